// C ABI of what a training step runs around the frozen-code products (declared
// in include/scaleqlora.h): host-side argument validation, then launches on the
// caller's stream.  Nothing here allocates device memory or synchronises.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "sq_checks.h"
#include "sq_launch.h"

namespace {

using namespace sq;

bool dtype_ok(int d) { return d == SQ_OUT_F32 || d == SQ_OUT_BF16; }

// ---------------------------------------------------------------- experts
constexpr int64_t kMoeExpertsMax = 2048;   // the sort's counters of one key each in LDS

int check_pairs(int64_t T, int64_t K, int64_t E) {
  if (T < 0 || K < 1 || E < 1 || T > kDimMax || K > kDimMax || E > kMoeExpertsMax) return SQ_ERR_SHAPE;
  return T * K > kDimMax ? SQ_ERR_SHAPE : SQ_OK;
}

int check_rows(int64_t T, int64_t K, int64_t E, int64_t H, const int32_t* slot, const int32_t* offsets) {
  const int st = check_pairs(T, K, E);
  if (st != SQ_OK) return st;
  if (H < 1 || H % 8 != 0 || H > kDimMax) return SQ_ERR_SHAPE;
  if (!offsets || (T > 0 && !slot)) return SQ_ERR_ARG;
  return aligned(slot, 4) && aligned(offsets, 4) ? SQ_OK : SQ_ERR_ALIGN;
}

}  // namespace

SQ_EXPORT size_t sq_moe_sort_workspace(int64_t T, int64_t K, int64_t E) {
  if (check_pairs(T, K, E) != SQ_OK || moe_sort_one(T * K)) return 0;
  return (size_t)((T * K + kMoeChunk - 1) / kMoeChunk + 1) * (size_t)(E + 1) * 4;
}

SQ_EXPORT int sq_moe_sort(int64_t T, int64_t K, int64_t E, const void* ids, int id_bytes, int32_t* offsets,
                          int32_t* token, int32_t* slot, void* workspace, size_t workspace_bytes, void* stream) {
  const int st = check_pairs(T, K, E);
  if (st != SQ_OK) return st;
  if (id_bytes != 4 && id_bytes != 8) return SQ_ERR_ARG;
  if (!offsets || (T > 0 && (!ids || !token || !slot))) return SQ_ERR_ARG;
  if (!aligned(ids, (uintptr_t)id_bytes) || !aligned(offsets, 4) || !aligned(token, 4) || !aligned(slot, 4))
    return SQ_ERR_ALIGN;
  const size_t need = sq_moe_sort_workspace(T, K, E);
  if (need > 0 && (!workspace || workspace_bytes < need)) return SQ_ERR_WORKSPACE;
  if (need > 0 && !aligned(workspace, 4)) return SQ_ERR_ALIGN;
  return hip_status(moe_sort_launch(T, (int)K, (int)E, ids, id_bytes, offsets, token, slot, workspace,
                                    static_cast<hipStream_t>(stream)));
}

SQ_EXPORT int sq_moe_gather(int64_t T, int64_t K, int64_t E, int64_t H, const void* X, int dtype, const int32_t* slot,
                            const int32_t* offsets, void* Xs, void* stream) {
  const int st = check_rows(T, K, E, H, slot, offsets);
  if (st != SQ_OK) return st;
  if (!dtype_ok(dtype) || (T > 0 && (!X || !Xs))) return SQ_ERR_ARG;
  if (!aligned(X, 16) || !aligned(Xs, 16)) return SQ_ERR_ALIGN;
  if (T == 0) return SQ_OK;
  return hip_status(moe_gather_launch(T, (int)K, (int)H, dtype == SQ_OUT_BF16, X, slot, offsets + E, Xs,
                                      static_cast<hipStream_t>(stream)));
}

SQ_EXPORT int sq_moe_combine(int64_t T, int64_t K, int64_t E, int64_t H, const void* Ys, int y_dtype,
                             const int32_t* slot, const int32_t* offsets, const float* weights, void* out,
                             int out_dtype, void* stream) {
  const int st = check_rows(T, K, E, H, slot, offsets);
  if (st != SQ_OK) return st;
  if (!dtype_ok(y_dtype) || !dtype_ok(out_dtype) || (T > 0 && (!Ys || !out))) return SQ_ERR_ARG;
  if (!aligned(Ys, 16) || !aligned(out, 16) || !aligned(weights, 4)) return SQ_ERR_ALIGN;
  if (T == 0) return SQ_OK;
  return hip_status(moe_combine_launch(T, (int)K, (int)H, Ys, y_dtype == SQ_OUT_BF16, slot, offsets + E, weights, out,
                                       out_dtype == SQ_OUT_BF16, static_cast<hipStream_t>(stream)));
}

SQ_EXPORT int sq_moe_combine_bwd(int64_t T, int64_t K, int64_t E, int64_t H, const void* dOut, int d_dtype,
                                 const void* Ys, int y_dtype, const int32_t* slot, const int32_t* offsets,
                                 const float* weights, void* dYs, int dy_dtype, float* dweights, void* stream) {
  const int st = check_rows(T, K, E, H, slot, offsets);
  if (st != SQ_OK) return st;
  if (!dtype_ok(d_dtype) || !dtype_ok(y_dtype) || !dtype_ok(dy_dtype)) return SQ_ERR_ARG;
  if (T > 0 && (!dOut || !Ys || !weights || !dYs || !dweights)) return SQ_ERR_ARG;
  if (!aligned(dOut, 16) || !aligned(Ys, 16) || !aligned(dYs, 16) || !aligned(weights, 4) || !aligned(dweights, 4))
    return SQ_ERR_ALIGN;
  if (T == 0) return SQ_OK;
  return hip_status(moe_combine_bwd_launch(T, (int)K, (int)H, dOut, d_dtype == SQ_OUT_BF16, Ys, y_dtype == SQ_OUT_BF16,
                                           slot, offsets + E, weights, dYs, dy_dtype == SQ_OUT_BF16, dweights,
                                           static_cast<hipStream_t>(stream)));
}

// ---------------------------------------------------------------- 8-bit activations
namespace {

constexpr int64_t kExpertsMax = 8192;      // the batched scale gradient's lists in LDS

bool act_ok(int act) { return act == SQ_ACT_INT8 || act == SQ_ACT_E4M3; }

int check_act(int act, int64_t T, int64_t I, const void* X, const uint8_t* codes, const uint8_t* scales) {
  if (!act_ok(act)) return SQ_ERR_ARG;
  // 32 values a work-item: a launch of 2^32 of them would be cut short
  if (T < 0 || I < 1 || T > kDimMax || I > kDimMax || I % 32 != 0 || T > (int64_t(1) << 36) / I) return SQ_ERR_SHAPE;
  if (T > 0 && (!X || !codes || !scales)) return SQ_ERR_ARG;
  return aligned(X, 16) && aligned(codes, 16) ? SQ_OK : SQ_ERR_ALIGN;
}

// The kept activation [Tx, I] and the scale gradient's other operands; N rows of dY.
int check_dscale8(int fmt, int act, int64_t Tx, int64_t N, int64_t O, int64_t I, const uint8_t* x, const uint8_t* xs,
                  const void* dY, const uint8_t* codes, const float* dS) {
  const int st = check_layer(fmt, 0, O, I);
  if (st != SQ_OK) return st;
  if (!act_ok(act)) return SQ_ERR_ARG;
  if (I % 32 != 0 || Tx < 0 || N < 0 || Tx > kDimMax || N > kDimMax / 4) return SQ_ERR_SHAPE;
  if (Tx * I > kOperandBytesMax || N * O * 2 > kOperandBytesMax) return SQ_ERR_SHAPE;
  if (O > (1 << 23) || I > (1 << 23)) return SQ_ERR_SHAPE;      // a 64-row stage within 32-bit offsets
  if (!codes || !dS || (N > 0 && !dY) || (Tx > 0 && (!x || !xs))) return SQ_ERR_ARG;
  return aligned(x, 16) && aligned(dY, 16) && aligned(codes, 4) && aligned(dS, 4) ? SQ_OK : SQ_ERR_ALIGN;
}

}  // namespace

SQ_EXPORT int sq_act_pack(int act, int64_t T, int64_t I, const void* X, uint8_t* codes_out, uint8_t* scales_out,
                          void* stream) {
  const int st = check_act(act, T, I, X, codes_out, scales_out);
  if (st != SQ_OK || T == 0) return st;
  return hip_status(act_pack_launch(act, T, I, X, codes_out, scales_out, static_cast<hipStream_t>(stream)));
}

SQ_EXPORT int sq_act_unpack(int act, int64_t T, int64_t I, const uint8_t* codes, const uint8_t* scales, void* X,
                            void* stream) {
  const int st = check_act(act, T, I, X, codes, scales);
  if (st != SQ_OK || T == 0) return st;
  return hip_status(act_unpack_launch(act, T, I, codes, scales, X, static_cast<hipStream_t>(stream)));
}

SQ_EXPORT size_t sq_bwd_dscale_act8_workspace(int fmt, int64_t T, int64_t O, int64_t I) {
  if (check_layer(fmt, T, O, I) != SQ_OK || I % 32 != 0) return 0;
  return dscale_act8_workspace(fmt, (int)T, (int)O, (int)I);
}

SQ_EXPORT int sq_bwd_dscale_act8(int fmt, int act, int64_t T, int64_t O, int64_t I, const uint8_t* x_codes,
                                 const uint8_t* x_scales, const void* dY, const uint8_t* codes, float* dS,
                                 void* workspace, size_t workspace_bytes, void* stream) {
  int st = check_layer(fmt, T, O, I);
  if (st == SQ_OK) st = check_dscale8(fmt, act, T, T, O, I, x_codes, x_scales, dY, codes, dS);
  if (st != SQ_OK) return st;
  const size_t need = sq_bwd_dscale_act8_workspace(fmt, T, O, I);
  if (need > 0 && (!workspace || workspace_bytes < need)) return SQ_ERR_WORKSPACE;
  if (need > 0 && !aligned(workspace, 16)) return SQ_ERR_ALIGN;
  return hip_status(dscale_act8(fmt, act, (int)T, (int)O, (int)I, x_codes, x_scales, dY, codes, dS, workspace,
                                static_cast<hipStream_t>(stream)));
}

SQ_EXPORT size_t sq_bwd_dscale_act8_batched_workspace(int64_t E, int64_t T, int64_t I) {
  if (E < 1 || E > kExpertsMax || T < 0 || I < 1 || T > kDimMax || I > kDimMax || I % 32 != 0 || T * I * 2 > kOperandBytesMax) return 0;
  return dscale_act8_batched_workspace((int)E, (int)T, (int)I);
}

SQ_EXPORT int sq_bwd_dscale_act8_batched(int fmt, int act, int64_t E, int64_t T, int64_t N, int64_t O, int64_t I,
                                         const uint8_t* x_codes, const uint8_t* x_scales, const int32_t* rows,
                                         const int32_t* offsets, const void* dY, const uint8_t* codes, float* dS,
                                         void* workspace, size_t workspace_bytes, void* stream) {
  const int st = check_dscale8(fmt, act, T, N, O, I, x_codes, x_scales, dY, codes, dS);
  if (st != SQ_OK) return st;
  if (T * I * 2 > kOperandBytesMax) return SQ_ERR_SHAPE;
  // the tiles of all experts are numbered in 32 bits
  if (E < 1 || E > kExpertsMax || E * ((O + 255) / 256) * ((I + 255) / 256) > kDimMax) return SQ_ERR_SHAPE;
  if (!offsets || (N > 0 && !rows && N != T)) return SQ_ERR_ARG;
  if (!aligned(rows, 4) || !aligned(offsets, 4)) return SQ_ERR_ALIGN;
  const size_t need = sq_bwd_dscale_act8_batched_workspace(E, T, I);
  if (need > 0 && (!workspace || workspace_bytes < need)) return SQ_ERR_WORKSPACE;
  if (need > 0 && !aligned(workspace, 16)) return SQ_ERR_ALIGN;
  return hip_status(dscale_act8_batched(fmt, act, (int)E, (int)T, (int)N, (int)O, (int)I, x_codes, x_scales, rows,
                                        offsets, dY, codes, dS, workspace, static_cast<hipStream_t>(stream)));
}

// ---------------------------------------------------------------- cross entropy
namespace {

static_assert(SQ_HEAD_MXFP4 == SQ_MXFP4 && SQ_HEAD_NVFP4 == SQ_NVFP4 && SQ_HEAD_BF16 == kCeBf16,
              "header and library agree on the head formats");

int check_head(int head, int64_t T, int64_t V, int64_t I) {
  if (head != SQ_HEAD_MXFP4 && head != SQ_HEAD_NVFP4 && head != SQ_HEAD_BF16) return SQ_ERR_FORMAT;
  if (T < 0 || V < 1 || I < 1 || T > kDimMax || V > kDimMax - 256 || I > kDimMax) return SQ_ERR_SHAPE;
  if (I % (head == SQ_HEAD_BF16 ? 8 : block_of(head)) != 0) return SQ_ERR_SHAPE;
  // X and a 256-row tile of the head go through 32-bit offsets
  if (T * I * 2 > kOperandBytesMax || I * 512 > kOperandBytesMax) return SQ_ERR_SHAPE;
  return ((V + 255) / 256) * ((T + 63) / 64) > kDimMax ? SQ_ERR_SHAPE : SQ_OK;
}

int check_ce(int head, int64_t T, int64_t V, int64_t I, const void* X, const void* W, const uint8_t* scales, float ws2,
             const void* targets, int target_bytes) {
  const int st = check_head(head, T, V, I);
  if (st != SQ_OK) return st;
  if (target_bytes != 4 && target_bytes != 8) return SQ_ERR_ARG;
  if (!W || (head != SQ_HEAD_BF16 && !scales) || (T > 0 && (!X || !targets))) return SQ_ERR_ARG;
  if (head == SQ_HEAD_NVFP4 && !ws2_ok(ws2)) return SQ_ERR_ARG;
  return aligned(X, 16) && aligned(W, head == SQ_HEAD_BF16 ? 16 : 4) && aligned(targets, (uintptr_t)target_bytes)
             ? SQ_OK : SQ_ERR_ALIGN;
}

int check_ce_workspace(int bwd, int head, int64_t T, int64_t V, int64_t I, const void* workspace, size_t bytes) {
  if (!workspace || bytes < ce_workspace(bwd, head, T, V, I)) return SQ_ERR_WORKSPACE;
  return aligned(workspace, 256) ? SQ_OK : SQ_ERR_ALIGN;
}

}  // namespace

SQ_EXPORT size_t sq_ce_fwd_workspace(int head, int64_t T, int64_t V, int64_t I) {
  return check_head(head, T, V, I) != SQ_OK || T == 0 ? 0 : ce_workspace(0, head, T, V, I);
}

SQ_EXPORT size_t sq_ce_bwd_workspace(int head, int64_t T, int64_t V, int64_t I) {
  return check_head(head, T, V, I) != SQ_OK || T == 0 ? 0 : ce_workspace(1, head, T, V, I);
}

SQ_EXPORT int sq_ce_fwd(int head, int64_t T, int64_t V, int64_t I, const void* X, const void* W, const uint8_t* scales,
                        float ws2, const void* targets, int target_bytes, float* loss, float* lse, void* workspace,
                        size_t workspace_bytes, void* stream) {
  int st = check_ce(head, T, V, I, X, W, scales, ws2, targets, target_bytes);
  if (st != SQ_OK) return st;
  if (T > 0 && (!loss || !lse)) return SQ_ERR_ARG;
  if (!aligned(loss, 4) || !aligned(lse, 4)) return SQ_ERR_ALIGN;
  if (T == 0) return SQ_OK;
  st = check_ce_workspace(0, head, T, V, I, workspace, workspace_bytes);
  if (st != SQ_OK) return st;
  return hip_status(ce_fwd_launch(head, (int)T, V, (int)I, X, W, scales, head == SQ_HEAD_NVFP4 ? ws2 : 1.0f, targets,
                                  target_bytes, loss, lse, workspace, static_cast<hipStream_t>(stream)));
}

SQ_EXPORT int sq_ce_bwd(int head, int64_t T, int64_t V, int64_t I, const void* X, const void* W, const uint8_t* scales,
                        float ws2, const void* targets, int target_bytes, const float* lse, const float* dloss, void* dX,
                        int dx_dtype, void* workspace, size_t workspace_bytes, void* stream) {
  int st = check_ce(head, T, V, I, X, W, scales, ws2, targets, target_bytes);
  if (st != SQ_OK) return st;
  if (!dtype_ok(dx_dtype) || (T > 0 && (!lse || !dloss || !dX))) return SQ_ERR_ARG;
  if (!aligned(lse, 4) || !aligned(dloss, 4) || !aligned(dX, 16)) return SQ_ERR_ALIGN;
  if (T == 0) return SQ_OK;
  st = check_ce_workspace(1, head, T, V, I, workspace, workspace_bytes);
  if (st != SQ_OK) return st;
  return hip_status(ce_bwd_launch(head, (int)T, V, (int)I, X, W, scales, head == SQ_HEAD_NVFP4 ? ws2 : 1.0f, targets,
                                  target_bytes, lse, dloss, dX, dx_dtype == SQ_OUT_BF16, workspace,
                                  static_cast<hipStream_t>(stream)));
}
