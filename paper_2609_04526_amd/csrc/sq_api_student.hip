// C ABI of the operators of a 4-bit student and its teacher (declared in
// include/scaleqlora.h): host-side argument validation, then launches on the
// caller's stream.  Nothing here allocates device memory or synchronises.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "sq_checks.h"
#include "sq_launch.h"

namespace {

using namespace sq;

bool dtype_ok(int d) { return d == SQ_OUT_F32 || d == SQ_OUT_BF16; }
bool fmt_ok(int fmt) { return fmt == SQ_MXFP4 || fmt == SQ_NVFP4; }

// ---------------------------------------------------------------- 4-bit activations
constexpr int64_t kExpertsMax = 8192;
constexpr int64_t kXcds = 8;                // the experts' chunks are dealt to them in turn

// X bf16 [T, I] and its 4-bit form.
int check_act4(int fmt, int64_t T, int64_t I, const void* X, float ws2, const uint8_t* codes, const uint8_t* scales) {
  if (!fmt_ok(fmt)) return SQ_ERR_FORMAT;
  // 8 values a work-item, 32 a launch's: one of 2^32 work-items would be cut short
  if (T < 0 || I < 1 || T > kDimMax || I > kDimMax || I % block_of(fmt) != 0 || T > (int64_t(1) << 36) / I) return SQ_ERR_SHAPE;
  if (fmt == SQ_NVFP4 && !ws2_ok(ws2)) return SQ_ERR_ARG;
  if (T > 0 && (!X || !codes || !scales)) return SQ_ERR_ARG;
  return aligned(X, 16) && aligned(codes, 4) ? SQ_OK : SQ_ERR_ALIGN;
}

// What the products of two 4-bit operands take, the same for one layer and for many.
int check_fwd_act4(int64_t T, int64_t N, const uint8_t* x, const uint8_t* xs, const uint8_t* codes, const uint8_t* scales,
                   const void* Y, int y_dtype) {
  if (!dtype_ok(y_dtype) || !codes || !scales || (T > 0 && (!x || !xs)) || (N > 0 && !Y)) return SQ_ERR_ARG;
  return aligned(x, 16) && aligned(codes, 16) && aligned(xs, 4) && aligned(scales, 4) && aligned(Y, 16) ? SQ_OK : SQ_ERR_ALIGN;
}

// (the kept rows as sq_fwd_act4 takes them and an expert's codes go through 32-bit offsets;
// Y, whose rows are N and not T, does not)
int check_batched(int fmt, int64_t E, int64_t T, int64_t N, int64_t O, int64_t I) {
  if (!fmt_ok(fmt)) return SQ_ERR_FORMAT;
  if (T < 0 || O < 1 || I < 1 || T > kDimMax || O > kDimMax || I > kDimMax) return SQ_ERR_SHAPE;
  if (O % 8 != 0 || I % block_of(fmt) != 0) return SQ_ERR_SHAPE;
  if (T * I * 2 > kOperandBytesMax || O * I / 2 > kOperandBytesMax) return SQ_ERR_SHAPE;
  if (fmt != SQ_MXFP4) return SQ_ERR_UNIMPLEMENTED;
  if (E < 1 || E > kExpertsMax || N < 0 || N > kDimMax) return SQ_ERR_SHAPE;
  // the workgroups of a launch: 64 rows by 128 outputs each at least (and 16 by 16 for the
  // fewest rows, of which there are fewer)
  const int64_t chunks = N / 64 + (E < N ? E : N) + kXcds;
  return chunks > kGroupsX || chunks * ((O + 127) / 128) > kGroupsX ? SQ_ERR_SHAPE : SQ_OK;
}

int check_workspace(size_t need, const void* workspace, size_t bytes) {
  if (need == 0) return SQ_OK;
  if (!workspace || bytes < need) return SQ_ERR_WORKSPACE;
  return aligned(workspace, 256) ? SQ_OK : SQ_ERR_ALIGN;
}

}  // namespace

SQ_EXPORT int sq_act4_pack(int fmt, int64_t T, int64_t I, const void* X, float ws2, uint8_t* codes_out, uint8_t* scales_out,
                           void* stream) {
  const int st = check_act4(fmt, T, I, X, ws2, codes_out, scales_out);
  if (st != SQ_OK || T == 0) return st;
  return hip_status(act4_pack_launch(fmt, T, I, X, ws2, codes_out, scales_out, static_cast<hipStream_t>(stream)));
}

SQ_EXPORT int sq_act4_unpack(int fmt, int64_t T, int64_t I, const uint8_t* codes, const uint8_t* scales, float ws2, void* X,
                             void* stream) {
  const int st = check_act4(fmt, T, I, X, ws2, codes, scales);
  if (st != SQ_OK || T == 0) return st;
  return hip_status(act4_unpack_launch(fmt, T, I, codes, scales, ws2, X, static_cast<hipStream_t>(stream)));
}

SQ_EXPORT size_t sq_fwd_act4_workspace(int fmt, int64_t T, int64_t O, int64_t I) {
  return check_layer(fmt, T, O, I) != SQ_OK || T == 0 ? 0 : act4_workspace(fmt, T, O, I);
}

SQ_EXPORT int sq_fwd_act4(int fmt, int64_t T, int64_t O, int64_t I, const uint8_t* x_codes, const uint8_t* x_scales, float x_ws2,
                          const uint8_t* codes, const uint8_t* scales, float ws2, void* Y, int y_dtype, void* workspace,
                          size_t workspace_bytes, void* stream) {
  int st = check_layer(fmt, T, O, I);
  if (st == SQ_OK) st = check_fwd_act4(T, T, x_codes, x_scales, codes, scales, Y, y_dtype);
  if (st != SQ_OK) return st;
  if (fmt == SQ_NVFP4 && (!ws2_ok(x_ws2) || !ws2_ok(ws2) || !ws2_ok(x_ws2 * ws2))) return SQ_ERR_ARG;
  if (T == 0) return SQ_OK;
  st = check_workspace(act4_workspace(fmt, T, O, I), workspace, workspace_bytes);
  if (st != SQ_OK) return st;
  return hip_status(act4_fwd(fmt, (int)T, (int)O, (int)I, x_codes, x_scales, x_ws2, codes, scales, ws2, Y, y_dtype == SQ_OUT_BF16,
                             workspace, static_cast<hipStream_t>(stream)));
}

SQ_EXPORT size_t sq_fwd_act4_batched_workspace(int fmt, int64_t E, int64_t T, int64_t N, int64_t O, int64_t I) {
  return check_batched(fmt, E, T, N, O, I) != SQ_OK || N == 0 ? 0 : act4_batched_workspace(E, T, N, O, I);
}

SQ_EXPORT int sq_fwd_act4_batched(int fmt, int64_t E, int64_t T, int64_t N, int64_t O, int64_t I, const uint8_t* x_codes,
                                  const uint8_t* x_scales, const int32_t* rows, const int32_t* offsets, const uint8_t* codes,
                                  const uint8_t* scales, void* Y, int y_dtype, void* workspace, size_t workspace_bytes,
                                  void* stream) {
  int st = check_batched(fmt, E, T, N, O, I);
  if (st == SQ_OK) st = check_fwd_act4(T, N, x_codes, x_scales, codes, scales, Y, y_dtype);
  if (st != SQ_OK) return st;
  if (!offsets || (N > 0 && !rows && N != T)) return SQ_ERR_ARG;
  if (!aligned(rows, 4) || !aligned(offsets, 4)) return SQ_ERR_ALIGN;
  if (N == 0) return SQ_OK;
  st = check_workspace(act4_batched_workspace(E, T, N, O, I), workspace, workspace_bytes);
  if (st != SQ_OK) return st;
  return hip_status(act4_fwd_batched((int)E, (int)T, (int)N, (int)O, (int)I, x_codes, x_scales, rows, offsets, codes, scales, Y,
                                     y_dtype == SQ_OUT_BF16, workspace, static_cast<hipStream_t>(stream)));
}

// ---------------------------------------------------------------- distillation
namespace {

// the head as the cross entropy takes it, with entries in the place of targets
int check_distill_head(int head, int64_t T, int64_t V, int64_t I, int64_t K) {
  if (head != SQ_HEAD_MXFP4 && head != SQ_HEAD_NVFP4 && head != SQ_HEAD_BF16) return SQ_ERR_FORMAT;
  if (T < 0 || V < 1 || I < 1 || T > kDimMax || V > kDimMax - 256 || I > kDimMax) return SQ_ERR_SHAPE;
  if (I % (head == SQ_HEAD_BF16 ? 8 : block_of(head)) != 0 || K < 1 || K > kDistillMax) return SQ_ERR_SHAPE;
  // X and a 256-row tile of the head go through 32-bit offsets
  if (T * I * 2 > kOperandBytesMax || I * 512 > kOperandBytesMax) return SQ_ERR_SHAPE;
  return ((V + 255) / 256) * ((T + 63) / 64) > kDimMax ? SQ_ERR_SHAPE : SQ_OK;
}

int check_distill(int head, int64_t T, int64_t V, int64_t I, int64_t K, const void* X, const void* W, const uint8_t* scales,
                  float ws2, const void* ids, int id_bytes, const void* logits, int logit_dtype, float temperature,
                  const float* picked) {
  const int st = check_distill_head(head, T, V, I, K);
  if (st != SQ_OK) return st;
  if ((id_bytes != 4 && id_bytes != 8) || !dtype_ok(logit_dtype)) return SQ_ERR_ARG;
  if (!W || (head != SQ_HEAD_BF16 && !scales) || (T > 0 && (!X || !ids || !logits || !picked))) return SQ_ERR_ARG;
  // the logits' factor, the gradient's and the temperature's square have to stay numbers
  if (!(temperature >= 0x1p-20f && temperature <= 0x1p20f)) return SQ_ERR_ARG;
  if (head == SQ_HEAD_NVFP4 && !(ws2_ok(ws2) && ws2_ok(ws2 / temperature) && ws2_ok(ws2 * temperature))) return SQ_ERR_ARG;
  return aligned(X, 16) && aligned(W, head == SQ_HEAD_BF16 ? 16 : 4) && aligned(ids, (uintptr_t)id_bytes) &&
                 aligned(logits, logit_dtype == SQ_OUT_BF16 ? 2 : 4) && aligned(picked, 4) ? SQ_OK : SQ_ERR_ALIGN;
}

}  // namespace

SQ_EXPORT size_t sq_distill_fwd_workspace(int head, int64_t T, int64_t V, int64_t I) {
  return check_distill_head(head, T, V, I, 1) != SQ_OK || T == 0 ? 0 : distill_workspace(0, head, T, V, I);
}

SQ_EXPORT size_t sq_distill_bwd_workspace(int head, int64_t T, int64_t V, int64_t I) {
  return check_distill_head(head, T, V, I, 1) != SQ_OK || T == 0 ? 0 : distill_workspace(1, head, T, V, I);
}

SQ_EXPORT int sq_distill_fwd(int head, int64_t T, int64_t V, int64_t I, int64_t K, const void* X, const void* W,
                             const uint8_t* scales, float ws2, const void* ids, int id_bytes, const void* logits, int logit_dtype,
                             float temperature, float* loss, float* lse, float* picked, void* workspace, size_t workspace_bytes,
                             void* stream) {
  int st = check_distill(head, T, V, I, K, X, W, scales, ws2, ids, id_bytes, logits, logit_dtype, temperature, picked);
  if (st != SQ_OK) return st;
  if (T > 0 && (!loss || !lse)) return SQ_ERR_ARG;
  if (!aligned(loss, 4) || !aligned(lse, 4)) return SQ_ERR_ALIGN;
  if (T == 0) return SQ_OK;
  st = check_workspace(distill_workspace(0, head, T, V, I), workspace, workspace_bytes);
  if (st != SQ_OK) return st;
  const Distill k{ids, logits, picked, id_bytes, logit_dtype == SQ_OUT_BF16, (int)K, temperature};
  return hip_status(distill_fwd_launch(head, (int)T, V, (int)I, X, W, scales, head == SQ_HEAD_NVFP4 ? ws2 : 1.0f, k, loss, lse,
                                       workspace, static_cast<hipStream_t>(stream)));
}

SQ_EXPORT int sq_distill_bwd(int head, int64_t T, int64_t V, int64_t I, int64_t K, const void* X, const void* W,
                             const uint8_t* scales, float ws2, const void* ids, int id_bytes, const void* logits, int logit_dtype,
                             float temperature, const float* lse, const float* picked, const float* dloss, void* dX, int dx_dtype,
                             void* workspace, size_t workspace_bytes, void* stream) {
  int st = check_distill(head, T, V, I, K, X, W, scales, ws2, ids, id_bytes, logits, logit_dtype, temperature, picked);
  if (st != SQ_OK) return st;
  if (!dtype_ok(dx_dtype) || (T > 0 && (!lse || !dloss || !dX))) return SQ_ERR_ARG;
  if (!aligned(lse, 4) || !aligned(dloss, 4) || !aligned(dX, 16)) return SQ_ERR_ALIGN;
  if (T == 0) return SQ_OK;
  st = check_workspace(distill_workspace(1, head, T, V, I), workspace, workspace_bytes);
  if (st != SQ_OK) return st;
  const Distill k{ids, logits, const_cast<float*>(picked), id_bytes, logit_dtype == SQ_OUT_BF16, (int)K, temperature};
  return hip_status(distill_bwd_launch(head, (int)T, V, (int)I, X, W, scales, head == SQ_HEAD_NVFP4 ? ws2 : 1.0f, k, lse, dloss,
                                       dX, dx_dtype == SQ_OUT_BF16, workspace, static_cast<hipStream_t>(stream)));
}

// ---------------------------------------------------------------- embedding
namespace {

// Places go by 32 bits, 64 past the last token among them, and columns in launches of
// 2048 each.
constexpr int64_t kEmbedTokensMax = int64_t(1) << 30, kEmbedColumnsMax = int64_t(1) << 26;

int check_table(int head, int64_t T, int64_t V, int64_t I, const void* ids, int id_bytes, float factor) {
  if (head != SQ_HEAD_MXFP4 && head != SQ_HEAD_NVFP4 && head != SQ_HEAD_BF16) return SQ_ERR_FORMAT;
  if (T < 0 || V < 1 || I < 1 || T > kEmbedTokensMax || V > kDimMax - 256 || I > kEmbedColumnsMax) return SQ_ERR_SHAPE;
  if (I % (head == SQ_HEAD_BF16 ? 8 : block_of(head)) != 0) return SQ_ERR_SHAPE;
  if ((id_bytes != 4 && id_bytes != 8) || !isfinite(factor) || (T > 0 && !ids)) return SQ_ERR_ARG;
  return aligned(ids, (uintptr_t)id_bytes) ? SQ_OK : SQ_ERR_ALIGN;
}

size_t embed_bwd_workspace(int64_t T, int64_t V, int64_t I) {
  if (T < 1 || V < 1 || I < 1 || T > kEmbedTokensMax || V > kDimMax - 256 || I > kEmbedColumnsMax || I % 8 != 0) return 0;
  return embed_workspace(T, V, I);
}

int embed_bwd(int head, int64_t T, int64_t V, int64_t I, const void* ids, int id_bytes, const void* dOut, int d_dtype, float factor,
              const uint8_t* codes, void* grad, int grad_bf16, void* workspace, size_t workspace_bytes, void* stream) {
  const int st = check_table(head, T, V, I, ids, id_bytes, factor);
  if (st != SQ_OK) return st;
  if (!dtype_ok(d_dtype) || !grad || (T > 0 && !dOut) || (head != SQ_HEAD_BF16 && !codes)) return SQ_ERR_ARG;
  if (!aligned(dOut, 16) || !aligned(grad, 16) || !aligned(codes, 4)) return SQ_ERR_ALIGN;
  const int sw = check_workspace(embed_bwd_workspace(T, V, I), workspace, workspace_bytes);
  if (sw != SQ_OK) return sw;
  return hip_status(embed_bwd_launch(head, (int)T, (int)V, (int)I, ids, id_bytes, dOut, d_dtype == SQ_OUT_BF16, factor, codes, grad,
                                     grad_bf16, workspace, static_cast<hipStream_t>(stream)));
}

}  // namespace

SQ_EXPORT int sq_embed_fwd(int head, int64_t T, int64_t V, int64_t I, const void* ids, int id_bytes, const void* W,
                           const uint8_t* scales, float ws2, float factor, void* out, int out_dtype, void* stream) {
  const int st = check_table(head, T, V, I, ids, id_bytes, factor);
  if (st != SQ_OK) return st;
  if (!dtype_ok(out_dtype) || !W || (head != SQ_HEAD_BF16 && !scales) || (T > 0 && !out)) return SQ_ERR_ARG;
  if (head == SQ_HEAD_NVFP4 && !ws2_ok(ws2)) return SQ_ERR_ARG;
  if (!aligned(W, head == SQ_HEAD_BF16 ? 16 : 4) || !aligned(out, 16)) return SQ_ERR_ALIGN;
  if (T == 0) return SQ_OK;
  return hip_status(embed_launch(head, T, (int)V, (int)I, ids, id_bytes, W, scales, ws2, factor, out, out_dtype == SQ_OUT_BF16,
                                 static_cast<hipStream_t>(stream)));
}

SQ_EXPORT size_t sq_embed_bwd_workspace(int64_t T, int64_t V, int64_t I) { return embed_bwd_workspace(T, V, I); }

SQ_EXPORT int sq_embed_bwd(int64_t T, int64_t V, int64_t I, const void* ids, int id_bytes, const void* dOut, int d_dtype,
                           float factor, void* dW, int dw_dtype, void* workspace, size_t workspace_bytes, void* stream) {
  if (!dtype_ok(dw_dtype)) return SQ_ERR_ARG;
  return embed_bwd(SQ_HEAD_BF16, T, V, I, ids, id_bytes, dOut, d_dtype, factor, nullptr, dW, dw_dtype == SQ_OUT_BF16, workspace,
                   workspace_bytes, stream);
}

SQ_EXPORT int sq_embed_bwd_dscale(int fmt, int64_t T, int64_t V, int64_t I, const void* ids, int id_bytes, const void* dOut,
                                  int d_dtype, float factor, const uint8_t* codes, float* dS, void* workspace,
                                  size_t workspace_bytes, void* stream) {
  if (!fmt_ok(fmt)) return SQ_ERR_FORMAT;
  return embed_bwd(fmt, T, V, I, ids, id_bytes, dOut, d_dtype, factor, codes, dS, 0, workspace, workspace_bytes, stream);
}
