// Distillation of a head from a teacher's top logits: what differs from the cross
// entropy, whose products over the vocabulary (sq_ce.hip) it shares.
//
//   s[t,v]  = l[t,v] / tau                       lse[t] = log sum_v exp s[t,v]
//   q[t,k]  = softmax over the entries k that count of z[t,k] / tau
//   loss[t] = tau^2 sum_k q[t,k] (log q[t,k] - s[t,ids[t,k]] + lse[t])
//   dX[t]   = dloss[t] tau sum_v (exp(s[t,v] - lse[t]) - sum_{k : ids[t,k] = v} q[t,k]) W[v]
//
// An entry counts if its id is in the vocabulary and its logit is not -inf; a token
// without one is ignored.  The entries touch K of V columns: the forward takes their
// logits as products of their own with K rows of the head, which the backward uses
// again to write (p - q) over the p of its piece before the product with W, in one
// rounding.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "sq_device.h"
#include "sq_distill.h"
#include "sq_gemm_args.h"
#include "sq_launch.h"
#include "sq_rows.h"

namespace sq {

namespace {

inline int ok() { return hipGetLastError() == hipSuccess ? 0 : -1; }

// Workgroups by token (or by 4 or 16), on in y where x is full: `most` of them, whose
// work-items stay below the 2^32 from which a launch is cut short without an error.
__device__ __forceinline__ int64_t group_at() { return (int64_t)blockIdx.y * gridDim.x + blockIdx.x; }
inline dim3 groups_of(int64_t n, int64_t most = kGroupsX) {
  return dim3((unsigned)(n < most ? n : most), (unsigned)((n + most - 1) / most));
}

__device__ __forceinline__ float max_of(float v) {
#pragma unroll
  for (int d = 32; d; d >>= 1) v = fmaxf(v, __shfl_xor(v, d));
  return v;
}
__device__ __forceinline__ float sum_of(float v) {
#pragma unroll
  for (int d = 32; d; d >>= 1) v += __shfl_xor(v, d);
  return v;
}

// Entry k of token t: its row of the head, or -1 where it does not count.
__device__ __forceinline__ int entry_at(const Distill& g, int64_t t, int k, int V, float* z) {
  if (k >= g.K) return -1;
  const int64_t at = t * g.K + k, v = id_at(g.ids, g.id_bytes, at);
  *z = g.z_bf16 ? __uint_as_float((uint32_t)static_cast<const uint16_t*>(g.z)[at] << 16) : static_cast<const float*>(g.z)[at];
  return v >= 0 && v < V && *z != -INFINITY ? (int)v : -1;
}

// A token's entries, one wave's: lane l has entries l, l + 64, .., P in all; the
// teacher's probabilities and their logarithms (0 where an entry does not count).
template <int P>
struct Entries {
  int id[P];
  float q[P], log_q[P];
};
template <int P>
__device__ __forceinline__ Entries<P> entries_of(const Distill& g, int64_t t, int V) {
  const int lane = threadIdx.x & 63;
  Entries<P> e;
  float z[P], top = -INFINITY, sum = 0.0f;
#pragma unroll
  for (int i = 0; i < P; ++i) {
    z[i] = -INFINITY;
    e.id[i] = entry_at(g, t, i * 64 + lane, V, &z[i]);
    // a NaN stays: fmax would drop it
    if (e.id[i] >= 0) top = z[i] != z[i] || top != top ? z[i] + top : fmaxf(top, z[i]);
  }
#pragma unroll
  for (int d = 32; d; d >>= 1) {
    const float o = __shfl_xor(top, d);
    top = o != o || top != top ? o + top : fmaxf(top, o);
  }
  const float f = 1.0f / g.tau;
#pragma unroll
  for (int i = 0; i < P; ++i) {
    e.log_q[i] = e.id[i] >= 0 ? (z[i] - top) * f : 0.0f;
    e.q[i] = e.id[i] >= 0 ? __expf(e.log_q[i]) : 0.0f;
    sum += e.q[i];
  }
  sum = sum_of(sum);
  const float log_sum = __logf(sum);
#pragma unroll
  for (int i = 0; i < P; ++i) {
    if (e.id[i] < 0) continue;
    e.q[i] /= sum;
    e.log_q[i] -= log_sum;
  }
  return e;
}

// ------------------------------------------------------------------ live tokens
// One wave's answer for token t.
__device__ __forceinline__ void put_live(const Distill& g, int64_t t, int V, int* y) {
  const int lane = threadIdx.x & 63;
  bool any = false;
  for (int k = lane; k < g.K; k += 64) {
    float z;
    any |= entry_at(g, t, k, V, &z) >= 0;
  }
  const bool live = __ballot(any) != 0;
  if (lane == 0) y[t] = live ? V : -1;
}
__global__ __launch_bounds__(256) void distill_live_kernel(Distill g, int T, int V, int* __restrict__ y) {
  const int64_t t = group_at() * 4 + (threadIdx.x >> 6);
  if (t < T) put_live(g, t, V, y);
}

// ------------------------------------------------------------------ their logits
// 16 entries of one token per workgroup, 4 per wave (all of a token's in one: 200 tokens of
// 50000 x 2048 bf16 with 256 entries each 124 us, so 29).  Bound by the gathered rows: 4096
// tokens of 131072 x 4096 bf16 with 64 entries 286 us, 2.1 GB at 7.5 TB/s.  The first
// workgroup of a token also finds whether it counts.
template <int HEAD>
__global__ __launch_bounds__(256) void distill_pick_kernel(Distill g, int T, int V, int H, const uint16_t* __restrict__ X,
                                                           const void* __restrict__ W, const uint8_t* __restrict__ scales,
                                                           float f, int* __restrict__ y) {
  const int64_t t = (int64_t)blockIdx.z * kGroupsX + blockIdx.x;
  if (t >= T) return;
  const int lane = threadIdx.x & 63, k0 = (int)blockIdx.y * 16 + (int)(threadIdx.x >> 6) * 4;
  if (blockIdx.y == 0 && threadIdx.x < 64) put_live(g, t, V, y);
  if (k0 >= g.K) return;
  int id[4];
  float sum[4] = {0.0f, 0.0f, 0.0f, 0.0f}, z;
  bool any = false;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    id[i] = __builtin_amdgcn_readfirstlane(entry_at(g, t, k0 + i, V, &z));
    any |= id[i] >= 0;
  }
  if (any) {
    if constexpr (HEAD == kCeBf16) {
      for (int h = lane * 8; h < H; h += 512) {
        float x[8];
        load8<true>(X, t * H + h, x);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          float w[8];
          table8<HEAD>(W, scales, 1.0f, (int64_t)max(id[i], 0) * H + h, w);
#pragma unroll
          for (int j = 0; j < 8; ++j) sum[i] = __builtin_fmaf(x[j], w[j], sum[i]);
        }
      }
    } else {
      // a block per lane: its codes in words (codes are 4-byte aligned), its scale once
      // (1999 tokens of 50001 x 4096 MXFP4, 64 entries each, 40% ignored: 76 -> 44 us)
      constexpr int B = ScaleOperand<HEAD>::kBlock;
      for (int h = lane * B; h < H; h += 64 * B) {
        uint32_t q[4][B / 8], b[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int64_t at = (int64_t)max(id[i], 0) * H + h;
          const uint32_t* c = reinterpret_cast<const uint32_t*>(static_cast<const uint8_t*>(W) + at / 2);
#pragma unroll
          for (int j = 0; j < B / 8; ++j) q[i][j] = c[j];
          b[i] = scales[at / B];
        }
        float part[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int j = 0; j < B / 8; ++j) {
          float x[8];
          load8<true>(X, t * H + h + 8 * j, x);
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            float w[8];
            codes8(q[i][j], w);
#pragma unroll
            for (int k = 0; k < 8; ++k) part[i] = __builtin_fmaf(x[k], w[k], part[i]);
          }
        }
#pragma unroll
        for (int i = 0; i < 4; ++i)
          sum[i] = __builtin_fmaf(part[i], HEAD == kMX ? e8m0_to_f32(b[i]) : e4m3_to_f32(b[i]), sum[i]);
      }
    }
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float v = sum_of(sum[i]) * f;
    if (lane == 0 && k0 + i < g.K) g.picked[t * g.K + k0 + i] = id[i] >= 0 ? v : 0.0f;
  }
}

// ------------------------------------------------------------------ loss
// 16 tokens per workgroup: its threads share the tiles' pairs, 64 to a token, then a
// wave takes a token.  Latency: 5 tokens of 4 tiles 3.7 us, 4096 of 512 tiles 9.
template <int P>
__global__ __launch_bounds__(1024) void distill_loss_kernel(Distill g, const float2* __restrict__ part, const int* __restrict__ rows,
                                                            const int* __restrict__ count, const int* __restrict__ y, int T, int V,
                                                            int tiles, float* __restrict__ loss, float* __restrict__ lse) {
  __shared__ float2 s_part[16][64 + 1];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int live = count ? min(*count, T) : T;
  auto join = [](float2 a, float2 b) {
    const float m = fmaxf(a.x, b.x), ref = m == -INFINITY ? 0.0f : m;
    return make_float2(m, a.y * __expf(a.x - ref) + b.y * __expf(b.x - ref));
  };
  {
    const int n = threadIdx.x & 15, first = threadIdx.x >> 4;
    const int64_t row = group_at() * 16 + n;
    float2 p = make_float2(-INFINITY, 0.0f);
    if (row < live) {
#pragma unroll 4
      for (int i = first; i < tiles; i += 64) p = join(p, part[(size_t)i * T + row]);
    }
    s_part[n][first] = p;
  }
  __syncthreads();
  const int64_t t0 = group_at() * 16 + wave;                  // tokens that are ignored
  if (lane == 0 && t0 < T && y[t0] < 0) loss[t0] = lse[t0] = 0.0f;
  if (t0 >= live) return;
  const int64_t t = rows ? rows[t0] : t0;
  if (y[t] < 0) return;
  float2 p = s_part[wave][lane];
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) p = join(p, make_float2(__shfl_xor(p.x, d), __shfl_xor(p.y, d)));
  const float most = p.x, rest = __logf(p.y);
  const Entries<P> e = entries_of<P>(g, t, V);
  float v = 0.0f;
#pragma unroll
  for (int k = 0; k < P; ++k) {
    // the distance to the largest logit first, as the cross entropy takes it
    const int at = k * 64 + lane;
    if (e.id[k] >= 0) v += e.q[k] != 0.0f ? e.q[k] * (e.log_q[k] + ((most - g.picked[t * g.K + at]) + rest)) : 0.0f;
  }
  v = sum_of(v);
  if (lane == 0) {
    loss[t] = g.tau * g.tau * v;
    lse[t] = most + rest;
  }
}

// ------------------------------------------------------------------ gradient
// A wave per live token.  Entries of one id are one column: each writes the same
// value, with all their probabilities taken off.  Latency: 5 tokens with 16 entries 5.6 us,
// 4096 with 64 11.
template <int P>
__global__ __launch_bounds__(256) void distill_put_kernel(Distill g, DistillPiece p, const float* __restrict__ lse,
                                                          const float* __restrict__ dloss) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int64_t row = group_at() * 4 + wave;
  if (row >= (p.count ? min(*p.count, p.T) : p.T)) return;
  const int64_t t = p.rows ? p.rows[row] : row;
  const Entries<P> e = entries_of<P>(g, t, p.V);
  const float z = lse[t], c = dloss[t];
  // each entry against all, one broadcast at a time: its column's probabilities, and
  // whether it is the first of them
  float q[P], lost[P];
  bool first[P];
#pragma unroll
  for (int i = 0; i < P; ++i) {
    q[i] = 0.0f;
    first[i] = true;
  }
#pragma unroll
  for (int j = 0; j < P; ++j) {
    const int n = min(g.K - j * 64, 64);
    for (int l0 = 0; l0 < n; l0 += 8)                         // (past the last entry: of no id, probability 0)
#pragma unroll
      for (int u = 0; u < 8; ++u) {
        const int l = l0 + u, id = __builtin_amdgcn_readlane(e.id[j], l);
        const float of = __uint_as_float((uint32_t)__builtin_amdgcn_readlane((int)__float_as_uint(e.q[j]), l));
#pragma unroll
        for (int i = 0; i < P; ++i) {
          const bool same = e.id[i] == id;
          q[i] += same ? of : 0.0f;
          if (j <= i) first[i] = first[i] && !(same && (j < i || l < lane));
        }
      }
  }
#pragma unroll
  for (int i = 0; i < P; ++i) {
    const int k = i * 64 + lane;
    lost[i] = 0.0f;
    if (e.id[i] < 0) continue;
    const int64_t at = e.id[i] - p.v0;
    const bool tail = p.dtail && e.id[i] >= p.main, here = at >= 0 && at < p.n;
    if (!tail && !here && !p.lost) continue;
    const float d = c * (__expf(g.picked[t * g.K + k] - z) - q[i]);
    if (tail) {
      p.dtail[t * 8 + (e.id[i] - p.main)] = d;
      continue;
    }
    const uint32_t b = bits_of(__builtin_convertvector((f32x2{d, d}), bf16x2));
    if (first[i]) lost[i] = d - __uint_as_float(b << 16);
    if (!here) continue;
    const int group = min((int)(at / p.width), p.groups - 1);
    const int64_t last = (int64_t)(p.groups - 1) * p.width - p.shift;     // the last group's first column
    const bool in_last = p.groups > 1 ? group == p.groups - 1 : true;
    const int64_t col = in_last ? at - last : at - (int64_t)group * p.width;
    p.d[(int64_t)group * p.width * p.T + row * p.width + col] = (uint16_t)b;
  }
  if (!p.lost) return;
  // the entries that lost the most: their rows of the head are added at the end (error
  // of dX against 64 bits, 5 tokens of 1000 x 512 with 16 entries 3.6e-3 -> 1.8e-3, of which
  // 1.7e-3 is dX's own rounding)
  for (int r = 0; r < kDistillLost; ++r) {
    float most = 0.0f;
    int which = 0;
#pragma unroll
    for (int i = 0; i < P; ++i)
      if (fabsf(lost[i]) > most) {
        most = fabsf(lost[i]);
        which = i;
      }
    const float top = max_of(most);
    const uint64_t who = __ballot(top > 0.0f && most == top);
    if (!who) {
      if (lane == 0) p.lost[row * kDistillLost + r] = DistillLost{-1, 0.0f};
      continue;
    }
    if (lane == __builtin_ctzll(who)) {
#pragma unroll
      for (int i = 0; i < P; ++i)
        if (i == which) {
          p.lost[row * kDistillLost + r] = DistillLost{e.id[i], lost[i]};
          lost[i] = 0.0f;
        }
    }
  }
}

}  // namespace

int distill_live_launch(const Distill& k, int T, int V, int* y, hipStream_t s) {
  hipLaunchKernelGGL(distill_live_kernel, groups_of(((int64_t)T + 3) / 4), dim3(256), 0, s, k, T, V, y);
  return ok();
}

int distill_pick_launch(const Distill& k, int head, int T, int V, int H, const void* X, const void* W, const uint8_t* scales,
                        float f, int* y, hipStream_t s) {
  const dim3 grid((unsigned)(T < kGroupsX ? T : kGroupsX), (unsigned)((k.K + 15) / 16), (unsigned)((T + kGroupsX - 1) / kGroupsX));
  auto go = [&](auto kernel) {
    hipLaunchKernelGGL(kernel, grid, dim3(256), 0, s, k, T, V, H, static_cast<const uint16_t*>(X), W, scales, f, y);
    return ok();
  };
  return head == kMX ? go(distill_pick_kernel<kMX>) : head == kNV ? go(distill_pick_kernel<kNV>) : go(distill_pick_kernel<kCeBf16>);
}

int distill_loss_launch(const Distill& k, const float2* part, const int* rows, const int* count, const int* y, int T, int V,
                        int tiles, float* loss, float* lse, hipStream_t s) {
  auto go = [&](auto kernel) {
    hipLaunchKernelGGL(kernel, groups_of(((int64_t)T + 15) / 16, kGroupsX / 2), dim3(1024), 0, s, k, part, rows, count, y, T, V, tiles, loss, lse);
    return ok();
  };
  return k.K <= 64 ? go(distill_loss_kernel<1>) : k.K <= 128 ? go(distill_loss_kernel<2>) : go(distill_loss_kernel<4>);
}

int distill_put_launch(const Distill& k, const DistillPiece& piece, const float* lse, const float* dloss, hipStream_t s) {
  auto go = [&](auto kernel) {
    hipLaunchKernelGGL(kernel, groups_of(((int64_t)piece.T + 3) / 4), dim3(256), 0, s, k, piece, lse, dloss);
    return ok();
  };
  return k.K <= 64 ? go(distill_put_kernel<1>) : k.K <= 128 ? go(distill_put_kernel<2>) : go(distill_put_kernel<4>);
}

}  // namespace sq
