// Embedding lookup and its gradients, for tables in bf16 and in the layer's 4-bit
// storage.
//
//   out[t]  = factor W[ids[t]]
//   dW[v]   = factor sum_{t : ids[t] = v} dOut[t]                      (bf16 table)
//   dS[v,g] = factor sum_{j in g} code[v,j] sum_{t : ids[t] = v} dOut[t,j]
//
// All of it is bound by memory.  The gradients sort the tokens by id (stable), sum
// the runs of one id in token order, and write zeros where an id has no token.
// Nothing is added atomically, so the same bits come out of every run.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <type_traits>

#include "sq_device.h"
#include "sq_launch.h"
#include "sq_rows.h"

namespace sq {

namespace {

inline int ok() { return hipGetLastError() == hipSuccess ? 0 : -1; }

// The id, or V where it is outside the table.
__device__ __forceinline__ int key_at(const void* ids, int bytes, int64_t t, int V) {
  const int64_t v = id_at(ids, bytes, t);
  return v >= 0 && v < V ? (int)v : V;
}

// ------------------------------------------------------------------ lookup
// One token per workgroup, 8 columns per lane and step.
template <int HEAD, bool BF16>
__global__ __launch_bounds__(256) void embed_kernel(const void* __restrict__ ids, int id_bytes, int64_t T, int V, int H,
                                                    const void* __restrict__ W, const uint8_t* __restrict__ scales, float ws2,
                                                    float factor, void* __restrict__ out) {
  const int64_t t = (int64_t)blockIdx.y * kGroupsX + blockIdx.x;
  if (t >= T) return;
  const int key = key_at(ids, id_bytes, t, V);
  for (int h = (int)threadIdx.x * 8; h < H; h += (int)blockDim.x * 8) {
    float v[8] = {};
    if (key < V) {
      table8<HEAD>(W, scales, ws2, (int64_t)key * H + h, v);
#pragma unroll
      for (int k = 0; k < 8; ++k) v[k] *= factor;
    }
    store8<BF16>(out, t * H + h, v);
  }
}

// ------------------------------------------------------------------ sort
// Place of each token in the stable order by id: the smaller keys, and the equal ones
// of earlier tokens.  A workgroup takes 64 tokens, one per lane; its waves share the
// other tokens, whose keys lie in LDS.  Every token meets every other: T^2 steps of
// two instructions, but one launch and no pass over the vocabulary.
// The other workgroups clear the gradient meanwhile.
__global__ __launch_bounds__(1024) void embed_rank_kernel(const void* __restrict__ ids, int id_bytes, int T, int V,
                                                          int* __restrict__ keys, int* __restrict__ tokens,
                                                          float* __restrict__ grad, int64_t grad_words) {
  const int sorters = (T + 63) / 64;
  if ((int)blockIdx.x >= sorters) {
    const int64_t n = (int64_t)(gridDim.x - sorters) * 1024, at = (int64_t)(blockIdx.x - sorters) * 1024 + threadIdx.x;
    for (int64_t i = at; i < grad_words / 4; i += n) reinterpret_cast<f32x4*>(grad)[i] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    if (at < grad_words % 4) grad[grad_words / 4 * 4 + at] = 0.0f;
    return;
  }
  __shared__ int s_key[kEmbedRankTokens];
  __shared__ int s_n[16][64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int padded = sorters * 64;
  for (int i = threadIdx.x; i < padded; i += 1024) s_key[i] = i < T ? key_at(ids, id_bytes, i, V) : 0x7FFFFFFF;
  __syncthreads();
  const int own = (int)blockIdx.x * 64, k = s_key[own + lane];
  // blocks of 64 tokens, wave w takes every 16th
  int n = 0;
  for (int b = wave; b < sorters; b += 16) {
    const int* s = s_key + b * 64;
    if (b == (int)blockIdx.x) {
      for (int j = 0; j < 64; ++j) n += s[j] < k || (s[j] == k && j < lane);
    } else if (b < (int)blockIdx.x) {
#pragma unroll 16
      for (int j = 0; j < 64; ++j) n += s[j] <= k;
    } else {
#pragma unroll 16
      for (int j = 0; j < 64; ++j) n += s[j] < k;
    }
  }
  s_n[wave][lane] = n;
  __syncthreads();
  if (wave == 0 && own + lane < T) {
#pragma unroll
    for (int w = 1; w < 16; ++w) n += s_n[w][lane];
    keys[n] = k;
    tokens[n] = own + lane;
  }
}

// More tokens: two stable sorts, by the low and by the high bits of the key.
// `bits` of the key from `shift` on, of tokens in the order `from` (null: as they come).
__global__ __launch_bounds__(256) void embed_digit_kernel(const void* __restrict__ ids, int id_bytes, int T, int V,
                                                          const int* __restrict__ from, int shift, int mask,
                                                          int* __restrict__ digit) {
  const int s = (int)blockIdx.x * 256 + threadIdx.x;
  if (s < T) digit[s] = (key_at(ids, id_bytes, from ? from[s] : s, V) >> shift) & mask;
}
// The order `place` of the tokens that stand in the order `from` (null: as they come).
__global__ __launch_bounds__(256) void embed_order_kernel(const void* __restrict__ ids, int id_bytes, int T, int V,
                                                          const int* __restrict__ from, const int* __restrict__ place,
                                                          int* __restrict__ keys, int* __restrict__ tokens) {
  const int s = (int)blockIdx.x * 256 + threadIdx.x;
  if (s >= T) return;
  const int t = from ? from[place[s]] : place[s];
  tokens[s] = t;
  if (keys) keys[s] = key_at(ids, id_bytes, t, V);
}

// ------------------------------------------------------------------ sums
struct EmbedArgs {
  const int* keys;          // sorted
  const int* tokens;
  const void* d;            // dOut [T, H]
  const uint8_t* codes;     // 4-bit tables
  void* grad;               // dW [V, H] or dS [V, G]
  float* part;              // sums of whole chunks of one id, [chunks, H]
  int T, V, H, chunk;
  float factor;
};

// v += the rows of tokens at places [a, b).
template <bool BF16>
__device__ __forceinline__ void add_rows(const EmbedArgs& g, int a, int b, int h, float (&v)[8]) {
  int s = a;
  for (; s + 8 <= b; s += 8) {
    float w[8][8];
#pragma unroll
    for (int u = 0; u < 8; ++u) load8<BF16>(g.d, (int64_t)g.tokens[s + u] * g.H + h, w[u]);
#pragma unroll
    for (int u = 0; u < 8; ++u)
#pragma unroll
      for (int k = 0; k < 8; ++k) v[k] += w[u][k];
  }
  for (; s < b; ++s) {
    float w[8];
    load8<BF16>(g.d, (int64_t)g.tokens[s] * g.H + h, w);
#pragma unroll
    for (int k = 0; k < 8; ++k) v[k] += w[k];
  }
}

// Chunks of places that one id holds whole: their sums, so that an id with many tokens
// is summed by many workgroups.
template <bool BF16>
__global__ __launch_bounds__(256) void embed_chunk_kernel(EmbedArgs g) {
  const int a = (int)blockIdx.x * g.chunk, b = a + g.chunk, h = ((int)blockIdx.y * (int)blockDim.x + (int)threadIdx.x) * 8;
  if (b > g.T || g.keys[a] != g.keys[b - 1] || g.keys[a] >= g.V || h >= g.H) return;
  float v[8] = {};
  add_rows<BF16>(g, a, b, h, v);
  store8<false>(g.part, (int64_t)blockIdx.x * g.H + h, v);
}

enum EmbedGrad { kDwF32 = 0, kDwBf16 = 1, kDsMx = 2, kDsNv = 3 };

// The first place of each id sums its run: its tokens in order, whole chunks by
// their sums.
template <int GRAD, bool BF16>
__global__ __launch_bounds__(256) void embed_sum_kernel(EmbedArgs g) {
  const int64_t at = (int64_t)blockIdx.z * kGroupsX + blockIdx.x;
  if (at >= g.T) return;
  const int s = (int)at, key = g.keys[s], lane = threadIdx.x & 63;
  if (key >= g.V || (s > 0 && g.keys[s - 1] == key)) return;
  int end = s;
  for (;;) {
    const uint64_t other = __ballot(end + lane >= g.T || g.keys[min(end + lane, g.T - 1)] != key);
    if (other) {
      end += __builtin_ctzll(other);
      break;
    }
    end += 64;
  }
  const int h = ((int)blockIdx.y * (int)blockDim.x + (int)threadIdx.x) * 8;
  const bool in = h < g.H;                                    // the lanes of a block are all in or all out
  float v[8] = {};
  if (in) {
    const int c0 = (s + g.chunk - 1) / g.chunk, c1 = end / g.chunk;
    if (c0 < c1) {
      add_rows<BF16>(g, s, c0 * g.chunk, h, v);
#pragma unroll 8
      for (int c = c0; c < c1; ++c) {
        float w[8];
        load8<false>(g.part, (int64_t)c * g.H + h, w);
#pragma unroll
        for (int k = 0; k < 8; ++k) v[k] += w[k];
      }
      add_rows<BF16>(g, c1 * g.chunk, end, h, v);
    } else {
      add_rows<BF16>(g, s, end, h, v);
    }
  }
  if constexpr (GRAD == kDwF32 || GRAD == kDwBf16) {
#pragma unroll
    for (int k = 0; k < 8; ++k) v[k] *= g.factor;
    if (in) store8<GRAD == kDwBf16>(g.grad, (int64_t)key * g.H + h, v);
  } else {
    constexpr int kLanes = GRAD == kDsMx ? 4 : 2;
    const uint32_t q = in ? *reinterpret_cast<const uint32_t*>(g.codes + ((int64_t)key * g.H + h) / 2) : 0u;
    const f32x2 c[4] = {__builtin_amdgcn_cvt_scalef32_pk_f32_fp4(q, 1.0f, 0), __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(q, 1.0f, 1),
                        __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(q, 1.0f, 2), __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(q, 1.0f, 3)};
    float sum = 0.0f;
#pragma unroll
    for (int k = 0; k < 4; ++k) sum += v[2 * k] * c[k].x + v[2 * k + 1] * c[k].y;
    sum += __shfl_xor(sum, 1);
    if (kLanes == 4) sum += __shfl_xor(sum, 2);
    constexpr int kBlock = 8 * kLanes;
    if (in && lane % kLanes == 0) static_cast<float*>(g.grad)[(int64_t)key * (g.H / kBlock) + h / kBlock] = sum * g.factor;
  }
}

// ------------------------------------------------------------------ plan
inline int64_t up(int64_t v, int64_t m) { return (v + m - 1) / m * m; }

// Tokens per chunk: about as many chunks as tokens in one, where one id has them all.
inline int chunk_of(int64_t T) {
  int c = 32;
  while ((int64_t)c * c * 16 < T) c *= 2;
  return c;
}

struct EmbedPlan {
  size_t keys, tokens, part, digit, orders[2], place, slot, offsets, sort, total;
};
EmbedPlan embed_plan(int64_t T, int64_t V, int64_t H) {
  EmbedPlan p{};
  size_t at = 0;
  auto take = [&](size_t bytes) {
    const size_t o = at;
    at += (bytes + 255) & ~(size_t)255;
    return o;
  };
  p.keys = take((size_t)T * 4);
  p.tokens = take((size_t)T * 4);
  p.part = take((size_t)(T / chunk_of(T)) * H * 4);
  if (T > kEmbedRankTokens) {
    p.digit = take((size_t)T * 4);
    for (size_t& o : p.orders) o = take((size_t)T * 4);
    p.place = take((size_t)T * 4);
    p.slot = take((size_t)T * 4);
    p.offsets = take((size_t)(kEmbedDigits + 1) * 4);
    p.sort = take((size_t)((T + kMoeChunk - 1) / kMoeChunk + 1) * (kEmbedDigits + 1) * 4);
  }
  p.total = at;
  return p;
}

__global__ __launch_bounds__(256) void embed_clear_kernel(float* __restrict__ grad, int64_t words) {
  const int64_t n = (int64_t)gridDim.x * 256, at = (int64_t)blockIdx.x * 256 + threadIdx.x;
  for (int64_t i = at; i < words / 4; i += n) reinterpret_cast<f32x4*>(grad)[i] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
  if (at < words % 4) grad[words / 4 * 4 + at] = 0.0f;
}

// Tokens sorted by id into the workspace, and `words` words of the gradient cleared.
int embed_sort(const EmbedPlan& p, const void* ids, int id_bytes, int T, int V, uint8_t* ws, void* grad, int64_t words, hipStream_t s) {
  int* keys = reinterpret_cast<int*>(ws + p.keys);
  int* tokens = reinterpret_cast<int*>(ws + p.tokens);
  const int64_t want = (words / 4 + 4095) / 4096;             // workgroups of the clearing, 4 steps each
  const int clear = (int)(want < 1 ? 1 : want < 2048 ? want : 2048);
  if (T <= kEmbedRankTokens) {
    hipLaunchKernelGGL(embed_rank_kernel, dim3((unsigned)((T + 63) / 64 + clear)), dim3(1024), 0, s, ids, id_bytes, T, V, keys,
                       tokens, static_cast<float*>(grad), words);
    return ok();
  }
  hipLaunchKernelGGL(embed_clear_kernel, dim3((unsigned)(4 * clear)), dim3(256), 0, s, static_cast<float*>(grad), words);
  if (ok() != 0) return -1;
  int* digit = reinterpret_cast<int*>(ws + p.digit);
  int* place = reinterpret_cast<int*>(ws + p.place);
  const dim3 grid((unsigned)((T + 255) / 256)), block(256);
  const int* from = nullptr;
  for (int pass = 0;; ++pass) {
    const int shift = pass * kEmbedDigitBits;
    hipLaunchKernelGGL(embed_digit_kernel, grid, block, 0, s, ids, id_bytes, T, V, from, shift, kEmbedDigits - 1, digit);
    if (ok() != 0) return -1;
    if (moe_sort_launch(T, 1, kEmbedDigits, digit, 4, reinterpret_cast<int*>(ws + p.offsets), place,
                        reinterpret_cast<int*>(ws + p.slot), ws + p.sort, s) != 0)
      return -1;
    const bool last = (int64_t)V >> (shift + kEmbedDigitBits) == 0;      // the keys are 0 .. V
    int* out = last ? tokens : reinterpret_cast<int*>(ws + p.orders[pass & 1]);
    hipLaunchKernelGGL(embed_order_kernel, grid, block, 0, s, ids, id_bytes, T, V, from, place, last ? keys : nullptr, out);
    if (ok() != 0) return -1;
    if (last) return 0;
    from = out;
  }
}

template <int GRAD, bool BF16>
int embed_sums(const EmbedArgs& g, hipStream_t s) {
  const int block = (int)(up(g.H / 8, 64) < 256 ? up(g.H / 8, 64) : 256);
  const unsigned slabs = (unsigned)((g.H / 8 + block - 1) / block);
  const int chunks = g.T / g.chunk;
  if (chunks > 0) {
    hipLaunchKernelGGL((embed_chunk_kernel<BF16>), dim3((unsigned)chunks, slabs), dim3(block), 0, s, g);
    if (ok() != 0) return -1;
  }
  const dim3 grid((unsigned)(g.T < kGroupsX ? g.T : kGroupsX), slabs, (unsigned)((g.T + kGroupsX - 1) / kGroupsX));
  hipLaunchKernelGGL((embed_sum_kernel<GRAD, BF16>), grid, dim3(block), 0, s, g);
  return ok();
}

}  // namespace

int embed_launch(int head, int64_t T, int V, int H, const void* ids, int id_bytes, const void* W, const uint8_t* scales,
                 float ws2, float factor, void* out, int out_bf16, hipStream_t s) {
  const int block = (int)(up(H / 8, 64) < 256 ? up(H / 8, 64) : 256);
  const dim3 grid((unsigned)(T < kGroupsX ? T : kGroupsX), (unsigned)((T + kGroupsX - 1) / kGroupsX));
  auto go = [&](auto kernel) {
    hipLaunchKernelGGL(kernel, grid, dim3(block), 0, s, ids, id_bytes, T, V, H, W, scales, ws2, factor, out);
    return ok();
  };
  if (head == kMX) return out_bf16 ? go(embed_kernel<kMX, true>) : go(embed_kernel<kMX, false>);
  if (head == kNV) return out_bf16 ? go(embed_kernel<kNV, true>) : go(embed_kernel<kNV, false>);
  return out_bf16 ? go(embed_kernel<kCeBf16, true>) : go(embed_kernel<kCeBf16, false>);
}

size_t embed_workspace(int64_t T, int64_t V, int64_t H) { return embed_plan(T, V, H).total; }

// head: kMX or kNV (grad fp32 [V, G]), or kCeBf16 (grad [V, H] in fp32 or bf16).
int embed_bwd_launch(int head, int T, int V, int H, const void* ids, int id_bytes, const void* dOut, int d_bf16, float factor,
                     const uint8_t* codes, void* grad, int grad_bf16, void* workspace, hipStream_t s) {
  const EmbedPlan p = embed_plan(T, V, H);
  uint8_t* ws = static_cast<uint8_t*>(workspace);
  const int64_t cols = head == kCeBf16 ? H : H / (head == kMX ? 32 : 16);
  const int64_t words = (int64_t)V * cols / (head == kCeBf16 && grad_bf16 ? 2 : 1);
  if (T == 0) {
    const int64_t want = (words / 4 + 1023) / 1024;
    hipLaunchKernelGGL(embed_clear_kernel, dim3((unsigned)(want < 1 ? 1 : want < 8192 ? want : 8192)), dim3(256), 0, s,
                       static_cast<float*>(grad), words);
    return ok();
  }
  if (embed_sort(p, ids, id_bytes, T, V, ws, grad, words, s) != 0) return -1;
  EmbedArgs g{};
  g.keys = reinterpret_cast<int*>(ws + p.keys);
  g.tokens = reinterpret_cast<int*>(ws + p.tokens);
  g.part = reinterpret_cast<float*>(ws + p.part);
  g.d = dOut; g.codes = codes; g.grad = grad;
  g.T = T; g.V = V; g.H = H; g.chunk = chunk_of(T); g.factor = factor;
  if (head == kMX) return d_bf16 ? embed_sums<kDsMx, true>(g, s) : embed_sums<kDsMx, false>(g, s);
  if (head == kNV) return d_bf16 ? embed_sums<kDsNv, true>(g, s) : embed_sums<kDsNv, false>(g, s);
  if (grad_bf16) return d_bf16 ? embed_sums<kDwBf16, true>(g, s) : embed_sums<kDwBf16, false>(g, s);
  return d_bf16 ? embed_sums<kDwF32, true>(g, s) : embed_sums<kDwF32, false>(g, s);
}

}  // namespace sq
