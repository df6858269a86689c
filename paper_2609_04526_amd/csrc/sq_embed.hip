// Embedding lookup and its gradients, for tables in bf16 and in the layer's 4-bit
// storage.
//
//   out[t]  = factor W[ids[t]]
//   dW[v]   = factor sum_{t : ids[t] = v} dOut[t]                      (bf16 table)
//   dS[v,g] = factor sum_{j in g} code[v,j] sum_{t : ids[t] = v} dOut[t,j]
//
// All of it is bound by memory.  The gradients sort the tokens by id (stable), sum
// the runs of one id in token order, and write zeros where an id has no token.  The
// only atomics count, so the same bits come out of every run.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <type_traits>

#include "sq_device.h"
#include "sq_launch.h"
#include "sq_rows.h"

namespace sq {

namespace {

inline int ok() { return hipGetLastError() == hipSuccess ? 0 : -1; }

// 16 bytes of a gradient that no token reaches.  They pass the caches by, which such a
// table would fill (gradient of 1999 tokens, 50001 x 2048 fp32: 89 -> 76 us; where nothing
// else runs, in embed_few_kernel, they go through: 80 MB 20 us, so 18).
__device__ __forceinline__ void zero16(u32x4* p) { __builtin_nontemporal_store(u32x4{0u, 0u, 0u, 0u}, p); }

// The id, or V where it is outside the table.
__device__ __forceinline__ int key_at(const void* ids, int bytes, int64_t t, int V) {
  const int64_t v = id_at(ids, bytes, t);
  return v >= 0 && v < V ? (int)v : V;
}

// ------------------------------------------------------------------ lookup
// One token per workgroup, 8 columns per lane and step.  Bound by memory: 16384 tokens of
// 4096 MXFP4 to bf16 27 us (170 MB, 6.3 TB/s).
// PAST: bf16 rows, whole lines at once, pass the caches by, where they and the table's are more
// than these hold: a product reads them next.  us of this kernel and with sq_fwd of 1024
// outputs behind it, through and past them: 2000 tokens of 4096 MXFP4 (21 MB) 6.0, 5.7 and
// 38, 42; 16384 (170) 27, 25.5 and 129, 150; 32768 (340) 74, 50 and 318, 303; bf16 2000 (33) 6.0, 5.2 and
// 38, 42; 16384 (268) 43, 40 and 148, 167; 24000 (393) 68, 57 and 267, 261.
template <int HEAD, bool BF16, bool PAST>
__global__ __launch_bounds__(256) void embed_kernel(const void* __restrict__ ids, int id_bytes, int64_t T, int V, int H,
                                                    const void* __restrict__ W, const uint8_t* __restrict__ scales, float ws2,
                                                    float factor, void* __restrict__ out) {
  static_assert(BF16 || !PAST, "bf16 rows");
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
    if constexpr (PAST) __builtin_nontemporal_store(bf16_of(v), reinterpret_cast<u32x4*>(static_cast<uint16_t*>(out) + t * H + h));
    else store8<BF16>(out, t * H + h, v);
  }
}

// ------------------------------------------------------------------ sort
// What a workgroup of 1024 does with counts [wave][digit] of its tokens: they become the
// places where each wave's tokens of a digit start, behind the smaller digits of all
// tokens, the digit's own before this workgroup (`before`, of digit threadIdx.x) and
// those of its earlier waves; `after`: the digit's tokens past this workgroup.  Gives
// this lane's place among its wave's tokens of digit d.
__device__ __forceinline__ int place_digits(int (&s_next)[16][kEmbedDigits], int (&s_sum)[8], int before, int after, int d, bool in) {
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  int total = 0, upto = 0;
  if (tid < kEmbedDigits) {
    total = before + after;
    for (int w = 0; w < 16; ++w) total += s_next[w][tid];
    upto = total;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const int v = __shfl_up(upto, o);
      upto += lane >= o ? v : 0;
    }
    if (lane == 63) s_sum[wave] = upto;
  }
  __syncthreads();
  if (tid < kEmbedDigits) {
    int at = upto - total + before;
    for (int w = 0; w < wave; ++w) at += s_sum[w];
    for (int w = 0; w < 16; ++w) {
      const int n = s_next[w][tid];
      s_next[w][tid] = at;
      at += n;
    }
  }
  __syncthreads();
  uint64_t same = __ballot(in);
#pragma unroll
  for (int b = 0; b < kEmbedDigitBits; ++b) {
    const uint64_t m = __ballot((d >> b) & 1);
    same &= (d >> b) & 1 ? m : ~m;
  }
  return __builtin_amdgcn_mbcnt_hi((uint32_t)(same >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)same, 0));
}

// Up to 1024 tokens: all passes in one workgroup, through LDS, while the others clear
// the gradient, so that the sums have nothing to clear (a launch and the marks less: 5
// tokens of 1000 x 256 bf16 with the lookup 26 -> 23 us, the host's calls).
__global__ __launch_bounds__(1024) void embed_few_kernel(const void* __restrict__ ids, int id_bytes, int T, int V, int passes,
                                                         int* __restrict__ keys, int* __restrict__ tokens, u32x4* __restrict__ grad,
                                                         int64_t units, int words) {
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  if (blockIdx.x > 0) {
    const int64_t n = (int64_t)(gridDim.x - 1) * 1024, at = (int64_t)(blockIdx.x - 1) * 1024 + tid;
    for (int64_t i = at; i < units; i += n) grad[i] = u32x4{0u, 0u, 0u, 0u};
    if (at < words) reinterpret_cast<uint32_t*>(grad + units)[at] = 0u;
    return;
  }
  __shared__ int s_next[16][kEmbedDigits], s_sum[8], s_key[1024], s_token[1024];
  const bool in = tid < T;
  int key = in ? key_at(ids, id_bytes, tid, V) : 0, token = tid;
  for (int p = 0; p < passes; ++p) {
    for (int i = tid; i < 16 * kEmbedDigits; i += 1024) (&s_next[0][0])[i] = 0;
    __syncthreads();
    const int d = (key >> (p * kEmbedDigitBits)) & (kEmbedDigits - 1);
    if (in) atomicAdd(&s_next[wave][d], 1);
    __syncthreads();
    const int rank = place_digits(s_next, s_sum, 0, 0, d, in);
    if (in) {
      const int at = s_next[wave][d] + rank;
      s_key[at] = key;
      s_token[at] = token;
    }
    __syncthreads();
    if (in) {
      key = s_key[tid];
      token = s_token[tid];
    }
  }
  if (in) {
    keys[tid] = key;
    tokens[tid] = token;
  }
}

// One pass of a stable sort by 9 bits of the keys, from `shift` on: of the ids (FIRST)
// or of the pass before.  A workgroup places 1024 tokens.  It counts the digits of all
// tokens and of those before its own by itself, from keys that stay in L2, so that a
// pass is one launch and nothing is exchanged between workgroups.  The other
// workgroups of the first pass clear `marks`; the last pass sets those of the ids that
// occur.  A pass leaves most CUs idle, so further workgroups clear part of the gradient
// meanwhile, which the sums would have to otherwise, and so they do in the launch of the
// chunks' sums (gradient of 1999 tokens, 50001 x 2048 fp32, 28 MiB a pass 80 us, 40 and 24
// with the chunks 75; 4000 tokens, bf16, 46.8, 42.7).
template <bool FIRST>
__global__ __launch_bounds__(1024) void embed_pass_kernel(const void* __restrict__ ids, int id_bytes, int T, int V,
                                                          const int* __restrict__ keys_in, const int* __restrict__ tokens_in,
                                                          int shift, int* __restrict__ keys, int* __restrict__ tokens,
                                                          uint8_t* __restrict__ marks, int64_t mark_words,
                                                          u32x4* __restrict__ part, int64_t part_words) {
  const int blocks = (T + 1023) / 1024;
  if ((int)blockIdx.x >= blocks) {
    const int64_t n = (int64_t)(gridDim.x - blocks) * 1024, i0 = (int64_t)(blockIdx.x - blocks) * 1024 + threadIdx.x;
    const u32x4 zero = {0u, 0u, 0u, 0u};
    if (FIRST)
      for (int64_t i = i0; i < mark_words; i += n) reinterpret_cast<u32x4*>(marks)[i] = zero;
    for (int64_t i = i0; i < part_words; i += n) zero16(&part[i]);
    return;
  }
  __shared__ int s_all[kEmbedDigits], s_before[kEmbedDigits], s_next[16][kEmbedDigits], s_sum[8];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  for (int d = tid; d < kEmbedDigits; d += 1024) s_all[d] = s_before[d] = 0;
  for (int i = tid; i < 16 * kEmbedDigits; i += 1024) (&s_next[0][0])[i] = 0;
  __syncthreads();
  auto key_of = [&](int i) { return FIRST ? key_at(ids, id_bytes, i, V) : keys_in[i]; };
  auto digit = [&](int k) { return (k >> shift) & (kEmbedDigits - 1); };
  const int own = (int)blockIdx.x * 1024, mine = own + tid;
#pragma unroll 4
  for (int i = tid; i < own; i += 1024) atomicAdd(&s_before[digit(key_of(i))], 1);
#pragma unroll 4
  for (int i = mine + 1024; i < T; i += 1024) atomicAdd(&s_all[digit(key_of(i))], 1);
  const bool in = mine < T;
  const int key = in ? key_of(mine) : 0, d = digit(key);
  if (in) atomicAdd(&s_next[wave][d], 1);
  __syncthreads();
  const int rank = place_digits(s_next, s_sum, tid < kEmbedDigits ? s_before[tid] : 0, tid < kEmbedDigits ? s_all[tid] : 0, d, in);
  if (!in) return;
  const int at = s_next[wave][d] + rank;
  keys[at] = key;
  tokens[at] = FIRST ? mine : tokens_in[mine];
  if (!FIRST && marks && key < V) marks[key] = 1;
}

// More tokens than every workgroup should read: the same passes by the sort of routed pairs.
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
                                                          int* __restrict__ keys, int* __restrict__ tokens,
                                                          uint8_t* __restrict__ marks) {
  const int s = (int)blockIdx.x * 256 + threadIdx.x;
  if (s >= T) return;
  const int t = from ? from[place[s]] : place[s];
  tokens[s] = t;
  if (!keys) return;
  const int key = key_at(ids, id_bytes, t, V);
  keys[s] = key;
  if (key < V) marks[key] = 1;
}

// ------------------------------------------------------------------ sums
struct EmbedArgs {
  const int* keys;          // sorted
  const int* tokens;
  const void* d;            // dOut [T, H]
  const uint8_t* codes;     // 4-bit tables
  void* grad;               // dW [V, H] or dS [V, G]
  float* part;              // sums of whole chunks of one id, [chunks, H]
  const uint8_t* marks;     // [V]: the ids that occur
  int T, V, H, chunk;
  int chunks;               // of which the sums are there
  int units, lanes;         // 16-byte (or 4-byte) units of a row of the gradient, and lanes that clear one, a power of 2
  int narrow;               // rows are not whole 16 bytes
  int heads;                // workgroups of the sums, before those that clear
  int64_t clear_from;       // the first row that is not clear yet
  int clear_rows;           // of a workgroup
  u32x4* clear;             // and what the chunks' launch clears, before that row
  int64_t clear_words;
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
  if ((int)blockIdx.x >= g.chunks) {                          // (as in a pass)
    if (blockIdx.y > 0) return;
    const int64_t n = (int64_t)((int)gridDim.x - g.chunks) * blockDim.x;
    for (int64_t i = (int64_t)((int)blockIdx.x - g.chunks) * blockDim.x + threadIdx.x; i < g.clear_words; i += n) zero16(&g.clear[i]);
    return;
  }
  const int a = (int)blockIdx.x * g.chunk, b = a + g.chunk, h = ((int)blockIdx.y * (int)blockDim.x + (int)threadIdx.x) * 8;
  if (b > g.T || g.keys[a] != g.keys[b - 1] || g.keys[a] >= g.V || h >= g.H) return;
  float v[8] = {};
  add_rows<BF16>(g, a, b, h, v);
  store8<false>(g.part, (int64_t)blockIdx.x * g.H + h, v);
}

enum EmbedGrad { kDwF32 = 0, kDwBf16 = 1, kDsMx = 2, kDsNv = 3 };

// Zeros in the rows of ids that do not occur: the i-th `clear_rows` of them, so that the
// workgroups, in their order, write through the memory from its start to its end (1999
// tokens, 50001 x 2048 fp32 in steps of all workgroups 76 us, so 66; 16384 tokens, 100000 x
// 2048 183, 150).
__device__ __forceinline__ void clear_rows(const EmbedArgs& g, int i) {
  const int per = (int)blockDim.x / g.lanes, sub = (int)threadIdx.x / g.lanes, l = (int)threadIdx.x % g.lanes;
  const int64_t r0 = g.clear_from + (int64_t)i * g.clear_rows, end = min(r0 + g.clear_rows, (int64_t)g.V);
  for (int64_t r = r0 + sub; r < end; r += per) {
    if (g.marks[r]) continue;
    for (int u = l; u < g.units; u += g.lanes) {
      if (g.narrow) reinterpret_cast<float*>(g.grad)[r * g.units + u] = 0.0f;
      else zero16(&reinterpret_cast<u32x4*>(g.grad)[r * g.units + u]);
    }
  }
}

// A workgroup has 8 places, and sums the runs that start there: their tokens in order,
// one row after another whichever run they belong to, 8 on their way together.  A run
// that goes on past the 64 places whose keys a wave holds takes whole chunks by their
// sums.  The workgroups past the places clear the rows of ids that do not occur.  16384
// tokens of 131072 x 4096 MXFP4 take 40 us, the rows' 134 MB at 3.4 TB/s: the round trips of
// places, rows and codes; 1999 of 50001 x 2048 bf16 43, of which zeros, 308 MB at 7.1.
template <int GRAD, bool BF16>
__global__ __launch_bounds__(256) void embed_sum_kernel(EmbedArgs g) {
  if ((int)blockIdx.x >= g.heads) {
    if (blockIdx.y == 0) clear_rows(g, (int)blockIdx.x - g.heads);
    return;
  }
  const int lane = threadIdx.x & 63;
  const int h = ((int)blockIdx.y * (int)blockDim.x + (int)threadIdx.x) * 8;
  const bool in = h < g.H;                                    // the lanes of a block are all in or all out
  float v[8];
  auto zero = [&]() {
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = 0.0f;
  };
  auto codes_of = [&](int key) { return in ? *reinterpret_cast<const uint32_t*>(g.codes + ((int64_t)key * g.H + h) / 2) : 0u; };
  // the sums in v to the row of `key`, whose codes are q
  auto put = [&](int key, uint32_t q) {
    if constexpr (GRAD == kDwF32 || GRAD == kDwBf16) {
#pragma unroll
      for (int j = 0; j < 8; ++j) v[j] *= g.factor;
      if (in) store8<GRAD == kDwBf16>(g.grad, (int64_t)key * g.H + h, v);
    } else {
      constexpr int kLanes = GRAD == kDsMx ? 4 : 2, kBlock = 8 * kLanes;
      const f32x2 c[4] = {__builtin_amdgcn_cvt_scalef32_pk_f32_fp4(q, 1.0f, 0), __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(q, 1.0f, 1),
                          __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(q, 1.0f, 2), __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(q, 1.0f, 3)};
      float sum = 0.0f;
#pragma unroll
      for (int j = 0; j < 4; ++j) sum += v[2 * j] * c[j].x + v[2 * j + 1] * c[j].y;
      sum += __shfl_xor(sum, 1);
      if (kLanes == 4) sum += __shfl_xor(sum, 2);
      if (in && lane % kLanes == 0) static_cast<float*>(g.grad)[(int64_t)key * (g.H / kBlock) + h / kBlock] = sum * g.factor;
    }
  };
  for (int64_t at = (int64_t)blockIdx.x * 8; at < g.T; at += (int64_t)g.heads * 8) {
    const int a = (int)at, i = min(a + lane, g.T - 1);
    const int k = g.keys[i], t = g.tokens[i], before = a + lane > 0 ? g.keys[min(a + lane, g.T) - 1] : -1;
    // the places where a run starts, the dropped ids' and the end of all among them
    const uint64_t starts = __ballot(a + lane == g.T || (a + lane < g.T && k != before));
    const uint64_t mine = starts & 0xFFull & __ballot(a + lane < g.T && k < g.V);
    if (!mine) continue;
    const int first = __builtin_ctzll(mine), last = 63 - __builtin_clzll(mine);
    const uint64_t after = starts & ~((2ull << last) - 1);
    const int end = after ? __builtin_ctzll(after) : last;    // of the runs that end inside the 64 places
    for (int p0 = first; p0 < end; p0 += 8) {
      Raw8<BF16> w[8];
      uint32_t q[8];
#pragma unroll
      for (int u = 0; u < 8; ++u) {
        const int p = min(p0 + u, end - 1);
        w[u].load(g.d, in ? (int64_t)__builtin_amdgcn_readlane(t, p) * g.H + h : 0);
        if constexpr (GRAD == kDsMx || GRAD == kDsNv) q[u] = codes_of(__builtin_amdgcn_readlane(k, p));
        else q[u] = 0;
      }
#pragma unroll
      for (int u = 0; u < 8; ++u) {
        const int p = p0 + u;
        if (p >= end) break;
        if ((starts >> p) & 1) zero();
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] += w[u].at(j);
        if (p + 1 == end || ((starts >> (p + 1)) & 1)) put(__builtin_amdgcn_readlane(k, p), q[u]);
      }
    }
    if (after) continue;
    const int s = a + last, key = __builtin_amdgcn_readlane(k, last);
    const uint32_t q = GRAD == kDsMx || GRAD == kDsNv ? codes_of(key) : 0u;
    // where it stops: 64 places at a time tried over what is left, which the first with
    // another key shortens (64 after 64 of them: 16000 tokens of 1000 x 1024 49 us, so 45)
    int stop = a + 64;
    for (int hi = g.T; stop < hi;) {
      const int step = (hi - stop + 63) / 64, p = stop + lane * step;
      const int n = __builtin_popcountll(__ballot(p < hi && g.keys[min(p, g.T - 1)] == key));
      if (n == 0) break;
      hi = min(hi, stop + n * step);
      stop += (n - 1) * step + 1;
    }
    zero();
    if (in) {
      const int c0 = (s + g.chunk - 1) / g.chunk, c1 = stop / g.chunk;
      if (c0 >= c1 || !g.chunks) {                            // no chunk inside the run, or none summed
        add_rows<BF16>(g, s, stop, h, v);
      } else {
        add_rows<BF16>(g, s, c0 * g.chunk, h, v);
#pragma unroll 8
        for (int c = c0; c < c1; ++c) {
          float w[8];
          load8<false>(g.part, (int64_t)c * g.H + h, w);
#pragma unroll
          for (int j = 0; j < 8; ++j) v[j] += w[j];
        }
        add_rows<BF16>(g, c1 * g.chunk, stop, h, v);
      }
    }
    put(key, q);
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
  size_t keys, tokens, part, marks, orders[2], others, place, slot, offsets, sort, total;
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
  p.marks = take((size_t)V);
  for (size_t& o : p.orders) o = take((size_t)T * 4);
  if (T > kEmbedPassTokens) {
    p.others = take((size_t)T * 4);
    p.place = take((size_t)T * 4);
    p.slot = take((size_t)T * 4);
    p.offsets = take((size_t)(kEmbedDigits + 1) * 4);
    p.sort = take((size_t)((T + kMoeChunk - 1) / kMoeChunk + 1) * (kEmbedDigits + 1) * 4);
  }
  p.total = at;
  return p;
}

__global__ __launch_bounds__(256) void embed_clear_kernel(u32x4* __restrict__ to, int64_t units, int words) {
  const int64_t n = (int64_t)gridDim.x * 256, at = (int64_t)blockIdx.x * 256 + threadIdx.x;
  for (int64_t i = at; i < units; i += n) zero16(&to[i]);
  if (at < words) reinterpret_cast<uint32_t*>(to + units)[at] = 0u;
}
int clear(void* to, int64_t bytes, hipStream_t s) {             // bytes a multiple of 4
  const int64_t want = (bytes / 16 + 1023) / 1024;
  hipLaunchKernelGGL(embed_clear_kernel, dim3((unsigned)(want < 1 ? 1 : want < 8192 ? want : 8192)), dim3(256), 0, s,
                     static_cast<u32x4*>(to), bytes / 16, (int)(bytes % 16 / 4));
  return ok();
}

// Tokens sorted by id into the workspace, and the ids that occur marked; *cleared: the
// bytes of the gradient that are zero by then.
constexpr int64_t kEmbedPassClears = int64_t(40) << 20, kEmbedChunkClears = int64_t(24) << 20, kEmbedClearsFrom = int64_t(48) << 20;   // bytes a pass, of so many or more
int embed_sort(const EmbedPlan& p, const void* ids, int id_bytes, int T, int V, uint8_t* ws, void* grad, int64_t bytes,
               int64_t* cleared, hipStream_t s) {
  auto at = [&](size_t o) { return reinterpret_cast<int*>(ws + o); };
  int passes = 1;
  while ((int64_t)V >> (passes * kEmbedDigitBits) > 0) ++passes;         // the keys are 0 .. V
  if (T <= 1024) {
    *cleared = bytes;
    // a store per lane, up to 16 GiB: 2^32 lanes would be cut short
    const int64_t want = bytes / 16 / 1024 + 1;
    hipLaunchKernelGGL(embed_few_kernel, dim3(1 + (unsigned)(want < (1 << 20) ? want : 1 << 20)), dim3(1024), 0, s, ids, id_bytes, T, V,
                       passes, at(p.keys), at(p.tokens), static_cast<u32x4*>(grad), bytes / 16, (int)(bytes % 16 / 4));
    return ok();
  }
  if (T <= kEmbedPassTokens) {
    passes = passes < 2 ? 2 : passes;
    const unsigned blocks = (unsigned)((T + 1023) / 1024);
    const int64_t words = (V + 15) / 16;                      // marks are padded to whole 256 bytes
    const int* keys_in = nullptr;
    const int* tokens_in = nullptr;
    *cleared = 0;
    for (int k = 0; k < passes; ++k) {
      u32x4* part = reinterpret_cast<u32x4*>(static_cast<uint8_t*>(grad) + *cleared);
      const int64_t left = bytes < kEmbedClearsFrom ? 0 : bytes - *cleared, part_words = (left < kEmbedPassClears ? left : kEmbedPassClears) / 16;
      const int64_t most = k == 0 && words > part_words ? words : part_words, more = (most + 4095) / 4096;
      const unsigned others = (unsigned)(more < 1024 ? more : 1024);
      *cleared += part_words * 16;
      const bool last = k + 1 == passes, even = (passes - k) % 2 == 0;
      int* keys = even ? at(p.orders[0]) : at(p.keys);
      int* tokens = even ? at(p.orders[1]) : at(p.tokens);
      uint8_t* marks = k == 0 || last ? ws + p.marks : nullptr;
      if (k == 0)
        hipLaunchKernelGGL((embed_pass_kernel<true>), dim3(blocks + others), dim3(1024), 0, s, ids, id_bytes, T, V, keys_in,
                           tokens_in, 0, keys, tokens, marks, words, part, part_words);
      else
        hipLaunchKernelGGL((embed_pass_kernel<false>), dim3(blocks + others), dim3(1024), 0, s, ids, id_bytes, T, V, keys_in,
                           tokens_in, k * kEmbedDigitBits, keys, tokens, marks, words, part, part_words);
      if (ok() != 0) return -1;
      keys_in = keys;
      tokens_in = tokens;
    }
    return 0;
  }
  *cleared = 0;
  if (clear(ws + p.marks, (int64_t)up(V, 16), s) != 0) return -1;
  const dim3 grid((unsigned)((T + 255) / 256)), block(256);
  const int* from = nullptr;
  for (int k = 0; k < passes; ++k) {
    hipLaunchKernelGGL(embed_digit_kernel, grid, block, 0, s, ids, id_bytes, T, V, from, k * kEmbedDigitBits, kEmbedDigits - 1, at(p.others));
    if (ok() != 0) return -1;
    if (moe_sort_launch(T, 1, kEmbedDigits, at(p.others), 4, at(p.offsets), at(p.place), at(p.slot), ws + p.sort, s) != 0) return -1;
    const bool last = k + 1 == passes;
    int* out = last ? at(p.tokens) : at(p.orders[k & 1]);
    hipLaunchKernelGGL(embed_order_kernel, grid, block, 0, s, ids, id_bytes, T, V, from, at(p.place), last ? at(p.keys) : nullptr, out,
                       ws + p.marks);
    if (ok() != 0) return -1;
    from = out;
  }
  return 0;
}

// What a workgroup clears of a gradient (gradient of 4000 tokens, 50001 x 2048 bf16, with 4, 8
// and 16 KiB 48.4, 42.8, 42.3 us; of 1999, fp32, 65.4, 65.6, 75.7).
constexpr int64_t kEmbedClearBytes = 8192;

// Up to these tokens a run is summed by one workgroup per 2048 columns, whatever its length:
// a launch less (us in a graph, without against with the chunks' sums: 128 tokens of
// 1000 x 4096 9.9, 11.4, all of one id 16.2, 13.4; 256 of one id 26.4, 13.5).
constexpr int kEmbedRunTokens = 128;

template <int GRAD, bool BF16>
int embed_sums(EmbedArgs g, hipStream_t s) {
  const int block = (int)(up(g.H / 8, 64) < 256 ? up(g.H / 8, 64) : 256);
  const int chunks = g.T / g.chunk;
  g.chunks = g.T > kEmbedRunTokens ? chunks : 0;
  if (g.chunks) {
    const int64_t more = (g.clear_words + 4095) / 4096;
    hipLaunchKernelGGL((embed_chunk_kernel<BF16>), dim3((unsigned)(chunks + (more < 1024 ? more : 1024)), (unsigned)((g.H / 8 + block - 1) / block)), dim3(block), 0, s, g);
    if (ok() != 0) return -1;
  }
  const int64_t cols = GRAD == kDsMx ? g.H / 32 : GRAD == kDsNv ? g.H / 16 : GRAD == kDwBf16 ? g.H / 2 : g.H;   // words of a row
  g.narrow = cols % 4 != 0;
  g.units = (int)(g.narrow ? cols : cols / 4);
  g.lanes = 1;
  while (g.lanes < g.units && g.lanes < block) g.lanes *= 2;
  if (block % g.lanes != 0) g.lanes = 64;                     // blocks of 192
  const int groups = (g.T + 7) / 8;
  g.heads = groups < (1 << 20) ? groups : 1 << 20;
  const int64_t row = cols * 4, per = block / g.lanes, some = up(kEmbedClearBytes / row < 1 ? 1 : kEmbedClearBytes / row, per);
  const int64_t most = up((g.V - g.clear_from + (1 << 20) - 1) >> 20, per);
  g.clear_rows = (int)(some > most ? some : most);
  const int64_t clears = (g.V - g.clear_from + g.clear_rows - 1) / g.clear_rows;
  hipLaunchKernelGGL((embed_sum_kernel<GRAD, BF16>), dim3((unsigned)(g.heads + clears), (unsigned)((g.H / 8 + block - 1) / block)),
                     dim3(block), 0, s, g);
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
  // the rows written, and those read, each once at most
  const int64_t row = head == kCeBf16 ? 2 * (int64_t)H : H / 2 + H / (head == kMX ? 32 : 16), bytes = 2 * T * H + (T < V ? T : V) * row;
  const bool past = out_bf16 && bytes > kCacheBytes;
  auto by = [&](auto HEAD) {
    constexpr int h = decltype(HEAD)::value;
    return past ? go(embed_kernel<h, true, true>) : out_bf16 ? go(embed_kernel<h, true, false>) : go(embed_kernel<h, false, false>);
  };
  if (head == kMX) return by(std::integral_constant<int, kMX>{});
  return head == kNV ? by(std::integral_constant<int, kNV>{}) : by(std::integral_constant<int, kCeBf16>{});
}

size_t embed_workspace(int64_t T, int64_t V, int64_t H) { return embed_plan(T, V, H).total; }

// head: kMX or kNV (grad fp32 [V, G]), or kCeBf16 (grad [V, H] in fp32 or bf16).
int embed_bwd_launch(int head, int T, int V, int H, const void* ids, int id_bytes, const void* dOut, int d_bf16, float factor,
                     const uint8_t* codes, void* grad, int grad_bf16, void* workspace, hipStream_t s) {
  const EmbedPlan p = embed_plan(T, V, H);
  uint8_t* ws = static_cast<uint8_t*>(workspace);
  const int64_t cols = head == kCeBf16 ? H : H / (head == kMX ? 32 : 16);
  if (T == 0) return clear(grad, V * cols * (head == kCeBf16 && grad_bf16 ? 2 : 4), s);
  const int64_t row = cols * (head == kCeBf16 && grad_bf16 ? 2 : 4);
  int64_t cleared;
  if (embed_sort(p, ids, id_bytes, T, V, ws, grad, V * row, &cleared, s) != 0) return -1;
  EmbedArgs g{};
  if (T > 1024 && T <= kEmbedPassTokens && V * row >= kEmbedClearsFrom) {      // more of it beside the chunks' sums
    const int64_t left = V * row - cleared;
    g.clear = reinterpret_cast<u32x4*>(static_cast<uint8_t*>(grad) + cleared);
    g.clear_words = (left < kEmbedChunkClears ? left : kEmbedChunkClears) / 16;
    cleared += g.clear_words * 16;
  }
  g.clear_from = cleared / row;
  g.keys = reinterpret_cast<int*>(ws + p.keys);
  g.tokens = reinterpret_cast<int*>(ws + p.tokens);
  g.part = reinterpret_cast<float*>(ws + p.part);
  g.marks = ws + p.marks;
  g.d = dOut; g.codes = codes; g.grad = grad;
  g.T = T; g.V = V; g.H = H; g.chunk = chunk_of(T); g.factor = factor;
  if (head == kMX) return d_bf16 ? embed_sums<kDsMx, true>(g, s) : embed_sums<kDsMx, false>(g, s);
  if (head == kNV) return d_bf16 ? embed_sums<kDsNv, true>(g, s) : embed_sums<kDsNv, false>(g, s);
  if (grad_bf16) return d_bf16 ? embed_sums<kDwBf16, true>(g, s) : embed_sums<kDwBf16, false>(g, s);
  return d_bf16 ? embed_sums<kDwF32, true>(g, s) : embed_sums<kDwF32, false>(g, s);
}

}  // namespace sq
