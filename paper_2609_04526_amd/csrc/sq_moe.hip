// Tokens to experts and back: the stable sort of routed (token, k) pairs by
// expert, the rows laid out expert by expert, and their weighted sum per token
// with its gradients.  All of it is bound by memory or, for few tokens, by
// launches.
//
// Pair p = t K + k.  key(p) = ids[p], or E when that is no expert (dropped).
//   slot[p]  = #{q : key(q) < key(p)} + #{q < p : key(q) = key(p)}
// is a permutation of 0 .. N - 1 (N = T K); dropped pairs come last, so a pair
// is routed when its slot lies below offsets[E].  Slots that the caller hands
// back are device data: one outside 0 .. N - 1 counts as dropped and is never
// used as an address.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <type_traits>

#include "sq_device.h"
#include "sq_launch.h"

namespace sq {

namespace {

typedef uint32_t u32x4m __attribute__((ext_vector_type(4)));

// ------------------------------------------------------------------ sort
template <typename ID>
__device__ __forceinline__ int key_of(const ID* ids, int64_t p, int64_t N, int E) {
  if (p >= N) return E + 1;                                   // no pair
  const ID v = ids[p];
  return v >= 0 && v < (ID)E ? (int)v : E;
}

__device__ __forceinline__ int lanes_below(uint64_t mask) {
  return __builtin_amdgcn_mbcnt_hi((uint32_t)(mask >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)mask, 0));
}

// 4 pairs from p on, of a step that ends at `end` (<= N): one access where they
// are whole, and its width is left to the ids' own alignment.
template <typename ID>
__device__ __forceinline__ void keys4(const ID* ids, int p, int end, int E, int (&k)[4]) {
  struct __attribute__((packed, aligned(alignof(ID)))) Four { ID v[4]; };
  if (p + 4 <= end) {
    const Four f = *reinterpret_cast<const Four*>(ids + p);
#pragma unroll
    for (int j = 0; j < 4; ++j) k[j] = (int)min((std::make_unsigned_t<ID>)f.v[j], (std::make_unsigned_t<ID>)E);
  } else {
#pragma unroll
    for (int j = 0; j < 4; ++j) k[j] = key_of(ids, p + j, end, E);
  }
}

// One launch, workgroup e owns key e: it counts the pairs of smaller keys (the
// key's first slot) and its own (its waves' shares, each wave a contiguous run
// of pairs), then numbers its own.  A lane takes 4 consecutive pairs of 256 and
// keeps one bit for each that is its key's, so the ids are read once, 4 steps'
// loads together, and 4 ballots order a step.  Every workgroup reads all ids,
// which stay in L2; nothing is exchanged between workgroups.  8 pairs take 3.7 us,
// 32768 of 128 experts 13.3: the ids' round trips and comparisons, since every key
// meets every id.
template <typename ID>
__global__ __launch_bounds__(1024) void moe_sort_kernel(const ID* __restrict__ ids, int N, int K, int E,
                                                        int* __restrict__ offsets, int* __restrict__ token,
                                                        int* __restrict__ slot) {
  __shared__ int s_eq[16], s_lt[16];
  const int e = (int)blockIdx.x;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), waves = blockDim.x >> 6;
  const int per = ((N + waves - 1) / waves + 255) & ~255;     // at most 16 steps
  const int p0 = wave * per, p1 = min(p0 + per, N);
  int lt = 0;
  uint64_t mine = 0;                                          // bit 4 step + j
  for (int st = 0; p0 + 256 * st < p1; st += 4) {
    int k[4][4];
#pragma unroll
    for (int u = 0; u < 4; ++u) keys4(ids, p0 + 256 * (st + u) + 4 * lane, p1, E, k[u]);
    uint32_t bits = 0;
#pragma unroll
    for (int u = 0; u < 4; ++u)
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        lt += k[u][j] < e;
        bits |= k[u][j] == e ? 1u << (4 * u + j) : 0u;
      }
    mine |= (uint64_t)bits << (4 * st);
  }
  int eq = __popcll(mine);
#pragma unroll
  for (int d = 32; d; d >>= 1) {
    eq += __shfl_xor(eq, d);
    lt += __shfl_xor(lt, d);
  }
  if (lane == 0) {
    s_eq[wave] = eq;
    s_lt[wave] = lt;
  }
  __syncthreads();
  int base = 0, before = 0;
  for (int w = 0; w < waves; ++w) {
    base += s_lt[w];
    before += w < wave ? s_eq[w] : 0;
  }
  if (threadIdx.x == 0) offsets[e] = base;       // key E, the dropped pairs: the routed count
  int next = base + before;
  if (eq == 0) return;                           // after the last barrier; uniform in the wave
  for (int st = 0; p0 + 256 * st < p1; ++st) {
    const uint32_t m = (uint32_t)(mine >> (4 * st)) & 15u;
    int rank = next;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const uint64_t b = __ballot((m >> j) & 1);
      rank += lanes_below(b);
      next += __popcll(b);
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      if (!((m >> j) & 1)) continue;
      const uint32_t q = (uint32_t)(p0 + 256 * st + 4 * lane + j);
      slot[q] = rank;
      token[rank] = (int)(q / (uint32_t)K);
      ++rank;
    }
  }
}

// Three launches for many pairs, whose ids every workgroup of the form above
// would read once per key: counts per chunk and key, running sums over the
// chunks of each key, and the numbering of each chunk's pairs.
template <typename ID>
__global__ __launch_bounds__(256) void moe_count_kernel(const ID* __restrict__ ids, int64_t N, int E,
                                                        int* __restrict__ count) {
  extern __shared__ int s_hist[];
  for (int e = threadIdx.x; e <= E; e += 256) s_hist[e] = 0;
  __syncthreads();
  const int64_t p0 = (int64_t)blockIdx.x * kMoeChunk;
#pragma unroll
  for (int i = 0; i < kMoeChunk / 256; ++i) {
    const int k = key_of(ids, p0 + i * 256 + threadIdx.x, N, E);
    if (k <= E) atomicAdd(&s_hist[k], 1);
  }
  __syncthreads();
  for (int e = threadIdx.x; e <= E; e += 256) count[(int64_t)blockIdx.x * (E + 1) + e] = s_hist[e];
}

// Workgroup e: count[c][e] becomes the pairs of key e in chunks before c; the
// sum goes to total[e].
__global__ __launch_bounds__(256) void moe_scan_kernel(int* __restrict__ count, int chunks, int E,
                                                       int* __restrict__ total) {
  __shared__ int s_wave[4];
  const int e = (int)blockIdx.x, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  int run = 0;
  for (int c0 = 0; c0 < chunks; c0 += 256) {
    const int c = c0 + (int)threadIdx.x;
    const int v = c < chunks ? count[(int64_t)c * (E + 1) + e] : 0;
    int s = v;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
      const int u = __shfl_up(s, d);
      if (lane >= d) s += u;
    }
    if (lane == 63) s_wave[wave] = s;
    __syncthreads();
    int before = run, all = 0;
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      before += w < wave ? s_wave[w] : 0;
      all += s_wave[w];
    }
    if (c < chunks) count[(int64_t)c * (E + 1) + e] = before + s - v;
    run += all;
    __syncthreads();
  }
  if (threadIdx.x == 0) total[e] = run;
}

// Workgroup c numbers the pairs of chunk c.  Its 4 waves take a quarter each;
// next[w][e] starts at the slot of wave w's first pair of key e, and 64 pairs
// at a time find the lanes of equal key by ballots over the key's bits.
template <typename ID>
__global__ __launch_bounds__(256) void moe_number_kernel(const ID* __restrict__ ids, int64_t N, int K, int E, int bits,
                                                         const int* __restrict__ count, const int* __restrict__ total,
                                                         int* __restrict__ offsets, int* __restrict__ token,
                                                         int* __restrict__ slot) {
  extern __shared__ int s_next[];                             // [4][E + 1], then the keys' first slots [E + 1]
  int* const s_base = s_next + 4 * (E + 1);
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  for (int i = tid; i < 4 * (E + 1); i += 256) s_next[i] = 0;
  if (wave == 0) {                                            // exclusive sums of total
    int run = 0;
    for (int e0 = 0; e0 <= E; e0 += 64) {
      const int e = e0 + lane, v = e <= E ? total[e] : 0;
      int s = v;
#pragma unroll
      for (int d = 1; d < 64; d <<= 1) {
        const int u = __shfl_up(s, d);
        if (lane >= d) s += u;
      }
      if (e <= E) s_base[e] = run + s - v;
      run += __shfl(s, 63);
    }
  }
  __syncthreads();
  constexpr int kPer = kMoeChunk / 4;
  const int64_t p0 = (int64_t)blockIdx.x * kMoeChunk + wave * kPer;
#pragma unroll 4
  for (int i = 0; i < kPer / 64; ++i) {
    const int k = key_of(ids, p0 + i * 64 + lane, N, E);
    if (k <= E) atomicAdd(&s_next[wave * (E + 1) + k], 1);
  }
  __syncthreads();
  for (int e = tid; e <= E; e += 256) {
    int at = s_base[e] + count[(int64_t)blockIdx.x * (E + 1) + e];
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      const int n = s_next[w * (E + 1) + e];
      s_next[w * (E + 1) + e] = at;
      at += n;
    }
    if (blockIdx.x == 0) offsets[e] = s_base[e];
  }
  __syncthreads();
  int* const next = s_next + wave * (E + 1);
#pragma unroll 4
  for (int i = 0; i < kPer / 64; ++i) {
    const int64_t p = p0 + i * 64 + lane;
    const int k = key_of(ids, p, N, E);
    uint64_t same = __ballot(k <= E);
    for (int b = 0; b < bits; ++b) {
      const uint64_t m = __ballot((k >> b) & 1);
      same &= (k >> b) & 1 ? m : ~m;
    }
    if (k <= E) {
      const int rank = lanes_below(same);
      const int at = next[k] + rank;
      slot[p] = at;
      token[at] = (int)(p / K);
      // the last lane of the key moves its counter; the wave's LDS operations
      // take effect in program order, so every lane has read it
      if ((same >> lane) == 1) next[k] = at + 1;
    }
    __builtin_amdgcn_wave_barrier();
  }
}

// ------------------------------------------------------------------ rows
// 8 elements of a row: 16 bytes of bf16 or 32 of fp32, as loaded and as fp32.
template <bool BF16>
struct Raw8 {
  u32x4m w[BF16 ? 1 : 2];
  template <bool STREAM = false>
  __device__ __forceinline__ void load(const void* base, int64_t at) {
    const u32x4m* q = reinterpret_cast<const u32x4m*>(static_cast<const uint8_t*>(base) + at * (BF16 ? 2 : 4));
#pragma unroll
    for (int i = 0; i < (BF16 ? 1 : 2); ++i) w[i] = STREAM ? __builtin_nontemporal_load(q + i) : q[i];
  }
  __device__ __forceinline__ float at(int i) const {
    if constexpr (BF16) return __uint_as_float(i & 1 ? w[0][i >> 1] & 0xFFFF0000u : w[0][i >> 1] << 16);
    else return __uint_as_float(w[i >> 2][i & 3]);
  }
};
template <bool BF16>
__device__ __forceinline__ void store8(const float (&v)[8], void* base, int64_t at) {
  u32x4m* q = reinterpret_cast<u32x4m*>(static_cast<uint8_t*>(base) + at * (BF16 ? 2 : 4));
  if constexpr (BF16) {
    u32x4m w;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const bf16x2 b = __builtin_convertvector((f32x2{v[2 * i], v[2 * i + 1]}), bf16x2);
      w[i] = bits_of(b);
    }
    q[0] = w;
  } else {
    q[0] = u32x4m{__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3])};
    q[1] = u32x4m{__float_as_uint(v[4]), __float_as_uint(v[5]), __float_as_uint(v[6]), __float_as_uint(v[7])};
  }
}

// Workgroups by token, on in y where x is full.
__device__ __forceinline__ int64_t group_at() { return (int64_t)blockIdx.y * kGroupsX + blockIdx.x; }
inline dim3 groups_of(int64_t n) {
  return dim3((unsigned)(n < kGroupsX ? n : kGroupsX), (unsigned)((n + kGroupsX - 1) / kGroupsX));
}

// Workgroup t: row t of X (units 16-byte pieces) to the slots of its K pairs;
// dropped pairs' rows are zeros.  Bound by memory: 4096 x 2048 bf16 to 8 rows each
// 22.9 us, 6.6 TB/s of reads and writes.
__global__ __launch_bounds__(256) void moe_gather_kernel(const u32x4m* __restrict__ X, const int* __restrict__ slot,
                                                         const int* __restrict__ routed, int64_t T, int K, int units,
                                                         int64_t N, u32x4m* __restrict__ Xs) {
  const int64_t t = group_at();
  if (t >= T) return;
  const int R = *routed;
  for (int c = threadIdx.x; c < units; c += blockDim.x) {
    const u32x4m v = X[t * units + c], zero = {0u, 0u, 0u, 0u};
    for (int k = 0; k < K; ++k) {
      const int at = slot[t * K + k];
      if ((uint32_t)at < (uint64_t)N) Xs[(int64_t)at * units + c] = at < R ? v : zero;
    }
  }
}

// Rows are taken kPairs at a time: the loads of a batch go out together and
// carry no branches but the uniform one on K (a dropped pair reads row 0 and
// its value is not used).
constexpr int kPairs = 8;

// Workgroup t: out[t] = sum over k of w[t,k] Ys[slot[t,k]] in k order, fp32,
// over the routed pairs.  Bound by memory: 8 rows of 2048 bf16 each to 16384 tokens
// 106 us (5.7 TB/s), weighted 113.  STREAM: rows that do not fit the caches, read
// past them, do not wait for what was written last to leave (120 and 143 us there
// without; 333 tokens, 2 rows of 4104 fp32, which fit: 4.9 us, with it 6.0).
template <bool YB, bool OB, bool WEIGHTED, bool STREAM>
__global__ __launch_bounds__(256) void moe_combine_kernel(const void* __restrict__ Ys, const int* __restrict__ slot,
                                                          const int* __restrict__ routed,
                                                          const float* __restrict__ weights, int64_t T, int K, int H,
                                                          int64_t N, void* __restrict__ out) {
  const int64_t t = group_at();
  if (t >= T) return;
  const uint32_t R = (uint32_t)min((int64_t)max(*routed, 0), N);
  for (int c = threadIdx.x * 8; c < H; c += blockDim.x * 8) {
    float acc[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) acc[i] = 0.0f;
    for (int k0 = 0; k0 < K; k0 += kPairs) {
      Raw8<YB> v[kPairs];
      uint32_t at[kPairs];
      float w[kPairs];
#pragma unroll
      for (int k = 0; k < kPairs; ++k) {
        at[k] = R;
        w[k] = 1.0f;
        if (k0 + k >= K) continue;
        at[k] = (uint32_t)slot[t * K + k0 + k];
        if (WEIGHTED) w[k] = weights[t * K + k0 + k];
        v[k].template load<STREAM>(Ys, (int64_t)(at[k] < R ? at[k] : 0u) * H + c);
      }
#pragma unroll
      for (int k = 0; k < kPairs; ++k) {
        if (k0 + k >= K) continue;
#pragma unroll
        for (int i = 0; i < 8; ++i) acc[i] = at[k] < R ? __builtin_fmaf(w[k], v[k].at(i), acc[i]) : acc[i];
      }
    }
    store8<OB>(acc, out, t * H + c);
  }
}

// Gradients of the weighted sum.  WAVES waves take token t: the rows of dYs
// are written as the rows of Ys are read for the weights' gradients.  Bound by
// memory: 16384 tokens, 8 rows of 2048 bf16 each 223 us, 5.1 TB/s.  Many tokens take a
// wave each, whose sums need no exchange; few take 4 (333 tokens, 2 rows of 4104 fp32:
// 8.2 us).
template <bool DB, bool YB, bool GB, int WAVES>
__global__ __launch_bounds__(256) void moe_combine_bwd_kernel(const void* __restrict__ dOut, const void* __restrict__ Ys,
                                                              const int* __restrict__ slot,
                                                              const int* __restrict__ routed,
                                                              const float* __restrict__ weights, int64_t T, int K, int H,
                                                              int64_t N, void* __restrict__ dYs,
                                                              float* __restrict__ dw) {
  constexpr int kTokens = 4 / WAVES;
  __shared__ float s_part[4][kPairs];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int wave_u = __builtin_amdgcn_readfirstlane(wave);
  const int64_t t = group_at() * kTokens + wave_u / WAVES;
  const int in = (wave % WAVES) * 64 + lane;                  // of the token's 64 WAVES lanes
  const uint32_t R = (uint32_t)min((int64_t)max(*routed, 0), N);
  for (int k0 = 0; k0 < K; k0 += kPairs) {
    float dot[kPairs];
#pragma unroll
    for (int k = 0; k < kPairs; ++k) dot[k] = 0.0f;
    if (t < T) {
      uint32_t at[kPairs];
      float w[kPairs];
#pragma unroll
      for (int k = 0; k < kPairs; ++k) {
        at[k] = ~0u;
        w[k] = 0.0f;
        if (k0 + k >= K) continue;
        at[k] = (uint32_t)slot[t * K + k0 + k];
        w[k] = weights[t * K + k0 + k];
      }
      for (int c = in * 8; c < H; c += WAVES * 64 * 8) {
        Raw8<DB> d;
        Raw8<YB> y[kPairs];
        d.load(dOut, t * H + c);
#pragma unroll
        for (int k = 0; k < kPairs; ++k)
          if (k0 + k < K) y[k].load(Ys, (int64_t)(at[k] < R ? at[k] : 0u) * H + c);
#pragma unroll
        for (int k = 0; k < kPairs; ++k) {
          if (k0 + k >= K) continue;
          const bool live = at[k] < R;
          float g[8];
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            dot[k] = live ? __builtin_fmaf(d.at(i), y[k].at(i), dot[k]) : dot[k];
            g[i] = live ? w[k] * d.at(i) : 0.0f;
          }
          if (at[k] < (uint64_t)N) store8<GB>(g, dYs, (int64_t)at[k] * H + c);
        }
      }
    }
#pragma unroll
    for (int k = 0; k < kPairs; ++k) {
#pragma unroll
      for (int s = 32; s; s >>= 1) dot[k] += __shfl_xor(dot[k], s);
    }
    if constexpr (WAVES == 1) {
      if (t < T && lane < kPairs && k0 + lane < K) {
        float v = dot[0];
#pragma unroll
        for (int k = 1; k < kPairs; ++k) v = lane == k ? dot[k] : v;
        dw[t * K + k0 + lane] = v;
      }
    } else {
      if (lane == 0) {
#pragma unroll
        for (int k = 0; k < kPairs; ++k) s_part[wave][k] = dot[k];
      }
      __syncthreads();
      if (t < T && in < kPairs && k0 + in < K) {
        const int w0 = wave / WAVES * WAVES;
        float v = s_part[w0][in];
#pragma unroll
        for (int w = 1; w < WAVES; ++w) v += s_part[w0 + w][in];
        dw[t * K + k0 + in] = v;
      }
      __syncthreads();
    }
  }
}

inline int ok() { return hipGetLastError() == hipSuccess ? 0 : -1; }

inline unsigned row_threads(int64_t pieces) {
  return (unsigned)(pieces >= 256 ? 256 : (pieces + 63) / 64 * 64);
}

template <typename ID>
int sort_go(int64_t N, int K, int E, const ID* ids, int* offsets, int* token, int* slot, int* workspace, hipStream_t s) {
  if (moe_sort_one(N)) {
    const int64_t need = (N + 255) / 256 * 64;                // a wave orders 256 pairs per step
    const unsigned threads = (unsigned)(need >= 1024 ? 1024 : (need < 64 ? 64 : need));
    hipLaunchKernelGGL((moe_sort_kernel<ID>), dim3((unsigned)(E + 1)), dim3(threads), 0, s, ids, (int)N, K, E, offsets, token, slot);
    return ok();
  }
  const int chunks = (int)((N + kMoeChunk - 1) / kMoeChunk);
  int* const total = workspace;
  int* const count = workspace + (E + 1);
  int bits = 0;
  while ((E >> bits) != 0) ++bits;
  hipLaunchKernelGGL((moe_count_kernel<ID>), dim3((unsigned)chunks), dim3(256), (size_t)(E + 1) * 4, s, ids, N, E, count);
  if (ok() != 0) return -1;
  hipLaunchKernelGGL(moe_scan_kernel, dim3((unsigned)(E + 1)), dim3(256), 0, s, count, chunks, E, total);
  if (ok() != 0) return -1;
  hipLaunchKernelGGL((moe_number_kernel<ID>), dim3((unsigned)chunks), dim3(256), (size_t)(E + 1) * 20, s, ids, N, K, E,
                     bits, count, total, offsets, token, slot);
  return ok();
}

}  // namespace

int moe_sort_launch(int64_t T, int K, int E, const void* ids, int id_bytes, int32_t* offsets, int32_t* token,
                    int32_t* slot, void* workspace, hipStream_t s) {
  const int64_t N = T * K;
  return id_bytes == 8 ? sort_go(N, K, E, static_cast<const int64_t*>(ids), offsets, token, slot, static_cast<int*>(workspace), s)
                       : sort_go(N, K, E, static_cast<const int32_t*>(ids), offsets, token, slot, static_cast<int*>(workspace), s);
}

int moe_gather_launch(int64_t T, int K, int H, int bf16, const void* X, const int32_t* slot, const int32_t* routed,
                      void* Xs, hipStream_t s) {
  const int units = H / (bf16 ? 8 : 4);
  hipLaunchKernelGGL(moe_gather_kernel, groups_of(T), dim3(row_threads(units)), 0, s,
                     static_cast<const u32x4m*>(X), slot, routed, T, K, units, T * K, static_cast<u32x4m*>(Xs));
  return ok();
}

int moe_combine_launch(int64_t T, int K, int H, const void* Ys, int y_bf16, const int32_t* slot, const int32_t* routed,
                       const float* weights, void* out, int out_bf16, hipStream_t s) {
  const dim3 grid = groups_of(T), block(row_threads(H / 8));
  const bool stream = T * K * H * (y_bf16 ? 2 : 4) >= kMoeStreamBytes;
  auto go = [&](auto YB, auto OB, auto W) {
    constexpr bool y = decltype(YB)::value, o = decltype(OB)::value, w = decltype(W)::value;
    if (stream)
      hipLaunchKernelGGL((moe_combine_kernel<y, o, w, true>), grid, block, 0, s, Ys, slot, routed, weights, T, K, H, T * K, out);
    else
      hipLaunchKernelGGL((moe_combine_kernel<y, o, w, false>), grid, block, 0, s, Ys, slot, routed, weights, T, K, H, T * K, out);
    return ok();
  };
  using Y = std::true_type;
  using F = std::false_type;
  auto by_weights = [&](auto YB, auto OB) { return weights ? go(YB, OB, Y{}) : go(YB, OB, F{}); };
  if (y_bf16) return out_bf16 ? by_weights(Y{}, Y{}) : by_weights(Y{}, F{});
  return out_bf16 ? by_weights(F{}, Y{}) : by_weights(F{}, F{});
}

int moe_combine_bwd_launch(int64_t T, int K, int H, const void* dOut, int d_bf16, const void* Ys, int y_bf16,
                           const int32_t* slot, const int32_t* routed, const float* weights, void* dYs, int g_bf16,
                           float* dw, hipStream_t s) {
  auto go = [&](auto DB, auto YB, auto GB) {
    constexpr bool d = decltype(DB)::value, y = decltype(YB)::value, g = decltype(GB)::value;
    if (T >= kMoeWaveTokens)
      hipLaunchKernelGGL((moe_combine_bwd_kernel<d, y, g, 1>), groups_of((T + 3) / 4), dim3(256), 0, s, dOut, Ys,
                         slot, routed, weights, T, K, H, T * K, dYs, dw);
    else
      hipLaunchKernelGGL((moe_combine_bwd_kernel<d, y, g, 4>), groups_of(T), dim3(256), 0, s, dOut, Ys, slot, routed,
                         weights, T, K, H, T * K, dYs, dw);
    return ok();
  };
  using Y = std::true_type;
  using F = std::false_type;
  auto by_g = [&](auto DB, auto YB) { return g_bf16 ? go(DB, YB, Y{}) : go(DB, YB, F{}); };
  if (d_bf16) return y_bf16 ? by_g(Y{}, Y{}) : by_g(Y{}, F{});
  return y_bf16 ? by_g(F{}, Y{}) : by_g(F{}, F{});
}

}  // namespace sq
