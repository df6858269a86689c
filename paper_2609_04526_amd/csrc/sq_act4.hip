// Activations in the layer's own 4-bit storage, and the products of two 4-bit
// operands: one layer, or stacked experts on rows whose ranges stay on the device.
//
//   x^[t,i] = code[t,i] sx[t, i/B]          block scale and code as the layer's
//   Y[t,o]  = sum_b sx[t,b] sw[o,b] sum_{i in b} cx[t,i] cw[o,i]
//
// MXFP4's blocks are the matrix cores' own: a scaled product takes 32 codes and
// one E8M0 byte per lane and operand and sums exact products in fp32, at four times
// the rate of bf16 from a quarter of its bytes.  NVFP4's blocks of 16 with E4M3
// scales are not, so its kept rows go through bf16 (code x scale is exact there)
// and the layer's bf16 product.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <type_traits>

#include "sq_device.h"
#include "sq_gemm_args.h"
#include "sq_launch.h"
#include "sq_rtn.h"
#include "sq_tiles.h"

namespace sq {

namespace {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef int i32x8 __attribute__((ext_vector_type(8)));

inline int ok() { return hipGetLastError() == hipSuccess ? 0 : -1; }

// ------------------------------------------------------------------ pack, unpack
constexpr int kSteps = 4;               // pieces of 8 values in flight per lane

// The codes and the scale byte of piece p (8 values; B / 8 adjacent lanes share a
// block): exactly the re-quantiser's nearest rule, but a block that holds an Inf or
// NaN gets the NaN scale and zero codes.
template <int FMT>
__device__ __forceinline__ void pack8(u32x4 h, float ws2, const RcpDivisor& wd, uint8_t* codes, uint8_t* scales, int64_t p) {
  constexpr int kLanes = ScaleOperand<FMT>::kBlock / 8;
  uint32_t am = 0;
#pragma unroll
  for (int k = 0; k < 4; ++k) am = max(am, max(h[k] & 0x7FFFu, (h[k] >> 16) & 0x7FFFu));
  am = max(am, (uint32_t)__shfl_xor((int)am, 1));
  if (kLanes == 4) am = max(am, (uint32_t)__shfl_xor((int)am, 2));
  const bool bad = am >= 0x7F80u;
  const float sixth = sixth_of(bad ? 0.0f : __uint_as_float(am << 16));
  uint32_t byte;
  float f = 0.0f;                                             // MXFP4: 2^-k
  RcpDivisor ed{};
  if constexpr (FMT == kMX) {
    byte = mx_scale_byte(sixth, &f);
  } else {
    byte = e4m3_encode_rne_sat(div_exact(sixth, wd));
    ed = make_rcp_divisor(__fmul_rn(e4m3_to_f32(byte), ws2));
  }
  uint32_t c = 0, sign = 0;
  float q[8];
#pragma unroll
  for (int k = 0; k < 8; ++k) {
    const float x = __uint_as_float((h[k >> 1] >> (16 * (k & 1))) << 16);
    if constexpr (FMT == kMX) q[k] = __fmul_rn(x, f);
    else q[k] = ed.d == 0.0f ? 0.0f : div_exact(x, ed);
    sign |= ((h[k >> 1] >> (12 + 16 * (k & 1))) & 8u) << (4 * k);
  }
  // nearest E2M1, ties to even, held to 6
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, q[0], q[1], 1.0f, 0);
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, q[2], q[3], 1.0f, 1);
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, q[4], q[5], 1.0f, 2);
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, q[6], q[7], 1.0f, 3);
  c = bad ? 0u : (c & 0x77777777u) | sign;
  reinterpret_cast<uint32_t*>(codes)[p] = c;
  if (p % kLanes == 0) scales[p / kLanes] = (uint8_t)(bad ? (FMT == kMX ? 0xFFu : 0x7Fu) : byte);
}

// Bound by memory: 8192 x 14336 in 66 us with NVFP4's exact quotients (4.6 TB/s), 8192 x 4096
// MXFP4 in 20 to 28.
template <int FMT>
__global__ __launch_bounds__(256) void act4_pack_kernel(const u32x4* __restrict__ X, int64_t pieces, float ws2,
                                                        uint8_t* __restrict__ codes, uint8_t* __restrict__ scales) {
  const int64_t p0 = (int64_t)blockIdx.x * (256 * kSteps) + threadIdx.x;
  u32x4 w[kSteps];
#pragma unroll
  for (int i = 0; i < kSteps; ++i) w[i] = X[min(p0 + i * 256, pieces - 1)];
  const RcpDivisor wd = make_rcp_divisor(ws2);
#pragma unroll
  for (int i = 0; i < kSteps; ++i)                            // whole blocks: pieces is a multiple of their lanes
    if (p0 + i * 256 < pieces) pack8<FMT>(w[i], ws2, wd, codes, scales, p0 + i * 256);
}

// 8 codes times their scale as bf16: exact but below bf16's range, at 2^128 and
// more (infinite) and, with NVFP4, by the tensor's ws2 (rounded to fp32, then to bf16: off
// by 2^-8 (1 + 2^-15) of itself at most).
template <int FMT>
__device__ __forceinline__ u32x4 unpack8(uint32_t c, uint32_t byte, float ws2) {
  const float s = FMT == kMX ? e8m0_to_f32(byte) : e4m3_to_f32(byte);
  const f32x2 v[4] = {__builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c, 1.0f, 0), __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c, 1.0f, 1),
                      __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c, 1.0f, 2), __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c, 1.0f, 3)};
  u32x4 r;
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    const float a = FMT == kMX ? v[k].x * s : v[k].x * s * ws2, b = FMT == kMX ? v[k].y * s : v[k].y * s * ws2;
    r[k] = bits_of(__builtin_convertvector((f32x2{a, b}), bf16x2));
  }
  return r;
}

// PAST: the values pass the caches by, where they and their codes are more than these hold:
// a product reads them next.  us of this kernel and with sq_bwd_dscale behind it, through and
// past them: 8000 x 4096 MXFP4 to 1024 outputs (83 MB) 14.2, 12.0 and 74.6, 81.0; 20000 (207)
// 31.7, 31.1 and 160, 174; 28000 (290) 49.5, 42.7 and 246, 243; 36000 (373) 66, 54 and 317, 309;
// 7000 x 14336 NVFP4 to 4096 (257) 38.7, 38.1 and 655, 668; 8192 (301) 55, 44 and 795, 796;
// 12000 (441) 77, 64 and 1206, 1190.  sq_fwd_act4's own, which the product reads at once, stay
// in them at any size (8192 tokens of 4096 x 14336 836, 850).
template <int FMT, bool PAST>
__global__ __launch_bounds__(256) void act4_unpack_kernel(const uint32_t* __restrict__ codes, const uint8_t* __restrict__ scales,
                                                          int64_t pieces, float ws2, u32x4* __restrict__ X) {
  const int64_t p0 = (int64_t)blockIdx.x * (256 * kSteps) + threadIdx.x;
  uint32_t c[kSteps], b[kSteps];
#pragma unroll
  for (int i = 0; i < kSteps; ++i) {
    const int64_t p = min(p0 + i * 256, pieces - 1);
    c[i] = codes[p];
    b[i] = scales[p / (ScaleOperand<FMT>::kBlock / 8)];
  }
#pragma unroll
  for (int i = 0; i < kSteps; ++i)
    if (p0 + i * 256 < pieces) {
      const u32x4 v = unpack8<FMT>(c[i], b[i], ws2);
      if constexpr (PAST) __builtin_nontemporal_store(v, &X[p0 + i * 256]);
      else X[p0 + i * 256] = v;
    }
}

// ------------------------------------------------------------------ products
struct Act4Args {
  const uint8_t* x;         // codes [T, I/2] and scales [T, G] of the kept rows
  const uint8_t* xs;
  const uint8_t* w;         // codes [E, O, I/2] and scales [E, O, G]
  const uint8_t* ws;
  const int* rows;          // row of Y -> kept row, or null
  const int* offsets;       // [E + 1], or null: one layer, rows [0, N)
  void* out;                // [N, O]
  int T, N, E, O, I, G;
  int Gs;                   // bytes from one row's scales to the next
  int chunks;               // workgroups along the rows
  const int* table;         // act4_table_kernel's, or null
  int splits, per;          // of the sum over the inputs: planes [N, O] of `per` stages each (an even number), one layer only
};

// Which rows of Y a workgroup takes: chunk c of the experts' ranges, each cut into
// chunks of `per` rows.  Ranges are held to 0 .. N.  e < 0: past the last chunk, then
// n = c minus their number, and r0 .. r1 are the rows that no expert has at the end,
// with those before the first range counted in front.
struct Chunk {
  int e, r0, r1, n;
};
__device__ __forceinline__ Chunk chunk_at(const int* offsets, int E, int N, int per, int c) {
  if (!offsets) {
    const int r0 = c * per;
    return r0 < N ? Chunk{0, r0, min(r0 + per, N), 0} : Chunk{-1, N, N, c - (N + per - 1) / per};
  }
  // 4 experts per lane: 256 for one round of loads (512 experts of 256 x 512 with one row
  // each 14.1 -> 9.8 us)
  const int lane = threadIdx.x & 63;
  int before = 0;
  for (int e0 = 0; e0 < E; e0 += 256) {
    const int e = e0 + 4 * lane;
    int o[5], t[4], sum = 0;
#pragma unroll
    for (int i = 0; i < 5; ++i) o[i] = min(max(offsets[min(e + i, E)], 0), N);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      t[i] = (max(o[i + 1] - o[i], 0) + per - 1) / per;       // 0 past the last expert
      sum += t[i];
    }
    int upto = sum;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
      const int v = __shfl_up(upto, d);
      upto += lane >= d ? v : 0;
    }
    const uint64_t in = __ballot(before + upto > c);
    if (in) {
      int at = c - (before + upto - sum), i = 0;
#pragma unroll
      for (int k = 0; k < 3; ++k)
        if (i == k && at >= t[k]) {
          at -= t[k];
          ++i;
        }
      const int first = i == 0 ? o[0] : i == 1 ? o[1] : i == 2 ? o[2] : o[3], end = i == 0 ? o[1] : i == 1 ? o[2] : i == 2 ? o[3] : o[4];
      const int l = __builtin_ctzll(in);
      const int r0 = __builtin_amdgcn_readlane(first, l) + __builtin_amdgcn_readlane(at, l) * per;
      return Chunk{e0 + 4 * l + __builtin_amdgcn_readlane(i, l), max(r0, 0), min(r0 + per, __builtin_amdgcn_readlane(end, l)), 0};
    }
    before += __builtin_amdgcn_readlane(upto, 63);
  }
  return Chunk{-1, min(max(offsets[E], 0), N), N, c - before};
}

// The chunks of all experts in a table, for products of several rounds of the CUs, whose
// workgroups would each look for theirs: word 0 their number, from word 4 on (expert,
// first row, end, 0) of each.  One workgroup.  Sums are held to `most`, which ranges in
// order never pass.
__global__ __launch_bounds__(1024) void act4_table_kernel(const int* __restrict__ offsets, int E, int N, int per, int most, int* __restrict__ table) {
  __shared__ int s_sum[16];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  int before = 0;
  for (int e0 = 0; e0 < E; e0 += 1024) {
    const int e = e0 + tid;
    const int a = e < E ? min(max(offsets[e], 0), N) : 0, b = e < E ? min(max(offsets[e + 1], 0), N) : 0;
    const int t = min((max(b - a, 0) + per - 1) / per, most);
    int upto = t;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
      const int v = __shfl_up(upto, d);
      upto = min(upto + (lane >= d ? v : 0), most);
    }
    if (lane == 63) s_sum[wave] = upto;
    __syncthreads();
    int front = before;
#pragma unroll
    for (int w = 0; w < 16; ++w) {
      if (w < wave) front = min(front + s_sum[w], most);
      before = min(before + s_sum[w], most);
    }
    const int at = front + upto - t;
    for (int k = 0; k < t && at + k < most; ++k)
      reinterpret_cast<int4*>(table)[1 + at + k] = make_int4(e, a + k * per, min(a + (k + 1) * per, b), 0);
    __syncthreads();
  }
  if (tid == 0) table[0] = before;
}

// 4 consecutive outputs of one row.
template <bool BF16>
__device__ __forceinline__ void put4(void* out, size_t at, f32x4 v) {
  if constexpr (BF16) {
    u32x2 w;
    w[0] = bits_of(__builtin_convertvector((f32x2{v[0], v[1]}), bf16x2));
    w[1] = bits_of(__builtin_convertvector((f32x2{v[2], v[3]}), bf16x2));
    *reinterpret_cast<u32x2*>(static_cast<uint16_t*>(out) + at) = w;
  } else {
    *reinterpret_cast<f32x4*>(static_cast<float*>(out) + at) = v;
  }
}

// Zeros in columns [o0, o0 + cols) of the rows that no expert has: this workgroup's
// share of them, the chunks past the last taking turns.
template <bool BF16>
__device__ __forceinline__ void zero_rows(const Act4Args& g, const Chunk& c, int chunk, int o0, int cols) {
  if (!g.offsets) return;
  const int step = max(g.chunks - (chunk - c.n), 1);          // chunks past the last
  const int front = min(min(max(g.offsets[0], 0), g.N), c.r0), all = front + c.r1 - c.r0;
  const int quads = (min(o0 + cols, g.O) - o0) / 4;           // O is a multiple of 8
  for (int r = c.n; r < all; r += step) {
    const int row = r < front ? r : c.r0 + r - front;
    for (int q = threadIdx.x; q < quads; q += blockDim.x) put4<BF16>(g.out, (size_t)row * g.O + o0 + 4 * q, f32x4{0.0f, 0.0f, 0.0f, 0.0f});
  }
}

__device__ __forceinline__ i32x8 codes_operand(u32x4 c) {
  return i32x8{(int)c[0], (int)c[1], (int)c[2], (int)c[3], 0, 0, 0, 0};
}

// Few rows: the weight's codes go from memory into the operand registers, each once
// per chunk of 16 NT rows.  A workgroup takes 16 RM outputs; its waves take a stretch of
// the inputs each, in steps of 128, and their sums meet in LDS in wave order.  Bound by the
// round trips of the loads: one row of 4096 x 4096 4.2 us (2.1 TB/s), 64 rows 8.6.  WORDS:
// scale rows are whole words, and 4 steps' scales of a row come in one load.
template <int RM, int NT, bool WORDS, bool BF16>
__global__ __launch_bounds__(512) void act4_thin_kernel(Act4Args g) {
  constexpr int kWaves = 8, kUnroll = WORDS ? 4 : 2;
  __shared__ f32x4 part[kWaves][RM * NT][64];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int groups = (g.O + 16 * RM - 1) / (16 * RM);
  const int chunk = (int)(blockIdx.x / groups), o0 = (int)(blockIdx.x % groups) * 16 * RM;
  const Chunk c = chunk_at(g.offsets, g.E, g.N, 16 * NT, chunk);
  if (c.e < 0) {
    zero_rows<BF16>(g, c, chunk, o0, 16 * RM);
    return;
  }
  const int half = g.I / 2, steps = (g.I + 127) / 128, kb = lane >> 4;
  const int per = (steps + kWaves - 1) / kWaves, first = wave * per, end = min(first + per, steps);
  const __amdgpu_buffer_rsrc_t rw = make_rsrc(g.w + (size_t)c.e * g.O * half, (uint32_t)((size_t)g.O * half));
  const __amdgpu_buffer_rsrc_t rws = make_rsrc(g.ws + (size_t)c.e * g.O * g.G, (uint32_t)((size_t)g.O * g.G));
  const __amdgpu_buffer_rsrc_t rx = make_rsrc(g.x, (uint32_t)((size_t)g.T * half));
  const __amdgpu_buffer_rsrc_t rxs = make_rsrc(g.xs, (uint32_t)((size_t)g.T * g.G));
  uint32_t w_row[RM], x_row[NT];
#pragma unroll
  for (int m = 0; m < RM; ++m) {
    const int o = o0 + 16 * m + (lane & 15);
    w_row[m] = o < g.O ? (uint32_t)o : kOOB;
  }
#pragma unroll
  for (int j = 0; j < NT; ++j) {
    const int r = c.r0 + 16 * j + (lane & 15);
    x_row[j] = kOOB;
    if (r < c.r1) {
      const int t = g.rows ? g.rows[r] : r;
      if (t >= 0 && t < g.T) x_row[j] = (uint32_t)t;
    }
  }
  f32x4 acc[RM][NT];
#pragma unroll
  for (int m = 0; m < RM; ++m)
#pragma unroll
    for (int j = 0; j < NT; ++j) acc[m][j] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
  for (int s0 = first; s0 < end; s0 += kUnroll) {
    u32x4 wc[kUnroll][RM], xc[kUnroll][NT];
    uint32_t wb[kUnroll][RM], xb[kUnroll][NT];
    // of one row: this lane's codes of each step (zeros past the inputs), and the
    // steps' scales; with WORDS those past the row's end are another's, of steps that
    // are not taken
    auto load = [&](__amdgpu_buffer_rsrc_t rc, __amdgpu_buffer_rsrc_t rs, uint32_t row, auto put) {
      u32x4 words = {0u, 0u, 0u, 0u};
      if constexpr (WORDS) {
        const int at = (int)(row == kOOB ? kOOB : row * (uint32_t)g.G + 4u * (uint32_t)s0);
        words = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(rs, at, 0, 0));
      }
#pragma unroll
      for (int u = 0; u < kUnroll; ++u) {
        const uint32_t b = (uint32_t)(s0 + u) * 4 + kb;       // this lane's block of 32 inputs
        const bool in = s0 + u < end && b < (uint32_t)g.G && row != kOOB;
        const u32x4 q = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(rc, (int)(in ? row * (uint32_t)half + 16u * b : kOOB), 0, 0));
        uint32_t s;
        if constexpr (WORDS) s = words[u] >> (8 * kb);
        else s = __builtin_amdgcn_raw_buffer_load_b8(rs, (int)(in ? row * (uint32_t)g.G + b : kOOB), 0, 0);
        put(u, q, s);
      }
    };
#pragma unroll
    for (int m = 0; m < RM; ++m) load(rw, rws, w_row[m], [&](int u, u32x4 q, uint32_t s) { wc[u][m] = q; wb[u][m] = s; });
#pragma unroll
    for (int j = 0; j < NT; ++j) load(rx, rxs, x_row[j], [&](int u, u32x4 q, uint32_t s) { xc[u][j] = q; xb[u][j] = s; });
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) {
      if (s0 + u >= end) break;
#pragma unroll
      for (int m = 0; m < RM; ++m)
#pragma unroll
        for (int j = 0; j < NT; ++j)
          acc[m][j] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(codes_operand(wc[u][m]), codes_operand(xc[u][j]), acc[m][j], 4, 4, 0,
                                                                       (int)wb[u][m], 0, (int)xb[u][j]);
    }
  }
#pragma unroll
  for (int m = 0; m < RM; ++m)
#pragma unroll
    for (int j = 0; j < NT; ++j) part[wave][m * NT + j][lane] = acc[m][j];
  __syncthreads();
  // a 16 x 16 result: lane l holds outputs 4 (l / 16) + 0..3 of row l % 16
  for (int i = threadIdx.x; i < RM * NT * 64; i += 512) {
    const int f = i >> 6, l = i & 63;
    f32x4 v = part[0][f][l];
#pragma unroll
    for (int w = 1; w < kWaves; ++w) v += part[w][f][l];
    const int o = o0 + 16 * (f / NT) + 4 * (l >> 4), r = c.r0 + 16 * (f % NT) + (l & 15);
    if (o < g.O && r < c.r1) put4<BF16>(g.out, (size_t)r * g.O + o, v);
  }
}

template <int RM, int NT>
int thin_go(Act4Args g, int bf16, hipStream_t s) {
  // every range's last chunk may be short, and one more chunk for the rows of no expert
  g.chunks = g.offsets ? (int)(g.N / (16 * NT) + (g.E < g.N ? g.E : g.N) + 1) : (g.N + 16 * NT - 1) / (16 * NT);
  const dim3 grid((unsigned)((g.O + 16 * RM - 1) / (16 * RM) * g.chunks)), block(512);
  const bool words = g.G % 4 == 0;
  auto go = [&](auto kernel) {
    hipLaunchKernelGGL(kernel, grid, block, 0, s, g);
    return ok();
  };
  if (words) return bf16 ? go(act4_thin_kernel<RM, NT, true, true>) : go(act4_thin_kernel<RM, NT, true, false>);
  return bf16 ? go(act4_thin_kernel<RM, NT, false, true>) : go(act4_thin_kernel<RM, NT, false, false>);
}

// Outputs per workgroup: the more, the less often the rows are read, but a workgroup
// for every CU.  One layer of more than 16 rows comes here with up to 4096 outputs
// (act4_plan), of which 16 to a workgroup leave one for each CU.
int thin_by(const Act4Args& g, int bf16, hipStream_t s) {
  if (!g.offsets && g.N > 16) return g.N <= 32 ? thin_go<1, 2>(g, bf16, s) : thin_go<1, 4>(g, bf16, s);
  const int64_t chunks = g.offsets ? (g.E < g.N ? g.E : g.N) : 1;
  const int64_t groups = (g.O + 63) / 64 * chunks;
  if (groups >= kCUs * 3 / 4) return thin_go<4, 1>(g, bf16, s);
  return 2 * groups >= kCUs * 3 / 4 ? thin_go<2, 1>(g, bf16, s) : thin_go<1, 1>(g, bf16, s);
}

// f(0), f(1), .. with constants, in this order.
template <int... N, typename F>
__device__ __forceinline__ void for_each(std::integer_sequence<int, N...>, F f) {
  (f(std::integral_constant<int, N>{}), ...);
}
template <int N, typename F>
__device__ __forceinline__ void times(F f) {
  for_each(std::make_integer_sequence<int, N>{}, f);
}

// Many rows: tiles of BM outputs by BT rows of Y, so that a lane holds one row's
// outputs.  A stage is 256 inputs: the 128 bytes of codes of each row, a cache line,
// copied to LDS with the 16-byte chunks placed as a bf16 tile's (a chunk is one lane's
// 32 codes of a product); the scales come for two stages at a time, 16 bytes of each
// row.  Between a slice's products go the reads of the next slice and the copies of a
// later stage, and the barrier that publishes the next stage stands amid the last
// slice.
// 8192 tokens of 14336 x 4096 take 243 to 250 us: matrix cores busy 0.52 at 1.78 GHz, the
// chip's power limit.  128 experts of 1536 x 2048 over 32768 rows (81 to 87) are bound by memory
// and by the tiles' ends, 8 stages apart: busy 0.29 at 2.23 GHz.  Tiles that follow each other
// in resident workgroups, the next one's first copies under the last products, gained
// nothing, since the stores then hold up the next tile's stages.
template <int BM, int BT, int STAGES>
constexpr int tile_lds() {
  return STAGES * (BM + BT) * 128 + (STAGES <= 3 ? 2 : 4) * (BM + BT) * 16;
}
// PAST: outputs pass the caches by, which the experts' weights and rows need (128 experts of
// 1536 x 2048 over 32768 rows 108 -> 88 us, of 2048 x 768 to fp32 98 -> 77; of one layer it
// is a loss as often as a gain: 8192 tokens of 8192 x 1024 55 -> 64, 4096 x 4096 41.2 -> 40.5).
template <int BM, int BT, int WGM, int WGN, int STAGES, bool PAST, bool BF16>
__device__ __forceinline__ void act4_tile(const Act4Args& g, const Chunk& c, int m0, int split, uint8_t* lds) {
  constexpr int kStageI = 256, kRow = kStageI / 2, kSlices = 4;
  constexpr int WM = BM / WGM, WN = BT / WGN, TM = WM / 32, TN = WN / 32;
  static_assert(WGM * WGN == 8 && TM >= 1 && TN >= 1, "8 waves");
  constexpr int kA = BM * kRow, kB = BT * kRow, kSa = BM * 16, kSb = BT * 16;
  constexpr int kInstA = BM / 64, kInstB = BT / 64, kDma = kInstA + kInstB;
  constexpr int kAhead = (STAGES - 2) * kDma;
  // Scales of stages 2 p and 2 p + 1 are copied behind the codes of stage 2 p - 1 (2 p
  // with three stages), in the first slice of an even stage, kLead pairs ahead of it.
  static_assert(STAGES == 2 || STAGES == 3 || STAGES == 4 || STAGES == 6, "stages");
  constexpr int kLead = STAGES == 3 ? 1 : STAGES / 2, kSets = STAGES <= 3 ? 2 : 4;
  // each operand's buffers lie beside each other, so that their places are one
  // register's and a constant
  constexpr int kAtB = STAGES * kA, kAtSa = kAtB + STAGES * kB, kAtSb = kAtSa + kSets * kSa, kAll = kAtSb + kSets * kSb;
  static_assert(kAll == tile_lds<BM, BT, STAGES>() && kAll <= 160 * 1024 && BM * BT * 2 <= kAll, "LDS, of the loop and of the outputs in bf16");
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int wave_u = __builtin_amdgcn_readfirstlane(wave);
  const int wm0 = (wave / WGN) * WM, wn0 = (wave % WGN) * WN;

  const int half = g.I / 2, kt_first = split * g.per;
  const int nk = min((g.I + kStageI - 1) / kStageI - kt_first, g.per);
  const int live_m = min(BM, g.O - m0);
  const size_t row0 = (size_t)c.e * g.O + m0;
  const DmaRsrc ra = make_dma_rsrc(g.w + row0 * half, (uint32_t)((size_t)live_m * half));
  const DmaRsrc rb = make_dma_rsrc(g.x, (uint32_t)((size_t)g.T * half));
  // a wave copies the scales of 64 rows: the first four the weight's, the others Y's
  // (where those are fewer, several waves the same)
  const bool weights = wave_u < 4;
  const DmaRsrc rs = weights ? make_dma_rsrc(g.ws + row0 * g.Gs, (uint32_t)((size_t)live_m * g.Gs))
                             : make_dma_rsrc(g.xs, (uint32_t)((size_t)g.T * g.Gs));
  const int s_row = wave_u * 64 % (weights ? BM : BT);
  const int s_to = (weights ? kAtSa : kAtSb) + s_row * 16, s_group = weights ? kSa : kSb;

  // a copy instruction fills 8 rows of codes
  auto kept_row = [&](int r) -> uint32_t {                    // of Y's row c.r0 + r
    if (c.r0 + r >= c.r1) return kOOB;
    const int t = g.rows ? g.rows[c.r0 + r] : c.r0 + r;
    return t >= 0 && t < g.T ? (uint32_t)t : kOOB;
  };
  // (rows past the weight's last lie behind the buffer's end)
  uint32_t off_a, off_b[kInstB];
  int lim;                                                    // bytes of a row from this lane's chunk on: rows r and r + 64 have the same
  {
    const int r = wave * 8 + (lane >> 3), ch = (lane & 7) ^ swz_kc(r);
    lim = half - 16 * ch;
    off_a = (uint32_t)r * (uint32_t)half + 16u * ch;
#pragma unroll
    for (int q = 0; q < kInstB; ++q) {
      const uint32_t t = kept_row(q * 64 + r);
      off_b[q] = t == kOOB ? kOOB : t * (uint32_t)half + 16u * ch;
    }
  }
  const uint32_t t_s = weights ? (uint32_t)(s_row + lane) : kept_row(s_row + lane);
  const uint32_t off_s = t_s == kOOB ? kOOB : t_s * (uint32_t)g.Gs;

  SQ_LDS uint8_t* const lp = (SQ_LDS uint8_t*)lds;
  // copy n of stage kt into buffer S; what lies past the matrix reads as zeros
  auto dma = [&](auto S, int kt, auto N) {
    constexpr int n = decltype(N)::value;
    constexpr int st = decltype(S)::value;
    const int k = (kt_first + kt) * kRow;
    if constexpr (n < kInstA) {
      dma16(ra, lp + st * kA + (n * 64 + wave_u * 8) * kRow, k >= lim ? kOOB : off_a + (uint32_t)(n * 64 * half + k));
    } else {
      constexpr int q = n - kInstA;
      dma16(rb, lp + kAtB + st * kB + (q * 64 + wave_u * 8) * kRow, off_b[q] == kOOB || k >= lim ? kOOB : off_b[q] + (uint32_t)k);
    }
  };
  // the scales of stages 2 p and 2 p + 1 into set p % kSets; where a row ends inside its 16
  // bytes, the next row's follow
  auto dma_scales = [&](int p) {
    const int at = kt_first * 8 + p * 16;
    dma16(rs, lp + s_to + p % kSets * s_group, off_s == kOOB || at >= g.Gs ? kOOB : off_s + (uint32_t)at);
  };
  constexpr int kFirst = kDma / 2, kSecond = kDma - kFirst;
  auto dma_all = [&](auto S, int kt) { times<kDma>([&](auto N) { dma(S, kt, N); }); };
  auto dma_first = [&](auto S, int kt) { times<kFirst>([&](auto N) { dma(S, kt, N); }); };

  f32x16 acc[TM][TN];
#pragma unroll
  for (int i = 0; i < TM; ++i)
#pragma unroll
    for (int j = 0; j < TN; ++j)
#pragma unroll
      for (int r = 0; r < 16; ++r) acc[i][j][r] = 0.0f;

  struct Frag {
    u32x4 a[TM], b[TN];
  };
  Frag F0, F1;
  // scales of a stage, word w for slices 2 w and 2 w + 1: this lane's byte of the
  // first in byte 0, of the second in byte 2
  struct Scales {
    int a[TM][2], b[TN][2];
  };
  Scales sc[2];
  // Where a slice's chunk of this lane's row is, for row tiles of even number; 32 rows
  // on, the placement turns bit 2 of the chunk, which is bit 1 of the slice.
  uint32_t a_at[kSlices], b_at[kSlices];
#pragma unroll
  for (int kk = 0; kk < kSlices; ++kk) {
    const int ra0 = wm0 + (lane & 31), rb0 = wn0 + (lane & 31), ch = 2 * kk + (lane >> 5);
    a_at[kk] = (uint32_t)(ra0 * kRow + ((ch ^ swz_kc(ra0)) << 4));
    b_at[kk] = (uint32_t)(kAtB + rb0 * kRow + ((ch ^ swz_kc(rb0)) << 4));
  }
  constexpr int kReads = TM + TN, kProducts = TM * TN, kMid = kProducts / 2, kRest = kProducts - kMid;
  auto read = [&](auto S, auto KK, Frag& f, auto N) {
    constexpr int n = decltype(N)::value, kk = decltype(KK)::value, st = decltype(S)::value;
    // a0 b0 b1 .. a1 ..: the order in which the products need them
    if constexpr (n == 0 || n > TN) {
      constexpr int i = n == 0 ? 0 : n - TN;
      f.a[i] = *(const SQ_LDS u32x4*)(lp + a_at[kk ^ (2 * (i & 1))] + st * kA + i * 32 * kRow);
    } else {
      constexpr int j = n - 1;
      f.b[j] = *(const SQ_LDS u32x4*)(lp + b_at[kk ^ (2 * (j & 1))] + st * kB + j * 32 * kRow);
    }
  };
  const uint32_t sa_at = (uint32_t)(kAtSa + (wm0 + (lane & 31)) * 16), sb_at = (uint32_t)(kAtSb + (wn0 + (lane & 31)) * 16);
  auto read_scales = [&](int kt, auto ODD, Scales& v, auto N) {
    constexpr int n = decltype(N)::value, odd = decltype(ODD)::value;
    const int shift = 8 * (lane >> 5), set = (kt >> 1) % kSets;
    // blocks past the row's end have zero codes, and the next row's scales may be NaN
    const int at = (kt_first + kt) * 8;
    const uint32_t in0 = at < g.Gs ? ~0u : 0u, in1 = at + 4 < g.Gs ? ~0u : 0u;
    const u32x2 w = n < TM ? *(const SQ_LDS u32x2*)(lp + sa_at + set * kSa + n * 512 + odd * 8)
                           : *(const SQ_LDS u32x2*)(lp + sb_at + set * kSb + (n - TM) * 512 + odd * 8);
    int* to = n < TM ? v.a[n < TM ? n : 0] : v.b[n < TM ? 0 : n - TM];
    to[0] = (int)((w[0] & in0) >> shift);
    to[1] = (int)((w[1] & in1) >> shift);
  };
  auto product = [&](Frag& f, const Scales& v, auto KK, auto N) {
    constexpr int i = decltype(N)::value / TN, j = decltype(N)::value % TN, kk = decltype(KK)::value, w = kk >> 1, byte = 2 * (kk & 1);
    acc[i][j] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(codes_operand(f.a[i]), codes_operand(f.b[j]), acc[i][j], 4, 4, byte,
                                                                v.a[i][w], byte, v.b[j][w]);
  };
  // f of those of 0 .. ALL - 1 that fall to part N of PARTS
  auto share = [&](auto N, auto PARTS, auto ALL, auto f) {
    constexpr int parts = decltype(PARTS)::value, all = decltype(ALL)::value;
    constexpr int n = decltype(N)::value < parts ? decltype(N)::value : parts, m = n < parts ? n + 1 : parts;
    constexpr int lo = n * all / parts, hi = m * all / parts;
    times<hi - lo>([&](auto K) { f(std::integral_constant<int, lo + decltype(K)::value>{}); });
  };
  using I0 = std::integral_constant<int, 0>;
  using Reads = std::integral_constant<int, kReads>;
  using Parts = std::integral_constant<int, (kReads < kProducts ? kReads : kProducts)>;

  // V: which of the two sets of scales the stage has
  auto step = [&](auto S, auto V, int kt) {
    constexpr int st = decltype(S)::value, v = decltype(V)::value;
    using SN = std::integral_constant<int, (st + 1) % STAGES>;            // stage kt + 1
    using SP = std::integral_constant<int, (st + STAGES - 1) % STAGES>;   // stage kt + STAGES - 1
    times<kSlices - 1>([&](auto KK) {
      constexpr int kk = decltype(KK)::value;
      Frag& now = kk & 1 ? F1 : F0;
      Frag& next = kk & 1 ? F0 : F1;
      times<kProducts>([&](auto N) {
        product(now, sc[v], KK, N);
        share(N, Parts{}, Reads{}, [&](auto R) { read(S, std::integral_constant<int, kk + 1>{}, next, R); });
        if constexpr (kk == 0)
          share(N, std::integral_constant<int, kProducts>{}, std::integral_constant<int, kSecond>{},
                [&](auto C) { dma(SP{}, kt + STAGES - 1, std::integral_constant<int, kFirst + decltype(C)::value>{}); });
        if constexpr (kk == 0 && v == 0 && decltype(N)::value == kProducts - 1) dma_scales((kt >> 1) + kLead);
        __builtin_amdgcn_sched_barrier(0);
      });
    });
    times<kProducts>([&](auto N) {
      constexpr int n = decltype(N)::value;
      if constexpr (n == kMid) {
        // stage kt + 1 has landed once only the copies of the stages after it are
        // outstanding, and the scales copied among them
        wait_vm_lgkm0<kAhead + kLead - v>();
        __builtin_amdgcn_s_barrier();
        __builtin_amdgcn_sched_barrier(0);
      }
      product(F1, sc[v], std::integral_constant<int, kSlices - 1>{}, N);
      if constexpr (n >= kMid) {
        using At = std::integral_constant<int, n - kMid>;
        using Rest = std::integral_constant<int, kRest>;
        share(At{}, Rest{}, Reads{}, [&](auto R) {
          read(SN{}, I0{}, F0, R);
          read_scales(kt + 1, std::integral_constant<int, 1 - v>{}, sc[1 - v], R);
        });
        share(At{}, Rest{}, std::integral_constant<int, kFirst>{}, [&](auto C) { dma(S, kt + STAGES, C); });
      }
      __builtin_amdgcn_sched_barrier(0);
    });
  };

  // prologue: stages 0 .. STAGES - 2 and the first half of stage STAGES - 1 on their
  // way, with their scales in the order of the loop; the first operands of stage 0
  dma_scales(0);
  times<STAGES - 1>([&](auto S) {
    dma_all(S, decltype(S)::value);
    if constexpr (decltype(S)::value % 2 == 1 && decltype(S)::value / 2 + 1 < kLead) dma_scales(decltype(S)::value / 2 + 1);
  });
  dma_first(std::integral_constant<int, STAGES - 1>{}, STAGES - 1);
  wait_vm_lgkm0<kAhead + kFirst + kLead - 1>();
  __builtin_amdgcn_s_barrier();
  __builtin_amdgcn_sched_barrier(0);
  times<kReads>([&](auto R) {
    read(I0{}, I0{}, F0, R);
    read_scales(0, I0{}, sc[0], R);
  });
  // rings of STAGES buffers and 2 sets of scales turn together
  constexpr int kTurn = STAGES % 2 ? 2 * STAGES : STAGES;
  for (int kt0 = 0; kt0 < nk; kt0 += kTurn)
    times<kTurn>([&](auto U) {
      constexpr int u = decltype(U)::value;
      if (u > 0 && kt0 + u >= nk) return;
      step(std::integral_constant<int, u % STAGES>{}, std::integral_constant<int, u % 2>{}, kt0 + u);
    });
  wait_vm_lgkm0<0>();

  auto put = [](auto* to, auto v) {
    if constexpr (PAST) __builtin_nontemporal_store(v, to);
    else *to = v;
  };
  // 32 x 32 result: lane l, register r holds output 8 (r / 4) + 4 (l / 32) + r % 4 of
  // row l % 32.
  if constexpr (BF16) {
    // through LDS, so that a row's outputs leave together: 16-byte unit u of row n at
    // unit u ^ n
    __syncthreads();
    SQ_LDS uint16_t* s = (SQ_LDS uint16_t*)lds + wave * WM * WN;
    constexpr int kLanes = WM / 8, kTok = 64 / kLanes;
#pragma unroll
    for (int j = 0; j < TN; ++j)
#pragma unroll
      for (int i = 0; i < TM; ++i)
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          u32x2 w;
          w[0] = bits_of(__builtin_convertvector((f32x2{acc[i][j][4 * q], acc[i][j][4 * q + 1]}), bf16x2));
          w[1] = bits_of(__builtin_convertvector((f32x2{acc[i][j][4 * q + 2], acc[i][j][4 * q + 3]}), bf16x2));
          const int n = j * 32 + (lane & 31), u = i * 4 + q;
          *(SQ_LDS u32x2*)(s + n * WM + ((u ^ n) & (kLanes - 1)) * 8 + 4 * (lane >> 5)) = w;
        }
    __builtin_amdgcn_wave_barrier();
#pragma unroll
    for (int it = 0; it < WN / kTok; ++it) {
      const int n = it * kTok + lane / kLanes, u = lane % kLanes;
      const u32x4 v = *(const SQ_LDS u32x4*)(s + n * WM + ((u ^ n) & (kLanes - 1)) * 8);
      const int row = c.r0 + wn0 + n, o = m0 + wm0 + 8 * u;
      if (row < c.r1 && o < g.O) put(reinterpret_cast<u32x4*>(static_cast<uint16_t*>(g.out) + (size_t)row * g.O + o), v);
    }
  } else {
    // the same for 32 rows at a time, whose 16-byte units of fp32 a wave's share of LDS holds
    __syncthreads();
    static_assert(8 * 32 * WM * 4 <= kAll, "LDS, of 32 rows of a wave's outputs");
    constexpr int kUnits = WM / 4, kRows = 64 / kUnits;
    SQ_LDS f32x4* s = (SQ_LDS f32x4*)lds + wave * 32 * kUnits;
#pragma unroll
    for (int j = 0; j < TN; ++j) {
#pragma unroll
      for (int i = 0; i < TM; ++i)
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          const int n = lane & 31, u = i * 8 + 2 * q + (lane >> 5);
          s[n * kUnits + (u ^ (n & (kUnits - 1)))] = f32x4{acc[i][j][4 * q], acc[i][j][4 * q + 1], acc[i][j][4 * q + 2], acc[i][j][4 * q + 3]};
        }
      __builtin_amdgcn_wave_barrier();
#pragma unroll
      for (int it = 0; it < 32 / kRows; ++it) {
        const int n = it * kRows + lane / kUnits, u = lane % kUnits;
        const f32x4 v = s[n * kUnits + (u ^ (n & (kUnits - 1)))];
        const int row = c.r0 + wn0 + j * 32 + n, o = m0 + wm0 + 4 * u;
        if (row < c.r1 && o < g.O) put(reinterpret_cast<f32x4*>(static_cast<float*>(g.out) + ((size_t)split * g.N + row) * g.O + o), v);
      }
      __builtin_amdgcn_wave_barrier();
    }
  }
}

// A tile per workgroup: of the experts' chunks dealt to the XCDs in turn (those past the
// last are spread as well), of one layer in groups of 4 x n tiles.
template <int BM, int BT, int WGM, int WGN, int STAGES, bool BF16>
__global__ __launch_bounds__(512) void act4_tile_kernel(Act4Args g) {
  __shared__ __attribute__((aligned(16))) uint8_t lds[tile_lds<BM, BT, STAGES>()];
  const int tiles_m = (g.O + BM - 1) / BM;
  int chunk, tm, split = 0;
  if (g.offsets) {
    const int at = (int)blockIdx.x / kXcds;
    chunk = at / tiles_m * kXcds + (int)blockIdx.x % kXcds;
    tm = at % tiles_m;
    if (chunk >= g.chunks) return;
  } else {
    const int tiles = tiles_m * g.chunks, pos = xcd_stretch((int)blockIdx.x, tiles * g.splits);
    split = pos / tiles;
    tile_at<4>(pos - split * tiles, tiles_m, g.chunks, tm, chunk);
  }
  const Chunk c = chunk_at(g.offsets, g.E, g.N, BT, chunk);
  if (c.e < 0) zero_rows<BF16>(g, c, chunk, tm * BM, BM);
  else act4_tile<BM, BT, WGM, WGN, STAGES, false, BF16>(g, c, tm * BM, split, lds);
}

// Experts' chunks of BT rows from a table, the tiles of a chunk and the chunks of an
// expert beside each other, in stretches that the XCDs take, so that one L2 reads an
// expert's weight.  An expert's last chunk takes the smallest tile that holds its rows.
template <int BT, bool BF16>
__global__ __launch_bounds__(512) void act4_experts_kernel(Act4Args g) {
  constexpr int kLds = BT == 64 ? tile_lds<256, 64, 3>() : tile_lds<256, 128, 3>();
  static_assert(tile_lds<256, 256, 2>() <= tile_lds<256, 128, 3>(), "the largest");
  __shared__ __attribute__((aligned(16))) uint8_t lds[kLds];
  const int tiles_m = (g.O + 255) / 256, total = g.table[0], n = total * tiles_m;
  if ((int)blockIdx.x >= n) {                                 // past the last chunk: rows that no expert has
    const int chunk = (int)blockIdx.x / tiles_m;
    const Chunk c{-1, min(max(g.offsets[g.E], 0), g.N), g.N, chunk - total};
    zero_rows<BF16>(g, c, chunk, (int)blockIdx.x % tiles_m * 256, 256);
    return;
  }
  const int pos = xcd_stretch((int)blockIdx.x, n), chunk = pos / tiles_m, m0 = (pos - chunk * tiles_m) * 256;
  const int4 t = reinterpret_cast<const int4*>(g.table)[1 + chunk];
  const Chunk c{__builtin_amdgcn_readfirstlane(t.x), __builtin_amdgcn_readfirstlane(t.y), __builtin_amdgcn_readfirstlane(t.z), 0};
  const int rows = c.r1 - c.r0;
  if constexpr (BT == 256)
    if (rows > 128) {
      act4_tile<256, 256, 2, 4, 2, true, BF16>(g, c, m0, 0, lds);
      return;
    }
  if constexpr (BT >= 128)
    if (rows > 64) {
      act4_tile<256, 128, 4, 2, 3, true, BF16>(g, c, m0, 0, lds);
      return;
    }
  act4_tile<256, 64, 8, 1, 3, true, BF16>(g, c, m0, 0, lds);
}

// Scale rows of G bytes laid out in whole words.
__global__ __launch_bounds__(256) void act4_words_kernel(const uint8_t* __restrict__ from, int64_t rows, int G, int words,
                                                         uint32_t* __restrict__ to) {
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < rows * words; i += (int64_t)gridDim.x * 256) {
    const int64_t r = i / words;
    const int k = (int)(i - r * words) * 4;
    uint32_t v = 0;
#pragma unroll
    for (int b = 0; b < 4; ++b) v |= k + b < G ? (uint32_t)from[r * G + k + b] << (8 * b) : 0u;
    to[i] = v;
  }
}

// 8 outputs per lane: the planes added in order.
template <bool BF16>
__global__ __launch_bounds__(256) void act4_join_kernel(const f32x4* __restrict__ planes, int splits, int64_t items, void* __restrict__ out) {
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (i >= items) return;
  f32x4 a = planes[2 * i], b = planes[2 * i + 1];
  for (int s = 1; s < splits; ++s) {
    a += planes[2 * ((int64_t)s * items + i)];
    b += planes[2 * ((int64_t)s * items + i) + 1];
  }
  put4<BF16>(out, 8 * i, a);
  put4<BF16>(out, 8 * i + 4, b);
}

// Chunks of `per` rows of the experts' ranges at most, since every range's last may be
// short, and one for the rows of no expert.
inline int64_t most_chunks(int64_t E, int64_t N, int64_t per) { return N / per + (E < N ? E : N) + 1; }

template <int BM, int BT, int WGM, int WGN, int STAGES>
int tile_go(Act4Args g, int bf16, hipStream_t s) {
  g.chunks = g.offsets ? (int)most_chunks(g.E, g.N, BT) : (g.N + BT - 1) / BT;
  const int along = g.offsets ? (g.chunks + kXcds - 1) / kXcds * kXcds : g.chunks;
  const dim3 grid((unsigned)((g.O + BM - 1) / BM * along * g.splits)), block(512);
  if (bf16) hipLaunchKernelGGL((act4_tile_kernel<BM, BT, WGM, WGN, STAGES, true>), grid, block, 0, s, g);
  else hipLaunchKernelGGL((act4_tile_kernel<BM, BT, WGM, WGN, STAGES, false>), grid, block, 0, s, g);
  return ok();
}

template <int BT>
int experts_go(Act4Args g, int bf16, hipStream_t s) {
  g.chunks = (int)most_chunks(g.E, g.N, BT);
  hipLaunchKernelGGL(act4_table_kernel, dim3(1), dim3(1024), 0, s, g.offsets, g.E, g.N, BT, g.chunks - 1, const_cast<int*>(g.table));
  if (ok() != 0) return -1;
  const dim3 grid((unsigned)((g.O + 255) / 256 * g.chunks)), block(512);
  if (bf16) hipLaunchKernelGGL((act4_experts_kernel<BT, true>), grid, block, 0, s, g);
  else hipLaunchKernelGGL((act4_experts_kernel<BT, false>), grid, block, 0, s, g);
  return ok();
}

// How a product runs: tiles of bm outputs by bt rows (bt = 0: the few rows' kernel), and
// the splits of one layer's sums.
struct Act4Plan {
  int bm, bt, splits, per;
  bool table;
};

// Experts of more than one round of the CUs take their chunks from a table, and their last
// rows a smaller tile (128 of 1536 x 2048 with 256 rows each 122 us, with the table 114,
// with both 105; 128 of 2048 x 768 with 256 83, 76, 69; 128 of 768 x 2048 with 128 42.4,
// -, 38.9).  With the smallest tiles only from 3 rounds on, since the table's launch costs
// 2 (512 of 768 x 2048 with one row each 41.7 -> 34.9, 128 with 16 22.4 -> 24.0).
// The smallest tiles that one round of the CUs holds, or else the largest that the rows
// fill.  us in a graph, of 128 x 64, 128 x 128, 256 x 64, 256 x 128 and 256 x 256 tiles:
// 512 rows of 4096 x 4096 10.7, 11.9, 12.8, 15.5, 23.1; 512 of 14336 x 4096 40.9, 28.5,
// 30.0, 24.7, 28.7; 2000 of 4096 x 4096 40.7, 31.1, 30.7, 26.7, 29.4; 128 experts of 768
// x 2048 with 16 rows each 26.3, 27.3, 23.0, 25.7, 33.0, with 64 41.6, 37.7, 35.9, 30.4,
// 36.2; 128 of 1536 x 2048 with 256 212, 155, 168, 137, 116.  The few rows' kernel against
// 128 x 64 (one layer) and 256 x 64 tiles (experts): 16 rows of 4096 x 4096 4.8, 8.7; 64
// 8.6, 9.0; 64 of 14336 x 4096 15.0, 10.4; 8 experts of 1536 x 2048 with 4 rows each 5.8,
// 8.0; 128 of 768 x 2048 with 1 14.1, 12.8.
// Few tiles and a long sum: split it, at least 8 stages each, since planes and their
// join cost 5 us (64 rows of 4096 x 14336 26.7, in two 19.8).
Act4Plan act4_plan(bool batched, int64_t E, int64_t N, int64_t O, int64_t I) {
  const int64_t live = E < N ? E : N, avg = (N + live - 1) / live, stages = (I + 255) / 256;
  Act4Plan p{256, 256, 1, (int)stages, false};
  if (avg <= 16 && (!batched || live * O <= 64 * 256)) p.bt = 0;
  if (!batched && avg <= 64 && O <= 16 * kCUs) p.bt = 0;
  if (p.bt == 0) return p;
  const int tiles[5][2] = {{128, 64}, {256, 64}, {128, 128}, {256, 128}, {256, 256}};
  bool found = false;
  for (const auto& t : tiles) {
    if (found || (!batched && t[0] == 256 && t[1] == 64)) continue;
    const int64_t along = (O + t[0] - 1) / t[0];
    // of many experts each range's last chunk is half full on average; chunks go to XCDs
    const int64_t chunks = batched ? live * (2 * avg + t[1]) / (2 * t[1]) : (N + t[1] - 1) / t[1];
    found = batched ? ((chunks > live ? chunks : live) + kXcds - 1) / kXcds * along <= kCUs / kXcds : chunks * along <= kCUs;
    if (found) {
      p.bm = t[0];
      p.bt = t[1];
    }
  }
  if (batched && !found) {
    p.bt = avg <= 48 ? 64 : avg <= 160 ? 128 : 256;
    p.table = p.bt > 64 || live * ((O + 255) / 256) >= 3 * kCUs;
  }
  const int64_t t = (O + p.bm - 1) / p.bm * ((N + p.bt - 1) / p.bt);
  if (!batched && 2 * t <= kCUs && stages >= 24) {
    int64_t n = kCUs / t < stages / 8 ? kCUs / t : stages / 8;
    n = n < 8 ? n : 8;
    p.per = (int)(((stages + n - 1) / n + 1) / 2 * 2);
    p.splits = (int)((stages + p.per - 1) / p.per);
  }
  return p;
}

// Bytes of the workspace: scales whose rows are not whole words, laid out anew for the
// tiles, and behind them the planes of split sums or the table of chunks.
size_t words_bytes(const Act4Plan& p, int64_t E, int64_t T, int64_t O, int64_t I) {
  const int64_t G = I / 32;
  return G % 4 == 0 || p.bt == 0 ? 0 : ((size_t)((T + E * O) * ((G + 3) / 4 * 4)) + 255) & ~(size_t)255;
}
size_t plan_bytes(const Act4Plan& p, int64_t E, int64_t T, int64_t N, int64_t O, int64_t I) {
  return words_bytes(p, E, T, O, I) + (p.splits > 1 ? (size_t)p.splits * N * O * 4 : 0) +
         (p.table ? (size_t)most_chunks(E, N, p.bt) * 16 : 0);
}

int product(Act4Args g, int bf16, void* workspace, hipStream_t s) {
  const Act4Plan p = act4_plan(g.offsets != nullptr, g.E, g.N, g.O, g.I);
  g.Gs = g.G;
  g.splits = p.splits;
  g.per = p.per;
  if (p.bt == 0) return thin_by(g, bf16, s);
  if (g.G % 4 != 0) {
    const int words = (g.G + 3) / 4;
    uint32_t* to = static_cast<uint32_t*>(workspace);
    auto lay = [&](const uint8_t* from, int64_t rows, uint32_t* at) {
      if (rows == 0) return 0;
      const int64_t groups = (rows * words + 255) / 256;
      hipLaunchKernelGGL(act4_words_kernel, dim3((unsigned)(groups < kGroupsX ? groups : kGroupsX)), dim3(256), 0, s, from, rows, g.G, words, at);
      return ok();
    };
    uint32_t* ws = to + (size_t)g.T * words;
    if (lay(g.xs, g.T, to) != 0 || lay(g.ws, (int64_t)g.E * g.O, ws) != 0) return -1;
    g.xs = reinterpret_cast<uint8_t*>(to);
    g.ws = reinterpret_cast<uint8_t*>(ws);
    g.Gs = 4 * words;
  }
  void* const out = g.out;
  uint8_t* const behind = static_cast<uint8_t*>(workspace) + words_bytes(p, g.E, g.T, g.O, g.I);
  if (p.splits > 1) g.out = behind;
  if (p.table) g.table = reinterpret_cast<int*>(behind);
  const int as_bf16 = bf16 && p.splits == 1;
  int rc;
  if (p.table) rc = p.bt == 64 ? experts_go<64>(g, as_bf16, s) : p.bt == 128 ? experts_go<128>(g, as_bf16, s) : experts_go<256>(g, as_bf16, s);
  else if (p.bm == 128) rc = p.bt == 64 ? tile_go<128, 64, 4, 2, 6>(g, as_bf16, s) : tile_go<128, 128, 4, 2, 4>(g, as_bf16, s);
  else if (p.bt == 64) rc = tile_go<256, 64, 8, 1, 3>(g, as_bf16, s);
  else rc = p.bt == 128 ? tile_go<256, 128, 4, 2, 3>(g, as_bf16, s) : tile_go<256, 256, 2, 4, 2>(g, as_bf16, s);
  if (rc != 0 || p.splits == 1) return rc;
  const int64_t items = (int64_t)g.N * g.O / 8;
  auto join = [&](auto kernel) {
    hipLaunchKernelGGL(kernel, dim3((unsigned)((items + 255) / 256)), dim3(256), 0, s, static_cast<const f32x4*>(g.out), p.splits, items, out);
    return ok();
  };
  return bf16 ? join(act4_join_kernel<true>) : join(act4_join_kernel<false>);
}

}  // namespace

int act4_pack_launch(int fmt, int64_t T, int64_t I, const void* X, float ws2, uint8_t* codes, uint8_t* scales, hipStream_t s) {
  const int64_t pieces = T * I / 8;
  const dim3 grid((unsigned)((pieces + 256 * kSteps - 1) / (256 * kSteps))), block(256);
  const u32x4* x = static_cast<const u32x4*>(X);
  if (fmt == kMX) hipLaunchKernelGGL((act4_pack_kernel<kMX>), grid, block, 0, s, x, pieces, 1.0f, codes, scales);
  else hipLaunchKernelGGL((act4_pack_kernel<kNV>), grid, block, 0, s, x, pieces, ws2, codes, scales);
  return ok();
}

static int unpack_go(int fmt, bool past, int64_t T, int64_t I, const uint8_t* codes, const uint8_t* scales, float ws2, void* X, hipStream_t s) {
  const int64_t pieces = T * I / 8;
  const dim3 grid((unsigned)((pieces + 256 * kSteps - 1) / (256 * kSteps))), block(256);
  auto go = [&](auto kernel) {
    hipLaunchKernelGGL(kernel, grid, block, 0, s, reinterpret_cast<const uint32_t*>(codes), scales, pieces, ws2, static_cast<u32x4*>(X));
    return ok();
  };
  if (past) return fmt == kMX ? go(act4_unpack_kernel<kMX, true>) : go(act4_unpack_kernel<kNV, true>);
  return fmt == kMX ? go(act4_unpack_kernel<kMX, false>) : go(act4_unpack_kernel<kNV, false>);
}

int act4_unpack_launch(int fmt, int64_t T, int64_t I, const uint8_t* codes, const uint8_t* scales, float ws2, void* X, hipStream_t s) {
  const int64_t bytes = 2 * T * I + T * I / 2 + T * I / (fmt == kMX ? 32 : 16);
  return unpack_go(fmt, bytes > kCacheBytes, T, I, codes, scales, fmt == kMX ? 1.0f : ws2, X, s);
}

size_t act4_workspace(int fmt, int64_t T, int64_t O, int64_t I) {
  return fmt == kMX ? plan_bytes(act4_plan(false, 1, T, O, I), 1, T, T, O, I) : (size_t)T * I * 2;
}

int act4_fwd(int fmt, int T, int O, int I, const uint8_t* x, const uint8_t* xs, float x_ws2, const uint8_t* codes,
             const uint8_t* scales, float ws2, void* Y, int y_bf16, void* workspace, hipStream_t s) {
  if (fmt == kNV) {
    if (unpack_go(fmt, false, T, I, x, xs, 1.0f, workspace, s) != 0) return -1;
    return gemm_fwd(fmt, T, O, I, workspace, codes, scales, x_ws2 * ws2, Y, y_bf16, s);
  }
  Act4Args g{};
  g.x = x; g.xs = xs; g.w = codes; g.ws = scales; g.out = Y;
  g.T = g.N = T; g.E = 1; g.O = O; g.I = I; g.G = I / 32;
  return product(g, y_bf16, workspace, s);
}

size_t act4_batched_workspace(int64_t E, int64_t T, int64_t N, int64_t O, int64_t I) {
  return plan_bytes(act4_plan(true, E, N, O, I), E, T, N, O, I);
}

int act4_fwd_batched(int E, int T, int N, int O, int I, const uint8_t* x, const uint8_t* xs, const int* rows,
                     const int* offsets, const uint8_t* codes, const uint8_t* scales, void* Y, int y_bf16, void* workspace,
                     hipStream_t s) {
  Act4Args g{};
  g.x = x; g.xs = xs; g.w = codes; g.ws = scales; g.out = Y; g.rows = rows; g.offsets = offsets;
  g.T = T; g.N = N; g.E = E; g.O = O; g.I = I; g.G = I / 32;
  return product(g, y_bf16, workspace, s);
}

}  // namespace sq
