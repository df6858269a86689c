// Activations kept in 8 bits between the forward and the backward pass, and
// the scale gradient that reads them.
//
// Blocks of 32 columns share one power of two 2^k (byte k + 127):
//   int8  k = floor(log2 amax) - 6, q = x 2^-k to the nearest whole number, ties
//         to even, held to +-127 (only 127.5 reaches past it)
//   e4m3  k = ceil(log2(amax / 448)), q = x 2^-k to the nearest E4M3, ties to even
// with k held to [-126, 127].  A block with an Inf or NaN takes byte 255 and
// reads as NaN.  An int8 value has 7 significant bits and an E4M3 value 4, so q
// 2^k is exact in bf16 and the products of the gradient are those of a bf16 X
// that holds these values.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <type_traits>

#include "sq_device.h"
#include "sq_gemm_args.h"
#include "sq_launch.h"
#include "sq_tiles.h"

namespace sq {

namespace {

enum Act { kInt8 = 0, kE4M3 = 1 };

// ------------------------------------------------------------------ pack
// One lane takes 8 columns (16 bytes of bf16), four lanes a block.  Streams
// 3.03 bytes per value.
template <int ACT>
__device__ __forceinline__ void pack8(const u32x4& w, uint8_t* __restrict__ codes, uint8_t* __restrict__ scales,
                                      int64_t at) {
  uint32_t amax = 0;                                          // of the bf16 bits without the sign: ordered as the values
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint32_t a = w[i] & 0x7FFF7FFFu;
    amax = max(amax, max(a & 0xFFFFu, a >> 16));
  }
  amax = max(amax, (uint32_t)__shfl_xor((int)amax, 1));
  amax = max(amax, (uint32_t)__shfl_xor((int)amax, 2));
  const int e = (int)(amax >> 7);                             // exponent field: floor(log2 amax) + 127 when not 0
  int byte = ACT == kInt8 ? e - 6 : e - 8 + ((amax & 0x7Fu) > 0x60u);
  byte = max(byte, 1);
  const bool bad = amax >= 0x7F80u;
  const float inv = __uint_as_float((uint32_t)(254 - byte) << 23);
  float v[8];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    v[2 * i] = __uint_as_float(w[i] << 16) * inv;
    v[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u) * inv;
  }
  u32x2 q;
  if constexpr (ACT == kInt8) {
    // adding 1.5 * 2^23 rounds to a whole number and leaves it in the low byte
    uint32_t r[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) r[i] = __float_as_uint(__builtin_amdgcn_fmed3f(v[i], -127.0f, 127.0f) + 12582912.0f);
#pragma unroll
    for (int h = 0; h < 2; ++h)
      q[h] = (r[4 * h] & 0xFFu) | (r[4 * h + 1] & 0xFFu) << 8 | (r[4 * h + 2] & 0xFFu) << 16 | r[4 * h + 3] << 24;
  } else {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      int c = __builtin_amdgcn_cvt_pk_fp8_f32(v[4 * h], v[4 * h + 1], 0, false);
      q[h] = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(v[4 * h + 2], v[4 * h + 3], c, true);
    }
  }
  if (bad) q = u32x2{0u, 0u};
  *reinterpret_cast<u32x2*>(codes + at * 8) = q;
  if ((at & 3) == 0) scales[at >> 2] = (uint8_t)(bad ? 255 : byte);
}

constexpr int kActSteps = 4;                                  // 8-column pieces per lane, all loaded first

template <int ACT>
__global__ __launch_bounds__(256) void act_pack_kernel(const u32x4* __restrict__ X, int64_t pieces,
                                                       uint8_t* __restrict__ codes, uint8_t* __restrict__ scales) {
  const int64_t p0 = (int64_t)blockIdx.x * (256 * kActSteps) + threadIdx.x;
  u32x4 w[kActSteps];
#pragma unroll
  for (int i = 0; i < kActSteps; ++i) {
    const int64_t p = p0 + i * 256;
    w[i] = X[p < pieces ? p : pieces - 1];
  }
#pragma unroll
  for (int i = 0; i < kActSteps; ++i)                         // whole blocks: pieces is a multiple of 4
    if (p0 + i * 256 < pieces) pack8<ACT>(w[i], codes, scales, p0 + i * 256);
}

// 8 values of one block as bf16 pairs, each product exact or rounded once
// (below the smallest bf16).
template <int ACT>
__device__ __forceinline__ u32x4 unpack8(u32x2 q, float scale) {
  u32x4 r;
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    f32x2 a, b;
    if constexpr (ACT == kInt8) {
      a = f32x2{(float)((int)(q[h] << 24) >> 24), (float)((int)(q[h] << 16) >> 24)};
      b = f32x2{(float)((int)(q[h] << 8) >> 24), (float)((int)q[h] >> 24)};
    } else {
      a = __builtin_amdgcn_cvt_pk_f32_fp8((int)q[h], false);
      b = __builtin_amdgcn_cvt_pk_f32_fp8((int)q[h], true);
    }
    r[2 * h] = bits_of(__builtin_convertvector((f32x2{a.x * scale, a.y * scale}), bf16x2));
    r[2 * h + 1] = bits_of(__builtin_convertvector((f32x2{b.x * scale, b.y * scale}), bf16x2));
  }
  return r;
}

template <int ACT>
__global__ __launch_bounds__(256) void act_unpack_kernel(const u32x2* __restrict__ codes,
                                                         const uint8_t* __restrict__ scales, int64_t pieces,
                                                         u32x4* __restrict__ X) {
  const int64_t p0 = (int64_t)blockIdx.x * (256 * kActSteps) + threadIdx.x;
  u32x2 q[kActSteps];
  uint32_t b[kActSteps];
#pragma unroll
  for (int i = 0; i < kActSteps; ++i) {
    const int64_t p = p0 + i * 256 < pieces ? p0 + i * 256 : pieces - 1;
    q[i] = codes[p];
    b[i] = scales[p >> 2];
  }
#pragma unroll
  for (int i = 0; i < kActSteps; ++i)
    if (p0 + i * 256 < pieces) X[p0 + i * 256] = unpack8<ACT>(q[i], e8m0_to_f32(b[i]));
}

// ------------------------------------------------------------------ dS
// dS[o,b] = sum_{j in block b} code[o,j] sum_t dY[t,o] x^[t,j], as the bf16
// product's tiles compute it (M = I, N = O, K = tokens), with x^ formed on
// chip: a lane loads 8 values of a row two stages ahead, turns them into bf16
// once per workgroup and writes them to the tile that the matrix cores read
// transposed.  dY is copied to LDS as it is.
//
// Groups share the grid: the experts of a layer (rows offsets[g] ..
// offsets[g + 1] of dY, their own codes and dS) or the parts of a long token
// sum (rows_per each, partial planes).  With `rows`, row s of dY meets row
// rows[s] of x^, so experts read the tokens' one copy.
struct Ds8Args {
  const uint8_t* x;         // [Tx, I]
  const uint8_t* xs;        // [Tx, I / 32]
  const int* rows;          // [N] or null
  const uint16_t* dy;       // [N, O]
  const uint8_t* codes;     // [O, I / 2] per group, code_step apart
  float* out;               // [O, G] per group, O * G apart
  const int* offsets;       // [groups + 1] or null: rows_per each
  int64_t code_step;
  int Tx, N, O, I, G;
  int groups, rows_per;
};

// Conversion of 8 kept values to bf16: int8 as (q + 128) s - 128 s, exact in
// one fused step; E4M3 by the scaled converts.
template <int ACT>
__device__ __forceinline__ u32x4 kept8(u32x2 q, uint32_t sb) {
  u32x4 r;
  if constexpr (ACT == kInt8) {
    const float s = e8m0_to_f32(sb), z = -128.0f * s;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const uint32_t u = q[h] ^ 0x80808080u;
      const float a = __builtin_fmaf((float)(u & 0xFFu), s, z), b = __builtin_fmaf((float)((u >> 8) & 0xFFu), s, z);
      const float c = __builtin_fmaf((float)((u >> 16) & 0xFFu), s, z), d = __builtin_fmaf((float)(u >> 24), s, z);
      r[2 * h] = pack_hi16(a, b);
      r[2 * h + 1] = pack_hi16(c, d);
    }
  } else {
    const float s = e8m0_as_scale_operand(sb);
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      r[2 * h] = bits_of(__builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((int)q[h], s, false));
      r[2 * h + 1] = bits_of(__builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((int)q[h], s, true));
    }
  }
  return r;
}

// One resident workgroup runs its share of the tiles as one pipeline of 64-row
// stages (two LDS buffers): a cursor two stages ahead loads x^'s items at the
// start of a step and, after the step's barrier, converts them and copies dY's
// stage into the buffer just read; with `rows`, the row numbers are read
// another stage ahead.  Every barrier waits for all loads.  A group without
// rows runs one stage of zeros, so its dS is 0.
template <int FMT, int ACT, int BM, int BN, int WGM, int WGN, bool ROWS>
__global__ __launch_bounds__(64 * WGM * WGN) void ds8_kernel(Ds8Args g) {
  constexpr int NT = 64 * WGM * WGN;
  constexpr int WM = BM / WGM, WN = BN / WGN;
  constexpr int TM = WM / 32, TN = WN / 32;
  constexpr int kA = BM * kBK * 2, kB = BN * kBK * 2;
  constexpr int kPer = kBK * (BM / 8) / NT;                   // 8-column items per thread and stage
  constexpr int kRowStep = NT / (BM / 8);
  static_assert(kPer * NT == kBK * (BM / 8) && kPer * kRowStep == kBK, "items split over the threads");
  using DB = DmaNat<BN, NT, kBK>;
  __shared__ __attribute__((aligned(16))) uint8_t lds0[kA + kB];
  __shared__ __attribute__((aligned(16))) uint8_t lds1[kA + kB];

  const int tid = threadIdx.x;
  const int lane = tid & 63, wave = tid >> 6;
  const int wave_u = __builtin_amdgcn_readfirstlane(wave);
  const int wm0 = (wave / WGN) * WM, wn0 = (wave % WGN) * WN;
  const int O = g.O, I = g.I, G = g.G;
  const int tiles_m = (I + BM - 1) / BM, tiles_n = (O + BN - 1) / BN, per = tiles_m * tiles_n;
  const int total = per * g.groups;

  // positions first, first + step, ... below end: XCD x takes the x-th
  // contiguous stretch, its workgroups deal it round robin
  const int w = (int)blockIdx.x, nwg = (int)gridDim.x, x = w % kXcds;
  const int step = nwg / kXcds + (x < nwg % kXcds ? 1 : 0);
  const int tq = total / kXcds, tr = total % kXcds;
  const int s0 = x < tr ? x * (tq + 1) : tr * (tq + 1) + (x - tr) * tq;
  const int first = s0 + w / kXcds, end = s0 + (x < tr ? tq + 1 : tq);
  if (first >= end) return;

  // One stage of a tile: group, corner, its rows [r0, r0 + n), stage kt of nk.
  struct Cursor {
    int pos, e, m0, n0, r0, n, kt, nk;
  };
  auto locate = [&](Cursor& c) {
    c.e = c.pos / per;
    int tm, tn;
    tile_at<8>(c.pos - c.e * per, tiles_m, tiles_n, tm, tn);
    c.m0 = tm * BM;
    c.n0 = tn * BN;
    int a, b;
    if (g.offsets) {                                          // device data: held to the rows there are
      a = min(max(g.offsets[c.e], 0), g.N);
      b = min(max(g.offsets[c.e + 1], a), g.N);
    } else {
      a = min(c.e * g.rows_per, g.N);
      b = min(a + g.rows_per, g.N);
    }
    c.r0 = a;
    c.n = b - a;
    c.kt = 0;
    c.nk = c.n > 0 ? (c.n + kBK - 1) / kBK : 1;
  };
  auto advance = [&](Cursor& c) {                             // c.pos >= end once past the last stage
    if (++c.kt == c.nk) {
      c.pos += step;
      if (c.pos < end) locate(c);
    }
  };

  const __amdgpu_buffer_rsrc_t rx = make_rsrc(g.x, (uint32_t)((size_t)g.Tx * I));
  const __amdgpu_buffer_rsrc_t rxs = make_rsrc(g.xs, (uint32_t)((size_t)g.Tx * (I / 32)));
  const __amdgpu_buffer_rsrc_t rrow = make_rsrc(g.rows, ROWS ? (uint32_t)g.N * 4u : 0u);
  const int irow = tid / (BM / 8), icol = (tid % (BM / 8)) * 8;

  int idx[ROWS ? kPer : 1];
  auto load_rows = [&](const Cursor& c) {
    if constexpr (ROWS) {
#pragma unroll
      for (int p = 0; p < kPer; ++p) {
        const int k = c.kt * kBK + irow + p * kRowStep;
        idx[p] = __builtin_amdgcn_raw_buffer_load_b32(rrow, (int)(k < c.n ? (uint32_t)(c.r0 + k) * 4u : kOOB), 0, 0);
      }
    }
  };
  u32x2 q[kPer];
  uint32_t sb[kPer];
  auto load_items = [&](const Cursor& c) {
#pragma unroll
    for (int p = 0; p < kPer; ++p) {
      const int k = c.kt * kBK + irow + p * kRowStep, col = c.m0 + icol;
      const uint32_t r = ROWS ? (uint32_t)idx[p] : (uint32_t)(c.r0 + k);
      const bool in = k < c.n && col < I && r < (uint32_t)g.Tx;
      const uint32_t oc = in ? r * (uint32_t)I + (uint32_t)col : kOOB;
      const uint32_t os = in ? r * (uint32_t)(I / 32) + (uint32_t)(col / 32) : kOOB;
      q[p] = __builtin_bit_cast(u32x2, __builtin_amdgcn_raw_buffer_load_b64(rx, (int)oc, 0, 0));
      sb[p] = __builtin_amdgcn_raw_buffer_load_b8(rxs, (int)os, 0, 0);
    }
  };
  auto commit_items = [&](SQ_LDS uint8_t* st) {
    SQ_LDS uint16_t* s = (SQ_LDS uint16_t*)st;
#pragma unroll
    for (int p = 0; p < kPer; ++p)
      *(SQ_LDS u32x4*)(s + nat_off<BM>(irow + p * kRowStep, icol)) = kept8<ACT>(q[p], sb[p]);
  };
  DB dB;
  auto copy_dy = [&](const Cursor& c, SQ_LDS uint8_t* st) {
    const DmaRsrc rb = make_dma_rsrc(g.dy + (size_t)c.r0 * O, (uint32_t)((size_t)c.n * O * 2));
    dB.init(O, O, c.n0, tid);
    dB.issue(rb, (SQ_LDS uint16_t*)(st + kA), (uint32_t)c.kt * kBK * (uint32_t)O * 2u, wave_u);
  };

  f32x16 acc[TM][TN];
  auto clear = [&]() {
#pragma unroll
    for (int i = 0; i < TM; ++i)
#pragma unroll
      for (int j = 0; j < TN; ++j)
#pragma unroll
        for (int r = 0; r < 16; ++r) acc[i][j][r] = 0.0f;
  };
  clear();
  struct Frag {
    bf16x8 a[TM];
    bf16x8 b[TN];
  };
  Frag F0, F1;
  auto read = [&](SQ_LDS uint8_t* st, auto KK, Frag& f) {
    constexpr int kk = decltype(KK)::value;
    const SQ_LDS uint16_t* a = (const SQ_LDS uint16_t*)st;
    const SQ_LDS uint16_t* b = (const SQ_LDS uint16_t*)(st + kA);
#pragma unroll
    for (int i = 0; i < TM; ++i) f.a[i] = nat_frag<BM>(a, kk, wm0 + i * 32, lane);
#pragma unroll
    for (int j = 0; j < TN; ++j) f.b[j] = nat_frag<BN>(b, kk, wn0 + j * 32, lane);
  };
  auto mma = [&](Frag& f) {
#pragma unroll
    for (int i = 0; i < TM; ++i)
#pragma unroll
      for (int j = 0; j < TN; ++j)
        acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(f.a[i], f.b[j], acc[i][j], 0, 0, 0);
  };
  using I0 = std::integral_constant<int, 0>;
  using I1 = std::integral_constant<int, 1>;
  using I2 = std::integral_constant<int, 2>;
  using I3 = std::integral_constant<int, 3>;

  Cursor cc, cd, cr;                                          // compute; items and dY, two ahead; rows, three ahead
  cc.pos = first;
  locate(cc);
  cd = cc;
  cr = cc;

  // prologue: stages 0 and 1 whole, the rows of stage 2
#pragma unroll
  for (int b = 0; b < 2; ++b) {
    if (cd.pos < end) {
      SQ_LDS uint8_t* st = b == 0 ? (SQ_LDS uint8_t*)lds0 : (SQ_LDS uint8_t*)lds1;
      load_rows(cd);
      load_items(cd);
      copy_dy(cd, st);
      commit_items(st);
      advance(cd);
    }
  }
  cr = cd;
  if (cr.pos < end) {
    load_rows(cr);
    advance(cr);
  }
  wait_vm_lgkm0<0>();
  __builtin_amdgcn_s_barrier();
  __builtin_amdgcn_sched_barrier(0);
  SQ_LDS uint8_t* cur = (SQ_LDS uint8_t*)lds0;
  SQ_LDS uint8_t* nxt = (SQ_LDS uint8_t*)lds1;
  read(cur, I0{}, F0);
  for (;;) {
    const bool ahead = cd.pos < end;
    if (ahead) load_items(cd);
    if constexpr (ROWS) {
      if (cr.pos < end) {
        load_rows(cr);
        advance(cr);
      }
    }
    read(cur, I1{}, F1);
    mma(F0);
    read(cur, I2{}, F0);
    mma(F1);
    read(cur, I3{}, F1);
    mma(F0);
    wait_vm_lgkm0<0>();
    __builtin_amdgcn_s_barrier();
    __builtin_amdgcn_sched_barrier(0);
    const bool last = cc.kt + 1 == cc.nk;
    const bool more = !last || cc.pos + step < end;
    if (more) read(nxt, I0{}, F0);
    if (ahead) copy_dy(cd, cur);
    mma(F1);
    if (ahead) {
      commit_items(cur);
      advance(cd);
    }
    if (last) {
      float* const dS = g.out + (size_t)cc.e * O * G;
      u32x4 cw[TM * TN];
      ds_codes<FMT, TM, TN>(cw, g.codes + (size_t)cc.e * g.code_step, O, I, cc.m0 + wm0, cc.n0 + wn0, lane);
      if (cc.m0 + BM <= I && cc.n0 + BN <= O)
        ds_store<FMT, TM, TN, true>(acc, cw, dS, O, I, G, cc.m0 + wm0, cc.n0 + wn0, lane);
      else
        ds_store<FMT, TM, TN, false>(acc, cw, dS, O, I, G, cc.m0 + wm0, cc.n0 + wn0, lane);
      if (!more) break;
      clear();
    }
    advance(cc);
    SQ_LDS uint8_t* t = cur;
    cur = nxt;
    nxt = t;
  }
  wait_vm_lgkm0<0>();
}

// One tile per workgroup, for long token sums.  Between two barriers a step reads
// and multiplies one 64-row stage; x^'s items of the stage two ahead are loaded
// at its start and written to the freed buffer after its barrier, dY's copy of
// that stage goes out half there and half in the next step's first slice.
template <int FMT, int ACT, int BM, int BN, int WGM, int WGN, bool ROWS>
__global__ __launch_bounds__(64 * WGM * WGN) void ds8_tile_kernel(Ds8Args g) {
  constexpr int NT = 64 * WGM * WGN;
  constexpr int WM = BM / WGM, WN = BN / WGN;
  constexpr int TM = WM / 32, TN = WN / 32;
  constexpr int kA = BM * kBK * 2, kB = BN * kBK * 2;
  constexpr int kPer = kBK * (BM / 8) / NT;                   // 8-column items per thread and stage
  constexpr int kRowStep = NT / (BM / 8);
  static_assert(kPer * NT == kBK * (BM / 8) && kPer * kRowStep == kBK, "items split over the threads");
  using DB = DmaNat<BN, NT, kBK>;
  __shared__ __attribute__((aligned(16))) uint8_t lds0[kA + kB];
  __shared__ __attribute__((aligned(16))) uint8_t lds1[kA + kB];

  const int tid = threadIdx.x;
  const int lane = tid & 63, wave = tid >> 6;
  const int wave_u = __builtin_amdgcn_readfirstlane(wave);
  const int wm0 = (wave / WGN) * WM, wn0 = (wave % WGN) * WN;
  const int O = g.O, I = g.I, G = g.G;
  const int tiles_m = (I + BM - 1) / BM, tiles_n = (O + BN - 1) / BN, per = tiles_m * tiles_n;
  const int pos = xcd_stretch((int)blockIdx.x, (int)gridDim.x);
  const int e = pos / per;
  int tm, tn;
  tile_at<8>(pos - e * per, tiles_m, tiles_n, tm, tn);
  const int m0 = tm * BM, n0 = tn * BN;
  int r0, n;
  if (g.offsets) {                                            // device data: held to the rows there are
    r0 = __builtin_amdgcn_readfirstlane(min(max(g.offsets[e], 0), g.N));
    n = __builtin_amdgcn_readfirstlane(min(max(g.offsets[e + 1], r0), g.N)) - r0;
  } else {
    r0 = min(e * g.rows_per, g.N);
    n = min(r0 + g.rows_per, g.N) - r0;
  }
  const int nk = (n + kBK - 1) / kBK;

  const int irow = tid / (BM / 8), icol = (tid % (BM / 8)) * 8;
  const bool icol_in = m0 + icol < I;
  // x^ by row number, or the group's rows from a base that moves with the stage
  const __amdgpu_buffer_rsrc_t rx = make_rsrc(g.x, (uint32_t)((size_t)g.Tx * I));
  const __amdgpu_buffer_rsrc_t rxs = make_rsrc(g.xs, (uint32_t)((size_t)g.Tx * (I / 32)));
  const __amdgpu_buffer_rsrc_t rrow = make_rsrc(g.rows, ROWS ? (uint32_t)g.N * 4u : 0u);
  uint32_t qoff[ROWS ? 1 : kPer], soff[ROWS ? 1 : kPer];
  if constexpr (!ROWS) {
#pragma unroll
    for (int p = 0; p < kPer; ++p) {
      const uint32_t r = (uint32_t)(irow + p * kRowStep);
      qoff[p] = icol_in ? r * (uint32_t)I + (uint32_t)(m0 + icol) : kOOB;
      soff[p] = icol_in ? r * (uint32_t)(I / 32) + (uint32_t)((m0 + icol) / 32) : kOOB;
    }
  }
  int idx[ROWS ? kPer : 1];
  auto load_rows = [&](int kt) {
    if constexpr (ROWS) {
#pragma unroll
      for (int p = 0; p < kPer; ++p) {
        const int k = kt * kBK + irow + p * kRowStep;
        idx[p] = __builtin_amdgcn_raw_buffer_load_b32(rrow, (int)(k < n ? (uint32_t)(r0 + k) * 4u : kOOB), 0, 0);
      }
    }
  };
  u32x2 q[kPer];
  uint32_t sb[kPer];
  auto load_items = [&](int kt) {
    if constexpr (ROWS) {
#pragma unroll
      for (int p = 0; p < kPer; ++p) {
        const uint32_t r = (uint32_t)idx[p];
        const bool in = kt * kBK + irow + p * kRowStep < n && icol_in && r < (uint32_t)g.Tx;
        const uint32_t oc = in ? r * (uint32_t)I + (uint32_t)(m0 + icol) : kOOB;
        const uint32_t os = in ? r * (uint32_t)(I / 32) + (uint32_t)((m0 + icol) / 32) : kOOB;
        q[p] = __builtin_bit_cast(u32x2, __builtin_amdgcn_raw_buffer_load_b64(rx, (int)oc, 0, 0));
        sb[p] = __builtin_amdgcn_raw_buffer_load_b8(rxs, (int)os, 0, 0);
      }
    } else {
      const int first = r0 + kt * kBK, left = n - kt * kBK;   // rows of the group from this stage on
      const __amdgpu_buffer_rsrc_t bx = make_rsrc(g.x + (size_t)first * I, (uint32_t)left * (uint32_t)I);
      const __amdgpu_buffer_rsrc_t bs = make_rsrc(g.xs + (size_t)first * (I / 32), (uint32_t)left * (uint32_t)(I / 32));
#pragma unroll
      for (int p = 0; p < kPer; ++p) {
        q[p] = __builtin_bit_cast(u32x2, __builtin_amdgcn_raw_buffer_load_b64(bx, (int)qoff[p], 0, 0));
        sb[p] = __builtin_amdgcn_raw_buffer_load_b8(bs, (int)soff[p], 0, 0);
      }
    }
  };
  auto stage = [&](auto S) { return decltype(S)::value == 0 ? (SQ_LDS uint8_t*)lds0 : (SQ_LDS uint8_t*)lds1; };
  auto commit_items = [&](auto S) {
    SQ_LDS uint16_t* s = (SQ_LDS uint16_t*)stage(S);
#pragma unroll
    for (int p = 0; p < kPer; ++p)
      *(SQ_LDS u32x4*)(s + nat_off<BM>(irow + p * kRowStep, icol)) = kept8<ACT>(q[p], sb[p]);
  };
  const DmaRsrc rb = make_dma_rsrc(g.dy + (size_t)r0 * O, (uint32_t)((size_t)n * O * 2));
  DB dB;
  dB.init(O, O, n0, tid);
  auto dma_half = [&](auto S, int kt, auto HALF) {
    constexpr int h = decltype(HALF)::value;
    dB.template issue_part<h * DB::kInst / 2, (h + 1) * DB::kInst / 2>(rb, (SQ_LDS uint16_t*)(stage(S) + kA),
                                                                      (uint32_t)kt * kBK * (uint32_t)O * 2u, wave_u);
  };

  f32x16 acc[TM][TN];
#pragma unroll
  for (int i = 0; i < TM; ++i)
#pragma unroll
    for (int j = 0; j < TN; ++j)
#pragma unroll
      for (int r = 0; r < 16; ++r) acc[i][j][r] = 0.0f;
  struct Frag {
    bf16x8 a[TM];
    bf16x8 b[TN];
  };
  Frag F0, F1;
  auto read = [&](auto S, auto KK, Frag& f) {
    constexpr int kk = decltype(KK)::value;
    const SQ_LDS uint16_t* a = (const SQ_LDS uint16_t*)stage(S);
    const SQ_LDS uint16_t* b = (const SQ_LDS uint16_t*)(stage(S) + kA);
#pragma unroll
    for (int i = 0; i < TM; ++i) f.a[i] = nat_frag<BM>(a, kk, wm0 + i * 32, lane);
#pragma unroll
    for (int j = 0; j < TN; ++j) f.b[j] = nat_frag<BN>(b, kk, wn0 + j * 32, lane);
  };
  auto mma = [&](Frag& f) {
#pragma unroll
    for (int i = 0; i < TM; ++i)
#pragma unroll
      for (int j = 0; j < TN; ++j)
        acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(f.a[i], f.b[j], acc[i][j], 0, 0, 0);
  };
  using I0 = std::integral_constant<int, 0>;
  using I1 = std::integral_constant<int, 1>;
  using I2 = std::integral_constant<int, 2>;
  using I3 = std::integral_constant<int, 3>;
  auto step = [&](auto S, int kt) {
    using SN = std::integral_constant<int, 1 - decltype(S)::value>;
    if (kt + 2 < nk) {
      load_items(kt + 2);
      load_rows(kt + 3);
    }
    read(S, I1{}, F1);
    if (kt + 1 < nk) dma_half(SN{}, kt + 1, I1{});
    mma(F0);
    read(S, I2{}, F0);
    mma(F1);
    read(S, I3{}, F1);
    mma(F0);
    wait_vm_lgkm0<0>();
    __builtin_amdgcn_s_barrier();
    __builtin_amdgcn_sched_barrier(0);
    if (kt + 1 < nk) read(SN{}, I0{}, F0);
    if (kt + 2 < nk) dma_half(S, kt + 2, I0{});
    mma(F1);
    if (kt + 2 < nk) commit_items(S);
  };
  // prologue: stage 0 whole, stage 1's items and the first half of its copy
  if (nk > 0) {
    load_rows(0);
    load_items(0);
    load_rows(1);
    dma_half(I0{}, 0, I0{});
    dma_half(I0{}, 0, I1{});
    commit_items(I0{});
    if (1 < nk) {
      load_items(1);
      load_rows(2);
      commit_items(I1{});
    }
    wait_vm_lgkm0<0>();
    __builtin_amdgcn_s_barrier();
    __builtin_amdgcn_sched_barrier(0);
    read(I0{}, I0{}, F0);
    if (1 < nk) dma_half(I1{}, 1, I0{});
  }
  for (int kt0 = 0; kt0 < nk; kt0 += 2) {
    step(I0{}, kt0);
    if (kt0 + 1 < nk) step(I1{}, kt0 + 1);
  }
  wait_vm_lgkm0<0>();

  float* const dS = g.out + (size_t)e * O * G;
  u32x4 cw[TM * TN];
  ds_codes<FMT, TM, TN>(cw, g.codes + (size_t)e * g.code_step, O, I, m0 + wm0, n0 + wn0, lane);
  if (m0 + BM <= I && n0 + BN <= O)
    ds_store<FMT, TM, TN, true>(acc, cw, dS, O, I, G, m0 + wm0, n0 + wn0, lane);
  else
    ds_store<FMT, TM, TN, false>(acc, cw, dS, O, I, G, m0 + wm0, n0 + wn0, lane);
}

// dS[i] = sum over s of part[s][i], s in increasing order; n is a multiple of 4.
__global__ __launch_bounds__(256) void ds8_reduce_kernel(const float* __restrict__ part, float* __restrict__ dS,
                                                         int64_t n, int splits) {
  const int64_t i4 = ((int64_t)blockIdx.x * 256 + threadIdx.x) * 4;
  if (i4 >= n) return;
  float4 acc = *reinterpret_cast<const float4*>(part + i4);
  for (int s = 1; s < splits; ++s) {
    const float4 v = *reinterpret_cast<const float4*>(part + (size_t)s * n + i4);
    acc.x += v.x; acc.y += v.y; acc.z += v.z; acc.w += v.w;
  }
  dS[i4] = acc.x; dS[i4 + 1] = acc.y; dS[i4 + 2] = acc.z; dS[i4 + 3] = acc.w;
}

inline int ok() { return hipGetLastError() == hipSuccess ? 0 : -1; }

template <int FMT, int ACT>
int ds8_go(const Ds8Args& g, bool large, hipStream_t s) {
  if (large) {
    const int64_t total = (int64_t)((g.I + 255) / 256) * ((g.O + 255) / 256) * g.groups;
    const dim3 grid((unsigned)total), block(512);
    if (g.rows) hipLaunchKernelGGL((ds8_tile_kernel<FMT, ACT, 256, 256, 2, 4, true>), grid, block, 0, s, g);
    else hipLaunchKernelGGL((ds8_tile_kernel<FMT, ACT, 256, 256, 2, 4, false>), grid, block, 0, s, g);
    return ok();
  }
  const int64_t total = (int64_t)((g.I + 127) / 128) * ((g.O + 127) / 128) * g.groups;
  const dim3 grid((unsigned)(total < 2 * kCUs ? total : 2 * kCUs)), block(512);
  if (g.rows) hipLaunchKernelGGL((ds8_kernel<FMT, ACT, 128, 128, 2, 4, true>), grid, block, 0, s, g);
  else hipLaunchKernelGGL((ds8_kernel<FMT, ACT, 128, 128, 2, 4, false>), grid, block, 0, s, g);
  return ok();
}

int ds8_launch(int fmt, int act, bool large, const Ds8Args& g, hipStream_t s) {
  auto go = [&](auto F, auto A) {
    constexpr int f = decltype(F)::value, a = decltype(A)::value;
    return ds8_go<f, a>(g, large, s);
  };
  using MX = std::integral_constant<int, kMX>;
  using NV = std::integral_constant<int, kNV>;
  using A0 = std::integral_constant<int, kInt8>;
  using A1 = std::integral_constant<int, kE4M3>;
  if (fmt == kMX) return act == kInt8 ? go(MX{}, A0{}) : go(MX{}, A1{});
  return act == kInt8 ? go(NV{}, A0{}) : go(NV{}, A1{});
}

// Parts of the token sum of one layer whose 256 x 256 tiles leave CUs idle (as
// the bf16 product splits it: at least 4 stages each, 8 parts at most).
int ds8_splits(int T, int O, int I) {
  const int64_t tiles = (int64_t)((I + 255) / 256) * ((O + 255) / 256);
  const int nk = (T + kBK - 1) / kBK;
  if (tiles >= kCUs) return 1;
  int splits = (int)(kCUs / tiles);
  splits = min(splits, min(nk / 4, 8));
  return splits < 2 ? 1 : splits;
}

}  // namespace

int act_pack_launch(int act, int64_t T, int64_t I, const void* X, uint8_t* codes, uint8_t* scales, hipStream_t s) {
  const int64_t pieces = T * I / 8, blocks = (pieces + 256 * kActSteps - 1) / (256 * kActSteps);
  const u32x4* x = static_cast<const u32x4*>(X);
  if (act == kInt8)
    hipLaunchKernelGGL((act_pack_kernel<kInt8>), dim3((unsigned)blocks), dim3(256), 0, s, x, pieces, codes, scales);
  else
    hipLaunchKernelGGL((act_pack_kernel<kE4M3>), dim3((unsigned)blocks), dim3(256), 0, s, x, pieces, codes, scales);
  return ok();
}

int act_unpack_launch(int act, int64_t T, int64_t I, const uint8_t* codes, const uint8_t* scales, void* X,
                      hipStream_t s) {
  const int64_t pieces = T * I / 8, blocks = (pieces + 256 * kActSteps - 1) / (256 * kActSteps);
  const u32x2* c = reinterpret_cast<const u32x2*>(codes);
  u32x4* x = static_cast<u32x4*>(X);
  if (act == kInt8)
    hipLaunchKernelGGL((act_unpack_kernel<kInt8>), dim3((unsigned)blocks), dim3(256), 0, s, c, scales, pieces, x);
  else
    hipLaunchKernelGGL((act_unpack_kernel<kE4M3>), dim3((unsigned)blocks), dim3(256), 0, s, c, scales, pieces, x);
  return ok();
}

size_t dscale_act8_workspace(int fmt, int T, int O, int I) {
  const int splits = ds8_splits(T, O, I);
  return splits < 2 ? 0 : (size_t)splits * O * (I / (fmt == kMX ? 32 : 16)) * sizeof(float);
}

int dscale_act8(int fmt, int act, int T, int O, int I, const uint8_t* x, const uint8_t* xs, const void* dY,
                const uint8_t* codes, float* dS, void* workspace, hipStream_t s) {
  Ds8Args g{};
  g.x = x; g.xs = xs; g.dy = static_cast<const uint16_t*>(dY); g.codes = codes;
  g.Tx = T; g.N = T; g.O = O; g.I = I; g.G = I / (fmt == kMX ? 32 : 16);
  const int64_t tiles = (int64_t)((I + 255) / 256) * ((O + 255) / 256);
  const int splits = ds8_splits(T, O, I);
  g.groups = splits;
  g.rows_per = splits < 2 ? T : ((T + kBK - 1) / kBK + splits - 1) / splits * kBK;
  g.out = splits < 2 ? dS : static_cast<float*>(workspace);
  const int rc = ds8_launch(fmt, act, splits >= 2 || tiles >= kCUs, g, s);
  if (rc != 0 || splits < 2) return rc;
  const int64_t n = (int64_t)O * g.G;                         // a multiple of 8: O % 8 == 0
  hipLaunchKernelGGL(ds8_reduce_kernel, dim3((unsigned)((n / 4 + 255) / 256)), dim3(256), 0, s,
                     static_cast<const float*>(workspace), dS, n, splits);
  return ok();
}

int dscale_act8_batched(int fmt, int act, int E, int Tx, int N, int O, int I, const uint8_t* x, const uint8_t* xs,
                        const int32_t* rows, const int32_t* offsets, const void* dY, const uint8_t* codes, float* dS,
                        hipStream_t s) {
  Ds8Args g{};
  g.x = x; g.xs = xs; g.rows = rows; g.dy = static_cast<const uint16_t*>(dY); g.codes = codes; g.out = dS;
  g.offsets = offsets;
  g.code_step = (int64_t)O * I / 2;
  g.Tx = Tx; g.N = N; g.O = O; g.I = I; g.G = I / (fmt == kMX ? 32 : 16);
  g.groups = E;
  // as the bf16 grouped product: large tiles where they fill the chip and the
  // experts average 512 rows
  const int64_t tiles = (int64_t)((I + 255) / 256) * ((O + 255) / 256) * E;
  return ds8_launch(fmt, act, tiles >= kCUs && N >= (int64_t)512 * E, g, s);
}

}  // namespace sq
