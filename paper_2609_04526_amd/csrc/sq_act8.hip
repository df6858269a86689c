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
// 3.03 bytes per value: 8192 x 14336 to E4M3 in 58 us (6.1 TB/s), and back in 53
// (6.6 TB/s, mostly writes that the cache takes).
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

// STREAM: an X that the caches do not hold is read past them (58 us there, 78
// without); one that they do is read from them (12106 x 2432 and back: 29, 31).
constexpr int64_t kActStreamBytes = int64_t(128) << 20;

template <int ACT, bool STREAM>
__global__ __launch_bounds__(256) void act_pack_kernel(const u32x4* __restrict__ X, int64_t pieces,
                                                       uint8_t* __restrict__ codes, uint8_t* __restrict__ scales) {
  const int64_t p0 = (int64_t)blockIdx.x * (256 * kActSteps) + threadIdx.x;
  u32x4 w[kActSteps];
#pragma unroll
  for (int i = 0; i < kActSteps; ++i) {
    const int64_t p = p0 + i * 256;
    const u32x4* x = X + (p < pieces ? p : pieces - 1);
    w[i] = STREAM ? __builtin_nontemporal_load(x) : *x;
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
// A long token sum is split over workgroups where the tiles leave compute units
// idle: groups of rows_per rows each, with partial planes.
struct Ds8Args {
  const uint8_t* x;         // [N, I]
  const uint8_t* xs;        // [N, I / 32]
  const uint16_t* dy;       // [N, O]
  const uint8_t* codes;     // [O, I / 2]
  float* out;               // [O, G] per group, O * G apart
  int N, O, I, G;
  int groups, rows_per;
};

// Conversion of 8 kept values to bf16, as unpack8 does it: int8 as q s, whose 7 bits
// pack_hi16 keeps; E4M3 by the scaled converts.  ((q + 128) s - 128 s would be one
// instruction shorter, but 128 s overflows where q s does not: under byte 248, which
// blocks of 2^127 and more have.)
template <int ACT>
__device__ __forceinline__ u32x4 kept8(u32x2 q, uint32_t sb) {
  u32x4 r;
  if constexpr (ACT == kInt8) {
    const float s = e8m0_to_f32(sb);
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const float a = (float)((int)(q[h] << 24) >> 24) * s, b = (float)((int)(q[h] << 16) >> 24) * s;
      const float c = (float)((int)(q[h] << 8) >> 24) * s, d = (float)((int)q[h] >> 24) * s;
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

// One tile per workgroup, for long token sums.  Between two barriers a step reads
// and multiplies one 64-row stage; x^'s items of the stage two ahead are loaded
// at its start and written to the freed buffer after its barrier, dY's copy of
// that stage goes out half there and half in the next step's first slice.
template <int FMT, int ACT, int BM, int BN, int WGM, int WGN>
__global__ __launch_bounds__(64 * WGM * WGN) void ds8_tile_kernel(Ds8Args g) {
  constexpr int NT = 64 * WGM * WGN;
  constexpr int WM = BM / WGM, WN = BN / WGN;
  constexpr int TM = WM / 32, TN = WN / 32;
  constexpr int kA = BM * kBK * 2, kB = BN * kBK * 2;
  constexpr int kPer = kBK * (BM / 8) / NT;                   // 8-column items per thread and stage
  constexpr int kRowStep = NT / (BM / 8);
  static_assert(kPer * NT == kBK * (BM / 8) && kPer * kRowStep == kBK, "items split over the threads");
  constexpr int kEvery = TM * TN / kPer;                      // products per item of the last slice
  static_assert(kEvery * kPer == TM * TN, "items spread over the slice");
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
  const int r0 = min(e * g.rows_per, g.N), n = min(r0 + g.rows_per, g.N) - r0;
  const int nk = (n + kBK - 1) / kBK;

  const int irow = tid / (BM / 8), icol = (tid % (BM / 8)) * 8;
  const bool icol_in = m0 + icol < I;
  uint32_t qoff[kPer], soff[kPer];                            // from the stage's first row
#pragma unroll
  for (int p = 0; p < kPer; ++p) {
    const uint32_t r = (uint32_t)(irow + p * kRowStep);
    qoff[p] = icol_in ? r * (uint32_t)I + (uint32_t)(m0 + icol) : kOOB;
    soff[p] = icol_in ? r * (uint32_t)(I / 32) + (uint32_t)((m0 + icol) / 32) : kOOB;
  }
  u32x2 q[kPer];
  uint32_t sb[kPer];
  auto load_items = [&](int kt) {
    const int first = r0 + kt * kBK, left = n - kt * kBK;     // rows of the part from this stage on
    const __amdgpu_buffer_rsrc_t bx = make_rsrc(g.x + (size_t)first * I, (uint32_t)left * (uint32_t)I);
    const __amdgpu_buffer_rsrc_t bs = make_rsrc(g.xs + (size_t)first * (I / 32), (uint32_t)left * (uint32_t)(I / 32));
#pragma unroll
    for (int p = 0; p < kPer; ++p) {
      q[p] = __builtin_bit_cast(u32x2, __builtin_amdgcn_raw_buffer_load_b64(bx, (int)qoff[p], 0, 0));
      sb[p] = __builtin_amdgcn_raw_buffer_load_b8(bs, (int)soff[p], 0, 0);
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
    if (kt + 2 < nk) load_items(kt + 2);
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
    // an item's conversion after every second product of the slice, so that the
    // vector units work while the matrix cores do (past the last stage the
    // buffer is read no more)
    SQ_LDS uint16_t* s = (SQ_LDS uint16_t*)stage(S);
#pragma unroll
    for (int m = 0; m < TM * TN; ++m) {
      const int i = m / TN, j = m % TN;
      acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(F1.a[i], F1.b[j], acc[i][j], 0, 0, 0);
      if (m % kEvery == kEvery - 1) {
        const int p = m / kEvery;
        *(SQ_LDS u32x4*)(s + nat_off<BM>(irow + p * kRowStep, icol)) = kept8<ACT>(q[p], sb[p]);
      }
    }
#pragma unroll
    for (int p = 0; p < kPer; ++p) {
      __builtin_amdgcn_sched_group_barrier(0x008, kEvery, 0);                       // MFMA
      __builtin_amdgcn_sched_group_barrier(0x002, ACT == kInt8 ? 24 : 8, 0);        // vector ALU
      __builtin_amdgcn_sched_group_barrier(0x200, 1, 0);                            // LDS write
    }
  };
  // prologue: stage 0 whole, stage 1's items and the first half of its copy
  if (nk > 0) {
    load_items(0);
    dma_half(I0{}, 0, I0{});
    dma_half(I0{}, 0, I1{});
    commit_items(I0{});
    if (1 < nk) {
      load_items(1);
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
  ds_codes<FMT, TM, TN>(cw, g.codes, O, I, m0 + wm0, n0 + wn0, lane);
  if (m0 + BM <= I && n0 + BN <= O)
    ds_store<FMT, TM, TN, true>(acc, cw, dS, O, I, G, m0 + wm0, n0 + wn0, lane);
  else
    ds_store<FMT, TM, TN, false>(acc, cw, dS, O, I, G, m0 + wm0, n0 + wn0, lane);
}

// ------------------------------------------------------------------ experts
// The experts' products from the tokens' unpacked x (each token is unpacked
// once, its row read by every expert that it goes to).  An expert has a few
// 64-row stages, and a workgroup per tile would spend most of its life filling
// and draining its pipeline, so each workgroup stays resident and runs its share
// of the tiles as one pipeline of stages in two LDS buffers: the copies go two
// stages ahead of the products, across the ends of tiles, and every barrier waits
// for all loads.  Tiles are 256 x 256, a wave's part 128 x 64: of the shapes that
// fit the registers the one that reads the fewest operand bytes from LDS.  Rows that
// are picked and rows in place take the same time (128 experts of 768 x 2048 over
// 32768 rows 140 and 146 us).
constexpr int kRowsBM = 256, kRowsBN = 256;
constexpr int kTakenStep = 64;          // a queue's count in a line of its own
constexpr int kQueueUnits = 1040;       // of one queue at most: 8192 experts, or 64 units and more of fewer

// The epilogue of a wave's 128 x 64 (input features r0 .., output features c0 ..):
// products with the codes summed over the scale blocks, as ds_store but with one
// fused step per element.  A lane holds 16 of a 32-feature tile's rows of one
// output feature, the lane 32 away the others.
//
// Scattered accesses of 4 and 16 bytes per row took as long as a third of a stage:
// each row's 64 bytes of codes come as 16 bytes per lane and load, the lane
// halves taking neighbouring ones and exchanging them (codes of pair p and both
// halves: tiles 2 p and 2 p + 1), and a row's sums leave 16 bytes at a time.
constexpr int kRowsTM = 4, kRowsTN = 2;
__device__ __forceinline__ void load_code_pairs(u32x4 (&cw)[kRowsTN][kRowsTM / 2], const uint8_t* codes, int O, int I,
                                                int r0, int c0, int lane) {
  const __amdgpu_buffer_rsrc_t rs = make_rsrc(codes, (uint32_t)((size_t)O * (I >> 1)));
#pragma unroll
  for (int j = 0; j < kRowsTN; ++j) {
    const int o = c0 + j * 32 + (lane & 31);
#pragma unroll
    for (int p = 0; p < kRowsTM / 2; ++p) {
      const int jb = r0 + 64 * p + 32 * (lane >> 5);
      const uint32_t off = o < O && jb < I ? (uint32_t)o * (uint32_t)(I >> 1) + (uint32_t)(jb >> 1) : kOOB;
      cw[j][p] = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(rs, (int)off, 0, 0));
    }
  }
}
// a and b by lane halves: {a.low, b.low} and {a.high, b.high}.
__device__ __forceinline__ void swap_halves(uint32_t& a, uint32_t& b) {
  const auto r = __builtin_amdgcn_permlane32_swap(a, b, false, false);
  a = r[0];
  b = r[1];
}
template <int FMT>
__device__ __forceinline__ void block_sums(const f32x16 (&acc)[kRowsTM][kRowsTN],
                                           const u32x4 (&cw)[kRowsTN][kRowsTM / 2], float* dS, int O, int I, int G,
                                           int r0, int c0, int lane) {
  constexpr int kB = FMT == kMX ? 32 : 16, kSums = 128 / kB;  // per output feature
  const int shift = 16 * (lane >> 5);
  float s[kRowsTN][kSums];
#pragma unroll
  for (int j = 0; j < kRowsTN; ++j)
#pragma unroll
    for (int p = 0; p < kRowsTM / 2; ++p) {
      u32x4 c[2] = {cw[j][p], cw[j][p]};                      // of tiles 2 p and 2 p + 1, in every lane
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        uint32_t x = c[0][q], y = c[1][q];
        swap_halves(x, y);
        c[0][q] = x;
        c[1][q] = y;
      }
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        const int i = 2 * p + t;
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          const uint32_t w = c[t][q] >> shift;                // zeros outside the layer
          const f32x2 v01 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, 1.0f, 0);
          const f32x2 v23 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, 1.0f, 1);
          float& sum = s[j][FMT == kMX ? i : 2 * i + q / 2];
          if (q % (FMT == kMX ? 4 : 2) == 0) sum = 0.0f;
          sum = __builtin_fmaf(acc[i][j][4 * q + 0], v01[0], sum);
          sum = __builtin_fmaf(acc[i][j][4 * q + 1], v01[1], sum);
          sum = __builtin_fmaf(acc[i][j][4 * q + 2], v23[0], sum);
          sum = __builtin_fmaf(acc[i][j][4 * q + 3], v23[1], sum);
        }
      }
    }
  // both halves' sums: of output feature c0 + lane
  const int o = c0 + lane;
  float v[kSums];
#pragma unroll
  for (int b = 0; b < kSums; ++b) {
    uint32_t x = __float_as_uint(s[0][b]), y = __float_as_uint(s[1][b]);
    swap_halves(x, y);
    v[b] = __uint_as_float(x) + __uint_as_float(y);
  }
  const __amdgpu_buffer_rsrc_t rs = make_rsrc(dS, (uint32_t)((size_t)O * G * 4));
  const uint32_t at = o < O ? (uint32_t)(o * G + r0 / kB) * 4u : kOOB;
  if (r0 + 128 <= I) {
#pragma unroll
    for (int b = 0; b < kSums; b += 4) {
      const u32x4 w = {__float_as_uint(v[b]), __float_as_uint(v[b + 1]), __float_as_uint(v[b + 2]), __float_as_uint(v[b + 3])};
      __builtin_amdgcn_raw_buffer_store_b128(w, rs, (int)(at == kOOB ? kOOB : at + 4u * b), 0, 0);
    }
  } else {
#pragma unroll
    for (int b = 0; b < kSums; ++b)
      __builtin_amdgcn_raw_buffer_store_b32(__float_as_uint(v[b]), rs,
                                            (int)(at == kOOB || r0 + kB * b >= I ? kOOB : at + 4u * b), 0, 0);
  }
}

struct DsRowsArgs {
  const uint16_t* x;        // [Tx, I] bf16
  const int* rows;          // [N] or null
  const uint16_t* dy;       // [N, O]
  const uint8_t* codes;     // [E, O, I / 2]
  float* out;               // [E, O, G]
  const int* offsets;       // [E + 1]
  const int* order;         // [E] experts by falling number of rows
  int* taken;               // tiles taken from each of the 8 queues, kTakenStep apart
  int Tx, N, O, I, G, E;
  int parts;                // units of an expert: runs of tiles of equal number
};

// An expert's tiles are cut into `parts` units, and the units dealt to 8 queues
// (one per XCD, whose workgroups share an L2 and so an expert's operands) by
// falling number of rows, there and back: queue x holds units x, 15 - x, 16 + x,
// 31 - x, ...  A queue's tiles go one at a time to whichever of its workgroups is
// free, long experts first.
__device__ __forceinline__ int queue_unit(int i, int x) { return 16 * (i >> 1) + (i & 1 ? 15 - x : x); }
__device__ __forceinline__ int queue_units(int units, int x) {
  const int rem = units % 16;
  return 2 * (units / 16) + (x < rem) + (15 - x < rem);
}

template <int FMT, bool ROWS>
__global__ __launch_bounds__(512) void ds_rows_kernel(DsRowsArgs g) {
  constexpr int BM = kRowsBM, BN = kRowsBN, BK = kBK, NT = 512;
  constexpr int TM = kRowsTM, TN = kRowsTN;                   // a wave's 128 x 64 of 32 x 32 products
  constexpr int kA = BM * BK * 2, kB = BN * BK * 2;
  using DB = DmaNat<BN, NT, BK>;
  __shared__ __attribute__((aligned(16))) uint8_t lds[2 * (kA + kB)];
  __shared__ int s_next[4];
  __shared__ int s_expert[kQueueUnits], s_first[kQueueUnits], s_rows[kQueueUnits];   // of the queue's units

  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wm0 = (wave >> 2) * 128, wn0 = (wave & 3) * 64;
  const int O = g.O, I = g.I, G = g.G;
  const int tiles_m = (I + BM - 1) / BM, tiles_n = (O + BN - 1) / BN;
  const int per = tiles_m * tiles_n / g.parts;                // tiles of a unit

  // this workgroup's queue, and the first tile it takes from it
  const int queue = (int)blockIdx.x % kXcds, units = queue_units(g.E * g.parts, queue), end = per * units;
  const int first = (int)blockIdx.x / kXcds;
  if (first >= end) return;
  for (int i = tid; i < units; i += NT) {
    const int e = g.order[queue_unit(i, queue) / g.parts];
    const int a = min(max(g.offsets[e], 0), g.N);             // device data: held to the rows there are
    s_expert[i] = e;
    s_first[i] = a;
    s_rows[i] = min(max(g.offsets[e + 1], a), g.N) - a;
  }
  __syncthreads();

  // A tile: expert, corner.  A stage of one: the expert's rows [r0, r0 + n), stage
  // kt of nk; an expert without rows runs one stage of zeros, so its dS is 0.
  auto uniform = [](int v) { return __builtin_amdgcn_readfirstlane(v); };
  auto corner = [&](int pos, int i, int& m0, int& n0) {       // of a tile in the queue's unit i
    const int t = queue_unit(i, queue) % g.parts * per + (pos - i * per), tn = t / tiles_m;
    m0 = (t - tn * tiles_m) * BM;
    n0 = tn * BN;
  };
  struct Cursor {
    int pos = 0, m0 = 0, n0 = 0, r0 = 0, n = 0, kt = 0, nk = 1;
  };
  auto locate = [&](Cursor& c, int pos) {
    c.pos = pos;
    c.kt = 0;
    if (pos >= end) return;
    const int i = pos / per;
    corner(pos, i, c.m0, c.n0);
    c.r0 = uniform(s_first[i]);
    c.n = uniform(s_rows[i]);
    c.nk = c.n > 0 ? (c.n + BK - 1) / BK : 1;
  };

  // The wave copies 8 rows of a stage of x, two per instruction: this lane's half
  // meets rows half, 2 + half, 4 + half, 6 + half.  (A tile's columns past the
  // layer hold other values of x: they reach no sum that is stored.)
  const int half = lane >> 5;
  const __amdgpu_buffer_rsrc_t rrow = make_rsrc(g.rows, ROWS ? (uint32_t)g.N * 4u : 0u);
  uint32_t xrow[4] = {0u, 0u, 0u, 0u};
  auto load_rows = [&](const Cursor& c) {
    if constexpr (ROWS) {
      const int at = (c.r0 + c.kt * BK + 8 * wave + half) * 4;
#pragma unroll
      for (int q = 0; q < 4; ++q) xrow[q] = __builtin_amdgcn_raw_buffer_load_b32(rrow, at + 8 * q, 0, 0);
    }
  };
  const uint32_t row_bytes = (uint32_t)I * 2u, x_bytes = (uint32_t)((size_t)g.Tx * I * 2);
  uint32_t acol[4], boff[DB::kInst];                          // from the tile's corner
#pragma unroll
  for (int q = 0; q < 4; ++q) acol[q] = (uint32_t)(((lane & 31) ^ swz_nat<BM>(2 * q + half)) << 4);
#pragma unroll
  for (int q = 0; q < DB::kInst; ++q) {
    const int k = q * (NT / 32) + (tid >> 5);
    boff[q] = (uint32_t)k * (uint32_t)O * 2u + (uint32_t)(((lane & 31) ^ swz_nat<BN>(k)) << 4);
  }
  // The copy of the cursor's stage into buffer b, in 8 instructions; rows that
  // there are not read zeros, and past the last tile everything does.
  struct Copy {
    DmaRsrc ra, rb;
    SQ_LDS uint8_t* st;
    int left;
    uint32_t row;
  };
  auto copy_begin = [&](const Cursor& c, int b) {
    Copy k;
    const bool any = c.pos < end;
    const int row0 = c.kt * BK;
    k.st = (SQ_LDS uint8_t*)lds + b * (kA + kB);
    k.left = any ? c.n - row0 : 0;
    k.row = (uint32_t)(c.r0 + row0 + 8 * wave + half);
    const uint32_t skip = (uint32_t)c.m0 * 2u;
    k.ra = make_dma_rsrc(g.x + c.m0, any && x_bytes > skip ? x_bytes - skip : 0u);
    k.rb = make_dma_rsrc(g.dy + (size_t)(c.r0 + row0) * O + c.n0, k.left > 0 ? (uint32_t)(((size_t)k.left * O - c.n0) * 2) : 0u);
    return k;
  };
  auto copy_part = [&](const Copy& k, auto Q) {
    constexpr int q = decltype(Q)::value % 4;
    if constexpr (decltype(Q)::value < 4) {
      uint32_t r = ROWS ? xrow[q] : k.row + 2 * q;
      r = 8 * wave + 2 * q + half < k.left ? min(r, (uint32_t)g.Tx) : (uint32_t)g.Tx;
      dma16(k.ra, (SQ_LDS uint16_t*)k.st + (8 * wave + 2 * q) * BM, r * row_bytes + acol[q]);
    } else {
      dma16(k.rb, (SQ_LDS uint16_t*)(k.st + kA) + (q * (NT / 64) + wave) * 64 * 8, boff[q]);
    }
  };
  static_assert(DB::kInst == 4, "a stage's copy is 4 instructions of either operand");
  auto copy = [&](const Cursor& c, int b) {
    const Copy k = copy_begin(c, b);
    copy_part(k, std::integral_constant<int, 0>{});
    copy_part(k, std::integral_constant<int, 1>{});
    copy_part(k, std::integral_constant<int, 2>{});
    copy_part(k, std::integral_constant<int, 3>{});
    copy_part(k, std::integral_constant<int, 4>{});
    copy_part(k, std::integral_constant<int, 5>{});
    copy_part(k, std::integral_constant<int, 6>{});
    copy_part(k, std::integral_constant<int, 7>{});
  };

  f32x16 acc[TM][TN];
  struct Frag {
    bf16x8 a[TM];
    bf16x8 b[TN];
  };
  Frag F0, F1;
  // Where this lane's operands of slice 0 are in the present buffer (nat_frag's
  // two reads each; a later slice is a fixed distance on), moved to the other
  // buffer and back: one set of addresses for both.
  uint32_t at_a[TM][2], at_b[TN][2];
  {
    const int i = lane & 15, gr = lane >> 4;
    const int row = 8 * (gr >> 1) + (i >> 2), col = 16 * (gr & 1) + 4 * (i & 3);
    const uint32_t base = (uint32_t)reinterpret_cast<uintptr_t>((SQ_LDS uint8_t*)lds);
#pragma unroll
    for (int h = 0; h < 2; ++h) {
#pragma unroll
      for (int m = 0; m < TM; ++m) at_a[m][h] = base + 2u * (uint32_t)nat_off<BM>(row + 4 * h, wm0 + m * 32 + col);
#pragma unroll
      for (int n = 0; n < TN; ++n) at_b[n][h] = base + kA + 2u * (uint32_t)nat_off<BN>(row + 4 * h, wn0 + n * 32 + col);
    }
  }
  int flip = kA + kB;
  auto other_buffer = [&]() {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
#pragma unroll
      for (int m = 0; m < TM; ++m) at_a[m][h] += (uint32_t)flip;
#pragma unroll
      for (int n = 0; n < TN; ++n) at_b[n][h] += (uint32_t)flip;
    }
    flip = -flip;
  };
  auto frag = [&](const uint32_t (&at)[2], int off) {
    const v4i16 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((SQ_LDS v4i16*)(uintptr_t)(at[0] + off));
    const v4i16 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((SQ_LDS v4i16*)(uintptr_t)(at[1] + off));
    bf16x8 r;
    __builtin_memcpy(&r, &lo, 8);
    __builtin_memcpy(reinterpret_cast<char*>(&r) + 8, &hi, 8);
    return r;
  };
  auto read = [&](auto KK, Frag& f) {
    constexpr int kk = decltype(KK)::value;
#pragma unroll
    for (int i = 0; i < TM; ++i) f.a[i] = frag(at_a[i], kk * 16 * BM * 2);
#pragma unroll
    for (int j = 0; j < TN; ++j) f.b[j] = frag(at_b[j], kk * 16 * BN * 2);
  };
  auto mma = [&](Frag& f) {
#pragma unroll
    for (int i = 0; i < TM; ++i)
#pragma unroll
      for (int j = 0; j < TN; ++j)
        acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(f.a[i], f.b[j], acc[i][j], 0, 0, 0);
  };
  auto mma_first = [&](Frag& f) {                             // a tile's first products: its sums start here
    const f32x16 zero = {};
#pragma unroll
    for (int i = 0; i < TM; ++i)
#pragma unroll
      for (int j = 0; j < TN; ++j) acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(f.a[i], f.b[j], zero, 0, 0, 0);
  };
  using I0 = std::integral_constant<int, 0>;
  using I1 = std::integral_constant<int, 1>;
  using I2 = std::integral_constant<int, 2>;
  using I3 = std::integral_constant<int, 3>;

  // Tiles are taken two ahead of the copies' present one: by the first wave, at
  // the start of the step after the one that needed the last, so that the answer
  // comes with the step's own wait; it goes to the others through LDS behind the
  // next barrier, four places in turn.  The first two come from the grid.
  int taken = 0, got = 0;                                     // tiles asked for; the answer
  bool ask = false;
  auto next_tile = [&]() { return uniform(*((volatile SQ_LDS int*)s_next + (taken & 3))); };

  // Copies go two stages ahead of the products; what stage they reached is kept
  // in turn for the products: tile (end or more: none) and whether it is its last.
  Cursor cd;
  locate(cd, first);
  if (tid == 0) {
    s_next[0] = first + kCUs / kXcds;
    s_next[1] = atomicAdd(g.taken + queue * kTakenStep, 1);
  }
  load_rows(cd);
  copy(cd, 0);
  int pos0 = cd.pos, pos1 = end, pos2 = end;
  bool last0 = ++cd.kt == cd.nk, last1 = false, last2 = false;
  __syncthreads();
  if (last0) {
    locate(cd, next_tile());
    ++taken;
    ask = true;
  }
  if (cd.pos < end) {
    load_rows(cd);
    copy(cd, 1);
    pos1 = cd.pos;
    last1 = ++cd.kt == cd.nk;
  }
  wait_vm_lgkm0<0>();
  __builtin_amdgcn_s_barrier();
  __builtin_amdgcn_sched_barrier(0);
  if (last1) {
    if (ask && tid == 0) s_next[2] = atomicAdd(g.taken + queue * kTakenStep, 1);   // two tiles of one stage each
    __syncthreads();
    locate(cd, next_tile());
    ++taken;
    ask = true;
  }
  int cur = 0;
  bool fresh = true;
  read(I0{}, F0);
  // one stage a turn, its first slice already in F0
  for (;;) {
    if (ask && tid == 0) got = atomicAdd(g.taken + queue * kTakenStep, 1);
    if (cd.pos < end) load_rows(cd);
    // a tile's codes come with its last stage, so that this step's wait is theirs
    u32x4 cw[TN][TM / 2];
    int e = 0, m0 = 0, n0 = 0;
    if (last0) {
      const int i = pos0 / per;
      e = uniform(s_expert[i]);
      corner(pos0, i, m0, n0);
      load_code_pairs(cw, g.codes + (size_t)e * O * (I / 2), O, I, m0 + wm0, n0 + wn0, lane);
    }
    read(I1{}, F1);
    if (fresh) mma_first(F0);
    else mma(F0);
    read(I2{}, F0);
    mma(F1);
    read(I3{}, F1);
    mma(F0);
    wait_vm_lgkm0<0>();
    __builtin_amdgcn_s_barrier();
    __builtin_amdgcn_sched_barrier(0);
    other_buffer();
    if (!last0) read(I0{}, F0);
    // the last slice's products, an instruction of the copy after each
    const Copy k = copy_begin(cd, cur);
    auto both = [&](auto Q) {
      constexpr int m = decltype(Q)::value;
      acc[m / TN][m % TN] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(F1.a[m / TN], F1.b[m % TN], acc[m / TN][m % TN], 0, 0, 0);
      copy_part(k, Q);
    };
    both(std::integral_constant<int, 0>{});
    both(std::integral_constant<int, 1>{});
    both(std::integral_constant<int, 2>{});
    both(std::integral_constant<int, 3>{});
    both(std::integral_constant<int, 4>{});
    both(std::integral_constant<int, 5>{});
    both(std::integral_constant<int, 6>{});
    both(std::integral_constant<int, 7>{});
    pos2 = cd.pos;
    last2 = cd.pos < end && ++cd.kt == cd.nk;
    if (ask && tid == 0) *((volatile SQ_LDS int*)s_next + ((taken + 1) & 3)) = got;
    ask = last2;
    if (last2) {
      locate(cd, next_tile());
      ++taken;
    }
    if (last0) {
      block_sums<FMT>(acc, cw, g.out + (size_t)e * O * G, O, I, G, m0 + wm0, n0 + wn0, lane);
      if (pos1 >= end) break;
      read(I0{}, F0);
    }
    fresh = last0;
    pos0 = pos1;
    pos1 = pos2;
    last0 = last1;
    last1 = last2;
    cur ^= 1;
  }
  wait_vm_lgkm0<0>();
}

// What the product needs, in one launch: x unpacked (kActSteps * 256 pieces per
// workgroup) and, in the last workgroup, the experts' order and the queues'
// counts (the workgroups' first two tiles are taken).  More than 1024 experts, whose
// order would take too long here, keep their own.
template <int ACT>
__global__ __launch_bounds__(256) void ds_rows_prepare_kernel(const u32x2* __restrict__ codes,
                                                              const uint8_t* __restrict__ scales, int64_t pieces,
                                                              u32x4* __restrict__ X, const int* __restrict__ offsets,
                                                              int E, int workgroups, int* __restrict__ order,
                                                              int* __restrict__ taken) {
  if (blockIdx.x + 1 < gridDim.x) {
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
    return;
  }
  const int tid = threadIdx.x;
  if (tid < kXcds) taken[tid * kTakenStep] = 2 * (workgroups / kXcds);
  if (E > 1024) {
    for (int e = tid; e < E; e += 256) order[e] = e;
    return;
  }
  __shared__ int s_n[1024];
  for (int e = tid; e < E; e += 256) s_n[e] = offsets[e + 1] - offsets[e];
  __syncthreads();
  for (int e = tid; e < E; e += 256) {
    const int n = s_n[e];
    int rank = 0;
    for (int o = 0; o < E; ++o) rank += s_n[o] > n || (s_n[o] == n && o < e);
    order[rank] = e;
  }
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
  const int ext = large ? 256 : 128;
  const dim3 grid((unsigned)((g.I + ext - 1) / ext * ((g.O + ext - 1) / ext) * g.groups)), block(512);
  if (large) hipLaunchKernelGGL((ds8_tile_kernel<FMT, ACT, 256, 256, 2, 4>), grid, block, 0, s, g);
  else hipLaunchKernelGGL((ds8_tile_kernel<FMT, ACT, 128, 128, 2, 4>), grid, block, 0, s, g);
  return ok();
}

int ds8_launch(int fmt, int act, bool large, const Ds8Args& g, hipStream_t s) {
  if (fmt == kMX) return act == kInt8 ? ds8_go<kMX, kInt8>(g, large, s) : ds8_go<kMX, kE4M3>(g, large, s);
  return act == kInt8 ? ds8_go<kNV, kInt8>(g, large, s) : ds8_go<kNV, kE4M3>(g, large, s);
}

template <int FMT>
int ds_rows_go(const DsRowsArgs& g, hipStream_t s) {
  static_assert(kCUs % kXcds == 0, "as many workgroups for every queue");
  if (g.rows) hipLaunchKernelGGL((ds_rows_kernel<FMT, true>), dim3(kCUs), dim3(512), 0, s, g);
  else hipLaunchKernelGGL((ds_rows_kernel<FMT, false>), dim3(kCUs), dim3(512), 0, s, g);
  return ok();
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

// Layers of many outputs meet each row of x^ in many tiles, and each of them would
// turn its 8 bits into bf16: beyond 2048 outputs, once the product is long enough
// to pay for another launch (some 20 us), x^ goes through the workspace in bf16 to
// the bf16 product.  MXFP4, us, tiles from 8 bits (int8, E4M3) against x^ first:
// 8192 tokens, 14336 x 4096: 855, 799 against 730, 726; 512 tokens of it: 73, 69
// against 65, 65; 4096 tokens, 4096 x 4096: 116, 110 against 108, 108.  And where
// the rule keeps the tiles: 8192 tokens, 2048 x 4096: 118, 112 against 119, 119;
// 512 tokens, 4096 x 4096: 20, 19 against 23, 22.
bool ds8_unpacks(int T, int O, int I) {
  return O > 2048 && (int64_t)T * O >= int64_t(24000000000) / I;
}

}  // namespace

int act_pack_launch(int act, int64_t T, int64_t I, const void* X, uint8_t* codes, uint8_t* scales, hipStream_t s) {
  const int64_t pieces = T * I / 8, blocks = (pieces + 256 * kActSteps - 1) / (256 * kActSteps);
  const u32x4* x = static_cast<const u32x4*>(X);
  auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, dim3((unsigned)blocks), dim3(256), 0, s, x, pieces, codes, scales); };
  const bool stream = T * I * 2 >= kActStreamBytes;
  if (act == kInt8) stream ? go(act_pack_kernel<kInt8, true>) : go(act_pack_kernel<kInt8, false>);
  else stream ? go(act_pack_kernel<kE4M3, true>) : go(act_pack_kernel<kE4M3, false>);
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
  if (ds8_unpacks(T, O, I)) return (size_t)T * I * 2 + gemm_dscale_workspace(fmt, T, O, I);   // I % 32 == 0
  const int splits = ds8_splits(T, O, I);
  return splits < 2 ? 0 : (size_t)splits * O * (I / (fmt == kMX ? 32 : 16)) * sizeof(float);
}

int dscale_act8(int fmt, int act, int T, int O, int I, const uint8_t* x, const uint8_t* xs, const void* dY,
                const uint8_t* codes, float* dS, void* workspace, hipStream_t s) {
  if (ds8_unpacks(T, O, I)) {
    if (act_unpack_launch(act, T, I, x, xs, workspace, s) != 0) return -1;
    return gemm_dscale(fmt, T, O, I, workspace, dY, codes, dS, static_cast<uint8_t*>(workspace) + (size_t)T * I * 2, s);
  }
  Ds8Args g{};
  g.x = x; g.xs = xs; g.dy = static_cast<const uint16_t*>(dY); g.codes = codes;
  g.N = T; g.O = O; g.I = I; g.G = I / (fmt == kMX ? 32 : 16);
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

// x in bf16, the order, the queues' counts
size_t dscale_act8_batched_workspace(int E, int T, int I) {
  return (size_t)T * I * 2 + (size_t)((E + 3) / 4) * 16 + kXcds * kTakenStep * 4;
}

int dscale_act8_batched(int fmt, int act, int E, int Tx, int N, int O, int I, const uint8_t* x, const uint8_t* xs,
                        const int32_t* rows, const int32_t* offsets, const void* dY, const uint8_t* codes, float* dS,
                        void* workspace, hipStream_t s) {
  uint8_t* ws = static_cast<uint8_t*>(workspace);
  u32x4* xb = reinterpret_cast<u32x4*>(ws);
  int* order = reinterpret_cast<int*>(ws + (size_t)Tx * I * 2);
  int* taken = order + (E + 3) / 4 * 4;
  const int64_t pieces = (int64_t)Tx * I / 8;
  const dim3 grid((unsigned)((pieces + 256 * kActSteps - 1) / (256 * kActSteps) + 1));
  const u32x2* c = reinterpret_cast<const u32x2*>(x);
  if (act == kInt8)
    hipLaunchKernelGGL((ds_rows_prepare_kernel<kInt8>), grid, dim3(256), 0, s, c, xs, pieces, xb, offsets, E, kCUs, order, taken);
  else
    hipLaunchKernelGGL((ds_rows_prepare_kernel<kE4M3>), grid, dim3(256), 0, s, c, xs, pieces, xb, offsets, E, kCUs, order, taken);
  if (ok() != 0) return -1;
  DsRowsArgs g{};
  g.x = reinterpret_cast<const uint16_t*>(xb); g.rows = N > 0 ? rows : nullptr;
  g.dy = static_cast<const uint16_t*>(dY); g.codes = codes; g.out = dS; g.offsets = offsets;
  g.order = order; g.taken = taken;
  g.Tx = Tx; g.N = N; g.O = O; g.I = I; g.G = I / (fmt == kMX ? 32 : 16); g.E = E;
  // enough units that the queues come out even: the smallest divisor of an
  // expert's tiles that gives 64 in all
  const int tiles = (I + kRowsBM - 1) / kRowsBM * ((O + kRowsBN - 1) / kRowsBN);
  g.parts = 1;
  while (g.parts < tiles && (tiles % g.parts != 0 || E * g.parts < 64)) ++g.parts;
  if ((int64_t)E * g.parts > 8192) g.parts = 1;               // the queues' lists
  return fmt == kMX ? ds_rows_go<kMX>(g, s) : ds_rows_go<kNV>(g, s);
}

}  // namespace sq
