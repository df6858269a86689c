// Softmax cross entropy of a language-model head over its whole vocabulary and
// the gradient of the head's input; large products' logits never reach memory.
//
//   l[t,v]  = X[t] . W[v]                       W bf16, or codes x scales
//   lse[t]  = log sum_v exp l[t,v]              loss[t] = lse[t] - l[t,y_t]
//   dX[t]   = dloss[t] sum_v (exp(l[t,v] - lse[t]) - [v = y_t]) W[v]
//
// Forward: tiles of the logits (256 rows of W by the tokens) leave only each
// token's maximum and sum of exponentials over the tile; a second kernel joins
// them.  Backward: pieces of the vocabulary; a piece's logits are formed again
// and leave as bf16 gradients of the logits, [tokens, piece], which the next
// product contracts with the same rows of W into fp32 sums.  Up to 4096 tokens
// an MXFP4 head of whole 512s is read as codes by all three products; other 4-bit heads' pieces are written
// out as bf16 before they are used (code x scale is exact in bf16; NVFP4's ws2 goes
// to the fp32 sums).
//
// Few tiles, whose sums are split, and a 4-bit head of few tokens, read by the
// layer's own products, pass fp32 logits through the workspace instead.
//
// Rows without a target in the vocabulary cost nothing beyond 256 tokens: the
// rows that have one are numbered first, and tiles past the last of them end at
// once.  The number stays on the device.
//
// The three products bound it (the forward's logits, the same again, dX), and the
// matrix cores' power bounds them: 4096 tokens of 131072 x 4096 bf16 10.0-10.6 ms,
// 1.24-1.32 PFLOP/s; 1999 tokens, 40% of them ignored, of 50001 x 4096 MXFP4 1.27 ms.
// One token of 131072 x 4096 bf16 takes 538 us, three reads of the head at 6.0 TB/s,
// of MXFP4 226.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <type_traits>

#include "sq_device.h"
#include "sq_gemm_args.h"
#include "sq_launch.h"
#include "sq_tiles.h"

namespace sq {

namespace {

constexpr float kLog2E = 1.44269504f;
constexpr int kCeGroup = 4;             // tile rows per group of the tile order

__device__ __forceinline__ int64_t target_at(const void* y, int bytes, int64_t t) {
  return bytes == 8 ? static_cast<const int64_t*>(y)[t] : (int64_t)static_cast<const int32_t*>(y)[t];
}

// fp32 of the low or high half of a pair of bf16.
__device__ __forceinline__ float bf16_half(uint32_t pair, int high) {
  return __uint_as_float(high ? pair & 0xFFFF0000u : pair << 16);
}

// ------------------------------------------------------------------ rows
// rows[0 .. n) = the tokens whose target is in the vocabulary, in order; *count
// = n.  One workgroup: 1024 tokens per step.
__global__ __launch_bounds__(1024) void ce_rows_kernel(const void* __restrict__ y, int y_bytes, int T, int64_t V,
                                                       int* __restrict__ count, int* __restrict__ rows) {
  __shared__ int s_n[16];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  int base = 0;
  for (int t0 = 0; t0 < T; t0 += 1024) {
    const int t = t0 + (int)threadIdx.x;
    bool in = false;
    if (t < T) {
      const int64_t v = target_at(y, y_bytes, t);
      in = v >= 0 && v < V;
    }
    const uint64_t b = __ballot(in);
    if (lane == 0) s_n[wave] = __popcll(b);
    __syncthreads();
    int at = base, all = 0;
#pragma unroll
    for (int w = 0; w < 16; ++w) {
      at += w < wave ? s_n[w] : 0;
      all += s_n[w];
    }
    if (in) rows[at + __builtin_amdgcn_mbcnt_hi((uint32_t)(b >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)b, 0))] = t;
    base += all;
    __syncthreads();
  }
  if (threadIdx.x == 0) *count = base;
}

// ------------------------------------------------------------------ 4-bit heads
// Rows [v0, v0 + n) of the head as bf16, 8 codes per lane.
template <int FMT>
__global__ __launch_bounds__(256) void ce_dequant_kernel(const uint8_t* __restrict__ codes,
                                                         const uint8_t* __restrict__ scales, int64_t first, int64_t items,
                                                         uint16_t* __restrict__ out) {
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (i >= items) return;
  const uint32_t w = reinterpret_cast<const uint32_t*>(codes)[first + i];
  const uint32_t b = scales[(first + i) / (ScaleOperand<FMT>::kBlock / 8)];
  reinterpret_cast<uint4*>(out)[i] = ScaleOperand<FMT>::dequant8(w, ScaleOperand<FMT>::of(b));
}

// ------------------------------------------------------------------ products
struct CeArgs {
  const uint16_t* x;        // X [T, H]
  const uint16_t* w;        // rows [v0, v0 + Vn) of W as bf16, [Vn, H] (with CODES their MXFP4 codes)
  const uint8_t* scales;    // with CODES: their scales
  uint16_t* d;              // gradients of the logits [T, ld], piece columns
  float* part;              // forward: (max, sum) [tile of all of W][T]
  float* tlogit;            // forward: the target's logit [T]; backward: what rounding took from its gradient
  float* sums;              // backward: fp32 sums of dX, planes of [live rows in whole tiles, H]
  const int* rows;          // compact row -> token, or null (row = token)
  const int* count;         // live rows, or null (T)
  const void* y;
  const float* lse;
  const float* dloss;
  int64_t v0;               // first row of W of this piece
  int64_t V;
  int T, H, Vn, ld;
  int y_bytes;
  int part_tile0;           // forward: tile of all of W that this piece starts at
  int split_stages;         // backward: 64-row stages of a whole piece
  int add;                  // backward: the sums hold earlier pieces
  float* logits;            // fp32 planes [splits][T][ldl] of a head of few tiles
  int ldl, splits;
  float ws2;
};

// K-contiguous rows picked by number: as DmaKC, with row r0 + r of the tile at
// row rows[r0 + r] of the matrix.
template <int R, int NT>
struct DmaRows {
  static constexpr int kInst = R / 8 / (NT / 64);
  static_assert(kInst * (NT / 64) * 8 == R, "tile rows must split over the waves");
  uint32_t off[kInst];
  int klim[kInst];
  __device__ __forceinline__ void init(int ld, int live, int kdim, int r0, int tid, const int* rows) {
    const int wave = tid >> 6, lane = tid & 63;
#pragma unroll
    for (int q = 0; q < kInst; ++q) {
      const int r = (q * (NT / 64) + wave) * 8 + (lane >> 3);
      const int c = (lane & 7) ^ swz_kc(r);
      const int gr = r0 + r;
      off[q] = kOOB;
      if (gr < live) off[q] = ((uint32_t)(rows ? rows[gr] : gr) * (uint32_t)ld + (uint32_t)c * 8u) * 2u;
      klim[q] = kdim - c * 8;
    }
  }
  template <int Q0, int Q1>
  __device__ __forceinline__ void issue_part(DmaRsrc rs, SQ_LDS uint16_t* s, int k0, int wave) const {
#pragma unroll
    for (int q = Q0; q < Q1; ++q) {
      const uint32_t o = off[q] == kOOB || k0 >= klim[q] ? kOOB : off[q] + (uint32_t)k0 * 2u;
      dma16(rs, s + (q * (NT / 64) + wave) * 8 * kBK, o);
    }
  }
};

// The copies of a 4-bit tile of R = NT / 2 rows, two 16-byte chunks each: 64 codes
// of a row and stage, chunk c of row r at place c ^ (r / 8 & 1) (a wave's reads of 8
// codes then meet each bank twice at most), or 32 scales of a row.
template <int NT, bool SCALES>
struct DmaPairs {
  static constexpr int kInst = 1;
  uint32_t off;
  int chunk;
  __device__ __forceinline__ void init(int row_bytes, int live, int tid) {
    const int r = tid >> 1;
    chunk = SCALES ? tid & 1 : (tid & 1) ^ ((r >> 3) & 1);
    off = r < live ? (uint32_t)r * (uint32_t)row_bytes + 16u * (uint32_t)chunk : kOOB;
  }
  // the 32 bytes of every row from byte `first` on; past the row's end zeros
  __device__ __forceinline__ void issue(DmaRsrc rs, SQ_LDS uint8_t* s, int first, int row_bytes, int wave) const {
    dma16(rs, s + wave * 1024, off == kOOB || first + 16 * chunk >= row_bytes ? kOOB : off + (uint32_t)first);
  }
};

// Split of the vocabulary rows of dX's contraction over workgroups: few tiles as often
// as they go into the CUs (at least 4 stages each); tiles that would leave the last
// round of the CUs poorly filled up to 6 times, by the time of the rounds and of the
// planes (tenths of us: 16 a stage, 1 a tile's plane).  4097 tokens of 131072 x 2048
// make 136 tiles: the gradient with one split 4.92 ms, with 5 4.39 (bf16).
constexpr int kCeMostGroups = 768;      // tiles times splits, where there are splits
__host__ __device__ inline int ce_splits(int tiles, int stages) {
  const int most = stages / 4;
  if (tiles < 1 || most < 2 || 2 * tiles > kCeMostGroups) return 1;
  if (3 * tiles <= kCUs) {
    const int n = kCUs / tiles < most ? kCUs / tiles : most;
    return n < 64 ? n : 64;
  }
  int best = 1, least = 0x7FFFFFFF;
#pragma unroll                            // divisions by constants: every workgroup works this out
  for (int s = 1; s <= 6; ++s) {
    if (s > most || s * tiles > kCeMostGroups) continue;
    const int cost = (s * tiles + kCUs - 1) / kCUs * (int)((unsigned)(stages + s - 1) / s) * 16 + s * tiles;
    if (cost < least) {
      least = cost;
      best = s;
    }
  }
  return best;
}

enum CeMode { kCeStats = 0, kCeGrad = 1, kCeDx = 2, kCeLogits = 3 };

// f(0), f(1), .. with constants, in this order.
template <int... N, typename F>
__device__ __forceinline__ void for_each(std::integer_sequence<int, N...>, F f) {
  (f(std::integral_constant<int, N>{}), ...);
}

// The tile product of them all, 256 x BN (logits: W's rows by tokens, so that
// a lane holds one token's logits and sums them without its neighbours) or BM x
// 256 (dX: tokens by columns of W).  64-deep stages copied global -> LDS, four
// 16-deep slices each.  The chip's power bounds it: what counts is that the matrix
// cores, at whatever clock is left, do not wait.  With a slice's reads and copies
// in a row and the barrier between two slices the products of 4096 tokens with
// 131072 x 4096 bf16 took 3.50 (statistics), 3.66 (gradients) and 3.45 ms (dX);
// in this order 3.27, 3.47 and 3.21.  4 waves of 128 x 128 instead of 8 (a third
// fewer LDS reads) took 3.44 ms and, in dX, 3.26: one wave per SIMD cannot overlap
// its exponentials.  Stages of 32 with up to 5 in LDS were 8% slower.
template <int MODE, int BM, int BN, int WGM, int WGN, int STAGES, bool CODES = false>
__global__ __launch_bounds__(64 * WGM * WGN) void ce_kernel(CeArgs g) {
  constexpr int NT = 64 * WGM * WGN;
  constexpr int WM = BM / WGM, WN = BN / WGN;
  constexpr int TM = WM / 32, TN = WN / 32;
  constexpr int kA = CODES && MODE != kCeDx ? BM * kBK / 2 : BM * kBK * 2, kB = BN * kBK * 2, kStage = kA + kB, kSlices = kBK / 16;
  constexpr bool kDxMode = MODE == kCeDx;
  constexpr int kGroup = 16;                                  // stages of a row's 32 scales
  constexpr bool kRowCodes = CODES && !kDxMode;               // W's codes through LDS
  using DA = std::conditional_t<kRowCodes, DmaPairs<NT, false>, DmaKC<BM, NT>>;
  using DB = std::conditional_t<kDxMode, DmaNat<BN, NT, kBK>, DmaRows<BN, NT>>;
  constexpr bool kItems = kDxMode && CODES;                   // W's codes through registers
  constexpr int kDmaB = kItems ? 0 : DB::kInst;
  constexpr int kDma = DA::kInst + kDmaB;
  // with CODES a stage is published a step before it is multiplied: its codes become
  // operands in the vector units meanwhile
  constexpr int kAhead = kItems ? 0 : (STAGES - (CODES ? 3 : 2)) * kDma;
  static_assert(!kRowCodes || (MODE != kCeLogits && BM == NT / 2 && STAGES == 3), "4-bit tiles");
  static_assert(!kItems || (BN == 256 && NT == 512 && STAGES == 2), "an item of 32 columns per thread");
  static_assert(STAGES >= 2 && STAGES <= 3 && kAhead < 63, "stages");
  __shared__ __attribute__((aligned(16))) uint8_t lds[STAGES * kStage + (kRowCodes ? 2 * BM * 32 : 0)];

  const int tid = threadIdx.x;
  const int lane = tid & 63, wave = tid >> 6;
  const int wave_u = __builtin_amdgcn_readfirstlane(wave);
  const int wm0 = (wave / WGN) * WM, wn0 = (wave % WGN) * WN;
  const int live = g.count ? min(*g.count, g.T) : g.T;

  // tile, and the stages [s_first, s_first + nk) of its contraction
  const int M = kDxMode ? live : g.Vn, N = kDxMode ? g.H : live, K = kDxMode ? g.Vn : g.H;
  const int tiles_m = (M + BM - 1) / BM, tiles_n = (N + BN - 1) / BN, tiles = tiles_m * tiles_n;
  const int splits = kDxMode ? ce_splits(tiles, g.split_stages) : MODE == kCeLogits ? g.splits : 1;
  if ((int)blockIdx.x >= tiles * splits) return;
  const int pos = xcd_stretch((int)blockIdx.x, tiles * splits);
  const int split = kDxMode || MODE == kCeLogits ? pos / tiles : 0;
  int tm, tn;
  tile_at<kCeGroup>(pos - split * tiles, tiles_m, tiles_n, tm, tn);
  const int m0 = tm * BM, n0 = tn * BN;
  const int nk_all = (K + kBK - 1) / kBK;
  const int per = (nk_all + splits - 1) / splits;
  const int s_first = min(split * per, nk_all), nk = min(per, nk_all - s_first);

  DmaRsrc ra, rb;
  DA dA;
  DB dB;
  if constexpr (kDxMode) {
    ra = make_dma_rsrc(g.d + (size_t)m0 * g.ld, (uint32_t)((size_t)min(BM, M - m0) * g.ld * 2));
    if constexpr (!kItems)
      rb = make_dma_rsrc(g.w + (size_t)s_first * kBK * g.H, (uint32_t)((size_t)(K - min(s_first * kBK, K)) * g.H * 2));
    dA.init(g.ld, min(BM, M - m0), g.ld, 0, tid);
    if constexpr (!kItems) dB.init(g.H, g.H, n0, tid);
  } else if constexpr (kRowCodes) {
    ra = make_dma_rsrc(reinterpret_cast<const uint8_t*>(g.w) + (size_t)m0 * (g.H / 2), (uint32_t)(min(BM, M - m0) * (g.H / 2)));
    rb = make_dma_rsrc(g.x, (uint32_t)((size_t)g.T * g.H * 2));
    dA.init(g.H / 2, min(BM, M - m0), tid);
    dB.init(g.H, live, g.H, n0, tid, g.rows);
  } else {
    ra = make_dma_rsrc(g.w + (size_t)m0 * g.H, (uint32_t)((size_t)min(BM, M - m0) * g.H * 2));
    rb = make_dma_rsrc(g.x, (uint32_t)((size_t)g.T * g.H * 2));
    dA.init(g.H, min(BM, M - m0), g.H, 0, tid);
    dB.init(g.H, live, g.H, n0, tid, g.rows);
  }

  // What the epilogue needs of this lane's tokens, a chain of loads that would hold
  // it up: whether they have a target (bit j of `has`), where in the lane's registers
  // it is, if there, and their loss's gradient and lse.
  const int vrow = m0 + wm0 + 4 * (lane >> 5);               // first row of W of this lane's registers
  uint32_t has = 0;
  int own[TN];
  float c_of[TN], z_of[TN];
  if constexpr (MODE == kCeStats || MODE == kCeGrad) {
    int t[TN];
    int64_t y[TN];
#pragma unroll
    for (int j = 0; j < TN; ++j) {
      const int row = n0 + wn0 + j * 32 + (lane & 31);
      t[j] = row < live ? g.rows ? g.rows[row] : row : -1;
    }
#pragma unroll
    for (int j = 0; j < TN; ++j) y[j] = t[j] >= 0 ? target_at(g.y, g.y_bytes, t[j]) : -1;
#pragma unroll
    for (int j = 0; j < TN; ++j) {
      const bool valid = y[j] >= 0 && y[j] < g.V;
      // the target's row counted from this lane's first, if this lane holds it
      const int64_t off = y[j] - g.v0 - vrow;
      own[j] = valid && off >= 0 && off < WM && (off & 4) == 0 ? (int)off : -1;
      has |= (uint32_t)valid << j;
      if constexpr (MODE == kCeGrad) {
        c_of[j] = valid ? g.dloss[t[j]] : 0.0f;
        z_of[j] = valid ? g.lse[t[j]] : 0.0f;
      }
    }
  }

  f32x16 acc[TM][TN];
  float* sums = nullptr;
  if constexpr (kDxMode) {
    // this split's plane of the live rows; earlier pieces' sums are carried on
    sums = g.sums + (size_t)split * tiles_m * BM * g.H;
#pragma unroll
    for (int i = 0; i < TM; ++i)
#pragma unroll
      for (int j = 0; j < TN; ++j) {
        const int col = n0 + wn0 + j * 32 + (lane & 31);
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          const int row = m0 + wm0 + i * 32 + 8 * (r >> 2) + 4 * (lane >> 5) + (r & 3);
          acc[i][j][r] = g.add && col < g.H ? sums[(size_t)row * g.H + col] : 0.0f;
        }
      }
  } else {
#pragma unroll
    for (int i = 0; i < TM; ++i)
#pragma unroll
      for (int j = 0; j < TN; ++j)
#pragma unroll
        for (int r = 0; r < 16; ++r) acc[i][j][r] = 0.0f;
  }

  auto stage_at = [&](auto S) { return (SQ_LDS uint8_t*)lds + decltype(S)::value * kStage; };
  using I0 = std::integral_constant<int, 0>;
  using I1 = std::integral_constant<int, 1>;

  // copy N of half HALF of stage kt into buffer S; what lies past the matrix reads
  // as zeros, so the copies need no condition on kt
  auto dma = [&](auto S, int kt, auto HALF, auto N) {
    constexpr int h = decltype(HALF)::value, n = decltype(N)::value;
    constexpr int a0 = h ? DA::kInst / 2 : 0, an = h ? DA::kInst - a0 : DA::kInst / 2, b0 = h ? kDmaB / 2 : 0;
    const int ka = (s_first + kt) * kBK;
    if constexpr (n < an) {
      if constexpr (kRowCodes) dA.issue(ra, stage_at(S), ka / 2, g.H / 2, wave_u);
      else dA.template issue_part<a0 + n, a0 + n + 1>(ra, (SQ_LDS uint16_t*)stage_at(S), ka, false, wave_u);
    } else {
      SQ_LDS uint16_t* b = (SQ_LDS uint16_t*)(stage_at(S) + kA);
      constexpr int q = b0 + n - an;
      if constexpr (kDxMode)
        dB.template issue_part<q, q + 1>(rb, b, (uint32_t)(kt * kBK) * (uint32_t)g.H * 2u, wave_u);
      else
        dB.template issue_part<q, q + 1>(rb, b, ka, wave_u);
    }
  };
  constexpr int kHalf[2] = {DA::kInst / 2 + kDmaB / 2, kDma - DA::kInst / 2 - kDmaB / 2};
  auto dma_half = [&](auto S, int kt, auto HALF) {
    for_each(std::make_integer_sequence<int, kHalf[decltype(HALF)::value]>{}, [&](auto N) { dma(S, kt, HALF, N); });
  };

  // A slice's operands, and its products and reads in the order in which each needs
  // the fewest before it: a0 b0 b1 .. a1 .., products row by row.
  struct Frag {
    bf16x8 a[TM];
    bf16x8 b[TN];
  };
  Frag F0, F1;
  constexpr int kReads = TM + TN, kProducts = TM * TN, kMid = kProducts / 2, kRest = kProducts - kMid;
  auto read = [&](auto S, auto KK, Frag& f, auto N) {
    constexpr int n = decltype(N)::value, kk = decltype(KK)::value;
    const int chunk = 2 * kk + (lane >> 5);
    if constexpr (n == 0 || n > TN) {
      static_assert(!kRowCodes, "operands from codes are converted");
      constexpr int i = n == 0 ? 0 : n - TN;
      f.a[i] = *(const SQ_LDS bf16x8*)((const SQ_LDS uint16_t*)stage_at(S) + kc_off(wm0 + i * 32 + (lane & 31), chunk));
    } else {
      constexpr int j = n - 1;
      const SQ_LDS uint16_t* b = (const SQ_LDS uint16_t*)(stage_at(S) + kA);
      if constexpr (kDxMode) f.b[j] = nat_frag<BN>(b, kk, wn0 + j * 32, lane);
      else f.b[j] = *(const SQ_LDS bf16x8*)(b + kc_off(wn0 + j * 32 + (lane & 31), chunk));
    }
  };
  auto product = [&](Frag& f, auto N) {
    constexpr int i = decltype(N)::value / TN, j = decltype(N)::value % TN;
    acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(f.a[i], f.b[j], acc[i][j], 0, 0, 0);
  };
  // CODES: this lane's codes and scales of a stage, 8 codes per row tile and slice,
  // and the operand made of them
  DmaPairs<NT, true> dS;
  DmaRsrc rscale;
  uint32_t cw[TM][4], sc[TM];
  SQ_LDS uint8_t* const scales = (SQ_LDS uint8_t*)lds + STAGES * kStage;
  if constexpr (kRowCodes) {
    rscale = make_dma_rsrc(g.scales + (size_t)m0 * (g.H / 32), (uint32_t)(min(BM, M - m0) * (g.H / 32)));
    dS.init(g.H / 32, min(BM, M - m0), tid);
  }
  auto dma_scales = [&](int group) { dS.issue(rscale, scales + (group & 1) * (BM * 32), group * 32, g.H / 32, wave_u); };
  auto read_codes = [&](auto S, int kt, auto I) {
    constexpr int i = decltype(I)::value;
    const int row = wm0 + i * 32 + (lane & 31), swap = (lane >> 3) & 1;
#pragma unroll
    for (int c = 0; c < 2; ++c) {
      const SQ_LDS uint32_t* p = (const SQ_LDS uint32_t*)(stage_at(S) + row * 32 + (c ^ swap) * 16 + (lane >> 5) * 4);
      cw[i][2 * c] = p[0];
      cw[i][2 * c + 1] = p[2];
    }
    sc[i] = *(const SQ_LDS uint16_t*)(scales + ((kt / kGroup) & 1) * (BM * 32) + row * 32 + kt % kGroup * 2);
  };
  auto convert = [&](Frag& f, auto KK, auto I) {
    constexpr int i = decltype(I)::value, kk = decltype(KK)::value;
    const uint4 v = ScaleOperand<kMX>::dequant8(cw[i][kk], ScaleOperand<kMX>::of((sc[i] >> (kk >= 2 ? 8 : 0)) & 0xFFu));
    f.a[i] = __builtin_bit_cast(bf16x8, v);
  };
  // dX from codes: a thread's item of a stage is a block of 32 columns of one row of
  // W, its codes and their scale loaded a step before it is written out as bf16
  const int irow = tid >> 3, icol = (tid & 7) * 32;
  const bool icol_in = n0 + icol < g.H;
  u32x4 iq = {0u, 0u, 0u, 0u};
  uint32_t isc = 0;
  auto load_item = [&](int kt) {
    const int first = min((s_first + kt) * kBK, K), left = min(K - first, kBK);
    const size_t row0 = (size_t)first;
    const __amdgpu_buffer_rsrc_t rc = make_rsrc(reinterpret_cast<const uint8_t*>(g.w) + row0 * (g.H / 2), (uint32_t)(left * (g.H / 2)));
    const __amdgpu_buffer_rsrc_t rs = make_rsrc(g.scales + row0 * (g.H / 32), (uint32_t)(left * (g.H / 32)));
    const uint32_t at = icol_in ? (uint32_t)irow * (uint32_t)(g.H / 2) + (uint32_t)((n0 + icol) / 2) : kOOB;
    const uint32_t as = icol_in ? (uint32_t)irow * (uint32_t)(g.H / 32) + (uint32_t)((n0 + icol) / 32) : kOOB;
    iq = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(rc, (int)at, 0, 0));
    isc = __builtin_amdgcn_raw_buffer_load_b8(rs, (int)as, 0, 0);
  };
  auto write_item = [&](auto S, auto C) {                     // columns 8 C .. 8 C + 7 of it
    constexpr int c = decltype(C)::value;
    SQ_LDS uint16_t* b = (SQ_LDS uint16_t*)(stage_at(S) + kA);
    const uint4 v = ScaleOperand<kMX>::dequant8(iq[c], ScaleOperand<kMX>::of(isc));
    *(SQ_LDS u32x4*)(b + nat_off<BN>(irow, icol + 8 * c)) = __builtin_bit_cast(u32x4, v);
  };
  // f of those of 0 .. ALL - 1 that fall to part N of PARTS
  auto share = [&](auto N, auto PARTS, auto ALL, auto f) {
    constexpr int parts = decltype(PARTS)::value, all = decltype(ALL)::value;
    constexpr int n = decltype(N)::value < parts ? decltype(N)::value : parts, m = n < parts ? n + 1 : parts;
    constexpr int lo = n * all / parts, hi = m * all / parts;
    for_each(std::make_integer_sequence<int, hi - lo>{}, [&](auto K) { f(std::integral_constant<int, lo + decltype(K)::value>{}); });
  };
  using Products = std::make_integer_sequence<int, kProducts>;
  using Reads = std::integral_constant<int, kReads>;

  // One stage.  Between a slice's products go the reads of the next slice and the
  // copies of the stage STAGES - 1 ahead, one at a time, so that neither holds the
  // matrix cores up; the barrier that publishes stage kt + 1 and frees this one
  // stands amid the last slice, whose other half covers its reads and copies.
  auto step = [&](auto S, int kt) {
    constexpr int s = decltype(S)::value;
    using SN = std::integral_constant<int, (s + 1) % STAGES>;            // stage kt + 1
    using SP = std::integral_constant<int, (s + STAGES - 1) % STAGES>;   // stage kt + STAGES - 1
    for_each(std::make_integer_sequence<int, kSlices - 1>{}, [&](auto KK) {
      constexpr int kk = decltype(KK)::value;
      Frag& now = kk & 1 ? F1 : F0;
      Frag& next = kk & 1 ? F0 : F1;
      for_each(Products{}, [&](auto N) {
        product(now, N);
        share(N, std::integral_constant<int, (kReads < kProducts ? kReads : kProducts)>{}, Reads{},
              [&](auto R) { read(S, std::integral_constant<int, kk + 1>{}, next, R); });
        if constexpr (kk == 0)
          share(N, std::integral_constant<int, kProducts>{}, std::integral_constant<int, kHalf[1]>{},
                [&](auto C) { dma(SP{}, kt + STAGES - 1, I1{}, C); });
        if constexpr (kItems && kk == 0 && decltype(N)::value == 0) load_item(kt + 2);
        __builtin_amdgcn_sched_barrier(0);
      });
    });
    for_each(Products{}, [&](auto N) {
      constexpr int n = decltype(N)::value;
      if constexpr (n == kMid) {
        // stage kt + 1 has landed once only the copies of the stages after it are
        // outstanding
        wait_vm_lgkm0<kAhead>();
        __builtin_amdgcn_s_barrier();
        __builtin_amdgcn_sched_barrier(0);
      }
      product(F1, N);
      if constexpr (n >= kMid) {
        using At = std::integral_constant<int, n - kMid>;
        using Rest = std::integral_constant<int, kRest>;
        share(At{}, Rest{}, Reads{}, [&](auto R) { read(SN{}, I0{}, F0, R); });
        share(At{}, Rest{}, std::integral_constant<int, kHalf[0]>{}, [&](auto C) { dma(S, kt + STAGES, I0{}, C); });
        if constexpr (kItems) share(At{}, Rest{}, std::integral_constant<int, 4>{}, [&](auto C) { write_item(S, C); });
      }
      __builtin_amdgcn_sched_barrier(0);
    });
  };
  // The same with CODES: the operands of the next slice are made of the codes that the
  // lane holds; the next stage's codes are read once the present ones are used up.
  auto step_codes = [&](auto S, int kt) {
    constexpr int s = decltype(S)::value;
    using SN = std::integral_constant<int, (s + 1) % STAGES>;
    using SP = std::integral_constant<int, (s + STAGES - 1) % STAGES>;
    using Parts = std::integral_constant<int, kProducts>;
    using Mid = std::integral_constant<int, kMid>;
    using Rest = std::integral_constant<int, kRest>;
    using Rows = std::integral_constant<int, TM>;
    using Cols = std::integral_constant<int, TN>;
    for_each(std::make_integer_sequence<int, kSlices - 1>{}, [&](auto KK) {
      constexpr int kk = decltype(KK)::value;
      using Next = std::integral_constant<int, kk + 1>;
      Frag& now = kk & 1 ? F1 : F0;
      Frag& next = kk & 1 ? F0 : F1;
      for_each(Products{}, [&](auto N) {
        constexpr int n = decltype(N)::value;
        product(now, N);
        share(N, Parts{}, Cols{}, [&](auto J) { read(S, Next{}, next, std::integral_constant<int, decltype(J)::value + 1>{}); });
        if constexpr (kk == kSlices - 2) {
          share(N, Mid{}, Rows{}, [&](auto I) { convert(next, Next{}, I); });
          if constexpr (n >= kMid)
            share(std::integral_constant<int, n - kMid>{}, Rest{}, Rows{}, [&](auto I) { read_codes(SN{}, kt + 1, I); });
        } else {
          share(N, Parts{}, Rows{}, [&](auto I) { convert(next, Next{}, I); });
        }
        if constexpr (kk == 0) share(N, Parts{}, std::integral_constant<int, kHalf[1]>{}, [&](auto C) { dma(SP{}, kt + STAGES - 1, I1{}, C); });
        __builtin_amdgcn_sched_barrier(0);
      });
    });
    for_each(Products{}, [&](auto N) {
      constexpr int n = decltype(N)::value;
      if constexpr (n == kMid) {
        wait_vm_lgkm0<kAhead>();
        __builtin_amdgcn_s_barrier();
        __builtin_amdgcn_sched_barrier(0);
      }
      product(F1, N);
      share(N, Mid{}, Cols{}, [&](auto J) { read(SN{}, I0{}, F0, std::integral_constant<int, decltype(J)::value + 1>{}); });
      if constexpr (n >= kMid) {
        using At = std::integral_constant<int, n - kMid>;
        share(At{}, Rest{}, Rows{}, [&](auto I) { convert(F0, I0{}, I); });
        share(At{}, Rest{}, std::integral_constant<int, kHalf[0]>{}, [&](auto C) { dma(S, kt + STAGES, I0{}, C); });
      }
      __builtin_amdgcn_sched_barrier(0);
    });
    if (kt % kGroup == 0) dma_scales(kt / kGroup + 1);
  };
  // prologue: stage 0 whole and its first operands, then stages 1 .. STAGES - 2
  // and the first half of stage STAGES - 1
  if (nk > 0) {
    dma_half(I0{}, 0, I0{});
    dma_half(I0{}, 0, I1{});
    if constexpr (kItems) {
      load_item(0);
      for_each(std::make_integer_sequence<int, 4>{}, [&](auto C) { write_item(I0{}, C); });
      load_item(1);
      for_each(std::make_integer_sequence<int, 4>{}, [&](auto C) { write_item(I1{}, C); });
    }
    if constexpr (kRowCodes) {
      dma_scales(0);
      dma_half(I1{}, 1, I0{});
      dma_half(I1{}, 1, I1{});
    }
    wait_vm_lgkm0<0>();
    __builtin_amdgcn_s_barrier();
    __builtin_amdgcn_sched_barrier(0);
    if constexpr (kRowCodes) {
      for_each(std::make_integer_sequence<int, TM>{}, [&](auto I) {
        read_codes(I0{}, 0, I);
        convert(F0, I0{}, I);
      });
      for_each(std::make_integer_sequence<int, TN>{}, [&](auto J) { read(I0{}, I0{}, F0, std::integral_constant<int, decltype(J)::value + 1>{}); });
    } else {
      for_each(std::make_integer_sequence<int, kReads>{}, [&](auto R) { read(I0{}, I0{}, F0, R); });
      if constexpr (STAGES > 2) {
        dma_half(I1{}, 1, I0{});
        dma_half(I1{}, 1, I1{});
      }
    }
    dma_half(std::integral_constant<int, STAGES - 1>{}, STAGES - 1, I0{});
  }
  for (int kt0 = 0; kt0 < nk; kt0 += STAGES)
    for_each(std::make_integer_sequence<int, STAGES>{}, [&](auto S) {
      constexpr int s = decltype(S)::value;
      if (s > 0 && kt0 + s >= nk) return;
      if constexpr (kRowCodes) step_codes(S, kt0 + s);
      else step(S, kt0 + s);
    });
  wait_vm_lgkm0<0>();

  // ---------------------------------------------------------------- epilogue
  // 32x32 output tile: lane l, register r holds row 8*(r/4) + 4*(l/32) + r%4,
  // column l%32.
  if constexpr (kDxMode) {
#pragma unroll
    for (int i = 0; i < TM; ++i)
#pragma unroll
      for (int j = 0; j < TN; ++j) {
        const int col = n0 + wn0 + j * 32 + (lane & 31);
        if (col >= g.H) continue;
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          const int row = m0 + wm0 + i * 32 + 8 * (r >> 2) + 4 * (lane >> 5) + (r & 3);
          sums[(size_t)row * g.H + col] = acc[i][j][r];
        }
      }
  } else if constexpr (MODE == kCeLogits) {
    // 4 consecutive rows of W per lane and quarter: 16 bytes of a token's logits
#pragma unroll
    for (int j = 0; j < TN; ++j) {
      const int row = n0 + wn0 + j * 32 + (lane & 31);
      if (row >= live) continue;
      float* out = g.logits + ((size_t)split * g.T + row) * g.ldl;
#pragma unroll
      for (int i = 0; i < TM; ++i)
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          const int v = m0 + wm0 + i * 32 + 8 * q + 4 * (lane >> 5);
          if (v < g.ldl)
            *reinterpret_cast<float4*>(out + v) = 
                make_float4(acc[i][j][4 * q] * g.ws2, acc[i][j][4 * q + 1] * g.ws2, acc[i][j][4 * q + 2] * g.ws2,
                            acc[i][j][4 * q + 3] * g.ws2);
        }
    }
  } else {
    __syncthreads();                     // the operand tiles are done with
    const int end = g.Vn - vrow;                              // rows of W from it on
    const bool whole = m0 + BM <= g.Vn;
#pragma unroll
    for (int j = 0; j < TN; ++j) {
      const int row = n0 + wn0 + j * 32 + (lane & 31);       // compact token row
      const bool valid = (has >> j) & 1;
      const int at = own[j];
      // most waves hold whole tiles and no token's target: their registers need
      // no comparison
      const bool plain = whole && __ballot(at >= 0) == 0;
      if constexpr (MODE == kCeStats) {
        // 4 running maxima and sums, so that none waits for the one before it
        float top, sum;
        auto stats = [&](auto PLAIN) {
          constexpr bool kPlain = decltype(PLAIN)::value;
          float tops[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY}, sums[4] = {0.0f, 0.0f, 0.0f, 0.0f}, l = 0.0f;
#pragma unroll
          for (int i = 0; i < TM; ++i)
#pragma unroll
            for (int r = 0; r < 16; ++r) {
              const int v = i * 32 + 8 * (r >> 2) + (r & 3);
              if (!kPlain) l = v == at ? acc[i][j][r] : l;
              tops[r & 3] = kPlain || v < end ? fmaxf(tops[r & 3], acc[i][j][r]) : tops[r & 3];
            }
          if (!kPlain && at >= 0) g.tlogit[row] = l * g.ws2;
          top = fmaxf(fmaxf(tops[0], tops[1]), fmaxf(tops[2], tops[3]));
          top = fmaxf(top, __shfl_xor(top, 32));
          const float ref = top == -INFINITY ? 0.0f : top;     // nothing to sum: exp(-inf) = 0
          const float scale = g.ws2 * kLog2E;
#pragma unroll
          for (int i = 0; i < TM; ++i)
#pragma unroll
            for (int r = 0; r < 16; ++r) {
              // the distance first: scaled by log2(e) before, logits from 1e4 on lost
              // their last bits and those from 2.36e38 on were infinite
              const float p = __builtin_amdgcn_exp2f((acc[i][j][r] - ref) * scale);
              sums[r & 3] += kPlain || i * 32 + 8 * (r >> 2) + (r & 3) < end ? p : 0.0f;
            }
          sum = (sums[0] + sums[1]) + (sums[2] + sums[3]);
          sum += __shfl_xor(sum, 32);
          top *= g.ws2;
        };
        if (plain) stats(std::true_type{});
        else stats(std::false_type{});
        SQ_LDS float* s = (SQ_LDS float*)lds + 2 * ((wave / WGN) * BN + wn0 + j * 32 + (lane & 31));
        if (lane < 32) {
          s[0] = top;
          s[1] = sum;
        }
      } else {
        // Rounded to bf16 for the product with W, as the layers' dY is.  The
        // target's own, by far the largest as a rule, would bring most of the
        // rounding's error into dX: what it lost is kept, and added with the
        // target's row of W at the end (error against 64 bits 2.5e-3 -> 1.8e-3, of
        // which 1.7e-3 is dX's own rounding to bf16).
        const float c = c_of[j], z = z_of[j];
        SQ_LDS uint16_t* s = (SQ_LDS uint16_t*)lds + wave * WM * WN;
        const int cj = j * 32 + (lane & 31);
        auto grads = [&](auto PLAIN) {
          constexpr bool kPlain = decltype(PLAIN)::value;
          float lost = 0.0f;
#pragma unroll
          for (int i = 0; i < TM; ++i)
#pragma unroll
            for (int q = 0; q < 4; ++q) {
              float e[4];
#pragma unroll
              for (int r = 0; r < 4; ++r) {
                const int v = i * 32 + 8 * q + r;
                const float p = __builtin_amdgcn_exp2f(__builtin_fmaf(acc[i][j][4 * q + r], g.ws2, -z) * kLog2E);
                e[r] = kPlain ? c * p : valid && v < end ? c * (p - (v == at ? 1.0f : 0.0f)) : 0.0f;
              }
              u32x2 pair;
              pair[0] = bits_of(__builtin_convertvector((f32x2{e[0], e[1]}), bf16x2));
              pair[1] = bits_of(__builtin_convertvector((f32x2{e[2], e[3]}), bf16x2));
              if constexpr (!kPlain) {
#pragma unroll
                for (int r = 0; r < 4; ++r) lost = i * 32 + 8 * q + r == at ? e[r] - bf16_half(pair[r >> 1], r & 1) : lost;
              }
              // 16-byte unit u of token cj at unit u ^ cj
              const int u = i * 4 + q;
              *(SQ_LDS u32x2*)(s + cj * WM + ((u ^ cj) & (WM / 8 - 1)) * 8 + 4 * (lane >> 5)) = pair;
            }
          if (!kPlain && at >= 0) g.tlogit[row] = lost;
        };
        // (an ignored token among the rows, as in a batch that is not compact,
        // takes the way with comparisons, which gives it zeros)
        if (plain && __ballot(row < live && !valid) == 0) grads(std::true_type{});
        else grads(std::false_type{});
      }
    }
    if constexpr (MODE == kCeStats) {
      __syncthreads();
      if (tid < BN && n0 + tid < live) {
        const SQ_LDS float* s = (const SQ_LDS float*)lds + 2 * tid;
        float top = s[0], sum = s[1];
#pragma unroll
        for (int w = 1; w < WGM; ++w) {
          const float b = s[2 * w * BN], bs = s[2 * w * BN + 1], m = fmaxf(top, b);
          const float ref = m == -INFINITY ? 0.0f : m;
          sum = sum * __expf(top - ref) + bs * __expf(b - ref);
          top = m;
        }
        float2* out = reinterpret_cast<float2*>(g.part) + (size_t)(g.part_tile0 + tm) * g.T + n0 + tid;
        *out = make_float2(top, sum);
      }
    } else {
      // a wave's own block: WM / 8 lanes take a token's row
      const SQ_LDS uint16_t* s = (const SQ_LDS uint16_t*)lds + wave * WM * WN;
      constexpr int kLanes = WM / 8, kTok = 64 / kLanes;
#pragma unroll
      for (int it = 0; it < WN / kTok; ++it) {
        const int cj = it * kTok + lane / kLanes, u = lane % kLanes;
        const u32x4 v = *(const SQ_LDS u32x4*)(s + cj * WM + ((u ^ cj) & (kLanes - 1)) * 8);
        const int row = n0 + wn0 + cj, col = m0 + wm0 + u * 8;
        if (row < live && col < g.ld) *reinterpret_cast<u32x4*>(g.d + (size_t)row * g.ld + col) = v;
      }
    }
  }
}

// ------------------------------------------------------------------ joins
// loss and lse of 64 tokens per workgroup: 16 waves share the tiles' pairs.
__global__ __launch_bounds__(1024) void ce_loss_kernel(const float2* __restrict__ part, const float* __restrict__ tlogit,
                                                       const int* __restrict__ rows, const int* __restrict__ count,
                                                       const void* __restrict__ y, int y_bytes, int T, int64_t V,
                                                       int tiles, float* __restrict__ loss, float* __restrict__ lse) {
  __shared__ float s_top[16][64], s_sum[16][64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int live = count ? min(*count, T) : T;
  const int row = (int)blockIdx.x * 64 + lane;
  float top = -INFINITY, sum = 0.0f;
  if (row < live) {
#pragma unroll 4
    for (int i = wave; i < tiles; i += 16) {
      const float2 p = part[(size_t)i * T + row];
      const float m = fmaxf(top, p.x), ref = m == -INFINITY ? 0.0f : m;
      sum = sum * __expf(top - ref) + p.y * __expf(p.x - ref);
      top = m;
    }
  }
  s_top[wave][lane] = top;
  s_sum[wave][lane] = sum;
  __syncthreads();
  if (wave == 0 && row < live) {
    for (int w = 1; w < 16; ++w) {
      const float b = s_top[w][lane], m = fmaxf(top, b), ref = m == -INFINITY ? 0.0f : m;
      sum = sum * __expf(top - ref) + s_sum[w][lane] * __expf(b - ref);
      top = m;
    }
    const int t = rows ? rows[row] : row;
    const int64_t v = target_at(y, y_bytes, t);
    if (v >= 0 && v < V) {
      // the largest logit's distance first: for a likely target little is left of
      // lse - logit, and lse's own rounding would be most of the error
      const float rest = __logf(sum);
      lse[t] = top + rest;
      loss[t] = (top - tlogit[row]) + rest;
    }
  }
  // tokens without a target (this workgroup's share of all tokens)
  const int t = (int)blockIdx.x * 64 + lane;
  if (wave == 1 && t < T) {
    const int64_t v = target_at(y, y_bytes, t);
    if (v < 0 || v >= V) lse[t] = loss[t] = 0.0f;
  }
}

// What the last kernel of the gradient adds beside the planes of sums: the
// target's row of the head times what rounding took from its logit's gradient,
// and the rows of a 4-bit head past a multiple of 8, which the layer's products
// do not take.
struct CeRest {
  const void* w;            // the head: bf16 rows or codes
  const uint8_t* scales;
  const float* lost;        // [T], by compact row
  const float* d;           // [T, 8] logit gradients of the rows from `first` on
  int64_t first;
  int rows;
};

// 8 values of a head from element i (a multiple of 8) of its rows on.
template <int HEAD>
__device__ __forceinline__ void head8(const void* w, const uint8_t* scales, int64_t i, float (&v)[8]) {
  if constexpr (HEAD == kCeBf16) {
    const u32x4 q = *reinterpret_cast<const u32x4*>(static_cast<const uint16_t*>(w) + i);
#pragma unroll
    for (int k = 0; k < 8; ++k) v[k] = bf16_half(q[k >> 1], k & 1);
  } else {
    const uint32_t q = *reinterpret_cast<const uint32_t*>(static_cast<const uint8_t*>(w) + (i >> 1));
    const uint32_t b = scales[i / (HEAD == kMX ? 32 : 16)];
    const float s = HEAD == kMX ? e8m0_to_f32(b) : e4m3_to_f32(b);
    const f32x2 c[4] = {__builtin_amdgcn_cvt_scalef32_pk_f32_fp4(q, 1.0f, 0), __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(q, 1.0f, 1),
                        __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(q, 1.0f, 2), __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(q, 1.0f, 3)};
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      v[2 * k] = c[k].x * s;
      v[2 * k + 1] = c[k].y * s;
    }
  }
}

// 1024 columns of one token's dX per workgroup: the planes added in order, times f (and the
// rest's rows times ws2); zeros where there is no target (their rows come after
// the live ones).  planes = 0: as many as the product split the vocabulary into.
template <bool BF16, int HEAD>
__global__ __launch_bounds__(128) void ce_dx_kernel(const float* __restrict__ sums, int planes, int64_t plane_rows,
                                                    const int* __restrict__ rows, const int* __restrict__ count,
                                                    const void* __restrict__ y, int y_bytes, int T, int64_t V, int H,
                                                    int bm, int tiles_n, int stages, float f, float ws2, CeRest rest,
                                                    void* __restrict__ dX) {
  const int live = count ? min(*count, T) : T;
  const int64_t at = (int64_t)blockIdx.z * kGroupsX + blockIdx.x;
  const int b = (int)at, h = ((int)blockIdx.y * 128 + (int)threadIdx.x) * 8;
  if (at >= T || h >= H) return;
  auto put = [&](int t, const float (&v)[8]) {
    if constexpr (BF16) {
      u32x4 w;
#pragma unroll
      for (int i = 0; i < 4; ++i) w[i] = bits_of(__builtin_convertvector((f32x2{v[2 * i], v[2 * i + 1]}), bf16x2));
      *reinterpret_cast<u32x4*>(static_cast<uint16_t*>(dX) + (size_t)t * H + h) = w;
    } else {
      float4* q = reinterpret_cast<float4*>(static_cast<float*>(dX) + (size_t)t * H + h);
      q[0] = make_float4(v[0], v[1], v[2], v[3]);
      q[1] = make_float4(v[4], v[5], v[6], v[7]);
    }
  };
  const int64_t target = target_at(y, y_bytes, b);
  const bool ignored = target < 0 || target >= V;
  if (b < live && (rows || !ignored)) {
    if (planes == 0) {
      const int tiles_m = (live + bm - 1) / bm;
      planes = ce_splits(tiles_m * tiles_n, stages);
      plane_rows = (int64_t)tiles_m * bm;
    }
    const size_t plane = (size_t)plane_rows * H;
    const int t = rows ? rows[b] : b;
    const int64_t own = rows ? target_at(y, y_bytes, t) : target;
    float v[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = 0.0f;
#pragma unroll 8
    for (int s = 0; s < planes; ++s) {
      const float4* q = reinterpret_cast<const float4*>(sums + s * plane + (size_t)b * H + h);
      const float4 a = q[0], c = q[1];
      v[0] += a.x; v[1] += a.y; v[2] += a.z; v[3] += a.w;
      v[4] += c.x; v[5] += c.y; v[6] += c.z; v[7] += c.w;
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] *= f;
    auto add = [&](float d, int64_t row) {
      float w[8];
      head8<HEAD>(rest.w, rest.scales, row * H + h, w);
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] = __builtin_fmaf(d, w[i], v[i]);
    };
    if (own < rest.first) add(rest.lost[b] * ws2, own);
    for (int r = 0; r < rest.rows; ++r) add(rest.d[b * 8 + r] * ws2, rest.first + r);
    put(t, v);
  }
  if (ignored) {
    const float zero[8] = {};
    put(b, zero);
  }
}

// ------------------------------------------------------------------ logits in pieces
// With few tokens the time is the head's bytes, and a 4-bit head written out in
// bf16 first is five times its own: there the layer's own products read the codes.
// And a head of few tiles leaves most of the chip idle: there the tiles' sums over
// I are split into planes.  Either way a piece of fp32 logits passes through the
// workspace, and these kernels do the rest.
//
// A piece's n logits of a token lie in groups of `width` columns, each group a [T,
// width] matrix of its own (width a multiple of 256; the last ends where the logits
// end, so it holds some of the one before it again), or in one matrix of row length
// `width` >= n; in `planes` planes, `plane` values apart, that add up.
struct CePiece {
  const float* logits;
  int n, width, planes;
  int64_t plane;
  int64_t v0;               // its first row of the head
  const int* rows;          // as CeArgs
  const int* count;
  const void* y;
  int y_bytes;
  int T;
  int64_t V;
  __device__ __forceinline__ int live() const { return count ? min(*count, T) : T; }
  __device__ __forceinline__ int token(int row) const { return rows ? rows[row] : row; }
  // where row `row`'s logit of column c < n is, those of the next columns beside it
  // as far as c's group goes
  __device__ __forceinline__ int64_t at(int row, int c) const {
    const int first = c / width * width, early = first > 0 && first + width > n ? first + width - n : 0;
    return (int64_t)first * T + (int64_t)row * width + (c - first + early);
  }
};

// The rows of a 4-bit head past a multiple of 8, fewer than 8, which the layer's
// products do not take: workgroups of their own in the two kernels below, each
// with one token (launches of their own cost 115 tokens of 16301 x 3648 24 us of 152).
struct CeTail {
  const uint16_t* x;        // X [T, H]
  const uint8_t* codes;     // from the first such row on
  const uint8_t* scales;
  int rows, H;              // 0: none
  float ws2;
  int64_t v0;
  float2* part;             // forward
  float* d;                 // backward: fp32 gradients [T, 8]
};

// Token t's logits of these rows, 2 per wave, to s_l; rows that are not there -inf.
template <int HEAD>
__device__ __forceinline__ void tail_logits(const CeTail& g, int t, float* s_l) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  float sum[2] = {0.0f, 0.0f};
#pragma unroll 4
  for (int h = lane * 8; h < g.H; h += 512) {
    const u32x4 q = *reinterpret_cast<const u32x4*>(g.x + (size_t)t * g.H + h);
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      const int r = min(2 * wave + k, g.rows - 1);            // a row past the last is not used
      float w[8];
      head8<HEAD>(g.codes, g.scales, (int64_t)r * g.H + h, w);
#pragma unroll
      for (int i = 0; i < 8; ++i) sum[k] = __builtin_fmaf(bf16_half(q[i >> 1], i & 1), w[i], sum[k]);
    }
  }
#pragma unroll
  for (int k = 0; k < 2; ++k) {
#pragma unroll
    for (int s = 32; s; s >>= 1) sum[k] += __shfl_xor(sum[k], s);
    if (lane == 0) s_l[2 * wave + k] = 2 * wave + k < g.rows ? sum[k] * g.ws2 : -INFINITY;
  }
  __syncthreads();
}

// (max, sum) of 256 logits of one token per wave, and the target's logit; past the
// n logits, a workgroup per token for the tail (HEAD a 4-bit format).
template <int HEAD>
__global__ __launch_bounds__(256) void ce_part_kernel(CePiece p, float2* __restrict__ part, float* __restrict__ tlogit,
                                                      CeTail tail) {
  const int extra = (int)blockIdx.x - (p.n + 255) / 256;
  if (HEAD != kCeBf16 && extra >= 0) {
    __shared__ float s_l[8];
    const int t = (int)blockIdx.y * 4 + extra;
    if (t >= p.T) return;
    tail_logits<HEAD>(tail, t, s_l);
    if (threadIdx.x == 0) {
      const int64_t at = target_at(p.y, p.y_bytes, t) - tail.v0;
      float top = -INFINITY, total = 0.0f;
      for (int r = 0; r < tail.rows; ++r) {
        top = fmaxf(top, s_l[r]);
        if (at == r) tlogit[t] = s_l[r];
      }
      const float ref = top == -INFINITY ? 0.0f : top;
      for (int r = 0; r < tail.rows; ++r) total += __expf(s_l[r] - ref);
      tail.part[t] = make_float2(top, total);
    }
    return;
  }
  const int lane = threadIdx.x & 63, row = (int)blockIdx.y * 4 + (threadIdx.x >> 6);
  if (row >= p.live()) return;
  const int c0 = (int)blockIdx.x * 256 + lane * 4;
  const int64_t at = target_at(p.y, p.y_bytes, p.token(row)) - p.v0 - c0;
  float l[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY}, top = -INFINITY;
  if (c0 < p.n) {
    const float* src = p.logits + p.at(row, c0);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if (c0 + i >= p.n) continue;
      l[i] = src[i];
      for (int s = 1; s < p.planes; ++s) l[i] += src[s * p.plane + i];
      if (at == i) tlogit[row] = l[i];
      top = fmaxf(top, l[i]);
    }
  }
#pragma unroll
  for (int d = 32; d; d >>= 1) top = fmaxf(top, __shfl_xor(top, d));
  const float ref = top == -INFINITY ? 0.0f : top;
  float sum = 0.0f;
#pragma unroll
  for (int i = 0; i < 4; ++i) sum += __expf(l[i] - ref);
#pragma unroll
  for (int d = 32; d; d >>= 1) sum += __shfl_xor(sum, d);
  if (lane == 0) part[(size_t)blockIdx.x * p.T + row] = make_float2(top, sum);
}

// The logits' gradients in bf16, 8 of one token per lane, in groups of d_width
// columns, each a [T, d_width] matrix; d_cols columns in all, whole groups.  The
// last group ends where the logits end, so it begins `shift` columns inside the
// one before it, and those columns are zeros in it; without groups (d_width =
// d_cols, shift 0) columns from n on are zeros.  All sizes are multiples of 8 but n.
// Past the columns, a workgroup per token for the tail (HEAD a 4-bit format).
template <int HEAD>
__global__ __launch_bounds__(256) void ce_grad_kernel(CePiece p, const float* __restrict__ lse,
                                                      const float* __restrict__ dloss, int d_cols, int d_width, int shift,
                                                      uint16_t* __restrict__ d, float* __restrict__ lost, CeTail tail) {
  if (HEAD != kCeBf16 && (int)blockIdx.x * 2048 >= d_cols) {
    __shared__ float s_l[8];
    const int t = (int)blockIdx.y, r = (int)threadIdx.x;
    tail_logits<HEAD>(tail, t, s_l);
    const int64_t y = target_at(p.y, p.y_bytes, t);
    if (r < tail.rows)
      tail.d[t * 8 + r] = y >= 0 && y < p.V ? dloss[t] * (__expf(s_l[r] - lse[t]) - (y - tail.v0 == r ? 1.0f : 0.0f)) : 0.0f;
    return;
  }
  const int row = (int)blockIdx.y, k = ((int)blockIdx.x * 256 + (int)threadIdx.x) * 8;
  if (row >= p.live() || k >= d_cols) return;
  const int first = k / d_width * d_width, early = first + d_width >= d_cols ? shift : 0;
  const int c = k - early, t = p.token(row);
  const int64_t target = target_at(p.y, p.y_bytes, t), at = target - p.v0 - c;
  const bool any = target >= 0 && target < p.V && c < p.n && k - first >= early;
  float x[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) x[i] = 0.0f;
  if (any) {
    const float* src = p.logits + p.at(row, c);
    for (int s = 0; s < p.planes; ++s) {
      const float4* l = reinterpret_cast<const float4*>(src + s * p.plane);
      const float4 a = l[0], b = l[1];
      x[0] += a.x; x[1] += a.y; x[2] += a.z; x[3] += a.w;
      x[4] += b.x; x[5] += b.y; x[6] += b.z; x[7] += b.w;
    }
  }
  const float f = any ? dloss[t] : 0.0f, z = any ? lse[t] : 0.0f;
  u32x4 w;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    f32x2 e;
    e.x = any && c + 2 * i < p.n ? f * (__expf(x[2 * i] - z) - (at == 2 * i ? 1.0f : 0.0f)) : 0.0f;
    e.y = any && c + 2 * i + 1 < p.n ? f * (__expf(x[2 * i + 1] - z) - (at == 2 * i + 1 ? 1.0f : 0.0f)) : 0.0f;
    w[i] = bits_of(__builtin_convertvector(e, bf16x2));
    if (any && at >= 0 && at >> 1 == i) lost[row] = at & 1 ? e.y - bf16_half(w[i], 1) : e.x - bf16_half(w[i], 0);
  }
  *reinterpret_cast<u32x4*>(d + (size_t)first * p.T + (size_t)row * d_width + (k - first)) = w;
}

inline int ok() { return hipGetLastError() == hipSuccess ? 0 : -1; }

// ------------------------------------------------------------------ plan
constexpr int64_t kCeSplitStages = 16;  // stages of the sum over I from which few tiles are split
constexpr int64_t kCePieceBytes = int64_t(256) << 20;        // a piece's logit gradients, and a 4-bit head's bf16 rows

struct CePlan {
  int bt, bx;               // token extent of the logits' tiles and of dX's
  bool compact;             // rows without a target are left out
  int splits;               // of the logits' sums over I, through fp32 planes (1: none)
  int64_t piece;            // rows of W per piece (a multiple of 256)
  int pieces;
  int ld;                   // columns of the logit gradients (and of the planes)
  int64_t groups;           // tiles times splits of dX, at most
  size_t rows, tlogit, part, wbuf, logits, d, sums, total;   // offsets in the workspace
};

inline int64_t up(int64_t v, int64_t m) { return (v + m - 1) / m * m; }

// Token extent of the logits' tiles: the least time in rounds of the CUs, where a
// round of 256 x 128 and 256 x 64 tiles takes 0.58 and 0.36 of one of 256 x 256
// tiles, and a last round from three quarters of a whole one on, as it is filled.
// us of the forward with 64-, 128- and 256-token tiles, bf16: 1024 tokens of
// 16384 x 4096 146, 123, 115; 180 of 72000 x 5120 277, 252, 279; 300 of 131072 x 4096
// 494, 434, 455; 420 of 36320 x 544 41, 44, 49; 130 of 40000 x 1024 26, 34, 32.  From
// codes: 180 of 72000 x 5120 165, 227, 224; 300 of 131072 x 4096 417, 444, 448.  The
// rule is the same for both, though codes would gain from 64 more often: then tiles
// of up to 128 tokens join the sums of codes in the order of their bf16 values', and
// give the same bits (256-token ones have their waves laid out otherwise).
int ce_tokens(int64_t T, int64_t vt) {
  auto cost = [&](int bt, double round) {
    const int64_t tiles = vt * (up(T, bt) / bt), last = tiles % kCUs;
    return round * (double)(tiles / kCUs) + (last ? round * (0.75 + 0.25 * (double)last / kCUs) : 0.0);
  };
  const double c64 = cost(64, 0.36), c128 = cost(128, 0.58), c256 = cost(256, 1.0);
  if (c64 < c128 && c64 < c256) return 64;
  return c128 < c256 ? 128 : 256;
}

// Token extent of dX's tiles: their products' time, with the idle CUs and what
// smaller tiles were measured to cost, and that of the fp32 planes, which double
// with the extent (bf16, us of the gradient with 64-, 128- and 256-token tiles: 256
// tokens of 50000 x 2048 133, 127, 142; 501 of 72471 x 4960 1437, 943, 877; 174 of
// 7717 x 736 31, 34, 37; 3947 of 2830 x 960 86, 83, 91).
int ce_dx_tokens(int64_t T, int64_t rows, int64_t cols) {
  auto cost = [&](int bx, double product) {
    const int64_t tiles = up(T, bx) / bx * cols;
    const int64_t groups = tiles > kCUs * 16 ? tiles : tiles * ce_splits((int)tiles, (int)((rows + kBK - 1) / kBK));
    const double us = product * 2e-9 / 1.3 * (double)up(groups, kCUs) / (double)groups * (double)(tiles * bx) * 256 * (double)rows;
    return us + 2 * 1024 / 5e6 * (double)(groups * bx);
  };
  const double c64 = cost(64, 2.0), c128 = cost(128, 1.25), c256 = cost(256, 1.0);
  if (c64 < c128 && c64 < c256) return 64;
  return c128 < c256 ? 128 : 256;
}

CePlan ce_plan(bool bwd, bool four_bit, int64_t T, int64_t V, int64_t H) {
  CePlan p{};
  const int64_t vt = (V + 255) / 256;
  p.bt = ce_tokens(T, vt);
  p.compact = T > 256;
  int64_t most = up(V, 256);
  if (bwd) most = kCePieceBytes / (2 * T);
  if (four_bit || bwd) {                                     // also 32-bit offsets into a piece of W
    // A 4-bit head's rows, written out and read while still in the cache at 256
    // MiB, but at least four tiles for every CU within 1 GiB (673 tokens, half of
    // them ignored, of 143596 x 8160 MXFP4: pieces of 256 MiB 6.6 ms, of 1 GiB 5.3)
    int64_t by_w = (int64_t(1) << 30) / (2 * H);
    if (four_bit) {
      const int64_t cached = kCePieceBytes / (2 * H), fill = 4 * kCUs * 256 / (up(T, p.bt) / p.bt), rows = cached > fill ? cached : fill;
      by_w = rows < by_w ? rows : by_w;
    }
    most = most < by_w ? most : by_w;
  }
  const int64_t by_grid = kGroupsX / (up(T, p.bt) / p.bt) * 256;   // the tiles of a launch
  most = most < by_grid ? most : by_grid;
  most = most / 256 * 256 > 256 ? most / 256 * 256 : 256;
  p.pieces = (int)((V + most - 1) / most);
  p.piece = up((V + p.pieces - 1) / p.pieces, 256);
  p.pieces = (int)((V + p.piece - 1) / p.piece);
  p.ld = (int)(p.piece < V ? p.piece : up(V, 64));
  // Few tiles (64-token ones then, by ce_tokens) and a long sum: split it, at least 4
  // stages each (bf16, us of loss and gradient, whole against split: 4 tokens of 1136
  // x 7296 104, 45; 300 of 3891 x 4864 108, 85; 100 of 8000 x 4096 82, 69).
  const int64_t tiles = vt * (up(T, p.bt) / p.bt), stages = (H + kBK - 1) / kBK;
  p.splits = 1;
  if (p.pieces == 1 && p.bt == 64 && 2 * tiles <= kCUs && stages >= kCeSplitStages) {
    const int64_t by_cu = kCUs / tiles, by_stages = stages / 4, n = by_cu < by_stages ? by_cu : by_stages;
    p.splits = (int)(n < 8 ? n : 8);
  }
  size_t at = 256;                                           // the count of live rows
  auto take = [&](size_t bytes) {
    const size_t o = at;
    at += (bytes + 255) & ~(size_t)255;
    return o;
  };
  p.rows = take(p.compact ? (size_t)T * 4 : 0);
  if (four_bit) p.wbuf = take((size_t)p.piece * H * 2);
  p.tlogit = take((size_t)T * 4);
  if (p.splits > 1) p.logits = take((size_t)p.splits * T * p.ld * 4);
  if (!bwd) {
    p.part = take((size_t)vt * T * 8);
  } else {
    p.d = take((size_t)T * p.ld * 2);
    const int64_t dx_cols = up(H, 256) / 256;
    p.bx = ce_dx_tokens(T, p.piece < V ? p.piece : V, dx_cols);
    // planes of whole tiles, for as many live rows as need the most
    const int64_t tt = up(T, p.bx) / p.bx;
    const int stages = (int)(((p.piece < V ? p.piece : V) + kBK - 1) / kBK);
    p.groups = tt * dx_cols;
    for (int64_t t = dx_cols; t <= tt * dx_cols && t <= kCeMostGroups; t += dx_cols) {
      const int64_t n = t * ce_splits((int)t, stages);
      p.groups = p.groups > n ? p.groups : n;
    }
    p.sums = take((size_t)p.groups * p.bx * 256 * 4);
  }
  p.total = at;
  return p;
}

// 256 x 64 tiles: where there are more than CUs two workgroups share one, with two
// stages each, otherwise one with three (us of the forward, bf16, three stages against
// two: 300 tokens of 50000 x 4096 226, 202; 420 of 36320 x 544 46, 42; 250 of 8000 x
// 4096 36, 42; 40 of 50000 x 2048 36, 39).
template <int MODE>
int ce_go(const CeArgs& g, int bt, int64_t blocks, hipStream_t s) {
  if (blocks == 0) return 0;
  const dim3 grid((unsigned)blocks), block(512);
  if constexpr (MODE == kCeLogits) {                          // of 64 tokens, as many as the CUs at most
    hipLaunchKernelGGL((ce_kernel<MODE, 256, 64, 8, 1, 3>), grid, block, 0, s, g);
  } else if constexpr (MODE == kCeDx) {
    if (bt == 64) hipLaunchKernelGGL((ce_kernel<MODE, 64, 256, 1, 8, 3>), grid, block, 0, s, g);
    else if (bt == 128) hipLaunchKernelGGL((ce_kernel<MODE, 128, 256, 2, 4, 3>), grid, block, 0, s, g);
    else hipLaunchKernelGGL((ce_kernel<MODE, 256, 256, 2, 4, 2>), grid, block, 0, s, g);
  } else {
    if (bt == 64 && blocks > kCUs) hipLaunchKernelGGL((ce_kernel<MODE, 256, 64, 8, 1, 2>), grid, block, 0, s, g);
    else if (bt == 64) hipLaunchKernelGGL((ce_kernel<MODE, 256, 64, 8, 1, 3>), grid, block, 0, s, g);
    else if (bt == 128) hipLaunchKernelGGL((ce_kernel<MODE, 256, 128, 4, 2, 3>), grid, block, 0, s, g);
    else hipLaunchKernelGGL((ce_kernel<MODE, 256, 256, 2, 4, 2>), grid, block, 0, s, g);
  }
  return ok();
}

// An MXFP4 head straight from its codes: rows that its 16-byte copies of codes and
// scales end with, and tiles enough.  Of the logits' tiles two waves convert each
// value, of dX's one thread, on its way to LDS, which costs the products up to 8%
// over bf16 operands; neither the head in bf16 nor the logits of the layer's own
// products go through memory, which counts for less with more tokens.  us of loss
// and gradient, without against with: 300 tokens of 50000 x 4096 806, 473; 1024 of
// 131072 x 4096 3318, 2879; 2048 of 50001 x 4096 2510, 2178; 4096 of it 4260, 4268;
// 8192 of 50001 x 2048 4322, 4504.  The forward of 64 and 256 tokens of 131072 x 4096:
// 109, 88 and 283, 225.  The gradient of up to 64 tokens stays with the layer's
// products (64 tokens of 131072 x 4096 307, from codes 326; 128 tokens 573, 490).
constexpr int kCeCodesTokens = 64, kCeCodesMost = 4096;

bool ce_codes(int head, int64_t T, int64_t V, int64_t H) {
  if (head != kMX || H % 512 != 0 || T < 1 || T > kCeCodesMost) return false;
  const CePlan p = ce_plan(false, false, T, V, H);
  return p.splits == 1 && p.pieces == 1;
}

template <int MODE>
int ce_codes_go(const CeArgs& g, int bt, int64_t blocks, hipStream_t s) {
  if (blocks == 0) return 0;
  const dim3 grid((unsigned)blocks), block(512);
  if constexpr (MODE == kCeDx) {
    if (bt == 64) hipLaunchKernelGGL((ce_kernel<MODE, 64, 256, 1, 8, 2, true>), grid, block, 0, s, g);
    else if (bt == 128) hipLaunchKernelGGL((ce_kernel<MODE, 128, 256, 2, 4, 2, true>), grid, block, 0, s, g);
    else hipLaunchKernelGGL((ce_kernel<MODE, 256, 256, 2, 4, 2, true>), grid, block, 0, s, g);
  } else {
    if (bt == 64) hipLaunchKernelGGL((ce_kernel<MODE, 256, 64, 8, 1, 3, true>), grid, block, 0, s, g);
    else if (bt == 128) hipLaunchKernelGGL((ce_kernel<MODE, 256, 128, 4, 2, 3, true>), grid, block, 0, s, g);
    else hipLaunchKernelGGL((ce_kernel<MODE, 256, 256, 4, 2, 3, true>), grid, block, 0, s, g);
  }
  return ok();
}

// The bf16 rows [v0, v0 + n) of the head: its own, or a 4-bit piece written out.
int ce_weight(int head, const void* W, const uint8_t* scales, int64_t v0, int64_t n, int64_t H, void* buf,
              const uint16_t** out, hipStream_t s) {
  if (head == kCeBf16) {
    *out = static_cast<const uint16_t*>(W) + v0 * H;
    return 0;
  }
  uint16_t* b = static_cast<uint16_t*>(buf);
  *out = b;
  const int64_t first = v0 * H / 8, items = n * H / 8;
  const dim3 grid((unsigned)((items + 255) / 256)), block(256);
  const uint8_t* codes = static_cast<const uint8_t*>(W);
  if (head == kMX) hipLaunchKernelGGL((ce_dequant_kernel<kMX>), grid, block, 0, s, codes, scales, first, items, b);
  else hipLaunchKernelGGL((ce_dequant_kernel<kNV>), grid, block, 0, s, codes, scales, first, items, b);
  return ok();
}

int ce_part_go(int head, const CePiece& c, float2* part, float* tlogit, const CeTail& tail, hipStream_t s) {
  const dim3 grid((unsigned)((c.n + 255) / 256 + (tail.rows > 0 ? 4 : 0)), (unsigned)((c.T + 3) / 4));
  auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, dim3(256), 0, s, c, part, tlogit, tail); };
  if (tail.rows == 0) go(ce_part_kernel<kCeBf16>);
  else head == kMX ? go(ce_part_kernel<kMX>) : go(ce_part_kernel<kNV>);
  return ok();
}

int ce_grad_go(int head, const CePiece& c, const float* lse, const float* dloss, int d_cols, int d_width, int shift,
               uint16_t* d, float* lost, const CeTail& tail, hipStream_t s) {
  const dim3 grid((unsigned)((d_cols / 8 + 255) / 256 + (tail.rows > 0 ? 1 : 0)), (unsigned)c.T);
  auto go = [&](auto kernel) {
    hipLaunchKernelGGL(kernel, grid, dim3(256), 0, s, c, lse, dloss, d_cols, d_width, shift, d, lost, tail);
  };
  if (tail.rows == 0) go(ce_grad_kernel<kCeBf16>);
  else head == kMX ? go(ce_grad_kernel<kMX>) : go(ce_grad_kernel<kNV>);
  return ok();
}

// Workgroups of the gradient's last step.
inline dim3 ce_dx_grid(int T, int H) {
  return dim3((unsigned)(T < kGroupsX ? T : kGroupsX), (unsigned)((H + 1023) / 1024), (unsigned)((T + kGroupsX - 1) / kGroupsX));
}

// The last step of the gradient, for each head and output type.
template <typename F>
int ce_dx_by(int head, int dx_bf16, F finish) {
  if (head == kMX) return dx_bf16 ? finish(ce_dx_kernel<true, kMX>) : finish(ce_dx_kernel<false, kMX>);
  if (head == kNV) return dx_bf16 ? finish(ce_dx_kernel<true, kNV>) : finish(ce_dx_kernel<false, kNV>);
  return dx_bf16 ? finish(ce_dx_kernel<true, kCeBf16>) : finish(ce_dx_kernel<false, kCeBf16>);
}

int ce_loss_go(const float2* part, const float* tlogit, const CePiece& c, int tiles, float* loss, float* lse, hipStream_t s) {
  hipLaunchKernelGGL(ce_loss_kernel, dim3((unsigned)((c.T + 63) / 64)), dim3(1024), 0, s, part, tlogit, c.rows, c.count, c.y,
                     c.y_bytes, c.T, c.V, tiles, loss, lse);
  return ok();
}

// ------------------------------------------------------------------ 4-bit heads, few tokens
constexpr int64_t kCeLogitBytes = int64_t(64) << 20;         // a piece's fp32 logits

struct CeFew {
  int64_t main;             // rows of the head that the layer's products take (a multiple of 8)
  int tail;                 // the others, fewer than 8
  int64_t piece;            // rows per piece of logits
  int group;                // rows per group of the logits' product (0: one product)
  int width, groups, shift; // backward: groups of dX's contraction, as ce_grad_kernel takes them
  size_t tlogit, part, logits, d, sums, dtail, total;
};

// One product over many rows would take strips or tiles made for a layer's few; as
// a grouped one over groups of 4096 rows it takes the grouped products' tiles
// (131072 x 4096, one product against groups, us of NVFP4's loss and gradient: 1
// token 297, 311; 64 tokens 442, 413; 128 tokens 721, 593; 256 tokens 966, 1104; of
// MXFP4's gradient: 1 token 180, 150; 64 tokens 275, 206).
constexpr int kCeGroupTokens = 128, kCeGroupRows = 4096, kCeGroupFrom = 8 * kCeGroupRows;

CeFew ce_few_plan(bool bwd, int64_t T, int64_t V, int64_t H) {
  CeFew p{};
  p.main = V / 8 * 8;
  p.tail = (int)(V - p.main);
  p.group = (T <= kCeGroupTokens && p.main >= kCeGroupFrom) || p.main * H > int64_t(1) << 31 ? kCeGroupRows : 0;
  int64_t rows = kCeLogitBytes / (4 * T);
  const int64_t by_codes = (int64_t(1) << 31) / H;           // operands below 1 GiB
  rows = rows < by_codes ? rows : by_codes;
  rows = rows / kCeGroupRows * kCeGroupRows;
  p.piece = rows > kCeGroupRows ? rows : kCeGroupRows;
  // dX in as many groups of equal width as their 256-column tiles need to fill the
  // CUs twice, over all of the head at once: its gradients are 2 bytes per logit
  const int64_t cols = (H + 255) / 256, want = (2 * kCUs + cols - 1) / cols;
  p.width = (int)up((p.main + (want < 64 ? want : 64) - 1) / (want < 64 ? want : 64), 64);
  if (p.width < 256) p.width = 256;
  if (p.width > p.main) p.width = (int)p.main;
  p.groups = (int)((p.main + p.width - 1) / p.width);
  p.shift = (int)((int64_t)p.groups * p.width - p.main);
  const int64_t most = bwd || p.piece > p.main ? p.main : p.piece;
  size_t at = 0;
  auto take = [&](size_t bytes) {
    const size_t o = at;
    at += (bytes + 255) & ~(size_t)255;
    return o;
  };
  p.logits = take((size_t)(p.group > 0 ? up(most, p.group) : most) * T * 4);
  p.tlogit = take((size_t)T * 4);
  if (!bwd) {
    p.part = take((size_t)((p.main + 255) / 256 + 1) * T * 8);
  } else {
    p.d = take((size_t)p.groups * p.width * T * 2);
    p.sums = take((size_t)p.groups * T * H * 4);
    p.dtail = take((size_t)T * 32);
  }
  p.total = at;
  return p;
}

// Whether the layer's products take the head (their operands within 32 bits).
bool ce_few(int head, int64_t T, int64_t V, int64_t H) {
  if (head == kCeBf16 || T > kCeFewTokens || V < 8) return false;
  const CeFew p = ce_few_plan(true, T, V, H);
  return p.width * H <= int64_t(1) << 31 && kCeGroupRows * H <= int64_t(1) << 31 && p.width * T * 4 <= int64_t(1) << 30 &&
         p.main * T * 4 <= int64_t(1) << 30;
}

// Logits of rows [v0, v0 + n) of the head to `logits`, and how they lie in *c.
int ce_few_logits(int head, int T, int64_t v0, int n, int H, const void* X, const uint8_t* codes, const uint8_t* scales,
                  float ws2, int group, float* logits, CePiece* c, hipStream_t s) {
  const int64_t G = H / (head == kMX ? 32 : 16);
  const uint8_t* cd = codes + v0 * H / 2;
  const uint8_t* sc = scales + v0 * G;
  c->logits = logits;
  c->v0 = v0;
  c->n = n;
  c->planes = 1;
  c->width = group > 0 && n > group ? group : n;
  if (c->width == n) return gemm_fwd(head, T, n, H, X, cd, sc, ws2, logits, 0, s);
  ExpertProblem e[kGroupMax];
  const int groups = (n + group - 1) / group;
  for (int k0 = 0; k0 < groups; k0 += kGroupMax) {
    const int m = groups - k0 < kGroupMax ? groups - k0 : kGroupMax;
    for (int k = 0; k < m; ++k) {
      const int64_t at = (int64_t)(k0 + k) * group, r = at + group < n ? at : n - group;
      e[k] = ExpertProblem{X, nullptr, cd + r * H / 2, sc + r * G, logits + at * T, T, ws2};
    }
    if (gemm_fwd_grouped(head, group, H, m, e, 0, s) != 0) return -1;
  }
  return 0;
}

CeTail ce_tail(const CeFew& p, int head, const void* X, const uint8_t* codes, const uint8_t* scales, int H, float ws2) {
  return CeTail{static_cast<const uint16_t*>(X), codes + p.main * H / 2, scales + p.main * (H / (head == kMX ? 32 : 16)),
                p.tail, H, ws2, p.main, nullptr, nullptr};
}

int ce_few_fwd(int head, int T, int64_t V, int H, const void* X, const uint8_t* codes, const uint8_t* scales, float ws2,
               const void* y, int y_bytes, float* loss, float* lse, uint8_t* ws, hipStream_t s) {
  const CeFew p = ce_few_plan(false, T, V, H);
  float* logits = reinterpret_cast<float*>(ws + p.logits);
  float2* part = reinterpret_cast<float2*>(ws + p.part);
  float* tlogit = reinterpret_cast<float*>(ws + p.tlogit);
  CePiece c{};
  c.y = y; c.y_bytes = y_bytes; c.T = T; c.V = V;
  int tiles = 0;
  for (int64_t v0 = 0; v0 < p.main; v0 += p.piece) {
    const int n = (int)(p.main - v0 < p.piece ? p.main - v0 : p.piece);
    if (ce_few_logits(head, T, v0, n, H, X, codes, scales, ws2, p.group, logits, &c, s) != 0) return -1;
    const bool last = v0 + n == p.main;
    const int own = (n + 255) / 256;
    CeTail tail{};
    if (last && p.tail > 0) tail = ce_tail(p, head, X, codes, scales, H, ws2);
    tail.part = part + (size_t)(tiles + own) * T;
    if (ce_part_go(head, c, part + (size_t)tiles * T, tlogit, tail, s) != 0) return -1;
    tiles += own + (tail.rows > 0);
  }
  return ce_loss_go(part, tlogit, c, tiles, loss, lse, s);
}

int ce_few_bwd(int head, int T, int64_t V, int H, const void* X, const uint8_t* codes, const uint8_t* scales, float ws2,
               const void* y, int y_bytes, const float* lse, const float* dloss, void* dX, int dx_bf16, uint8_t* ws,
               hipStream_t s) {
  const CeFew p = ce_few_plan(true, T, V, H);
  const int64_t G = H / (head == kMX ? 32 : 16);
  uint16_t* d = reinterpret_cast<uint16_t*>(ws + p.d);
  float* sums = reinterpret_cast<float*>(ws + p.sums);
  float* dtail = reinterpret_cast<float*>(ws + p.dtail);
  float* lost = reinterpret_cast<float*>(ws + p.tlogit);
  CePiece c{};
  c.y = y; c.y_bytes = y_bytes; c.T = T; c.V = V;
  if (ce_few_logits(head, T, 0, (int)p.main, H, X, codes, scales, ws2, p.group, reinterpret_cast<float*>(ws + p.logits), &c, s) != 0)
    return -1;
  CeTail tail{};
  if (p.tail > 0) tail = ce_tail(p, head, X, codes, scales, H, ws2);
  tail.d = dtail;
  if (ce_grad_go(head, c, lse, dloss, p.groups * p.width, p.width, p.shift, d, lost, tail, s) != 0) return -1;
  // dX of every group of rows, as the layer's grouped product
  ExpertProblem e[64];
  for (int k = 0; k < p.groups; ++k) {
    const int64_t v0 = (int64_t)k * p.width - (k + 1 == p.groups ? p.shift : 0);
    e[k] = ExpertProblem{d + (size_t)k * p.width * T, nullptr, codes + v0 * H / 2, scales + v0 * G, sums + (size_t)k * T * H, T, ws2};
  }
  if (gemm_dx_grouped(head, p.width, H, p.groups, e, 0, s) != 0) return -1;
  const CeRest rest{codes, scales, lost, dtail, p.main, p.tail};
  auto finish = [&](auto kernel) {
    hipLaunchKernelGGL(kernel, ce_dx_grid(T, H), dim3(128), 0, s, sums, p.groups, (int64_t)T, nullptr, nullptr, y, y_bytes,
                       T, V, H, 0, 0, 0, 1.0f, ws2, rest, dX);
    return ok();
  };
  return ce_dx_by(head, dx_bf16, finish);
}

}  // namespace

size_t ce_workspace(int bwd, int head, int64_t T, int64_t V, int64_t H) {
  const size_t n = ce_few(head, T, V, H) ? ce_few_plan(bwd != 0, T, V, H).total : ce_plan(bwd != 0, head != kCeBf16, T, V, H).total;
  if (!ce_codes(head, T, V, H)) return n;
  const size_t codes = ce_plan(bwd != 0, false, T, V, H).total;  // either way: what decides is where the operands are
  return n > codes ? n : codes;
}

// What both directions set up: the arguments, and the live rows numbered.
static int ce_begin(const CePlan& p, int T, int64_t V, int H, const void* X, float ws2, const void* y, int y_bytes, uint8_t* ws,
                    CeArgs* g, CePiece* c, hipStream_t s) {
  g->x = static_cast<const uint16_t*>(X);
  g->y = y; g->y_bytes = y_bytes; g->T = T; g->H = H; g->V = V; g->ws2 = ws2;
  g->tlogit = reinterpret_cast<float*>(ws + p.tlogit);
  g->ld = g->ldl = p.ld;
  g->splits = p.splits;
  g->logits = reinterpret_cast<float*>(ws + p.logits);
  if (p.compact) {
    int* count = reinterpret_cast<int*>(ws);
    int* rows = reinterpret_cast<int*>(ws + p.rows);
    g->count = count;
    g->rows = rows;
    hipLaunchKernelGGL(ce_rows_kernel, dim3(1), dim3(1024), 0, s, y, y_bytes, T, V, count, rows);
    if (ok() != 0) return -1;
  }
  c->logits = g->logits;
  c->n = (int)V; c->width = p.ld; c->planes = p.splits; c->plane = (int64_t)T * p.ld;
  c->rows = g->rows; c->count = g->count; c->y = y; c->y_bytes = y_bytes; c->T = T; c->V = V;
  return 0;
}

int ce_fwd_launch(int head, int T, int64_t V, int H, const void* X, const void* W, const uint8_t* scales, float ws2,
                  const void* y, int y_bytes, float* loss, float* lse, void* workspace, hipStream_t s) {
  uint8_t* ws = static_cast<uint8_t*>(workspace);
  if (ce_codes(head, T, V, H) && ((uintptr_t)W | (uintptr_t)scales) % 16 == 0) {
    const CePlan p = ce_plan(false, false, T, V, H);
    CeArgs g{};
    CePiece c{};
    if (ce_begin(p, T, V, H, X, ws2, y, y_bytes, ws, &g, &c, s) != 0) return -1;
    g.w = static_cast<const uint16_t*>(W);
    g.scales = scales;
    g.Vn = (int)V;
    g.part = reinterpret_cast<float*>(ws + p.part);
    const int tiles = (int)((V + 255) / 256);
    if (ce_codes_go<kCeStats>(g, p.bt, (int64_t)tiles * ((T + p.bt - 1) / p.bt), s) != 0) return -1;
    return ce_loss_go(reinterpret_cast<float2*>(g.part), g.tlogit, c, tiles, loss, lse, s);
  }
  if (ce_few(head, T, V, H))
    return ce_few_fwd(head, T, V, H, X, static_cast<const uint8_t*>(W), scales, ws2, y, y_bytes, loss, lse, ws, s);
  const CePlan p = ce_plan(false, head != kCeBf16, T, V, H);
  CeArgs g{};
  CePiece c{};
  if (ce_begin(p, T, V, H, X, ws2, y, y_bytes, ws, &g, &c, s) != 0) return -1;
  g.part = reinterpret_cast<float*>(ws + p.part);
  float2* part = reinterpret_cast<float2*>(g.part);
  const int64_t tt = (T + p.bt - 1) / p.bt;
  for (int64_t v0 = 0; v0 < V; v0 += p.piece) {
    const int64_t n = V - v0 < p.piece ? V - v0 : p.piece, tiles = (n + 255) / 256 * tt;
    if (ce_weight(head, W, scales, v0, n, H, ws + p.wbuf, &g.w, s) != 0) return -1;
    g.v0 = v0;
    g.Vn = (int)n;
    g.part_tile0 = (int)(v0 / 256);
    if (p.splits > 1) {
      if (ce_go<kCeLogits>(g, p.bt, tiles * p.splits, s) != 0 || ce_part_go(head, c, part, g.tlogit, CeTail{}, s) != 0) return -1;
    } else if (ce_go<kCeStats>(g, p.bt, tiles, s) != 0) {
      return -1;
    }
  }
  return ce_loss_go(part, g.tlogit, c, (int)((V + 255) / 256), loss, lse, s);
}

int ce_bwd_launch(int head, int T, int64_t V, int H, const void* X, const void* W, const uint8_t* scales, float ws2,
                  const void* y, int y_bytes, const float* lse, const float* dloss, void* dX, int dx_bf16,
                  void* workspace, hipStream_t s) {
  uint8_t* ws = static_cast<uint8_t*>(workspace);
  const bool codes = T > kCeCodesTokens && ce_codes(head, T, V, H) && ((uintptr_t)W | (uintptr_t)scales) % 16 == 0;
  if (!codes && ce_few(head, T, V, H))
    return ce_few_bwd(head, T, V, H, X, static_cast<const uint8_t*>(W), scales, ws2, y, y_bytes, lse, dloss, dX, dx_bf16,
                      ws, s);
  const CePlan p = ce_plan(true, head != kCeBf16 && !codes, T, V, H);
  CeArgs g{};
  CePiece c{};
  if (ce_begin(p, T, V, H, X, ws2, y, y_bytes, ws, &g, &c, s) != 0) return -1;
  g.lse = lse; g.dloss = dloss;
  g.d = reinterpret_cast<uint16_t*>(ws + p.d);
  g.sums = reinterpret_cast<float*>(ws + p.sums);
  g.split_stages = (int)(((p.piece < V ? p.piece : V) + kBK - 1) / kBK);
  const int64_t tt = (T + p.bt - 1) / p.bt, tn = (H + 255) / 256;
  for (int64_t v0 = 0; v0 < V; v0 += p.piece) {
    const int64_t n = V - v0 < p.piece ? V - v0 : p.piece, tiles = (n + 255) / 256 * tt;
    g.v0 = v0;
    g.Vn = (int)n;
    g.add = v0 > 0;
    if (codes) {
      g.w = reinterpret_cast<const uint16_t*>(static_cast<const uint8_t*>(W) + v0 * (H / 2));
      g.scales = scales + v0 * (H / 32);
      if (ce_codes_go<kCeGrad>(g, p.bt, tiles, s) != 0 || ce_codes_go<kCeDx>(g, p.bx, p.groups, s) != 0) return -1;
      continue;
    }
    if (ce_weight(head, W, scales, v0, n, H, ws + p.wbuf, &g.w, s) != 0) return -1;
    if (p.splits > 1) {
      if (ce_go<kCeLogits>(g, p.bt, tiles * p.splits, s) != 0 ||
          ce_grad_go(head, c, lse, dloss, p.ld, p.ld, 0, g.d, g.tlogit, CeTail{}, s) != 0)
        return -1;
    } else if (ce_go<kCeGrad>(g, p.bt, tiles, s) != 0) {
      return -1;
    }
    if (ce_go<kCeDx>(g, p.bx, p.groups, s) != 0) return -1;
  }
  const CeRest rest{W, scales, g.tlogit, nullptr, V, 0};
  auto finish = [&](auto kernel) {
    hipLaunchKernelGGL(kernel, ce_dx_grid(T, H), dim3(128), 0, s, g.sums, 0, (int64_t)0, g.rows, g.count, y, y_bytes, T, V,
                       H, p.bx, (int)tn, g.split_stages, ws2, ws2, rest, dX);
    return ok();
  };
  return ce_dx_by(head, dx_bf16, finish);
}

}  // namespace sq
