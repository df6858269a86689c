// Tile layouts in LDS, their global -> LDS copies, the tile order and the dS
// epilogue, shared by the kernels that feed the matrix cores from them.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "sq_device.h"
#include "sq_gemm_args.h"

namespace sq {

constexpr int kBK = 64;                 // K per LDS stage

// ------------------------------------------------------------------ layouts
// KC: K-contiguous [rows][64] bf16; 16-byte chunk c of row r lives at chunk
// c ^ swz_kc(r), so 8 consecutive rows read at one logical chunk hit 8
// different bank groups.
__device__ __forceinline__ int swz_kc(int r) { return (r ^ (r >> 3)) & 7; }
__device__ __forceinline__ int kc_off(int r, int c) { return r * kBK + ((c ^ swz_kc(r)) << 3); }

// NAT: [BK][R] bf16 with R elements per k-row; 16-byte chunk c of row k lives
// at chunk c ^ swz_nat(k): each of the 4 rows a 16-lane transpose read spans
// lands in its own 64-byte slot.
template <int R>
__device__ __forceinline__ int swz_nat(int k) { return (4 * (k & 7)) & (R / 8 - 1); }
template <int R>
__device__ __forceinline__ int nat_off(int k, int col) {
  return k * R + ((((col >> 3) ^ swz_nat<R>(k))) << 3) + (col & 7);
}

// MFMA operand (8 consecutive k at one m) from a NAT tile: rows
// 16*kk + 8*(lane/32) + 0..7 of column mbase + lane%32.
template <int R>
__device__ __forceinline__ bf16x8 nat_frag(const SQ_LDS uint16_t* s, int kk, int mbase, int lane) {
  const int i = lane & 15, g = lane >> 4;
  const int col = mbase + 16 * (g & 1) + 4 * (i & 3);
  const int row0 = 16 * kk + 8 * (g >> 1) + (i >> 2);
  const v4i16 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((SQ_LDS v4i16*)(s + nat_off<R>(row0, col)));
  const v4i16 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((SQ_LDS v4i16*)(s + nat_off<R>(row0 + 4, col)));
  bf16x8 r;
  __builtin_memcpy(&r, &lo, 8);
  __builtin_memcpy(reinterpret_cast<char*>(&r) + 8, &hi, 8);
  return r;
}

// ------------------------------------------------------------------ DMA issue
// Each thread issues the same set of 16-byte buffer->LDS loads every stage,
// at byte offsets that advance by a fixed step per stage.  The offsets, their
// per-stage step and the K limit of each load are computed once.
//
// KC tile: rows [r0, r0+R) of a [rows_total, ld] bf16 matrix, k in
// [k0, k0+64); one wave instruction fills 8 consecutive LDS rows (1 KiB).
// Rows past the matrix read zeros from the buffer bound; k past kdim is
// masked explicitly on a ragged last stage.
template <int R, int NT>
struct DmaKC {
  static constexpr int kInst = R / 8 / (NT / 64);
  static_assert(kInst * (NT / 64) * 8 == R, "tile rows must split over the waves");
  uint32_t off[kInst];      // byte offset at k0 = 0 (kOOB if the row is outside)
  int klim[kInst];          // the load is valid while k0 < klim
  __device__ __forceinline__ void init(int ld, int rows_total, int kdim, int r0, int tid) {
    const int wave = tid >> 6, lane = tid & 63;
#pragma unroll
    for (int q = 0; q < kInst; ++q) {
      const int blk = q * (NT / 64) + wave;
      const int r = blk * 8 + (lane >> 3);
      const int c = (lane & 7) ^ swz_kc(r);
      const int gr = r0 + r;
      off[q] = gr < rows_total ? (uint32_t)((size_t)gr * ld + c * 8) * 2u : kOOB;
      klim[q] = kdim - c * 8;
    }
  }
  __device__ __forceinline__ void issue(DmaRsrc rs, SQ_LDS uint16_t* s, int k0, bool full,
                                        int wave) const {
    issue_part<0, kInst>(rs, s, k0, full, wave);
  }
  template <int Q0, int Q1>
  __device__ __forceinline__ void issue_part(DmaRsrc rs, SQ_LDS uint16_t* s, int k0, bool full,
                                             int wave) const {
#pragma unroll
    for (int q = Q0; q < Q1; ++q) {
      const int blk = q * (NT / 64) + wave;
      uint32_t o = off[q] + (uint32_t)k0 * 2u;
      if (!full && k0 >= klim[q]) o = kOOB;
      dma16(rs, s + blk * 8 * kBK, o);
    }
  }
};

// NAT tile: k-rows [k0, k0+BK) of a [kdim, ld] bf16 matrix, columns [m0, m0+R).
// Rows past kdim fall past the buffer's end and read zeros; columns past mdim
// only feed accumulators of rows/columns that are never stored.
template <int R, int NT, int BK>
struct DmaNat {
  static constexpr int kCpr = R / 8;                       // chunks per row
  static constexpr int kInst = BK * kCpr / 64 / (NT / 64);
  static_assert(kInst * (NT / 64) * 64 == BK * kCpr, "tile must split over the waves");
  uint32_t off[kInst];
  __device__ __forceinline__ void init(int ld, int mdim, int m0, int tid) {
    const int wave = tid >> 6, lane = tid & 63;
#pragma unroll
    for (int q = 0; q < kInst; ++q) {
      const int blk = q * (NT / 64) + wave;
      const int p = blk * 64 + lane;
      const int k = p / kCpr, pc = p % kCpr;
      const int c = pc ^ swz_nat<R>(k);
      const int gm = m0 + c * 8;
      off[q] = gm < mdim ? (uint32_t)((size_t)k * ld + gm) * 2u : kOOB;
    }
  }
  __device__ __forceinline__ void issue(DmaRsrc rs, SQ_LDS uint16_t* s, uint32_t kstep_bytes,
                                        int wave) const {
    issue_part<0, kInst>(rs, s, kstep_bytes, wave);
  }
  template <int Q0, int Q1>
  __device__ __forceinline__ void issue_part(DmaRsrc rs, SQ_LDS uint16_t* s, uint32_t kstep_bytes,
                                             int wave) const {
#pragma unroll
    for (int q = Q0; q < Q1; ++q) {
      const int blk = q * (NT / 64) + wave;
      const uint32_t o = off[q] == kOOB ? kOOB : off[q] + kstep_bytes;
      dma16(rs, s + blk * 64 * 8, o);
    }
  }
};

// ------------------------------------------------------------------ tile order
// Tile (tm, tn) at position idx of the grouped column-by-column order.
template <int kGroupM>
__device__ __forceinline__ void tile_at(int idx, int tiles_m, int tiles_n, int& tm, int& tn) {
  const int per_group = kGroupM * tiles_n;
  const int group = idx / per_group;
  const int first_m = group * kGroupM;
  const int gm = min(kGroupM, tiles_m - first_m);
  const int in = idx - group * per_group;
  tm = first_m + in % gm;
  tn = in / gm;
}

template <int kGroupM>
__device__ __forceinline__ void tile_of(int bid, int nb, int tiles_m, int tiles_n, int& tm, int& tn) {
  tile_at<kGroupM>(xcd_stretch(bid, nb), tiles_m, tiles_n, tm, tn);
}

// ------------------------------------------------------------------ dS epilogue
// A dS tile's rows are input features j, its columns output features o.  In
// 32x32 MFMA tile (i, j) lane l holds rows 8 q + 4 (l / 32) + 0..3 (q = 0..3)
// of column l % 32, and each group of 4 rows takes its 4 codes from one
// 16-bit pair of the packed plane.  The 16 bytes of codes of row o and the
// tile's 32 features hold the pairs of both lane halves; cw[j TM + i] is that
// chunk, zeros for a row outside the layer.  The chunk starts at byte
// o I / 2 + jb / 2: 16-byte aligned for MXFP4 (I is a multiple of 32), 8-byte
// aligned for NVFP4 (a multiple of 16), which loads it as two halves.
template <int FMT, int TM, int TN>
__device__ __forceinline__ void ds_codes(u32x4 (&cw)[TM * TN], const uint8_t* codes, int O, int I, int r0, int c0,
                                         int lane) {
  const __amdgpu_buffer_rsrc_t rs = make_rsrc(codes, (uint32_t)((size_t)O * (I >> 1)));
#pragma unroll
  for (int j = 0; j < TN; ++j) {
    const int o = c0 + j * 32 + (lane & 31);
#pragma unroll
    for (int i = 0; i < TM; ++i) {
      const int jb = r0 + i * 32;
      const uint32_t off = o < O && jb < I ? (uint32_t)o * (uint32_t)(I >> 1) + (uint32_t)(jb >> 1) : kOOB;
      if constexpr (FMT == kMX) {
        cw[j * TM + i] = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(rs, (int)off, 0, 0));
      } else {
        const u32x2 lo = __builtin_bit_cast(u32x2, __builtin_amdgcn_raw_buffer_load_b64(rs, (int)off, 0, 0));
        const u32x2 hi = __builtin_bit_cast(
            u32x2, __builtin_amdgcn_raw_buffer_load_b64(rs, (int)(off == kOOB ? kOOB : off + 8u), 0, 0));
        cw[j * TM + i] = u32x4{lo[0], lo[1], hi[0], hi[1]};
      }
    }
  }
}

// Products with the codes, summed over each scale block (32 features for
// MXFP4, 16 for NVFP4; the 32 rows of an MFMA tile are split over the two
// lane halves) and stored to dS[o, block].
// INTERIOR: the tile lies inside the layer (every row below I, every column
// below O), so no element needs a range check.
template <int FMT, int TM, int TN, bool INTERIOR>
__device__ __forceinline__ void ds_store(const f32x16 (&acc)[TM][TN], const u32x4 (&cw)[TM * TN], float* dS, int O,
                                         int I, int G, int r0, int c0, int lane) {
  const int lrow = 4 * (lane >> 5);
#pragma unroll
  for (int j = 0; j < TN; ++j) {
    const int o = c0 + j * 32 + (lane & 31);
    const bool o_ok = INTERIOR || o < O;
#pragma unroll
    for (int i = 0; i < TM; ++i) {
      const int jb = r0 + i * 32;          // first feature of this 32-row tile
      float prod[16];
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        // the pair of rows jb + 8 q + lrow .. + 3: bytes 4 q + lrow / 2 of the
        // chunk, decoded two codes per convert (E2M1 values are exact in fp32)
        const uint32_t c = INTERIOR || jb + 8 * q + lrow < I ? cw[j * TM + i][q] >> (4 * lrow) : 0u;
        typedef float f32x2 __attribute__((ext_vector_type(2)));
        const f32x2 v01 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c, 1.0f, 0);
        const f32x2 v23 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c, 1.0f, 1);
        prod[4 * q + 0] = acc[i][j][4 * q + 0] * v01[0];
        prod[4 * q + 1] = acc[i][j][4 * q + 1] * v01[1];
        prod[4 * q + 2] = acc[i][j][4 * q + 2] * v23[0];
        prod[4 * q + 3] = acc[i][j][4 * q + 3] * v23[1];
      }
      if constexpr (FMT == kMX) {
        float s = 0.0f;
#pragma unroll
        for (int r = 0; r < 16; ++r) s += prod[r];
        s += __shfl_xor(s, 32);
        if (lane < 32 && o_ok && (INTERIOR || jb < I)) dS[(size_t)o * G + jb / 32] = s;
      } else {
        float s0 = 0.0f, s1 = 0.0f;
#pragma unroll
        for (int r = 0; r < 8; ++r) { s0 += prod[r]; s1 += prod[8 + r]; }
        s0 += __shfl_xor(s0, 32);
        s1 += __shfl_xor(s1, 32);
        const int b = jb / 16 + (lane >> 5);
        const float s = (lane < 32) ? s0 : s1;
        if (o_ok && (INTERIOR || b * 16 < I)) dS[(size_t)o * G + b] = s;
      }
    }
  }
}

}  // namespace sq
