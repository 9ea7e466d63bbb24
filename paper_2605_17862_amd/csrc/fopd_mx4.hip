// Matrices in microscaled 4-bit floating point, and their product on the matrix cores of gfx950 (CDNA4).
//
//   fopd_mx4_pack       rows of fp32 / bf16 into blocks of 32 entries that share a power of two
//   fopd_mx4_unpack     the values of a packed matrix (both bound by HBM: [151,936, 4096] in bf16 245 - 252 us each, 6.3 TB/s;
//                       in fp32 479 us, 5.9 TB/s, and 1037, 2.7 TB/s)
//   fopd_mx4_few        Out[t, v] = sum_k H[t, k] W[v, k] for few rows of H: the weight streamed past them once
//   fopd_mx4_tiles      the same for many rows, in 256 x 256 tiles
//
// A block holds x_k ~ 2^(s - 127) e_k with e_k one of 0, 0.5, 1, 1.5, 2, 3, 4, 6 and its sign: s is the exponent of the block's
// largest magnitude less 2, which puts that entry at 4 .. 7.99; entries are rounded to nearest, ties to even, those past 6 to 6.
// A block with an infinity or a NaN has s = 255, and all its values are NaN.
//
// A packed matrix of R rows of d entries is in the order in which wavefronts take it.  64 rows and a step of 256 entries are 8704
// bytes, one step of the rows after the other, then the next 64 rows, zeros in the place of entries that do not exist:
//   codes    in v_mfma_scale_f32_16x16x128_f8f6f4 lane 16 q + r holds row r, entries 32 q .. + 31 of 128, in 16 bytes, two entries a
//            byte, the first in the low half.  These fragments follow each other lane by lane, 1 KB each: rows 0 - 15 with
//            entries 0 - 127 of the step, with 128 - 255, rows 16 - 31, ..
//   scales   512 bytes: byte 8 (16 q + r % 16) + 2 (r / 16) + h is that of row r's block 4 h + q of the step: the 8 bytes of a lane are
//            the scales of its fragments, one read where bytes in the order of the matrix would take eight and a shift each.
// A load of a wavefront is then 1 KB in a row, and lies in the LDS as it is read from there, free of bank conflicts.  (Rows of codes
// one after the other, whose fragments are 64-byte pieces of sixteen rows: one row x [151,936, 4096] 69 us.)

#ifndef FOPD_MX4_HIP_
#define FOPD_MX4_HIP_

#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>
#include <type_traits>

#include "fopd_kernels.hip"
#include "fopd_lm_head.hip"
#include "fopd_gemm.hip"

namespace fopd {

constexpr int kMxStep = 256;                  // entries of a step
constexpr int kMxFragment = 1024;             // bytes of 16 rows of 128 entries
constexpr int kMxCodeBytes = 8192;            // of 64 rows and a step
constexpr int kMxScaleBytes = 512;
constexpr int kMxStepBytes = kMxCodeBytes + kMxScaleBytes;
constexpr int kMxThreads = 256;
constexpr int kMxPackThreads = 512;          // of the two kernels that change the order
constexpr int64_t kMxMaxEntries = 1 << 24;     // of a row: its packed bytes are counted in 32 bits

struct Mx4Layout {
  int64_t steps, groups, total;               // groups of 64 rows; bytes
  __host__ __device__ Mx4Layout(int64_t R, int64_t d)
      : steps((d + kMxStep - 1) / kMxStep), groups((R + 63) / 64), total(groups * steps * kMxStepBytes) {}
};

typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef int i32x8 __attribute__((ext_vector_type(8)));

namespace {

// Places in the bytes of 64 rows and a step: of entry k of a row (the byte that holds it), and of the scale of its block b.
__host__ __device__ __forceinline__ int mx_code_at(int row, int k) {
  return ((row >> 4) * 2 + (k >> 7)) * kMxFragment + (16 * ((k >> 5) & 3) + (row & 15)) * 16 + ((k & 31) >> 1);
}
__host__ __device__ __forceinline__ int mx_scale_at(int row, int b) { return kMxCodeBytes + 8 * (16 * (b & 3) + (row & 15)) + 2 * (row >> 4) + (b >> 2); }

// A block whose largest magnitude has these bits: the power it shares, as it is held (magnitudes order as their bits do, infinities and
// NaN above the rest: 255), and 2^(127 - that), with which a product is exact wherever it is not rounded to zero anyway.
__device__ __forceinline__ int mx_block_scale(uint32_t top) {
  const int exponent = static_cast<int>(top >> 23);
  return exponent == 255 ? 255 : max(exponent - 2, 0);
}
__device__ __forceinline__ float mx_block_factor(int scale) {
  return scale == 255 ? 0.f : __uint_as_float(static_cast<uint32_t>(254 - scale) << 23);
}
// Codes of N (4 or 8) entries; of a block of NaN zeros.
template <int N>
__device__ __forceinline__ uint32_t mx_codes(const float* x, int scale) {
  const float f = mx_block_factor(scale);
  uint32_t codes = 0;
  codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, x[0] * f, x[1] * f, 1.f, 0);
  codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, x[2] * f, x[3] * f, 1.f, 1);
  if constexpr (N == 8) {
    codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, x[4] * f, x[5] * f, 1.f, 2);
    codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, x[6] * f, x[7] * f, 1.f, 3);
  }
  return scale == 255 ? 0u : codes;
}
template <int N>
__device__ __forceinline__ uint32_t mx_largest(const float* x, uint32_t top) {
#pragma unroll
  for (int e = 0; e < N; ++e) top = max(top, __float_as_uint(x[e]) & 0x7fffffffu);
  return top;
}

// acc += A B over 128 entries; the scales are bytes SA of sa and SB of sb.
template <int SA, int SB>
__device__ __forceinline__ f32x4 mx_multiply(const i32x4& a, const i32x4& b, const f32x4& acc, int sa, int sb) {
  const i32x8 a8 = __builtin_shufflevector(a, a, 0, 1, 2, 3, -1, -1, -1, -1);
  const i32x8 b8 = __builtin_shufflevector(b, b, 0, 1, 2, 3, -1, -1, -1, -1);
  return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a8, b8, acc, 4, 4, SA, sa, SB, sb);
}

// (the bytes are constants of the instruction; in an unrolled loop one case remains)
__device__ __forceinline__ f32x4 mx_multiply(const i32x4& a, const i32x4& b, const f32x4& acc, int sa, int byte_a, int sb, int byte_b) {
  switch (byte_a * 4 + byte_b) {
    case 0: return mx_multiply<0, 0>(a, b, acc, sa, sb);
    case 1: return mx_multiply<0, 1>(a, b, acc, sa, sb);
    case 2: return mx_multiply<0, 2>(a, b, acc, sa, sb);
    case 3: return mx_multiply<0, 3>(a, b, acc, sa, sb);
    case 4: return mx_multiply<1, 0>(a, b, acc, sa, sb);
    case 5: return mx_multiply<1, 1>(a, b, acc, sa, sb);
    case 6: return mx_multiply<1, 2>(a, b, acc, sa, sb);
    case 7: return mx_multiply<1, 3>(a, b, acc, sa, sb);
    case 8: return mx_multiply<2, 0>(a, b, acc, sa, sb);
    case 9: return mx_multiply<2, 1>(a, b, acc, sa, sb);
    case 10: return mx_multiply<2, 2>(a, b, acc, sa, sb);
    case 11: return mx_multiply<2, 3>(a, b, acc, sa, sb);
    case 12: return mx_multiply<3, 0>(a, b, acc, sa, sb);
    case 13: return mx_multiply<3, 1>(a, b, acc, sa, sb);
    case 14: return mx_multiply<3, 2>(a, b, acc, sa, sb);
    default: return mx_multiply<3, 3>(a, b, acc, sa, sb);
  }
}

}  // namespace

// Workgroup (group - first_group) x steps + step: 64 rows of one step.  A block is 32 / E neighbouring lanes of E entries.
// Columns d and on are zeros and are not read; so are rows past the last.
template <int DT>
__global__ void __launch_bounds__(kMxPackThreads)
fopd_mx4_pack(const void* __restrict__ in, int64_t ld, int64_t R, int64_t d, unsigned char* __restrict__ packed, int64_t first_group) {
  constexpr int E = Elem<DT>::kPerVec, kLanesPerRow = kMxStep / E, kRows = 64 / kLanesPerRow;   // rows of a wavefront at a time
  constexpr int kWaveRows = 64 * 64 / kMxPackThreads;
  const Mx4Layout at(R, d);
  const unsigned steps = static_cast<unsigned>(at.steps), in_launch = blockIdx.x / steps;
  const int64_t group = first_group + in_launch;
  const int step = static_cast<int>(blockIdx.x - in_launch * steps);
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int part = lane % kLanesPerRow;                    // of a row's step
  const int64_t col = static_cast<int64_t>(step) * kMxStep + part * E;
  __shared__ __align__(16) unsigned char bytes[kMxStepBytes];
  const int row0 = wave * kWaveRows + lane / kLanesPerRow;
  u32x4 q[kWaveRows / kRows];
#pragma unroll
  for (int u = 0; u < kWaveRows / kRows; ++u) {
    const int64_t r = group * 64 + row0 + u * kRows;
    q[u] = u32x4{0u, 0u, 0u, 0u};
    if (r >= R || col >= d) continue;
    const char* p = static_cast<const char*>(in) + (r * ld + col) * Elem<DT>::kBytes;
    if (col + E <= d) {
      q[u] = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(p));
    } else {
      float x[E];
#pragma unroll
      for (int e = 0; e < E; ++e) x[e] = col + e < d ? load_elem<DT>(p, e) : 0.f;
      q[u] = pack<DT>(x);
    }
  }
#pragma unroll
  for (int u = 0; u < kWaveRows / kRows; ++u) {
    const int in_group = row0 + u * kRows;
    float x[E];
    unpack<DT>(q[u], x);
    uint32_t top = mx_largest<E>(x, 0);
#pragma unroll
    for (int off = 1; off < 32 / E; off <<= 1) top = max(top, static_cast<uint32_t>(__shfl_xor(static_cast<int>(top), off, 64)));
    const int scale = mx_block_scale(top);
    const uint32_t codes = mx_codes<E>(x, scale);
    unsigned char* to = bytes + mx_code_at(in_group, part * E);
    if constexpr (E == 8) *reinterpret_cast<uint32_t*>(to) = codes;
    else *reinterpret_cast<uint16_t*>(to) = static_cast<uint16_t>(codes);
    if (part % (32 / E) == 0) bytes[mx_scale_at(in_group, part / (32 / E))] = static_cast<unsigned char>(scale);
  }
  __syncthreads();
  u32x4* out = reinterpret_cast<u32x4*>(packed + (group * at.steps + step) * kMxStepBytes);
  for (int k = tid; k < kMxStepBytes / 16; k += kMxPackThreads) __builtin_nontemporal_store(reinterpret_cast<const u32x4*>(bytes)[k], out + k);
}

// Workgroup (group - first_group) x steps + step, eight entries a lane.
template <int DT>
__global__ void __launch_bounds__(kMxPackThreads)
fopd_mx4_unpack(const unsigned char* __restrict__ packed, int64_t R, int64_t d, void* __restrict__ out, int64_t ldo,
                int64_t first_group) {
  typedef float f32x2v __attribute__((ext_vector_type(2)));
  const Mx4Layout at(R, d);
  const unsigned steps = static_cast<unsigned>(at.steps), in_launch = blockIdx.x / steps;
  const int64_t group = first_group + in_launch;
  const int step = static_cast<int>(blockIdx.x - in_launch * steps);
  const int tid = threadIdx.x, part = tid & 31;
  const int64_t col = static_cast<int64_t>(step) * kMxStep + part * 8, row0 = group * 64 + (tid >> 5);
  __shared__ __align__(16) unsigned char bytes[kMxStepBytes];
  const u32x4* from = reinterpret_cast<const u32x4*>(packed + (group * at.steps + step) * kMxStepBytes);
  for (int k = tid; k < kMxStepBytes / 16; k += kMxPackThreads) reinterpret_cast<u32x4*>(bytes)[k] = __builtin_nontemporal_load(from + k);
  __syncthreads();
  if (col >= d) return;
#pragma unroll
  for (int u = 0; u < 64 * 32 / kMxPackThreads; ++u) {
    const int64_t r = row0 + (kMxPackThreads / 32) * u;
    if (r >= R) break;
    const int in_group = (tid >> 5) + (kMxPackThreads / 32) * u;
    const uint32_t codes = *reinterpret_cast<const uint32_t*>(bytes + mx_code_at(in_group, part * 8));
    const int scale = bytes[mx_scale_at(in_group, part >> 2)];
    const float unit = scale == 255 ? __builtin_nanf("") : __uint_as_float(scale == 0 ? 0x00400000u : static_cast<uint32_t>(scale) << 23);
    const f32x2v p0 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, 1.f, 0), p1 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, 1.f, 1);
    const f32x2v p2 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, 1.f, 2), p3 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, 1.f, 3);
    const float x[8] = {p0.x * unit, p0.y * unit, p1.x * unit, p1.y * unit, p2.x * unit, p2.y * unit, p3.x * unit, p3.y * unit};
    char* o = static_cast<char*>(out) + (r * ldo + col) * Elem<DT>::kBytes;
    if (col + 8 <= d) {
      u32x4* ov = reinterpret_cast<u32x4*>(o);
      if constexpr (DT == FOPD_BF16) {
        __builtin_nontemporal_store(pack<FOPD_BF16>(x), ov);
      } else {
        __builtin_nontemporal_store(pack<FOPD_F32>(x), ov);
        __builtin_nontemporal_store(pack<FOPD_F32>(x + 4), ov + 1);
      }
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if (col + e < d) store_elem<DT>(o, e, x[e]);
    }
  }
}

// Few rows of H, or few of W: workgroup (x, y) has vocabulary rows 64 x .. + 63 and the up to 64 rows 64 y .. of H, 16 BLOCKS of them
// at most.  Its wavefronts take the steps in turn and their sums are added
// in the LDS; the weight goes from memory to the registers of the one wavefront that needs it.  Bound by HBM: one row 48 us = 6.8
// TB/s; with results to write the rate falls to that of mixed traffic, 45 rows (14 MB of bf16) 65 us = 5.3 TB/s.  Results of 49 - 64
// rows past the caches: 64 x 32,000 18.2 -> 17.8 us, 128 x 24,000 in fp32, d = 512, 13.0 -> 11.6, of fewer no faster (30 x 151,936 63.8 / 65.1).  (H in the LDS of one workgroup a compute unit, whose
// wavefronts stream sixteen vocabulary rows each: 1 / 45 / 64 rows 58.6 / 72 / 76 us where this takes 54 / 70 / 75; eight
// wavefronts a workgroup: 95 for one row, with the codes row by row, where four took 69.)
// RAW (BLOCKS 1): the up to 16 rows of H as they are, of that type with pitch ldh.  A fragment's lane holds one row's block, so it
// quantises that block by itself, while the weight is on its way, and the launch that packs H falls away.  The same bits either way.
constexpr int kMxPacked = -1;

template <int DT, int BLOCKS, bool CACHED, int RAW = kMxPacked>
__global__ void __launch_bounds__(kMxThreads)
fopd_mx4_few(const unsigned char* __restrict__ W, int64_t V, const void* __restrict__ H, int64_t ldh, int64_t T, int64_t d,
             void* __restrict__ out, int64_t ldo) {
  static_assert(RAW == kMxPacked || BLOCKS == 1, "sixteen rows at most");
  constexpr int kWaves = kMxThreads / 64;
  __shared__ __align__(16) float sums[kWaves / 2][16 * BLOCKS][64 + 4];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int steps = static_cast<int>(Mx4Layout(V, d).steps);
  const int64_t v0 = static_cast<int64_t>(blockIdx.x) * 64, t0 = static_cast<int64_t>(blockIdx.y) * 64;
  const unsigned char* w = W + (v0 >> 6) * steps * kMxStepBytes;
  const unsigned char* h = static_cast<const unsigned char*>(H) + (RAW == kMxPacked ? (t0 >> 6) * steps * kMxStepBytes : 0);
  f32x4 acc[4][BLOCKS];
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int j = 0; j < BLOCKS; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
  for (int s = wave; s < steps; s += kWaves) {
    const unsigned char *ws = w + static_cast<int64_t>(s) * kMxStepBytes, *hs = h + static_cast<int64_t>(s) * kMxStepBytes;
    i32x4 a[4][2], b[BLOCKS][2];
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int ks = 0; ks < 2; ++ks) a[i][ks] = __builtin_bit_cast(i32x4, load_vec<CACHED>(reinterpret_cast<const u32x4*>(ws + (2 * i + ks) * kMxFragment) + lane));
    const uint2 sa = reinterpret_cast<const uint2*>(ws + kMxCodeBytes)[lane];
    uint64_t sb;
    if constexpr (RAW == kMxPacked) {
#pragma unroll
      for (int j = 0; j < BLOCKS; ++j)
#pragma unroll
        for (int ks = 0; ks < 2; ++ks) b[j][ks] = reinterpret_cast<const i32x4*>(hs + (2 * j + ks) * kMxFragment)[lane];
      sb = reinterpret_cast<const uint64_t*>(hs + kMxCodeBytes)[lane];
    } else {
      constexpr int E = Elem<RAW>::kPerVec;
      const char* row = static_cast<const char*>(H) + std::min<int64_t>(lane & 15, T - 1) * ldh * Elem<RAW>::kBytes;
      u32x4 raw[2][32 / E];
#pragma unroll
      for (int ks = 0; ks < 2; ++ks) {
        const int64_t k = static_cast<int64_t>(s) * kMxStep + 128 * ks + 32 * (lane >> 4);
#pragma unroll
        for (int c = 0; c < 32 / E; ++c) {
          const char* p = row + (k + c * E) * Elem<RAW>::kBytes;
          raw[ks][c] = u32x4{0u, 0u, 0u, 0u};
          if (k + (c + 1) * E <= d) {
            raw[ks][c] = *reinterpret_cast<const u32x4*>(p);
          } else if (k + c * E < d) {
            float x[E];
#pragma unroll
            for (int e = 0; e < E; ++e) x[e] = k + c * E + e < d ? load_elem<RAW>(p, e) : 0.f;
            raw[ks][c] = pack<RAW>(x);
          }
        }
      }
      sb = 0;
#pragma unroll
      for (int ks = 0; ks < 2; ++ks) {
        float x[32];
        uint32_t top = 0;
#pragma unroll
        for (int c = 0; c < 32 / E; ++c) {
          unpack<RAW>(raw[ks][c], x + c * E);
          top = mx_largest<E>(x + c * E, top);
        }
        const int scale = mx_block_scale(top);
#pragma unroll
        for (int c = 0; c < 4; ++c) b[0][ks][c] = static_cast<int>(mx_codes<8>(x + 8 * c, scale));
        sb |= static_cast<uint64_t>(scale) << (8 * ks);
      }
    }
#pragma unroll
    for (int ks = 0; ks < 2; ++ks)
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < BLOCKS; ++j)
          acc[i][j] = mx_multiply(a[i][ks], b[j][ks], acc[i][j], static_cast<int>(i < 2 ? sa.x : sa.y), 2 * (i & 1) + ks,
                                  static_cast<int>(j < 2 ? sb : sb >> 32), 2 * (j & 1) + ks);
  }
  // register r of acc[i][j]: vocabulary row 16 i + 4 (lane / 16) + r, row 16 j + lane % 16 of H
  // (the upper half of the wavefronts hands its sums to the lower one)
  auto place = [&](int i, int j) { return reinterpret_cast<f32x4*>(&sums[wave & (kWaves / 2 - 1)][16 * j + (lane & 15)][16 * i + 4 * (lane >> 4)]); };
  if (wave >= kWaves / 2) {
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int j = 0; j < BLOCKS; ++j) *place(i, j) = acc[i][j];
  }
  __syncthreads();
  if (wave < kWaves / 2) {
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int j = 0; j < BLOCKS; ++j) *place(i, j) += acc[i][j];
  }
  __syncthreads();
  for (int k = tid; k < 16 * BLOCKS * 16; k += kMxThreads) {            // four neighbouring results each
    const int t = k >> 4, v = 4 * (k & 15);
    f32x4 z = *reinterpret_cast<const f32x4*>(&sums[0][t][v]);
#pragma unroll
    for (int u = 1; u < kWaves / 2; ++u) z += *reinterpret_cast<const f32x4*>(&sums[u][t][v]);
    if (t0 + t >= T || v0 + v >= V) continue;
    char* o = static_cast<char*>(out) + ((t0 + t) * ldo + v0 + v) * Elem<DT>::kBytes;
    if (v0 + v + 4 <= V) {
      typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
      u32x2* o16 = reinterpret_cast<u32x2*>(o);
      f32x4* o32 = reinterpret_cast<f32x4*>(o);
      const u32x2 z16 = {pack_bf16x2(z[0], z[1]), pack_bf16x2(z[2], z[3])};
      if constexpr (DT == FOPD_BF16 && BLOCKS < 4) *o16 = z16;
      else if constexpr (DT == FOPD_BF16) __builtin_nontemporal_store(z16, o16);
      else if constexpr (BLOCKS < 4) *o32 = z;
      else __builtin_nontemporal_store(z, o32);
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (v0 + v + e < V) store_elem<DT>(o, e, z[e]);
    }
  }
}

// ---- some rows of H ------------------------------------------------------------------------------------------------
// Up to 16 BLOCKS rows of H and a workgroup for every 128 vocabulary rows: the weight is read once, by the wavefront that
// multiplies it (32 rows of it), straight into registers a step of 256 entries ahead; H's step, 8.5 KB of 64 rows, goes through one of two
// places in the LDS, so the workgroup reads it once where fopd_mx4_few's wavefronts all would.  Two workgroups a compute unit (of 8 blocks:
// 206 registers; with at most 168, for three, they spill: 297 us where this takes 83).  Bound by HBM, reads and writes mixed: 128 rows x
// 151,936, d = 4096, 331 MB read and 39 written, 76 us = 4.9 TB/s (81 with the launch that packs H; so counted, fopd_mx4_tiles, half of whose tile is columns that do not exist, 111;
// fopd_mx4_few with eight blocks 106).  H's loads are asked for first, since they are waited for first, to be placed: the other way round the
// wait took in the weight's, 128 x 40,000 32.7 us instead of 27.5.  Weights two steps ahead: no faster (128 x 151,936 88).  Ordinary
// stores: 93.
template <int BLOCKS>
struct MxStream {
  static constexpr int kBlocks = BLOCKS;
  static constexpr int kGroups = (BLOCKS + 3) / 4;                     // of 64 rows of H
  static constexpr int kVocabulary = 128;                              // rows of W a workgroup
  static constexpr int kStage = kGroups * kMxStepBytes;
  static constexpr int kSums = 64 * (kVocabulary + 4) * 4;
  static constexpr int kLds = 2 * kStage > kSums ? 2 * kStage : kSums;
};

template <int DT, int BLOCKS, bool CACHED>
__global__ void __launch_bounds__(kMxThreads, 2)
fopd_mx4_stream(const unsigned char* __restrict__ W, int64_t V, const unsigned char* __restrict__ H, int64_t T, int64_t d,
                void* __restrict__ out, int64_t ldo) {
  using S = MxStream<BLOCKS>;
  static_assert(kMxThreads == 4 * 64, "four wavefronts of 32 vocabulary rows");
  __shared__ __align__(16) unsigned char lds[S::kLds];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int steps = static_cast<int>(Mx4Layout(V, d).steps);
  const int64_t v0 = static_cast<int64_t>(blockIdx.x) * S::kVocabulary;
  // (groups that do not exist: the last one again, whose results are not written)
  const unsigned char* w = W + std::min<int64_t>((v0 >> 6) + (wave >> 1), ((V + 63) >> 6) - 1) * steps * kMxStepBytes;
  const int last_group = static_cast<int>((T + 63) >> 6) - 1;
  f32x4 acc[2][BLOCKS];
#pragma unroll
  for (int i = 0; i < 2; ++i)
#pragma unroll
    for (int j = 0; j < BLOCKS; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};

  struct Weight { i32x4 codes[2][2]; uint32_t scales; };
  constexpr int kVecs = kMxStepBytes / 16;                             // of a step of 64 rows
  constexpr int kLoads = (S::kGroups * kVecs + kMxThreads - 1) / kMxThreads;
  auto load_weight = [&](int s, Weight& a) {
    const unsigned char* ws = w + static_cast<int64_t>(s) * kMxStepBytes;
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
      for (int ks = 0; ks < 2; ++ks)
        a.codes[i][ks] = __builtin_bit_cast(i32x4, load_vec<CACHED>(reinterpret_cast<const u32x4*>(ws + (4 * (wave & 1) + 2 * i + ks) * kMxFragment) + lane));
    a.scales = *reinterpret_cast<const uint32_t*>(ws + kMxCodeBytes + 8 * lane + 4 * (wave & 1));
  };
  auto load_rows = [&](int s, u32x4 (&h)[kLoads]) {
#pragma unroll
    for (int u = 0; u < kLoads; ++u) {
      const int k = tid + u * kMxThreads, g = k / kVecs;
      if (k < S::kGroups * kVecs)
        h[u] = *reinterpret_cast<const u32x4*>(H + (static_cast<int64_t>(min(g, last_group)) * steps + s) * kMxStepBytes + (k - g * kVecs) * 16);
    }
  };
  auto place_rows = [&](int s, const u32x4 (&h)[kLoads]) {
#pragma unroll
    for (int u = 0; u < kLoads; ++u) {
      const int k = tid + u * kMxThreads;
      if (k < S::kGroups * kVecs) *reinterpret_cast<u32x4*>(lds + (s & 1) * S::kStage + k * 16) = h[u];
    }
  };
  auto meet = [&] {
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup", "local");
    __builtin_amdgcn_s_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup", "local");
  };
  auto multiply = [&](int s, const Weight& a) {
    const unsigned char* hs = lds + (s & 1) * S::kStage;
#pragma unroll
    for (int g = 0; g < S::kGroups; ++g) {
      const uint64_t sb = reinterpret_cast<const uint64_t*>(hs + g * kMxStepBytes + kMxCodeBytes)[lane];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        if (4 * g + j >= BLOCKS) break;
#pragma unroll
        for (int ks = 0; ks < 2; ++ks) {
          const i32x4 b = reinterpret_cast<const i32x4*>(hs + g * kMxStepBytes + (2 * j + ks) * kMxFragment)[lane];
#pragma unroll
          for (int i = 0; i < 2; ++i)
            acc[i][4 * g + j] = mx_multiply(a.codes[i][ks], b, acc[i][4 * g + j], static_cast<int>(a.scales), 2 * i + ks,
                                            static_cast<int>(j < 2 ? sb : sb >> 32), 2 * (j & 1) + ks);
        }
      }
    }
  };

  Weight a0, a1;
  u32x4 h[kLoads];
  auto step = [&](int s, const Weight& now, Weight& next) {
    if (s + 1 < steps) {
      load_rows(s + 1, h);                                               // (they are waited for first)
      load_weight(s + 1, next);
    }
    __builtin_amdgcn_sched_barrier(0);
    multiply(s, now);
    __builtin_amdgcn_sched_barrier(0);
    if (s + 1 < steps) place_rows(s + 1, h);
    meet();
  };
  load_rows(0, h);
  load_weight(0, a0);
  place_rows(0, h);
  meet();
  for (int s = 0; s < steps; s += 2) {
    step(s, a0, a1);
    if (s + 1 < steps) step(s + 1, a1, a0);
  }
  // register r of acc[i][j]: vocabulary row 32 wave + 16 i + 4 (lane / 16) + r, row 16 j + lane % 16 of H; 64 rows at a time
  float(*sums)[S::kVocabulary + 4] = reinterpret_cast<float(*)[S::kVocabulary + 4]>(lds);
#pragma unroll
  for (int g = 0; g < S::kGroups; ++g) {
    constexpr int kRows = 64;
    if (g > 0) meet();
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      if (4 * g + j >= BLOCKS) break;
#pragma unroll
      for (int i = 0; i < 2; ++i) *reinterpret_cast<f32x4*>(&sums[16 * j + (lane & 15)][32 * wave + 16 * i + 4 * (lane >> 4)]) = acc[i][4 * g + j];
    }
    meet();
    const int rows = min(kRows, 16 * (BLOCKS - 4 * g));
    for (int k = tid; k < rows * (S::kVocabulary / 4); k += kMxThreads) {
      const int t = k / (S::kVocabulary / 4), v = 4 * (k % (S::kVocabulary / 4));
      const f32x4 z = *reinterpret_cast<const f32x4*>(&sums[t][v]);
      if (64 * g + t >= T || v0 + v >= V) continue;
      char* o = static_cast<char*>(out) + ((64 * g + t) * ldo + v0 + v) * Elem<DT>::kBytes;
      if (v0 + v + 4 <= V) {
        typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
        const u32x2 z16 = {pack_bf16x2(z[0], z[1]), pack_bf16x2(z[2], z[3])};
        if constexpr (DT == FOPD_BF16) __builtin_nontemporal_store(z16, reinterpret_cast<u32x2*>(o));
        else __builtin_nontemporal_store(z, reinterpret_cast<f32x4*>(o));
      } else {
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if (v0 + v + e < V) store_elem<DT>(o, e, z[e]);
      }
    }
  }
}

// ---- many rows of H: 256 x 256 tiles -------------------------------------------------------------------------------
// The loop of fopd_lm_head.hip (matrix_step) on 4-bit operands: a half tile is 16 KB of a step there and here, 128 rows of 64 bf16 or
// 256 4-bit entries, the fragments are the same 16 bytes a lane and the instruction takes as long; a product does four times the
// work.  A wavefront fetches one 16-row block, two fragments, of each half tile.  The scales of a step are one more load
// a wavefront, 512 bytes of 64 rows (the four groups of A's tile, then B's four), requested with B0 and, like B0, all
// read in the step's first slot:
//
//   phase   reads              multiplies   requests                              waits for (besides its own LDS reads)
//     1     B0, A0, scales     A0 x B0      A1 of the next step
//     2     B1                 A0 x B1      B0 and scales of the next but one     A1 of this step                    (12 loads stay in flight)
//     3     A1                 A1 x B1      A0 of the next but one
//     4                        A1 x B0      B1 of the next but one                B0, scales, A0, B1 of the next step    (9)

// 4096 rows x 151,936, d = 4096: 1.19 - 1.25 ms = 4.1 - 4.3 PFLOP/s (three times the rate of a large bf16 product), d = 32,768 4.85; the instruction
// alone, operands in registers, reaches 8.7.  Counters: 2.0 GHz, matrix cores 0.51 busy, LDS conflicts 3.5 %; with all loads to one
// step, so from the L2, 6 % less time: what is left is the slots, in which four wavefronts' reads through the LDS take as long as the
// other four's products.  Slower or no faster: the 32 x 32 x 64 instruction with a layout for it (9.8 PFLOP/s alone; 1246 us where this took
// 1219, and 45 rows 78 us where fopd_mx4_few took 70), B0 and the scales read a phase ahead, in the phase without reads (1242 /
// 1234), four wavefronts of 128 x 128, whose LDS reads are a third fewer but whose requests hold up the only
// wavefront a SIMD has (1310 / 1225; walking the tiles, with spilled registers, 1454), non-temporal loads of the weight (1287 / 1244; with one tile
// of rows 3 % faster).  Codes row by row instead of in fragments: 1240 / 1220.

constexpr int kMxScaleLds = 8 * 1024;                     // scales of a step (half of each 1 KB is not read)
constexpr int kMxTileLds = kLoopLdsBytes + 2 * kMxScaleLds;

namespace {

// One operand's half tiles: the wavefront's 16 rows of each.
struct MxSource {
  const unsigned char* base;
  int groups;
  const char* src[2];
  __device__ __forceinline__ void locate(int r0, int steps, int wave) {
#pragma unroll
    for (int h = 0; h < 2; ++h)
      src[h] = reinterpret_cast<const char*>(base) + static_cast<int64_t>(min((r0 >> 6) + 2 * h + (wave >> 2), groups - 1)) * steps * kMxStepBytes +
               (wave & 3) * (2 * kMxFragment);
  }
};

struct MxLoader {
  MxSource a, b;
  int steps, wave;
  uint32_t lds, scale_lds;
  uint32_t code_lane, scale_lane;                          // lane's bytes in a fragment and in the scales, from the tile's first step on
  const char* scale_src;
  uint32_t at;                                             // bytes of the steps before this one
  __device__ __forceinline__ void locate(const GemmTile& t) {
    a.locate(t.m0, steps, wave);
    b.locate(t.n0, steps, wave);
    const int group = wave < 4 ? min((t.m0 >> 6) + wave, a.groups - 1) : min((t.n0 >> 6) + wave - 4, b.groups - 1);
    scale_src = reinterpret_cast<const char*>(wave < 4 ? a.base : b.base) + static_cast<int64_t>(group) * steps * kMxStepBytes + kMxCodeBytes;
    at = 0;
  }
  __device__ __forceinline__ void step(bool on = true) { at += on ? kMxStepBytes : 0; }
  __device__ __forceinline__ void request(int half, int buf) {
    const uint32_t dst = lds + buf * kStepBytes + half * kHalfBytes;
    const char* src = half == kHalfA0 ? a.src[0] : half == kHalfA1 ? a.src[1] : half == kHalfB0 ? b.src[0] : b.src[1];
    load_to_lds(src, code_lane + at, dst);
    load_to_lds(src, code_lane + at + kMxFragment, dst + kMxFragment);
    if (half == kHalfB0) load_to_lds(scale_src, scale_lane + at, scale_lds + buf * kMxScaleLds);
  }
};

// Where the wavefront's fragments of a step lie in the LDS.
struct MxFragments {
  uint32_t a_off, b_off;
  __device__ __forceinline__ explicit MxFragments(const MatrixPlace& p) {
    const int lane = threadIdx.x & 63;
    a_off = p.wm * (8 * kMxFragment) + lane * 16;
    b_off = 2 * kHalfBytes + p.wn * (4 * kMxFragment) + lane * 16;
  }
  __device__ __forceinline__ i32x4 a(const unsigned char* step, int half, int i, int ks) const {
    return *reinterpret_cast<const i32x4*>(step + half * kHalfBytes + a_off + (2 * i + ks) * kMxFragment);
  }
  __device__ __forceinline__ i32x4 b(const unsigned char* step, int half, int j, int ks) const {
    return *reinterpret_cast<const i32x4*>(step + half * kHalfBytes + b_off + (2 * j + ks) * kMxFragment);
  }
};

typedef f32x4 MxAcc[2][4][2][2];                          // [A half][16-row block][B half][16-row block]

template <int FLIGHT>
__device__ __forceinline__ void mx_wait() {
  static_assert(FLIGHT <= 63, "the counter's range");
  asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"(FLIGHT) : "memory");
}

__device__ __forceinline__ void mx_product(MxAcc& acc, int a, int b, const i32x4 (&fa)[4][2], const i32x4 (&fb)[2][2], uint2 sa, uint32_t sb) {
#pragma unroll
  for (int ks = 0; ks < 2; ++ks)
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int j = 0; j < 2; ++j)
        acc[a][i][b][j] = mx_multiply(fa[i][ks], fb[j][ks], acc[a][i][b][j], static_cast<int>(i < 2 ? sa.x : sa.y), 2 * (i & 1) + ks,
                                      static_cast<int>(sb), 2 * j + ks);
}

// STORES: stores of the tile before that are still in flight behind the requests that this step waits for (loads and stores
// count and end in order).
template <int STORES, typename Request>
__device__ __forceinline__ void mx_step(MxAcc& acc, const MxFragments& frags, const unsigned char* here, const unsigned char* scales_a,
                                        const unsigned char* scales_b, Request request) {
  i32x4 fa[4][2], fb0[2][2], fb1[2][2];
#pragma unroll
  for (int j = 0; j < 2; ++j)
#pragma unroll
    for (int ks = 0; ks < 2; ++ks) fb0[j][ks] = frags.b(here, 0, j, ks);
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int ks = 0; ks < 2; ++ks) fa[i][ks] = frags.a(here, 0, i, ks);
  const uint2 sa0 = *reinterpret_cast<const uint2*>(scales_a), sa1 = *reinterpret_cast<const uint2*>(scales_a + 2048);
  const uint32_t sb0 = *reinterpret_cast<const uint32_t*>(scales_b), sb1 = *reinterpret_cast<const uint32_t*>(scales_b + 2048);
  request(kHalfA1);
  asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
  slot_end();
  mx_product(acc, 0, 0, fa, fb0, sa0, sb0);
  slot_end();
#pragma unroll
  for (int j = 0; j < 2; ++j)
#pragma unroll
    for (int ks = 0; ks < 2; ++ks) fb1[j][ks] = frags.b(here, 1, j, ks);
  request(kHalfB0);
  mx_wait<12 + STORES>();
  slot_end();
  mx_product(acc, 0, 1, fa, fb1, sa0, sb1);
  slot_end();
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int ks = 0; ks < 2; ++ks) fa[i][ks] = frags.a(here, 1, i, ks);
  request(kHalfA0);
  asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
  slot_end();
  mx_product(acc, 1, 1, fa, fb1, sa1, sb1);
  slot_end();
  request(kHalfB1);
  mx_wait<9 + STORES>();
  slot_end();
  mx_product(acc, 1, 0, fa, fb0, sa1, sb0);
  slot_end();
}

// Lanes 8 .. 15 of each sixteen of `low` change places with lanes 0 .. 7 of `high`.
__device__ __forceinline__ void swap_eights(uint32_t& low, uint32_t& high) {
  const int l = static_cast<int>(low), h = static_cast<int>(high);
  low = static_cast<uint32_t>(__builtin_amdgcn_update_dpp(l, h, 0x128, 0xf, 0xc, false));      // row_ror:8, lanes 8 .. 15
  high = static_cast<uint32_t>(__builtin_amdgcn_update_dpp(h, l, 0x128, 0xf, 0x3, false));     // lanes 0 .. 7
}

// 16 bytes of results of row t from column v on.
template <int DT, bool WHOLE>
__device__ __forceinline__ void mx_store(void* out, int64_t ldo, int64_t t, int64_t v, int64_t T, int64_t V, const u32x4& q) {
  constexpr int E = Elem<DT>::kPerVec;
  char* o = static_cast<char*>(out) + (t * ldo + v) * Elem<DT>::kBytes;
  if (WHOLE || (t < T && v + E <= V)) {
    __builtin_nontemporal_store(q, reinterpret_cast<u32x4*>(o));
  } else if (t < T) {
    float x[E];
    unpack<DT>(q, x);
#pragma unroll
    for (int e = 0; e < E; ++e)
      if (v + e < V) store_elem<DT>(o, e, x[e]);
  }
}

// Register r of acc[a][i][b][j] is vocabulary row 128 a + 64 wm + 16 i + 4 (lane / 16) + r of the tile, row 128 b + 32 wn + 16 j +
// lane % 16 of H's.  Lanes change places until a store writes whole 128-byte lines of eight rows, 16 bytes a lane.
template <int DT, bool WHOLE>
__device__ __forceinline__ void mx_store_block(const MxAcc& acc, const MatrixPlace& place, int m0, int n0, int64_t T, int64_t V,
                                               void* __restrict__ out, int64_t ldo) {
  const int lane = threadIdx.x & 63, n = lane & 7, upper = (lane >> 3) & 1, q = lane >> 4;
#pragma unroll
  for (int a = 0; a < 2; ++a)
#pragma unroll
    for (int b = 0; b < 2; ++b)
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        const int64_t t = n0 + 128 * b + 32 * place.wn + 16 * j + n;
        const int64_t v = m0 + 128 * a + 64 * place.wm;
        if constexpr (DT == FOPD_F32) {
#pragma unroll
          for (int i = 0; i < 4; i += 2) {
            u32x4 x = __builtin_bit_cast(u32x4, acc[a][i][b][j]), y = __builtin_bit_cast(u32x4, acc[a][i + 1][b][j]);
#pragma unroll
            for (int r = 0; r < 4; ++r) {
              uint32_t lo = x[r], hi = y[r];
              swap_eights(lo, hi);
              x[r] = lo;
              y[r] = hi;
            }
            mx_store<DT, WHOLE>(out, ldo, t, v + 16 * (i + upper) + 4 * q, T, V, x);
            mx_store<DT, WHOLE>(out, ldo, t + 8, v + 16 * (i + upper) + 4 * q, T, V, y);
          }
        } else {
          u32x4 u[2];                                      // columns 8 q .. + 7 of the first and of the second 32
#pragma unroll
          for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int r = 0; r < 2; ++r) {
              const f32x4 &x = acc[a][2 * h][b][j], &y = acc[a][2 * h + 1][b][j];
              const auto s32 = __builtin_amdgcn_permlane32_swap(pack_bf16x2(x[2 * r], x[2 * r + 1]), pack_bf16x2(y[2 * r], y[2 * r + 1]), false, false);
              const auto s16 = __builtin_amdgcn_permlane16_swap(s32[0], s32[1], false, false);
              u[h][r] = s16[0];
              u[h][r + 2] = s16[1];
            }
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            uint32_t lo = u[0][r], hi = u[1][r];
            swap_eights(lo, hi);
            u[0][r] = lo;
            u[1][r] = hi;
          }
          mx_store<DT, WHOLE>(out, ldo, t, v + 32 * upper + 8 * q, T, V, u[0]);
          mx_store<DT, WHOLE>(out, ldo, t + 8, v + 32 * upper + 8 * q, T, V, u[1]);
        }
      }
}

}  // namespace

// Launched as fopd_gemm_nt is (TileWalk): m the vocabulary, n the rows of H.
template <int DT, bool WALK>
__global__ void __launch_bounds__(kLmThreads)
fopd_mx4_tiles(const unsigned char* __restrict__ W, int64_t V, const unsigned char* __restrict__ H, int64_t T, int64_t d,
               void* __restrict__ out, int64_t ldo, int tiles_m, int tiles_n) {
  extern __shared__ __align__(16) unsigned char mx_smem[];
  const int steps = static_cast<int>(Mx4Layout(V, d).steps);
  TileWalk<true, WALK> walk = {tiles_m, tiles_n, steps, 1};
  GemmTile tile;
  if (!walk.first(tile, blockIdx.x)) return;               // whole workgroup, before any barrier

  const MatrixPlace mine = matrix_place(mx_smem);
  const MxFragments frags(mine);
  const int lane = threadIdx.x & 63, wave = mine.wm * 4 + mine.wn;
  const unsigned char* scales = mx_smem + kLoopLdsBytes;
  const unsigned char* scales_a = scales + mine.wm * 1024 + lane * 8;
  const unsigned char* scales_b = scales + (4 + (mine.wn >> 1)) * 1024 + lane * 8 + (mine.wn & 1) * 4;
  MxLoader load = {{W, static_cast<int>((V + 63) >> 6), {}}, {H, static_cast<int>((T + 63) >> 6), {}}, steps, wave, mine.lds,
                   mine.lds - wave * 2048u + kLoopLdsBytes + wave * 1024u, lane * 16u, (lane & 31) * 16u, nullptr, 0};

  // the stream of steps, as matrix_tiles
  constexpr int kStores = DT == FOPD_F32 ? 32 : 16;        // of a whole tile, by a wavefront
  GemmTile ahead_tile = tile;
  TileWalk<true, WALK> ahead = walk;
  int left = steps;
  load.locate(tile);
  auto advance = [&]() {
    if constexpr (!WALK) {
      const bool more = left > 1;
      left -= more ? 1 : 0;
      load.step(more);
    } else if (--left > 0) {
      load.step();
    } else if (ahead.next(ahead_tile)) {
      left = steps;
      load.locate(ahead_tile);
    } else {
      left = 1;                                            // the last step again, never read
    }
  };
#pragma unroll
  for (int buf = 0; buf < 2; ++buf) {
    load.request(kHalfB0, buf);
    load.request(kHalfA0, buf);
    load.request(kHalfB1, buf);
    if (buf == 0) {
      load.request(kHalfA1, buf);
      advance();
    }
  }
  asm volatile("s_waitcnt vmcnt(9)" ::: "memory");
  slot_end();
  if (mine.wm == 1) slot_end();
  int cur = 0;
  bool stored = false;
  MxAcc acc;
  while (true) {
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int b = 0; b < 2; ++b)
#pragma unroll
          for (int j = 0; j < 2; ++j) acc[h][i][b][j] = f32x4{0.f, 0.f, 0.f, 0.f};
    auto run = [&](auto stores_tag, auto switch_tag) {
      mx_step<decltype(stores_tag)::value>(acc, frags, mx_smem + cur * kStepBytes, scales_a + cur * kMxScaleLds, scales_b + cur * kMxScaleLds,
                                           [&](int half) {
        load.request(half, half == kHalfA1 ? 1 - cur : cur);
        if (half == kHalfA1) {
          if constexpr (decltype(switch_tag)::value) {
            advance();
          } else {
            --left;
            load.step();
          }
        }
      });
      cur = 1 - cur;
    };
    typedef std::integral_constant<int, 0> None;
    typedef std::integral_constant<int, kStores> Some;
    int kt = steps;
    if constexpr (!WALK) {
      for (; kt > 0; --kt) run(None(), std::true_type());
      matrix_end(mine);
      if (tile.m0 + kGemmTile <= V && tile.n0 + kGemmTile <= T) mx_store_block<DT, true>(acc, mine, tile.m0, tile.n0, T, V, out, ldo);
      else mx_store_block<DT, false>(acc, mine, tile.m0, tile.n0, T, V, out, ldo);
      return;
    }
    if (stored) {
      if (left > 1) run(Some(), std::false_type());
      else run(Some(), std::true_type());
      --kt;
    }
    while (kt > 0) {
      const int plain = min(kt, left - 1);
      for (int i = 0; i < plain; ++i) run(None(), std::false_type());
      kt -= plain;
      if (kt > 0) {
        run(None(), std::true_type());
        --kt;
      }
    }
    stored = tile.m0 + kGemmTile <= V && tile.n0 + kGemmTile <= T;
    if (stored) {
      mx_store_block<DT, true>(acc, mine, tile.m0, tile.n0, T, V, out, ldo);
    } else {                                               // an unknown number of stores: waited for
      mx_store_block<DT, false>(acc, mine, tile.m0, tile.n0, T, V, out, ldo);
      asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    }
    if (!walk.next(tile)) break;
  }
  matrix_end(mine);
}

}  // namespace fopd

#endif  // FOPD_MX4_HIP_
