// Global norm of a list of gradient tensors and their scaling by it, for gfx950 (CDNA4).
//
//   fopd_grad_sum_squares   sum of squares of a workgroup's pieces of the list, in 64 bits
//   fopd_grad_norm_final    the workgroups' sums in their order: sum of squares and norm
//   fopd_grad_scale         out = c grad,  c = min(1, max_norm / (norm + eps))
//
// Bound by HBM: the norm reads the list once, the scaling reads it and writes it.  Squares are formed and added in 64 bits, at
// the rate of 32-bit fused multiply-adds on this part: entries of 1e-30 or 1e30 neither vanish nor overflow, and the result
// does not depend on the size of the list.
//
// A launch gets up to kGradTable tensors by value, in its kernel arguments: nothing is copied to the device beforehand, and a
// captured launch keeps its own table.  A tensor is rows of `cols` entries; rows that follow each other without a gap are one
// long row.  It is cut into pieces of kGradPiece entries of a row, dealt to the workgroups in turn.

#ifndef FOPD_GRAD_HIP_
#define FOPD_GRAD_HIP_

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "fopd_kernels.hip"

namespace fopd {

constexpr int kGradTable = 48;
constexpr int kGradPiece = 8192;              // entries: 16 or 32 KB
constexpr int kGradLanes = 256;
constexpr int kGradMaxGroups = 4096;          // workgroups of a launch of fopd_grad_sum_squares
constexpr int64_t kGradMaxPieces = 1LL << 30; // pieces of a launch

struct GradEntry {
  const void* grad;
  void* out;
  int64_t cols, ld, ld_out;
  int32_t rows, row_pieces, first_piece;      // pieces of a row; pieces of the launch's tensors before this one
  int8_t bf16, out_bf16;
};

struct GradTable {
  int32_t n, pieces;
  GradEntry t[kGradTable];
};

namespace {

struct GradPlace {
  int64_t row, col;
  int count;                                  // entries of this piece
};

// Tensor and place of a piece.  The table is searched by the scalar unit: the piece is the same for the whole workgroup.
__device__ __forceinline__ int grad_tensor_of(const GradTable& g, int piece) {
  int lo = 0, hi = g.n - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (g.t[mid].first_piece <= piece) lo = mid;
    else hi = mid - 1;
  }
  return lo;
}

__device__ __forceinline__ GradPlace grad_place(const GradEntry& t, int piece) {
  const int local = piece - t.first_piece;
  const int row = local / t.row_pieces;
  const int64_t col = static_cast<int64_t>(local - row * t.row_pieces) * kGradPiece;
  const int64_t left = t.cols - col;
  return GradPlace{row, col, static_cast<int>(left < kGradPiece ? left : kGradPiece)};
}

template <int DT>
__device__ __forceinline__ double grad_piece_squares(const char* p, int count) {
  constexpr int E = Elem<DT>::kPerVec, B = Elem<DT>::kBytes;
  const int tid = threadIdx.x;
  // entries up to the first 16-byte boundary, then vectors, then the rest
  const int head = min(count, static_cast<int>((16 - (reinterpret_cast<uintptr_t>(p) & 15)) & 15) / B);
  const int nvec = (count - head) / E;
  double a[4] = {0.0, 0.0, 0.0, 0.0};
  if (tid < head) {
    const double x = load_elem<DT>(p, tid);
    a[0] = fma(x, x, a[0]);
  }
  const u32x4* v = reinterpret_cast<const u32x4*>(p + head * B);
#pragma unroll 4
  for (int j = tid; j < nvec; j += kGradLanes) {
    float x[E];
    unpack<DT>(v[j], x);
#pragma unroll
    for (int e = 0; e < E; ++e) a[e & 3] = fma(static_cast<double>(x[e]), static_cast<double>(x[e]), a[e & 3]);
  }
  const int rest = head + nvec * E + tid;
  if (rest < count) {
    const double x = load_elem<DT>(p, rest);
    a[1] = fma(x, x, a[1]);
  }
  return (a[0] + a[1]) + (a[2] + a[3]);
}

template <int DT, int DT_OUT>
__device__ __forceinline__ void grad_piece_scale(const char* p, char* o, int count, float c) {
  constexpr int E = Elem<DT>::kPerVec, B = Elem<DT>::kBytes, BO = Elem<DT_OUT>::kBytes;
  const int tid = threadIdx.x;
  // vectors of E entries on both sides where input and output reach their boundaries at the same entry
  int head = min(count, static_cast<int>((16 - (reinterpret_cast<uintptr_t>(p) & 15)) & 15) / B);
  const bool wide = ((reinterpret_cast<uintptr_t>(o) + head * BO) & (E * BO < 16 ? E * BO - 1 : 15)) == 0;
  if (!wide) {
    for (int k = tid; k < count; k += kGradLanes) store_elem<DT_OUT>(o, k, c * load_elem<DT>(p, k));
    return;
  }
  const int nvec = (count - head) / E;
  if (tid < head) store_elem<DT_OUT>(o, tid, c * load_elem<DT>(p, tid));
  const u32x4* v = reinterpret_cast<const u32x4*>(p + head * B);
  char* ov = o + head * BO;
#pragma unroll 4
  for (int j = tid; j < nvec; j += kGradLanes) {
    float x[E];
    unpack<DT>(v[j], x);
#pragma unroll
    for (int e = 0; e < E; ++e) x[e] *= c;
    if constexpr (E * BO == 8) {
      reinterpret_cast<uint2*>(ov)[j] = make_uint2(pack_bf16x2(x[0], x[1]), pack_bf16x2(x[2], x[3]));
    } else {
#pragma unroll
      for (int h = 0; h < E * BO / 16; ++h) reinterpret_cast<u32x4*>(ov)[j * (E * BO / 16) + h] = pack<DT_OUT>(x + h * (16 / BO));
    }
  }
  const int rest = head + nvec * E + tid;
  if (rest < count) store_elem<DT_OUT>(o, rest, c * load_elem<DT>(p, rest));
}

}  // namespace

__global__ void __launch_bounds__(kGradLanes)
fopd_grad_sum_squares(GradTable g, double* __restrict__ partial) {
  double sum = 0.0;
  for (int piece = blockIdx.x; piece < g.pieces; piece += gridDim.x) {
    const GradEntry& t = g.t[grad_tensor_of(g, piece)];
    const GradPlace at = grad_place(t, piece);
    const int64_t first = at.row * t.ld + at.col;
    if (t.bf16) sum += grad_piece_squares<FOPD_BF16>(static_cast<const char*>(t.grad) + first * 2, at.count);
    else sum += grad_piece_squares<FOPD_F32>(static_cast<const char*>(t.grad) + first * 4, at.count);
  }
  __shared__ double sh[kGradLanes / 64];
  sum = block_sum<kGradLanes>(sum, sh);
  if (threadIdx.x == 0) partial[blockIdx.x] = sum;
}

// sum_sq = (add: sum_sq +) the n partial sums; norm (last launch of a list, else NULL) = its root.
__global__ void __launch_bounds__(kGradLanes)
fopd_grad_norm_final(const double* __restrict__ partial, int n, bool add, double* __restrict__ sum_sq, float* __restrict__ norm) {
  double sum = 0.0;
  for (int k = threadIdx.x; k < n; k += kGradLanes) sum += partial[k];
  __shared__ double sh[kGradLanes / 64];
  sum = block_sum<kGradLanes>(sum, sh);
  if (threadIdx.x != 0) return;
  if (add) sum += sum_sq[0];
  sum_sq[0] = sum;
  if (norm != nullptr) norm[0] = static_cast<float>(sqrt(sum));
}

// c < 1 or NaN as it is, else 1: a norm that is no number makes every entry one.
__device__ __forceinline__ float grad_coefficient(double sum_sq, float max_norm, float eps) {
  const double c = static_cast<double>(max_norm) / (sqrt(sum_sq) + static_cast<double>(eps));
  return static_cast<float>(c >= 1.0 ? 1.0 : c);
}

__global__ void __launch_bounds__(kGradLanes)
fopd_grad_scale(GradTable g, const double* __restrict__ sum_sq, float max_norm, float eps, float* __restrict__ coef) {
  const float c = grad_coefficient(sum_sq[0], max_norm, eps);
  if (coef != nullptr && blockIdx.x == 0 && threadIdx.x == 0) coef[0] = c;
  for (int piece = blockIdx.x; piece < g.pieces; piece += gridDim.x) {
    const GradEntry& t = g.t[grad_tensor_of(g, piece)];
    if (c == 1.f && t.out == t.grad) continue;               // in place and not clipped: as it is
    const GradPlace at = grad_place(t, piece);
    const char* p = static_cast<const char*>(t.grad) + (at.row * t.ld + at.col) * (t.bf16 ? 2 : 4);
    char* o = static_cast<char*>(t.out) + (at.row * t.ld_out + at.col) * (t.out_bf16 ? 2 : 4);
    if (t.bf16) {
      if (t.out_bf16) grad_piece_scale<FOPD_BF16, FOPD_BF16>(p, o, at.count, c);
      else grad_piece_scale<FOPD_BF16, FOPD_F32>(p, o, at.count, c);
    } else {
      if (t.out_bf16) grad_piece_scale<FOPD_F32, FOPD_BF16>(p, o, at.count, c);
      else grad_piece_scale<FOPD_F32, FOPD_F32>(p, o, at.count, c);
    }
  }
}

}  // namespace fopd

#endif  // FOPD_GRAD_HIP_
