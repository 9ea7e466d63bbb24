// Global norm of a list of gradient tensors and their scaling by it, for gfx950 (CDNA4).
//
//   fopd_grad_sum_squares   sum of squares of a workgroup's pieces of the list, in 64 bits; the last workgroup of a list's last launch
//                           adds the workgroups' sums up, in their order: sum of squares and norm
//   fopd_grad_scale         out = c grad,  c = min(1, max_norm / (norm + eps))
//
// Bound by HBM: the norm reads the list once, the scaling reads it and writes it.  622 M fp32 entries: 345 us (7.2 TB/s, the end
// of the list out of the Infinity Cache on repeated calls) and 882 us (5.6 TB/s, the rate of the fastest copy).  Squares are formed and
// added in 64 bits, at the rate of 32-bit fused multiply-adds on this part: entries of 1e-30 or 1e30 neither vanish nor overflow, and
// the result does not depend on the size of the list.  Outputs leave by non-temporal stores (ordinary ones 1359 us for both
// calls, so 1250), and so do inputs come in the scaling (ordinary loads 1305).
//
// A launch gets up to kGradTable tensors by value, in its kernel arguments: nothing is copied to the device beforehand, and a
// captured launch keeps its own table.  A tensor is rows of `cols` entries; rows that follow each other without a gap are one
// long row.  It is cut into pieces of kGradPieceBytes of a row, dealt to the workgroups in turn; a lane has all 16-byte loads of a
// piece in flight at once.  The norm goes through the list from the front, the scaling from the back: what the norm read
// last is still in the Infinity Cache.  (The scaling's own traffic leaves that there: tensors from the front, each from its end, take
// as long, 8 layers of width 4096 in bf16 646 us, so 648.)

#ifndef FOPD_GRAD_HIP_
#define FOPD_GRAD_HIP_

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "fopd_kernels.hip"

namespace fopd {

constexpr int kGradTable = 48;
constexpr int kGradPieceBytes = 32768;
constexpr int kGradLanes = 256;
constexpr int kGradVecs = kGradPieceBytes / 16 / kGradLanes;
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
  const int most = kGradPieceBytes >> (t.bf16 ? 1 : 2);
  const int64_t col = static_cast<int64_t>(local - row * t.row_pieces) * most;
  const int64_t left = t.cols - col;
  return GradPlace{row, col, static_cast<int>(left < most ? left : most)};
}

// Calls with the vectors' 16-byte loads all under way: body(vector, its value), vectors first + lane + 256 u.
template <bool CACHED, typename Body>
__device__ __forceinline__ void grad_vectors(const u32x4* v, int n, Body body) {
  u32x4 q[kGradVecs];
  if (n == kGradVecs * kGradLanes) {
#pragma unroll
    for (int u = 0; u < kGradVecs; ++u) q[u] = load_vec<CACHED>(v + threadIdx.x + u * kGradLanes);
#pragma unroll
    for (int u = 0; u < kGradVecs; ++u) body(static_cast<int>(threadIdx.x) + u * kGradLanes, q[u]);
  } else {
#pragma unroll
    for (int u = 0; u < kGradVecs; ++u)
      if (static_cast<int>(threadIdx.x) + u * kGradLanes < n) q[u] = load_vec<CACHED>(v + threadIdx.x + u * kGradLanes);
#pragma unroll
    for (int u = 0; u < kGradVecs; ++u)
      if (static_cast<int>(threadIdx.x) + u * kGradLanes < n) body(static_cast<int>(threadIdx.x) + u * kGradLanes, q[u]);
  }
}

// Entries before the first 16-byte boundary.
template <int DT>
__device__ __forceinline__ int grad_head(const char* p, int count) {
  return min(count, static_cast<int>((16 - (reinterpret_cast<uintptr_t>(p) & 15)) & 15) / Elem<DT>::kBytes);
}

template <int DT, bool CACHED>
__device__ __forceinline__ double grad_piece_squares(const char* p, int count) {
  constexpr int E = Elem<DT>::kPerVec;
  const int tid = threadIdx.x, head = grad_head<DT>(p, count), nvec = (count - head) / E;
  double a[4] = {0.0, 0.0, 0.0, 0.0};
  grad_vectors<CACHED>(reinterpret_cast<const u32x4*>(p + head * Elem<DT>::kBytes), nvec, [&](int, const u32x4& q) {
    float x[E];
    unpack<DT>(q, x);
#pragma unroll
    for (int e = 0; e < E; ++e) a[e & 3] = fma(static_cast<double>(x[e]), static_cast<double>(x[e]), a[e & 3]);
  });
  const int rest = count - nvec * E;           // fewer than two vectors' entries, before and behind them
  if (tid < rest) {
    const double x = load_elem<DT>(p, tid < head ? tid : nvec * E + tid);
    a[0] = fma(x, x, a[0]);
  }
  return (a[0] + a[1]) + (a[2] + a[3]);
}

template <int DT, int DT_OUT>
__device__ __forceinline__ void grad_piece_scale(const char* p, char* o, int count, float c) {
  constexpr int E = Elem<DT>::kPerVec, B = Elem<DT>::kBytes, BO = Elem<DT_OUT>::kBytes;
  const int tid = threadIdx.x, head = grad_head<DT>(p, count);
  // vectors on both sides where input and output reach their boundaries at the same entry
  if (((reinterpret_cast<uintptr_t>(o) + head * BO) & (E * BO < 16 ? E * BO - 1 : 15)) != 0) {
    for (int k = tid; k < count; k += kGradLanes) store_elem<DT_OUT>(o, k, c * load_elem<DT>(p, k));
    return;
  }
  const int nvec = (count - head) / E;
  char* ov = o + head * BO;
  grad_vectors<false>(reinterpret_cast<const u32x4*>(p + head * B), nvec, [&](int j, const u32x4& q) {
    float x[E];
    unpack<DT>(q, x);
#pragma unroll
    for (int e = 0; e < E; ++e) x[e] *= c;
    if constexpr (E * BO == 8) {
      typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
      __builtin_nontemporal_store(u32x2{pack_bf16x2(x[0], x[1]), pack_bf16x2(x[2], x[3])}, reinterpret_cast<u32x2*>(ov) + j);
    } else {
#pragma unroll
      for (int h = 0; h < E * BO / 16; ++h)
        __builtin_nontemporal_store(pack<DT_OUT>(x + h * (16 / BO)), reinterpret_cast<u32x4*>(ov) + j * (E * BO / 16) + h);
    }
  });
  const int rest = count - nvec * E;
  if (tid < rest) {
    const int k = tid < head ? tid : nvec * E + tid;
    store_elem<DT_OUT>(o, k, c * load_elem<DT>(p, k));
  }
}

}  // namespace

// What the last launch of a list leaves behind: the root and sum of `count` partial sums (of earlier launches too).
struct GradFinish {
  int count;                                  // 0: not the last launch
  bool add;                                   // to what sum_sq holds
  double* sum_sq;
  float* norm;                                // may be NULL
  int32_t* ticket;                            // 0 before and after
};

// Pieces from first_cached on stay in the Infinity Cache.  partial: this launch's first.
__global__ void __launch_bounds__(kGradLanes)
fopd_grad_sum_squares(GradTable g, double* partial, int first_cached, GradFinish finish) {
  double sum = 0.0;
  for (int piece = blockIdx.x; piece < g.pieces; piece += gridDim.x) {
    const GradEntry& t = g.t[grad_tensor_of(g, piece)];
    const GradPlace at = grad_place(t, piece);
    const int64_t first = at.row * t.ld + at.col;
    const char* p = static_cast<const char*>(t.grad) + first * (t.bf16 ? 2 : 4);
    if (piece >= first_cached) sum += t.bf16 ? grad_piece_squares<FOPD_BF16, true>(p, at.count) : grad_piece_squares<FOPD_F32, true>(p, at.count);
    else sum += t.bf16 ? grad_piece_squares<FOPD_BF16, false>(p, at.count) : grad_piece_squares<FOPD_F32, false>(p, at.count);
  }
  __shared__ double sh[kGradLanes / 64];
  __shared__ int last;
  sum = block_sum<kGradLanes>(sum, sh);
  if (threadIdx.x == 0) {
    // The sum goes to where all XCDs' caches meet, and is there before the ticket is drawn: whoever draws the last ticket finds
    // them all.  (Which workgroup that is does not matter, the order of the additions is that of the list.)
    __hip_atomic_store(partial + blockIdx.x, sum, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    last = finish.count > 0 && __hip_atomic_fetch_add(finish.ticket, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == static_cast<int>(gridDim.x) - 1;
  }
  __syncthreads();
  if (last == 0) return;
  const double* from = partial + gridDim.x - finish.count;
  sum = 0.0;
  for (int k = threadIdx.x; k < finish.count; k += kGradLanes) sum += __hip_atomic_load(from + k, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  sum = block_sum<kGradLanes>(sum, sh);
  if (threadIdx.x != 0) return;
  if (finish.add) sum += finish.sum_sq[0];
  finish.sum_sq[0] = sum;
  if (finish.norm != nullptr) finish.norm[0] = static_cast<float>(sqrt(sum));
  *finish.ticket = 0;
}

// c < 1 or NaN as it is, else 1: a norm that is no number makes every entry one.
__device__ __forceinline__ float grad_coefficient(double sum_sq, float max_norm, float eps) {
  const double norm = sqrt(sum_sq) + static_cast<double>(eps);
  if (norm == 0.0) return 1.f;                             // nothing but zeros, whatever max_norm
  const double c = static_cast<double>(max_norm) / norm;
  return static_cast<float>(c >= 1.0 ? 1.0 : c);
}

__global__ void __launch_bounds__(kGradLanes)
fopd_grad_scale(GradTable g, const double* __restrict__ sum_sq, float max_norm, float eps, float* __restrict__ coef) {
  const float c = grad_coefficient(sum_sq[0], max_norm, eps);
  if (coef != nullptr && blockIdx.x == 0 && threadIdx.x == 0) coef[0] = c;
  for (int piece = g.pieces - 1 - static_cast<int>(blockIdx.x); piece >= 0; piece -= static_cast<int>(gridDim.x)) {
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
