// Verification of drafted tokens for gfx950 (CDNA4): how many tokens of each draft the student keeps, and the token after them.
//
//   fopd_verify_rows     one pass over the target's and the drafter's rows: (maximum, sum) of each piece of a row
//   fopd_verify_race     per sample the decisions from those, then the race for the next token over the entries of one row
//   fopd_verify_finish   per sample the winner among the pieces of that race
//
// Row j of a sample has p_j = softmax(z_j / tau), q_j = softmax(z'_j / tau) (without the drafter's logits: all of it on the drafted
// token x_j) and a uniform u_j.  Draft j is kept while u_j q_j(x_j) < p_j(x_j); at the first one that is not, a, the next token is
// distributed as max(p_a - q_a, 0) made to add up to 1, after a whole draft as p_a.  It is found by a race: token v arrives at e_v
// / r_v, e_v given exponential variates, and the first one wins, which it does with probability r_v / sum r.  A race needs no
// running sum over the vocabulary, whose borders would have to be known to far more digits than the terms have, and splits over
// any number of workgroups; the lowest index wins a tie.  tau = 0: the largest logit instead of either.
//
// Bound by HBM: every row is read once by the first kernel, and one row of either kind again, mostly from the Infinity Cache,
// together with the variates by the second.

#ifndef FOPD_VERIFY_HIP_
#define FOPD_VERIFY_HIP_

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "fopd_kernels.hip"

namespace fopd {

constexpr int kVerifyThreads = 256;
constexpr int kVerifyMaxDraft = 1023;         // (the decisions of a sample are made in one workgroup's LDS)
constexpr int kVerifyMaxSplits = 64;          // pieces of a row in the first kernel, a power of two
constexpr int32_t kFlagDist = 16;

// What the entry point was given, as the three kernels see it.
struct VerifyArgs {
  const void* target;
  const void* draft;                          // NULL: all of a draft's probability is on its token
  int64_t ld, ld_draft, rows, ld_noise;
  int V, B, K;
  const int32_t* draft_ids;
  const int64_t* row_begin;
  const int32_t* draft_lens;
  const float* temperature;
  const float* accept_u;
  const float* noise;                         // NULL: every sample greedily
  int32_t* n_accepted;
  int32_t* out_ids;
  float* out_logp;
  uint8_t* out_mask;
};

// (maximum, sum of exp2((x - maximum) c), first index of the maximum) of a piece of a row; an empty piece has sum 0.
struct RowPart {
  float top, sum;
  int32_t at, pad;
};

// The winner among the entries of a piece: by max(p - q, 0) and, where that is zero everywhere, by p.
struct RacePart {
  float left, full;
  int32_t left_at, full_at;
};

// What the second kernel decided: tokens kept (-1: the sample's rows are not there), whether there is a next token, and the
// row's maximum and sum for that token's log-probability.
struct Verdict {
  int32_t kept, next;
  float top, sum;
};

namespace {

constexpr float kLowest = -3.402823466e38f;   // reference of an empty piece: an entry of the type's lowest value counts

struct VerifySample {
  int64_t row;
  int len;
  bool there, greedy;
  float c;                                    // log2(e) / tau; NaN where tau is negative or no number
};

__device__ __forceinline__ VerifySample verify_sample(const VerifyArgs& a, int i) {
  VerifySample s;
  s.len = a.draft_lens != nullptr ? a.draft_lens[i] : a.K;
  s.row = a.row_begin != nullptr ? a.row_begin[i] : static_cast<int64_t>(i) * (a.K + 1);
  s.there = s.len >= 0 && s.len <= a.K && s.row >= 0 && s.row <= a.rows - 1 - s.len;
  const float tau = a.temperature != nullptr ? a.temperature[i] : 1.f;
  s.greedy = a.noise == nullptr || tau == 0.f;
  s.c = s.greedy ? kLog2e : (tau > 0.f ? kLog2e / tau : __builtin_nanf(""));
  return s;
}

// Entries of `x` into the lane's piece.  The maximum is subtracted before the temperature is applied: entries of the type's
// lowest value keep a finite difference among themselves, and -inf gives exp2(-inf) = 0.
template <int N>
__device__ __forceinline__ void verify_add(const float* x, float c, float& top, float& sum) {
  float m = top;
#pragma unroll
  for (int e = 0; e < N; ++e) m = fmaxf(m, x[e]);
  if (m > top) {
    sum *= fast_exp2((top - m) * c);
    top = m;
  }
  float s0 = 0.f, s1 = 0.f;
#pragma unroll
  for (int e = 0; e < N; e += 2) {
    s0 += fast_exp2((x[e] - top) * c);
    if (e + 1 < N) s1 += fast_exp2((x[e + 1] - top) * c);
  }
  sum += s0 + s1;
}

// (a piece that is empty or holds NaN keeps what it is: 0 x anything finite, NaN + anything)
__device__ __forceinline__ void verify_merge(float c, float& top, float& sum, float top2, float sum2) {
  const float m = fmaxf(top, top2);
  sum = sum * fast_exp2((top - m) * c) + sum2 * fast_exp2((top2 - m) * c);
  top = m;
}

__device__ __forceinline__ void race_merge(float& s, int& at, float s2, int at2) {
  if (s2 > s || (s2 == s && at2 < at)) {
    s = s2;
    at = at2;
  }
}

}  // namespace

// Workgroup ((tensor B + sample) (K + 1) + row) splits + piece; parts[(tensor R + row of the tensor) splits + piece].
template <int DT>
__global__ void __launch_bounds__(kVerifyThreads)
fopd_verify_rows(VerifyArgs a, int splits, int piece_vecs, RowPart* __restrict__ parts) {
  constexpr int E = Elem<DT>::kPerVec;
  const unsigned unit = blockIdx.x / static_cast<unsigned>(splits);
  const int piece = static_cast<int>(blockIdx.x - unit * splits);
  const unsigned per = static_cast<unsigned>(a.K + 1);
  const int j = static_cast<int>(unit % per);
  unsigned i = unit / per;
  const bool drafter = i >= static_cast<unsigned>(a.B);
  if (drafter) i -= a.B;
  const VerifySample s = verify_sample(a, static_cast<int>(i));
  if (!s.there || j > s.len || (drafter && (s.greedy || j == s.len))) return;
  const int64_t r = s.row + j;
  const char* row = drafter ? static_cast<const char*>(a.draft) + r * a.ld_draft * Elem<DT>::kBytes
                            : static_cast<const char*>(a.target) + r * a.ld * Elem<DT>::kBytes;
  const u32x4* rv = reinterpret_cast<const u32x4*>(row);
  const int tid = threadIdx.x;
  const int nvec = a.V / E;
  const int end = min(nvec, (piece + 1) * piece_vecs);
  float top = kLowest, sum = 0.f;
  int at = 0x7fffffff;
  auto add = [&](auto count, const float* x, int first) {
    constexpr int N = decltype(count)::value;
    if (s.greedy) {                           // first index of the largest entry: a lane's indices only grow
#pragma unroll
      for (int e = 0; e < N; ++e)
        if (x[e] > top || (x[e] == top && at == 0x7fffffff)) {
          sum *= fast_exp2((top - x[e]) * s.c);
          top = x[e];
          at = first + e;
        }
    }
    verify_add<N>(x, s.c, top, sum);
  };
  int v = piece * piece_vecs + tid;
  if (!s.greedy) {
    for (; v + 3 * kVerifyThreads < end; v += 4 * kVerifyThreads) {
      u32x4 q[4];
#pragma unroll
      for (int u = 0; u < 4; ++u) q[u] = rv[v + u * kVerifyThreads];
      float x[4 * E];
#pragma unroll
      for (int u = 0; u < 4; ++u) unpack<DT>(q[u], x + u * E);
      verify_add<4 * E>(x, s.c, top, sum);
    }
  }
  for (; v < end; v += kVerifyThreads) {
    float x[E];
    unpack<DT>(rv[v], x);
    add(std::integral_constant<int, E>(), x, v * E);
  }
  if (piece == splits - 1 && nvec * E + tid < a.V) {                   // fewer than a vector's entries
    const float x = load_elem<DT>(row, nvec * E + tid);
    add(std::integral_constant<int, 1>(), &x, nvec * E + tid);
  }
  __shared__ RowPart sh[kVerifyThreads / 64];
  auto take = [&](float top2, float sum2, int at2) {
    if (top2 > top || (top2 == top && at2 < at)) at = at2;
    verify_merge(s.c, top, sum, top2, sum2);
  };
#pragma unroll
  for (int off = 32; off > 0; off >>= 1) take(__shfl_xor(top, off, 64), __shfl_xor(sum, off, 64), __shfl_xor(at, off, 64));
  if ((tid & 63) == 0) sh[tid >> 6] = RowPart{top, sum, at, 0};
  __syncthreads();
  if (tid == 0) {
    for (int w = 1; w < kVerifyThreads / 64; ++w) take(sh[w].top, sh[w].sum, sh[w].at);
    parts[((drafter ? a.rows : 0) + r) * splits + piece] = RowPart{top, sum, at, 0};
  }
}

// Workgroup sample x pieces + piece.  Every workgroup of a sample makes the sample's decisions, the first one writes them down;
// dynamic LDS: 2 (K + 1) RowParts.
template <int DT>
__global__ void __launch_bounds__(kVerifyThreads)
fopd_verify_race(VerifyArgs a, int splits, const RowPart* __restrict__ parts, int pieces, int piece_vecs,
                 RacePart* __restrict__ races, Verdict* __restrict__ verdicts, int32_t* __restrict__ flags) {
  constexpr int E = Elem<DT>::kPerVec;
  extern __shared__ __align__(16) unsigned char verify_smem[];
  RowPart* rows = reinterpret_cast<RowPart*>(verify_smem);             // [target, drafter][K + 1]
  __shared__ int sh_kept, sh_next;
  const int i = static_cast<int>(blockIdx.x / static_cast<unsigned>(pieces));
  const int piece = static_cast<int>(blockIdx.x - static_cast<unsigned>(i) * pieces);
  const int tid = threadIdx.x, lane = tid & 63;
  const VerifySample s = verify_sample(a, i);
  const int per = a.K + 1;
  const bool writes = piece == 0;
  if (!s.there) {
    if (writes) {
      if (tid == 0) {
        atomicOr(flags, kFlagSegments);
        a.n_accepted[i] = 0;
        verdicts[i] = Verdict{-1, 0, 0.f, 0.f};
      }
      if (a.row_begin == nullptr)             // the rows are this sample's own
        for (int j = tid; j < per; j += kVerifyThreads) {
          const int64_t r = static_cast<int64_t>(i) * per + j;
          a.out_ids[r] = -1;
          a.out_logp[r] = 0.f;
          a.out_mask[r] = 0;
        }
    }
    return;
  }
  // the pieces of each row, `splits` lanes a row
  const bool with_draft = a.draft != nullptr && !s.greedy;
  const int items = (with_draft ? 2 : 1) * (s.len + 1);
  for (int base = 0; base < items; base += kVerifyThreads / splits) {
    const int item = base + tid / splits;
    const bool drafter = item > s.len;
    const int j = drafter ? item - s.len - 1 : item;
    RowPart p = {kLowest, 0.f, 0x7fffffff, 0};
    if (item < items && !(drafter && j == s.len))
      p = parts[((drafter ? a.rows : 0) + s.row + j) * splits + (tid & (splits - 1))];
    for (int off = splits >> 1; off > 0; off >>= 1) {
      const float top2 = __shfl_xor(p.top, off, 64), sum2 = __shfl_xor(p.sum, off, 64);
      const int at2 = __shfl_xor(p.at, off, 64);
      if (top2 > p.top || (top2 == p.top && at2 < p.at)) p.at = at2;
      verify_merge(s.c, p.top, p.sum, top2, sum2);
    }
    if (item < items && (tid & (splits - 1)) == 0) rows[(drafter ? per : 0) + j] = p;
  }
  __syncthreads();
  if (tid < 64) {
    int kept = s.len, next = 1, bad = 0;
    for (int base = 0; base <= s.len && kept == s.len; base += 64) {
      const int j = base + lane;
      bool keeps = true, usable = true;
      int problem = 0;
      if (j <= s.len) {
        const RowPart p = rows[j];
        const int64_t r = s.row + j;
        usable = p.sum > 0.f && p.sum < __builtin_inff();              // (false for NaN)
        if (!usable) problem = kFlagDist;
        keeps = j < s.len && usable;
        const int x = j < s.len ? a.draft_ids[r] : 0;
        const bool in_range = x >= 0 && x < a.V;
        if (j < s.len && !in_range) problem |= kFlagToken;
        keeps = keeps && in_range;
        if (s.greedy) {
          keeps = keeps && x == p.at;
        } else {
          RowPart q = {0.f, 1.f, 0, 0};
          if (with_draft && j < s.len) {
            q = rows[per + j];
            if (!(q.sum > 0.f && q.sum < __builtin_inff())) {
              usable = keeps = false;
              problem |= kFlagDist;
            }
          }
          if (keeps) {
            const double c = static_cast<double>(s.c);
            const double zp = load_elem<DT>(static_cast<const char*>(a.target) + r * a.ld * Elem<DT>::kBytes, x);
            const double px = exp2((zp - static_cast<double>(p.top)) * c) / static_cast<double>(p.sum);
            double qx = 1.0;
            if (with_draft) {
              const double zq = load_elem<DT>(static_cast<const char*>(a.draft) + r * a.ld_draft * Elem<DT>::kBytes, x);
              qx = exp2((zq - static_cast<double>(q.top)) * c) / static_cast<double>(q.sum);
            }
            keeps = static_cast<double>(a.accept_u[r]) * qx < px;
          }
        }
      }
      const unsigned long long stops = __ballot(j <= s.len && !keeps);
      if (stops != 0) {
        const int first = __ffsll(static_cast<unsigned long long>(stops)) - 1;
        kept = base + first;
        next = __shfl(usable ? 1 : 0, first, 64);
        bad = __shfl(problem, first, 64);
      }
      if (stops != 0) break;
    }
    if (lane == 0) {
      sh_kept = kept;
      sh_next = next;
      if (writes) {
        if (bad != 0) atomicOr(flags, bad);
        a.n_accepted[i] = kept;
        verdicts[i] = Verdict{kept, next, rows[kept].top, rows[kept].sum};
      }
    }
  }
  __syncthreads();
  const int kept = sh_kept;
  const RowPart p = rows[kept];
  if (writes) {                               // the drafted tokens that are kept, nothing in the rows behind the next one
    const int last = a.row_begin == nullptr ? a.K : s.len;
    for (int j = tid; j <= last; j += kVerifyThreads) {
      if (j == kept) continue;
      const int64_t r = s.row + j;
      float lp = 0.f;
      int x = -1;
      if (j < kept) {
        x = a.draft_ids[r];
        const double z = load_elem<DT>(static_cast<const char*>(a.target) + r * a.ld * Elem<DT>::kBytes, x);
        lp = static_cast<float>(((z - static_cast<double>(rows[j].top)) * static_cast<double>(s.c) -
                                 log2(static_cast<double>(rows[j].sum))) * kLn2);
      }
      a.out_ids[r] = x;
      a.out_logp[r] = lp;
      a.out_mask[r] = j < kept ? 1 : 0;
    }
  }
  float left = -1.f, full = -1.f;
  int left_at = 0x7fffffff, full_at = 0x7fffffff;
  if (sh_next != 0 && s.greedy) {
    if (writes && tid == 0) left = full = 1.f, left_at = full_at = p.at;
  } else if (sh_next != 0) {
    // r = max(p - q, 0) and p, each over the variate; both in units of the target row's sum
    const int64_t r = s.row + kept;
    const bool rejected = kept < s.len;
    const bool minus = rejected && a.draft != nullptr;
    const int out = rejected && a.draft == nullptr ? a.draft_ids[r] : -1;        // the token that is taken out
    const RowPart q = minus ? rows[per + kept] : RowPart{0.f, 1.f, 0, 0};
    const float ratio = p.sum / q.sum;
    const char* zrow = static_cast<const char*>(a.target) + r * a.ld * Elem<DT>::kBytes;
    const char* qrow = minus ? static_cast<const char*>(a.draft) + r * a.ld_draft * Elem<DT>::kBytes : zrow;
    const float* noise = a.noise + static_cast<int64_t>(i) * a.ld_noise;
    auto enter = [&](int v, float z, float zq, float e) {
      const float pv = fast_exp2((z - p.top) * s.c);
      const float rv = minus ? pv - ratio * fast_exp2((zq - q.top) * s.c) : (v == out ? 0.f : pv);
      const float inv = __builtin_amdgcn_rcpf(e);          // (an error of one unit in the last place, as the terms have)
      if (pv > 0.f && pv * inv > full) full = pv * inv, full_at = v;   // (a lane's indices only grow)
      if (rv > 0.f && rv * inv > left) left = rv * inv, left_at = v;
    };
    const int nvec = a.V / E, end = min(nvec, (piece + 1) * piece_vecs);
    for (int v = piece * piece_vecs + tid; v < end; v += kVerifyThreads) {
      float z[E], zq[E], e[E];
      unpack<DT>(reinterpret_cast<const u32x4*>(zrow)[v], z);
      unpack<DT>(reinterpret_cast<const u32x4*>(qrow)[v], zq);
#pragma unroll
      for (int h = 0; h < E / 4; ++h) unpack<FOPD_F32>(reinterpret_cast<const u32x4*>(noise)[v * (E / 4) + h], e + 4 * h);
#pragma unroll
      for (int k = 0; k < E; ++k) enter(v * E + k, z[k], zq[k], e[k]);
    }
    const int v = nvec * E + tid;
    if (piece == pieces - 1 && v < a.V) enter(v, load_elem<DT>(zrow, v), load_elem<DT>(qrow, v), noise[v]);
  }
#pragma unroll
  for (int off = 32; off > 0; off >>= 1) {
    race_merge(left, left_at, __shfl_xor(left, off, 64), __shfl_xor(left_at, off, 64));
    race_merge(full, full_at, __shfl_xor(full, off, 64), __shfl_xor(full_at, off, 64));
  }
  __shared__ RacePart sh_race[kVerifyThreads / 64];
  if (lane == 0) sh_race[tid >> 6] = RacePart{left, full, left_at, full_at};
  __syncthreads();
  if (tid == 0) {
    for (int w = 1; w < kVerifyThreads / 64; ++w) {
      race_merge(left, left_at, sh_race[w].left, sh_race[w].left_at);
      race_merge(full, full_at, sh_race[w].full, sh_race[w].full_at);
    }
    races[static_cast<int64_t>(i) * pieces + piece] = RacePart{left, full, left_at, full_at};
  }
}

// One wavefront a sample.
template <int DT>
__global__ void __launch_bounds__(64)
fopd_verify_finish(VerifyArgs a, int pieces, const RacePart* __restrict__ races, const Verdict* __restrict__ verdicts,
                   int32_t* __restrict__ flags) {
  const int i = blockIdx.x, lane = threadIdx.x;
  const Verdict d = verdicts[i];
  if (d.kept < 0) return;
  float left = -1.f, full = -1.f;
  int left_at = 0x7fffffff, full_at = 0x7fffffff;
  for (int k = lane; k < pieces; k += 64) {
    const RacePart p = races[static_cast<int64_t>(i) * pieces + k];
    race_merge(left, left_at, p.left, p.left_at);
    race_merge(full, full_at, p.full, p.full_at);
  }
#pragma unroll
  for (int off = 32; off > 0; off >>= 1) {
    race_merge(left, left_at, __shfl_xor(left, off, 64), __shfl_xor(left_at, off, 64));
    race_merge(full, full_at, __shfl_xor(full, off, 64), __shfl_xor(full_at, off, 64));
  }
  if (lane != 0) return;
  const VerifySample s = verify_sample(a, i);
  const int64_t r = s.row + d.kept;
  const int at = left > 0.f ? left_at : full_at;
  const bool found = d.next != 0 && at < a.V;
  if (d.next != 0 && !found) atomicOr(flags, kFlagDist);               // no variate is a number
  float lp = __builtin_nanf("");
  if (found) {
    const double z = load_elem<DT>(static_cast<const char*>(a.target) + r * a.ld * Elem<DT>::kBytes, at);
    lp = static_cast<float>(((z - static_cast<double>(d.top)) * static_cast<double>(s.c) - log2(static_cast<double>(d.sum))) * kLn2);
  }
  a.out_ids[r] = found ? at : -1;
  a.out_logp[r] = lp;
  a.out_mask[r] = found ? 1 : 0;
}

}  // namespace fopd

#endif  // FOPD_VERIFY_HIP_
