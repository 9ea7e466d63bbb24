// Verification of drafted tokens for gfx950 (CDNA4): how many tokens of each draft the student keeps, and the token after them.
//
//   fopd_verify_rows     one pass over the target's and the drafter's rows: (maximum, sum) of each piece of a row
//   fopd_verify_race     per sample the decisions from those, then the race for the next token over the entries of one row
//
// Row j of a sample has p_j = softmax(z_j / tau), q_j = softmax(z'_j / tau) (without the drafter's logits: all of it on the drafted
// token x_j) and a uniform u_j.  Draft j is kept while u_j q_j(x_j) < p_j(x_j); at the first one that is not, a, the next token is
// distributed as max(p_a - q_a, 0) made to add up to 1, after a whole draft as p_a.  It is found by a race: token v arrives at e_v
// / r_v, e_v given exponential variates, and the first one wins, which it does with probability r_v / sum r.  A race needs no
// running sum over the vocabulary, whose borders would have to be known to far more digits than the terms have, and splits over
// any number of workgroups; the lowest index wins a tie.  tau = 0: the largest logit instead of either.
//
// Bound by HBM where there are many samples: every row is read once by the first kernel, and one row of either kind again by the
// second, with the variates.  192 samples of 7 drafts x 151,936 in bf16: rows 145 - 151 us (875 MB, 5.8 - 6.0 TB/s), race 42 us (234 MB,
// 200 MB of rows left in the Infinity Cache on purpose: 219 MB fetched).  Bound by latency where there are few: one sample of 4 drafts
// 5 + 8 us, of which reading its 3.3 MB would be 0.5.  A batch of two 16-byte vectors a lane is the best of 2, 4 and 8 (37 samples of up to
// 5 looked-up drafts x 262,144: 32.2 / 34.4 / 37.8 us), and asking for the next one ahead of this one's arithmetic is slower
// (34.2).
//
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

// What the entry point was given, as the two kernels see it.
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

// The entries of a piece of a row: the largest, the sum over the others of exp2((x - top) c), and of a greedy sample's row the first
// index of the largest.  Without the largest entry's 1 the sum keeps its digits where it is small: log p of the likeliest
// token is -log(1 + others).  A piece without entries above -inf has top = -inf.
struct RowPart {
  float top, others;
  int32_t at, pad;
};

// The state of a sample's race across its workgroups: the best score so far in the upper half (scores are positive, so their
// bits order as they do) and all ones less its index in the lower, and how many workgroups are through.
struct RaceState {
  unsigned long long best;
  int32_t through, pad;
};

namespace {

struct RaceEntry {
  float score;
  int32_t at;
};

constexpr float kMinusInf = -__builtin_inff();
constexpr int kNowhere = 0x7fffffff;

struct VerifySample {
  int64_t row;
  int len;
  bool there, greedy;
  float c;                                    // log2(e) / tau; NaN where tau is negative, infinite or NaN
};

__device__ __forceinline__ VerifySample verify_sample(const VerifyArgs& a, int i) {
  VerifySample s;
  s.len = a.draft_lens != nullptr ? a.draft_lens[i] : a.K;
  s.row = a.row_begin != nullptr ? a.row_begin[i] : static_cast<int64_t>(i) * (a.K + 1);
  s.there = s.len >= 0 && s.len <= a.K && s.row >= 0 && s.row <= a.rows - 1 - s.len;
  const float tau = a.temperature != nullptr ? a.temperature[i] : 1.f;
  s.greedy = a.noise == nullptr || tau == 0.f;
  // (a temperature whose inverse is past the type's range is as good as one that is not: entries differ, or they do not)
  s.c = s.greedy ? kLog2e : (tau > 0.f && tau < __builtin_inff() ? fminf(kLog2e / tau, __FLT_MAX__) : __builtin_nanf(""));
  return s;
}

// A lane's entries: the sum over all of them in units of 2^ref, ref = max(top, -1e30) c as rounded, so that a term is one
// multiply-add and an exponential.  Batches of entries are summed in 32 bits and added up in 64; `batch` is the one that the
// largest entry is in, and ref has not changed since.
struct VerifyLane {
  float top = kMinusInf, ref = 0.f;
  double sum = 0.0;
  int batch = -1;
};

// As rounded wherever it goes: a difference of references that took in the product unrounded would be a rounding of |top| c away
// from what the terms were formed with (logits near 1000: 5e-5 of the sum).
__device__ __forceinline__ float verify_reference(float top, float c) {
#pragma clang fp contract(off)
  return fmaxf(top, -1e30f) * c;
}

template <int N>
__device__ __forceinline__ float verify_batch(const float* x, float c, float ref) {
  float s0 = 0.f, s1 = 0.f;
#pragma unroll
  for (int e = 0; e < N; e += 2) {
    s0 += fast_exp2(fmaf(x[e], c, -ref));
    if (e + 1 < N) s1 += fast_exp2(fmaf(x[e + 1], c, -ref));
  }
  return s0 + s1;
}

template <int N>
__device__ __forceinline__ void verify_add(const float* x, float c, int batch, VerifyLane& s) {
  float m = s.top;
#pragma unroll
  for (int e = 0; e < N; ++e) m = fmaxf(m, x[e]);
  if (m > s.top) {
    const float ref = verify_reference(m, c);
    // (ref only grows, except from an empty sum's 0 to logits below it: no factor there, which may be infinite)
    s.sum *= static_cast<double>(fast_exp2(fminf(s.ref - ref, 0.f)));
    s.top = m;
    s.ref = ref;
    s.batch = batch;
  }
  s.sum += static_cast<double>(verify_batch<N>(x, c, s.ref));
}

// What leaving one entry of size s.top out of its batch takes from the sum: the batch as it was added, and without.
template <int N>
__device__ __forceinline__ void verify_leave_out(float* x, float c, VerifyLane& s) {
  s.sum -= static_cast<double>(verify_batch<N>(x, c, s.ref));
  bool met = false;
#pragma unroll
  for (int e = 0; e < N; ++e) {
    const bool first = !met && x[e] == s.top;
    met = met || first;
    x[e] = first ? kMinusInf : x[e];
  }
  s.sum += static_cast<double>(verify_batch<N>(x, c, s.ref));
}

// A piece of -inf alone adds what it has: 0, or NaN.
__device__ __forceinline__ void verify_merge(float c, RowPart& p, RowPart q) {
  if (q.top > p.top || (q.top == p.top && q.at < p.at)) {
    const RowPart was = p;
    p = q;
    q = was;
  }
  p.others += q.top == kMinusInf ? q.others : (q.others + 1.f) * fast_exp2((q.top - p.top) * c);
}

__device__ __forceinline__ RowPart shuffled(const RowPart& p, int off) {
  return RowPart{__shfl_xor(p.top, off, 64), __shfl_xor(p.others, off, 64), __shfl_xor(p.at, off, 64), 0};
}

__device__ __forceinline__ bool is_distribution(const RowPart& p) {
  return p.top > kMinusInf && p.top < __builtin_inff() && p.others < __builtin_inff();          // (false for NaN)
}

// Of an entry z of the row: log of its probability, and the probability.
__device__ __forceinline__ double verify_log(const RowPart& p, float c, float z) {
  return (static_cast<double>(z) - static_cast<double>(p.top)) * static_cast<double>(c) * kLn2 - log1p(static_cast<double>(p.others));
}
__device__ __forceinline__ double verify_probability(const RowPart& p, float c, float z) {
  return exp2((static_cast<double>(z) - static_cast<double>(p.top)) * static_cast<double>(c)) / (1.0 + static_cast<double>(p.others));
}

}  // namespace

// Workgroup ((sample, tensor) (K + 1) + row) splits + piece, the tensors of a sample one after the other; parts[(tensor R + row of
// the tensor) splits + piece].  Rows of workgroups from first_cached on stay in the Infinity Cache for the race.  Also puts the
// drafted tokens' logits down (drafted[tensor R + row]) and starts the samples' races.
template <int DT>
__global__ void __launch_bounds__(kVerifyThreads)
fopd_verify_rows(VerifyArgs a, int splits, int piece_vecs, RowPart* __restrict__ parts, float* __restrict__ drafted,
                 RaceState* __restrict__ races, unsigned first_cached) {
  constexpr int E = Elem<DT>::kPerVec, U = 2;
  const unsigned unit = blockIdx.x / static_cast<unsigned>(splits);
  const int piece = static_cast<int>(blockIdx.x - unit * splits);
  const unsigned per = static_cast<unsigned>(a.K + 1);
  const unsigned side = unit / per, i = a.draft != nullptr ? side >> 1 : side;
  const int j = static_cast<int>(unit - side * per);
  const bool drafter = a.draft != nullptr && (side & 1) != 0;
  const int tid = threadIdx.x;
  if (!drafter && j == 0 && piece == 0 && tid == 0) races[i] = RaceState{0, 0, 0};
  const VerifySample s = verify_sample(a, static_cast<int>(i));
  if (!s.there || j > s.len || (drafter && (s.greedy || j == s.len))) return;
  const int64_t r = s.row + j;
  const char* row = drafter ? static_cast<const char*>(a.draft) + r * a.ld_draft * Elem<DT>::kBytes
                            : static_cast<const char*>(a.target) + r * a.ld * Elem<DT>::kBytes;
  const u32x4* rv = reinterpret_cast<const u32x4*>(row);
  const int nvec = a.V / E, begin = piece * piece_vecs;
  const int end = min(nvec, begin + piece_vecs);
  const bool last_piece = piece == splits - 1;
  const int x_id = tid == 0 && j < s.len ? a.draft_ids[r] : -1;
  const int tail = nvec * E + tid;            // fewer entries than a vector has
  const bool has_tail = last_piece && tail < a.V;
  VerifyLane mine;
  auto walk = [&](auto cached_tag) {
    constexpr bool CACHED = decltype(cached_tag)::value;
    int v = begin + tid;
    for (; v + (U - 1) * kVerifyThreads < end; v += U * kVerifyThreads) {
      u32x4 q[U];
#pragma unroll
      for (int u = 0; u < U; ++u) q[u] = load_vec<CACHED>(rv + v + u * kVerifyThreads);
      float x[U * E];
#pragma unroll
      for (int u = 0; u < U; ++u) unpack<DT>(q[u], x + u * E);
      verify_add<U * E>(x, s.c, v, mine);
    }
    for (; v < end; v += kVerifyThreads) {
      float x[E];
      unpack<DT>(load_vec<CACHED>(rv + v), x);
      verify_add<E>(x, s.c, v, mine);
    }
  };
  if (blockIdx.x >= first_cached) walk(std::true_type());
  else walk(std::false_type());
  if (has_tail) {
    const float x = load_elem<DT>(row, tail);
    verify_add<1>(&x, s.c, nvec, mine);
  }
  __shared__ float sh_top[kVerifyThreads / 64], sh_sum[kVerifyThreads / 64];
  __shared__ int sh_holder, sh_at;
  const float wave_top = wave_max(mine.top);
  if ((tid & 63) == 0) sh_top[tid >> 6] = wave_top;
  if (tid == 0) {
    sh_holder = kVerifyThreads;
    sh_at = kNowhere;
  }
  __syncthreads();
  float top = sh_top[0];
#pragma unroll
  for (int w = 1; w < kVerifyThreads / 64; ++w) top = fmaxf(top, sh_top[w]);
  const bool holds = mine.batch >= 0 && mine.top == top;
  if (holds) atomicMin(&sh_holder, tid);
  __syncthreads();
  if (holds && (s.greedy || sh_holder == tid)) {           // the largest entry's batch once more: a lane or two
    const bool leave_out = sh_holder == tid;
    int first = tail;
    if (mine.batch == nvec) {
      float x = load_elem<DT>(row, tail);
      if (leave_out) verify_leave_out<1>(&x, s.c, mine);
    } else {
      float x[U * E];
      const bool whole = mine.batch + (U - 1) * kVerifyThreads < end;
#pragma unroll
      for (int u = U - 1; u >= 0; --u) {
        const int w = mine.batch + u * kVerifyThreads;
        unpack<DT>(rv[whole || u == 0 ? w : mine.batch], x + u * E);
#pragma unroll
        for (int e = E - 1; e >= 0; --e)
          if ((whole || u == 0) && x[u * E + e] == top) first = w * E + e;
      }
      if (leave_out && whole) verify_leave_out<U * E>(x, s.c, mine);
      if (leave_out && !whole) verify_leave_out<E>(x, s.c, mine);
    }
    if (s.greedy) atomicMin(&sh_at, first);
  }
  auto total = [&](float x) {                              // over the workgroup, in every lane
    x = wave_sum(x);
    __syncthreads();
    if ((tid & 63) == 0) sh_sum[tid >> 6] = x;
    __syncthreads();
    float all = sh_sum[0];
#pragma unroll
    for (int w = 1; w < kVerifyThreads / 64; ++w) all += sh_sum[w];
    return all;
  };
  // into units of the largest entry, which may be a rounding of its reference away from it
  const float ref = verify_reference(top, s.c);
  const float to_top = top == kMinusInf ? 1.f : fast_exp2(-fmaf(top, s.c, -ref));
  float others = total(mine.batch < 0 ? static_cast<float>(mine.sum) : static_cast<float>(mine.sum) * fast_exp2(mine.ref - ref) * to_top);
  if (top > kMinusInf && (!(fabsf(top) < 1e30f) || !(fabsf(top * s.c) < 1e38f) || !(others < __builtin_inff()))) {
    // a largest entry whose product with c is no finite number (rows of the type's lowest value), or NaN: again, with the
    // largest entry subtracted first.  (Entries of that size are equal or too far apart to count: the sum is a whole number.)
    float sum = 0.f;
    for (int w = begin + tid; w < end; w += kVerifyThreads) {
      float x[E];
      unpack<DT>(rv[w], x);
#pragma unroll
      for (int e = 0; e < E; ++e) sum += fast_exp2((x[e] - top) * s.c);
    }
    if (has_tail) sum += fast_exp2((load_elem<DT>(row, tail) - top) * s.c);
    others = total(sum) - 1.f;
  }
  if (tid != 0) return;
  const RowPart p = {top, others, sh_at, 0};
  const int64_t at = (drafter ? a.rows : 0) + r;
  parts[at * splits + piece] = p;
  if (x_id >= begin * E && x_id < (last_piece ? a.V : end * E)) drafted[at] = load_elem<DT>(row, x_id);
}

// Workgroup (B - 1 - sample) pieces + piece: the samples whose rows were read last come first.  Every workgroup of a sample makes the sample's decisions, the first one writes them down;
// the last one to finish its piece has the winner.  Dynamic LDS: 2 (K + 1) RowParts.
template <int DT>
__global__ void __launch_bounds__(kVerifyThreads)
fopd_verify_race(VerifyArgs a, int splits, const RowPart* __restrict__ parts, const float* __restrict__ drafted, int pieces,
                 int piece_vecs, RaceState* races, int32_t* __restrict__ flags) {
  constexpr int E = Elem<DT>::kPerVec;
  extern __shared__ __align__(16) unsigned char verify_smem[];
  RowPart* rows = reinterpret_cast<RowPart*>(verify_smem);             // [target, drafter][K + 1]
  __shared__ int sh_kept, sh_next, sh_last, sh_nothing;
  __shared__ RaceEntry sh_race[kVerifyThreads / 64];
  const unsigned nth = blockIdx.x / static_cast<unsigned>(pieces);
  const int i = a.B - 1 - static_cast<int>(nth), piece = static_cast<int>(blockIdx.x - nth * pieces);
  const int tid = threadIdx.x, lane = tid & 63;
  const VerifySample s = verify_sample(a, i);
  const int per = a.K + 1;
  const bool writes = piece == 0;
  if (!s.there) {
    if (writes) {
      if (tid == 0) {
        atomicOr(flags, kFlagSegments);
        a.n_accepted[i] = 0;
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
  // what the decisions take, asked for together: lane j of the first wavefront has draft j
  const bool with_draft = a.draft != nullptr && !s.greedy;
  const int64_t r_lane = s.row + min(lane, s.len);
  int x_lane = -1;
  float u_lane = 0.f, z_lane = 0.f, zq_lane = 0.f;
  if (tid < min(64, s.len)) {
    x_lane = a.draft_ids[r_lane];
    z_lane = drafted[r_lane];
    if (!s.greedy) u_lane = a.accept_u[r_lane];
    if (with_draft) zq_lane = drafted[a.rows + r_lane];
  }
  // the pieces of each row, `splits` lanes a row
  const int items = (with_draft ? 2 : 1) * (s.len + 1);
  for (int base = 0; base < items; base += kVerifyThreads / splits) {
    const int item = base + tid / splits;
    const bool drafter = item > s.len;
    const int j = drafter ? item - s.len - 1 : item;
    RowPart p = {kMinusInf, 0.f, kNowhere, 0};
    if (item < items && !(drafter && j == s.len))
      p = parts[((drafter ? a.rows : 0) + s.row + j) * splits + (tid & (splits - 1))];
    for (int off = splits >> 1; off > 0; off >>= 1) verify_merge(s.c, p, shuffled(p, off));
    if (item < items && (tid & (splits - 1)) == 0) rows[(drafter ? per : 0) + j] = p;
  }
  __syncthreads();
  if (tid < 64) {
    int kept = s.len, next = 1, bad = 0;
    for (int base = 0; base <= s.len; base += 64) {
      const int j = base + lane;
      bool keeps = true, usable = true;
      int problem = 0;
      if (j <= s.len) {
        const RowPart p = rows[j];
        if (base > 0 && j < s.len) {
          const int64_t r = s.row + j;
          x_lane = a.draft_ids[r];
          z_lane = drafted[r];
          if (!s.greedy) u_lane = a.accept_u[r];
          if (with_draft) zq_lane = drafted[a.rows + r];
        }
        const bool in_range = x_lane >= 0 && x_lane < a.V;
        usable = is_distribution(p);
        if (!usable) problem = kFlagDist;
        if (j < s.len && !in_range) problem |= kFlagToken;
        keeps = j < s.len && usable && in_range;
        if (s.greedy) {
          keeps = keeps && x_lane == p.at;
        } else {
          RowPart q = {0.f, 0.f, 0, 0};
          if (with_draft && j < s.len) {
            q = rows[per + j];
            if (!is_distribution(q)) {
              usable = keeps = false;
              problem |= kFlagDist;
            }
          }
          if (keeps) {
            const double qx = with_draft ? verify_probability(q, s.c, zq_lane) : 1.0;
            keeps = static_cast<double>(u_lane) * qx < verify_probability(p, s.c, z_lane);
          }
        }
      }
      const unsigned long long stops = __ballot(j <= s.len && !keeps);
      if (stops != 0) {                       // (row n always stops)
        const int first = __ffsll(stops) - 1;
        kept = base + first;
        next = __shfl(usable ? 1 : 0, first, 64);
        bad = __shfl(problem, first, 64);
        break;
      }
    }
    if (lane == 0) {
      sh_kept = kept;
      sh_next = next;
      if (writes) {
        if (bad != 0) atomicOr(flags, bad);
        a.n_accepted[i] = kept;
      }
    }
  }
  __syncthreads();
  const int kept = sh_kept, next = sh_next;
  const RowPart p = rows[kept];
  const int64_t r = s.row + kept;
  if (writes) {                               // the drafted tokens that are kept, nothing in the rows behind the next one
    const int last = a.row_begin == nullptr ? a.K : s.len;
    for (int j = tid; j <= last; j += kVerifyThreads) {
      if (j == kept) continue;
      a.out_ids[s.row + j] = j < kept ? a.draft_ids[s.row + j] : -1;
      a.out_logp[s.row + j] = j < kept ? static_cast<float>(verify_log(rows[j], s.c, drafted[s.row + j])) : 0.f;
      a.out_mask[s.row + j] = j < kept ? 1 : 0;
    }
  }
  const char* zrow = static_cast<const char*>(a.target) + r * a.ld * Elem<DT>::kBytes;
  const bool rejected = kept < s.len, minus = rejected && with_draft;
  const int out = rejected && !with_draft && !s.greedy ? a.draft_ids[r] : -1;             // the token that is taken out
  const RowPart q = minus ? rows[per + kept] : RowPart{0.f, 0.f, 0, 0};
  const float ratio = (1.f + p.others) / (1.f + q.others);             // r in units of the target's sum: pv - ratio qv
  const char* qrow = minus ? static_cast<const char*>(a.draft) + r * a.ld_draft * Elem<DT>::kBytes : zrow;
  const float* noise = a.noise + static_cast<int64_t>(i) * a.ld_noise;
  const int nvec = a.V / E;
  RaceEntry best = {-1.f, kNowhere};
  auto merge = [&](float score, int at) {
    if (score > best.score || (score == best.score && at < best.at)) best = RaceEntry{score, at};
  };
  // entries of vectors begin .. end - 1 (and the tail) into the race; FULL: by p
  auto enter = [&](auto full_tag, auto minus_tag, int begin, int end, bool with_tail) {
    constexpr bool FULL = decltype(full_tag)::value, MINUS = decltype(minus_tag)::value;
    auto one = [&](int v, float z, float zq, float e) {
      float w = fast_exp2((z - p.top) * s.c);
      if (MINUS) w -= ratio * fast_exp2((zq - q.top) * s.c);
      else if (!FULL && v == out) w = 0.f;
      const float score = w * __builtin_amdgcn_rcpf(e);                // (an error of one unit in the last place, as w has)
      if (w > 0.f && score > best.score) best = RaceEntry{score, v};    // (a lane's indices only grow)
    };
    for (int v = begin + tid; v < end; v += kVerifyThreads) {
      float z[E], zq[E], e[E];
      unpack<DT>(reinterpret_cast<const u32x4*>(zrow)[v], z);
      if (MINUS) unpack<DT>(reinterpret_cast<const u32x4*>(qrow)[v], zq);
#pragma unroll
      for (int h = 0; h < E / 4; ++h) unpack<FOPD_F32>(reinterpret_cast<const u32x4*>(noise)[v * (E / 4) + h], e + 4 * h);
#pragma unroll
      for (int k = 0; k < E; ++k) one(v * E + k, z[k], MINUS ? zq[k] : 0.f, e[k]);
    }
    const int v = nvec * E + tid;
    if (with_tail && v < a.V) one(v, load_elem<DT>(zrow, v), MINUS ? load_elem<DT>(qrow, v) : 0.f, noise[v]);
  };
  auto reduce = [&]() {                       // the workgroup's first, in every lane of the first wavefront
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) merge(__shfl_xor(best.score, off, 64), __shfl_xor(best.at, off, 64));
    __syncthreads();
    if (lane == 0) sh_race[tid >> 6] = best;
    __syncthreads();
    if (tid < 64)
      for (int w = 0; w < kVerifyThreads / 64; ++w) merge(sh_race[w].score, sh_race[w].at);
  };
  bool found = next != 0;
  if (s.greedy || next == 0) {                // nothing to race for
    if (!writes) return;
    best = RaceEntry{1.f, p.at};
  } else {
    const int begin = piece * piece_vecs, end = min(nvec, begin + piece_vecs);
    if (minus) enter(std::false_type(), std::true_type(), begin, end, piece == pieces - 1);
    else enter(std::false_type(), std::false_type(), begin, end, piece == pieces - 1);
    reduce();
    if (pieces > 1) {
      // Both atomics are done where all XCDs' caches meet and the first has come back before the second is sent, so whoever is
      // the last one through finds every workgroup's best there.  (A release and an acquire around them instead write
      // back and drop whole L2s, once a workgroup: 192 samples x 10 workgroups 148 us, 56 with a kernel of its own for this.)
      if (tid == 0) {
        unsigned long long key = best.at == kNowhere ? 0ull : (static_cast<unsigned long long>(__float_as_uint(best.score)) << 32) | (0xffffffffu - best.at);
        key = max(key, __hip_atomic_fetch_max(&races[i].best, key, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT));
        asm volatile("s_waitcnt vmcnt(0)" ::"v"(key) : "memory");
        sh_last = __hip_atomic_fetch_add(&races[i].through, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == pieces - 1;
      }
      __syncthreads();
      if (sh_last == 0) return;
      if (tid == 0) {
        const unsigned long long key = __hip_atomic_fetch_max(&races[i].best, 0ull, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        best = key == 0 ? RaceEntry{-1.f, kNowhere} : RaceEntry{__uint_as_float(static_cast<uint32_t>(key >> 32)), static_cast<int32_t>(0xffffffffu - static_cast<uint32_t>(key))};
      }
    }
    if (tid == 0) sh_nothing = best.at == kNowhere;        // (not sh_last, which other wavefronts may still have to read)
    __syncthreads();
    if (sh_nothing != 0) {                     // p nowhere above q, by rounding or because accept_u is 1: p itself
      best = RaceEntry{-1.f, kNowhere};
      enter(std::true_type(), std::false_type(), 0, nvec, true);
      reduce();
    }
  }
  if (tid != 0) return;
  if (found && best.at == kNowhere) {         // no variate is a number
    atomicOr(flags, kFlagDist);
    found = false;
  }
  a.out_ids[r] = found ? best.at : -1;
  a.out_logp[r] = found ? static_cast<float>(verify_log(p, s.c, load_elem<DT>(zrow, best.at))) : __builtin_nanf("");
  a.out_mask[r] = found ? 1 : 0;
}

}  // namespace fopd

#endif  // FOPD_VERIFY_HIP_
