// Verification of proposed tokens against the target's distributions, from given random numbers.  Question u has T_u rows of
// the target, row a checking proposal x_a, the last one checking none.  With p_a and q_a the distributions of the target and
// of what proposed,
//   x_a stands           iff all before it stand and U_a q_a(x_a) < p_a(x_a);
//   after n that stand   w = max(p_n - q_n, 0) if proposal n was refused, w = p_n if there was none;
//   the token            = the first i with  sum_{j <= i} w_j > U_last sum_j w_j.
// A choice among 10^5 tokens lies next to a border often enough that 32 bits would choose another one now and then: weights,
// sums and their prefixes are held in 64 bits throughout.
//
// verify_stats_kernel   logits only: largest value, sum of exponentials around it and place of the largest, of each piece of
//                       every row (the one pass over all of them)
// verify_weigh_kernel   which proposals stand; sums of w over pieces of the row that decides
// verify_pick_kernel    the piece in which the running sum passes its share, the token in it, what is written
#include <cmath>
#include <cstdint>

#include "kernels.hpp"

namespace {

typedef unsigned uintx4 __attribute__((ext_vector_type(4)));

constexpr int kThreads = 256;
constexpr int kPiece = 8192;   // values of a piece of statistics
constexpr int kShare = 4096;   // values of a piece of weights

struct Decision {
  int32_t row, stands;  // row of the target that the token is drawn from (-1: no rows); proposals that stand
  int32_t refused;      // 0: w = p; 1: w = max(p - q, 0); 2: w = p without the proposal
  int32_t token;        // greedy: the token; else -1
  int32_t proposal;
  float top_p, top_q;
  int32_t pad;
  double inv_p, inv_q;  // 1 / sum of exponentials
};

// pieces of the workspace
struct Work {
  double* sum;      // [2 n_tokens][pieces]: target rows, then the rows of what proposed
  float* top;
  int32_t* place;
  double *weight, *plain;  // [n_queries][shares]: sums of w and of p
  Decision* decision;      // [n_queries]
  int pieces, shares;
};
__host__ __device__ inline int64_t pieces_of(int64_t n, int64_t size) { return (n + size - 1) / size; }
__host__ __device__ inline Work work_of(void* base, int64_t n_tokens, int64_t n_queries, int64_t vocab) {
  Work w;
  // (a row may begin up to seven values off a 16-byte address)
  w.pieces = static_cast<int>(pieces_of(vocab + 7, kPiece));
  w.shares = static_cast<int>(pieces_of(vocab, kShare));
  char* at = static_cast<char*>(base);
  w.decision = reinterpret_cast<Decision*>(at);
  at += n_queries * static_cast<int64_t>(sizeof(Decision));
  w.weight = reinterpret_cast<double*>(at);
  at += n_queries * w.shares * 8;
  w.plain = reinterpret_cast<double*>(at);
  at += n_queries * w.shares * 8;
  const int64_t cells = 2 * n_tokens * w.pieces;
  w.sum = reinterpret_cast<double*>(at);
  at += cells * 8;
  w.top = reinterpret_cast<float*>(at);
  at += cells * 4;
  w.place = reinterpret_cast<int32_t*>(at);
  return w;
}

// 2^t for t <= 0 in 64 bits, to 2e-12 of it: the nearest whole number goes to the exponent, the rest through the polynomial
// that meets 2^f at the nine Chebyshev points of [-1/2, 1/2].  No number and what lies below 2^-1074 give 0.
__device__ inline double exp2_below(double t) {
  t = fmax(t, -1100.0);
  const double shifted = t + 6755399441055744.0;  // 3 * 2^51: the sum's low bits hold the whole number
  const double f = t - (shifted - 6755399441055744.0);
  double y = 0x1.63d1363930791p-20;
  y = fma(y, f, 0x1.00dc4a53395d3p-16);
  y = fma(y, f, 0x1.4308ac85a7718p-13);
  y = fma(y, f, 0x1.5d8745a72831bp-10);
  y = fma(y, f, 0x1.3b2ab7181b778p-7);
  y = fma(y, f, 0x1.c6b08dd6fd236p-5);
  y = fma(y, f, 0x1.ebfbdff823cedp-3);
  y = fma(y, f, 0x1.62e42fef84cf0p-1);
  y = fma(y, f, 1.0);
  return ldexp(y, static_cast<int>(__double2loint(shifted)));
}

// e^((x - top) / T): factor = log2(e) / T.  Infinite values share everything between them; a row of none above -infinity has
// no weight.
__device__ inline double weight_of(float x, float top, double factor) {
  if (top == INFINITY) return x == INFINITY ? 1.0 : 0.0;
  if (!(top > -INFINITY)) return 0.0;
  return exp2_below((static_cast<double>(x) - static_cast<double>(top)) * factor);
}

__device__ inline float widen(float x) { return x; }
__device__ inline float widen(__bf16 x) { return static_cast<float>(x); }
template <typename T>
__device__ inline float at(const T* p, int64_t i) { return widen(p[i]); }

// a probability that is no number, negative or infinite counts as none
__device__ inline double clean(float p) { return p > 0.f && p < INFINITY ? static_cast<double>(p) : 0.0; }

__device__ inline float wave_max(float v) {
#pragma unroll
  for (int s = 32; s > 0; s >>= 1) v = fmaxf(v, __shfl_xor(v, s));
  return v;
}
__device__ inline double wave_sum(double v) {
#pragma unroll
  for (int s = 32; s > 0; s >>= 1) v += __shfl_xor(v, s);
  return v;
}
__device__ inline int wave_min(int v) {
#pragma unroll
  for (int s = 32; s > 0; s >>= 1) v = min(v, __shfl_xor(v, s));
  return v;
}

struct Span {
  int begin, end;
};
__device__ inline Span span_of(const VerifyParams& p, int u) {
  const int begin = min(max(p.cu[u], 0), p.n_tokens);
  return {begin, min(max(p.cu[u + 1], begin), p.n_tokens)};
}
// 1 / T as the factor of base-2 exponents; a temperature that is not above 0 is greedy, its statistics those of T = 1
__device__ inline bool greedy_of(const VerifyParams& p, int u) { return p.heat && !(p.heat[u] > 0.f); }
__device__ inline double factor_of(const VerifyParams& p, int u, bool greedy) {
  const double heat = p.heat && !greedy ? static_cast<double>(p.heat[u]) : 1.0;
  return 1.4426950408889634074 / heat;
}
template <typename T>
__device__ inline const T* target_row(const VerifyParams& p, int64_t row) { return static_cast<const T*>(p.target) + row * p.target_stride; }
template <typename T>
__device__ inline const T* draft_row(const VerifyParams& p, int64_t u, int64_t step) {
  return static_cast<const T*>(p.draft) + u * p.draft_query + step * p.draft_step;
}
// whether row t checks a proposal: a token of the vocabulary that a row of probabilities belongs to
__device__ inline bool proposes(const VerifyParams& p, const Span& s, int row) {
  if (row + 1 >= s.end) return false;
  const int x = p.tokens[row + 1];
  return x >= 0 && x < p.vocab && (!p.draft || row - s.begin < p.draft_steps);
}

// One workgroup: a piece of a row.  Values stay in registers between the maximum and the sum.
template <typename T>
__global__ __launch_bounds__(kThreads) void verify_stats_kernel(VerifyParams p) {
  constexpr int kWide = 16 / sizeof(T), kLoads = kPiece / kThreads / kWide;
  const Work w = work_of(p.workspace, p.n_tokens, p.n_queries, p.vocab);
  const int64_t cell = blockIdx.x;
  const int piece = static_cast<int>(cell % w.pieces);
  const int64_t which = cell / w.pieces;
  const bool of_draft = which >= p.n_tokens;
  const int row = static_cast<int>(of_draft ? which - p.n_tokens : which);
  __shared__ float top_sh[kThreads / 64];
  __shared__ double sum_sh[kThreads / 64];
  __shared__ int place_sh[kThreads / 64];
  // the question: as many as end at or before this row
  int u = 0;
  for (int i = 0; i < p.n_queries; i += kThreads) {
    const int mine = i + static_cast<int>(threadIdx.x);
    u += __syncthreads_count(mine < p.n_queries && p.cu[mine + 1] <= row);
  }
  if (u >= p.n_queries) return;
  const Span s = span_of(p, u);
  if (row < s.begin || row >= s.end) return;
  const bool greedy = greedy_of(p, u);
  if (of_draft && (greedy || !proposes(p, s, row))) return;
  const double factor = factor_of(p, u, greedy);
  const T* const from = of_draft ? draft_row<T>(p, u, row - s.begin) : target_row<T>(p, row);
  // 16-byte pieces from the address at or before the row's first value
  const int lead = static_cast<int>(reinterpret_cast<uintptr_t>(from) % 16 / sizeof(T));
  float x[kLoads][kWide];
  float top = -INFINITY;
#pragma unroll
  for (int i = 0; i < kLoads; ++i) {
    const int64_t first = static_cast<int64_t>(piece) * kPiece + (i * kThreads + threadIdx.x) * kWide - lead;
    if (first >= 0 && first + kWide <= p.vocab) {
      const uintx4 v = *reinterpret_cast<const uintx4*>(from + first);
#pragma unroll
      for (int e = 0; e < kWide; ++e)
        x[i][e] = sizeof(T) == 2 ? __uint_as_float(e % 2 ? v[e / 2] & 0xffff0000u : v[e / 2] << 16) : __uint_as_float(v[e % 4]);
    } else {
#pragma unroll
      for (int e = 0; e < kWide; ++e) x[i][e] = first + e >= 0 && first + e < p.vocab ? at(from, first + e) : -INFINITY;
    }
#pragma unroll
    for (int e = 0; e < kWide; ++e) top = fmaxf(top, x[i][e]);  // (passes over what is no number)
  }
  top = wave_max(top);
  const int wave = threadIdx.x / 64;
  if (threadIdx.x % 64 == 0) top_sh[wave] = top;
  __syncthreads();
#pragma unroll
  for (int i = 0; i < kThreads / 64; ++i) top = fmaxf(top, top_sh[i]);
  double sum = 0;
  if (top == INFINITY) {
#pragma unroll
    for (int i = 0; i < kLoads; ++i)
#pragma unroll
      for (int e = 0; e < kWide; ++e) sum += x[i][e] == INFINITY ? 1.0 : 0.0;
  } else if (top > -INFINITY) {
#pragma unroll
    for (int i = 0; i < kLoads; ++i)
#pragma unroll
      for (int e = 0; e < kWide; ++e) sum += exp2_below((static_cast<double>(x[i][e]) - static_cast<double>(top)) * factor);
  }
  int place = p.vocab;
  if (greedy && top > -INFINITY) {
#pragma unroll
    for (int i = kLoads - 1; i >= 0; --i)
#pragma unroll
      for (int e = kWide - 1; e >= 0; --e) {
        const int64_t index = static_cast<int64_t>(piece) * kPiece + (i * kThreads + threadIdx.x) * kWide - lead + e;
        if (x[i][e] == top && index >= 0 && index < p.vocab) place = static_cast<int>(index);
      }
  }
  sum = wave_sum(sum);
  place = wave_min(place);
  if (threadIdx.x % 64 == 0) {
    sum_sh[wave] = sum;
    place_sh[wave] = place;
  }
  __syncthreads();
  if (threadIdx.x == 0) {
    for (int i = 1; i < kThreads / 64; ++i) {
      sum += sum_sh[i];
      place = min(place, place_sh[i]);
    }
    w.sum[cell] = sum;
    w.top[cell] = top;
    w.place[cell] = place;
  }
}

// Statistics of a whole row from its pieces, by one wave.
struct RowStats {
  float top;
  double sum;
  int place;
};
__device__ inline RowStats row_stats(const Work& w, int64_t which, double factor) {
  const int lane = threadIdx.x % 64;
  RowStats r{-INFINITY, 0.0, INT32_MAX};
  for (int i = lane; i < w.pieces; i += 64) r.top = fmaxf(r.top, w.top[which * w.pieces + i]);
  r.top = wave_max(r.top);
  for (int i = lane; i < w.pieces; i += 64) {
    const float top = w.top[which * w.pieces + i];
    r.sum += w.sum[which * w.pieces + i] * (top == r.top ? 1.0 : weight_of(top, r.top, factor));
    if (top == r.top) r.place = min(r.place, w.place[which * w.pieces + i]);
  }
  r.sum = wave_sum(r.sum);
  r.place = wave_min(r.place);
  return r;
}
__device__ inline double inverse(double sum) { return sum > 0 ? 1.0 / sum : 0.0; }

// Which proposals of question u stand, by a whole workgroup: every thread gets the decision.
template <typename T, bool kLogits>
__device__ Decision decide(const VerifyParams& p, const Work& w, int u, const Span& s, bool greedy, double factor) {
  __shared__ int stop_sh;
  __shared__ Decision decision_sh;
  const int wave = threadIdx.x / 64;
  if (threadIdx.x == 0) stop_sh = s.end - 1;
  __syncthreads();
  for (int first = s.begin; first < s.end - 1; first += kThreads / 64) {
    const int row = first + wave;
    if (row < s.end - 1) {
      bool stands = proposes(p, s, row);
      if (stands) {
        const int x = p.tokens[row + 1];
        double px, qx = 1.0;
        if constexpr (kLogits) {
          const RowStats a = row_stats(w, row, factor);
          if (greedy) {
            px = x == a.place ? 1.0 : 0.0;
            qx = 0.0;
          } else {
            px = weight_of(at(target_row<T>(p, row), x), a.top, factor) * inverse(a.sum);
            if (p.draft) {
              const RowStats b = row_stats(w, static_cast<int64_t>(p.n_tokens) + row, factor);
              qx = weight_of(at(draft_row<T>(p, u, row - s.begin), x), b.top, factor) * inverse(b.sum);
            }
          }
        } else {
          px = clean(at(target_row<T>(p, row), x));
          if (p.draft) qx = clean(at(draft_row<T>(p, u, row - s.begin), x));
        }
        stands = static_cast<double>(p.uniform[row]) * qx < px;
      }
      if (!stands && threadIdx.x % 64 == 0) atomicMin(&stop_sh, row);
    }
    __syncthreads();
    const bool done = stop_sh < first + kThreads / 64;
    __syncthreads();
    if (done) break;
  }
  const int stop = stop_sh;
  if (wave == 0) {
    Decision d{};
    d.row = stop;
    d.stands = stop - s.begin;
    d.token = -1;
    d.refused = proposes(p, s, stop) ? (p.draft ? 1 : 2) : 0;
    d.proposal = d.refused ? p.tokens[stop + 1] : -1;
    if constexpr (kLogits) {
      const RowStats a = row_stats(w, stop, factor);
      d.top_p = a.top;
      d.inv_p = inverse(a.sum);
      if (greedy) d.token = a.place < p.vocab ? a.place : -1;
      else if (d.refused == 1) {
        const RowStats b = row_stats(w, static_cast<int64_t>(p.n_tokens) + stop, factor);
        d.top_q = b.top;
        d.inv_q = inverse(b.sum);
      }
    }
    if (threadIdx.x == 0) decision_sh = d;
  }
  __syncthreads();
  return decision_sh;
}

// (w, p) of value i of the row that decides.  Both products are rounded, so that equal distributions leave exactly nothing.
struct Pair {
  double w, p;
};
template <typename T, bool kLogits>
__device__ inline Pair pair_at(const Decision& d, const T* target, const T* draft, int i, double factor) {
#pragma clang fp contract(off)
  const float x = at(target, i);
  double a, b = 0.0;
  if constexpr (kLogits) a = weight_of(x, d.top_p, factor) * d.inv_p;
  else a = clean(x);
  if (d.refused == 1) {
    const float y = at(draft, i);
    if constexpr (kLogits) b = weight_of(y, d.top_q, factor) * d.inv_q;
    else b = clean(y);
  }
  const double left = d.refused == 2 && i == d.proposal ? 0.0 : fmax(a - b, 0.0);
  return {left, a};
}

// Exclusive prefix of v over the workgroup, and its total.
__device__ inline double scan(double v, double& total) {
  __shared__ double part[kThreads / 64];
  const int lane = threadIdx.x % 64, wave = threadIdx.x / 64;
  double up = v;
#pragma unroll
  for (int s = 1; s < 64; s <<= 1) {
    const double other = __shfl_up(up, s);
    if (lane >= s) up += other;
  }
  __syncthreads();
  if (lane == 63) part[wave] = up;
  __syncthreads();
  double before = 0;
  total = 0;
  for (int i = 0; i < kThreads / 64; ++i) {
    if (i < wave) before += part[i];
    total += part[i];
  }
  return before + up - v;
}

// One workgroup: a share of the row that decides for question u.
template <typename T, bool kLogits>
__global__ __launch_bounds__(kThreads) void verify_weigh_kernel(VerifyParams p) {
  const Work w = work_of(p.workspace, p.n_tokens, p.n_queries, p.vocab);
  const int share = static_cast<int>(blockIdx.x % w.shares), u = static_cast<int>(blockIdx.x / w.shares);
  const Span s = span_of(p, u);
  if (s.begin == s.end) {
    if (share == 0 && threadIdx.x == 0) w.decision[u].row = -1;
    return;
  }
  const bool greedy = kLogits && greedy_of(p, u);
  const double factor = kLogits ? factor_of(p, u, greedy) : 0.0;
  const Decision d = decide<T, kLogits>(p, w, u, s, greedy, factor);
  if (share == 0 && threadIdx.x == 0) w.decision[u] = d;
  if (greedy) return;
  const T* const target = target_row<T>(p, d.row);
  const T* const draft = d.refused == 1 ? draft_row<T>(p, u, d.row - s.begin) : nullptr;
  double weight = 0, plain = 0;
#pragma unroll 4
  for (int i = share * kShare + threadIdx.x; i < min((share + 1) * kShare, p.vocab); i += kThreads) {
    const Pair x = pair_at<T, kLogits>(d, target, draft, i, factor);
    weight += x.w;
    plain += x.p;
  }
  double all_weight, all_plain;
  scan(weight, all_weight);
  scan(plain, all_plain);
  if (threadIdx.x == 0) {
    w.weight[static_cast<int64_t>(u) * w.shares + share] = all_weight;
    w.plain[static_cast<int64_t>(u) * w.shares + share] = all_plain;
  }
}

// One workgroup: question u.
template <typename T, bool kLogits>
__global__ __launch_bounds__(kThreads) void verify_pick_kernel(VerifyParams p) {
  const Work w = work_of(p.workspace, p.n_tokens, p.n_queries, p.vocab);
  const int u = blockIdx.x;
  const Span s = span_of(p, u);
  const int tid = threadIdx.x;
  __shared__ int token_sh, share_sh, last_sh;
  __shared__ double before_sh;
  Decision d = w.decision[u];
  if (s.begin == s.end) {
    if (tid == 0) {
      p.accepted[u] = 0;
      if (p.new_len) p.new_len[u] = p.self_len[u];
    }
    return;
  }
  const bool greedy = kLogits && greedy_of(p, u);
  const double factor = kLogits ? factor_of(p, u, greedy) : 0.0;
  int token = d.token;
  if (!greedy) {
    const double* sums = w.weight + static_cast<int64_t>(u) * w.shares;
    double total = 0;
    for (int i = tid; i < w.shares; i += kThreads) total += sums[i];
    double all;
    scan(total, all);
    if (!(all > 0)) {  // the target lies nowhere above what proposed
      d.refused = 0;
      sums = w.plain + static_cast<int64_t>(u) * w.shares;
      total = 0;
      for (int i = tid; i < w.shares; i += kThreads) total += sums[i];
      scan(total, all);
    }
    if (all > 0) {
      const double want = static_cast<double>(p.uniform[s.end - 1]) * all;
      // the share in which the running sum passes `want`; behind the last, the last that has any
      if (tid == 0) {
        share_sh = INT32_MAX;
        last_sh = 0;
        token_sh = p.vocab;
      }
      double before = 0;
      for (int i = 0; i < w.shares; i += kThreads) {
        const double here = i + tid < w.shares ? sums[i + tid] : 0.0;
        double round;
        const double mine = before + scan(here, round);  // (its barriers are behind the lines above, and the last round's)
        if (here > 0) atomicMax(&last_sh, i + tid);
        if (here > 0 && mine + here > want) atomicMin(&share_sh, i + tid);
        __syncthreads();
        if (i + tid == share_sh || (share_sh == INT32_MAX && i + tid == last_sh)) before_sh = mine;
        before += round;
        if (share_sh != INT32_MAX) break;
      }
      __syncthreads();
      const int share = share_sh != INT32_MAX ? share_sh : last_sh;
      const T* const target = target_row<T>(p, d.row);
      const T* const draft = d.refused == 1 ? draft_row<T>(p, u, d.row - s.begin) : nullptr;
      constexpr int kMine = kShare / kThreads;
      const int first = share * kShare + tid * kMine;
      double mine[kMine], sum = 0;
      int last = -1;
#pragma unroll
      for (int e = 0; e < kMine; ++e) {
        mine[e] = first + e < p.vocab ? pair_at<T, kLogits>(d, target, draft, first + e, factor).w : 0.0;
        sum += mine[e];
        if (mine[e] > 0) last = first + e;
      }
      double unused, run = before_sh + scan(sum, unused);
      int found = p.vocab;
#pragma unroll
      for (int e = 0; e < kMine; ++e) {
        run += mine[e];
        if (found == p.vocab && run > want && mine[e] > 0) found = first + e;
      }
      found = wave_min(found);
      if (tid % 64 == 0) atomicMin(&token_sh, found);
      __syncthreads();
      token = token_sh;
      if (token == p.vocab) {  // (by rounding, or a number of 1 and more)
        __syncthreads();
        if (tid == 0) token_sh = -1;
        __syncthreads();
        last = -wave_min(-last);
        if (tid % 64 == 0) atomicMax(&token_sh, last);
        __syncthreads();
        token = token_sh;
      }
    } else {
      token = -1;
    }
  }
  for (int row = s.begin + tid; row < s.end; row += kThreads)
    p.out[row] = row < d.row ? p.tokens[row + 1] : row == d.row ? token : -1;
  if (tid == 0) {
    p.accepted[u] = d.stands;
    if (p.new_len) p.new_len[u] = p.self_len[u] - (s.end - 1 - d.row);
  }
  if (p.logp) {
    for (int row = s.begin + tid / 64; row < s.end; row += kThreads / 64) {
      double lp = 0;
      const int x = row < d.row ? p.tokens[row + 1] : row == d.row ? token : -1;
      if (x >= 0) {
        const float v = at(target_row<T>(p, row), x);
        if constexpr (kLogits) {
          const RowStats a = row_stats(w, row, factor);
          lp = (a.top == INFINITY ? 0.0 : (static_cast<double>(v) - static_cast<double>(a.top)) * factor * 0.69314718055994530942) - log(a.sum);
        } else {
          lp = log(clean(v));
        }
      }
      if (tid % 64 == 0) p.logp[row] = static_cast<float>(lp);
    }
  }
}

template <typename T>
void launch(const VerifyParams& p, bool logits, hipStream_t stream) {
  const Work w = work_of(p.workspace, p.n_tokens, p.n_queries, p.vocab);
  const dim3 threads(kThreads);
  if (logits) {
    const int64_t rows = (p.draft ? 2 : 1) * static_cast<int64_t>(p.n_tokens);
    if (rows > 0) verify_stats_kernel<T><<<dim3(static_cast<unsigned>(rows * w.pieces)), threads, 0, stream>>>(p);
    verify_weigh_kernel<T, true><<<dim3(static_cast<unsigned>(p.n_queries * w.shares)), threads, 0, stream>>>(p);
    verify_pick_kernel<T, true><<<dim3(p.n_queries), threads, 0, stream>>>(p);
  } else {
    verify_weigh_kernel<T, false><<<dim3(static_cast<unsigned>(p.n_queries * w.shares)), threads, 0, stream>>>(p);
    verify_pick_kernel<T, false><<<dim3(p.n_queries), threads, 0, stream>>>(p);
  }
}

}  // namespace

size_t verify_workspace_bytes(int64_t n_tokens, int64_t n_queries, int64_t vocab) {
  const Work w = work_of(nullptr, n_tokens, n_queries, vocab);
  const size_t all = reinterpret_cast<size_t>(w.place) + static_cast<size_t>(2 * n_tokens * w.pieces) * 4;
  return (all + 15) / 16 * 16;
}

hipError_t launch_verify(const VerifyParams& p, bool bf16, bool logits, hipStream_t stream) {
  if (bf16) launch<__bf16>(p, logits, stream);
  else launch<float>(p, logits, stream);
  return hipGetLastError();
}
