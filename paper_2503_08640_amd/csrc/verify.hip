// Verification of proposed tokens against the target's distributions, from given random numbers.  Question u has T_u rows of
// the target, row a checking proposal x_a, the last one checking none.  With p_a and q_a the distributions of the target and
// of what proposed,
//   x_a stands           iff all before it stand and U_a q_a(x_a) < p_a(x_a);
//   after n that stand   w = max(p_n - q_n, 0) if proposal n was refused, w = p_n if there was none;
//   the token            = the first i with  sum_{j <= i} w_j > U_last sum_j w_j.
// A choice among 10^5 tokens lies next to a border often enough that 32 bits would choose another one now and then: weights,
// sums and their prefixes are held in 64 bits throughout.
//
// verify_stats_kernel   logits only: the sum of exponentials (and where it is asked for, the place of the largest value) of each
//                       piece of every row, the one pass over all of them
// verify_decide_kernel  many questions, from logits: which proposals stand
// verify_draw_kernel    else the same, first; then sums of w over shares of the row that decides, and the last workgroup of a question
//                       to be done finds the share in which the running sum passes its part, and the token in it
// 128 questions of 4 rows over 128256 words, proposals' logits beside them, a quarter greedy: 131 us in fp32 (92 + 6 + 31, 460 MB), 113
// in bf16 (82 + 6 + 28); one question of 5 rows over 32000 words: 16 us, two launches of chains of loads (4.5 + 9).
#include <cfloat>
#include <cmath>
#include <cstdint>

#include "kernels.hpp"

namespace {

typedef unsigned uintx4 __attribute__((ext_vector_type(4)));
typedef uintx4 loose_uintx4 __attribute__((aligned(2)));  // rows begin where they like: 16 bytes at any address of a value

constexpr int kThreads = 256, kWaves = kThreads / 64;
constexpr int kPieceLeast = 2048;  // values of a wave's piece of statistics
constexpr int kShare = 512;        // values whose weights a wave sums up as one
constexpr int kGroup = 16;         // lanes that look at one row, the next as many at the row of what proposed
constexpr int kRows = kThreads / (2 * kGroup);
constexpr int kApart = 64;         // counters lie 256 bytes apart

// What a row gives its weights from.
struct Decision {
  int row, step;        // that the token is drawn from, and its number in the question; row -1: no rows
  int refused;          // 0: w = p; 1: w = max(p - q, 0); 2: w = p without the proposal
  int proposal, place;  // place: of the largest value
  float top_p, top_q, number;
  double log_p, inv_p, inv_q;  // logarithm and inverse of the sums of exponentials
};

// pieces of the workspace
struct Work {
  double* sum;   // [2 n_tokens][pieces]: target rows, then the rows of what proposed
  double* rest;  // [n_tokens][pieces], where no distribution proposed: the same without the proposal
  float* top;    // what its weights are counted from
  float* peak;   // greedy: largest value and its place
  int32_t* place;
  double* weight;          // [n_queries][shares]: sums of w
  Decision* decision;      // [n_queries]
  unsigned* done;          // [n_queries][kApart]: workgroups that have left theirs
  int pieces, shares;
};
__host__ __device__ inline int64_t pieces_of(int64_t n, int64_t size) { return (n + size - 1) / size; }
__host__ __device__ inline Work work_of(void* base, int64_t n_tokens, int64_t n_queries, int64_t vocab, int64_t piece) {
  Work w;
  w.pieces = static_cast<int>(pieces_of(vocab, piece));
  w.shares = static_cast<int>(pieces_of(vocab, kShare));
  char* at = static_cast<char*>(base);
  w.decision = reinterpret_cast<Decision*>(at);
  at += n_queries * static_cast<int64_t>(sizeof(Decision));
  w.weight = reinterpret_cast<double*>(at);
  at += n_queries * w.shares * 8;
  const int64_t cells = 2 * n_tokens * w.pieces;
  w.sum = reinterpret_cast<double*>(at);
  at += cells * 8;
  w.rest = reinterpret_cast<double*>(at);
  at += cells * 4;
  w.top = reinterpret_cast<float*>(at);
  at += cells * 4;
  w.peak = reinterpret_cast<float*>(at);
  at += cells * 4;
  w.place = reinterpret_cast<int32_t*>(at);
  at += cells * 4;
  w.done = reinterpret_cast<unsigned*>(at);
  return w;
}

// 2^f for f in [-1/2, 1/2], to 2e-12 of it: the polynomial that meets it at the interval's nine Chebyshev points.
__device__ inline double exp2_part(double f) {
  double y = 0x1.63d1363930791p-20;
  y = fma(y, f, 0x1.00dc4a53395d3p-16);
  y = fma(y, f, 0x1.4308ac85a7718p-13);
  y = fma(y, f, 0x1.5d8745a72831bp-10);
  y = fma(y, f, 0x1.3b2ab7181b778p-7);
  y = fma(y, f, 0x1.c6b08dd6fd236p-5);
  y = fma(y, f, 0x1.ebfbdff823cedp-3);
  y = fma(y, f, 0x1.62e42fef84cf0p-1);
  return fma(y, f, 1.0);
}
// 2^t for any t; nothing below 2^-1074, however far
__device__ inline double exp2_of(double t) {
#pragma clang fp contract(off)  // (f would take what the product behind a large t was rounded by)
  const double whole = rint(t);
  int exponent;
  asm("v_cvt_i32_f64 %0, %1" : "=v"(exponent) : "v"(whole));  // (stays at the ends of its range)
  return __builtin_amdgcn_ldexp(exp2_part(t - whole), exponent);
}

// Weights 2^(x factor - reference), factor = log2(e) / T, are counted from the value `top`.  Where x factor stays within 2^20 the
// reference is the nearest whole number to top factor, which then enters the exponent alone: fourteen operations of 64 bits, four
// cycles each, which bound the statistics in bf16.  Where it does not, from top itself.
struct Scale {
  double factor, shift;  // shift: 3 * 2^51 less the reference: x factor + shift holds the exponent in its low bits
  float top, least, most;  // values beyond least and most weigh nothing, and more than 64 bits hold
  bool plain;
};
__device__ inline Scale scale_of(float top, double factor) {
  Scale s{factor, 0.0, top, 0.f, 0.f, false};
  const double reference = rint(static_cast<double>(top) * factor);
  s.plain = fabs(reference) < 0x1p20 && factor < 0x1p100;
  s.shift = 6755399441055744.0 - reference;
  const double inverse = 1.0 / factor;
  s.least = static_cast<float>((reference - 2000.0) * inverse);
  s.most = static_cast<float>((reference + 1100.0) * inverse);
  return s;
}
__device__ inline double plain_weight(float x, const Scale& s) {
  const double v = __builtin_amdgcn_fmed3f(x, s.least, s.most);  // (what is no number becomes the least)
  const double shifted = fma(v, s.factor, s.shift), whole = shifted - s.shift;
  return __builtin_amdgcn_ldexp(exp2_part(fma(v, s.factor, -whole)), __double2loint(shifted));
}
// What is no number, and -infinity, has no weight; infinite values share everything between them; a row of none above -infinity
// has no weight.
__device__ inline double weight_of(float x, const Scale& s) {
  if (s.plain) return plain_weight(x, s);
  if (s.top == INFINITY) return x == INFINITY ? 1.0 : 0.0;
  return x >= -FLT_MAX && s.top >= -FLT_MAX ? exp2_of((static_cast<double>(x) - static_cast<double>(s.top)) * s.factor) : 0.0;
}
// what weights counted from `from` are to be multiplied by to be counted from `to`, which is not lower
__device__ inline double rescale(const Scale& from, const Scale& to) {
  if (from.plain && to.plain) return exp2_of(to.shift - from.shift);
  if (from.top == to.top) return 1.0;
  if (to.top == INFINITY) return 0.0;
  if (from.plain || to.plain) return exp2_of((from.plain ? 6755399441055744.0 - from.shift : from.top * from.factor) -
                                             (to.plain ? 6755399441055744.0 - to.shift : to.top * to.factor));
  return exp2_of((static_cast<double>(from.top) - static_cast<double>(to.top)) * to.factor);
}

__device__ inline float widen(float x) { return x; }
__device__ inline float widen(__bf16 x) { return static_cast<float>(x); }
template <typename T>
__device__ inline float at(const T* p, int64_t i) { return widen(p[i]); }

// a probability that is no number, negative or infinite counts as none
__device__ inline double clean(float p) { return p > 0.f && p < INFINITY ? static_cast<double>(p) : 0.0; }

// natural logarithm of the probability of value x, from that of the sum of the weights counted from top
constexpr double kLn2 = 0.69314718055994530942;
template <bool kLogits>
__device__ inline double log_of(float x, float top, double log_sum, double factor) {
  if constexpr (!kLogits) return log(clean(x));
  return (top == INFINITY ? 0.0 : (static_cast<double>(x) - static_cast<double>(top)) * factor * kLn2) - log_sum;
}
__device__ inline double log_sum_of(double sum, const Scale& s) {  // counted from top
  return log(sum) + (s.plain ? (6755399441055744.0 - s.shift - static_cast<double>(s.top) * s.factor) * kLn2 : 0.0);
}

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
  const int from = p.cu[u], to = p.cu[u + 1], begin = min(max(from, 0), p.n_tokens);
  return {begin, min(max(to, begin), p.n_tokens)};
}
// A temperature that is not above 0 is greedy, its statistics those of T = 1.  (Above 1e30 it would give weight to what is masked
// with the type's lowest value.)
struct Heat {
  bool greedy;
  double factor;  // log2(e) / T
};
__device__ inline Heat heat_of(const VerifyParams& p, int u) {
  const float t = p.heat ? p.heat[u] : 1.f;
  const bool greedy = !(t > 0.f);
  return {greedy, 1.4426950408889634074 / (greedy ? 1.0 : static_cast<double>(fminf(t, 1e30f)))};
}
template <typename T>
__device__ inline const T* target_row(const VerifyParams& p, int64_t row) { return static_cast<const T*>(p.target) + row * p.target_stride; }
template <typename T>
__device__ inline const T* draft_row(const VerifyParams& p, int64_t u, int64_t step) {
  return static_cast<const T*>(p.draft) + u * p.draft_query + step * p.draft_step;
}
// whether row t checks proposal x: a token of the vocabulary that a row of probabilities belongs to
__device__ inline bool proposes(const VerifyParams& p, const Span& s, int row, int x) {
  return row + 1 < s.end && x >= 0 && x < p.vocab && row - s.begin < p.draft_steps;
}

// 16 / sizeof(T) values from the first-th on, in two steps, so that several loads are in flight before one is waited for: the
// load (behind the row's end: of its last 16 bytes), then the values, `none` behind the end.
template <typename T>
__device__ inline uintx4 load_wide(const T* row, int first, int vocab) {
  constexpr int n = 16 / sizeof(T);
  return vocab < n ? uintx4{} : *reinterpret_cast<const loose_uintx4*>(row + min(first, vocab - n));
}
template <typename T, int n = 16 / sizeof(T)>
__device__ inline void widen_all(uintx4 v, float (&x)[n]) {
#pragma unroll
  for (int e = 0; e < n; ++e)
    x[e] = sizeof(T) == 2 ? __uint_as_float(e % 2 ? v[e / 2] & 0xffff0000u : v[e / 2] << 16) : __uint_as_float(v[e % 4]);
}
template <typename T, int n = 16 / sizeof(T)>
__device__ inline void values_of(uintx4 v, const T* row, int first, int vocab, float none, float (&x)[n]) {
  if (first + n <= vocab) {
    widen_all<T>(v, x);
  } else {
#pragma unroll
    for (int e = 0; e < n; ++e) x[e] = first + e < vocab ? at(row, first + e) : none;
  }
}

// One wave: a piece of a row, in chunks of kLoads times 16 bytes a lane, the next chunk on its way while one is summed up.  The
// exponents are counted from the largest value of the first chunk that has one: 64 bits leave 2^1000 on either side, so that the
// maximum need not be followed.  A piece that holds more than that (or +infinity) is gone through again with its own, twice and a value
// at a time: also one whose first chunk with a value above -infinity holds finite masks alone (-1e9, the type's lowest value), which
// -infinity does not cost.  512 rows of 128256 values, the front half masked: 232 us in bf16 and 176 in fp32 with -1e9, 60 and 68 with
// -infinity; 1 in 100 left anywhere, with the lowest value: 78 and 112, 60 and 66.
// 800 rows of 128256 values: 92 us in fp32, memory (4.5 TB/s; a copy on this card reaches 5.0), 82 in bf16, operations (20.7 of a wave
// for 64 values, 82 % of the rate that such operations reach).  With a maximum and barriers per workgroup 100 and 95 us; pieces of half
// the size 3 to 5 % more, four loads on their way instead of two no less.
template <typename T>
__global__ __launch_bounds__(kThreads) void verify_stats_kernel(VerifyParams p, int piece) {
  constexpr int kWide = 16 / sizeof(T), kLoads = 2, kStep = 64 * kWide, kChunk = kLoads * kStep;
  const Work w = work_of(p.workspace, p.n_tokens, p.n_queries, p.vocab, piece);
  const int lane = threadIdx.x % 64;
  // (the counters of the kernels behind this one)
  for (int64_t i = static_cast<int64_t>(blockIdx.x) * kThreads + threadIdx.x; i < p.n_queries; i += static_cast<int64_t>(gridDim.x) * kThreads) w.done[i * kApart] = 0;
  const int64_t cell = static_cast<int64_t>(blockIdx.x) * kWaves + threadIdx.x / 64;
  const int64_t which = cell / w.pieces;
  if (which >= (p.draft ? 2 : 1) * static_cast<int64_t>(p.n_tokens)) return;
  const bool of_draft = which >= p.n_tokens;
  const int row = static_cast<int>(of_draft ? which - p.n_tokens : which);
  const int begin = static_cast<int>(cell - which * w.pieces) * piece, end = min(begin + piece, p.vocab);
  const int mine = begin + lane * kWide;
  uintx4 raw[kLoads];
  const T* from = target_row<T>(p, row);
  if (!of_draft) {  // (asked for before it is known what for)
#pragma unroll
    for (int i = 0; i < kLoads; ++i) raw[i] = load_wide(from, mine + i * kStep, p.vocab);
  }
  // the question: as many as end at or before this row, 64 bounds a step (2048 rows of 32000 values in bf16: 57 us for 2048 questions, 48
  // for 512; 4096 rows of 8000 in fp32: 69 us for 4096, 39 for 1024)
  int u = 0;
  for (int i = 0; i < p.n_queries; i += 64) u += __popcll(__ballot(i + lane < p.n_queries && p.cu[min(i + lane, p.n_queries - 1) + 1] <= row));
  if (u >= p.n_queries) return;
  const Span s = span_of(p, u);
  const Heat heat = heat_of(p, u);
  if (row < s.begin || row >= s.end) return;
  if (of_draft) {
    if (heat.greedy || row + 1 >= s.end || !proposes(p, s, row, p.tokens[row + 1])) return;
    from = draft_row<T>(p, u, row - s.begin);
#pragma unroll
    for (int i = 0; i < kLoads; ++i) raw[i] = load_wide(from, mine + i * kStep, p.vocab);
  }
  const bool sums = !heat.greedy || p.logp;
  // where no distribution proposed, the sum without the proposal is kept, too (a difference would leave what it was rounded by)
  int proposal = -1;
  if (!p.draft && !heat.greedy && row + 1 < s.end) proposal = p.tokens[row + 1];
  if (proposal < begin || proposal >= end) proposal = -1;
  float peak = -INFINITY;
  double sum = 0;
  int place = INT32_MAX;
  Scale scale{};
  scale.top = -INFINITY;
  for (int chunk = begin; chunk < end; chunk += kChunk) {
    float x[kLoads][kWide];
    const int first = chunk + lane * kWide;
    if (chunk + kChunk <= end) {
#pragma unroll
      for (int i = 0; i < kLoads; ++i) widen_all<T>(raw[i], x[i]);
    } else {
#pragma unroll
      for (int i = 0; i < kLoads; ++i) values_of(raw[i], from, first + i * kStep, end, -INFINITY, x[i]);
    }
    if (chunk + kChunk < end) {
#pragma unroll
      for (int i = 0; i < kLoads; ++i) raw[i] = load_wide(from, first + kChunk + i * kStep, p.vocab);
    }
    if (!(scale.top > -INFINITY)) {
      float top = -INFINITY;
#pragma unroll
      for (int i = 0; i < kLoads; ++i)
#pragma unroll
        for (int e = 0; e < kWide; ++e) top = fmaxf(top, x[i][e]);  // (passes over what is no number)
      top = wave_max(top);
      if (!(top > -INFINITY)) continue;
      scale = scale_of(top, heat.factor);
    }
    if (heat.greedy) {
#pragma unroll
      for (int i = 0; i < kLoads; ++i)
#pragma unroll
        for (int e = 0; e < kWide; ++e)
          if (x[i][e] > peak) {
            peak = x[i][e];
            place = first + i * kStep + e;
          }
    }
    if (proposal >= chunk && proposal < chunk + kChunk) {
#pragma unroll
      for (int i = 0; i < kLoads; ++i)
#pragma unroll
        for (int e = 0; e < kWide; ++e) x[i][e] = first + i * kStep + e == proposal ? -INFINITY : x[i][e];
    }
    if (sums) {
#pragma unroll
      for (int i = 0; i < kLoads; ++i)
#pragma unroll
        for (int e = 0; e < kWide; ++e) sum += plain_weight(x[i][e], scale);
    }
  }
  float top = scale.top;
  sum = wave_sum(sum);
  double proposed = proposal >= 0 ? weight_of(at(from, proposal), scale) : 0.0;
  if (sums && top > -INFINITY && !(scale.plain && sum + proposed < 0x1p1000)) {
    for (int i = begin + lane; i < end; i += 64) top = fmaxf(top, at(from, i));
    top = wave_max(top);
    scale = scale_of(top, heat.factor);
    sum = 0;
    for (int i = begin + lane; i < end; i += 64) sum += i == proposal ? 0.0 : weight_of(at(from, i), scale);
    sum = wave_sum(sum);
    if (proposal >= 0) proposed = weight_of(at(from, proposal), scale);
  }
  if (heat.greedy) {
    const float all = wave_max(peak);
    place = wave_min(peak == all ? place : INT32_MAX);
    peak = all;
  }
  if (lane == 0) {
    if (!p.draft) w.rest[cell] = sum;
    w.sum[cell] = sum + proposed;
    w.top[cell] = top;
    w.peak[cell] = peak;
    w.place[cell] = place;
  }
}

__global__ void verify_clear_kernel(VerifyParams p, int piece) {
  const Work w = work_of(p.workspace, p.n_tokens, p.n_queries, p.vocab, piece);
  const int u = blockIdx.x * kThreads + threadIdx.x;
  if (u < p.n_queries) w.done[static_cast<int64_t>(u) * kApart] = 0;
}

// Statistics of a whole row from its pieces, by the lanes of a group.
__device__ inline float group_max(float v) {
#pragma unroll
  for (int s = kGroup / 2; s > 0; s >>= 1) v = fmaxf(v, __shfl_xor(v, s));
  return v;
}
struct RowSum {
  Scale scale;
  double sum;
};
// first: the lane's first piece, asked for beforehand
struct Piece {
  float top;
  double sum;
};
__device__ inline Piece first_piece(const Work& w, int64_t which) {
  const int lane = threadIdx.x % kGroup;
  const int64_t cell = which * w.pieces + min(lane, w.pieces - 1);
  return {w.top[cell], w.sum[cell]};
}
__device__ inline RowSum row_sum(const Work& w, int64_t which, Piece first, double factor) {
  const int lane = threadIdx.x % kGroup;
  const int64_t base = which * w.pieces;
  float top = first.top;
  for (int i = lane + kGroup; i < w.pieces; i += kGroup) top = fmaxf(top, w.top[base + i]);
  const Scale scale = scale_of(group_max(top), factor);
  double sum = 0;
  for (int i = lane; i < w.pieces; i += kGroup) {
    if (i > lane) first = {w.top[base + i], w.sum[base + i]};
    if (first.sum > 0) sum += first.sum * rescale(scale_of(first.top, factor), scale);
  }
#pragma unroll
  for (int s = kGroup / 2; s > 0; s >>= 1) sum += __shfl_xor(sum, s);
  return {scale, sum};
}
// (an index into the row, whatever the pieces hold: those of rows that belong to no question, or to one of other bounds, are not written)
__device__ inline int row_place(const Work& w, int64_t which, int vocab) {
  const int lane = threadIdx.x % kGroup;
  const int64_t base = which * w.pieces;
  float peak = -INFINITY;
  int place = INT32_MAX;
  for (int i = lane; i < w.pieces; i += kGroup) {
    const float here = w.peak[base + i];
    if (here > peak) {
      peak = here;
      place = w.place[base + i];
    }
  }
  const float all = group_max(peak);
  place = peak == all ? place : INT32_MAX;
#pragma unroll
  for (int s = kGroup / 2; s > 0; s >>= 1) place = min(place, __shfl_xor(place, s));
  return place >= 0 && place < vocab ? place : -1;
}
__device__ inline double inverse(double sum) { return sum > 0 ? 1.0 / sum : 0.0; }

// Which proposals of question u stand, by a whole workgroup, eight rows at a time: every thread gets the decision.  `tells`: this
// workgroup writes the rows in front of the one that decides, and behind it.
template <typename T, bool kLogits>
__device__ Decision decide(const VerifyParams& p, const Work& w, int u, const Span& s, const Heat& heat, bool tells) {
  __shared__ unsigned falls_sh[kWaves];
  __shared__ Decision decision_sh;
  const int lane = threadIdx.x % (2 * kGroup), group = threadIdx.x / (2 * kGroup);
  const bool speaks = lane == 0, of_draft = lane >= kGroup;
  const bool sums = kLogits && (!heat.greedy || p.logp);
  const float number = p.uniform[s.end - 1];
  for (int first = s.begin;; first += kRows) {
    const int row = first + group;
    Decision d{};
    bool stands = false;
    int x = -1;
    float v = 0;
    if (row < s.end) {
      if (row + 1 < s.end) x = p.tokens[row + 1];
      const float number_of_row = p.uniform[row];
      Piece piece{};
      const int64_t which = row + (of_draft && p.draft ? static_cast<int64_t>(p.n_tokens) : 0);
      if (sums) piece = first_piece(w, which);
      const bool asks = proposes(p, s, row, x), drawn = asks && p.draft && !(kLogits && heat.greedy);
      const T* const from = of_draft && drawn ? draft_row<T>(p, u, row - s.begin) : target_row<T>(p, row);
      if (asks) v = at(from, x);
      d.row = row;
      d.step = row - s.begin;
      d.number = number;
      d.proposal = x;
      d.refused = asks ? p.draft ? 1 : 2 : 0;
      double mine;  // p(x), in the other half of the lanes q(x)
      if constexpr (kLogits) {
        mine = 0.0;
        if (heat.greedy) d.place = row_place(w, row, p.vocab);
        if (sums) {
          const RowSum sum = row_sum(w, which, piece, heat.factor);
          d.top_p = sum.scale.top;
          d.inv_p = inverse(sum.sum);
          mine = weight_of(v, sum.scale) * d.inv_p;
          if (p.logp) d.log_p = log_sum_of(sum.sum, sum.scale);
          d.top_q = __shfl_xor(d.top_p, kGroup);
          d.inv_q = __shfl_xor(d.inv_p, kGroup);
        }
      } else {
        mine = clean(v);
      }
      const double other = __shfl_xor(mine, kGroup), qx = drawn ? other : 1.0;
      stands = asks && static_cast<double>(number_of_row) * qx < mine;  // (counts in the lanes that speak)
      if (kLogits && heat.greedy) stands = asks && x == d.place;        // (whatever the number is)
    }
    const uint64_t mask = __ballot(!stands);
    if (threadIdx.x % 64 == 0) falls_sh[threadIdx.x / 64] = static_cast<unsigned>((mask & 1) | (mask >> 2 * kGroup & 1) << 1) << group;
    __syncthreads();
    unsigned falls = 0;
#pragma unroll
    for (int i = 0; i < kWaves; ++i) falls |= falls_sh[i];
    const int stop = falls ? __ffs(falls) - 1 : kRows;
    if (group == stop && speaks) {  // (field by field: copied as a whole it goes through scratch memory)
      decision_sh.row = d.row;
      decision_sh.step = d.step;
      decision_sh.refused = d.refused;
      decision_sh.proposal = d.proposal;
      decision_sh.number = d.number;
      if constexpr (kLogits) {
        decision_sh.place = d.place;
        decision_sh.top_p = d.top_p;
        decision_sh.top_q = d.top_q;
        decision_sh.log_p = d.log_p;
        decision_sh.inv_p = d.inv_p;
        decision_sh.inv_q = d.inv_q;
      }
    }
    if (tells && speaks && row < s.end && group != stop) {
      p.out[row] = group < stop ? x : -1;
      if (p.logp) p.logp[row] = group < stop ? static_cast<float>(log_of<kLogits>(v, d.top_p, d.log_p, heat.factor)) : 0.f;
    }
    __syncthreads();
    if (falls) break;
  }
  const Decision d = decision_sh;
  if (tells) {
    for (int row = s.begin + d.step / kRows * kRows + kRows + threadIdx.x; row < s.end; row += kThreads) {
      p.out[row] = -1;
      if (p.logp) p.logp[row] = 0.f;
    }
    if (threadIdx.x == 0) {
      p.accepted[u] = d.step;
      if (p.new_len) p.new_len[u] = p.self_len[u] - (s.end - 1 - d.row);
    }
  }
  return d;
}

// A question without rows.
__device__ inline void tell_nothing(const VerifyParams& p, int u) {
  if (threadIdx.x == 0) {
    p.accepted[u] = 0;
    if (p.new_len) p.new_len[u] = p.self_len[u];
  }
}
template <typename T, bool kLogits>
__device__ inline void tell_token(const VerifyParams& p, const Decision& d, int token, double factor) {
  p.out[d.row] = token;
  if (p.logp)
    p.logp[d.row] = token < 0 ? 0.f : static_cast<float>(log_of<kLogits>(at(target_row<T>(p, d.row), token), d.top_p, d.log_p, factor));
}

// One workgroup: question u, from logits.
template <typename T>
__global__ __launch_bounds__(kThreads) void verify_decide_kernel(VerifyParams p, int piece) {
  const Work w = work_of(p.workspace, p.n_tokens, p.n_queries, p.vocab, piece);
  const int u = blockIdx.x;
  const Span s = span_of(p, u);
  if (s.begin == s.end) {
    if (threadIdx.x == 0) w.decision[u].row = -1;
    tell_nothing(p, u);
    return;
  }
  const Heat heat = heat_of(p, u);
  Decision d = decide<T, true>(p, w, u, s, heat, true);
  if (threadIdx.x > 0) return;
  if (heat.greedy) {
    tell_token<T, true>(p, d, d.place, heat.factor);
    d.row = -1;
  }
  w.decision[u] = d;
}

// w of value i of the row that decides.  Both products are rounded, so that equal distributions leave exactly nothing.
template <bool kLogits>
__device__ inline double weight_at(const Decision& d, float x, float y, int i, const Scale& of_p, const Scale& of_q) {
#pragma clang fp contract(off)
  double a, b = 0.0;
  if constexpr (kLogits) a = weight_of(x, of_p) * d.inv_p;
  else a = clean(x);
  if (d.refused == 1) {
    if constexpr (kLogits) b = weight_of(y, of_q) * d.inv_q;
    else b = clean(y);
  }
  return d.refused == 2 && i == d.proposal ? 0.0 : fmax(a - b, 0.0);
}

// Exclusive prefix of v over the workgroup, and its total.
__device__ inline double scan(double v, double& total) {
  __shared__ double part[kWaves];
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
#pragma unroll
  for (int i = 0; i < kWaves; ++i) {
    if (i < wave) before += part[i];
    total += part[i];
  }
  return before + up - v;
}

// Sums go from workgroup to workgroup past the caches in between (stores and loads of the device's scope), and a workgroup is
// counted once its stores have been acknowledged: nothing else is handed over, so that the count needs no fence, which
// would write back a whole L2 for each workgroup (64 questions over 102400 words: 76 us instead of 34).
__device__ inline double left(const double* p) { return __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }
__device__ inline void leave(double* p, double v) { __hip_atomic_store(p, v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }
__device__ inline void wait_for_stores() { asm volatile("s_waitcnt vmcnt(0)" ::: "memory"); }

// Threads hold runs of items one after the other, of sums `mine` with `front` in front of them.  The thread in whose run the
// running sum passes `want`; where none does, the last that has any; 0 if none has.  (By ballots: an atomic of many lanes becomes a loop over
// them, 1.5 us each.)
__device__ inline int passing_thread(double mine, double front, double want) {
  __shared__ int found_sh[kWaves], last_sh[kWaves];
  const int lane = threadIdx.x % 64, wave = threadIdx.x / 64;
  const uint64_t any = __ballot(mine > 0), found = __ballot(mine > 0 && front + mine > want);
  if (lane == 0) {  // (nobody reads these of an earlier call any more: a barrier lies between)
    found_sh[wave] = found ? wave * 64 + __builtin_ctzll(found) : -1;
    last_sh[wave] = any ? wave * 64 + 63 - __builtin_clzll(any) : -1;
  }
  __syncthreads();
  int it = 0;
#pragma unroll
  for (int i = 0; i < kWaves; ++i) it = max(it, last_sh[i]);
#pragma unroll
  for (int i = kWaves - 1; i >= 0; --i) it = found_sh[i] >= 0 ? found_sh[i] : it;
  return it;
}

// The piece of the row that decides in which the running sum passes `number` of the whole, from the sums that the statistics left:
// where w is p (or p without the proposal) nothing has to be weighed for it.  -1 without weights.
struct Place {
  int piece;
  double before, want;  // running sum in front of it
};
__device__ inline Place place_of(const Work& w, Decision& d, const Scale& of_p) {
  __shared__ Place place_sh;
  const int tid = threadIdx.x, run = (w.pieces + kThreads - 1) / kThreads;
  const int64_t base = static_cast<int64_t>(d.row) * w.pieces;
  auto sum_of = [&](int i) {
    const double sum = (d.refused == 2 ? w.rest : w.sum)[base + i];
    return sum > 0 ? sum * rescale(scale_of(w.top[base + i], of_p.factor), of_p) * d.inv_p : 0.0;
  };
  for (;;) {
    double mine = 0, all;
#pragma unroll 1
    for (int i = tid * run; i < min(tid * run + run, w.pieces); ++i) mine += sum_of(i);
    const double front = scan(mine, all);
    if (!(all > 0)) {
      if (d.refused == 0) return {-1, 0.0, 0.0};
      d.refused = 0;  // the proposal has all there is
      continue;
    }
    const double want = static_cast<double>(d.number) * all;
    if (tid == passing_thread(mine, front, want)) {
      double before = front, in_front = front;
      int chosen = tid * run;
#pragma unroll 1
      for (int i = tid * run; i < min(tid * run + run, w.pieces); ++i) {
        const double here = run == 1 ? mine : sum_of(i);
        if (!(here > 0)) continue;
        chosen = i;
        in_front = before;
        before += here;
        if (before > want) break;
      }
      place_sh = {chosen, in_front, want};
    }
    __syncthreads();
    return place_sh;
  }
}

// One workgroup: shares part * each .. of the row that decides for question u, a wave a share at a time and the next one on its way;
// where the statistics have the sums already, one workgroup alone and the piece that the token lies in (a draw for each of 128 rows
// without proposals: 54 us with every row weighed, so 27, statistics included; this kernel 11 of it, a chain: the pieces summed up,
// weighed, the token's piece read).  Two kernels, the sums first and then the draws, were
// 24 us instead of 19 for probabilities of 64 questions over 102400 words (2.8 TB/s of the rows that decide, the launch and the draw
// included) and 25 instead of 16 for one question.
template <typename T, bool kLogits, bool kDecided>
__global__ __launch_bounds__(kThreads) void verify_draw_kernel(VerifyParams p, int piece, int parts, int each) {
  constexpr int kWide = 16 / sizeof(T), kStep = 64 * kWide, kLoads = kShare / kStep;
  constexpr float kNone = kLogits ? -INFINITY : 0.f;
  const Work w = work_of(p.workspace, p.n_tokens, p.n_queries, p.vocab, piece);
  // (workgroup i runs on the chip's part i % 8: the first parts, which have more to do, are not to lie on one of them)
  const int u = blockIdx.x / parts, part = (blockIdx.x + u) % parts, tid = threadIdx.x, lane = tid % 64, wave = tid / 64;
  __shared__ bool last_sh;
  __shared__ int chosen_sh;
  __shared__ double before_sh, weight_sh[kPieceLeast];
  const Heat heat = heat_of(p, u);
  Decision d;
  if constexpr (kDecided) {
    d = w.decision[u];
    if (d.row < 0 || (kLogits && d.refused != 1 && part > 0)) return;
  } else {
    const Span s = span_of(p, u);
    const bool greedy = kLogits && heat.greedy;
    if (greedy && part > 0) return;  // (nothing to weigh)
    if (s.begin == s.end) {
      if (part == 0) tell_nothing(p, u);
      return;
    }
    d = decide<T, kLogits>(p, w, u, s, heat, part == 0);
    if (kLogits && d.refused != 1 && part > 0) return;
    if (greedy) {
      if (tid == 0) tell_token<T, kLogits>(p, d, d.place, heat.factor);
      return;
    }
  }
  const T* const target = target_row<T>(p, d.row);
  const T* const draft = d.refused == 1 ? draft_row<T>(p, u, d.step) : nullptr;
  double* const sums = w.weight + static_cast<int64_t>(u) * w.shares;
  const Scale of_p = kLogits ? scale_of(d.top_p, heat.factor) : Scale{}, of_q = kLogits ? scale_of(d.top_q, heat.factor) : Scale{};
  int share_begin = part * each, share_end = min(share_begin + each, w.shares);
  // keep: the weights stay in LDS for the draw, those of a short piece, or of the share that the token lies in, which is gone through
  // once more when its sum is there (the same instructions: what runs for the first time waits for them)
  bool alone = false, keep = false;
  double base = 0, want = 0;
  if constexpr (kLogits) {
    if (d.refused != 1) {
      const Place place = place_of(w, d, of_p);
      if (place.piece < 0) {
        if (tid == 0) tell_token<T, kLogits>(p, d, -1, heat.factor);
        return;
      }
      base = place.before;
      want = place.want;
      share_begin = place.piece * (piece / kShare);
      share_end = min(share_begin + piece / kShare, w.shares);
      alone = true;
      keep = piece <= kPieceLeast;
      before_sh = base;
    }
  }
  const bool known = alone;  // `want` is
  for (;;) {
    int share = share_begin + wave;
    uintx4 of_target[kLoads], of_draft[kLoads];
    if (share < share_end) {
#pragma unroll
      for (int k = 0; k < kLoads; ++k) {
        of_target[k] = load_wide(target, share * kShare + k * kStep + lane * kWide, p.vocab);
        if (d.refused == 1) of_draft[k] = load_wide(draft, share * kShare + k * kStep + lane * kWide, p.vocab);
      }
    }
    while (share < share_end) {
      const int first = share * kShare + lane * kWide, next = share + kWaves;
      float x[kLoads][kWide], y[kLoads][kWide];
      if ((share + 1) * kShare <= p.vocab) {
#pragma unroll
        for (int k = 0; k < kLoads; ++k) {
          widen_all<T>(of_target[k], x[k]);
          widen_all<T>(of_draft[k], y[k]);
        }
      } else {
#pragma unroll
        for (int k = 0; k < kLoads; ++k) {
          values_of(of_target[k], target, first + k * kStep, p.vocab, kNone, x[k]);
          if (d.refused == 1) values_of(of_draft[k], draft, first + k * kStep, p.vocab, kNone, y[k]);
        }
      }
      if (next < share_end) {
#pragma unroll
        for (int k = 0; k < kLoads; ++k) {
          of_target[k] = load_wide(target, next * kShare + k * kStep + lane * kWide, p.vocab);
          if (d.refused == 1) of_draft[k] = load_wide(draft, next * kShare + k * kStep + lane * kWide, p.vocab);
        }
      }
      double sum = 0;
#pragma unroll
      for (int k = 0; k < kLoads; ++k)
#pragma unroll
        for (int e = 0; e < kWide; ++e) {
          const double here = weight_at<kLogits>(d, x[k][e], y[k][e], first + k * kStep + e, of_p, of_q);
          sum += here;
          if (keep) weight_sh[(share - share_begin) * kShare + k * kStep + lane * kWide + e] = here;
        }
      if (!keep) {
        sum = wave_sum(sum);
        if (lane == 0) leave(sums + share, sum);
      }
      share = next;
    }
    if (keep) break;
    wait_for_stores();
    __syncthreads();
    if (!alone) {
      if (tid == 0)
        last_sh = __hip_atomic_fetch_add(w.done + static_cast<int64_t>(u) * kApart, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == static_cast<unsigned>(parts - 1);
      __syncthreads();
      if (!last_sh) return;
      share_begin = 0;
      share_end = w.shares;
    }
    const int run = (share_end - share_begin + kThreads - 1) / kThreads, first = share_begin + tid * run, end = min(first + run, share_end);
    double mine = 0, all;
    for (int i = first; i < end; ++i) mine += left(sums + i);
    const double front = base + scan(mine, all);
    if (!known) {
      if (!(all > 0)) {
        if (d.refused == 0) {
          if (tid == 0) tell_token<T, kLogits>(p, d, -1, heat.factor);
          return;
        }
        d.refused = 0;  // the target lies nowhere above what proposed: this workgroup goes through all of the target
        alone = true;
        continue;
      }
      want = static_cast<double>(d.number) * all;
    }
    if (tid == passing_thread(mine, front, want)) {
      double before = front, in_front = front;
      int chosen = first;
      for (int i = first; i < end; ++i) {
        const double here = run == 1 ? mine : left(sums + i);
        if (!(here > 0)) continue;
        chosen = i;
        in_front = before;
        before += here;
        if (before > want) break;
      }
      chosen_sh = chosen;
      before_sh = in_front;
    }
    __syncthreads();
    share_begin = chosen_sh;
    share_end = share_begin + 1;
    keep = true;
  }
  __syncthreads();
  const int run = (share_end - share_begin) * (kShare / kThreads);
  double mine = 0, all;
#pragma unroll 2
  for (int e = 0; e < run; ++e) mine += weight_sh[tid * run + e];
  const double front = before_sh + scan(mine, all);
  if (tid != passing_thread(mine, front, want)) return;
  double before = front;
  int token = -1;
#pragma unroll 1
  for (int e = 0; e < run; ++e) {
    const double here = weight_sh[tid * run + e];
    if (!(here > 0)) continue;
    token = share_begin * kShare + tid * run + e;
    before += here;
    if (before > want) break;
  }
  tell_token<T, kLogits>(p, d, token, heat.factor);
}

template <typename T, bool kLogits>
void launch(const VerifyParams& p, hipStream_t stream) {
  const int64_t rows = (p.draft ? 2 : 1) * static_cast<int64_t>(p.n_tokens);
  // A wave's piece: short ones fill the chip, long ones pay less often for the search, the scale and the reductions.  Calls with pieces
  // of 2048 and of 8192, in bf16: 16 x 8 looked up over 50257 words (2^22.6 values) 19.4 and 26.7 us, 128 rows of 128256 (2^24) 26.6 and
  // 30.7, 256 (2^25) 39.7 and 40.2, 512 (2^26) 67.0 and 59.4; with proposals' logits 32 x 4 (2^25) 51.2 and 45.7, 48 x 4 68.0 and 58.8,
  // 128 x 4 (2^27) 133 and 119; fp32 84 and 79 for 64 x 4, 157 and 145 for 128 x 4.
  const int piece = rows * p.vocab >= int64_t{1} << 25 ? 4 * kPieceLeast : kPieceLeast;
  const Work w = work_of(p.workspace, p.n_tokens, p.n_queries, p.vocab, piece);
  const dim3 threads(kThreads);
  // workgroups that fill the chip (logits: half as many 123 us instead of 114 for 128 x 4 in bf16; probabilities of 128 questions in
  // fp32 37 us, twice as many 41, four times 39)
  constexpr int64_t kFull = kLogits ? 2048 : 1024;
  // shares of a workgroup, a multiple of its waves; nothing is weighed by more than one where no distribution is taken off
  const int64_t most = pieces_of(w.shares, kWaves), per = kLogits && !p.draft ? most : (p.n_queries * most + kFull - 1) / kFull;
  const int each = static_cast<int>(per * kWaves), parts = static_cast<int>(pieces_of(w.shares, each));
  const dim3 grid(static_cast<unsigned>(p.n_queries) * parts);
  if (kLogits && rows > 0) {
    const int64_t cells = rows * w.pieces;
    verify_stats_kernel<T><<<dim3(static_cast<unsigned>((cells + kWaves - 1) / kWaves)), threads, 0, stream>>>(p, piece);
  } else {
    verify_clear_kernel<<<dim3((p.n_queries + kThreads - 1) / kThreads), threads, 0, stream>>>(p, piece);
  }
  if constexpr (kLogits) {
    // Each workgroup of a question decides for itself, which takes 3 us, while they all run at once; for more of them one does, 6.5 us
    // before the others begin: 128 x 4 in bf16 114 us against 119, 128 x 3 over 20000 words (1280 workgroups) 36 against 35.  (From
    // probabilities it takes less: never apart, 45 against 43 and 25 against 24 us.)
    if (static_cast<int64_t>(p.n_queries) * parts > 1536) {
      verify_decide_kernel<T><<<dim3(p.n_queries), threads, 0, stream>>>(p, piece);
      verify_draw_kernel<T, true, true><<<grid, threads, 0, stream>>>(p, piece, parts, each);
      return;
    }
  }
  verify_draw_kernel<T, kLogits, false><<<grid, threads, 0, stream>>>(p, piece, parts, each);
}

}  // namespace

size_t verify_workspace_bytes(int64_t n_tokens, int64_t n_queries, int64_t vocab) {
  const Work w = work_of(nullptr, n_tokens, n_queries, vocab, kPieceLeast);
  const size_t all = reinterpret_cast<size_t>(w.done) + static_cast<size_t>(n_queries) * kApart * 4;
  return (all + 15) / 16 * 16;
}

hipError_t launch_verify(const VerifyParams& p, bool bf16, bool logits, hipStream_t stream) {
  if (bf16) logits ? launch<__bf16, true>(p, stream) : launch<__bf16, false>(p, stream);
  else logits ? launch<float, true>(p, stream) : launch<float, false>(p, stream);
  return hipGetLastError();
}
