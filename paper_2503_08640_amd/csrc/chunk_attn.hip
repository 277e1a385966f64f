// Chunk attention (stage 2 for several new tokens per question, Sec. 2.2) on gfx950: every new token attends the sink, its
// question's selected groups and its own keys up to itself, the own keys lying in pages.
//
// Mathematics.  One softmax per row (a new token times a query head) over all its keys, taken in one pass over tiles of
// keys: with m the running maximum of the scores and l the running sum of 2^(s - m),
//     m' = max(m, max s),  l' = l 2^(m - m') + sum 2^(s - m'),  acc' = acc 2^(m - m') + sum 2^(s - m') v,   o = acc / l.
// m, l and acc are held in fp32.  acc and l are only rescaled when a row's maximum has grown by more than kSlack: until then
// the probabilities stay below 2^kSlack, far inside fp32 and bf16.  Scores are transposed, S^T = K Q^T, so that a lane
// holds 16 keys of ONE row per block of 32 keys: maxima and sums need one exchange between the two half-waves and no LDS,
// and the probabilities are in place as the operand of O^T = V^T P^T.  bf16 products (8-bit caches are widened as they are
// staged, exactly: every e4m3 value is a bf16 value), fp32 products for fp32 tensors; the only rounding to fewer bits besides
// the output's is that of the probabilities to bf16, relative 2^-9 each and unbiased, while l sums them unrounded.
//
// Work.  Workers and their records come from the host's plan (chunk_plan.cpp).  A record is a block of rows and a run of
// 64-key tiles: pool tiles from the lists, then a part of the question's own keys, whose number the device knows
// (self_len).  It leaves finished rows, or partial softmax states that the merge kernel joins.
#include <atomic>
#include <cstdint>

#include "kernels.hpp"
#include "layout.hpp"
#include "mfma_common.hpp"

namespace {
using namespace dbsa_mfma;

constexpr float kSlack = 8.f;  // log2 units a row's scores may exceed its running maximum by before acc is rescaled

struct E4m3 {};  // storage of 8-bit caches; q and o are bf16 then

template <typename T>
struct Kind;
template <>
struct Kind<__bf16> {
  typedef __bf16 Q;     // elements of q, o and of the staged tiles
  static constexpr int kStoredBytes = 2, kBytes = 2;
};
template <>
struct Kind<E4m3> {
  typedef __bf16 Q;
  static constexpr int kStoredBytes = 1, kBytes = 2;
};
template <>
struct Kind<float> {
  typedef float Q;
  static constexpr int kStoredBytes = 4, kBytes = 4;
};

typedef unsigned uintx4 __attribute__((ext_vector_type(4)));

// sixteen e4m3 bytes as bf16
__device__ DBSA_INLINE void widen16(const uintx4& raw, uintx4& lo, uintx4& hi) {
  union {
    bf16x2 p2[8];
    uintx4 v[2];
  } out;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    out.p2[2 * i] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(raw[i], 1.f, false);
    out.p2[2 * i + 1] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(raw[i], 1.f, true);
  }
  lo = out.v[0];
  hi = out.v[1];
}

// whether any of a piece's elements is not finite (e4m3: NaN, the format has no infinities)
template <typename T>
__device__ DBSA_INLINE bool not_finite(const uintx4& x) {
  bool bad = false;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if constexpr (Kind<T>::kStoredBytes == 1) {
      const unsigned off = (x[i] & 0x7F7F7F7Fu) ^ 0x7F7F7F7Fu;  // a zero byte where the magnitude is 0x7F
      bad |= ((off - 0x01010101u) & ~off & 0x80808080u) != 0;
    } else if constexpr (Kind<T>::kStoredBytes == 2) {
      bad |= (x[i] & 0x7F80u) == 0x7F80u || (x[i] & 0x7F800000u) == 0x7F800000u;
    } else {
      bad |= (x[i] & 0x7F800000u) == 0x7F800000u;
    }
  }
  return bad;
}

// channel ch of a stored row
template <typename T>
__device__ DBSA_INLINE float stored_value(const unsigned char* row, int ch) {
  if constexpr (Kind<T>::kStoredBytes == 1) return __builtin_amdgcn_cvt_f32_fp8(row[ch], 0);
  else if constexpr (Kind<T>::kStoredBytes == 2) return static_cast<float>(reinterpret_cast<const __bf16*>(row)[ch]);
  else return reinterpret_cast<const float*>(row)[ch];
}

// kBN keys per step (a 64-key tile is one or two steps), kNW waves of kRB blocks of 32 rows.
template <typename T, int kD, int kNW, int kRB, int kBN>
struct Chunk {
  typedef typename Kind<T>::Q Q;
  static constexpr int kThreads = 64 * kNW, kRows = 32 * kRB * kNW;
  static constexpr int kRowBytes = kD * Kind<T>::kBytes, kTileBytes = kBN * kRowBytes;  // as staged
  static constexpr int kSlots = kRowBytes / 16;                                         // 16-byte places of a staged row
  static constexpr int kPieces = kD * Kind<T>::kStoredBytes / 16;                       // 16-byte pieces of a stored row
  static constexpr int kOperand = kBN * kPieces;                                        // pieces of K, and of V, of a step
  static constexpr int kLoads = 2 * kOperand / kThreads;                                // pieces per thread
  static constexpr bool kApart = kOperand < kThreads;                                   // half the waves fetch K, half V
  static constexpr int kKeyBlocks = kBN / 32, kChBlocks = kD / 32;
  static constexpr int kStages = 2;
  static constexpr int kLds = kStages * (2 * kTileBytes + kNW * 8);  // tiles, and each wave's mask of poisoned rows
  static_assert(kPieces <= 32 && 64 % kPieces == 0, "a stored row is fetched by neighbouring lanes of one wave");
  static_assert(kApart ? kOperand * 2 == kThreads : kOperand % kThreads == 0, "whole pieces per thread");
  // K places: xor by row, so that the 16 rows a quarter wave reads of one column lie on different banks; V rows of 16-bit
  // elements are read transposed, four rows at a time (as in attn_prefill64.hip), V rows of fp32 element by element, the two
  // half-waves four rows apart.
  __device__ static DBSA_INLINE int k_swizzle(int row) { return kSlots >= 16 ? row % 16 : (row / 2) % 8; }
  __device__ static DBSA_INLINE int v_swizzle(int row) {
    if (Kind<T>::kBytes == 4) return 8 * ((row / 4) % 2);
    return kSlots >= 16 ? 4 * (row % 4) : 4 * ((row / 2) % 2);
  }
};

template <typename T, int kD, int kNW, int kRB, int kBN>
__global__ __launch_bounds__(64 * kNW, 2) void chunk_attn_kernel(ChunkParams p) {
  typedef Chunk<T, kD, kNW, kRB, kBN> C;
  typedef typename C::Q Q;
  constexpr bool kF32 = Kind<T>::kBytes == 4;
  constexpr int kB = C::kKeyBlocks, kO = C::kChBlocks;
  extern __shared__ __attribute__((aligned(1024))) unsigned char smem[];

  const int tid = threadIdx.x, lane = tid % 64, l32 = lane % 32, half = lane / 32;
  const int wave = __builtin_amdgcn_readfirstlane(tid / 64);
  const int hk = static_cast<int>(blockIdx.x) % p.n_kv_heads, worker = static_cast<int>(blockIdx.x) / p.n_kv_heads;
  const int r = p.n_q_heads / p.n_kv_heads;
  // scores in log2 units: scale * log2 e (and the keys' scale) goes onto them in fp32.  A negative key scale turns the
  // rows of Q around; a scale of nothing stays above zero, so that a masked -inf stays one.
  float c2 = p.scale_log2e;
  if (p.k_scale) c2 *= p.k_scale[hk];
  const bool negate = c2 < 0.f;
  c2 = fmaxf(fabsf(c2), 1e-30f);
  const float v_scale = p.v_scale ? p.v_scale[hk] : 1.f;

  const unsigned char* const kpool = static_cast<const unsigned char*>(p.k_pool.ptr) + hk * p.k_pool.stride_head * Kind<T>::kStoredBytes;
  const unsigned char* const vpool = static_cast<const unsigned char*>(p.v_pool.ptr) + hk * p.v_pool.stride_head * Kind<T>::kStoredBytes;
  const unsigned char* const kown = static_cast<const unsigned char*>(p.k_own.ptr) + hk * p.k_own.stride_head * Kind<T>::kStoredBytes;
  const unsigned char* const vown = static_cast<const unsigned char*>(p.v_own.ptr) + hk * p.v_own.stride_head * Kind<T>::kStoredBytes;

  const int64_t kpool_stride = p.k_pool.stride_tok * Kind<T>::kStoredBytes, vpool_stride = p.v_pool.stride_tok * Kind<T>::kStoredBytes;
  // this thread's first piece of a whole step
  const int64_t k_lane = (tid % C::kOperand / C::kPieces) * kpool_stride + (tid % C::kPieces) * 16;
  const int64_t v_lane = (tid % C::kOperand / C::kPieces) * vpool_stride + (tid % C::kPieces) * 16;

  int stage = 0;
  const int rec_end = p.ptr[worker + 1];
  for (int rec = p.ptr[worker]; rec < rec_end; ++rec) {
    const int32_t* const w = p.rec + rec * kChunkWords;
    const int tok_begin = w[0], n_tok = w[1], ent_begin = w[2], n_ent = w[3], own_u = w[4], part_base = w[8];
    const int cu = w[9], t_new = w[10];

    // ---- rows ----
    int row_tok[kRB], row_head[kRB], row_pos[kRB];
    bool row_ok[kRB];
    int own_n = 0;  // own keys there are
    if (own_u >= 0) own_n = min(max(p.self_len[own_u], 0), p.own_capacity);
#pragma unroll
    for (int rb = 0; rb < kRB; ++rb) {
      const int i = (wave * kRB + rb) * 32 + l32;
      const int t = i / r;
      row_ok[rb] = t < n_tok;
      row_tok[rb] = min(t, n_tok - 1);
      row_head[rb] = hk * r + i % r;
    }
    typedef typename std::conditional<kF32, floatx4, bf16x8>::type Piece;
    Piece qf[kRB][C::kSlots / 2];
#pragma unroll
    for (int rb = 0; rb < kRB; ++rb) {
      const int tok = p.toks[tok_begin + row_tok[rb]];
      row_pos[rb] = own_n - t_new + (tok - cu);  // the row's own index: it sees own keys 0 .. row_pos
      const Q* const qp = static_cast<const Q*>(p.q.ptr) + tok * p.q.stride_tok + row_head[rb] * p.q.stride_head;
#pragma unroll
      for (int c = 0; c < C::kSlots / 2; ++c) {
        qf[rb][c] = *reinterpret_cast<const Piece*>(qp + (2 * c + half) * (16 / static_cast<int>(sizeof(Q))));
        if (negate) qf[rb][c] = -qf[rb][c];
      }
    }
    // own tiles of this record: its share of those up to the last token's own key
    int own_first = 0, own_steps = 0;
    if (own_u >= 0) {
      const int last = own_n - t_new + (p.toks[tok_begin + n_tok - 1] - cu);
      const int64_t tiles = max(0, (last + kChunkTile) / kChunkTile);
      const int lo = static_cast<int>(w[5] * tiles / w[7]), hi = static_cast<int>(w[6] * tiles / w[7]);
      own_first = lo * kChunkTile;
      own_steps = (hi - lo) * (kChunkTile / kBN);
    }
    const int first_pos = own_n - t_new + (p.toks[tok_begin] - cu);  // (tokens of a question ascend)
    const int pool_steps = n_ent * (kChunkTile / kBN), steps = pool_steps + own_steps;

    // ---- the stream of steps ----
    // raw: what a step hangs off (its list entry, or the page of this lane's key), requested two steps ahead
    struct Ahead {
      int start, len, page;
    };
    auto fetch = [&](int s) DBSA_INLINE {
      Ahead x{0, 0, -1};
      if (s < pool_steps) {
        const int32_t* const e = p.ent + 2 * static_cast<int64_t>(ent_begin + s / (kChunkTile / kBN));
        x.start = e[0];
        x.len = e[1];
      } else if (s < steps) {
        const int j = own_first + (s - pool_steps) * kBN + lane;
        if (lane < kBN && j < own_n) x.page = p.page_table[static_cast<int64_t>(own_u) * p.table_stride + (j >> p.page_log2)];
      }
      return x;
    };
    // a step's keys: row of this lane's key in the pool or in the pages (-1: nothing there), and what the rows see of them
    struct Keys {
      int row;
      bool own, whole;  // whole: every row sees all kBN keys
      int first, len;   // pool: keys; own: index of the first key
    };
    auto place = [&](int s, const Ahead& x) DBSA_INLINE {
      Keys k;
      k.own = s >= pool_steps;
      if (!k.own) {
        const int off = (s % (kChunkTile / kBN)) * kBN;
        k.len = min((x.len & 0xFFFF) - off, kBN);
        k.first = 0;
        k.row = k.len > 0 ? x.start + off + min(lane, k.len - 1) : -1;
        k.whole = k.len == kBN;
      } else {
        k.first = own_first + (s - pool_steps) * kBN;
        k.len = kBN;
        const int j = k.first + lane;
        k.row = x.page >= 0 && x.page < p.n_pages ? (x.page << p.page_log2) + (j & ((1 << p.page_log2) - 1)) : -1;
        k.whole = k.first + kBN - 1 <= first_pos && __builtin_amdgcn_ballot_w64(lane < kBN && k.row < 0) == 0;
      }
      return k;
    };
    // This thread's pieces of a step: piece tid + i threads of K, then of V; the operand of piece i is the wave's.
    uintx4 raw[C::kLoads];
    auto is_v = [&](int i) DBSA_INLINE { return C::kApart ? wave >= kNW / 2 : i >= C::kLoads / 2; };
    auto piece_row = [&](int i) DBSA_INLINE { return (tid + i * C::kThreads) % C::kOperand / C::kPieces; };
    auto load = [&](const Keys& k) DBSA_INLINE {
      if (!k.own && k.whole) {
        const int64_t first = __builtin_amdgcn_readfirstlane(k.row);
#pragma unroll
        for (int i = 0; i < C::kLoads; ++i) {
          const unsigned char* const base = is_v(i) ? vpool : kpool;
          const int64_t stride = is_v(i) ? vpool_stride : kpool_stride;
          const int row0 = i * C::kThreads % C::kOperand / C::kPieces;  // (whole rows per pass of the threads)
          raw[i] = *reinterpret_cast<const uintx4*>(base + (first + row0) * stride + (is_v(i) ? v_lane : k_lane));
        }
        return;
      }
      const int shift = k.own ? p.page_log2 : 31;
#pragma unroll
      for (int i = 0; i < C::kLoads; ++i) {
        const unsigned char* const base = k.own ? (is_v(i) ? vown : kown) : (is_v(i) ? vpool : kpool);
        const int64_t stride = k.own ? (is_v(i) ? p.v_own.stride_tok : p.k_own.stride_tok) * Kind<T>::kStoredBytes
                                     : (is_v(i) ? vpool_stride : kpool_stride);
        const int row = __shfl(k.row, piece_row(i));
        raw[i] = uintx4{0, 0, 0, 0};
        if (row >= 0) {
          const int64_t page = row >> shift, in = row - (page << shift);
          raw[i] = *reinterpret_cast<const uintx4*>(base + page * p.stride_page * Kind<T>::kStoredBytes + in * stride + (tid % C::kPieces) * 16);
        }
      }
    };
    // Where some rows do not see every key (the chunk's own diagonal), a non-finite value must not reach the others through
    // 0 * NaN: such rows of V are staged as zeros, and their keys added one by one to the rows that see them.
    uint64_t* const poison = reinterpret_cast<uint64_t*>(smem + C::kStages * 2 * C::kTileBytes);
    auto take_poison = [&](int st) DBSA_INLINE {
      uint64_t mask = 0;
      constexpr uint64_t kRowLanes = (1ull << C::kPieces) - 1;
#pragma unroll
      for (int i = 0; i < C::kLoads; ++i) {
        if (!is_v(i)) continue;
        const uint64_t bad = __builtin_amdgcn_ballot_w64(not_finite<T>(raw[i]));
        if (bad == 0) continue;
        const int row0 = (64 * wave + i * C::kThreads) % C::kOperand / C::kPieces;
        for (int rr = 0; rr < 64 / C::kPieces; ++rr)
          if ((bad >> (rr * C::kPieces)) & kRowLanes) mask |= 1ull << (row0 + rr);
        if ((bad >> (lane / C::kPieces * C::kPieces)) & kRowLanes) raw[i] = uintx4{0, 0, 0, 0};
      }
      if (lane == 0) poison[st * kNW + wave] = mask;
    };
    auto store = [&](int st) DBSA_INLINE {
#pragma unroll
      for (int i = 0; i < C::kLoads; ++i) {
        const int row = piece_row(i), col = tid % C::kPieces;
        unsigned char* const at = smem + (2 * st + (is_v(i) ? 1 : 0)) * C::kTileBytes + row * C::kRowBytes;
        const int swizzle = is_v(i) ? C::v_swizzle(row) : C::k_swizzle(row);
        if constexpr (Kind<T>::kStoredBytes == 1) {
          uintx4 lo, hi;
          widen16(raw[i], lo, hi);
          *reinterpret_cast<uintx4*>(at + ((2 * col) ^ swizzle) * 16) = lo;
          *reinterpret_cast<uintx4*>(at + ((2 * col + 1) ^ swizzle) * 16) = hi;
        } else {
          *reinterpret_cast<uintx4*>(at + (col ^ swizzle) * 16) = raw[i];
        }
      }
    };

    // ---- softmax state ----
    floatx16 acc[kRB][kO];
    float m[kRB], l[kRB];  // l: this lane's keys' share
#pragma unroll
    for (int rb = 0; rb < kRB; ++rb) {
      m[rb] = -INFINITY;
      l[rb] = 0.f;
#pragma unroll
      for (int ob = 0; ob < kO; ++ob)
#pragma unroll
        for (int i = 0; i < 16; ++i) acc[rb][ob][i] = 0.f;
    }

    // the keys that take_poison kept out of the product
    auto add_poison = [&](const Keys& k, int st, floatx16 (&s)[kRB][kB]) DBSA_INLINE {
      uint64_t mask = 0;
#pragma unroll
      for (int i = 0; i < kNW; ++i) mask |= poison[st * kNW + i];
      mask = uniform64(mask);
      while (mask) {
        const int key = __builtin_ctzll(mask);
        mask &= mask - 1;
        const int row = __shfl(k.row, key);
        const unsigned char* const v = vown + (row >> p.page_log2) * p.stride_page * Kind<T>::kStoredBytes +
                                       (row & ((1 << p.page_log2) - 1)) * p.v_own.stride_tok * Kind<T>::kStoredBytes;
#pragma unroll
        for (int rb = 0; rb < kRB; ++rb) {
          float mine = 0.f;  // the key's probability, in the half-wave that holds the key
#pragma unroll
          for (int kb = 0; kb < kB; ++kb)
#pragma unroll
            for (int i = 0; i < 16; ++i)
              if (key == 32 * kb + 8 * (i / 4) + 4 * half + i % 4) mine = s[rb][kb][i];
          const float other = __shfl_xor(mine, 32);
          const float prob = (key / 4) % 2 == half ? mine : other;
#pragma unroll
          for (int ob = 0; ob < kO; ++ob)
#pragma unroll
            for (int i = 0; i < 16; ++i) {
              const float x = stored_value<T>(v, 32 * ob + 8 * (i / 4) + 4 * half + i % 4);
              if (prob != 0.f) acc[rb][ob][i] = fmaf(prob, x, acc[rb][ob][i]);
            }
        }
      }
    };

    auto compute = [&](const Keys& k, int st) DBSA_INLINE {
      const unsigned char* const kt = smem + st * 2 * C::kTileBytes;
      const unsigned char* const vt = kt + C::kTileBytes;
      floatx16 s[kRB][kB];
#pragma unroll
      for (int rb = 0; rb < kRB; ++rb)
#pragma unroll
        for (int kb = 0; kb < kB; ++kb)
#pragma unroll
          for (int i = 0; i < 16; ++i) s[rb][kb][i] = 0.f;
      // scores: K fragment (kb, c) is row 32 kb + l32, place 2 c + half
#pragma unroll
      for (int kb = 0; kb < kB; ++kb) {
        const int row = 32 * kb + l32;
#pragma unroll
        for (int c = 0; c < C::kSlots / 2; ++c) {
          const unsigned char* const at = kt + row * C::kRowBytes + (((2 * c + half) ^ C::k_swizzle(row)) * 16);
          if constexpr (kF32) {
            const floatx4 kf = *reinterpret_cast<const floatx4*>(at);
#pragma unroll
            for (int e = 0; e < 4; ++e)
#pragma unroll
              for (int rb = 0; rb < kRB; ++rb) s[rb][kb] = __builtin_amdgcn_mfma_f32_32x32x2f32(kf[e], qf[rb][c][e], s[rb][kb], 0, 0, 0);
          } else {
            const bf16x8 kf = *reinterpret_cast<const bf16x8*>(at);
#pragma unroll
            for (int rb = 0; rb < kRB; ++rb) s[rb][kb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf, qf[rb][c], s[rb][kb], 0, 0, 0);
          }
        }
      }
      // masks: element i of block kb is key 32 kb + 8 (i / 4) + 4 half + i % 4 of the step
      if (!k.whole) {
        const uint64_t there = k.own ? __builtin_amdgcn_ballot_w64(k.row >= 0) : ~0ull;
#pragma unroll
        for (int rb = 0; rb < kRB; ++rb) {
          const int last = k.own ? row_pos[rb] - k.first : k.len - 1;
#pragma unroll
          for (int kb = 0; kb < kB; ++kb)
#pragma unroll
            for (int i = 0; i < 16; ++i) {
              const int key = 32 * kb + 8 * (i / 4) + 4 * half + i % 4;
              if (key > last || !((there >> key) & 1)) s[rb][kb][i] = -INFINITY;
            }
        }
      }
#pragma unroll
      for (int rb = 0; rb < kRB; ++rb) {
        float top = s[rb][0][0];
#pragma unroll
        for (int kb = 0; kb < kB; ++kb)
#pragma unroll
          for (int i = 0; i < 16; ++i) top = fmaxf(top, s[rb][kb][i]);
        top = half_swap_max(top) * c2;
        if (__builtin_amdgcn_ballot_w64(top > m[rb] + kSlack) != 0) {
          const float next = fmaxf(m[rb], top);
          const float alpha = m[rb] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m[rb] - next);
          m[rb] = next;
          l[rb] *= alpha;
#pragma unroll
          for (int ob = 0; ob < kO; ++ob)
#pragma unroll
            for (int i = 0; i < 16; ++i) acc[rb][ob][i] *= alpha;
        }
        const float less = m[rb] == -INFINITY ? 0.f : -m[rb];
        float sum = 0.f;
#pragma unroll
        for (int kb = 0; kb < kB; ++kb)
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            s[rb][kb][i] = __builtin_amdgcn_exp2f(fmaf(s[rb][kb][i], c2, less));
            sum += s[rb][kb][i];
          }
        l[rb] += sum;
      }
      // output
      if (k.own && !k.whole) add_poison(k, st, s);
      if constexpr (kF32) {
#pragma unroll
        for (int kb = 0; kb < kB; ++kb)
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            const int row = 32 * kb + 8 * (i / 4) + 4 * half + i % 4;
#pragma unroll
            for (int ob = 0; ob < kO; ++ob) {
              const int ch = 32 * ob + l32;
              const float vf = *reinterpret_cast<const float*>(vt + row * C::kRowBytes + (((ch / 4) ^ C::v_swizzle(row)) * 16) + (ch % 4) * 4);
#pragma unroll
              for (int rb = 0; rb < kRB; ++rb) acc[rb][ob] = __builtin_amdgcn_mfma_f32_32x32x2f32(vf, s[rb][kb][i], acc[rb][ob], 0, 0, 0);
            }
          }
      } else {
        // V fragment (kb, ch, ob): keys 32 kb + 16 ch + 4 half + {0..3, 8..11}, the order the probabilities lie in; read transposed:
        // lane j of 16 fetches four channels of one key and gets four keys of one channel
        const int j = (lane % 16) / 4;
        const unsigned char* const vbase = vt + (4 * half + j) * C::kRowBytes + (lane % 2) * 8;
        const int slot0 = (2 * (l32 / 16) + (lane % 4) / 2) ^ C::v_swizzle(j);
#pragma unroll
        for (int kb = 0; kb < kB; ++kb)
#pragma unroll
          for (int ch = 0; ch < 2; ++ch) {
            bf16x8 pf[kRB];
#pragma unroll
            for (int rb = 0; rb < kRB; ++rb) {
              union {
                bf16x8 v;
                bf16x2 p2[4];
              } x;
#pragma unroll
              for (int e = 0; e < 4; ++e)
                x.p2[e] = __builtin_convertvector(floatx2{s[rb][kb][8 * ch + 2 * e], s[rb][kb][8 * ch + 2 * e + 1]}, bf16x2);
              pf[rb] = x.v;
            }
#pragma unroll
            for (int ob = 0; ob < kO; ++ob) {
              const unsigned char* const at = vbase + (32 * kb + 16 * ch) * C::kRowBytes + ((slot0 ^ (4 * ob)) * 16);
              const bf16x4 lo = lds_read_tr(reinterpret_cast<const __bf16*>(at));
              const bf16x4 hi = lds_read_tr(reinterpret_cast<const __bf16*>(at + 8 * C::kRowBytes));
              const bf16x8 vf = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
#pragma unroll
              for (int rb = 0; rb < kRB; ++rb) acc[rb][ob] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf, pf[rb], acc[rb][ob], 0, 0, 0);
            }
          }
      }
    };

    Ahead next{};
    Keys cur{}, ahead{};
    if (steps > 0) {
      ahead = place(0, fetch(0));
      load(ahead);
      next = fetch(1);
    }
    for (int s = 0; s < steps; ++s) {
      cur = ahead;
      if (cur.own && !cur.whole) take_poison(stage);
      store(stage);
      if (s + 1 < steps) {
        ahead = place(s + 1, next);
        load(ahead);
        next = fetch(s + 2);
      }
      // one barrier per step: the other stage was last read before the barrier of the step that filled this one
      __syncthreads();
      compute(cur, stage);
      stage ^= 1;
    }

    // ---- what the record leaves ----
#pragma unroll
    for (int rb = 0; rb < kRB; ++rb) {
      const float sum = half_swap_sum(l[rb]);
      if (!row_ok[rb]) continue;
      if (part_base >= 0) {
        float* const out = p.partial + (static_cast<int64_t>(part_base + row_tok[rb]) * p.n_q_heads + row_head[rb]) * (kD + kPartialPad);
#pragma unroll
        for (int ob = 0; ob < kO; ++ob)
#pragma unroll
          for (int g = 0; g < 4; ++g) {
            const floatx4 x = {acc[rb][ob][4 * g], acc[rb][ob][4 * g + 1], acc[rb][ob][4 * g + 2], acc[rb][ob][4 * g + 3]};
            *reinterpret_cast<floatx4*>(out + 32 * ob + 8 * g + 4 * half) = x;
          }
        if (half == 0) *reinterpret_cast<floatx2*>(out + kD) = floatx2{m[rb], sum};
      } else {
        const int tok = p.toks[tok_begin + row_tok[rb]];
        // (a row that saw no key is zero)
        const float inv = sum > 0.f || sum != sum ? v_scale / sum : 0.f;
        Q* const out = static_cast<Q*>(const_cast<void*>(p.o.ptr)) + tok * p.o.stride_tok + row_head[rb] * p.o.stride_head;
#pragma unroll
        for (int ob = 0; ob < kO; ++ob)
#pragma unroll
          for (int g = 0; g < 4; ++g) {
            typedef Q four __attribute__((ext_vector_type(4)));
            *reinterpret_cast<four*>(out + 32 * ob + 8 * g + 4 * half) =
                four{static_cast<Q>(acc[rb][ob][4 * g] * inv), static_cast<Q>(acc[rb][ob][4 * g + 1] * inv),
                     static_cast<Q>(acc[rb][ob][4 * g + 2] * inv), static_cast<Q>(acc[rb][ob][4 * g + 3] * inv)};
          }
        if (p.lse && half == 0)
          p.lse[static_cast<int64_t>(row_head[rb]) * p.n_rows + tok] = (m[rb] + __builtin_amdgcn_logf(sum)) * 0.6931471805599453f;
      }
    }
  }
}

// Joins the partial states of one (token, query head): m* = max m_s, o = sum acc_s 2^(m_s - m*) / sum l_s 2^(m_s - m*).  One wave
// each, kD / 64 channels per lane; maxima and sums are read with one state per lane.
template <typename Q, int kD>
__global__ __launch_bounds__(256) void chunk_merge_kernel(ChunkParams p) {
  constexpr int kRow = kD + kPartialPad, kPer = kD / 64;
  const int lane = threadIdx.x % 64;
  const int64_t pair = static_cast<int64_t>(blockIdx.x) * 4 + threadIdx.x / 64;
  if (pair >= static_cast<int64_t>(p.n_rows) * p.n_q_heads) return;
  const int tok = static_cast<int>(pair / p.n_q_heads), head = static_cast<int>(pair % p.n_q_heads);
  const int lo = p.tok_ptr[tok], n = p.tok_ptr[tok + 1] - lo;
  if (n == 0) return;  // finished by its record
  const float v_scale = p.v_scale ? p.v_scale[head / (p.n_q_heads / p.n_kv_heads)] : 1.f;
  const float* const base = p.partial + static_cast<int64_t>(head) * kRow;
  const int64_t stride = static_cast<int64_t>(p.n_q_heads) * kRow;
  float m = -INFINITY;
  for (int i = lane; i < n; i += 64) m = fmaxf(m, base[p.tok_part[lo + i] * stride + kD]);
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor(m, o, 64));
  float sum = 0.f, acc[kPer] = {};
  for (int at = 0; at < n; at += 64) {
    int part = 0;
    float weight = 0.f;
    if (at + lane < n) {
      part = p.tok_part[lo + at + lane];
      const float ms = base[part * stride + kD], ls = base[part * stride + kD + 1];
      weight = ms == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(ms - m);
      sum = fmaf(ls, weight, sum);
    }
    const int here = min(64, n - at);
    for (int i = 0; i < here; ++i) {
      const float* const row = base + __shfl(part, i) * stride + lane * kPer;
      const float wi = __shfl(weight, i);
#pragma unroll
      for (int e = 0; e < kPer; ++e) acc[e] = fmaf(row[e], wi, acc[e]);
    }
  }
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) sum += __shfl_xor(sum, o, 64);
  const float inv = sum > 0.f || sum != sum ? v_scale / sum : 0.f;
  Q* const out = static_cast<Q*>(const_cast<void*>(p.o.ptr)) + tok * p.o.stride_tok + head * p.o.stride_head + lane * kPer;
#pragma unroll
  for (int e = 0; e < kPer; ++e) out[e] = static_cast<Q>(acc[e] * inv);
  if (p.lse && lane == 0) p.lse[static_cast<int64_t>(head) * p.n_rows + tok] = (m + __builtin_amdgcn_logf(sum)) * 0.6931471805599453f;
}

template <typename T, int kD, int kNW, int kRB, int kBN>
hipError_t launch_shape(const ChunkParams& p, hipStream_t stream) {
  typedef Chunk<T, kD, kNW, kRB, kBN> C;
  const void* const f = reinterpret_cast<const void*>(chunk_attn_kernel<T, kD, kNW, kRB, kBN>);
  static std::atomic<bool> attr_set{false};  // setting it twice from two threads is harmless
  if (!attr_set) {
    const hipError_t e = hipFuncSetAttribute(f, hipFuncAttributeMaxDynamicSharedMemorySize, C::kLds);
    if (e != hipSuccess) return e;
    attr_set = true;
  }
  chunk_attn_kernel<T, kD, kNW, kRB, kBN><<<dim3(static_cast<unsigned>(p.n_workers) * p.n_kv_heads), dim3(C::kThreads), C::kLds, stream>>>(p);
  return hipGetLastError();
}

template <typename T, int kD>
hipError_t launch_kind(const ChunkParams& p, hipStream_t stream) {
  constexpr int kWide = Kind<T>::kBytes == 4 ? 32 : 64;
  hipError_t e = hipErrorInvalidValue;
  if (p.rows == 32) e = launch_shape<T, kD, 1, 1, 32>(p, stream);
  else if (p.rows == 64) e = launch_shape<T, kD, 2, 1, 32>(p, stream);
  else if (p.rows == 128) e = launch_shape<T, kD, 4, 1, kWide>(p, stream);
  else if (p.rows == 256) e = launch_shape<T, kD, 8, 1, kWide>(p, stream);
  if (e != hipSuccess || !p.merge) return e;
  const int64_t pairs = static_cast<int64_t>(p.n_rows) * p.n_q_heads;
  chunk_merge_kernel<typename Kind<T>::Q, kD><<<dim3(static_cast<unsigned>((pairs + 3) / 4)), dim3(256), 0, stream>>>(p);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_chunk_attn(const ChunkParams& p, int head_dim, ChunkKind kind, hipStream_t stream) {
  if (head_dim == 64) {
    return kind == ChunkKind::kBf16 ? launch_kind<__bf16, 64>(p, stream) : kind == ChunkKind::kF32 ? launch_kind<float, 64>(p, stream)
                                                                                                   : launch_kind<E4m3, 64>(p, stream);
  }
  return kind == ChunkKind::kBf16 ? launch_kind<__bf16, 128>(p, stream) : kind == ChunkKind::kF32 ? launch_kind<float, 128>(p, stream)
                                                                                                  : launch_kind<E4m3, 128>(p, stream);
}
