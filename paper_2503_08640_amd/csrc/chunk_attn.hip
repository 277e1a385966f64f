// Chunk attention (stage 2 for several new tokens per question, Sec. 2.2) on gfx950: every new token attends the sink, its
// question's selected groups and its own keys up to itself, the own keys lying in pages.
//
// Mathematics.  One softmax per row (a new token times a query head) over all its keys, taken in one pass over tiles of
// keys: with m the running maximum of the scores and l the running sum of 2^(s - m),
//     m' = max(m, max s),  l' = l 2^(m - m') + sum 2^(s - m'),  acc' = acc 2^(m - m') + sum 2^(s - m') v,   o = acc / l.
// m, l and acc are held in fp32.  Any m will do that keeps the probabilities in range, so m stays what the row's first keys
// give it while no score exceeds it by kRoom (walk).  Scores are transposed, S^T = K Q^T, so that a lane
// holds 16 keys of ONE row per block of 32 keys: maxima and sums need one exchange between the two half-waves and no LDS,
// and the probabilities are in place as the operand of O^T = V^T P^T.  bf16 products (8-bit caches are widened as they are
// staged, exactly: every e4m3 value is a bf16 value), fp32 products for fp32 tensors; the only rounding to fewer bits besides
// the output's is that of the probabilities to bf16, half a step (2^-8) at most and unbiased, while l sums them unrounded.  (Dividing
// by the sum of the rounded ones changed nothing, 2.332e-3 to 2.330e-3 of the result's norm, for 3 % of the time.)
//
// Work.  Workers and their records come from the host's plan (chunk_plan.cpp).  A record is a block of rows and a run of
// 64-key tiles: pool tiles from the lists, then a part of the question's own keys, whose number the device knows
// (self_len).  It leaves finished rows, or partial softmax states that the merge kernel joins.
//
// What bounds it.  Many rows: a tile of 256 rows and 64 keys of 128 channels is 2048 cycles of the matrix pipes, 2300 of LDS
// reads and 2000 of vector work (exponentials above all) on a compute unit; one barrier per step keeps the two waves of a
// SIMD side by side, and what does not overlap brings a tile to 2.0 us.  2048 tokens behind 90k and 30k own keys: 1860 us, 1080
// TFLOP/s (the library's product of 8192^3: 1212).  Few rows: memory, and the start of a record, a chain of loads (record,
// token, row of Q, list, first rows) of 3 us; a workgroup's waves without rows only fetch.  16 questions of 8 tokens over 30 % of
// 90k: 120 us, 3.3 TB/s of unique bytes; one token over 1200 keys: 17 us, 6 of them the merge.  8-bit caches of 64 channels:
// each wave fetches K or V alone, the choice ends up as pointers in scratch memory, and every request waits for the rows in
// flight (178 us for 6 prompts of 16 heads, 113 for the same in bf16).  Two row blocks per wave with one wave to a SIMD, which halves the LDS
// reads, were slower (2203 us for the 2048 tokens, 2028 then): nothing fills the waits of a lone wave.
#include <atomic>
#include <cstdint>

#include "kernels.hpp"
#include "layout.hpp"
#include "mfma_common.hpp"

namespace {
using namespace dbsa_mfma;

constexpr float kRoom = 24.f;    // log2 units a row's scores may exceed its reference maximum by
constexpr float kShrink = 24.f;  // log2 units that probabilities stay below 1 by where values are huge

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
typedef __attribute__((address_space(3))) uintx4 lds_piece;
typedef const __attribute__((address_space(3))) float lds_float;

// dma16 (mfma_common.hpp) with an address of its own per lane
__device__ inline void dma16_wide(uint64_t address, unsigned lds_addr) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off" : : "s"(lds_addr), "v"(address) : "memory");
}

// O += V P, as statements that change the accumulators where they are (left to itself the compiler keeps two sets of them and
// copies one to the other in every step).  It does not know what these are, so the spacing rules are kept by the order of the
// code: an accumulator's next product is at least two matrix instructions away, and the vector ALU reads or writes one only
// behind product_fence(), which passes the accumulators on, so that no use of them can be moved in front of its waits.
__device__ DBSA_INLINE void product_bf16(floatx16& o, const bf16x8& v, const bf16x8& p) {
  asm volatile("v_mfma_f32_32x32x16_bf16 %0, %1, %2, %0" : "+v"(o) : "v"(v), "v"(p));
}
__device__ DBSA_INLINE void product_f32(floatx16& o, float v, float p) {
  asm volatile("v_mfma_f32_32x32x2_f32 %0, %1, %2, %0" : "+v"(o) : "v"(v), "v"(p));
}
template <int kO>
__device__ DBSA_INLINE void product_fence(floatx16 (&acc)[kO]) {
  static_assert(kO == 2 || kO == 4, "head_dim 64 or 128");
  if constexpr (kO == 2) asm volatile("s_nop 15\n\ts_nop 15" : "+v"(acc[0]), "+v"(acc[1])::"memory");
  else asm volatile("s_nop 15\n\ts_nop 15" : "+v"(acc[0]), "+v"(acc[1]), "+v"(acc[2]), "+v"(acc[3])::"memory");
}

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

// kBN keys per step (a 64-key tile is one or two steps), kNW waves of 32 rows.
template <typename T, int kD, int kNW, int kBN>
struct Chunk {
  typedef typename Kind<T>::Q Q;
  static constexpr bool kF32 = Kind<T>::kBytes == 4;
  static constexpr int kThreads = 64 * kNW, kRows = 32 * kNW;
  static constexpr int kRowBytes = kD * Kind<T>::kBytes, kTileBytes = kBN * kRowBytes;  // as staged
  static constexpr int kSlots = kRowBytes / 16;                                         // 16-byte places of a staged row
  static constexpr int kPieces = kD * Kind<T>::kStoredBytes / 16;                       // 16-byte pieces of a stored row
  static constexpr int kOperand = kBN * kPieces;                                        // pieces of K, and of V, of a step
  static constexpr int kLoads = 2 * kOperand / kThreads;                                // pieces per thread
  static constexpr bool kApart = kOperand < kThreads;                                   // half the waves fetch K, half V
  static constexpr int kKeyBlocks = kBN / 32, kChBlocks = kD / 32;
  // Steps requested ahead of the one that is about to be read.  16-bit and fp32 rows go from memory straight into their
  // stage; 8-bit rows into a ring of the wave's own, from where the same lanes widen them into the stages.
  static constexpr bool kDirect = Kind<T>::kStoredBytes != 1;
  static constexpr int kFlight = kDirect ? (kNW == 8 || !kF32 ? 3 : 1) : kNW == 8 ? 3 : 4;
  // Eight waves of 16-bit operands run as a pipeline over half steps (walk): V is read one step behind K.
  static constexpr bool kPipelined = kNW == 8 && !kF32;
  static constexpr int kKStages = kDirect ? kFlight + 1 : 2, kVStages = kKStages + (kPipelined ? 1 : 0);
  static constexpr int kRingAt = (kKStages + kVStages) * kTileBytes;
  static constexpr int kRingBytes = kThreads * kLoads * 16;
  static constexpr int kPoisonAt = kRingAt + (kDirect ? 0 : kFlight * kRingBytes);  // per stage of V: each wave's mask of poisoned rows
  static constexpr int kVotesAt = kPoisonAt + kVStages * kNW * 8, kLds = kVotesAt + kNW * 4;
  static_assert(kPieces <= 32 && 64 % kPieces == 0, "a stored row is fetched by neighbouring lanes of one wave");
  static_assert(kApart ? kOperand * 2 == kThreads : kOperand % kThreads == 0, "whole pieces per thread");
  // K places: xor by row, so that the 16 rows a quarter wave reads of one column lie on different banks; V rows of 16-bit
  // elements are read transposed, four rows at a time (as in attn_prefill64.hip), V rows of fp32 element by element, the two
  // half-waves four rows apart.
  __device__ static DBSA_INLINE int k_swizzle(int row) { return kSlots >= 16 ? row % 16 : (row / 2) % 8; }
  __device__ static DBSA_INLINE int v_swizzle(int row) {
    if (kF32) return 8 * ((row / 4) % 2);
    return kSlots >= 16 ? 4 * (row % 4) : 4 * ((row / 2) % 2);
  }
};

// The lane index counted anew, for rare blocks of the step loop: what they derive from it is then not kept in registers
// through the loop.
__device__ DBSA_INLINE int lane_here() {
  int x;
  asm volatile("v_mbcnt_lo_u32_b32 %0, -1, 0\n\tv_mbcnt_hi_u32_b32 %0, -1, %0" : "=v"(x));
  return x;
}

template <typename T, int kD, int kNW, int kBN>
__global__ __launch_bounds__(64 * kNW, 2) void chunk_attn_kernel(ChunkParams p) {
  typedef Chunk<T, kD, kNW, kBN> C;
  typedef typename C::Q Q;
  constexpr bool kF32 = C::kF32;
  constexpr int kB = C::kKeyBlocks, kO = C::kChBlocks, kC = C::kSlots / 2;
  constexpr int kSteps = kChunkTile / kBN;  // steps of a tile
  constexpr int kEs = Kind<T>::kStoredBytes;
  extern __shared__ __attribute__((aligned(1024))) unsigned char smem[];

  const int tid = threadIdx.x, lane = tid % 64, l32 = lane % 32, half = lane / 32;
  const int wave = __builtin_amdgcn_readfirstlane(tid / 64);
  const int hk = __builtin_amdgcn_readfirstlane(static_cast<int>(blockIdx.x) % p.n_kv_heads);
  const int worker = __builtin_amdgcn_readfirstlane(static_cast<int>(blockIdx.x) / p.n_kv_heads);
  const int r = p.n_q_heads / p.n_kv_heads;
  // scores in log2 units: scale * log2 e (and the keys' scale) goes onto them in fp32.  The softmax takes a positive factor
  // (a masked -inf stays one, the largest score the largest): the sign of a negative key scale goes onto the rows of Q, and so
  // do a factor of nothing and one that is no number.
  float c2 = p.scale_log2e, on_rows = 1.f;
  if constexpr (kEs == 1) {
    const float c = c2 * p.k_scale[hk];
    on_rows = c > 0.f ? 1.f : c < 0.f ? -1.f : c;
    c2 = c == 0.f || c != c ? 1.f : fabsf(c);
  }

  const unsigned lds0 = static_cast<unsigned>(reinterpret_cast<uintptr_t>((lds_byte*)smem));
  // What the step loop reads of the arguments, in registers of its own: the compiler otherwise picks the ADDRESS of the
  // argument (pool or own) and loads it anew in every step, four scalar loads one behind the other.
  auto own_register = [](auto x) DBSA_INLINE {
    decltype(x) y;
    if constexpr (sizeof(x) == 8) y = static_cast<decltype(x)>(uniform64(static_cast<uint64_t>(x)));
    else y = __builtin_amdgcn_readfirstlane(x);
    asm volatile("" : "+s"(y));
    return y;
  };
  const const_words entries = (const_words)(own_register(reinterpret_cast<uintptr_t>(p.ent)));
  const const_words page_table = (const_words)(own_register(reinterpret_cast<uintptr_t>(p.page_table)));
  const uint64_t kpool = own_register(reinterpret_cast<uint64_t>(p.k_pool.ptr) + hk * p.k_pool.stride_head * kEs);
  const uint64_t vpool = own_register(reinterpret_cast<uint64_t>(p.v_pool.ptr) + hk * p.v_pool.stride_head * kEs);
  const uint64_t kown = own_register(reinterpret_cast<uint64_t>(p.k_own.ptr) + hk * p.k_own.stride_head * kEs);
  const uint64_t vown = own_register(reinterpret_cast<uint64_t>(p.v_own.ptr) + hk * p.v_own.stride_head * kEs);
  // (bytes; used where they fit: narrow)
  const int kpool_stride = own_register(static_cast<int>(p.k_pool.stride_tok * kEs)), vpool_stride = own_register(static_cast<int>(p.v_pool.stride_tok * kEs));
  const int kown_stride = own_register(static_cast<int>(p.k_own.stride_tok * kEs)), vown_stride = own_register(static_cast<int>(p.v_own.stride_tok * kEs));
  const int64_t page_bytes = own_register(p.stride_page * kEs);
  const int page_log2 = own_register(p.page_log2), n_pages = own_register(p.n_pages), table_stride = own_register(p.table_stride);
  const bool narrow = own_register(p.narrow) != 0;
  const int page_mask = (1 << page_log2) - 1;
  // LDS addresses of fragments: K fragment (kb, c) is row 32 kb + l32, place 2 c + half; V fragment (16-bit: kb, ch, ob) keys
  // 32 kb + 16 ch + 4 half + {0..3, 8..11}, the order the probabilities lie in, read transposed: lane j of 16 fetches four
  // channels of one key and gets four keys of one channel.  (A place is xor-ed: base ^ (32 c), base ^ (64 ob).)
  const int k_at = l32 * C::kRowBytes + ((half ^ C::k_swizzle(l32)) * 16);
  const int v_at = (4 * half + (lane % 16) / 4) * C::kRowBytes +
                   (((2 * (l32 / 16) + (lane % 4) / 2) ^ C::v_swizzle((lane % 16) / 4)) * 16) + (lane % 2) * 8;

  // Where a step's K and V lie in LDS (8 bits: and the ring place it lands in); steps take the places in turn, over all records.
  struct Place {
    unsigned k, v, ring, k0;
    __device__ DBSA_INLINE void next_k() { k = k == k0 + (C::kKStages - 1) * C::kTileBytes ? k0 : k + C::kTileBytes; }
    __device__ DBSA_INLINE void next_v() { v = v == k0 + (C::kKStages + C::kVStages - 1) * C::kTileBytes ? k0 + C::kKStages * C::kTileBytes : v + C::kTileBytes; }
    __device__ DBSA_INLINE void next_ring() { ring = ring == k0 + C::kRingAt + (C::kFlight - 1) * C::kRingBytes ? k0 + C::kRingAt : ring + C::kRingBytes; }
    // a step that lands in its stage
    __device__ DBSA_INLINE void next_direct() {
      if (C::kDirect) {
        next_k();
        next_v();
      } else {
        next_ring();
      }
    }
  };
  const Place start{lds0, lds0 + C::kKStages * C::kTileBytes, lds0 + C::kRingAt, lds0};
  Place wanted = start, arrived = start, read = start;  // of the step requested next, put next; K and V read next
  const const_words workers = (const_words)(reinterpret_cast<uintptr_t>(p.ptr));
  const const_words tokens = (const_words)(reinterpret_cast<uintptr_t>(p.toks));
  const const_words lengths = (const_words)(reinterpret_cast<uintptr_t>(p.self_len));
  const int rec_end = workers[worker + 1];
  for (int rec = workers[worker]; rec < rec_end; ++rec) {
    const const_words w = (const_words)(reinterpret_cast<uintptr_t>(p.rec)) + rec * kChunkWords;
    const int tok_begin = w[0], n_tok = w[1], ent_begin = w[2], n_ent = w[3], own_u = w[4], part_base = w[8];
    const int cu = w[9], t_new = w[10];

    // ---- the row of this lane (both half-waves hold it) ----
    int own_n = 0;  // own keys there are
    if (own_u >= 0) own_n = min(max(lengths[own_u], 0), p.own_capacity);
    const int row_index = wave * 32 + l32;
    const bool row_ok = row_index / r < n_tok;
    const int row_in = min(row_index / r, n_tok - 1);
    const int row_tok = p.toks[tok_begin + row_in];
    const int row_pos = own_n - t_new + (row_tok - cu);  // the row's own index: it sees own keys 0 .. row_pos
    typedef typename std::conditional<kF32, floatx4, bf16x8>::type Piece;
    Piece qf[kC];
    {
      const Q* const qp = static_cast<const Q*>(p.q.ptr) + row_tok * p.q.stride_tok + (hk * r + row_index % r) * p.q.stride_head;
#pragma unroll
      for (int c = 0; c < kC; ++c) {
        qf[c] = *reinterpret_cast<const Piece*>(qp + (2 * c + half) * (16 / static_cast<int>(sizeof(Q))));
        if constexpr (kEs == 1) {
          if (on_rows != 1.f) {
#pragma unroll
            for (int e = 0; e < 8; ++e) qf[c][e] = static_cast<Q>(static_cast<float>(qf[c][e]) * on_rows);
          }
        }
      }
    }
    // own tiles of this record: its share of those up to the last token's own key
    int own_first = 0, own_steps = 0;
    const int first_pos = own_n - t_new + (tokens[tok_begin] - cu);  // (tokens of a question ascend)
    if (own_u >= 0) {
      const int last = own_n - t_new + (tokens[tok_begin + n_tok - 1] - cu);
      const int64_t tiles = max(0, (last + kChunkTile) / kChunkTile);
      const int lo = static_cast<int>(w[5] * tiles / w[7]), hi = static_cast<int>(w[6] * tiles / w[7]);
      own_first = lo * kChunkTile;
      own_steps = (hi - lo) * kSteps;
    }
    const int pool_steps = n_ent * kSteps, steps = pool_steps + own_steps;

    // ---- the stream of steps ----
    // What a step hangs off: its list entry, or the pages of its keys.  Own steps never straddle a page of kBN tokens or more;
    // smaller pages are at most kPages to a step.
    constexpr int kPages = kBN / 16;
    struct Ahead {
      int start, len;
      int page[kPages];
    };
    auto fetch = [&](int s) DBSA_INLINE {
      Ahead x{0, 0, {}};
      if (s < pool_steps) {
        const const_words e = entries + 2 * static_cast<int64_t>(ent_begin + s / kSteps);
        x.start = e[0];
        x.len = e[1];
      } else {
        const int first = (own_first + (s - pool_steps) * kBN) >> page_log2;
        const const_words table = page_table + static_cast<int64_t>(own_u) * table_stride;
        x.page[0] = table[min(first, table_stride - 1)];
        if (page_mask < kBN - 1) {
#pragma unroll
          for (int i = 1; i < kPages; ++i) x.page[i] = table[min(first + i, table_stride - 1)];  // (those behind the step are not used)
        }
      }
      return x;
    };
    auto page_there = [&](int page) DBSA_INLINE { return page >= 0 && page < n_pages; };
    // page of key `key` of an own step
    auto page_of = [&](const Ahead& x, int key) DBSA_INLINE {
      int page = x.page[0];
      if (page_mask < kBN - 1) {
        const int at = key >> page_log2;
#pragma unroll
        for (int i = 1; i < kPages; ++i) page = at == i ? x.page[i] : page;
      }
      return page;
    };
    // Which own keys of a step there are: bit key.
    auto keys_there = [&](const Ahead& x, int first) DBSA_INLINE {
      const int ln = lane_here();
      return __builtin_amdgcn_ballot_w64(ln < kBN && first + ln < own_n && page_there(page_of(x, ln)));
    };
    constexpr uint64_t kAllKeys = ~0ull >> (64 - kBN);

    // This thread's pieces of a step: piece tid + i threads of K, then of V; the operand of piece i is the wave's.
    auto is_v = [&](int i) DBSA_INLINE { return C::kApart ? wave >= kNW / 2 : i >= C::kLoads / 2; };
    auto piece_row = [&](int i, int t) DBSA_INLINE { return (t + i * C::kThreads) % C::kOperand / C::kPieces; };
    // first row of the rows that wave and pass i fetch (1 KiB: 64 pieces)
    auto wave_row = [&](int i) DBSA_INLINE { return (64 * wave + i * C::kThreads) % C::kOperand / C::kPieces; };
    // where piece i of the step at `place` lands: places of a stage are xor-ed on the way (the lane fetches the piece that belongs
    // there), the ring holds pieces as they come
    auto landing = [&](const Place& place, int i) DBSA_INLINE {
      unsigned at;
      if constexpr (C::kDirect) at = (is_v(i) ? place.v : place.k) + wave_row(i) * C::kRowBytes;
      else at = place.ring + (i * kNW + wave) * 1024;
      return static_cast<unsigned>(__builtin_amdgcn_readfirstlane(static_cast<int>(at)));
    };
    auto fetched_col = [&](int i, int t) DBSA_INLINE {
      const int col = t % C::kPieces, row = piece_row(i, t);
      return (C::kDirect ? col ^ (is_v(i) ? C::v_swizzle(row) : C::k_swizzle(row)) : col) * 16;
    };
    bool again;           // the quick walk does not do for this record (see there)
    bool beyond;          // its sums of values left fp32
    uint32_t partly;      // bit s % 32: some row does not see some key of step s (kept until its product is done)
    uint32_t lacking;     // the same: some key of step s is not there
    // That of 64 steps, one per lane.  (Scalar loads in every step would be waited for by its first LDS read, which cannot
    // tell them from its own: they come back in no order.)
    int window, hung[kPages];
    auto look_ahead = [&](int s) DBSA_INLINE {
      window = s;
      const int at = s + lane_here();
#pragma unroll
      for (int i = 0; i < kPages; ++i) hung[i] = 0;
      if (at < pool_steps) {
        const int32_t* const e = p.ent + 2 * (static_cast<int64_t>(ent_begin) + at / kSteps);
        hung[0] = e[0];
        hung[1] = e[1];
      } else if (at < steps) {
        const int first = (own_first + (at - pool_steps) * kBN) >> page_log2;
        const int32_t* const table = p.page_table + static_cast<int64_t>(own_u) * table_stride;
        hung[0] = table[min(first, table_stride - 1)];
        if (page_mask < kBN - 1) {
#pragma unroll
          for (int i = 1; i < kPages; ++i) hung[i] = table[min(first + i, table_stride - 1)];
        }
      }
      // (not left in flight: the waits for rows count)
      wait_vmcnt<0>();
    };
    auto hangs_off = [&](int s) DBSA_INLINE {  // s in the window
      Ahead x;
#pragma unroll
      for (int i = 0; i < kPages; ++i) x.page[i] = __builtin_amdgcn_readlane(hung[i], s - window);
      x.start = x.page[0];
      x.len = x.page[1];
      return x;
    };
    auto recall = [&](int s) DBSA_INLINE { return s >= window ? hangs_off(s) : fetch(s); };  // s was requested
    auto request = [&](int s) DBSA_INLINE {  // s < steps, one after the other
      if (__builtin_expect(s == window + 64, 0)) look_ahead(s);
      const Ahead x = hangs_off(s);
      const bool own = s >= pool_steps;
      uint64_t kt = kpool, vt = vpool;
      int ks = kpool_stride, vs = vpool_stride, off, len, row;
      bool whole, in_line;  // every row sees every key; kBN rows one after the other
      bool lacks = false;   // some key is not there
      if (!own) {
        off = kSteps == 1 ? 0 : (s % kSteps) * kBN;
        len = min((x.len & 0xFFFF) - off, kBN);
        row = x.start + off;
        whole = in_line = len == kBN;
      } else {
        off = own_first + (s - pool_steps) * kBN;
        len = min(own_n - off, kBN);
        whole = len == kBN && off + kBN - 1 <= first_pos;
        row = off & page_mask;
        in_line = false;
        if (page_mask >= kBN - 1) {
          in_line = len == kBN && page_there(x.page[0]);
          lacks = !in_line;
        } else {
          lacks = len < kBN;
#pragma unroll
          for (int i = 0; i < kPages; ++i) lacks |= i << page_log2 < kBN && !page_there(x.page[i]);
        }
        whole = whole && !lacks;
        kt = kown + x.page[0] * page_bytes;
        vt = vown + x.page[0] * page_bytes;
        ks = kown_stride;
        vs = vown_stride;
      }
      const uint32_t bit = 1u << (s % 32);
      partly = whole ? partly & ~bit : partly | bit;
      lacking = lacks ? lacking | bit : lacking & ~bit;
      if (__builtin_expect(in_line && narrow, 1)) {
        kt += static_cast<int64_t>(row) * ks;
        vt += static_cast<int64_t>(row) * vs;
#pragma unroll
        for (int i = 0; i < C::kLoads; ++i) {
          const int stride = is_v(i) ? vs : ks;
          const int row0 = i * C::kThreads % C::kOperand / C::kPieces;  // (whole rows per pass of the threads)
          dma16(uniform64((is_v(i) ? vt : kt) + static_cast<unsigned>(row0 * stride)),
                static_cast<unsigned>(piece_row(0, tid) * stride + fetched_col(i, tid)), landing(wanted, i));
        }
      } else if (own && !lacks && narrow) {
        // smaller pages: the rows a wave fetches in one pass, at most 16, lie in one
        static_assert(64 / C::kPieces <= 16, "no page is smaller");
#pragma unroll
        for (int i = 0; i < C::kLoads; ++i) {
          const int row0 = __builtin_amdgcn_readfirstlane(wave_row(i)), stride = is_v(i) ? vs : ks;
          dma16(uniform64((is_v(i) ? vown : kown) + page_of(x, row0) * page_bytes + static_cast<unsigned>(((off + row0) & page_mask) * stride)),
                static_cast<unsigned>(lane / C::kPieces * stride + fetched_col(i, tid)), landing(wanted, i));
        }
      } else {
        const int t = 64 * wave + lane_here();
        const int64_t ks64 = (own ? p.k_own.stride_tok : p.k_pool.stride_tok) * kEs, vs64 = (own ? p.v_own.stride_tok : p.v_pool.stride_tok) * kEs;
#pragma unroll
        for (int i = 0; i < C::kLoads; ++i) {
          const int key = piece_row(i, t);
          int64_t at;
          if (own) {
            const int page = page_of(x, key);
            at = key < len && page_there(page) ? page * page_bytes + ((off + key) & page_mask) * (is_v(i) ? vs64 : ks64) : 0;
          } else {
            at = (x.start + (len > 0 ? off + min(key, len - 1) : 0)) * (is_v(i) ? vs64 : ks64);
          }
          dma16_wide((own ? (is_v(i) ? vown : kown) : (is_v(i) ? vpool : kpool)) + at + fetched_col(i, t), landing(wanted, i));
        }
      }
      wanted.next_direct();
    };
    // step s has landed, as far as this wave fetched it; `newer` steps were requested since
    auto wait_for = [&](int s, auto NEWER) DBSA_INLINE {
      constexpr int kNewer = decltype(NEWER)::value;
      if (s + kNewer < steps) wait_vmcnt<kNewer * C::kLoads>();
      else wait_vmcnt<0>();
    };
    // Where some rows do not see every key (the chunk's own diagonal, keys that are not there), nothing may reach them through
    // 0 * NaN: keys that are not there, and rows of V with a non-finite value, are staged as zeros, the latter's keys added
    // one by one to the rows that see them.
    uint64_t* const poison = reinterpret_cast<uint64_t*>(smem + C::kPoisonAt);
    auto clean = [&](int s, uintx4 (&raw)[C::kLoads]) DBSA_INLINE {  // -> whether it changed any
      uint64_t mask = 0;
      constexpr uint64_t kRowLanes = (1ull << C::kPieces) - 1;
      const int ln = lane_here();
      const int first = own_first + (s - pool_steps) * kBN;
      const bool lacks = (lacking >> (s % 32)) & 1;
      const uint64_t there = lacks ? keys_there(recall(s), first) : kAllKeys;
#pragma unroll
      for (int i = 0; i < C::kLoads; ++i) {
        const bool missing = !((there >> piece_row(i, 64 * wave + ln)) & 1);
        uint64_t bad = 0;
        if (is_v(i)) {
          bad = __builtin_amdgcn_ballot_w64(!missing && not_finite<T>(raw[i]));
          if (__builtin_expect(bad != 0, 0))
            for (int rr = 0; rr < 64 / C::kPieces; ++rr)
              if ((bad >> (rr * C::kPieces)) & kRowLanes) mask |= 1ull << (wave_row(i) + rr);
        }
        if (missing || ((bad >> (ln / C::kPieces * C::kPieces)) & kRowLanes)) raw[i] = uintx4{0, 0, 0, 0};
      }
      if (ln == 0) poison[(arrived.v - start.v) / C::kTileBytes * kNW + wave] = mask;
      again |= mask != 0;
      return lacks || mask != 0;
    };
    // What this wave does to its landed pieces of step s before the others read them.
    auto put = [&](int s) DBSA_INLINE {
      const bool own_partly = s >= pool_steps && ((partly >> (s % 32)) & 1);
      if constexpr (C::kDirect) {
        if (__builtin_expect(own_partly, 0)) {
          uintx4 raw[C::kLoads];
          const int ln = lane_here();
#pragma unroll
          for (int i = 0; i < C::kLoads; ++i) raw[i] = *reinterpret_cast<const lds_piece*>(static_cast<uintptr_t>(landing(arrived, i) + ln * 16));
          if (clean(s, raw)) {
#pragma unroll
            for (int i = 0; i < C::kLoads; ++i) *reinterpret_cast<lds_piece*>(static_cast<uintptr_t>(landing(arrived, i) + ln * 16)) = raw[i];
          }
        }
        arrived.next_k();
        arrived.next_v();
      } else {
        uintx4 raw[C::kLoads];
#pragma unroll
        for (int i = 0; i < C::kLoads; ++i) raw[i] = *reinterpret_cast<const lds_piece*>(static_cast<uintptr_t>(landing(arrived, i) + lane * 16));
        if (__builtin_expect(own_partly, 0)) clean(s, raw);
#pragma unroll
        for (int i = 0; i < C::kLoads; ++i) {
          const int row = piece_row(i, tid), col = tid % C::kPieces;
          const unsigned at = (is_v(i) ? arrived.v : arrived.k) + row * C::kRowBytes;
          const int swizzle = is_v(i) ? C::v_swizzle(row) : C::k_swizzle(row);
          uintx4 lo, hi;
          widen16(raw[i], lo, hi);
          *reinterpret_cast<lds_piece*>(static_cast<uintptr_t>(at + ((2 * col) ^ swizzle) * 16)) = lo;
          *reinterpret_cast<lds_piece*>(static_cast<uintptr_t>(at + ((2 * col + 1) ^ swizzle) * 16)) = hi;
        }
        arrived.next_k();
        arrived.next_v();
        arrived.next_ring();
      }
    };

    // ---- softmax state ----
    floatx16 acc[kO];
    float m, l;                       // l: this lane's keys' share
    float shrink = 1.f;               // on the probabilities of the careful walk (see there)
    floatx16 s[kB];                   // scores, then (fp32) probabilities
    bf16x8 pf[kF32 ? 1 : kB][2];      // probabilities as operands of the product

    // element i of block kb is key 32 kb + 8 (i / 4) + 4 half + i % 4 of the step
    auto mask = [&](int st, auto KB) DBSA_INLINE {
      constexpr int kb = decltype(KB)::value;
      const int ln = lane_here();
      uint64_t there = ~0ull;
      int last;
      if (st < pool_steps) {
        last = (recall(st).len & 0xFFFF) - (st % kSteps) * kBN - 1;
      } else {
        const int first = own_first + (st - pool_steps) * kBN;
        if ((lacking >> (st % 32)) & 1) there = keys_there(recall(st), first);
        last = row_pos - first;
      }
      last -= 4 * (ln / 32);
      there >>= 4 * (ln / 32);
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const int key = 32 * kb + 8 * (i / 4) + i % 4;
        if (key > last || !((there >> key) & 1)) s[kb][i] = -INFINITY;
      }
    };
    auto row_max = [&](auto KB) DBSA_INLINE {
      constexpr int kb = decltype(KB)::value;
      float top = s[kb][0];
#pragma unroll
      for (int i = 1; i < 16; ++i) top = fmaxf(top, s[kb][i]);
      return half_swap_max(top) * c2;
    };
    // the scores of half step (st, kb) masked, and a reference maximum for rows that had none
    auto prepare = [&](int st, auto KB) DBSA_INLINE {
      if (__builtin_expect((partly >> (st % 32)) & 1, 0)) mask(st, KB);
      if (__builtin_expect(__builtin_amdgcn_ballot_w64(m == -INFINITY) != 0, 0)) {
        const float top = row_max(KB);
        m = m == -INFINITY ? top : m;
      }
    };
    // a step's sum of probabilities in one lane above this: some score has outgrown its reference by more than kRoom, give or take
    const float outgrown = __builtin_exp2f(kRoom);
    // one probability and its share of the sum
    auto probability = [&](float score, float less) DBSA_INLINE { return __builtin_amdgcn_exp2f(fmaf(score, c2, less)); };
    auto pack = [&](auto KB) DBSA_INLINE {
      constexpr int kb = decltype(KB)::value;
      if constexpr (!kF32) {
#pragma unroll
        for (int ch = 0; ch < 2; ++ch) {
          union {
            bf16x8 v;
            bf16x2 p2[4];
          } x;
#pragma unroll
          for (int e = 0; e < 4; ++e) x.p2[e] = __builtin_convertvector(floatx2{s[kb][8 * ch + 2 * e], s[kb][8 * ch + 2 * e + 1]}, bf16x2);
          pf[kb][ch] = x.v;
        }
      }
    };
    auto softmax = [&](auto CAREFUL, int st) DBSA_INLINE {
      static_for<kB>([&](auto KB) DBSA_INLINE {
        constexpr int kb = decltype(KB)::value;
        if constexpr (!decltype(CAREFUL)::value) {
          prepare(st, KB);
        } else {
          if ((partly >> (st % 32)) & 1) mask(st, KB);
          const float top = row_max(KB), bigger = fmaxf(m, shrink == 1.f ? top : ceilf(top));
          const float alpha = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m - bigger);
          m = bigger;
          l *= alpha;
#pragma unroll
          for (int ob = 0; ob < kO; ++ob) acc[ob] *= alpha;
          if constexpr (kb > 0) {  // (the first half's probabilities go by the same maximum)
#pragma unroll
            for (int i = 0; i < 16; ++i) s[0][i] *= alpha;
          }
        }
        const float less = m == -INFINITY ? 0.f : -m;
        float sum = 0.f;
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          s[kb][i] = probability(s[kb][i], less);
          if constexpr (decltype(CAREFUL)::value) s[kb][i] *= shrink;
          sum += s[kb][i];
        }
        l += sum;
        if constexpr (!decltype(CAREFUL)::value) again |= sum > outgrown;
      });
      static_for<kB>([&](auto KB) DBSA_INLINE { pack(KB); });
    };
    // the keys that clean() kept out of the product
    auto add_poison = [&](int st) DBSA_INLINE {
      uint64_t keys = 0;
      for (int i = 0; i < kNW; ++i) keys |= poison[(read.v - start.v) / C::kTileBytes * kNW + i];
      keys = uniform64(keys);
      const int h = lane_here() / 32;
      while (keys) {
        const int key = __builtin_ctzll(keys);
        keys &= keys - 1;
        const int j = own_first + (st - pool_steps) * kBN + key;
        const int64_t page = page_table[static_cast<int64_t>(own_u) * table_stride + (j >> page_log2)];
        const unsigned char* const v = static_cast<const unsigned char*>(p.v_own.ptr) +
            (hk * p.v_own.stride_head + page * p.stride_page + (j & page_mask) * p.v_own.stride_tok) * kEs;
        float mine = 0.f;  // the key's probability, in the half-wave that holds the key
#pragma unroll
        for (int kb = 0; kb < kB; ++kb)
#pragma unroll
          for (int i = 0; i < 16; ++i)
            if (key == 32 * kb + 8 * (i / 4) + 4 * h + i % 4) {
              if constexpr (kF32) mine = s[kb][i];
              else mine = static_cast<float>(pf[kb][i / 8][i % 8]);
            }
        const float other = __shfl_xor(mine, 32);
        const float prob = (key / 4) % 2 == h ? mine : other;
#pragma unroll
        for (int ob = 0; ob < kO; ++ob)
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            const float x = stored_value<T>(v, 32 * ob + 8 * (i / 4) + 4 * h + i % 4);
            if (prob != 0.f) acc[ob][i] = fmaf(prob, x, acc[ob][i]);
          }
      }
    };
    // A run of matrix instructions: S = K Q for half QK of the step whose K is read next, and O += V P for half PV of the step
    // whose V is read next (-1: left out).  Fragments are read from LDS kDist matrix instructions before the one that takes
    // them, in an order the compiler is not left to change: it would otherwise read each right before its use and wait for
    // it.  Half SM's scores become probabilities on the way, a few vector instructions behind every matrix instruction.
    auto run = [&](auto QK, auto PV, auto SM) DBSA_INLINE {
      constexpr int kq = decltype(QK)::value, kv = decltype(PV)::value, ks = decltype(SM)::value;
      constexpr int nK = kq >= 0 ? kC : 0, nV = kv >= 0 ? (kF32 ? 16 * kO : 2 * kO) : 0, n = nK + nV;
      constexpr int kDist = kF32 ? 4 : 6;
      // K fragments among the first j: two to each of V, so that scores are ready some instructions before the run ends
      constexpr auto k_before = [](int j) { return nV == 0 ? j : (2 * j + 2) / 3 < nK ? (2 * j + 2) / 3 : nK; };
      const unsigned vt = read.v, kt = read.k;
      int k_here = k_at, v_here = v_at;  // (a fragment's address is one instruction from these; kept, they are twelve registers)
      asm volatile("" : "+v"(k_here), "+v"(v_here));
      if constexpr (nK > 0) {
#pragma unroll
        for (int i = 0; i < 16; ++i) s[kq][i] = 0.f;
      }
      const float less = m == -INFINITY ? 0.f : -m;
      float sum = 0.f, two[2];
      bf16x2 packed[8];
      Piece ring[kDist];  // (fp32: V fragments are single floats)
      auto read_fragment = [&](auto F) DBSA_INLINE {
        constexpr int f = decltype(F)::value, k = k_before(f), v = f - k;
        if constexpr (k_before(f + 1) > k) {
          ring[f % kDist] = *(reinterpret_cast<const __attribute__((address_space(3))) Piece*>(static_cast<uintptr_t>(kt + (k_here ^ (32 * k)))) +
                              32 * kq * C::kRowBytes / 16);
        } else if constexpr (kF32) {
          constexpr int ob = v % kO, i = v / kO, row = 32 * kv + 8 * (i / 4) + i % 4;
          const int ch = 32 * ob + l32;
          ring[f % kDist][0] = *reinterpret_cast<lds_float*>(static_cast<uintptr_t>(
              vt + (row + 4 * half) * C::kRowBytes + (((ch / 4) ^ (8 * ((row / 4 + half) % 2))) * 16) + (ch % 4) * 4));
        } else {
          constexpr int ob = v % kO, ch = v / kO;
          const lds_byte* const at = reinterpret_cast<const lds_byte*>(static_cast<uintptr_t>(vt + (v_here ^ (64 * ob)))) + (32 * kv + 16 * ch) * C::kRowBytes;
          const bf16x4 lo = lds_read_tr(at), hi = lds_read_tr(at + 8 * C::kRowBytes);
          ring[f % kDist] = __builtin_bit_cast(Piece, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
        }
      };
      __builtin_amdgcn_sched_barrier(0);
      static_for<(kDist < n ? kDist : n)>([&](auto F) DBSA_INLINE { read_fragment(F); });
      __builtin_amdgcn_sched_barrier(0);
      static_for<n>([&](auto F) DBSA_INLINE {
        constexpr int f = decltype(F)::value, k = k_before(f), v = f - k;
        if constexpr (k_before(f + 1) > k) {
          if constexpr (kF32) {
#pragma unroll
            for (int e = 0; e < 4; ++e) s[kq] = __builtin_amdgcn_mfma_f32_32x32x2f32(ring[f % kDist][e], qf[k][e], s[kq], 0, 0, 0);
          } else {
            s[kq] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, ring[f % kDist]), __builtin_bit_cast(bf16x8, qf[k]), s[kq], 0, 0, 0);
          }
        } else if constexpr (kF32) {
          product_f32(acc[v % kO], ring[f % kDist][0], s[kv][v / kO]);
        } else {
          product_bf16(acc[v % kO], __builtin_bit_cast(bf16x8, ring[f % kDist]), pf[kv][v / kO]);
        }
        if constexpr (f + kDist < n) read_fragment(std::integral_constant<int, f + kDist>{});
        if constexpr (ks >= 0) {
          // 16 probabilities over n slots; a pair is packed and summed behind the next one (a result of the transcendental unit
          // cannot be used by the very next instructions)
          static_for<16 * (f + 1) / n - 16 * f / n>([&](auto J) DBSA_INLINE {
            constexpr int i = 16 * f / n + decltype(J)::value;
            if constexpr (i % 2 == 0 && i > 0) {
              packed[i / 2 - 1] = __builtin_convertvector(floatx2{two[0], two[1]}, bf16x2);
              sum += two[0] + two[1];
              asm volatile("" : "+v"(packed[i / 2 - 1]), "+v"(sum));  // (else it sinks behind the run)
            }
            two[i % 2] = probability(s[ks][i], less);
            asm volatile("" : "+v"(two[i % 2]));
          });
        }
        __builtin_amdgcn_sched_barrier(0);
      });
      if constexpr (ks >= 0) {
        packed[7] = __builtin_convertvector(floatx2{two[0], two[1]}, bf16x2);
        sum += two[0] + two[1];
        l += sum;
        again |= sum > outgrown;
#pragma unroll
        for (int ch = 0; ch < 2; ++ch) {
          union {
            bf16x8 v;
            bf16x2 p2[4];
          } x;
#pragma unroll
          for (int e = 0; e < 4; ++e) x.p2[e] = packed[4 * ch + e];
          pf[ks][ch] = x.v;
        }
      }
    };

    // What happens to step n while step n - 1 is still being read.  (A wave's own ring place is free again once it has read it.)
    auto lds_done = [] { asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory"); };
    auto barrier = [&] {
      lds_done();
      __builtin_amdgcn_s_barrier();
      asm volatile("" ::: "memory");
    };
    constexpr std::integral_constant<int, -1> kNone{};
    constexpr std::integral_constant<int, 0> k0{};
    constexpr std::integral_constant<int, kB - 1> k1{};  // the second half of a step, where it has one
    // All steps of the record.  The quick walk never touches the accumulators but in the product (a block that sometimes
    // scales them costs a copy of all of them in every step): a row's reference maximum is that of the first step in which it
    // sees a key, and later scores may exceed it by kRoom, where probabilities and their sums are still far inside fp32 and
    // bf16.  Rows whose scores grow further, values that are not finite under a mask, and accumulators that are not finite
    // send the workgroup through the record once more, carefully: with the running maximum, and the poisoned keys one by
    // one.  Where it was the accumulators, the probabilities are held 2^kShrink times smaller, so that 2^kShrink of the largest
    // values add up to no more than one of them; the maximum is then kept to whole numbers, which take kShrink without a
    // rounding.  (Only there: next to huge values a channel of tiny ones, 2^-102 and below, loses bits by it.)
    auto begin_walk = [&]() DBSA_INLINE {
      m = -INFINITY;
      l = 0.f;
      again = beyond = false;
#pragma unroll
      for (int ob = 0; ob < kO; ++ob)
#pragma unroll
        for (int i = 0; i < 16; ++i) acc[ob][i] = 0.f;
      partly = lacking = 0;
      look_ahead(0);
    };
    // Step n is put, and the one kFlight behind it requested.  One barrier per step: behind it, step n has landed for all
    // waves, and all have read what they read before it, whose stages the step requested now takes (8 bits: whose stages the
    // step put before the next barrier takes).
    auto advance = [&](int n) DBSA_INLINE {
      if (n >= 0) {
        wait_for(n, std::integral_constant<int, C::kFlight - 1>{});
        put(n);
        barrier();
      }
      if (n + C::kFlight < steps) request(n + C::kFlight);
    };
    auto walk = [&]() DBSA_INLINE {
      begin_walk();
      if constexpr (C::kPipelined) {
        // Half steps of 32 keys in three stages, one apart: while the probabilities of a half are made, the scores of the next
        // half and the product of the one before it run on the matrix pipe; no instruction waits for one of its own half.
        // (One barrier per step keeps the two waves of a SIMD side by side, so that each has to mix its matrix and vector
        // instructions itself.)
        for (int n = -C::kFlight; n <= 0; ++n) advance(n);
        run(k0, kNone, kNone);
        prepare(0, k0);
        run(k1, kNone, k0);
        read.next_k();
        for (int st = 0; st < steps - 1; ++st) {
          advance(st + 1);
          prepare(st, k1);
          run(k0, k0, k1);
          prepare(st + 1, k0);
          run(k1, k1, k0);
          read.next_k();
          read.next_v();
        }
        prepare(steps - 1, k1);
        run(kNone, k0, k1);
        run(kNone, k1, kNone);
        read.next_v();
      } else {
        for (int st = -C::kFlight; st < steps; ++st) {
          advance(st);
          if (st < 0) continue;
          run(k0, kNone, kNone);
          softmax(std::false_type{}, st);
          run(kNone, k0, kNone);
          read.next_k();
          read.next_v();
        }
      }
      product_fence(acc);
      if constexpr (kEs != 1) {  // (sums of bytes stay far inside fp32)
        float nothing[kO] = {};  // 0, or NaN
#pragma unroll
        for (int i = 0; i < 16; ++i)
#pragma unroll
          for (int ob = 0; ob < kO; ++ob) nothing[ob] = fmaf(acc[ob][i], 0.f, nothing[ob]);
#pragma unroll
        for (int ob = 0; ob < kO; ++ob) beyond |= nothing[ob] != 0.f;
      }
    };
    // a wave without rows brings its pieces
    auto walk_idle = [&]() DBSA_INLINE {
      begin_walk();
      for (int n = -C::kFlight; n < steps; ++n) advance(n);
      for (int n = 0; n < steps; ++n) {
        read.next_k();
        read.next_v();
      }
    };
    // Rows behind a pool tile's end are copies of one that is there, and 0 * inf makes NaN of an infinity that the rows do see:
    // the quick walk's accumulators are not finite then, and the careful one takes these rows out.  (Bytes have no infinities.)
    auto take_copies = [&](int s, unsigned v) DBSA_INLINE {
      const int ln = lane_here(), len = (recall(s).len & 0xFFFF) - (s % kSteps) * kBN;
#pragma unroll
      for (int i = 0; i < C::kLoads; ++i) {
        const int row = piece_row(i, 64 * wave + ln);
        if (is_v(i) && row >= len) *reinterpret_cast<lds_piece*>(static_cast<uintptr_t>(v + wave_row(i) * C::kRowBytes + ln * 16)) = uintx4{0, 0, 0, 0};
      }
    };
    // step by step, nothing ahead
    auto walk_carefully = [&]() DBSA_INLINE {
      begin_walk();
      for (int st = 0; st < steps; ++st) {
        request(st);
        wait_vmcnt<0>();
        put(st);
        if constexpr (C::kDirect) {
          if (st < pool_steps && ((partly >> (st % 32)) & 1)) take_copies(st, read.v);
        }
        barrier();
        static_for<kB>([&](auto KB) DBSA_INLINE { run(KB, kNone, kNone); });
        softmax(std::true_type{}, st);
        if (st >= pool_steps && ((partly >> (st % 32)) & 1)) add_poison(st);
        product_fence(acc);
        static_for<kB>([&](auto KB) DBSA_INLINE { run(kNone, KB, kNone); });
        product_fence(acc);
        read.next_k();
        read.next_v();
        barrier();
      }
    };
    if (steps > 0) {
      if (wave * 32 < n_tok * r) walk();
      else walk_idle();
      // (behind this barrier every wave is done with the stages: the next walk's first steps may land)
      uint32_t* const votes = reinterpret_cast<uint32_t*>(smem + C::kVotesAt);
      const uint32_t any = __builtin_amdgcn_ballot_w64(again) != 0, far = __builtin_amdgcn_ballot_w64(beyond) != 0;
      if (lane == 0) votes[wave] = any | 2 * far;
      barrier();
      uint32_t all = 0;
#pragma unroll
      for (int i = 0; i < kNW; ++i) all |= votes[i];
      all = __builtin_amdgcn_readfirstlane(static_cast<int>(all));
      if (__builtin_expect(all != 0, 0)) {
        barrier();
        if (all & 2) shrink = __builtin_exp2f(-kShrink);
        walk_carefully();
        if (all & 2) m += kShrink;
      }
    } else {
      m = -INFINITY;
      l = 0.f;
#pragma unroll
      for (int ob = 0; ob < kO; ++ob)
#pragma unroll
        for (int i = 0; i < 16; ++i) acc[ob][i] = 0.f;
    }

    // ---- what the record leaves ----
    const float sum = half_swap_sum(l);
    const int row_head = hk * r + row_index % r;
    if (!row_ok) {
    } else if (part_base >= 0) {
      float* const out = p.partial + (static_cast<int64_t>(part_base + row_in) * p.n_q_heads + row_head) * (kD + kPartialPad);
#pragma unroll
      for (int ob = 0; ob < kO; ++ob)
#pragma unroll
        for (int g = 0; g < 4; ++g)
          *reinterpret_cast<floatx4*>(out + 32 * ob + 8 * g + 4 * half) =
              floatx4{acc[ob][4 * g], acc[ob][4 * g + 1], acc[ob][4 * g + 2], acc[ob][4 * g + 3]};
      if (half == 0) *reinterpret_cast<floatx2*>(out + kD) = floatx2{m, sum};
    } else {
      // (A row that saw no key is zero.  The values' scale comes behind the division: over a large sum a small one would lose its bits.)
      const bool any_key = sum > 0.f || sum != sum;
      const float inv = any_key ? 1.f / sum : 0.f, v_scale = kEs == 1 && any_key ? p.v_scale[hk] : 1.f;
      Q* const out = static_cast<Q*>(const_cast<void*>(p.o.ptr)) + row_tok * p.o.stride_tok + row_head * p.o.stride_head;
#pragma unroll
      for (int ob = 0; ob < kO; ++ob)
#pragma unroll
        for (int g = 0; g < 4; ++g) {
          typedef Q four __attribute__((ext_vector_type(4)));
          *reinterpret_cast<four*>(out + 32 * ob + 8 * g + 4 * half) =
              four{static_cast<Q>(acc[ob][4 * g] * inv * v_scale), static_cast<Q>(acc[ob][4 * g + 1] * inv * v_scale),
                   static_cast<Q>(acc[ob][4 * g + 2] * inv * v_scale), static_cast<Q>(acc[ob][4 * g + 3] * inv * v_scale)};
        }
      if (p.lse && half == 0) p.lse[static_cast<int64_t>(row_head) * p.n_rows + row_tok] = (m + __builtin_amdgcn_logf(sum)) * 0.6931471805599453f;
    }
  }
}

// Joins the partial states of one (token, query head): m* = max m_s, o = sum acc_s 2^(m_s - m*) / sum l_s 2^(m_s - m*).  Memory
// bound (100 MB of states of 512 tokens and 32 heads: 22 us), and for few tokens bound by its chain of loads (the token, its
// states, their maxima, their rows: 6 us): sixteen lanes take a pair, kD / 16 channels each, the maxima and sums are read with
// one state per lane, and four rows are in flight.  (A wave to a pair, one row in flight: 26 us.)
template <typename Q, int kD>
__global__ __launch_bounds__(256) void chunk_merge_kernel(ChunkParams p) {
  constexpr int kRow = kD + kPartialPad, kPer = kD / 16, kTeam = 16;
  const int in = threadIdx.x % kTeam;
  const int64_t pair = static_cast<int64_t>(blockIdx.x) * (256 / kTeam) + threadIdx.x / kTeam;
  if (pair >= static_cast<int64_t>(p.n_merge) * p.n_q_heads) return;  // (whole teams, which exchange among themselves alone)
  const int at = static_cast<int>(pair / p.n_q_heads), head = static_cast<int>(pair % p.n_q_heads);
  const int tok = p.merge[3 * static_cast<int64_t>(at)], n = p.merge[3 * static_cast<int64_t>(at) + 2];
  const int32_t* const parts = p.tok_part + p.merge[3 * static_cast<int64_t>(at) + 1];
  const float* const base = p.partial + static_cast<int64_t>(head) * kRow;
  const int64_t stride = static_cast<int64_t>(p.n_q_heads) * kRow;
  float m = -INFINITY;
  for (int i = in; i < n; i += kTeam) m = fmaxf(m, base[parts[i] * stride + kD]);
#pragma unroll
  for (int o = kTeam / 2; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor(m, o, kTeam));
  // (weights below 1 / n: n states of the largest values add up to no more than one)
  const float below = __builtin_exp2f(static_cast<float>(__builtin_clz(n) - 32));
  float sum = 0.f;
  floatx4 acc[kPer / 4] = {};
  for (int first = 0; first < n; first += kTeam) {
    const int part = parts[min(first + in, n - 1)];  // (behind the last: the last again, with nothing as its weight)
    float weight = 0.f;
    if (first + in < n) {
      const floatx2 ml = *reinterpret_cast<const floatx2*>(base + part * stride + kD);
      weight = ml[0] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(ml[0] - m) * below;
      sum = fmaf(ml[1], weight, sum);
    }
    const int here = min(kTeam, n - first);
    for (int i = 0; i < here; i += 4) {
      floatx4 x[4][kPer / 4];
      float w[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int from = min(i + j, here - 1);
        const float* const row = base + __shfl(part, from, kTeam) * stride + in * kPer;
        w[j] = i + j < here ? __shfl(weight, from, kTeam) : 0.f;
#pragma unroll
        for (int e = 0; e < kPer / 4; ++e) x[j][e] = *reinterpret_cast<const floatx4*>(row + 4 * e);
      }
#pragma unroll
      for (int j = 0; j < 4; ++j)
        if (i + j < here) {  // (a state's rows may hold what is not finite)
#pragma unroll
          for (int e = 0; e < kPer / 4; ++e)
#pragma unroll
            for (int f = 0; f < 4; ++f) acc[e][f] = fmaf(x[j][e][f], w[j], acc[e][f]);
        }
    }
  }
#pragma unroll
  for (int o = kTeam / 2; o > 0; o >>= 1) sum += __shfl_xor(sum, o, kTeam);
  const bool any_key = sum > 0.f || sum != sum;
  const float inv = any_key ? 1.f / sum : 0.f, v_scale = any_key && p.v_scale ? p.v_scale[head / (p.n_q_heads / p.n_kv_heads)] : 1.f;
  Q* const out = static_cast<Q*>(const_cast<void*>(p.o.ptr)) + tok * p.o.stride_tok + head * p.o.stride_head + in * kPer;
  typedef Q four __attribute__((ext_vector_type(4)));
#pragma unroll
  for (int e = 0; e < kPer / 4; ++e)
    *reinterpret_cast<four*>(out + 4 * e) = four{static_cast<Q>(acc[e][0] * inv * v_scale), static_cast<Q>(acc[e][1] * inv * v_scale),
                                                 static_cast<Q>(acc[e][2] * inv * v_scale), static_cast<Q>(acc[e][3] * inv * v_scale)};
  if (p.lse && in == 0) p.lse[static_cast<int64_t>(head) * p.n_rows + tok] = (m + __builtin_amdgcn_logf(sum / below)) * 0.6931471805599453f;
}

template <typename T, int kD, int kNW, int kBN>
hipError_t launch_shape(const ChunkParams& p, hipStream_t stream) {
  typedef Chunk<T, kD, kNW, kBN> C;
  const void* const f = reinterpret_cast<const void*>(chunk_attn_kernel<T, kD, kNW, kBN>);
  static std::atomic<bool> attr_set{false};  // setting it twice from two threads is harmless
  if (!attr_set) {
    const hipError_t e = hipFuncSetAttribute(f, hipFuncAttributeMaxDynamicSharedMemorySize, C::kLds);
    if (e != hipSuccess) return e;
    attr_set = true;
  }
  chunk_attn_kernel<T, kD, kNW, kBN><<<dim3(static_cast<unsigned>(p.n_workers) * p.n_kv_heads), dim3(C::kThreads), C::kLds, stream>>>(p);
  return hipGetLastError();
}

template <typename T, int kD>
hipError_t launch_kind(const ChunkParams& p, hipStream_t stream) {
  constexpr int kWide = Kind<T>::kBytes == 4 ? 32 : 64;
  hipError_t e = hipErrorInvalidValue;
  if (p.rows == 128) e = launch_shape<T, kD, 4, 32>(p, stream);
  else if (p.rows == 256) e = launch_shape<T, kD, 8, kWide>(p, stream);
  if (e != hipSuccess || p.n_merge == 0) return e;
  const int64_t pairs = static_cast<int64_t>(p.n_merge) * p.n_q_heads;
  chunk_merge_kernel<typename Kind<T>::Q, kD><<<dim3(static_cast<unsigned>((pairs + 15) / 16)), dim3(256), 0, stream>>>(p);
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
