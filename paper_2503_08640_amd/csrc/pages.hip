// Pages of the caches that the chunk attention reads: sharing, making room, giving back, tidying up, copying.  The books (page
// table, counts of the entries that name a page, lengths) are the caller's arrays; a page is free while its count is not above 0.
// These calls move little and are bound by the launch and by chains of loads, the copies by memory: 1.07 GB moved by a compaction in 8
// layers 215 us with its plan (5.0 TB/s, what a large copy reaches), 48 shared last pages in 16 layers 40 us (196 MB, three caches in
// turn; 32 with one, partly from the last-level cache).
#include <cstdint>

#include "kernels.hpp"

namespace {

typedef unsigned uintx4 __attribute__((ext_vector_type(4)));
typedef int intx4 __attribute__((ext_vector_type(4)));

__device__ inline bool is_page(int entry, const BookParams& p) { return entry >= 0 && entry < p.n_pages; }

__device__ inline int pages_for(int64_t tokens, const BookParams& p) {
  return static_cast<int>((tokens + (int64_t{1} << p.page_log2) - 1) >> p.page_log2);
}
// Pages of a row with so many tokens, as far as the row reaches.
__device__ inline int pages_used(int length, const BookParams& p) {
  return length < 0 ? 0 : min(pages_for(length, p), p.table_stride);
}

// ---- fork ------------------------------------------------------------------------------------------------------

constexpr int kForkEach = 8;  // entries of a thread

// A workgroup takes 2^columns_log2 columns of all rows: what the copies read of a column is in registers before any row of that
// column is written, so that rows may go round in a circle.  The counts are nearly half of its time (device-wide integer atomics; their
// order does not matter), so that an entry's whole change is one: the copies made of its row less the row's own loss of it.
// alone: the one workgroup of the launch, which sees to the lengths as well.  512 rows of 375 pages, half of them forked: 9.0 us with 8
// columns to a workgroup (12.5 with 16; before that 18 with a change for the loss and one for the copy, 71 with the loads one after the
// other), 8 rows of 57 pages 2.4.  One change for neighbours that name the same page, a thread having eight rows in a column, gained
// 1 us of 13 in beams that share most pages and lost as much in rows that share none and in small tables.
__global__ __launch_bounds__(1024) void pages_fork_kernel(BookParams p, const int32_t* source, int columns_log2, bool alone) {
  __shared__ int length_sh[kBookQuestions];
  __shared__ int copies_sh[kBookQuestions];       // copies made of the row
  __shared__ uint16_t source_sh[kBookQuestions];  // kStays: the row stays as it is
  constexpr uint16_t kStays = 0xffff;
  const int tid = threadIdx.x;
  for (int u = tid; u < p.n_queries; u += 1024) {
    const int s = source[u];
    copies_sh[u] = 0;
    length_sh[u] = p.self_len[u];
    source_sh[u] = s >= 0 && s < p.n_queries && s != u ? static_cast<uint16_t>(s) : kStays;
  }
  __syncthreads();
  for (int u = tid; u < p.n_queries; u += 1024)
    if (source_sh[u] != kStays) atomicAdd(&copies_sh[source_sh[u]], 1);
  __syncthreads();
  const int c = (blockIdx.x << columns_log2) + (tid & ((1 << columns_log2) - 1)), first = tid >> columns_log2, step = 1024 >> columns_log2;
  int old[kForkEach], now[kForkEach];
#pragma unroll
  for (int i = 0; i < kForkEach; ++i) {
    const int u = first + i * step;
    old[i] = now[i] = -1;
    if (u >= p.n_queries || c >= p.table_stride) continue;
    const int s = source_sh[u];
    if (s != kStays || copies_sh[u] > 0) old[i] = p.table[static_cast<int64_t>(u) * p.table_stride + c];
    if (s != kStays && c < pages_used(length_sh[s], p)) now[i] = p.table[static_cast<int64_t>(s) * p.table_stride + c];
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < kForkEach; ++i) {
    const int u = first + i * step;
    if (u >= p.n_queries || c >= p.table_stride) continue;
    const bool forks = source_sh[u] != kStays;
    const int change = (c < pages_used(length_sh[u], p) ? copies_sh[u] : 0) - forks;
    if (is_page(old[i], p) && change != 0) atomicAdd(p.refs + old[i], change);
    if (!is_page(now[i], p)) now[i] = -1;
    if (forks && now[i] != old[i]) p.table[static_cast<int64_t>(u) * p.table_stride + c] = now[i];
  }
  if (alone && tid < p.n_queries && source_sh[tid] != kStays) p.self_len[tid] = length_sh[source_sh[tid]];
}

__global__ __launch_bounds__(1024) void pages_fork_lengths_kernel(BookParams p, const int32_t* source) {
  __shared__ int length_sh[kBookQuestions];
  for (int u = threadIdx.x; u < p.n_queries; u += 1024) length_sh[u] = p.self_len[u];
  __syncthreads();
  for (int u = threadIdx.x; u < p.n_queries; u += 1024) {
    const int s = source[u];
    if (s >= 0 && s < p.n_queries && s != u) p.self_len[u] = length_sh[s];
  }
}

// ---- what one workgroup of 1024 threads shares -----------------------------------------------------------------

// Exclusive prefix over the workgroup, and the total.
__device__ inline uint64_t scan1024(uint64_t v, uint64_t& total) {
  __shared__ uint64_t part[16];
  const int lane = threadIdx.x % 64, wave = threadIdx.x / 64;
  uint64_t up = v;
#pragma unroll
  for (int s = 1; s < 64; s <<= 1) {
    const uint64_t other = __shfl_up(up, s);
    if (lane >= s) up += other;
  }
  __syncthreads();
  if (lane == 63) part[wave] = up;
  __syncthreads();
  // (a wave adds the sixteen up by its lanes: kept apart in every thread they take its registers)
  uint64_t sum = lane < 16 ? part[lane] : 0;
#pragma unroll
  for (int s = 1; s < 16; s <<= 1) {
    const uint64_t other = __shfl_up(sum, s);
    if (lane >= s) sum += other;
  }
  total = __shfl(sum, 15);
  return (wave > 0 ? __shfl(sum, wave - 1) : 0) + up - v;
}

// Counts of the kEach pages from the first-th on; those behind the last count as used.
template <int kEach>
__device__ inline void refs_of(const BookParams& p, int64_t first, int (&r)[kEach]) {
  if (first + kEach <= p.n_pages && reinterpret_cast<uintptr_t>(p.refs) % 16 == 0) {
#pragma unroll
    for (int e = 0; e < kEach; e += 4) {
      const intx4 v = *reinterpret_cast<const intx4*>(p.refs + first + e);
#pragma unroll
      for (int k = 0; k < 4; ++k) r[e + k] = v[k];
    }
  } else {
#pragma unroll
    for (int e = 0; e < kEach; ++e) r[e] = first + e < p.n_pages ? p.refs[first + e] : INT32_MAX;
  }
}
template <int kEach>
__device__ inline unsigned free_of(const int (&r)[kEach]) {
  unsigned free = 0;
#pragma unroll
  for (int e = 0; e < kEach; ++e) free |= (r[e] <= 0 ? 1u : 0u) << e;
  return free;
}

// ---- reserve ---------------------------------------------------------------------------------------------------

// What question u asks for.
struct Ask {
  int64_t tokens;
  int rows;           // of its last page that are in use
  int tail;           // that page, -1 if it is whole
  int first, behind;  // pages the new tokens reach into, behind the last one in use
  bool fits;
};
__device__ inline Ask ask_of(const BookParams& p, int length, int add, int u) {
  Ask a;
  const int64_t n = length < 0 ? 0 : length, more = add;
  a.tokens = n;
  a.rows = static_cast<int>(n & ((int64_t{1} << p.page_log2) - 1));
  a.tail = -1;
  a.fits = more > 0 && n + more <= static_cast<int64_t>(p.table_stride) << p.page_log2 && n + more <= INT32_MAX;
  a.first = a.behind = 0;
  if (a.fits) {
    a.first = pages_for(n, p);
    a.behind = pages_for(n + more, p);
    if (a.rows) {
      a.tail = p.table[static_cast<int64_t>(u) * p.table_stride + (n >> p.page_log2)];
      if (!is_page(a.tail, p)) {
        a.tail = -1;
        a.fits = false;
      }
    }
  }
  if (!a.fits) a.behind = a.first;
  return a;
}

constexpr int kNarrow = 4;     // entries that the thread of a question looks at by itself; more: sixteen lanes
constexpr int kSpareSh = 8192; // free pages that are kept in LDS

// One workgroup, in the order of the questions, kQ of them to a thread: what each asks for, the pages it gets, the books.  A chain
// of loads (lengths, entries, counts of the last pages); the first 8192 counts are asked for in front of it.  64 questions with 48
// replacements 8 us, 128 prompts of 450 to 900 tokens in pages of 16 (5500 pages out of 32768) 11.4 (64 with a question after the other).
// Counts are looked through from page 0 on, 8192 with a scan: a page for each of 128 questions 6.9 us in an arena of 8192 pages, 10.8 of
// 32768 and 42 of 262144 with the first four fifths in use.
template <int kQ>
__global__ __launch_bounds__(1024) void pages_reserve_kernel(BookParams p, const int32_t* add, int32_t* got, int32_t* copies,
                                                            int32_t* n_copies, int32_t* spare) {
  constexpr int kEach = 8;
  __shared__ __align__(16) int tail_sh[1024 * kQ];  // the last page that question u would write to, -1 if none
  __shared__ int lacks_sh[1024 * kQ];               // wide questions: entries that name no page yet; then, where their pages begin
  __shared__ uint16_t wide_sh[1024 * kQ];           // questions with many entries to look at, and which
  __shared__ int wide_first_sh[1024 * kQ], wide_behind_sh[1024 * kQ];
  __shared__ int spare_sh[kSpareSh];
  __shared__ int wide_count_sh;
  __shared__ bool shared_sh;
  const int tid = threadIdx.x, lane = tid % 64;
  int r[kEach];
  refs_of<kEach>(p, static_cast<int64_t>(tid) * kEach, r);
  if (tid == 0) {
    wide_count_sh = 0;
    shared_sh = false;
  }
  // An entry behind the tokens lacks a page of the question's own if it names none, or one that others name too.  Those are given back
  // below, all that were shared as the call began, so that the order does not matter: until then the workspace keeps which pages are.
  auto shared = [&](int page) {
    const bool several = p.refs[page] > 1;
    spare[page] = several;
    if (several) shared_sh = true;
    return several;
  };
  Ask a[kQ];
  int more[kQ], lacks[kQ];
#pragma unroll
  for (int i = 0; i < kQ; ++i) {
    const int u = tid * kQ + i;
    a[i] = Ask{};
    a[i].tail = -1;
    more[i] = lacks[i] = 0;
    if (u < p.n_queries) {
      more[i] = add[u];
      a[i] = ask_of(p, p.self_len[u], more[i], u);
    }
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < kQ; ++i) {
    const int u = tid * kQ + i, wide = a[i].behind - a[i].first;
    if (wide > 0 && wide <= kNarrow) {
      const int32_t* const row = p.table + static_cast<int64_t>(u) * p.table_stride;
      int entry[kNarrow], named = 0;
#pragma unroll
      for (int c = 0; c < kNarrow; ++c) {
        entry[c] = row[min(a[i].first + c, a[i].behind - 1)];
        named += c < wide && is_page(entry[c], p);
      }
      lacks[i] = wide - named;
      if (named) {
#pragma unroll
        for (int c = 0; c < kNarrow; ++c) lacks[i] += c < wide && is_page(entry[c], p) && shared(entry[c]);
      }
    }
    const uint64_t many = __ballot(wide > kNarrow);
    if (many) {
      int at = 0;
      if (lane == 0) at = atomicAdd(&wide_count_sh, __popcll(many));
      at = __shfl(at, 0) + __popcll(many & ((uint64_t{1} << lane) - 1));
      if (wide > kNarrow) {
        wide_sh[at] = static_cast<uint16_t>(u);
        wide_first_sh[at] = a[i].first;
        wide_behind_sh[at] = a[i].behind;
      }
    }
    tail_sh[u] = a[i].tail;
  }
  __syncthreads();
  const int n_wide = wide_count_sh;
  for (int i = tid / 16; i < n_wide; i += 64) {
    const int u = wide_sh[i], behind = wide_behind_sh[i];
    const int32_t* const row = p.table + static_cast<int64_t>(u) * p.table_stride;
    int n = 0;
    bool named = false;
#pragma unroll 2
    for (int c = wide_first_sh[i] + tid % 16; c < behind; c += 16) {
      const int lacking = !is_page(row[c], p);
      n += lacking;
      named |= !lacking;
    }
    if (named)
      for (int c = wide_first_sh[i] + tid % 16; c < behind; c += 16) n += is_page(row[c], p) && shared(row[c]);
#pragma unroll
    for (int s = 8; s > 0; s >>= 1) n += __shfl_xor(n, s);
    if (tid % 16 == 0) lacks_sh[u] = n;
  }
  __syncthreads();
  if (shared_sh) {
    auto give_back = [&](int32_t* entry) {
      const int page = *entry;
      if (!is_page(page, p) || !spare[page]) return;
      atomicAdd(p.refs + page, -1);
      *entry = -1;
    };
#pragma unroll
    for (int i = 0; i < kQ; ++i) {
      const int wide = a[i].behind - a[i].first;
      int32_t* const row = p.table + static_cast<int64_t>(tid * kQ + i) * p.table_stride;
      if (wide <= kNarrow)
#pragma unroll 1
        for (int c = a[i].first; c < a[i].behind; ++c) give_back(row + c);
    }
    for (int i = tid / 16; i < n_wide; i += 64) {
      int32_t* const row = p.table + static_cast<int64_t>(wide_sh[i]) * p.table_stride;
      for (int c = wide_first_sh[i] + tid % 16; c < wide_behind_sh[i]; c += 16) give_back(row + c);
    }
    // (the counts changed behind the first cache: done before the barrier, and nothing of before is kept behind it)
    __threadfence();
    __syncthreads();
    __threadfence();
    refs_of<kEach>(p, static_cast<int64_t>(tid) * kEach, r);
  }
  // a page that several name is replaced while, behind the replacements of earlier questions, more than one still does
  bool replaced[kQ];
#pragma unroll
  for (int i = 0; i < kQ; ++i) {
    const int u = tid * kQ + i, tail = a[i].tail;
    const int count = tail >= 0 ? p.refs[tail] : 0;
    int before = 0;
    if (count > 1) {
      int v = 0;
#pragma unroll 2
      for (; v + 4 <= u; v += 4) {
        const intx4 t = *reinterpret_cast<const intx4*>(tail_sh + v);
        before += (t[0] == tail) + (t[1] == tail) + (t[2] == tail) + (t[3] == tail);
      }
#pragma unroll 1
      for (; v < u; ++v) before += tail_sh[v] == tail;
    }
    replaced[i] = count - before > 1;
  }
  constexpr uint64_t kOne = (uint64_t{1} << 48) + 1, low = (uint64_t{1} << 48) - 1;
  uint64_t asks = 0;  // pages, and in the upper sixteen bits replacements, of this thread's questions
#pragma unroll
  for (int i = 0; i < kQ; ++i) {
    if (a[i].behind - a[i].first > kNarrow) lacks[i] = lacks_sh[tid * kQ + i];
    asks += lacks[i] + (replaced[i] ? kOne : 0);
  }
  uint64_t all, mine = scan1024(asks, all);
  const uint64_t total = all & low;
  // the lowest free pages
  uint64_t found = 0;
  for (int64_t base = 0; base < p.n_pages && found < total; base += 1024 * kEach) {
    const unsigned free = free_of(r);
    const int64_t first = base + static_cast<int64_t>(tid) * kEach;
    if (base + 1024 * kEach < p.n_pages) refs_of<kEach>(p, first + 1024 * kEach, r);
    uint64_t here, at = found + scan1024(__popc(free), here);
#pragma unroll 1
    for (unsigned left = free; left && at < total; left &= left - 1, ++at) {
      const int page = static_cast<int>(first) + __builtin_ctz(left);
      if (at < kSpareSh) spare_sh[at] = page;
      else spare[at] = page;
    }
    found += here;
  }
  __syncthreads();
  auto spare_at = [&](uint64_t i) { return i < kSpareSh ? spare_sh[i] : spare[i]; };
  // in order, as long as they last
  int copied = 0;
#pragma unroll
  for (int i = 0; i < kQ; ++i) {
    const int u = tid * kQ + i, wide = a[i].behind - a[i].first;
    uint64_t at = mine & low;
    const bool served = at + lacks[i] + replaced[i] <= found;
    if (u < p.n_queries) {
      got[u] = a[i].fits && served ? more[i] : 0;
      if (a[i].fits && served) p.self_len[u] = static_cast<int>(a[i].tokens + more[i]);
    }
    int32_t* const row = p.table + static_cast<int64_t>(u) * p.table_stride;
    if (served && replaced[i]) {
      const int page = spare_at(at++), number = static_cast<int>(mine >> 48);
      copies[3 * number] = a[i].tail;
      copies[3 * number + 1] = page;
      copies[3 * number + 2] = a[i].rows;
      ++copied;
      atomicAdd(p.refs + a[i].tail, -1);
      p.refs[page] = 1;
      row[a[i].tokens >> p.page_log2] = page;
    }
    if (wide > kNarrow) {
      lacks_sh[u] = served ? static_cast<int>(at) : -1;
    } else if (served && lacks[i] > 0) {
#pragma unroll 1
      for (int c = a[i].first; c < a[i].behind; ++c) {
        if (is_page(row[c], p)) continue;
        const int page = spare_at(at++);
        row[c] = page;
        p.refs[page] = 1;
      }
    }
    mine += lacks[i] + (replaced[i] ? kOne : 0);
  }
  uint64_t all_copied;
  scan1024(static_cast<uint64_t>(copied), all_copied);  // (and a barrier)
  if (tid == 0) *n_copies = static_cast<int>(all_copied);
  for (int i = tid / 16; i < n_wide; i += 64) {
    const int u = wide_sh[i], behind = wide_behind_sh[i], in = tid % 16, from = lane & 48;
    if (lacks_sh[u] < 0) continue;
    uint64_t at = static_cast<unsigned>(lacks_sh[u]);
    int32_t* const row = p.table + static_cast<int64_t>(u) * p.table_stride;
    int next = row[min(wide_first_sh[i] + in, behind - 1)];
#pragma unroll 1
    for (int c = wide_first_sh[i]; c < behind; c += 16) {
      const bool lacking = c + in < behind && !is_page(next, p);
      next = row[min(c + 16 + in, behind - 1)];
      const unsigned which = static_cast<unsigned>(__ballot(lacking) >> from) & 0xffffu;
      if (lacking) {
        const int page = spare_at(at + __popc(which & ((1u << in) - 1)));
        row[c + in] = page;
        p.refs[page] = 1;
      }
      at += __popc(which);
    }
  }
}

// ---- trim ------------------------------------------------------------------------------------------------------

// Four entries to a thread: 512 rows of 2048 entries, 91000 pages given back, 7.9 us (their atomics), 16 rows of 256 2.3.
__global__ __launch_bounds__(256) void pages_trim_kernel(BookParams p) {
  const int per_row = (p.table_stride + 1023) / 1024;
  const int u = blockIdx.x / per_row, first = (blockIdx.x % per_row) * 1024 + threadIdx.x;
  const int keep = pages_used(p.self_len[u], p);
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const int c = first + 256 * e;
    if (c < keep || c >= p.table_stride) continue;
    int32_t* const entry = p.table + static_cast<int64_t>(u) * p.table_stride + c;
    if (!is_page(*entry, p)) continue;
    atomicAdd(p.refs + *entry, -1);
    *entry = -1;
  }
}

// ---- compact ---------------------------------------------------------------------------------------------------

constexpr int kMovesSh = 4096;    // moves that are kept in LDS
constexpr int kChunksSh = 16;     // chunks of which the pages in use are kept there
constexpr int kRenameHere = 32768;  // entries that the one workgroup renames itself

// One workgroup: with L pages in use, those at L and behind go, in order, to the free ones before L.  160 pages 4.9 us, 1024 with a
// table of 128 rows of 64 entries 9.4.
template <int kEach>
__global__ __launch_bounds__(1024) void pages_compact_kernel(BookParams p, int32_t* copies, int32_t* counts, int32_t* new_place, bool renames) {
  constexpr int kChunk = 1024 * kEach;
  __shared__ uint16_t free_sh[kChunksSh][1024];
  __shared__ int from_sh[kMovesSh], to_sh[kMovesSh];
  const int tid = threadIdx.x;
  auto free_at = [&](int64_t base) {
    int r[kEach];
    refs_of<kEach>(p, base + static_cast<int64_t>(tid) * kEach, r);
    return free_of(r);
  };
  uint64_t used = 0, live;
#pragma unroll 2
  for (int64_t base = 0; base < p.n_pages; base += kChunk) {
    const unsigned free = free_at(base);
    const int64_t left = p.n_pages - base - static_cast<int64_t>(tid) * kEach;
    used += left <= 0 ? 0 : (left < kEach ? left : kEach) - __popc(free);
    if (base / kChunk < kChunksSh) free_sh[base / kChunk][tid] = static_cast<uint16_t>(free);
  }
  scan1024(used, live);
  uint64_t holes = 0, moves = 0;
  for (int64_t base = 0; base < p.n_pages; base += kChunk) {
    const int64_t first = base + static_cast<int64_t>(tid) * kEach;
    const unsigned free = base / kChunk < kChunksSh ? free_sh[base / kChunk][tid] : free_at(base);
    const int there = static_cast<int>(first >= p.n_pages ? 0 : p.n_pages - first < kEach ? p.n_pages - first : kEach);
    const int front = static_cast<int>(static_cast<int64_t>(live) <= first ? 0 : static_cast<int64_t>(live) - first < there ? static_cast<int64_t>(live) - first : there);
    const unsigned in_front = (1u << front) - 1, hole = free & in_front, move = ~free & ((1u << there) - 1) & ~in_front;
    uint64_t all;
    const uint64_t mine = scan1024(static_cast<uint64_t>(__popc(hole)) | static_cast<uint64_t>(__popc(move)) << 32, all);
    uint64_t h = holes + (mine & 0xffffffffu), m = moves + (mine >> 32);
    int place[kEach];
#pragma unroll
    for (int e = 0; e < kEach; ++e) {
      const int page = static_cast<int>(first + e);
      place[e] = free >> e & 1 ? -1 : page;
      if (hole >> e & 1) {
        if (h < kMovesSh) to_sh[h] = page;
        copies[3 * h++ + 1] = page;
      }
      if (move >> e & 1) {
        if (m < kMovesSh) from_sh[m] = page;
        copies[3 * m++] = page;
      }
    }
    if (there == kEach && reinterpret_cast<uintptr_t>(new_place) % 16 == 0) {
#pragma unroll
      for (int e = 0; e < kEach; e += 4) *reinterpret_cast<intx4*>(new_place + first + e) = intx4{place[e], place[e + 1], place[e + 2], place[e + 3]};
    } else {
      for (int e = 0; e < there; ++e) new_place[first + e] = free >> e & 1 ? -1 : static_cast<int>(first + e);
    }
    holes += all & 0xffffffffu;
    moves += all >> 32;
  }
  __syncthreads();
  for (uint64_t i = tid; i < moves; i += 1024) {
    const int from = i < kMovesSh ? from_sh[i] : copies[3 * i], to = i < kMovesSh ? to_sh[i] : copies[3 * i + 1];
    copies[3 * i + 2] = 1 << p.page_log2;
    p.refs[to] = p.refs[from];
    p.refs[from] = 0;
    new_place[from] = to;
  }
  if (tid == 0) {
    counts[0] = static_cast<int>(moves);
    counts[1] = static_cast<int>(live);
  }
  if (!renames) return;
  __syncthreads();
  const int entries = p.n_queries * p.table_stride;
#pragma unroll 4
  for (int i = tid; i < entries; i += 1024) {
    const int entry = p.table[i];
    if (is_page(entry, p)) p.table[i] = new_place[entry];
  }
}

__global__ __launch_bounds__(256) void pages_rename_kernel(BookParams p, const int32_t* new_place) {
  const int64_t entries = static_cast<int64_t>(p.n_queries) * p.table_stride, step = static_cast<int64_t>(gridDim.x) * 256;
  for (int64_t i = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x; i < entries; i += step) {
    const int entry = p.table[i];
    if (is_page(entry, p)) p.table[i] = new_place[entry];
  }
}

// ---- copy ------------------------------------------------------------------------------------------------------

constexpr int kSlice = 2048;  // 16-byte units that a workgroup copies at a time

// Workgroups walk (copy, layer, K or V, slice of the page); the copies that do not count end a walk.
__global__ __launch_bounds__(256) void pages_copy_kernel(PagesCopyParams p) {
  const int count = min(max(*p.n_copies, 0), p.max_copies);
  const int units = (p.page_tokens * p.heads) << p.row_log2;
  const int slices = (units + kSlice - 1) / kSlice;
  const int64_t per_copy = static_cast<int64_t>(p.n_layers) * 2 * slices, all = count * per_copy;
  for (int64_t item = blockIdx.x; item < all; item += gridDim.x) {
    const int64_t copy = item / per_copy;
    const int rest = static_cast<int>(item % per_copy), slice = rest % slices, plane = rest / slices;
    const int from = p.copies[3 * copy], to = p.copies[3 * copy + 1], rows = min(p.copies[3 * copy + 2], p.page_tokens);
    if (from < 0 || from >= p.n_pages || to < 0 || to >= p.n_pages || from == to || rows <= 0) continue;
    const TensorView& view = plane & 1 ? p.v : p.k;
    char* const base = static_cast<char*>(const_cast<void*>(view.ptr)) + (plane >> 1) * p.stride_layer * p.elem_bytes;
    const char* const src = base + from * p.stride_page * p.elem_bytes;
    char* const dst = base + to * p.stride_page * p.elem_bytes;
    const int n = (rows * p.heads) << p.row_log2;
    uintx4 part[kSlice / 256];
    int64_t at[kSlice / 256];
#pragma unroll
    for (int e = 0; e < kSlice / 256; ++e) {
      const int unit = slice * kSlice + e * 256 + static_cast<int>(threadIdx.x);
      if (p.flat) {
        at[e] = static_cast<int64_t>(unit) * 16;
      } else {
        const int row = unit >> p.row_log2;
        at[e] = ((row / p.heads) * view.stride_tok + (row % p.heads) * view.stride_head) * p.elem_bytes + (unit & ((1 << p.row_log2) - 1)) * 16;
      }
      if (unit < n) part[e] = *reinterpret_cast<const uintx4*>(src + at[e]);
    }
#pragma unroll
    for (int e = 0; e < kSlice / 256; ++e)
      if (slice * kSlice + e * 256 + static_cast<int>(threadIdx.x) < n) *reinterpret_cast<uintx4*>(dst + at[e]) = part[e];
  }
}

}  // namespace

hipError_t launch_pages_fork(const BookParams& p, const int32_t* source, hipStream_t stream) {
  // as many columns as the workgroup's registers hold; a table that fits into one workgroup is one launch, others have 8 columns
  // to a workgroup at most, however few rows there are: the loads and atomics of a workgroup are the time.  With the lengths, of 4, 8, 16,
  // 64 and any columns: 512 rows of 1024 entries, 375 in use, 11.0 10.7 14.3 14.3 14.3 us; 128 rows 5.6 5.8 6.7 13.0 13.0; 16 rows 4.3 4.3 4.5
  // 5.0 12.4; 16 rows of 4096, 2000 in use, 6.3 4.9 4.8 5.2 14.4
  int columns_log2 = 0;
  while ((1 << columns_log2) < p.table_stride && (p.n_queries << (columns_log2 + 1)) <= 1024 * kForkEach && (1 << columns_log2) < 1024) ++columns_log2;
  const bool alone = (1 << columns_log2) >= p.table_stride && p.n_queries <= 1024;
  if (!alone && columns_log2 > 3) columns_log2 = 3;
  const int blocks = (p.table_stride + (1 << columns_log2) - 1) >> columns_log2;
  pages_fork_kernel<<<dim3(blocks), dim3(1024), 0, stream>>>(p, source, columns_log2, alone);
  if (const hipError_t e = hipGetLastError(); e != hipSuccess || alone) return e;
  pages_fork_lengths_kernel<<<dim3(1), dim3(1024), 0, stream>>>(p, source);
  return hipGetLastError();
}

hipError_t launch_pages_reserve(const BookParams& p, const int32_t* add, int32_t* got, int32_t* copies, int32_t* n_copies, int32_t* spare,
                                hipStream_t stream) {
  if (p.n_queries <= 1024) pages_reserve_kernel<1><<<dim3(1), dim3(1024), 0, stream>>>(p, add, got, copies, n_copies, spare);
  else pages_reserve_kernel<kBookQuestions / 1024><<<dim3(1), dim3(1024), 0, stream>>>(p, add, got, copies, n_copies, spare);
  return hipGetLastError();
}

hipError_t launch_pages_trim(const BookParams& p, hipStream_t stream) {
  const int64_t blocks = static_cast<int64_t>(p.n_queries) * ((p.table_stride + 1023) / 1024);
  pages_trim_kernel<<<dim3(static_cast<unsigned>(blocks)), dim3(256), 0, stream>>>(p);
  return hipGetLastError();
}

hipError_t launch_pages_compact(const BookParams& p, int32_t* copies, int32_t* counts, int32_t* new_place, hipStream_t stream) {
  const int64_t entries = static_cast<int64_t>(p.n_queries) * p.table_stride;
  const bool renames = entries <= kRenameHere;
  if (p.n_pages <= 8192) pages_compact_kernel<4><<<dim3(1), dim3(1024), 0, stream>>>(p, copies, counts, new_place, renames);
  else pages_compact_kernel<16><<<dim3(1), dim3(1024), 0, stream>>>(p, copies, counts, new_place, renames);
  if (const hipError_t e = hipGetLastError(); e != hipSuccess || renames) return e;
  const int64_t blocks = (entries + 255) / 256;
  pages_rename_kernel<<<dim3(static_cast<unsigned>(blocks < 65536 ? blocks : 65536)), dim3(256), 0, stream>>>(p, new_place);
  return hipGetLastError();
}

hipError_t launch_pages_copy(const PagesCopyParams& p, hipStream_t stream) {
  const int64_t slices = (((static_cast<int64_t>(p.page_tokens) * p.heads) << p.row_log2) + kSlice - 1) / kSlice;
  const int64_t items = slices * 2 * p.n_layers * p.max_copies;
  if (items == 0) return hipSuccess;
  pages_copy_kernel<<<dim3(static_cast<unsigned>(items < 4096 ? items : 4096)), dim3(256), 0, stream>>>(p);
  return hipGetLastError();
}
