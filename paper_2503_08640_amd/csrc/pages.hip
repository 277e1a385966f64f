// Pages of the caches that the chunk attention reads: sharing, making room, giving back, tidying up, copying.  The books (page
// table, counts of the entries that name a page, lengths) are the caller's arrays; a page is free while its count is not above 0.
// These calls move little and are bound by the launch and by chains of loads, the copies by memory.
#include <cstdint>

#include "kernels.hpp"

namespace {

typedef unsigned uintx4 __attribute__((ext_vector_type(4)));

__device__ inline bool is_page(int entry, const BookParams& p) { return entry >= 0 && entry < p.n_pages; }

// Tokens of row u, as far as the row reaches.
__device__ inline int64_t tokens_of(const BookParams& p, int u) {
  const int64_t most = static_cast<int64_t>(p.table_stride) << p.page_log2;
  const int64_t n = p.self_len[u];
  return n < 0 ? 0 : n < most ? n : most;
}
__device__ inline int pages_for(int64_t tokens, const BookParams& p) {
  return static_cast<int>((tokens + (int64_t{1} << p.page_log2) - 1) >> p.page_log2);
}

// ---- fork ------------------------------------------------------------------------------------------------------

// A workgroup takes a range of columns of all rows: what a row's copy reads of a column is in LDS before any row of that
// column is written, so that rows may go round in a circle.  Counts: integer atomics, whose order does not matter.
__global__ __launch_bounds__(256) void pages_fork_kernel(BookParams p, const int32_t* source, int columns) {
  extern __shared__ int copy_sh[];
  const int first = blockIdx.x * columns, here = min(columns, p.table_stride - first);
  const int n = p.n_queries * here;
  for (int i = threadIdx.x; i < n; i += 256) {
    const int u = i / here, c = first + i % here, s = source[u];
    if (s < 0 || s >= p.n_queries || s == u) continue;
    const int old = p.table[static_cast<int64_t>(u) * p.table_stride + c];
    int now = c < pages_for(tokens_of(p, s), p) ? p.table[static_cast<int64_t>(s) * p.table_stride + c] : -1;
    if (!is_page(now, p)) now = -1;
    copy_sh[i] = now;
    if (now != old) {
      if (is_page(old, p)) atomicAdd(p.refs + old, -1);
      if (now >= 0) atomicAdd(p.refs + now, 1);
    }
  }
  __syncthreads();
  for (int i = threadIdx.x; i < n; i += 256) {
    const int u = i / here, c = first + i % here, s = source[u];
    if (s < 0 || s >= p.n_queries || s == u) continue;
    p.table[static_cast<int64_t>(u) * p.table_stride + c] = copy_sh[i];
  }
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

// ---- reserve ---------------------------------------------------------------------------------------------------

// Exclusive prefix over the workgroup's 1024 threads, and the total.
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
  uint64_t before = 0;
  total = 0;
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    if (i < wave) before += part[i];
    total += part[i];
  }
  return before + up - v;
}

// What question u asks for.
struct Ask {
  int64_t tokens;
  int rows;           // of its last page that are in use
  int tail;           // that page, -1 if it is whole
  int first, behind;  // pages the new tokens reach into, behind the last one in use
  bool fits;
};
__device__ inline Ask ask_of(const BookParams& p, const int32_t* add, int u) {
  Ask a;
  const int64_t n = p.self_len[u] < 0 ? 0 : p.self_len[u], more = add[u];
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

// One workgroup, in the order of the questions: what each asks for, the pages it gets, the books.
__global__ __launch_bounds__(1024) void pages_reserve_kernel(BookParams p, const int32_t* add, int32_t* got, int32_t* copies,
                                                            int32_t* n_copies, int32_t* spare) {
  __shared__ int tail_sh[kBookQuestions];   // the last page that question u would write to, -1 if none
  __shared__ int lacks_sh[kBookQuestions];  // entries that name no page yet; the lowest bit: the last page is to be replaced
  __shared__ int copied_sh;
  const int tid = threadIdx.x, lane = tid % 64, wave = tid / 64;
  if (tid == 0) copied_sh = 0;
  // (a wave to a question where many entries are looked at, a thread to a question else)
  for (int base = wave * 64; base < p.n_queries; base += 1024) {
    const int u = base + lane;
    Ask a{};
    int lacks = 0;
    if (u < p.n_queries) {
      a = ask_of(p, add, u);
      tail_sh[u] = a.tail;
      if (a.behind - a.first <= 4)
        for (int c = a.first; c < a.behind; ++c) lacks += !is_page(p.table[static_cast<int64_t>(u) * p.table_stride + c], p);
    }
    uint64_t many = __ballot(u < p.n_queries && a.behind - a.first > 4);
    while (many) {
      const int who = __ffsll(static_cast<unsigned long long>(many)) - 1;
      many &= many - 1;
      const int first = __shfl(a.first, who), behind = __shfl(a.behind, who);
      int all = 0;
      for (int c = first; c < behind; c += 64)
        all += __popcll(__ballot(c + lane < behind && !is_page(p.table[static_cast<int64_t>(base + who) * p.table_stride + min(c + lane, behind - 1)], p)));
      if (lane == who) lacks = all;
    }
    if (u < p.n_queries) lacks_sh[u] = 2 * lacks;
  }
  __syncthreads();
  // a page that several name is replaced while, behind the replacements of earlier questions, more than one still does
  for (int u = tid; u < p.n_queries; u += 1024) {
    const int tail = tail_sh[u];
    if (tail < 0) continue;
    const int count = p.refs[tail];
    if (count <= 1) continue;
    int before = 0;
    for (int v = 0; v < u; ++v) before += tail_sh[v] == tail;
    if (count - before > 1) lacks_sh[u] |= 1;
  }
  __syncthreads();
  uint64_t total = 0;  // pages asked for
  for (int base = 0; base < p.n_queries; base += 1024) {
    const int u = base + tid;
    uint64_t all;
    scan1024(u < p.n_queries ? (lacks_sh[u] >> 1) + (lacks_sh[u] & 1) : 0, all);
    total += all;
  }
  // the lowest free pages
  uint64_t found = 0;
  for (int64_t base = 0; base < p.n_pages && found < total; base += 4096) {
    int free = 0;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int64_t page = base + 4 * tid + e;
      if (page < p.n_pages && p.refs[page] <= 0) free |= 1 << e;
    }
    uint64_t here;
    uint64_t at = found + scan1024(__popc(free), here);
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (free >> e & 1) {
        if (at < total) spare[at] = static_cast<int>(base + 4 * tid + e);
        ++at;
      }
    found += here;
  }
  __syncthreads();
  // in order, as long as they last
  uint64_t before = 0;
  for (int base = 0; base < p.n_queries; base += 1024) {
    const int u = base + tid;
    const bool there = u < p.n_queries;
    const int word = there ? lacks_sh[u] : 0, ask = (word >> 1) + (word & 1);
    uint64_t all;
    const uint64_t mine = before + scan1024(static_cast<uint64_t>(ask) | static_cast<uint64_t>(word & 1) << 48, all);
    before += all;
    const uint64_t low = (uint64_t{1} << 48) - 1;
    uint64_t at = mine & low;
    Ask a{};
    bool served = false;
    if (there) {
      a = ask_of(p, add, u);
      served = at + ask <= found;
      got[u] = a.fits && served ? add[u] : 0;
      if (served && (word & 1)) {
        const int page = spare[at++], number = static_cast<int>(mine >> 48);
        copies[3 * number] = a.tail;
        copies[3 * number + 1] = page;
        copies[3 * number + 2] = a.rows;
        atomicAdd(&copied_sh, 1);
        atomicAdd(p.refs + a.tail, -1);
        p.refs[page] = 1;
        p.table[static_cast<int64_t>(u) * p.table_stride + (a.tokens >> p.page_log2)] = page;
      }
      if (served && a.fits) p.self_len[u] = static_cast<int>(a.tokens + add[u]);
      if (served && a.behind - a.first <= 4) {
        for (int c = a.first; c < a.behind; ++c) {
          int32_t* const entry = p.table + static_cast<int64_t>(u) * p.table_stride + c;
          if (is_page(*entry, p)) continue;
          const int page = spare[at++];
          *entry = page;
          p.refs[page] = 1;
        }
      }
    }
    uint64_t many = __ballot(there && served && a.behind - a.first > 4);
    while (many) {
      const int who = __ffsll(static_cast<unsigned long long>(many)) - 1;
      many &= many - 1;
      const int first = __shfl(a.first, who), behind = __shfl(a.behind, who);
      uint64_t next = __shfl(at, who);
      int32_t* const row = p.table + static_cast<int64_t>(base + wave * 64 + who) * p.table_stride;
      for (int c = first; c < behind; c += 64) {
        const bool lacks = c + lane < behind && !is_page(row[min(c + lane, behind - 1)], p);
        const uint64_t which = __ballot(lacks);
        if (lacks) {
          const int page = spare[next + __popcll(which & ((uint64_t{1} << lane) - 1))];
          row[c + lane] = page;
          p.refs[page] = 1;
        }
        next += __popcll(which);
      }
    }
  }
  __syncthreads();
  if (tid == 0) *n_copies = copied_sh;
}

// ---- trim ------------------------------------------------------------------------------------------------------

__global__ __launch_bounds__(256) void pages_trim_kernel(BookParams p) {
  const int per_row = (p.table_stride + 1023) / 1024;
  const int u = blockIdx.x / per_row, first = (blockIdx.x % per_row) * 1024 + threadIdx.x;
  const int keep = pages_for(tokens_of(p, u), p);
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

// One workgroup: with L pages in use, those at L and behind go, in order, to the free ones before L.
__global__ __launch_bounds__(1024) void pages_compact_kernel(BookParams p, int32_t* copies, int32_t* counts, int32_t* new_place) {
  const int tid = threadIdx.x;
  uint64_t live = 0;
  for (int64_t base = 0; base < p.n_pages; base += 4096) {
    int here = 0;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int64_t page = base + 4 * tid + e;
      here += page < p.n_pages && p.refs[page] > 0;
    }
    uint64_t all;
    scan1024(here, all);
    live += all;
  }
  uint64_t holes = 0, moves = 0;
  for (int64_t base = 0; base < p.n_pages; base += 4096) {
    int hole = 0, move = 0;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int64_t page = base + 4 * tid + e;
      if (page >= p.n_pages) continue;
      const bool used = p.refs[page] > 0, front = static_cast<uint64_t>(page) < live;
      if (front && !used) hole |= 1 << e;
      if (!front && used) move |= 1 << e;
      new_place[page] = used ? static_cast<int>(page) : -1;
    }
    uint64_t all;
    const uint64_t mine = scan1024(static_cast<uint64_t>(__popc(hole)) | static_cast<uint64_t>(__popc(move)) << 32, all);
    uint64_t h = holes + (mine & 0xffffffffu), m = moves + (mine >> 32);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int page = static_cast<int>(base + 4 * tid + e);
      if (hole >> e & 1) copies[3 * h++ + 1] = page;
      if (move >> e & 1) copies[3 * m++] = page;
    }
    holes += all & 0xffffffffu;
    moves += all >> 32;
  }
  __syncthreads();
  for (uint64_t i = tid; i < moves; i += 1024) {
    const int from = copies[3 * i], to = copies[3 * i + 1];
    copies[3 * i + 2] = 1 << p.page_log2;
    p.refs[to] = p.refs[from];
    p.refs[from] = 0;
    new_place[from] = to;
  }
  if (tid == 0) {
    counts[0] = static_cast<int>(moves);
    counts[1] = static_cast<int>(live);
  }
}

__global__ __launch_bounds__(256) void pages_rename_kernel(BookParams p, const int32_t* new_place) {
  const int64_t i = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x;
  if (i >= static_cast<int64_t>(p.n_queries) * p.table_stride) return;
  const int entry = p.table[i];
  if (is_page(entry, p)) p.table[i] = new_place[entry];
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
  // 64 KiB of LDS hold the columns of a workgroup
  int columns = 16384 / p.n_queries;
  columns = columns > 64 ? 64 : columns;
  const int blocks = (p.table_stride + columns - 1) / columns;
  pages_fork_kernel<<<dim3(blocks), dim3(256), static_cast<size_t>(p.n_queries) * columns * 4, stream>>>(p, source, columns);
  if (const hipError_t e = hipGetLastError()) return e;
  pages_fork_lengths_kernel<<<dim3(1), dim3(1024), 0, stream>>>(p, source);
  return hipGetLastError();
}

hipError_t launch_pages_reserve(const BookParams& p, const int32_t* add, int32_t* got, int32_t* copies, int32_t* n_copies, int32_t* spare,
                                hipStream_t stream) {
  pages_reserve_kernel<<<dim3(1), dim3(1024), 0, stream>>>(p, add, got, copies, n_copies, spare);
  return hipGetLastError();
}

hipError_t launch_pages_trim(const BookParams& p, hipStream_t stream) {
  const int64_t blocks = static_cast<int64_t>(p.n_queries) * ((p.table_stride + 1023) / 1024);
  pages_trim_kernel<<<dim3(static_cast<unsigned>(blocks)), dim3(256), 0, stream>>>(p);
  return hipGetLastError();
}

hipError_t launch_pages_compact(const BookParams& p, int32_t* copies, int32_t* counts, int32_t* new_place, hipStream_t stream) {
  pages_compact_kernel<<<dim3(1), dim3(1024), 0, stream>>>(p, copies, counts, new_place);
  if (const hipError_t e = hipGetLastError()) return e;
  const int64_t entries = static_cast<int64_t>(p.n_queries) * p.table_stride;
  if (entries > 0) pages_rename_kernel<<<dim3(static_cast<unsigned>((entries + 255) / 256)), dim3(256), 0, stream>>>(p, new_place);
  return hipGetLastError();
}

hipError_t launch_pages_copy(const PagesCopyParams& p, hipStream_t stream) {
  const int64_t slices = (((static_cast<int64_t>(p.page_tokens) * p.heads) << p.row_log2) + kSlice - 1) / kSlice;
  const int64_t items = slices * 2 * p.n_layers * p.max_copies;
  if (items == 0) return hipSuccess;
  pages_copy_kernel<<<dim3(static_cast<unsigned>(items < 4096 ? items : 4096)), dim3(256), 0, stream>>>(p);
  return hipGetLastError();
}
