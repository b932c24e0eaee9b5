// The pages of a paged cache, managed on the device for gfx950 (CDNA4): sequences fork, end, grow and give
// tokens back, pages move together. Tables and counts are small and every kernel here is a chain of
// latencies; only the copies of pages are bound by the memory. For 256 sequences and 5000 pages fork's two take 2.7
// and 2.4 us, extend's 4.1 and 5.3; compact's three, for 818 pages, 1.9, 3.1 and 3.1. Each workgroup of extend's second and of
// compact's sums up all chunks' counts, and one puts extend's requests in a row: with 2^20 pages and 16384 sequences fork takes 16 us,
// extend 140 and compact 30, with 2^24 and 2^20, the most, 0.9 ms, 9.1 and 0.8.
//
// refs[p] counts the rows of the page table that hold page p (and whatever else the caller counts);
// a page of count 0 is free. A sequence of n tokens holds the first ceil(n / page size) entries of its row.
#include <hip/hip_runtime.h>

#include "cache_attn.hpp"
#include "pages.hpp"

namespace csg {
namespace {

constexpr int kThreads = 256;
constexpr int kSlots = 1024;  // entries of a row that a workgroup has

__device__ __forceinline__ void tell(int32_t* status, int bit) {
  if (status) atomicOr(status, bit);
}

// A sequence's tokens, as far as its row goes, and the entries that it holds.
struct Held {
  int tokens, pages;
  bool bad;
};
__device__ __forceinline__ Held held(const PagesArgs& a, int tokens) {
  const int room = static_cast<int>(min(static_cast<int64_t>(a.max_pages) << a.page_shift, int64_t{1} << 30));
  Held h;
  h.tokens = min(max(tokens, 0), room);
  h.bad = h.tokens != tokens;
  h.pages = (h.tokens + (1 << a.page_shift) - 1) >> a.page_shift;
  return h;
}

__device__ __forceinline__ bool names_page(const PagesArgs& a, int p) { return p >= 0 && p < a.n_pages; }
__device__ __forceinline__ void count(const PagesArgs& a, int p, int by) {
  if (names_page(a, p)) atomicAdd(a.refs_out + p, by);
}

// ---- fork ------------------------------------------------------------------------------------
__device__ __forceinline__ Held parent_of(const PagesArgs& a, int b, int* parent) {
  int p = a.change[b];
  if (p >= a.batch) {
    if (threadIdx.x == 0) tell(a.status, kCacheBadLength);
    p = -1;
  }
  *parent = p;
  return held(a, p < 0 ? 0 : a.lens[p]);
}

// Rows of the new table, and the counts as they were.
__global__ __launch_bounds__(kThreads) void fork_rows(PagesArgs a, int row_blocks, int across) {
  const int tid = threadIdx.x;
  if (static_cast<int>(blockIdx.x) >= row_blocks) {
    const int64_t p0 = static_cast<int64_t>(blockIdx.x - row_blocks) * kPageChunk;
    for (int64_t p = p0 + tid; p < min(p0 + kPageChunk, static_cast<int64_t>(a.n_pages)); p += kThreads) a.refs_out[p] = a.refs[p];
    return;
  }
  const int b = blockIdx.x / across, s0 = blockIdx.x % across * kSlots;
  int parent;
  const Held h = parent_of(a, b, &parent);
  const int32_t* from = a.table + static_cast<int64_t>(max(parent, 0)) * a.max_pages;
  int32_t* to = a.table_out + static_cast<int64_t>(b) * a.max_pages;
  for (int s = s0 + tid; s < min(s0 + kSlots, a.max_pages); s += kThreads) {
    const int p = s < h.pages ? from[s] : -1;
    if (s < h.pages && !names_page(a, p)) tell(a.status, kCacheBadPage);
    to[s] = p;
  }
  if (s0 == 0 && tid == 0) {
    a.lens_out[b] = h.tokens;
    if (h.bad) tell(a.status, kCacheBadLength);
  }
}

// The counts: less the old rows, more the new ones.
__global__ __launch_bounds__(kThreads) void fork_counts(PagesArgs a, int across) {
  const int b = blockIdx.x / across, s0 = blockIdx.x % across * kSlots;
  int parent;
  const Held now = parent_of(a, b, &parent);
  if (parent == b) return;
  const Held old = held(a, a.lens[b]);
  if (old.bad && s0 == 0 && threadIdx.x == 0) tell(a.status, kCacheBadLength);  // (fork_rows looks at lengths that are kept)
  const int64_t row = static_cast<int64_t>(b) * a.max_pages;
  for (int s = s0 + static_cast<int>(threadIdx.x); s < min(s0 + kSlots, max(old.pages, now.pages)); s += kThreads) {
    if (s < old.pages) {
      const int p = a.table[row + s];
      if (!names_page(a, p)) tell(a.status, kCacheBadPage);
      count(a, p, -1);
    }
    if (s < now.pages) count(a, a.table_out[row + s], 1);
  }
}

// ---- sums ------------------------------------------------------------------------------------
template <class V>
__device__ __forceinline__ V sum_before(V x, V* total, V (&s_wave)[kThreads / 64]) {
  // exclusive, over the workgroup's threads
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  V sum = x;
#pragma unroll
  for (int d = 1; d < 64; d *= 2) {
    const V up = __shfl_up(sum, d);
    if (lane >= d) sum += up;
  }
  __syncthreads();  // (s_wave is free)
  if (lane == 63) s_wave[wave] = sum;
  __syncthreads();
  V before = sum - x, all = 0;
#pragma unroll
  for (int w = 0; w < kThreads / 64; ++w) {
    if (w < wave) before += s_wave[w];
    all += s_wave[w];
  }
  *total = all;
  return before;
}

// The workspace of extend and compact.
struct Sums {
  int32_t used, moving;  // compact: pages in use, and how many of them move
};
__device__ __forceinline__ Sums* sums_in(const PagesArgs& a) { return reinterpret_cast<Sums*>(a.ws); }
__device__ __forceinline__ int32_t* counts_in(const PagesArgs& a) { return reinterpret_cast<int32_t*>(a.ws + 64); }
__device__ __forceinline__ int32_t* list_in(const PagesArgs& a) { return counts_in(a) + 2 * (page_chunks(a.n_pages) / 2 + 1); }
__device__ __forceinline__ int32_t* ranks_in(const PagesArgs& a) { return list_in(a) + a.n_pages; }
__device__ __forceinline__ int64_t* first_in(const PagesArgs& a) { return reinterpret_cast<int64_t*>(ranks_in(a) + a.n_pages); }
__device__ __forceinline__ int32_t* splits_in(const PagesArgs& a) { return reinterpret_cast<int32_t*>(first_in(a) + a.batch); }

constexpr int kEach = kPageChunk / kThreads;  // pages of a thread, one after the other

// Whether this thread's pages of chunk c are in use, one bit each (pages that there are not: 0), and `there`.
__device__ __forceinline__ uint32_t used_bits(const PagesArgs& a, int c, uint32_t* there) {
  const int p0 = c * kPageChunk + static_cast<int>(threadIdx.x) * kEach;
  uint32_t used = 0, is = 0;
#pragma unroll
  for (int i = 0; i < kEach; ++i) {
    const int p = p0 + i;
    if (p < a.n_pages) {
      is |= 1u << i;
      if (a.refs[p] != 0) used |= 1u << i;
    }
  }
  *there = is;
  return used;
}

// Pages in use in the chunks before `c`, and in all.
__device__ __forceinline__ int used_before(const PagesArgs& a, int c, int* all, int (&s_wave)[kThreads / 64]) {
  int before = 0, total = 0;
  for (int i = threadIdx.x; i < page_chunks(a.n_pages); i += kThreads) {
    const int n = counts_in(a)[i];
    total += n;
    if (i < c) before += n;
  }
  int sum_b, sum_t;
  sum_before(before, &sum_b, s_wave);
  sum_before(total, &sum_t, s_wave);
  *all = sum_t;
  return sum_b;
}

// ---- extend ----------------------------------------------------------------------------------
// What sequence b asks for. Its requests are places first .. first + need - 1 of the row of all requests, and request
// i takes the i-th lowest free page.
struct Growth {
  Held before, after;
  int need;
  bool split;  // the last page is to be written and not the sequence's alone: it gets a copy
  bool fits;   // (in its row)
};
__device__ __forceinline__ Growth growth_of(const PagesArgs& a, int b) {
  Growth g;
  g.before = held(a, a.lens[b]);
  const int by = a.change[b];
  const int64_t tokens = static_cast<int64_t>(g.before.tokens) + by;
  const int64_t room = min(static_cast<int64_t>(a.max_pages) << a.page_shift, int64_t{1} << 30);
  g.fits = tokens <= room;
  const int want = static_cast<int>(max(int64_t{0}, min(tokens, int64_t{1} << 30)));
  g.after.tokens = want;
  g.after.pages = (want + (1 << a.page_shift) - 1) >> a.page_shift;
  g.after.bad = tokens < 0 || !g.fits;
  g.split = false;
  if (by > 0 && (g.before.tokens & ((1 << a.page_shift) - 1)) != 0) {
    const int last = a.table[static_cast<int64_t>(b) * a.max_pages + g.before.pages - 1];
    g.split = names_page(a, last) && a.refs[last] > 1;
  }
  g.need = max(0, g.after.pages - g.before.pages) + g.split;
  return g;
}

// The chunks' pages in use, and the counts as they were; the last workgroup puts the sequences' requests in a row.
__global__ __launch_bounds__(kThreads) void extend_count(PagesArgs a) {
  __shared__ int s_wave[kThreads / 64];
  __shared__ int64_t s_wave64[kThreads / 64];
  const int chunks = page_chunks(a.n_pages), c = blockIdx.x, tid = threadIdx.x;
  if (c < chunks) {
    uint32_t there;
    const uint32_t used = used_bits(a, c, &there);
    const int64_t p0 = static_cast<int64_t>(c) * kPageChunk;
    for (int64_t p = p0 + tid; p < min(p0 + kPageChunk, static_cast<int64_t>(a.n_pages)); p += kThreads) a.refs_out[p] = a.refs[p];
    int all;
    sum_before(static_cast<int>(__popc(used)), &all, s_wave);
    if (tid == 0) counts_in(a)[c] = all;
    return;
  }
  int64_t need = 0;
  int splits = 0;
  for (int b0 = 0; b0 < a.batch; b0 += kThreads) {
    const int b = b0 + tid;
    Growth g{};
    if (b < a.batch) g = growth_of(a, b);
    int64_t all;
    const int64_t first = need + sum_before(static_cast<int64_t>(g.need), &all, s_wave64);
    need += all;
    int all_splits;
    const int split = splits + sum_before(g.split && g.fits ? 1 : 0, &all_splits, s_wave);
    splits += all_splits;
    if (b < a.batch) {
      first_in(a)[b] = first;
      splits_in(a)[b] = split;
    }
  }
  if (tid == 0) *a.n_moves = 0;
}

// Free pages before the chunks' (the workgroup's threads have one each of 256 at a time); *all: of all chunks.
// If the page of rank q is in one of them, *chunk is it, and *before the free pages before it.
__device__ __forceinline__ void find_free(const PagesArgs& a, int64_t q, int* all, int* chunk, int* before, int (&s_wave)[kThreads / 64],
                                          int (&s_found)[2]) {
  const int chunks = page_chunks(a.n_pages);
  int sum = 0;
  for (int c0 = 0; c0 < chunks; c0 += kThreads) {
    const int c = c0 + static_cast<int>(threadIdx.x);
    const int free = c < chunks ? min(kPageChunk, a.n_pages - c * kPageChunk) - counts_in(a)[c] : 0;
    int total;
    const int first = sum + sum_before(free, &total, s_wave);
    if (first <= q && q < first + free) {
      s_found[0] = c;
      s_found[1] = first;
    }
    sum += total;
  }
  __syncthreads();
  *all = sum;
  *chunk = s_found[0];
  *before = s_found[1];
}

// The new rows. A workgroup finds the free pages that its entries get itself: usually they are in one chunk.
__global__ __launch_bounds__(kThreads) void extend_rows(PagesArgs a, int across) {
  __shared__ int s_wave[kThreads / 64], s_found[2];
  __shared__ int s_new[kSlots + 1];
  const int b = blockIdx.x / across, s0 = blockIdx.x % across * kSlots, tid = threadIdx.x;
  Growth g = growth_of(a, b);
  const int last = g.before.pages - 1;
  const int64_t first = g.need > 0 ? first_in(a)[b] : 0;
  bool granted = g.fits;
  int64_t q0 = 0;
  if (g.need > 0 && g.fits) {
    // its requests: the copy's, if the entry is its own, then its new entries'
    const bool copies = g.split && last >= s0 && last < s0 + kSlots;
    const int from = max(s0, g.before.pages), count_new = max(0, min(s0 + kSlots, g.after.pages) - from);
    q0 = copies ? first : first + g.split + (from - g.before.pages);
    const int m = count_new + copies;
    int all, chunk, before;
    find_free(a, q0, &all, &chunk, &before, s_wave, s_found);
    granted = first + g.need <= all;
    if (granted) {
      for (int64_t at = before; m > 0 && at < q0 + m && chunk < page_chunks(a.n_pages); ++chunk) {
        uint32_t there;
        const uint32_t bits = ~used_bits(a, chunk, &there) & there;
        int total;
        int64_t rank = at + sum_before(static_cast<int>(__popc(bits)), &total, s_wave);
        for (int i = 0; i < kEach; ++i)
          if (bits >> i & 1) {
            if (rank >= q0 && rank < q0 + m) s_new[rank - q0] = chunk * kPageChunk + tid * kEach + i;
            ++rank;
          }
        at += total;
      }
      __syncthreads();
    } else if (s0 == 0 && tid == 0) {
      tell(a.status, kPagesNone);
    }
  }
  if (s0 == 0 && tid == 0 && (g.before.bad || g.after.bad)) tell(a.status, kCacheBadLength);
  if (!granted) {
    g.after = g.before;
    g.split = false;
  }
  const int64_t row = static_cast<int64_t>(b) * a.max_pages;
  for (int s = s0 + tid; s < min(s0 + kSlots, a.max_pages); s += kThreads) {
    const int old = s < g.before.pages ? a.table[row + s] : -1;
    if (s < g.before.pages && !names_page(a, old)) tell(a.status, kCacheBadPage);
    int now = s < g.after.pages ? old : -1;
    if (s == last && g.split) {
      now = s_new[first - q0];
      count(a, old, -1);
      count(a, now, 1);
      const int at = splits_in(a)[b];
      a.moves[2 * at] = old;
      a.moves[2 * at + 1] = now;
      atomicMax(a.n_moves, at + 1);
    } else if (s > last && s < g.after.pages) {
      now = s_new[first + g.split + (s - g.before.pages) - q0];
      count(a, now, 1);
    } else if (s < g.before.pages && s >= g.after.pages) {
      count(a, old, -1);
    }
    a.table_out[row + s] = now;
  }
  if (s0 == 0 && tid == 0) a.lens_out[b] = g.after.tokens;
}

// ---- compact ---------------------------------------------------------------------------------
// With U pages in use, those at U and beyond go, in ascending order, to the free ones before U, in ascending order.
__global__ __launch_bounds__(kThreads) void compact_count(PagesArgs a) {
  __shared__ int s_wave[kThreads / 64];
  uint32_t there;
  const uint32_t used = used_bits(a, blockIdx.x, &there);
  int all;
  sum_before(static_cast<int>(__popc(used)), &all, s_wave);
  if (threadIdx.x == 0) counts_in(a)[blockIdx.x] = all;
}

// The free pages before U by their rank, the ranks of the pages in use among all in use, and the sums.
__global__ __launch_bounds__(kThreads) void compact_list(PagesArgs a) {
  __shared__ int s_wave[kThreads / 64];
  const int c = blockIdx.x;
  int u;
  const int before = used_before(a, c, &u, s_wave);
  uint32_t there;
  const uint32_t bits = used_bits(a, c, &there);
  int all;
  int used = before + sum_before(static_cast<int>(__popc(bits)), &all, s_wave);
  if (c == 0 && threadIdx.x == 0) sums_in(a)->used = u;
  for (int i = 0; i < kEach; ++i) {
    const int p = c * kPageChunk + static_cast<int>(threadIdx.x) * kEach + i;
    if (p >= a.n_pages) break;
    if (p == u - 1) sums_in(a)->moving = u - used - (bits >> i & 1);  // the free pages before U
    if (bits >> i & 1) {
      ranks_in(a)[p] = used++;
    } else if (p < u) {
      list_in(a)[p - used] = p;
    }
  }
}

// Where a page in use lies afterwards. As many pages in use lie at U and beyond as are free before it, `moving`; the
// one of rank r among all in use is number r - (U - moving) of them.
__device__ __forceinline__ int place_of(const PagesArgs& a, int p, const Sums& sums) {
  return p < sums.used ? p : list_in(a)[sums.moving - (sums.used - ranks_in(a)[p])];
}

__global__ __launch_bounds__(kThreads) void compact_rows(PagesArgs a, int page_blocks, int across) {
  const int tid = threadIdx.x;
  const Sums sums = {sums_in(a)->used, sums_in(a)->used > 0 ? sums_in(a)->moving : 0};
  if (static_cast<int>(blockIdx.x) < page_blocks) {
    if (blockIdx.x == 0 && tid == 0) *a.n_moves = sums.moving;
    const int p = blockIdx.x * kThreads + tid;
    if (p >= a.n_pages) return;
    const int refs = a.refs[p];
    if (refs == 0) {
      a.renamed[p] = -1;
      if (p >= sums.used) a.refs_out[p] = 0;
      return;
    }
    const int to = place_of(a, p, sums);
    a.renamed[p] = to;
    a.refs_out[to] = refs;
    if (p >= sums.used) {
      const int at = sums.moving - (sums.used - ranks_in(a)[p]);
      a.refs_out[p] = 0;
      a.moves[2 * at] = p;
      a.moves[2 * at + 1] = to;
    }
    return;
  }
  const int item = blockIdx.x - page_blocks;
  const int b = item / across, s0 = item % across * kSlots;
  const Held h = held(a, a.lens[b]);
  if (h.bad && s0 == 0 && tid == 0) tell(a.status, kCacheBadLength);
  const int64_t row = static_cast<int64_t>(b) * a.max_pages;
  for (int s = s0 + tid; s < min(s0 + kSlots, a.max_pages); s += kThreads) {
    int now = -1;
    if (s < h.pages) {
      const int p = a.table[row + s];
      if (names_page(a, p) && a.refs[p] != 0)
        now = place_of(a, p, sums);
      else
        tell(a.status, kCacheBadPage);
    }
    a.table_out[row + s] = now;
  }
}

// ---- copy ------------------------------------------------------------------------------------
// Pieces of 8 KiB of the pages that move, buffer by buffer, dealt to the workgroups in turn. Bound by the memory: 1750
// pages of 128 KiB in two buffers, 917 MB of traffic, in 152 us, 6.0 TB/s (a large copy: 5.1); in pieces of 16 KiB by 8
// workgroups a CU and through the caches 203. Stores go past the caches (copies of 32 pages in eight buffers 28 us with the
// tables, through the caches 31); loads only where they cannot lie in them (the large copy gains 13 us, the small one loses 4).
typedef unsigned int u32x4_t __attribute__((ext_vector_type(4)));
constexpr int kPiece = 8192, kGroupsPerCu = 64;
constexpr int64_t kCached = int64_t{256} << 20;  // bytes that the caches hold

template <bool past>
__device__ __forceinline__ void copy_piece(const u32x4_t* src, u32x4_t* dst, int bytes) {
  constexpr int kEachThread = kPiece / 16 / kThreads;
  u32x4_t x[kEachThread];
#pragma unroll
  for (int i = 0; i < kEachThread; ++i) {
    const int k = i * kThreads + static_cast<int>(threadIdx.x);
    if (16 * k < bytes) x[i] = past ? __builtin_nontemporal_load(src + k) : src[k];
  }
#pragma unroll
  for (int i = 0; i < kEachThread; ++i) {
    const int k = i * kThreads + static_cast<int>(threadIdx.x);
    if (16 * k < bytes) __builtin_nontemporal_store(x[i], dst + k);
  }
}

__global__ __launch_bounds__(kThreads) void copy_pages(CopyArgs a) {
  const int n = min(max(*a.n_moves, 0), a.max_moves);
  const int64_t pieces = (a.page_bytes + kPiece - 1) / kPiece;
  const int64_t items = pieces * n * a.n_buffers;
  const bool past = a.page_bytes * n * a.n_buffers > kCached;
  for (int64_t item = blockIdx.x; item < items; item += gridDim.x) {
    const int64_t page = item / pieces;
    const int move = static_cast<int>(page % n), buffer = static_cast<int>(page / n);
    const int from = a.moves[2 * move], to = a.moves[2 * move + 1];
    if (from < 0 || from >= a.n_pages || to < 0 || to >= a.n_pages) {
      if (threadIdx.x == 0) tell(a.status, kCacheBadPage);
      continue;
    }
    const int64_t at = (item - page * pieces) * kPiece;
    const int bytes = static_cast<int>(min(static_cast<int64_t>(kPiece), a.page_bytes - at));
    const u32x4_t* src = reinterpret_cast<const u32x4_t*>(a.buffers[buffer] + from * a.page_bytes + at);
    u32x4_t* dst = reinterpret_cast<u32x4_t*>(a.buffers[buffer] + to * a.page_bytes + at);
    if (past)
      copy_piece<true>(src, dst, bytes);
    else
      copy_piece<false>(src, dst, bytes);
  }
}

int rows_across(const PagesArgs& a) { return (a.max_pages + kSlots - 1) / kSlots; }

}  // namespace

hipError_t launch_pages_fork(const PagesArgs& a, hipStream_t s) {
  const int across = rows_across(a), rows = a.batch * across;
  hipLaunchKernelGGL(fork_rows, dim3(rows + page_chunks(a.n_pages)), dim3(kThreads), 0, s, a, rows, across);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || rows == 0) return e;
  hipLaunchKernelGGL(fork_counts, dim3(rows), dim3(kThreads), 0, s, a, across);
  return hipGetLastError();
}

hipError_t launch_pages_extend(const PagesArgs& a, hipStream_t s) {
  const int across = rows_across(a), rows = a.batch * across, chunks = page_chunks(a.n_pages);
  hipLaunchKernelGGL(extend_count, dim3(chunks + 1), dim3(kThreads), 0, s, a);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || rows == 0) return e;
  hipLaunchKernelGGL(extend_rows, dim3(rows), dim3(kThreads), 0, s, a, across);
  return hipGetLastError();
}

hipError_t launch_pages_compact(const PagesArgs& a, hipStream_t s) {
  const int across = rows_across(a), rows = a.batch * across, chunks = page_chunks(a.n_pages);
  hipLaunchKernelGGL(compact_count, dim3(chunks), dim3(kThreads), 0, s, a);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(compact_list, dim3(chunks), dim3(kThreads), 0, s, a);
  e = hipGetLastError();
  if (e != hipSuccess) return e;
  const int page_blocks = (a.n_pages + kThreads - 1) / kThreads;
  hipLaunchKernelGGL(compact_rows, dim3(page_blocks + rows), dim3(kThreads), 0, s, a, page_blocks, across);
  return hipGetLastError();
}

hipError_t launch_pages_copy(const CopyArgs& a, int cus, hipStream_t s) {
  const int64_t items = (a.page_bytes + kPiece - 1) / kPiece * a.max_moves * a.n_buffers;
  const int64_t most = int64_t{kGroupsPerCu} * cus;
  hipLaunchKernelGGL(copy_pages, dim3(static_cast<uint32_t>(items < most ? items : most)), dim3(kThreads), 0, s, a);
  return hipGetLastError();
}

}  // namespace csg
