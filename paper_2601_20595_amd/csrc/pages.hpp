// Interface between the host runtime and the kernels that manage a cache's pages.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

namespace csg {

constexpr int kPageChunk = 1024;               // pages that a workgroup counts
constexpr int32_t kMaxPoolPages = 1 << 24;     // as many chunks as a workgroup sums up in 64 turns
constexpr int32_t kMaxPoolBatch = 1 << 20;
constexpr int kCopyBuffers = 64;               // buffers of one launch

// status bits beyond those of the cache's calls
constexpr int kPagesNone = 4;  // no page was free

struct PagesArgs {
  const int32_t* table;  // [batch][max_pages]
  const int32_t* lens;   // [batch]
  const int32_t* refs;   // [n_pages]
  const int32_t* change;  // [batch]: parents (fork), tokens (extend)
  int32_t* table_out;
  int32_t* lens_out;
  int32_t* refs_out;
  int32_t* renamed;  // [n_pages] (compact)
  int32_t* moves;    // [][2]
  int32_t* n_moves;
  int32_t* status;   // or null
  unsigned char* ws;
  int32_t n_pages, page_shift, batch, max_pages;
};

struct CopyArgs {
  unsigned char* buffers[kCopyBuffers];
  const int32_t* moves;
  const int32_t* n_moves;
  int32_t* status;
  int64_t page_bytes;
  int32_t n_buffers, max_moves, n_pages;
};

constexpr int32_t page_chunks(int32_t n_pages) { return (n_pages + kPageChunk - 1) / kPageChunk; }
// Workspace: sums, counts of the chunks, two words a page, and of a sequence the places of its requests and its copy.
inline int64_t pages_workspace(int32_t n_pages, int32_t batch) {
  return 64 + int64_t{8} * (page_chunks(n_pages) / 2 + 1) + int64_t{8} * n_pages + int64_t{16} * batch;
}

hipError_t launch_pages_fork(const PagesArgs& a, hipStream_t stream);
hipError_t launch_pages_extend(const PagesArgs& a, hipStream_t stream);
hipError_t launch_pages_compact(const PagesArgs& a, hipStream_t stream);
hipError_t launch_pages_copy(const CopyArgs& a, int cus, hipStream_t stream);

}  // namespace csg
