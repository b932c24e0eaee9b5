// Entry points that manage the pages of a paged cache: checks of the arguments, then the launches.
#include <algorithm>
#include <initializer_list>

#include "csg.h"
#include "errors.hpp"
#include "pages.hpp"

namespace {

using csg::aligned16;
using csg::device_cus;
using csg::DeviceGuard;
using csg::fail;
using csg::hip_fail;

constexpr int64_t kMaxTableBlocks = 0xffffffff / 512;  // a launch's threads are counted in 32 bits
constexpr int64_t kMaxPageBytes = int64_t{1} << 31;

#define CSG_CHECK(expr)                \
  do {                                 \
    csg_status s_ = (expr);            \
    if (s_ != CSG_OK) return s_;       \
  } while (0)

csg_status check_pool(const csg_pages_cfg* c) {
  if (!c) return fail(CSG_ERR_INVALID, "cfg is NULL");
  if (c->n_pages < 1 || c->batch < 0 || c->max_pages < 1 || c->page_size < 1 || c->reserved != 0)
    return fail(CSG_ERR_INVALID, "bad shape of the cache");
  if (c->page_size != 16 && c->page_size != 32 && c->page_size != 64 && c->page_size != 128 && c->page_size != 256)
    return fail(CSG_ERR_UNSUPPORTED, "page_size must be 16, 32, 64, 128 or 256");
  if (c->n_pages > csg::kMaxPoolPages || c->batch > csg::kMaxPoolBatch)
    return fail(CSG_ERR_UNSUPPORTED, "at most 2^24 pages and 2^20 sequences");
  if (static_cast<int64_t>(c->max_pages) * c->page_size > (int64_t{1} << 30))
    return fail(CSG_ERR_UNSUPPORTED, "a sequence may have at most 2^30 tokens");
  if ((c->max_pages / 1024 + 1) * static_cast<int64_t>(c->batch) > kMaxTableBlocks)
    return fail(CSG_ERR_UNSUPPORTED, "the page table is too large for one launch");
  return CSG_OK;
}

struct Span {
  const void* p;
  int64_t words;
};

// Outputs are written while inputs are still read: no two may share memory, but inputs.
csg_status check_apart(std::initializer_list<Span> in, std::initializer_list<Span> out) {
  auto meet = [](const Span& a, const Span& b) {
    const uintptr_t x = reinterpret_cast<uintptr_t>(a.p), y = reinterpret_cast<uintptr_t>(b.p);
    return a.words > 0 && b.words > 0 && x < y + 4 * static_cast<uint64_t>(b.words) && y < x + 4 * static_cast<uint64_t>(a.words);
  };
  for (const Span* o = out.begin(); o != out.end(); ++o) {
    for (const Span& i : in)
      if (meet(*o, i)) return fail(CSG_ERR_INVALID, "outputs may not overlap inputs");
    for (const Span* p = out.begin(); p != o; ++p)
      if (meet(*o, *p)) return fail(CSG_ERR_INVALID, "outputs may not overlap each other");
  }
  return CSG_OK;
}

csg::PagesArgs pool_args(const csg_pages_cfg& c) {
  csg::PagesArgs a{};
  a.n_pages = c.n_pages;
  while ((1 << a.page_shift) < c.page_size) ++a.page_shift;
  a.batch = c.batch;
  a.max_pages = c.max_pages;
  return a;
}

int64_t table_words(const csg_pages_cfg& c) { return static_cast<int64_t>(c.batch) * c.max_pages; }

csg_status check_workspace(const csg_pages_cfg& c, const void* workspace, size_t bytes) {
  const int64_t need = csg::pages_workspace(c.n_pages, c.batch);
  if (!workspace) return fail(CSG_ERR_INVALID, "NULL buffer");
  if (!aligned16(workspace)) return fail(CSG_ERR_INVALID, "the workspace must be 16-byte aligned");
  if (static_cast<int64_t>(bytes) < need)
    return fail(CSG_ERR_INVALID, "the workspace holds %zu bytes; the call needs %lld", bytes, static_cast<long long>(need));
  return CSG_OK;
}

}  // namespace

csg_status csg_pages_workspace(const csg_pages_cfg* cfg, size_t* bytes) {
  CSG_CHECK(check_pool(cfg));
  if (!bytes) return fail(CSG_ERR_INVALID, "NULL argument");
  *bytes = static_cast<size_t>(csg::pages_workspace(cfg->n_pages, cfg->batch));
  return CSG_OK;
}

csg_status csg_pages_fork(const csg_pages_cfg* cfg, const int32_t* page_table, const int32_t* lens, const int32_t* refs,
                          const int32_t* parent, int32_t* table_out, int32_t* lens_out, int32_t* refs_out, int32_t* status,
                          int device, void* stream) {
  CSG_CHECK(check_pool(cfg));
  if (!refs || !refs_out || (cfg->batch > 0 && (!page_table || !lens || !parent || !table_out || !lens_out)))
    return fail(CSG_ERR_INVALID, "NULL buffer");
  const int64_t words = table_words(*cfg), b = cfg->batch, n = cfg->n_pages;
  CSG_CHECK(check_apart({{page_table, words}, {lens, b}, {refs, n}, {parent, b}}, {{table_out, words}, {lens_out, b}, {refs_out, n}}));
  int32_t cus = 0;
  CSG_CHECK(device_cus(device, &cus));
  DeviceGuard g(device);
  if (g.err != hipSuccess) return hip_fail(g.err, "hipSetDevice");
  csg::PagesArgs a = pool_args(*cfg);
  a.table = page_table;
  a.lens = lens;
  a.refs = refs;
  a.change = parent;
  a.table_out = table_out;
  a.lens_out = lens_out;
  a.refs_out = refs_out;
  a.status = status;
  CSG_HIP(csg::launch_pages_fork(a, static_cast<hipStream_t>(stream)));
  return CSG_OK;
}

csg_status csg_pages_extend(const csg_pages_cfg* cfg, const int32_t* page_table, const int32_t* lens, const int32_t* refs,
                            const int32_t* grow, int32_t* table_out, int32_t* lens_out, int32_t* refs_out, int32_t* moves,
                            int32_t* n_moves, void* workspace, size_t workspace_bytes, int32_t* status, int device,
                            void* stream) {
  CSG_CHECK(check_pool(cfg));
  if (!refs || !refs_out || !n_moves ||
      (cfg->batch > 0 && (!page_table || !lens || !grow || !table_out || !lens_out || !moves)))
    return fail(CSG_ERR_INVALID, "NULL buffer");
  CSG_CHECK(check_workspace(*cfg, workspace, workspace_bytes));
  const int64_t words = table_words(*cfg), b = cfg->batch, n = cfg->n_pages;
  CSG_CHECK(check_apart({{page_table, words}, {lens, b}, {refs, n}, {grow, b}},
                        {{table_out, words}, {lens_out, b}, {refs_out, n}, {moves, 2 * b}, {n_moves, 1},
                         {workspace, csg::pages_workspace(cfg->n_pages, cfg->batch) / 4}}));
  int32_t cus = 0;
  CSG_CHECK(device_cus(device, &cus));
  DeviceGuard g(device);
  if (g.err != hipSuccess) return hip_fail(g.err, "hipSetDevice");
  csg::PagesArgs a = pool_args(*cfg);
  a.table = page_table;
  a.lens = lens;
  a.refs = refs;
  a.change = grow;
  a.table_out = table_out;
  a.lens_out = lens_out;
  a.refs_out = refs_out;
  a.moves = moves;
  a.n_moves = n_moves;
  a.status = status;
  a.ws = static_cast<unsigned char*>(workspace);
  CSG_HIP(csg::launch_pages_extend(a, static_cast<hipStream_t>(stream)));
  return CSG_OK;
}

csg_status csg_pages_compact(const csg_pages_cfg* cfg, const int32_t* page_table, const int32_t* lens, const int32_t* refs,
                             int32_t* table_out, int32_t* refs_out, int32_t* renamed, int32_t* moves, int32_t* n_moves,
                             void* workspace, size_t workspace_bytes, int32_t* status, int device, void* stream) {
  CSG_CHECK(check_pool(cfg));
  if (!refs || !refs_out || !renamed || !n_moves || (cfg->n_pages > 1 && !moves) ||
      (cfg->batch > 0 && (!page_table || !lens || !table_out)))
    return fail(CSG_ERR_INVALID, "NULL buffer");
  CSG_CHECK(check_workspace(*cfg, workspace, workspace_bytes));
  const int64_t words = table_words(*cfg), b = cfg->batch, n = cfg->n_pages;
  CSG_CHECK(check_apart({{page_table, words}, {lens, b}, {refs, n}},
                        {{table_out, words}, {refs_out, n}, {renamed, n}, {moves, n / 2 * 2}, {n_moves, 1},
                         {workspace, csg::pages_workspace(cfg->n_pages, cfg->batch) / 4}}));
  int32_t cus = 0;
  CSG_CHECK(device_cus(device, &cus));
  DeviceGuard g(device);
  if (g.err != hipSuccess) return hip_fail(g.err, "hipSetDevice");
  csg::PagesArgs a = pool_args(*cfg);
  a.table = page_table;
  a.lens = lens;
  a.refs = refs;
  a.table_out = table_out;
  a.refs_out = refs_out;
  a.renamed = renamed;
  a.moves = moves;
  a.n_moves = n_moves;
  a.status = status;
  a.ws = static_cast<unsigned char*>(workspace);
  CSG_HIP(csg::launch_pages_compact(a, static_cast<hipStream_t>(stream)));
  return CSG_OK;
}

csg_status csg_pages_copy(int32_t n_pages, int64_t page_bytes, int32_t n_buffers, void* const* buffers, const int32_t* moves,
                          int32_t max_moves, const int32_t* n_moves, int32_t* status, int device, void* stream) {
  if (n_pages < 1 || n_buffers < 0 || max_moves < 0 || page_bytes < 0)
    return fail(CSG_ERR_INVALID, "bad shape of the buffers");
  if (page_bytes % 16 != 0) return fail(CSG_ERR_INVALID, "page_bytes must be a multiple of 16");
  if (page_bytes > kMaxPageBytes) return fail(CSG_ERR_UNSUPPORTED, "page_bytes must be at most 2^31");
  if (n_buffers == 0 || max_moves == 0 || page_bytes == 0) return CSG_OK;
  if (!buffers || !moves || !n_moves) return fail(CSG_ERR_INVALID, "NULL buffer");
  for (int32_t i = 0; i < n_buffers; ++i) {
    if (!buffers[i]) return fail(CSG_ERR_INVALID, "NULL buffer");
    if (!aligned16(buffers[i])) return fail(CSG_ERR_INVALID, "buffers must be 16-byte aligned");
  }
  int32_t cus = 0;
  CSG_CHECK(device_cus(device, &cus));
  DeviceGuard g(device);
  if (g.err != hipSuccess) return hip_fail(g.err, "hipSetDevice");
  csg::CopyArgs a{};
  a.moves = moves;
  a.n_moves = n_moves;
  a.status = status;
  a.page_bytes = page_bytes;
  a.max_moves = max_moves;
  a.n_pages = n_pages;
  for (int32_t first = 0; first < n_buffers; first += csg::kCopyBuffers) {
    a.n_buffers = std::min(n_buffers - first, csg::kCopyBuffers);
    for (int32_t i = 0; i < a.n_buffers; ++i) a.buffers[i] = static_cast<unsigned char*>(buffers[first + i]);
    CSG_HIP(csg::launch_pages_copy(a, cus, static_cast<hipStream_t>(stream)));
  }
  return CSG_OK;
}
