// Entry points of attention over packed documents and of the paged key/value cache: checks of
// the arguments, then the launches. Nothing here allocates, waits or keeps state, apart from
// what is known of each device.
#include <algorithm>
#include <cmath>
#include <mutex>
#include <initializer_list>
#include <numeric>

#include "cache_attn.hpp"
#include "csg.h"
#include "doc_attn.hpp"
#include "errors.hpp"

namespace {

using csg::aligned16;
using csg::DeviceGuard;
using csg::fail;
using csg::hip_fail;

constexpr int kMaxDevices = 64;
constexpr int64_t kMaxRows = int64_t{1} << 30;
constexpr int64_t kMaxStride = int64_t{1} << 23;  // 63 rows of it stay within 32-bit byte offsets
constexpr int64_t kMaxGrid = 0xffffffff / 512;  // workgroups: a launch's threads are counted in 32 bits
constexpr int32_t kDefaultCus = 256;
// Rows of a cache's attention: four are a workgroup of the merge, and the tiles of as many as 2048 entries
// with all of the rows each are still counted in 32 bits.
constexpr int64_t kMaxCacheRows = int64_t{1} << 25;
static_assert(kMaxCacheRows / 4 <= kMaxGrid * 2, "workgroups of 256 threads");
static_assert(kMaxCacheRows / csg::kCacheTileRows * csg::kMaxCacheEntries < (int64_t{1} << 32), "tiles");

// Compute units of `device`, checked once to be the one this library is built for.
csg_status device_cus(int device, int32_t* cus) {
  static std::mutex mu;
  static int32_t known[kMaxDevices] = {};
  if (device < 0 || device >= kMaxDevices) return fail(CSG_ERR_INVALID, "device %d out of range", device);
  std::lock_guard<std::mutex> lock(mu);
  if (!known[device]) {
    char arch[64];
    csg_status st = csg_device_check(device, arch, sizeof arch);
    if (st != CSG_OK) return st;
    int n = 0;
    CSG_HIP(hipDeviceGetAttribute(&n, hipDeviceAttributeMultiprocessorCount, device));
    known[device] = n > 0 ? n : kDefaultCus;
  }
  *cus = known[device];
  return CSG_OK;
}

csg_status check_heads(int32_t n_heads, int32_t n_kv_heads, int32_t head_dim, int32_t dtype) {
  if (n_heads < 1 || n_kv_heads < 1 || n_heads % n_kv_heads != 0 || n_heads > 65536)
    return fail(CSG_ERR_INVALID, "n_heads must be a multiple of n_kv_heads, and at most 65536");
  if (dtype != CSG_BF16 && dtype != CSG_F16 && dtype != CSG_F32) return fail(CSG_ERR_INVALID, "unknown dtype %d", dtype);
  if (dtype == CSG_F32) return fail(CSG_ERR_UNSUPPORTED, "attention takes bf16 and f16");
  if (head_dim != 64 && head_dim != 128) return fail(CSG_ERR_UNSUPPORTED, "head_dim must be 64 or 128");
  return CSG_OK;
}

constexpr float kLog2e = 1.4426950408889634f;

csg::Scoring scoring(float scale, float softcap, const float* slopes) {
  csg::Scoring s{};
  s.unit = softcap > 0.0f ? softcap : scale;
  if (softcap > 0.0f) s.cap_in = 2.0f * scale * kLog2e / softcap;
  s.slopes = slopes;
  return s;
}

csg_status check_scores(float* scale, float softcap, int32_t head_dim) {
  if (*scale == 0.0f) *scale = 1.0f / std::sqrt(static_cast<float>(head_dim));
  if (!(*scale > 0.0f) || !std::isfinite(*scale)) return fail(CSG_ERR_INVALID, "scale must be positive and finite");
  if (!(softcap >= 0.0f) || !std::isfinite(softcap)) return fail(CSG_ERR_INVALID, "softcap must be finite and not negative");
  // the kernels' factors: 0 times an infinite one would be NaN
  const csg::Scoring s = scoring(*scale, softcap, nullptr);
  if (!std::isnormal(s.unit) || !std::isfinite(s.unit * kLog2e) || (softcap > 0.0f && !std::isnormal(s.cap_in)))
    return fail(CSG_ERR_INVALID, "scale and softcap, and scale / softcap, must be normal numbers");
  return CSG_OK;
}

// Default and check of a row stride.
csg_status check_stride(int64_t* stride, int64_t row, const char* what) {
  if (*stride == 0) *stride = row;
  if (*stride < row || *stride % 8 != 0)
    return fail(CSG_ERR_INVALID, "%s must be 0, or at least a row and a multiple of 8 elements", what);
  if (*stride > kMaxStride) return fail(CSG_ERR_UNSUPPORTED, "%s must be at most 2^23 elements", what);
  return CSG_OK;
}

#define CSG_CHECK(expr)                \
  do {                                 \
    csg_status s_ = (expr);            \
    if (s_ != CSG_OK) return s_;       \
  } while (0)

csg_status check_docs(csg_doc_attn_cfg* c, bool gradient) {
  CSG_CHECK(check_heads(c->n_heads, c->n_kv_heads, c->head_dim, c->dtype));
  CSG_CHECK(check_scores(&c->scale, c->softcap, c->head_dim));
  if (c->causal != 0 && c->causal != 1) return fail(CSG_ERR_INVALID, "causal must be 0 or 1");
  if (c->joined != 0 && c->joined != 1) return fail(CSG_ERR_INVALID, "joined must be 0 or 1");
  if (c->n_docs < 0 || c->q_rows < 0 || c->k_rows < 0 || c->q_rows > kMaxRows || c->k_rows > kMaxRows ||
      c->n_docs > kMaxRows)
    return fail(CSG_ERR_INVALID, "rows or documents out of range");
  const int64_t q_row = static_cast<int64_t>(c->n_heads) * c->head_dim;
  const int64_t k_row = static_cast<int64_t>(c->n_kv_heads) * c->head_dim;
  CSG_CHECK(check_stride(&c->q_stride, q_row, "q_stride"));
  CSG_CHECK(check_stride(&c->k_stride, k_row, "k_stride"));
  CSG_CHECK(check_stride(&c->v_stride, k_row, "v_stride"));
  if (gradient) {
    CSG_CHECK(check_stride(&c->dq_stride, q_row, "dq_stride"));
    CSG_CHECK(check_stride(&c->dk_stride, k_row, "dk_stride"));
    CSG_CHECK(check_stride(&c->dv_stride, k_row, "dv_stride"));
  }
  // (the smallest tiles: one row of workgroups per head)
  if ((std::max(c->q_rows, c->k_rows) / 32 + c->n_docs) * c->n_heads > kMaxGrid)
    return fail(CSG_ERR_UNSUPPORTED, "too many rows, documents and heads for one launch");
  return CSG_OK;
}

csg::DocAttnArgs doc_args(const csg_doc_attn_cfg& c, int32_t cus, const void* q, const void* k, const void* v, const int32_t* q_ptr,
                          const int32_t* k_ptr, const int32_t* prefix, const float* slopes) {
  csg::DocAttnArgs a{};
  a.Q = static_cast<const uint16_t*>(q);
  a.K = static_cast<const uint16_t*>(k);
  a.V = static_cast<const uint16_t*>(v);
  a.q_ptr = q_ptr;
  a.k_ptr = k_ptr;
  a.prefix = prefix;
  a.q_stride = c.q_stride;
  a.k_stride = c.k_stride;
  a.v_stride = c.v_stride;
  a.dq_stride = c.dq_stride;
  a.dk_stride = c.dk_stride;
  a.dv_stride = c.dv_stride;
  a.q_rows = static_cast<int32_t>(c.q_rows);
  a.k_rows = static_cast<int32_t>(c.k_rows);
  a.n_docs = c.n_docs;
  a.H = c.n_heads;
  a.Hkv = c.n_kv_heads;
  a.tile_heads = std::gcd(c.n_heads / c.n_kv_heads, 4);
  a.causal = c.causal;
  a.joined = c.joined;
  a.cus = cus;
  a.row_parts = 1;
  a.scale = c.scale;
  a.scoring = scoring(c.scale, c.softcap, slopes);
  return a;
}

// Bytes of the rows' statistics, and of everything: the sums of the parts behind them.
int64_t stats_bytes(const csg_doc_attn_cfg& c) { return (2 * c.q_rows * c.n_heads * 4 + 15) / 16 * 16; }
int64_t part_bytes(const csg_doc_attn_cfg& c, int64_t rows) { return rows * c.n_kv_heads * 2 * c.head_dim * 4; }
int32_t row_parts(const csg_doc_attn_cfg& c, int32_t cus) {
  return csg::doc_row_parts(c.q_rows, c.k_rows, c.n_docs, c.n_heads, c.n_kv_heads, c.head_dim, cus);
}
int64_t grad_workspace(const csg_doc_attn_cfg& c, int32_t cus) {
  const int32_t parts = row_parts(c, cus);
  return stats_bytes(c) + (parts > 1 ? part_bytes(c, parts * c.k_rows) : 0);
}
// What any call of up to cfg's rows and keys needs, whatever its documents are.
int64_t max_grad_workspace(const csg_doc_attn_cfg& c, int32_t cus) {
  return stats_bytes(c) + part_bytes(c, csg::doc_max_part_rows(c.q_rows, c.k_rows, c.n_heads, c.n_kv_heads, c.head_dim, cus));
}

csg_status check_cache(csg_cache_cfg* c) {
  CSG_CHECK(check_heads(c->n_heads, c->n_kv_heads, c->head_dim, c->dtype));
  if (c->n_pages < 1 || c->batch < 0 || c->max_pages < 1 || c->tokens < 0 || c->tokens > kMaxRows || c->n_groups < 0)
    return fail(CSG_ERR_INVALID, "bad cache shape");
  if (c->page_size < 1) return fail(CSG_ERR_INVALID, "bad page size");
  if (c->page_size != 16 && c->page_size != 32 && c->page_size != 64 && c->page_size != 128 && c->page_size != 256)
    return fail(CSG_ERR_UNSUPPORTED, "page_size must be 16, 32, 64, 128 or 256");
  if (static_cast<int64_t>(c->max_pages) * c->page_size > kMaxRows)
    return fail(CSG_ERR_UNSUPPORTED, "a sequence may have at most 2^30 tokens");
  CSG_CHECK(check_stride(&c->q_stride, static_cast<int64_t>(c->n_heads) * c->head_dim, "q_stride"));
  return CSG_OK;
}

csg_status check_cache_attn(csg_cache_cfg* c) {
  CSG_CHECK(check_cache(c));
  CSG_CHECK(check_scores(&c->scale, c->softcap, c->head_dim));
  if (c->n_groups > c->batch) return fail(CSG_ERR_INVALID, "more groups than sequences");
  if (static_cast<int64_t>(c->batch) + c->n_groups > csg::kMaxCacheEntries)
    return fail(CSG_ERR_UNSUPPORTED, "at most %d sequences and groups", csg::kMaxCacheEntries);
  if (c->tokens * c->n_heads > kMaxCacheRows) return fail(CSG_ERR_UNSUPPORTED, "too many tokens and heads for one launch");
  // blocks of keys times tasks that read them, at most; they are counted in 32 bits. (A task has at
  // least a tile, one of four tiles and more as many as four go into it, rounded up.)
  const int64_t tiles = csg::cache_max_tiles(c->n_heads, c->n_kv_heads, c->tokens, c->batch, c->n_groups);
  const int64_t tasks = tiles / 4 + c->batch + c->n_groups;
  const int64_t blocks = static_cast<int64_t>(c->max_pages) * c->page_size / csg::kCacheBlock + 1;
  if (tasks > 0 && blocks + csg::kCacheTaskCost > 0x7fffffff / tasks)
    return fail(CSG_ERR_UNSUPPORTED, "max_pages pages for every sequence are too many keys for one launch");
  return CSG_OK;
}

int64_t cache_workspace(const csg_cache_cfg& c, int32_t cus) {
  return csg::cache_plan_bytes() + csg::cache_part_bytes(c.head_dim) *
                                       csg::cache_max_parts(c.n_heads, c.n_kv_heads, c.tokens, c.batch, c.n_groups,
                                                            csg::cache_head_workers(cus, c.n_kv_heads));
}

csg::CacheArgs cache_args(const csg_cache_cfg& c, const void* k_pages, const void* v_pages, const void* q, const int32_t* q_ptr,
                          const int32_t* lens, const int32_t* table, int32_t* status) {
  csg::CacheArgs a{};
  a.k_pages = static_cast<uint16_t*>(const_cast<void*>(k_pages));
  a.v_pages = static_cast<uint16_t*>(const_cast<void*>(v_pages));
  a.q_ptr = q_ptr;
  a.lens = lens;
  a.table = table;
  a.status = status;
  a.n_pages = c.n_pages;
  while ((1 << a.page_shift) < c.page_size) ++a.page_shift;
  a.batch = c.batch;
  a.max_pages = c.max_pages;
  a.H = c.n_heads;
  a.Hkv = c.n_kv_heads;
  a.tokens = static_cast<int32_t>(c.tokens);
  a.Q = static_cast<const uint16_t*>(q);
  a.q_stride = c.q_stride;
  return a;
}

bool all_aligned(std::initializer_list<const void*> list) {
  for (const void* p : list)
    if (!aligned16(p)) return false;
  return true;
}

}  // namespace

csg_status csg_doc_attn(const csg_doc_attn_cfg* cfg, const void* q, const void* k, const void* v, const int32_t* q_ptr,
                        const int32_t* k_ptr, const int32_t* prefix, const float* slopes, void* o, void* lse, int device,
                        void* stream) {
  if (!cfg) return fail(CSG_ERR_INVALID, "cfg is NULL");
  csg_doc_attn_cfg c = *cfg;
  CSG_CHECK(check_docs(&c, false));
  if (c.q_rows == 0 || c.n_docs == 0) return CSG_OK;
  if (!q || !o || !lse || !q_ptr || !k_ptr || (c.k_rows > 0 && (!k || !v))) return fail(CSG_ERR_INVALID, "NULL buffer");
  if (!all_aligned({q, k, v, o, lse})) return fail(CSG_ERR_INVALID, "buffers must be 16-byte aligned");
  int32_t cus = 0;
  CSG_CHECK(device_cus(device, &cus));
  DeviceGuard g(device);
  if (g.err != hipSuccess) return hip_fail(g.err, "hipSetDevice");
  csg::DocAttnArgs a = doc_args(c, cus, q, k, v, q_ptr, k_ptr, prefix, slopes);
  a.O = static_cast<uint16_t*>(o);
  a.LSE = static_cast<float*>(lse);
  CSG_HIP(csg::launch_doc_forward(a, c.dtype == CSG_F16, c.head_dim, static_cast<hipStream_t>(stream)));
  return CSG_OK;
}

csg_status csg_doc_attn_grad_workspace(const csg_doc_attn_cfg* cfg, int device, size_t* bytes) {
  if (!cfg || !bytes) return fail(CSG_ERR_INVALID, "NULL argument");
  csg_doc_attn_cfg c = *cfg;
  CSG_CHECK(check_docs(&c, true));
  int32_t cus = kDefaultCus;
  if (device >= 0) CSG_CHECK(device_cus(device, &cus));
  *bytes = static_cast<size_t>(max_grad_workspace(c, cus));
  return CSG_OK;
}

csg_status csg_doc_attn_grad(const csg_doc_attn_cfg* cfg, const void* q, const void* k, const void* v, const int32_t* q_ptr,
                             const int32_t* k_ptr, const int32_t* prefix, const float* slopes, const void* o,
                             const void* lse, const void* d_o, void* dq, void* dk, void* dv, void* workspace,
                             size_t workspace_bytes, int device, void* stream) {
  if (!cfg) return fail(CSG_ERR_INVALID, "cfg is NULL");
  csg_doc_attn_cfg c = *cfg;
  CSG_CHECK(check_docs(&c, true));
  if (c.n_docs == 0 || (c.q_rows == 0 && c.k_rows == 0)) return CSG_OK;
  // (without rows there are no statistics and no parts: the workspace is empty)
  if (!q_ptr || !k_ptr || (c.q_rows > 0 && (!q || !o || !lse || !d_o || !dq || !workspace)) ||
      (c.k_rows > 0 && (!k || !v || !dk || !dv)))
    return fail(CSG_ERR_INVALID, "NULL buffer");
  if (!all_aligned({q, k, v, o, lse, d_o, dq, dk, dv, workspace}))
    return fail(CSG_ERR_INVALID, "buffers must be 16-byte aligned");
  int32_t cus = 0;
  CSG_CHECK(device_cus(device, &cus));
  if (static_cast<int64_t>(workspace_bytes) < grad_workspace(c, cus))
    return fail(CSG_ERR_INVALID, "the workspace holds %zu bytes; the call needs %lld", workspace_bytes,
                static_cast<long long>(grad_workspace(c, cus)));
  DeviceGuard g(device);
  if (g.err != hipSuccess) return hip_fail(g.err, "hipSetDevice");
  csg::DocAttnArgs a = doc_args(c, cus, q, k, v, q_ptr, k_ptr, prefix, slopes);
  a.O = static_cast<uint16_t*>(const_cast<void*>(o));
  a.LSE = static_cast<float*>(const_cast<void*>(lse));
  a.dO = static_cast<const uint16_t*>(d_o);
  a.dQ = static_cast<uint16_t*>(dq);
  a.dK = static_cast<uint16_t*>(dk);
  a.dV = static_cast<uint16_t*>(dv);
  a.stats = static_cast<float*>(workspace);
  a.row_parts = row_parts(c, cus);
  a.parts = reinterpret_cast<float*>(static_cast<unsigned char*>(workspace) + stats_bytes(c));
  CSG_HIP(csg::launch_doc_grad(a, c.dtype == CSG_F16, c.head_dim, static_cast<hipStream_t>(stream)));
  return CSG_OK;
}

csg_status csg_cache_append(const csg_cache_cfg* cfg, void* k_pages, void* v_pages, const void* k, const void* v, const void* q,
                            void* q_out, const int32_t* q_ptr, const int32_t* lens, const int32_t* page_table,
                            const double* inv_freq, int32_t* status, int device, void* stream) {
  if (!cfg) return fail(CSG_ERR_INVALID, "cfg is NULL");
  csg_cache_cfg c = *cfg;
  CSG_CHECK(check_cache(&c));
  const int64_t k_row = static_cast<int64_t>(c.n_kv_heads) * c.head_dim;
  CSG_CHECK(check_stride(&c.k_stride, k_row, "k_stride"));
  CSG_CHECK(check_stride(&c.v_stride, k_row, "v_stride"));
  if (c.tokens > kMaxGrid) return fail(CSG_ERR_UNSUPPORTED, "too many tokens for one launch");
  if (c.rot_dim < 0 || c.rot_dim > c.head_dim || c.rot_dim % 16 != 0)
    return fail(CSG_ERR_INVALID, "rot_dim must be a multiple of 16 up to head_dim");
  if (c.interleaved != 0 && c.interleaved != 1) return fail(CSG_ERR_INVALID, "interleaved must be 0 or 1");
  if ((q != nullptr) != (q_out != nullptr)) return fail(CSG_ERR_INVALID, "q and q_out go together");
  if (q && q == q_out && c.q_stride != static_cast<int64_t>(c.n_heads) * c.head_dim)
    return fail(CSG_ERR_INVALID, "q_out is dense: it can be q only if q is");
  if (c.tokens == 0 || c.batch == 0) return CSG_OK;
  if (!k_pages || !v_pages || !k || !v || !q_ptr || !lens || !page_table || (c.rot_dim > 0 && !inv_freq))
    return fail(CSG_ERR_INVALID, "NULL buffer");
  if (!all_aligned({k_pages, v_pages, k, v, q, q_out})) return fail(CSG_ERR_INVALID, "buffers must be 16-byte aligned");
  int32_t cus = 0;
  CSG_CHECK(device_cus(device, &cus));
  DeviceGuard g(device);
  if (g.err != hipSuccess) return hip_fail(g.err, "hipSetDevice");
  csg::AppendArgs a{};
  a.c = cache_args(c, k_pages, v_pages, q, q_ptr, lens, page_table, status);
  a.K = static_cast<const uint16_t*>(k);
  a.V = static_cast<const uint16_t*>(v);
  a.q_out = static_cast<uint16_t*>(q_out);
  a.inv_freq = inv_freq;
  a.k_stride = c.k_stride;
  a.v_stride = c.v_stride;
  a.half = c.rot_dim / 2;
  a.interleaved = c.interleaved;
  CSG_HIP(csg::launch_cache_append(a, c.dtype == CSG_F16, c.head_dim, static_cast<hipStream_t>(stream)));
  return CSG_OK;
}

csg_status csg_cache_attn_workspace(const csg_cache_cfg* cfg, int device, size_t* bytes) {
  if (!cfg || !bytes) return fail(CSG_ERR_INVALID, "NULL argument");
  csg_cache_cfg c = *cfg;
  CSG_CHECK(check_cache_attn(&c));
  int32_t cus = kDefaultCus;
  if (device >= 0) CSG_CHECK(device_cus(device, &cus));
  *bytes = static_cast<size_t>(cache_workspace(c, cus));
  return CSG_OK;
}

csg_status csg_cache_attn(const csg_cache_cfg* cfg, const void* q, const void* k_pages, const void* v_pages,
                          const int32_t* q_ptr, const int32_t* lens, const int32_t* page_table, const int32_t* group_ptr,
                          const int32_t* prefix, const float* slopes, void* o, void* lse, void* workspace,
                          size_t workspace_bytes, int32_t* status, int device, void* stream) {
  if (!cfg) return fail(CSG_ERR_INVALID, "cfg is NULL");
  csg_cache_cfg c = *cfg;
  CSG_CHECK(check_cache_attn(&c));
  if (c.tokens == 0 || c.batch == 0) return CSG_OK;
  if (!q || !k_pages || !v_pages || !q_ptr || !lens || !page_table || !o || !workspace ||
      (c.n_groups > 0 && (!group_ptr || !prefix)))
    return fail(CSG_ERR_INVALID, "NULL buffer");
  if (!all_aligned({q, k_pages, v_pages, o, workspace})) return fail(CSG_ERR_INVALID, "buffers must be 16-byte aligned");
  int32_t cus = 0;
  CSG_CHECK(device_cus(device, &cus));
  if (static_cast<int64_t>(workspace_bytes) < cache_workspace(c, cus))
    return fail(CSG_ERR_INVALID, "the workspace holds %zu bytes; the call needs %lld", workspace_bytes,
                static_cast<long long>(cache_workspace(c, cus)));
  DeviceGuard g(device);
  if (g.err != hipSuccess) return hip_fail(g.err, "hipSetDevice");
  csg::CacheAttnArgs a{};
  a.c = cache_args(c, k_pages, v_pages, q, q_ptr, lens, page_table, status);
  a.O = static_cast<uint16_t*>(o);
  a.LSE = static_cast<float*>(lse);
  a.group_ptr = group_ptr;
  a.prefix = prefix;
  a.n_groups = c.n_groups;
  a.head_workers = csg::cache_head_workers(cus, c.n_kv_heads);
  a.dies = 8 / std::gcd(8, c.n_kv_heads);
  a.max_parts = csg::cache_max_parts(c.n_heads, c.n_kv_heads, c.tokens, c.batch, c.n_groups, a.head_workers);
  a.max_tiles = csg::cache_max_tiles(c.n_heads, c.n_kv_heads, c.tokens, c.batch, c.n_groups);
  a.ws = static_cast<unsigned char*>(workspace);
  a.scoring = scoring(c.scale, c.softcap, slopes);
  CSG_HIP(csg::launch_cache_attn(a, c.dtype == CSG_F16, c.head_dim, static_cast<hipStream_t>(stream)));
  return CSG_OK;
}
