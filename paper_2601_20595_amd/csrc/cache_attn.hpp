// Interface between the host runtime and the kernels of the paged key/value cache.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

#include "attn_scores.hpp"

namespace csg {

constexpr int kCacheTileRows = 32;     // (token, head) rows of a tile
constexpr int kCacheBlock = 32;        // keys per inner step of a wave
constexpr int kMaxCacheEntries = 2048; // sequences and groups of one call

// status bits
constexpr int kCacheBadPage = 1, kCacheBadLength = 2;

struct CacheArgs {
  uint16_t* k_pages;  // [n_pages][Hkv][page size][D]
  uint16_t* v_pages;
  const int32_t* q_ptr;  // [batch + 1]
  const int32_t* lens;   // [batch]
  const int32_t* table;  // [batch][max_pages]
  int32_t* status;       // or null
  int32_t n_pages, page_shift, batch, max_pages;
  int32_t H, Hkv;
  int32_t tokens;
  const uint16_t* Q;  // may be null in an append
  int64_t q_stride;
};

struct AppendArgs {
  CacheArgs c;
  const uint16_t* K;
  const uint16_t* V;
  uint16_t* q_out;         // [tokens][H][D]
  const double* inv_freq;  // [half], or null
  int64_t k_stride, v_stride;
  int32_t half;  // pairs rotated
  int32_t interleaved;
};

struct CacheAttnArgs {
  CacheArgs c;
  uint16_t* O;   // [tokens][H][D]
  float* LSE;    // [H][tokens]
  const int32_t* group_ptr;  // [n_groups + 1]
  const int32_t* prefix;     // [n_groups]
  int32_t n_groups;
  int32_t workers;   // workgroups that share the blocks of keys
  int32_t max_parts; // partial results the workspace holds
  unsigned char* ws;
  Scoring scoring;
};

// Workspace: the plan of a call, then partial results of 32 rows each.
constexpr int64_t cache_plan_bytes() { return 16 + kMaxCacheEntries * 16 + 240; }
constexpr int64_t cache_part_bytes(int head_dim) { return kCacheTileRows * (head_dim + 2) * 4; }
// Every task (a key/value head, one tile of rows, the keys of a sequence or the shared ones of
// a group) is cut where the work of one workgroup ends: no more parts than tasks and cuts.
inline int64_t cache_max_parts(int32_t H, int32_t Hkv, int64_t tokens, int32_t batch, int32_t n_groups, int32_t workers) {
  const int64_t tiles = tokens * (H / Hkv) / kCacheTileRows * (n_groups > 0 ? 2 : 1) + batch + n_groups;
  return tiles * Hkv + workers;
}

hipError_t launch_cache_append(const AppendArgs& a, bool f16, int head_dim, hipStream_t stream);
hipError_t launch_cache_attn(const CacheAttnArgs& a, bool f16, int head_dim, hipStream_t stream);

}  // namespace csg
