// Interface between the host runtime and the kernels of the paged key/value cache.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

#include "attn_scores.hpp"

namespace csg {

constexpr int kCacheTileRows = 32;     // (token, head) rows of a tile, one wave's
constexpr int kCacheWideRows = 128;    // rows of a wide task: a tile for each of four waves
constexpr int kCacheBlock = 32;        // keys per inner step of a wave, and unit of work
constexpr int kCacheWideBlock = 64;    // keys per inner step of a wide task
// What beginning and ending a task costs, in blocks. 64 sequences on four shared prompts 47.9 us with 3,
// 48.8 with 4, 49.0 with 6, 49.6 with 8; 12 sequences of 5 tokens on one 23.1, 22.5, 20.7, 22.0; 64 unrelated
// sequences 99.4, 100, 99.7, 98.7: it matters where the cuts happen to fall, and no value is best for all.
constexpr int kCacheTaskCost = 4;
constexpr int kCacheMinRun = 4;  // units a workgroup takes at least: a block for each wave
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
  int32_t head_workers;  // workgroups that share the blocks of keys of a key/value head
  int32_t dies;          // dies that its workgroups are on
  int64_t max_parts;     // places of partial results in the workspace
  int64_t max_tiles;     // tiles of a key/value head, if the bounds ascend
  unsigned char* ws;
  Scoring scoring;
};

// Workspace: the plan of a call, then partial results of 32 rows each.
constexpr int64_t cache_plan_bytes() { return 256 + kMaxCacheEntries * 32; }
constexpr int64_t cache_part_bytes(int head_dim) { return kCacheTileRows * (head_dim + 2) * 4; }
// Workgroups for each key/value head, all of them as many as are on the device at once (two a
// CU, by their registers and, for 128 elements a head, 64 KiB of LDS).
constexpr int32_t cache_head_workers(int32_t cus, int32_t Hkv) { return 2 * cus > Hkv ? 2 * cus / Hkv : 1; }
// Tiles of a key/value head, at most: every token in its sequence and, maybe, its group.
inline int64_t cache_max_tiles(int32_t H, int32_t Hkv, int64_t tokens, int32_t batch, int32_t n_groups) {
  return tokens * (H / Hkv) / kCacheTileRows * (n_groups > 0 ? 2 : 1) + batch + n_groups;
}
// Places of parts: the tiles and four for each workgroup.
inline int64_t cache_max_parts(int32_t H, int32_t Hkv, int64_t tokens, int32_t batch, int32_t n_groups, int32_t head_workers) {
  return (cache_max_tiles(H, Hkv, tokens, batch, n_groups) + int64_t{4} * head_workers) * Hkv;
}

hipError_t launch_cache_append(const AppendArgs& a, bool f16, int head_dim, hipStream_t stream);
hipError_t launch_cache_attn(const CacheAttnArgs& a, bool f16, int head_dim, hipStream_t stream);

}  // namespace csg
