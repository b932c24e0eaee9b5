// Interface between the host runtime and the kernels of the paged cache in 4 bits.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

#include "cache_attn.hpp"

namespace csg {

// A head's rows of a page: page size rows of D / 2 bytes, then page size times D / 32 scales.
constexpr int cache4_row_bytes(int head_dim) { return head_dim / 2 + head_dim / 32; }

// Attention's kernel for few rows has more workgroups on a CU than the other, whose number is the 16-bit cache's.
constexpr int kCache4Few = 3;
// kCacheTaskCost here, where a block is a quarter of the bytes. With 4, 8, 10, 12, 16: 64 unrelated sequences 41.9 us, 40.2, 39.7,
// 38.7, 39.6; 64 on four shared prompts 40.6, then 38.3 with any; 16 on one of 8192 31.2, 26.4, 28.0, 27.5, 26.6; 24 on two 26.2, 25.8,
// 24.2, 24.1, 25.3; 64 of up to 100 keys on one of 2000 27.0, 25.0, 24.5, 25.3, 25.0; 64 new tokens on 6000 to 9000 keys, two
// sequences (heads of 64) 32.4, 30.0, 29.6, 29.9, 29.5. From 8 on the cuts of each call's runs decide, not the cost.
constexpr int kCache4TaskCost = 10;
// Waves with runs of their own, four tasks of a workgroup at a time: 128 sequences of 20 to 300 keys 22.1 -> 18.2 us, 256 of 500 to
// 2000 80.4 -> 78.3; 64 of 100 to 8000, 58 blocks each, take 39.7 either way (heads of 64: 28.4 -> 27.0, so twice as many there).
// A task's cost 2: 19.0 us (128 sequences), 4: 18.2, 8: 19.6.
constexpr int kCache4AloneCost = 4;
constexpr int kCache4AloneBlocks = 48;  // of 128 elements a head, on average; 64: twice as many
// Units of a wave's run that a unit of another task counts for, where workgroups are divided between the two (undivided; 2, 4, 6,
// 8): 64 sequences of 20 to 1000 keys on four prompts 40.7 us; 36.5, 38.3, 38.5, 42.1; 256 of 300 to 2000 134; 98.2, 89.4, 90.7,
// 92.5; 96 of up to 400 on three (heads of 64) 31.5; 23.5, 23.1, 23.2, 23.5. With fewer than half as many small tasks as workgroups
// it gains nothing (24 sequences on two prompts 24.1, divided 24.4).
constexpr int kCache4OtherUnits = 4;
// Whether the sequences' rows (new tokens times heads of a key/value head) are few, on average; with groups, whose
// sequences' rows go through the shared keys together, never.
inline bool cache4_few(int64_t tokens, int32_t H, int32_t Hkv, int32_t batch, int32_t n_groups) {
  return n_groups == 0 && tokens * (H / Hkv) <= int64_t{16} * batch;
}
// Units of a run, at least. A part of a wide task writes 66 KB: with runs of 4, 8, 16, 64 sequences of up to 100 keys on a prompt of
// 2000 take 26.3 us, 24.5, 28.4; 96 of up to 400 on three (heads of 64) 23.1, 23.1, 26.5; 16 on one of 8192 27.9, 28.0, 28.8. Without
// groups shorter ones end sooner (16 rows of a head on 500 keys, two sequences, where this was tried without groups too: 14.3, 16.5, 16.6).
constexpr int kCache4WideRun = 8;
inline int32_t cache4_min_run(int64_t tokens, int32_t H, int32_t Hkv, int32_t batch, int32_t n_groups) {
  return n_groups > 0 && tokens * (H / Hkv) > int64_t{kCacheTileRows} * n_groups ? kCache4WideRun : kCacheMinRun;
}
constexpr int kReadRows = 32;  // rows of the outputs that a workgroup reads
// Heads that it reads: as many as leave four workgroups a CU, up to 8.
inline int32_t cache4_read_heads(int64_t tokens, int32_t Hkv, int32_t cus) {
  int32_t heads = 1;
  while (heads < 8 && Hkv % (2 * heads) == 0 && (tokens / kReadRows + 1) * (Hkv / (2 * heads)) >= 4 * cus) heads *= 2;
  return heads;
}

struct ReadArgs {
  CacheArgs c;      // q_ptr: first rows of the sequences; tokens: rows of the outputs
  uint16_t* K;      // rows of Hkv heads, k_stride elements apart
  uint16_t* V;
  int64_t k_stride, v_stride;
  int32_t heads;    // that a workgroup reads, a divisor of Hkv
};

// The pages of these calls hold bytes (CacheArgs::k_pages and v_pages point at them).
hipError_t launch_cache4_append(const AppendArgs& a, bool f16, int head_dim, hipStream_t stream);
hipError_t launch_cache4_read(const ReadArgs& a, bool f16, int head_dim, hipStream_t stream);
hipError_t launch_cache4_attn(const CacheAttnArgs& a, bool f16, int head_dim, hipStream_t stream);

}  // namespace csg
