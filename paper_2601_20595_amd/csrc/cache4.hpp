// Interface between the host runtime and the kernels of the paged cache in 4 bits.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

#include "cache_attn.hpp"

namespace csg {

// A head's rows of a page: page size rows of D / 2 bytes, then page size times D / 32 scales.
constexpr int cache4_row_bytes(int head_dim) { return head_dim / 2 + head_dim / 32; }

constexpr int kReadRows = 32;  // rows of the outputs that a workgroup reads

struct ReadArgs {
  CacheArgs c;      // q_ptr: first rows of the sequences; tokens: rows of the outputs
  uint16_t* K;      // rows of Hkv heads, k_stride elements apart
  uint16_t* V;
  int64_t k_stride, v_stride;
};

// The pages of these calls hold bytes (CacheArgs::k_pages and v_pages point at them).
hipError_t launch_cache4_append(const AppendArgs& a, bool f16, int head_dim, hipStream_t stream);
hipError_t launch_cache4_read(const ReadArgs& a, bool f16, int head_dim, hipStream_t stream);
hipError_t launch_cache4_attn(const CacheAttnArgs& a, bool f16, int head_dim, hipStream_t stream);

}  // namespace csg
