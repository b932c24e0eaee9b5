// Interface between the host runtime and the kernels of attention over packed documents.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

#include "attn_scores.hpp"

namespace csg {

constexpr int kDocTileRows = 128;  // (row, head) pairs of a tile: 4 waves of 32
constexpr int kDocBlock = 64;      // keys (gradient of keys and values: rows) per inner step

struct DocAttnArgs {
  const uint16_t* Q;   // rows of H heads of D elements, q_stride elements apart; K, V: Hkv heads
  const uint16_t* K;
  const uint16_t* V;
  uint16_t* O;         // [q_rows][H][D]
  float* LSE;          // [H][q_rows]
  const uint16_t* dO;  // [q_rows][H][D]
  uint16_t* dQ;
  uint16_t* dK;
  uint16_t* dV;
  float* stats;        // [2][H][q_rows]: log-sum-exp in base 2, then less sum_j P_ij (dO_i . V_j)
  const int32_t* q_ptr;   // [n_docs + 1]
  const int32_t* k_ptr;   // [n_docs + 1]
  const int32_t* prefix;  // [n_docs], or null
  int64_t q_stride, k_stride, v_stride, dq_stride, dk_stride, dv_stride;
  int32_t q_rows, k_rows, n_docs;
  int32_t H, Hkv;
  int32_t tile_heads;  // heads of a group that share a tile: 1, 2 or 4, a divisor of H / Hkv
  int32_t causal;
  float scale;
  Scoring scoring;
};

// `f16`: elements are IEEE half precision, otherwise bfloat16. head_dim: 64 or 128.
hipError_t launch_doc_forward(const DocAttnArgs& a, bool f16, int head_dim, hipStream_t stream);
hipError_t launch_doc_grad(const DocAttnArgs& a, bool f16, int head_dim, hipStream_t stream);

}  // namespace csg
