// Interface between the host runtime and the kernels of attention over packed documents.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

#include "attn_scores.hpp"

namespace csg {

constexpr int kDocTileRows = 128;  // keys of a tile of the keys' gradient: 4 waves of 32
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
  float* stats;        // [2][H][q_rows]: log-sum-exp in base 2 (f16: less 14), then less sum_j P_ij (dO_i . V_j)
  float* parts;        // [row_parts][k_rows][Hkv][2][D]: their sums (row_parts 1: none)
  const int32_t* q_ptr;   // [n_docs + 1]
  const int32_t* k_ptr;   // [n_docs + 1]
  const int32_t* prefix;  // [n_docs], or null
  int64_t q_stride, k_stride, v_stride, dq_stride, dk_stride, dv_stride;
  int32_t q_rows, k_rows, n_docs;
  int32_t H, Hkv;
  int32_t tile_heads;  // heads of a group that share a tile of rows: 1, 2 or 4, a divisor of H / Hkv
  int32_t causal;
  int32_t joined;      // gradient: o and lse are of more keys
  int32_t cus;         // of the device
  int32_t row_parts;   // parts into which the keys' gradient cuts its rows
  float scale;
  Scoring scoring;
};

// Tiles of keys, at most.
inline int64_t doc_key_tiles(int64_t k_rows, int64_t n_docs) { return k_rows / kDocTileRows + n_docs; }
// A tile of keys walks the rows of all heads of its group one after the other: where the tiles
// leave CUs idle, the rows are cut into parts, whose sums are added up in a kernel of their own.
// There is a part for every CU while each has four steps (documents being of the same length),
// and two for every workgroup that the CUs hold (one each, of heads of 64 two), which evens out the
// causal tiles, while each has 16; at most 16. The whole gradient, causal: 32 heads on 8 of 128, 512
// rows 106 -> 47 us (7 parts), 1024 rows 194 -> 82 (7), 3000 rows 457 -> 331 (2), 4096 rows 685 -> 540 (2), with
// half as many again 2048 rows 180 -> 198; 32 on 8 of 64, 8192 rows 1237 -> 1070 (2); but 16 documents of 250
// rows, 256 tiles of 16 steps of 128 elements, 110 -> 129 us with two parts.
constexpr int32_t kDocMaxParts = 16;
inline int64_t doc_steps(int64_t q_rows, int64_t n_docs, int32_t H, int32_t Hkv) {
  return (q_rows / (n_docs < 1 ? 1 : n_docs) + kDocBlock - 1) / kDocBlock * (H / Hkv);
}
// The most tiles of keys that are cut into that many parts (0: not even one is).
inline int64_t doc_part_tiles(int32_t parts, int64_t steps, int32_t head_dim, int32_t cus) {
  if (steps >= 16 * parts) return (head_dim == 64 ? 4 : 2) * static_cast<int64_t>(cus) / parts;
  return steps >= 4 * parts ? cus / parts : 0;
}
inline int32_t doc_row_parts(int64_t q_rows, int64_t k_rows, int64_t n_docs, int32_t H, int32_t Hkv, int32_t head_dim, int32_t cus) {
  const int64_t tiles = ((k_rows + kDocTileRows - 1) / kDocTileRows + n_docs / 2) * Hkv;
  const int64_t steps = doc_steps(q_rows, n_docs, H, Hkv);
  int32_t parts = 1;
  if (k_rows == 0) return parts;
  while (parts < kDocMaxParts && tiles <= doc_part_tiles(parts + 1, steps, head_dim, cus)) ++parts;
  return parts;
}
// Parts times their keys, 0 if there is one, at most, of any call of up to so many rows and keys. Fewer
// keys may be cut into more parts: for each number of parts, the most keys that have it.
inline int64_t doc_max_part_rows(int64_t q_rows, int64_t k_rows, int32_t H, int32_t Hkv, int32_t head_dim, int32_t cus) {
  const int64_t steps = doc_steps(q_rows, 1, H, Hkv);  // (fewer rows, or more documents: fewer steps)
  int64_t most = 0;
  for (int32_t parts = 2; parts <= kDocMaxParts; ++parts) {
    const int64_t keys = doc_part_tiles(parts, steps, head_dim, cus) / Hkv * kDocTileRows;
    const int64_t rows = parts * (keys < k_rows ? keys : k_rows);
    if (rows > most) most = rows;
  }
  return most;
}

// `f16`: elements are IEEE half precision, otherwise bfloat16. head_dim: 64 or 128.
hipError_t launch_doc_forward(const DocAttnArgs& a, bool f16, int head_dim, hipStream_t stream);
hipError_t launch_doc_grad(const DocAttnArgs& a, bool f16, int head_dim, hipStream_t stream);

}  // namespace csg
