// How products of queries and keys become scores, shared by host and device.
#pragma once

namespace csg {

struct Scoring {
  float scale;          // no cap: products to scores
  float cap_in;         // cap c: products to twice tanh's argument in base 2: 2 scale log2 e / c
  float cap;            // c; 0: no cap
  const float* slopes;  // [n_heads], or null
  bool plain() const { return cap == 0.0f && !slopes; }
};

}  // namespace csg
