// How products of queries and keys become scores, shared by host and device.
#pragma once

namespace csg {

// A score is unit times x, where x is the product less a distance's share, or with a cap (unit
// is the cap) tanh of the product's share less that of the distance. Kernels keep x: the unit
// goes into the factor of the exponent.
struct Scoring {
  float unit;           // softmax scale; cap c: c
  float cap_in;         // cap: products to twice tanh's argument in base 2: 2 scale log2 e / c; 0: no cap
  const float* slopes;  // [n_heads], or null
  bool plain() const { return cap_in == 0.0f && !slopes; }
};

}  // namespace csg
