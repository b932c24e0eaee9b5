// Device pieces shared by the attention kernels over documents and over a paged cache:
// element types, LDS tiles of rows, the loads that fill them, fragments, and scores.
//
// Matrix products are v_mfma_f32_32x32x16: the first operand's lane (l32 = lane % 32, hlf =
// lane / 32) holds row l32, inner positions 8 hlf .. + 7; the second operand's lane holds
// column l32, the same inner positions; the result's lane holds column l32, rows
// 8 (r / 4) + 4 hlf + r % 4 for its registers r = 0 .. 15.
//
// A tile holds rows of D elements, unpadded, and serves both kinds of fragments:
//   row fragments (16 bytes of one row per lane: products that sum over the D elements),
//   column fragments (products that sum over the rows), by transposing reads.
// The 16-byte piece p of row R sits at piece p ^ swz(R) of the row. With r0 .. r3 the low
// bits of R, swz is (r1, r0, r1 ^ r3, r2) for D = 128 and (r1, r0 ^ r3, r2) for D = 64, the
// first of them the highest bit. A row fragment read touches 16 consecutive rows at one p:
// 16 (D = 64: 8, each at two rows of different halves of 256 bytes) distinct places; a
// transposing read 4 consecutive rows x 2 or 4 neighbouring pieces: the two highest bits
// (D = 64: the row's half and the highest) are distinct over r0, r1. Neither has bank
// conflicts, with 32 or with 64 banks.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

#include "attn_scores.hpp"

namespace csg {
namespace tile {

typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x4_t __attribute__((ext_vector_type(4)));
typedef _Float16 f16x8_t __attribute__((ext_vector_type(8)));
typedef _Float16 f16x4_t __attribute__((ext_vector_type(4)));
typedef float f32x16_t __attribute__((ext_vector_type(16)));
typedef float f32x8_t __attribute__((ext_vector_type(8)));
typedef float f32x4_t __attribute__((ext_vector_type(4)));
typedef unsigned int u32x4_t __attribute__((ext_vector_type(4)));
typedef unsigned int u32x2_t __attribute__((ext_vector_type(2)));
typedef short i16x4_t __attribute__((ext_vector_type(4)));
typedef short i16x8_t __attribute__((ext_vector_type(8)));
typedef __attribute__((address_space(3))) void* lds_ptr_t;
typedef __attribute__((address_space(3))) unsigned char lds_u8_t;
typedef __attribute__((address_space(3))) i16x4_t lds_i16x4_t;

constexpr int kBufferDword3 = 0x00020000;  // raw buffer resource word 3 (gfx9 family)
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;

struct Bf16 {
  using x8 = bf16x8_t;
  using x4 = bf16x4_t;
  // Largest sum of a row's weights in one block that is taken against the running
  // reference; a larger one moves the reference to the row's maximum. Weights stay exact
  // to their type's 8 bits at any size.
  static constexpr float kRowSumLimit = 65536.0f;
  static constexpr bool kShortRange = false;
  static __device__ __forceinline__ f32x16_t mfma(x8 a, x8 b, f32x16_t c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
  }
};

struct F16 {
  using x8 = f16x8_t;
  using x4 = f16x4_t;
  // (the type ends at 65504, and what is below 2^-14 loses bits: weights stay near 1)
  static constexpr float kRowSumLimit = 1024.0f;
  static constexpr bool kShortRange = true;
  static __device__ __forceinline__ f32x16_t mfma(x8 a, x8 b, f32x16_t c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0);
  }
};

template <int D>
__device__ __forceinline__ constexpr int swz(int r) {
  const int r0 = r & 1, r1 = (r >> 1) & 1, r2 = (r >> 2) & 1, r3 = (r >> 3) & 1;
  return D == 128 ? (r1 << 3) | (r0 << 2) | ((r1 ^ r3) << 1) | r2 : (r1 << 2) | ((r0 ^ r3) << 1) | r2;
}

// Buffer resource over [base, base + bytes): reads beyond it give zero. Built from values
// that are the same in every lane, so that it lives in SGPRs.
__device__ __forceinline__ __amdgpu_buffer_rsrc_t make_rsrc(const void* base, int bytes) {
  const uint64_t p = reinterpret_cast<uint64_t>(base);
  const uint32_t lo = __builtin_amdgcn_readfirstlane(static_cast<uint32_t>(p));
  const uint32_t hi = __builtin_amdgcn_readfirstlane(static_cast<uint32_t>(p >> 32));
  void* ub = reinterpret_cast<void*>((static_cast<uint64_t>(hi) << 32) | lo);
  return __builtin_amdgcn_make_buffer_rsrc(ub, 0, __builtin_amdgcn_readfirstlane(bytes), kBufferDword3);
}

__device__ __forceinline__ uint32_t lds_address(const void* p) {
  return __builtin_amdgcn_readfirstlane(static_cast<uint32_t>(reinterpret_cast<uintptr_t>((lds_ptr_t)p)));
}

// One 16-byte-per-lane load of 1 KiB into LDS at lds (lane l: byte 16 l), from byte voff of
// the resource. In inline asm (M0 saved and restored), so that the compiler does not wait for
// it before every LDS read: the caller waits (wait_vm) before the tile is read. A load to LDS
// may read M0 no sooner than one instruction after it was written (s_nop), and the compiler
// does not look for such pairs inside of asm.
__device__ __forceinline__ void load_to_lds(__amdgpu_buffer_rsrc_t rs, uint32_t lds, int voff) {
  uint32_t saved;
  asm volatile(
      "s_mov_b32 %0, m0\n\t"
      "s_mov_b32 m0, %1\n\t"
      "s_nop 0\n\t"
      "buffer_load_dwordx4 %2, %3, 0 offen lds\n\t"
      "s_mov_b32 m0, %0"
      : "=&s"(saved)
      : "s"(lds), "v"(voff), "s"(rs)
      : "memory");
}

// The same with 4 bytes per lane.
__device__ __forceinline__ void load_dword_to_lds(__amdgpu_buffer_rsrc_t rs, uint32_t lds, int voff) {
  uint32_t saved;
  asm volatile(
      "s_mov_b32 %0, m0\n\t"
      "s_mov_b32 m0, %1\n\t"
      "s_nop 0\n\t"
      "buffer_load_dword %2, %3, 0 offen lds\n\t"
      "s_mov_b32 m0, %0"
      : "=&s"(saved)
      : "s"(lds), "v"(voff), "s"(rs)
      : "memory");
}

template <int n>
__device__ __forceinline__ void wait_vm() {
  asm volatile("s_waitcnt vmcnt(%0)" ::"n"(n) : "memory");
}

__device__ __forceinline__ void wait_lds() { asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory"); }

// The values, loaded by ordinary loads, are there. To be called ahead of a loop that only
// uses them: the compiler, which does not see the loads to LDS, would otherwise wait before
// their use in each turn until nothing is in flight, the tiles that the turn has just asked for included.
template <class X8, int N>
__device__ __forceinline__ void arrived(X8 (&f)[N]) {
#pragma unroll
  for (int s = 0; s < N; ++s) {
    u32x4_t raw = __builtin_bit_cast(u32x4_t, f[s]);
    asm volatile("" : "+v"(raw));
    f[s] = __builtin_bit_cast(X8, raw);
  }
}
__device__ __forceinline__ float arrived(float x) {
  asm volatile("" : "+v"(x));
  return x;
}

// Rows one load_to_lds fills (1 KiB), and the loads of a tile of `rows` rows.
template <int D>
constexpr int kLoadRows = 512 / D;

// A lane's part of a tile's loads. Load i fills rows kLoadRows i .. + kLoadRows - 1; the lane
// brings the piece of row kLoadRows i + row that belongs at its place. The row's low four
// bits take bit 2 and 3 (D = 64: bit 3) from i, which turns the piece by an XOR that is the
// same in every lane.
template <int D>
struct LoadLane {
  int row, piece;
  __device__ __forceinline__ explicit LoadLane(int lane) {
    constexpr int kPieces = D / 8;
    row = lane / kPieces;
    piece = (lane % kPieces) ^ swz<D>(row);
  }
  // byte offset in the source of what load i brings, rows `stride` bytes apart
  __device__ __forceinline__ int offset(int i, int stride) const {
    const int turn = swz<D>(kLoadRows<D> * (i % (16 / kLoadRows<D>)));
    return (kLoadRows<D> * i + row) * stride + 16 * (piece ^ turn);
  }
};

// Lane offsets of the fragments of a tile whose rows follow each other in LDS.
template <int D>
struct Frags {
  int row[D / 16];      // row fragment s: elements 16 s + 8 hlf .. + 7 of row l32
  int col[D / 32][2];   // column fragments: see cols()
  __device__ __forceinline__ explicit Frags(int lane) {
    const int l32 = lane & 31, hlf = lane >> 5;
#pragma unroll
    for (int s = 0; s < D / 16; ++s) row[s] = 2 * D * l32 + 16 * ((2 * s + hlf) ^ swz<D>(l32));
    // ds_read_b64_tr_b16 transposes 4 x 16 blocks among each 16 lanes: lane i points at
    // row k0 + i / 4, elements d0 + 4 (i % 4) .. + 3, and receives element d0 + i of rows
    // k0 .. k0 + 3. Rows 4 hlf + 0..3 (first read) and 8 + 4 hlf + 0..3 (second).
    const int i = lane & 15, h = (lane >> 4) & 1;
#pragma unroll
    for (int db = 0; db < D / 32; ++db)
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const int r = 8 * e + 4 * hlf + (i >> 2);
        col[db][e] = 2 * D * r + 16 * ((4 * db + 2 * h + ((i & 3) >> 1)) ^ swz<D>(r)) + 8 * (i & 1);
      }
  }
};

// Row fragment s of rows r0 .. r0 + 31 (r0 a multiple of 16) of a tile.
template <class T, int D>
__device__ __forceinline__ typename T::x8 row_frag(const unsigned char* t, const Frags<D>& f, int s, int r0) {
  return *reinterpret_cast<const typename T::x8*>(t + f.row[s] + 2 * D * r0);
}

// Column fragment: elements 32 db + l32 of rows r0 .. r0 + 15, as first operand, the rows in
// the order in which a result's registers 0 .. 7 (or 8 .. 15, for r0 + 16) list them.
template <class T, int D>
__device__ __forceinline__ typename T::x8 col_frag(const lds_u8_t* t, const Frags<D>& f, int db, int r0) {
  const i16x4_t lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4_t*)(t + f.col[db][0] + 2 * D * r0));
  const i16x4_t hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4_t*)(t + f.col[db][1] + 2 * D * r0));
  return __builtin_bit_cast(typename T::x8, (i16x8_t{lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]}));
}

// Registers 8 t .. 8 t + 7 of a result, rounded, as second operand (the order of col_frag).
template <class T>
__device__ __forceinline__ typename T::x8 pack(const f32x16_t& x, int t) {
  f32x8_t w;
#pragma unroll
  for (int r = 0; r < 8; ++r) w[r] = x[8 * t + r];
  return __builtin_convertvector(w, typename T::x8);
}

// Combination with lane ^ 32 (the other half of a row) by v_permlane32_swap: swapping the
// halves of two copies of x leaves x of both lanes in each, without an LDS round trip.
__device__ __forceinline__ float max_halves(float x) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float sum_halves(float x) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

// Row of a tile that a result's register r holds in this lane.
__device__ __forceinline__ constexpr int result_row(int r, int hlf) { return 8 * (r >> 2) + 4 * hlf + (r & 3); }

// tanh(x) = 1 - 2 / (1 + e^(2x)) from y = 2 x log2 e; off by 2^-22 at most, and +-1 where e^(2x)
// overflows or vanishes.
__device__ __forceinline__ float tanh_from_log2(float y) {
  return 1.0f - 2.0f * __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(y));
}
// The same, off by 2^-20 of itself at most: below 0.3 by the series
// x - x^3/3 + 2 x^5/15 - 17 x^7/315 + 62 x^9/2835, whose next term is 5e-8 of it there.
__device__ __forceinline__ float tanh_from_log2_near_0(float y) {
  const float x = y * (0.5f * kLn2), z = x * x;
  const float p = fmaf(z, fmaf(z, fmaf(z, fmaf(z, 62.0f / 2835.0f, -17.0f / 315.0f), 2.0f / 15.0f), -1.0f / 3.0f), 1.0f) * x;
  return fabsf(x) < 0.3f ? p : tanh_from_log2(y);
}
// Caps up to this take the short form: a score is off by 2^-22 times the cap, 1.5e-5 at 64, which is nothing
// beside the rounding of weights. Larger ones would lose their small scores' digits (0.1 at a cap of 1e6).
constexpr float kNearCap = 64.0f;

// A head's slope in units of x.
__device__ __forceinline__ float slope_of(const Scoring& p, int h) { return p.slopes ? p.slopes[h] / p.unit : 0.0f; }

// Products of N tiles to x, where the scores are not plain. `at`: what stands at the tile's row
// (or column) of register 0, lane hlf 0, less the other side's place; `sign`: it counts down
// (-1: keys in the registers) or up (1: rows) with the tile's rows.
template <int N>
__device__ __forceinline__ void cap_scores(const Scoring& p, f32x16_t (&x)[N]) {
  if (p.cap_in == 0.0f) return;
  if (p.unit <= kNearCap) {
#pragma unroll
    for (int n = 0; n < N; ++n)
#pragma unroll
      for (int r = 0; r < 16; ++r) x[n][r] = tanh_from_log2(x[n][r] * p.cap_in);
  } else {
#pragma unroll
    for (int n = 0; n < N; ++n)
#pragma unroll
      for (int r = 0; r < 16; ++r) x[n][r] = tanh_from_log2_near_0(x[n][r] * p.cap_in);
  }
}
template <int N, int sign>
__device__ __forceinline__ void bias_scores(const Scoring& p, float slope, int at, int hlf, f32x16_t (&x)[N]) {
  if (!p.slopes) return;
  const float from = static_cast<float>(at + sign * 4 * hlf);
#pragma unroll
  for (int n = 0; n < N; ++n)
#pragma unroll
    for (int r = 0; r < 16; ++r) x[n][r] = fmaf(-slope, fabsf(from + sign * static_cast<float>(32 * n + result_row(r, 0))), x[n][r]);
}

// A row's softmax so far, over blocks of N tiles of 32 keys each. x weighs 2^(c (x - m)), c =
// unit log2 e. The reference m moves to the row's largest x only where a block's weights would leave their
// range; on the first block, where it is -inf, and as long as every score is -inf, always.
// Both lanes of a row see the same sums and maxima, so they keep the same reference.
struct RowSoftmax {
  float m = -__builtin_inff();
  float mc = -__builtin_inff();  // c m
  float l = 0.0f;                // this lane's weights, summed before they are rounded
  bool wide = false;             // the row's c m may overflow: c x - c m would lose its weights

  // Weights of one block, rounded, as second operand of the value product, and the factor
  // by which what was summed before has to be multiplied if `moved`.
  template <class T, int N>
  __device__ __forceinline__ float block(const f32x16_t (&x)[N], float c, typename T::x8 (&pb)[2 * N], bool& moved) {
    float sum = weights<T, N, false>(x, c, mc, pb);
    const bool move = wide || !(sum_halves(sum) <= T::kRowSumLimit);
    float alpha = 1.0f;
    moved = __builtin_amdgcn_ballot_w64(move) != 0;
    if (moved) {
      float mx = -__builtin_inff();
#pragma unroll
      for (int n = 0; n < N; ++n)
#pragma unroll
        for (int r = 0; r < 16; ++r) mx = fmaxf(mx, x[n][r]);
      mx = max_halves(mx);
      const float to = move ? fmaxf(m, mx) : m;
      const bool none = to == -__builtin_inff();  // against -inf the weights would be NaN: they are 0
      alpha = m == -__builtin_inff() ? 0.0f : __builtin_amdgcn_exp2f((m - to) * c);
      m = to;
      mc = m * c;
      wide = !none && fabsf(mc) > 1e37f;
      l *= alpha;
      sum = weights<T, N, true>(x, c, none ? 0.0f : mc, pb, none ? 0.0f : m, wide);
    }
    l += sum;
    return alpha;
  }

 private:
  // (A row that stays takes the same weights on both paths: its result is its own, whatever the
  // wave's other rows hold.)
  template <class T, int N, bool kAgain>
  static __device__ __forceinline__ float weights(const f32x16_t (&x)[N], float c, float refc, typename T::x8 (&pb)[2 * N],
                                                  float ref = 0.0f, bool far = false) {
    float sum = 0.0f;
#pragma unroll
    for (int t = 0; t < 2 * N; ++t) {
      f32x8_t w;
#pragma unroll
      for (int r = 0; r < 8; ++r) {
        const float v = x[t >> 1][8 * (t & 1) + r];
        w[r] = __builtin_amdgcn_exp2f(kAgain && far ? (v - ref) * c : fmaf(v, c, -refc));
        sum += w[r];
      }
      pb[t] = __builtin_convertvector(w, typename T::x8);
    }
    return sum;
  }
};

// What sums against reference m count against reference top; nothing if they saw no key.
__device__ __forceinline__ float factor(float m, float top, float c) {
  return m == -__builtin_inff() ? 0.0f : __builtin_amdgcn_exp2f((m - top) * c);
}

// The last d of 0 .. n - 1 with below(d), which holds for the first few only (0 if for none),
// searched by a whole wave: 64 entries a turn.
template <class F>
__device__ __forceinline__ int last_below(int n, F below) {
  const int lane = threadIdx.x & 63;
  int lo = 0, len = n;  // the entry lies in lo .. lo + len - 1
  while (len > 1) {
    const int stride = (len + 63) / 64;
    const int at = lane * stride;
    const uint64_t m = __builtin_amdgcn_ballot_w64(at < len && below(lo + at));
    const int last = m ? 63 - __builtin_clzll(m) : 0;
    lo += last * stride;
    len = min(stride, len - last * stride);
  }
  return __builtin_amdgcn_readfirstlane(lo);
}

__device__ __forceinline__ int clamped(int x, int lo, int hi) { return x < lo ? lo : x > hi ? hi : x; }

}  // namespace tile
}  // namespace csg
