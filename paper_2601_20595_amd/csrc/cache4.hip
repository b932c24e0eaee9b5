// A paged key/value cache in 4 bits for gfx950 (CDNA4): new tokens go in, rows come out, attention
// reads it. Pages, tables and lengths are those of the cache in 16 bits.
//
// An element is a sign and one of 0, 0.5, 1, 1.5, 2, 3, 4, 6 (e2m1, in the order of its code); each 32
// elements of a head share a scale 2^e, held as the byte e + 127 (e8m0): the OCP microscaling format
// MXFP4, whose conversions the hardware has. e is the least with |x| <= 7 2^e in the block: what
// lies between 6 and 7 is off by no more than half the step above 4, as a rounding is; with the largest
// element below 8 2^e instead, an element of 7.9 would be off by 1.9.
// e is held within what leaves every value a normal number of bf16 (-125 .. 125), or exact in f16
// (-23 .. 13). A head's rows of a page lie behind each other, elements 2 i and 2 i + 1 in the low and the
// high half of byte i, and the page's scales behind them.
#include <hip/hip_runtime.h>

#include "cache4.hpp"
#include "cache_plan.hpp"

namespace csg {
namespace {

using namespace cache;

typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));
typedef _Float16 f16x2_t __attribute__((ext_vector_type(2)));

template <class T>
struct Four;  // conversions between T and 4 bits, and the limits of the scales' bytes
template <>
struct Four<Bf16> {
  static constexpr int kLeast = 127 - 125, kMost = 127 + 125;
  template <int byte>
  static __device__ __forceinline__ uint32_t from(uint32_t codes, float scale) {
    return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, byte));
  }
  template <int byte>
  static __device__ __forceinline__ uint32_t to(uint32_t old, uint32_t pair, float scale) {
    return __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(old, __builtin_bit_cast(bf16x2_t, pair), scale, byte);
  }
  static __device__ __forceinline__ float widen(uint32_t bits) { return __uint_as_float(bits << 16); }
};
template <>
struct Four<F16> {
  static constexpr int kLeast = 127 - 23, kMost = 127 + 13;
  template <int byte>
  static __device__ __forceinline__ uint32_t from(uint32_t codes, float scale) {
    return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(codes, scale, byte));
  }
  template <int byte>
  static __device__ __forceinline__ uint32_t to(uint32_t old, uint32_t pair, float scale) {
    return __builtin_amdgcn_cvt_scalef32_pk_fp4_f16(old, __builtin_bit_cast(f16x2_t, pair), scale, byte);
  }
  static __device__ __forceinline__ float widen(uint32_t bits) {
    return static_cast<float>(__builtin_bit_cast(_Float16, static_cast<uint16_t>(bits)));
  }
};

constexpr uint32_t kNanScale = 255;  // (the format's)

// The factor that a scale's byte stands for.
__device__ __forceinline__ float scale_of(uint32_t byte) {
  return __uint_as_float(byte == kNanScale ? 0x7fc00000u : byte << 23);
}

// Eight elements from their codes, of one block.
template <class T>
__device__ __forceinline__ u32x4_t values(uint32_t codes, float scale) {
  return u32x4_t{Four<T>::template from<0>(codes, scale), Four<T>::template from<1>(codes, scale),
                 Four<T>::template from<2>(codes, scale), Four<T>::template from<3>(codes, scale)};
}

// Bytes of a head's rows of a page, and where they begin.
template <int D>
__device__ __forceinline__ int64_t head_bytes(const CacheArgs& c) {
  return static_cast<int64_t>(cache4_row_bytes(D)) << c.page_shift;
}
template <int D>
__device__ __forceinline__ int64_t head_of(const CacheArgs& c, int page, int kvh) {
  return (static_cast<int64_t>(page) * c.Hkv + kvh) * head_bytes<D>(c);
}

// ---- new tokens into the cache --------------------------------------------------------------
// A workgroup per token, as in the cache of 16 bits; but keys are rotated in 64 bits (sines and cosines
// once a token, 6 operations a pair and head), so that what they are rounded to, next to a border too, does not depend on
// the order of a kernel's operations: to 32 bits (which the conversions to T take), from there to T, and to a code. The
// step through 32 bits is part of the definition: where it ends halfway between two numbers of T (one result in 2^16, f16:
// 2^13), a single rounding may take the other one. Eight
// lanes (D = 64: four) have a head; its rotated elements go through LDS, since a block's elements come from
// pairs of two places, and two lanes quantise a block. 64 tokens of 32 query heads on 8 of 128 take 4.6 us, a chain of latencies;
// 11322 of 64 on 8, 426 MB, 90 us, 4.7 TB/s (a large copy: 5.1).
template <class T, int D>
__global__ __launch_bounds__(kThreads) void cache4_append(AppendArgs a) {
  constexpr int kCols = D / 16, kHeads = kThreads / kCols;
  __shared__ double s_cos[D / 2], s_sin[D / 2];
  __shared__ __attribute__((aligned(16))) uint16_t s_row[kHeads][D];
  const CacheArgs& c = a.c;
  const int t = blockIdx.x;
  if (t < first_token(c, 0) || t >= first_token(c, c.batch)) return;  // (a row of no sequence)
  const int b = last_below(c.batch, [&](int i) { return c.q_ptr[i] <= t; });
  const int pos = c.lens[b] - (c.q_ptr[b + 1] - t);
  const int slot = pos >> c.page_shift;
  int page = -1;
  if (pos < 0 || slot >= c.max_pages) {
    if (threadIdx.x == 0) tell(c, kCacheBadLength);
  } else {
    page = c.table[static_cast<int64_t>(b) * c.max_pages + slot];
    if (page < 0 || page >= c.n_pages) {
      page = -1;
      if (threadIdx.x == 0) tell(c, kCacheBadPage);
    }
  }
  if (static_cast<int>(threadIdx.x) < a.half) {
    double sn, cs;
    sincos(static_cast<double>(pos) * a.inv_freq[threadIdx.x], &sn, &cs);
    s_cos[threadIdx.x] = cs;
    s_sin[threadIdx.x] = sn;
  }
  __syncthreads();
  const int lane_head = threadIdx.x / kCols, col = threadIdx.x % kCols;
  const bool turns = 8 * col < a.half;
  const bool split = turns && !a.interleaved;
  const int x0 = split ? 8 * col : 16 * col, x1 = split ? a.half + 8 * col : 16 * col + 8;
  if (c.Q) {
    float cs[8], sn[8];
    if (turns) {
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        cs[e] = static_cast<float>(s_cos[8 * col + e]);
        sn[e] = static_cast<float>(s_sin[8 * col + e]);
      }
    }
    for (int i = lane_head; i < c.H; i += kHeads) {
      const uint16_t* src = c.Q + t * c.q_stride + i * D;
      uint16_t* dst = a.q_out + (static_cast<int64_t>(t) * c.H + i) * D;
      const typename T::x8 y[2] = {*reinterpret_cast<const typename T::x8*>(src + x0), *reinterpret_cast<const typename T::x8*>(src + x1)};
      f32x8_t z[2] = {__builtin_convertvector(y[0], f32x8_t), __builtin_convertvector(y[1], f32x8_t)};
      if (turns) {
        if (split) {
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            const float u = z[0][e], v = z[1][e];
            z[0][e] = fmaf(u, cs[e], -v * sn[e]);
            z[1][e] = fmaf(v, cs[e], u * sn[e]);
          }
        } else {
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            const float u = z[e / 4][2 * (e & 3)], v = z[e / 4][2 * (e & 3) + 1];
            z[e / 4][2 * (e & 3)] = fmaf(u, cs[e], -v * sn[e]);
            z[e / 4][2 * (e & 3) + 1] = fmaf(v, cs[e], u * sn[e]);
          }
        }
      }
      // (a head that is not turned keeps its bits: the type's own values are exact in 32 bits)
      *reinterpret_cast<typename T::x8*>(dst + x0) = turns ? __builtin_convertvector(z[0], typename T::x8) : y[0];
      *reinterpret_cast<typename T::x8*>(dst + x1) = turns ? __builtin_convertvector(z[1], typename T::x8) : y[1];
    }
  }
  if (page < 0) return;
  const int row = pos & ((1 << c.page_shift) - 1);
  for (int i = lane_head; i < 2 * c.Hkv; i += kHeads) {
    const bool is_v = i >= c.Hkv;
    const int h = i - (is_v ? c.Hkv : 0);
    const uint16_t* src = (is_v ? a.V + t * a.v_stride : a.K + t * a.k_stride) + h * D;
    u32x4_t w[2];  // elements 16 col .. + 15
    if (is_v || a.half == 0) {
      w[0] = *reinterpret_cast<const u32x4_t*>(src + 16 * col);
      w[1] = *reinterpret_cast<const u32x4_t*>(src + 16 * col + 8);
    } else {
      uint16_t* mine = s_row[lane_head];
      typename T::x8 y[2] = {*reinterpret_cast<const typename T::x8*>(src + x0), *reinterpret_cast<const typename T::x8*>(src + x1)};
      if (turns) {
        f32x8_t z[2];
        auto turn = [&](int e, float x, float y, float& u, float& v) {
          const double cs = s_cos[8 * col + e], sn = s_sin[8 * col + e];
          u = static_cast<float>(x * cs - y * sn);
          v = static_cast<float>(y * cs + x * sn);
        };
        float u, v;
        if (split) {
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            turn(e, static_cast<float>(y[0][e]), static_cast<float>(y[1][e]), u, v);
            z[0][e] = u;
            z[1][e] = v;
          }
        } else {
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            turn(e, static_cast<float>(y[e / 4][2 * (e & 3)]), static_cast<float>(y[e / 4][2 * (e & 3) + 1]), u, v);
            z[e / 4][2 * (e & 3)] = u;
            z[e / 4][2 * (e & 3) + 1] = v;
          }
        }
        y[0] = __builtin_convertvector(z[0], typename T::x8);
        y[1] = __builtin_convertvector(z[1], typename T::x8);
      }
      *reinterpret_cast<u32x4_t*>(mine + x0) = __builtin_bit_cast(u32x4_t, y[0]);
      *reinterpret_cast<u32x4_t*>(mine + x1) = __builtin_bit_cast(u32x4_t, y[1]);
      // the lanes of a head are of one wave, whose LDS accesses are done in order
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
      __builtin_amdgcn_wave_barrier();
      w[0] = *reinterpret_cast<const u32x4_t*>(mine + 16 * col);
      w[1] = *reinterpret_cast<const u32x4_t*>(mine + 16 * col + 8);
      __builtin_amdgcn_wave_barrier();
    }
    // the largest absolute value, compared as bits (a NaN is larger than all)
    uint32_t top = 0;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const uint32_t pair = w[j / 4][j % 4];
      top = max(top, max(pair & 0x7fffu, pair >> 16 & 0x7fffu));
    }
    top = max(top, __shfl_xor(top, 1));
    const uint32_t wide = __float_as_uint(Four<T>::widen(top));
    // m 2^k with 1 <= m < 2: e = k - 2 up to m = 1.75, k - 1 beyond
    const int e = static_cast<int>((wide + 0x1fffffu) >> 23) - 2;
    const bool none = wide >= 0x7f800000u;
    const uint32_t byte = none ? kNanScale : static_cast<uint32_t>(clamped(e, Four<T>::kLeast, Four<T>::kMost));
    const float scale = __uint_as_float(byte << 23);
    u32x2_t codes{0u, 0u};
    if (!none) {
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        codes[j] = Four<T>::template to<0>(codes[j], w[j][0], scale);
        codes[j] = Four<T>::template to<1>(codes[j], w[j][1], scale);
        codes[j] = Four<T>::template to<2>(codes[j], w[j][2], scale);
        codes[j] = Four<T>::template to<3>(codes[j], w[j][3], scale);
      }
    }
    unsigned char* head = reinterpret_cast<unsigned char*>(is_v ? c.v_pages : c.k_pages) + head_of<D>(c, page, h);
    *reinterpret_cast<u32x2_t*>(head + row * (D / 2) + 8 * col) = codes;
    if (col % 2 == 0) head[((D / 2) << c.page_shift) + row * (D / 32) + col / 2] = static_cast<unsigned char>(byte);
  }
}

// ---- rows out of the cache ------------------------------------------------------------------
// A workgroup has kReadRows rows of some heads, keys and values. D / 8 lanes have a row: 4 bytes in, 16 bytes out; the
// rows of a page lie behind each other, and so do the heads of the output's rows. Bound by the memory: 115000 tokens of
// 2 x 8 heads of 128, 603 MB in 125 us, 4.8 TB/s (a large copy: 5.1). With a head a workgroup 162 us, with ordinary stores
// 130, with 64 or 128 rows a workgroup 138.
template <class T, int D>
__global__ __launch_bounds__(kThreads) void cache4_read(ReadArgs a) {
  constexpr int kLanes = D / 8, kAtOnce = kThreads / kLanes, kTurns = kReadRows / kAtOnce;
  static_assert(kReadRows % kAtOnce == 0, "whole turns");
  __shared__ int s_page[kReadRows], s_row[kReadRows];
  const CacheArgs& c = a.c;
  const int groups = c.Hkv / a.heads, row0 = blockIdx.x / groups * kReadRows, head0 = blockIdx.x % groups * a.heads;
  if (threadIdx.x < kReadRows) {
    const int t = row0 + threadIdx.x;
    int page = -1, row = -1;  // row -1: a row of no sequence
    if (t >= first_token(c, 0) && t < first_token(c, c.batch)) {
      int b = 0;
      for (int n = c.batch; n > 1;) {  // the last sequence that starts by then
        const int half = n / 2;
        const bool up = c.q_ptr[b + half] <= t;
        b = up ? b + half : b;
        n = up ? n - half : half;
      }
      const int pos = c.lens[b] - (c.q_ptr[b + 1] - t);
      const int slot = pos >> c.page_shift;
      row = pos & ((1 << c.page_shift) - 1);
      if (pos < 0 || slot >= c.max_pages) {
        tell(c, kCacheBadLength);
      } else {
        page = c.table[static_cast<int64_t>(b) * c.max_pages + slot];
        if (page < 0 || page >= c.n_pages) {
          page = -1;
          tell(c, kCacheBadPage);
        }
      }
    }
    s_page[threadIdx.x] = page;
    s_row[threadIdx.x] = row;
  }
  __syncthreads();
  const int col = threadIdx.x % kLanes, lane_row = threadIdx.x / kLanes;
#pragma unroll
  for (int i = 0; i < kTurns; ++i) {
    const int at = lane_row + i * kAtOnce;
    const int page = s_page[at], row = s_row[at];
    if (row < 0) continue;
    const int64_t from = head_of<D>(c, max(page, 0), head0) + row * (D / 2) + 4 * col;
    const int64_t scale_from = head_of<D>(c, max(page, 0), head0) + ((D / 2) << c.page_shift) + row * (D / 32) + col / 4;
    uint16_t* const k_to = a.K + (row0 + at) * a.k_stride + head0 * D + 8 * col;
    uint16_t* const v_to = a.V + (row0 + at) * a.v_stride + head0 * D + 8 * col;
    const unsigned char* const k_from = reinterpret_cast<const unsigned char*>(c.k_pages);
    const unsigned char* const v_from = reinterpret_cast<const unsigned char*>(c.v_pages);
#pragma unroll 4
    for (int h = 0; h < a.heads; ++h) {
      const int64_t skip = h * head_bytes<D>(c);
      u32x4_t k{0u, 0u, 0u, 0u}, v{0u, 0u, 0u, 0u};
      if (page >= 0) {
        k = values<T>(*reinterpret_cast<const uint32_t*>(k_from + from + skip), scale_of(k_from[scale_from + skip]));
        v = values<T>(*reinterpret_cast<const uint32_t*>(v_from + from + skip), scale_of(v_from[scale_from + skip]));
      }
      // (past the caches, which the codes and the tables need)
      __builtin_nontemporal_store(k, reinterpret_cast<u32x4_t*>(k_to + h * D));
      __builtin_nontemporal_store(v, reinterpret_cast<u32x4_t*>(v_to + h * D));
    }
  }
}

// ---- attention over the cache ---------------------------------------------------------------
// Entries, tasks and runs are those of the cache in 16 bits (cache_plan.hpp), and so are the parts, which
// its cache_merge joins. Codes become 16-bit numbers in registers, two an instruction, exactly: products and roundings are
// those of attention over the same values in 16 bits.
// With a quarter of the bytes, what is done for a key counts: a key of 4 rows costs its SIMD as much in products of 32 rows
// as in those of 16 twice over, so that up to 16 rows are one tile here. Bound by the memory where keys are many: 2
// sequences of over 100000, 244 MB in 51 us and the join 7, 4.8 TB/s (with 32-row products and every key through LDS 134);
// 64 sequences of up to 8000, 129 MB, 34 and 5, of which the plan, the first loads and the last parts' ends are 8. With few
// keys by a chain of latencies, 7.7 us for 900 keys. Where 16 sequences' rows share up to 8192 keys by the beginnings and ends of
// wide parts and their 26 MB of partial results (30 and 9); a wide block of 64 keys takes 2.3 us beside another workgroup's, 0.93 PFLOP/s.

// Combination of the four lanes of a row: lane ^ 16, then lane ^ 32, swapped as in max_halves.
__device__ __forceinline__ float max_quarters(float x) {
  const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return max_halves(fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1])));
}
__device__ __forceinline__ float sum_quarters(float x) {
  const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return sum_halves(__uint_as_float(r[0]) + __uint_as_float(r[1]));
}

// RowSoftmax for rows of four lanes, N / 4 tiles of 16 keys at a time. Weights are rounded to T, which the products with the values take; their
// sum is of 32 bits, before that rounding, so that the log-sum-exp has none of it (outputs of 64 sequences are off by 0.0021 of their
// size in bf16, with weights of 32 bits by 0.0017). The reference moves where one of the row's lanes finds
// its weights' sum beyond the limit: until then the lanes need not know each other's.
struct QuarterSoftmax {
  float m = -__builtin_inff();
  float mc = -__builtin_inff();
  float l = 0.0f;
  bool wide = false;

  template <class T, int N>
  __device__ __forceinline__ float block(const float (&x)[N], float c, int l16, typename T::x8 (&pb)[N / 8], bool& moved) {
    float sum = weights<T, N, false>(x, c, mc, pb);
    const uint64_t beyond = __builtin_amdgcn_ballot_w64(wide || !(sum <= T::kRowSumLimit));
    moved = beyond != 0;
    float alpha = 1.0f;
    if (moved) {
      const bool move = (beyond >> l16 & 0x0001000100010001ull) != 0;
      float mx = x[0];
#pragma unroll
      for (int r = 1; r < N; ++r) mx = fmaxf(mx, x[r]);
      mx = max_quarters(mx);
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
  template <class T, int N, bool kAgain>
  static __device__ __forceinline__ float weights(const float (&x)[N], float c, float refc, typename T::x8 (&pb)[N / 8], float ref = 0.0f,
                                                  bool far = false) {
    float sum = 0.0f;
#pragma unroll
    for (int t = 0; t < N / 8; ++t) {
      f32x8_t w;
#pragma unroll
      for (int r = 0; r < 8; ++r) {
        const float v = x[8 * t + r];
        w[r] = __builtin_amdgcn_exp2f(kAgain && far ? (v - ref) * c : fmaf(v, c, -refc));
        sum += w[r];
      }
      pb[t] = __builtin_convertvector(w, typename T::x8);
    }
    return sum;
  }
};

template <class T>
struct Mfma16;
template <>
struct Mfma16<Bf16> {
  static __device__ __forceinline__ f32x4_t run(bf16x8_t a, bf16x8_t b, f32x4_t c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }
};
template <>
struct Mfma16<F16> {
  static __device__ __forceinline__ f32x4_t run(f16x8_t a, f16x8_t b, f32x4_t c) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0); }
};

// Where the 16-byte pieces of a row of a wave's values lie: piece p at p ^ swz16(row). A store puts one piece of 16 rows, a
// transposing read takes two neighbouring pieces of 4 rows for each 16 lanes. With r0 .. r3 the row's bits, 8 rows in a
// row have distinct places in 128 bytes for a store, 16 in 256, and the pairs of 4 rows, and of 8, likewise for a read:
// neither has bank conflicts, with 32 or with 64 banks.
template <int D>
__device__ __forceinline__ constexpr int swz16(int r) {
  const int r0 = r & 1, r1 = r >> 1 & 1, r2 = r >> 2 & 1, r3 = r >> 3 & 1;
  return D == 128 ? (r2 ^ r3) << 3 | r1 << 2 | r0 << 1 | r2 : r1 << 2 | (r0 ^ r2) << 1 | (r2 ^ r3);
}

// A quarter of a row's codes, D / 4 elements, and its scale. `head`: where the head's rows of the page begin; the lane's
// row and quarter are in `at` and `scale_at`, from row0 on. Every row of a page may be read, so nothing is checked here:
// scores of keys that are not the part's are masked, and their values get scale 0 (which the
// conversions take for 2^-127: a weight of 0 makes zeros of them, and codes of 0 of keys without a page).
template <int D>
struct Quarter {
  uint32_t codes[D / 32];
  uint32_t scales;  // four of them: a byte would be widened at the end of the loop that loads it, which waits for it
  static __device__ __forceinline__ uint32_t code_place(int row, int quarter) { return row * (D / 2) + quarter * (D / 8); }
  static __device__ __forceinline__ uint32_t scale_place(int row, int quarter) { return row * (D / 32) + quarter * (D / 32) / 4; }
  __device__ __forceinline__ void load(const CacheArgs& c, const unsigned char* head, int row0, uint32_t at, uint32_t scale_at) {
    const unsigned char* from = head + row0 * (D / 2);
    if constexpr (D == 128) {
      const u32x4_t x = *reinterpret_cast<const u32x4_t*>(from + at);
#pragma unroll
      for (int i = 0; i < 4; ++i) codes[i] = x[i];
    } else {
      const u32x2_t x = *reinterpret_cast<const u32x2_t*>(from + at);
      codes[0] = x[0];
      codes[1] = x[1];
    }
    scales = *reinterpret_cast<const uint32_t*>(head + (((D / 2) << c.page_shift) + row0 * (D / 32)) + (scale_at & ~3u));
  }
  __device__ __forceinline__ void clear() {
#pragma unroll
    for (uint32_t& x : codes) x = 0;
    scales = 0;
  }
  __device__ __forceinline__ float scale(uint32_t scale_at) const { return scale_of(__builtin_amdgcn_ubfe(scales, 8 * (scale_at & 3u), 8)); }
};

// Half a row's codes and all of its scales, of rows l32 of 32: the first 16 from row0 of head, the others from row1 of head1.
template <int D>
struct Half {
  uint32_t codes[D / 16];
  uint32_t scales;
  __device__ __forceinline__ void load(const CacheArgs& c, const unsigned char* head, int row0, const unsigned char* head1, int row1, int l32,
                                       int hlf) {
    const bool second = l32 >= 16;
    const unsigned char* from = second ? head1 : head;
    const int row = (second ? row1 : row0) + (l32 & 15);
#pragma unroll
    for (int i = 0; i < D / 64; ++i) {
      const u32x4_t x = *reinterpret_cast<const u32x4_t*>(from + row * (D / 2) + hlf * (D / 4) + 16 * i);
#pragma unroll
      for (int k = 0; k < 4; ++k) codes[4 * i + k] = x[k];
    }
    const uint32_t at = ((D / 2) << c.page_shift) + row * (D / 32);
    if constexpr (D == 128)
      scales = *reinterpret_cast<const uint32_t*>(from + at);
    else
      scales = *reinterpret_cast<const uint16_t*>(from + at);
  }
  __device__ __forceinline__ void clear() {
#pragma unroll
    for (uint32_t& x : codes) x = 0;
    scales = 0;
  }
  // of codes[s]
  __device__ __forceinline__ float scale(int s, int hlf) const {
    return scale_of(__builtin_amdgcn_ubfe(scales, 8 * (hlf * (D / 64) + s / 4), 8));
  }
};

// Where the head's rows of the page of keys key .. key + 15 begin, of page 0 if they have none; without: the lanes whose
// keys are the part's and have none.
template <int D>
__device__ __forceinline__ int64_t head_at(const CacheArgs& c, const Part& p, int key, uint64_t& without) {
  const int page = page_of(c, p, key);
  without = __builtin_amdgcn_ballot_w64(page < 0 && key < p.end && key + 16 > p.lo);
  return head_of<D>(c, max(page, 0), p.kvh);
}

// Where 16 keys' rows of the head begin, of those that lane `at` of `heads` knows.
__device__ __forceinline__ const unsigned char* head_in(const uint16_t* pages, int64_t heads, int at) {
  const uint32_t lo = __builtin_amdgcn_readlane(static_cast<int>(heads), at), hi = __builtin_amdgcn_readlane(static_cast<int>(heads >> 32), at);
  return reinterpret_cast<const unsigned char*>(pages) + (static_cast<uint64_t>(hi) << 32 | lo);
}

// A narrow part: up to 16 R rows, whose four waves take every fourth step of 16 kTiles keys, each at its own pace, or
// (alone) one wave all of them. Keys go from
// the loads' registers into the products (the elements of a head in the order in which the lanes have them, which
// the queries follow); values through LDS, in 16 bits, where the transposing reads find them. The next
// step's codes are asked for as soon as the last ones are converted, and waited for where they are; two steps ahead took
// as long.
template <class T, int D, bool kPlain, int R, int kTiles, bool alone>
__device__ __forceinline__ void narrow_part(const CacheAttnArgs& a, const Entry& x, const KeptEntry* local, const Part& p, int row0, unsigned char* stage,
                                            float (&s_ref)[4][32], float (&s_sum)[4][32], float* out, int lane, int wave) {
  using x8 = typename T::x8;
  constexpr int kStep = 16 * kTiles, kAtOnce = 64 / kTiles;
  constexpr int kParts = D / 32;  // products that a score sums
  const CacheArgs& c = a.c;
  asm("" : "+v"(lane));  // (what a part makes of it is made again in each, and not kept through the others)
  const int l16 = lane & 15, g = lane >> 4;
  unsigned char* mine = stage + wave * 32 * 2 * D;
  const int steps = (p.end - p.key0 + kStep - 1) / kStep;
  const int mine_n = alone ? steps : steps > wave ? (steps - wave + 3) / 4 : 0;
  const int stride = alone ? kStep : 4 * kStep, my_key0 = p.key0 + (alone ? 0 : wave * kStep);
  auto key_of = [&](int n) { return my_key0 + n * stride; };
  // lane n holds where the 16 keys n % kTiles of the wave's step n / kTiles have the head's rows of their page (kAtOnce steps
  // at a time); where there is none, those of page 0 are read, and zeros put in their place if bit n of `without` says so
  auto heads_at = [&](int n, uint64_t& without) { return head_at<D>(c, p, key_of(n + lane / kTiles) + 16 * (lane % kTiles), without); };
  int64_t heads = 0, next_heads = 0;
  uint64_t without = 0, next_without = 0;
  const uint32_t code_at = Quarter<D>::code_place(l16, g), scale_at = Quarter<D>::scale_place(l16, g);
  Quarter<D> k[kTiles], v[kTiles];
  auto load = [&](int n, const uint16_t* from, Quarter<D> (&to)[kTiles]) {
#pragma unroll
    for (int t = 0; t < kTiles; ++t)
      to[t].load(c, head_in(from, heads, kTiles * (n % kAtOnce) + t), (key_of(n) + 16 * t) & ((1 << c.page_shift) - 1), code_at, scale_at);
  };
  if (mine_n > 0) heads = heads_at(0, without);
  Part pr[R];
  x8 qf[R][kParts];
  float slope[R];
#pragma unroll
  for (int i = 0; i < R; ++i) {
    pr[i] = p;
    locate_row(a, x, local, row0 + 16 * i + l16, pr[i]);
    const uint16_t* q = c.Q + pr[i].token * c.q_stride + pr[i].h * D + (D / 4) * g;
#pragma unroll
    for (int s = 0; s < kParts; ++s) {
      const u32x4_t raw = pr[i].ok ? *reinterpret_cast<const u32x4_t*>(q + 8 * s) : u32x4_t{0u, 0u, 0u, 0u};
      qf[i][s] = __builtin_bit_cast(x8, raw);
    }
    slope[i] = kPlain ? 0.0f : slope_of(a.scoring, pr[i].h);
  }
  if (mine_n > 0) {
    load(0, c.k_pages, k);
    load(0, c.v_pages, v);
  }
#pragma unroll
  for (int i = 0; i < R; ++i) {
    arrived(qf[i]);
    slope[i] = arrived(slope[i]);
  }
  const float cexp = a.scoring.unit * kLog2e;
  // places in LDS: a lane's stores (piece (D / 32) g + s of row l16), its transposing reads (4 rows of the lane's
  // group, elements 16 db ..)
  const int to = 2 * D * l16 + 16 * (((D / 32) * g) ^ swz16<D>(l16));
  const int row = 4 * g + (l16 >> 2);
  const int from = 2 * D * row + 16 * (((l16 & 3) >> 1) ^ swz16<D>(row)) + 8 * (l16 & 1);
  f32x4_t acc[R][D / 16];
#pragma unroll
  for (int i = 0; i < R; ++i)
#pragma unroll
    for (int db = 0; db < D / 16; ++db) acc[i][db] = f32x4_t{};
  QuarterSoftmax sm[R];
  for (int n = 0; n < mine_n; ++n) {
    const uint32_t zeros = static_cast<uint32_t>(without >> kTiles * (n % kAtOnce));
    if (n % kAtOnce == kAtOnce / 2) next_heads = heads_at(n + kAtOnce / 2, next_without);
    if (n % kAtOnce == kAtOnce - 1) {
      heads = next_heads;
      without = next_without;
    }
    if (zeros & ((1u << kTiles) - 1)) {
      asm volatile("");  // (a branch: as selections, this would wait for the values here)
#pragma unroll
      for (int t = 0; t < kTiles; ++t)
        if (zeros >> t & 1) {
          k[t].clear();
          v[t].clear();
        }
    }
    f32x4_t tile[R][kTiles];
#pragma unroll
    for (int t = 0; t < kTiles; ++t) {
      const float scale = k[t].scale(scale_at);
#pragma unroll
      for (int i = 0; i < R; ++i) tile[i][t] = f32x4_t{};
#pragma unroll
      for (int s = 0; s < kParts; ++s) {
        const x8 kf = __builtin_bit_cast(x8, values<T>(k[t].codes[s], scale));
#pragma unroll
        for (int i = 0; i < R; ++i) tile[i][t] = Mfma16<T>::run(kf, qf[i][s], tile[i][t]);
      }
    }
    load(n + 1, c.k_pages, k);
    x8 pb[R][kTiles / 2];
#pragma unroll
    for (int i = 0; i < R; ++i) {
      float sc[4 * kTiles];  // of keys 16 (r / 4) + 4 g + r % 4
#pragma unroll
      for (int r = 0; r < 4 * kTiles; ++r) sc[r] = tile[i][r / 4][r % 4];
      const int key0 = key_of(n);
      if constexpr (!kPlain) {
        if (a.scoring.cap_in != 0.0f) {
          if (a.scoring.unit <= kNearCap) {
#pragma unroll
            for (float& y : sc) y = tanh_from_log2(y * a.scoring.cap_in);
          } else {
#pragma unroll
            for (float& y : sc) y = tanh_from_log2_near_0(y * a.scoring.cap_in);
          }
        }
        if (a.scoring.slopes) {
          const float at = static_cast<float>(pr[i].pos - key0 - 4 * g);
#pragma unroll
          for (int r = 0; r < 4 * kTiles; ++r) sc[r] = fmaf(-slope[i], fabsf(at - static_cast<float>(16 * (r / 4) + r % 4)), sc[r]);
        }
      }
      if (key0 + kStep > pr[i].all_hi || key0 < p.lo) {
#pragma unroll
        for (int r = 0; r < 4 * kTiles; ++r) {
          const int key = key0 + 16 * (r / 4) + 4 * g + r % 4;
          if (key >= pr[i].hi || key < p.lo) sc[r] = -__builtin_inff();
        }
      }
      bool moved;
      const float alpha = sm[i].template block<T>(sc, cexp, l16, pb[i], moved);
      if (moved) {
#pragma unroll
        for (int db = 0; db < D / 16; ++db) acc[i][db] *= alpha;
      }
    }
#pragma unroll
    for (int u = 0; u < kTiles / 2; ++u) {
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        const Quarter<D>& y = v[2 * u + t];
        const int key = key_of(n) + 32 * u + 16 * t + l16;
        const float scale = key >= p.lo && key < p.end ? y.scale(scale_at) : 0.0f;
#pragma unroll
        for (int s = 0; s < kParts; ++s) *reinterpret_cast<u32x4_t*>(mine + 32 * D * t + (to ^ 16 * s)) = values<T>(y.codes[s], scale);
      }
      if (u == kTiles / 2 - 1) load(n + 1, c.v_pages, v);
      asm volatile("" ::: "memory");  // (a wave's LDS accesses are done in order)
      x8 vf[D / 16];
#pragma unroll
      for (int db = 0; db < D / 16; ++db) {
        const lds_u8_t* at = (const lds_u8_t*)mine + (from ^ 32 * db);
        const i16x4_t lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4_t*)at);
        const i16x4_t hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4_t*)(at + 32 * D));
        vf[db] = __builtin_bit_cast(x8, (i16x8_t{lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]}));
      }
      __builtin_amdgcn_sched_barrier(0);  // (all of them are asked for before the first is waited for)
#pragma unroll
      for (int db = 0; db < D / 16; ++db)
#pragma unroll
        for (int i = 0; i < R; ++i) acc[i][db] = Mfma16<T>::run(vf[db], pb[i][u], acc[i][db]);
      asm volatile("" ::: "memory");
    }
  }

  // the waves' results against their common reference, summed in the order of the waves; the
  // 16-byte pieces of a row are turned by its number, against bank conflicts
  asm("" : "+v"(lane));  // (these places are not made ahead of the loop, and kept through it)
  const int r16 = lane & 15, quarter = lane >> 4;
  const int rows = x.rows - p.tile * kCacheTileRows - row0;
  float l[R];
#pragma unroll
  for (int i = 0; i < R; ++i) l[i] = sum_quarters(sm[i].l);
  if constexpr (alone) {
#pragma unroll
    for (int i = 0; i < R; ++i) {
      if (!out || 16 * i + r16 >= rows) continue;
      const int r = row0 + 16 * i + r16;
#pragma unroll
      for (int db = 0; db < D / 16; ++db) *reinterpret_cast<f32x4_t*>(out + r * D + 16 * db + 4 * quarter) = acc[i][db];
      if (quarter == 0) {
        out[32 * D + r] = sm[i].m;
        out[32 * D + 32 + r] = l[i];
      }
    }
    return;
  }
#pragma unroll
  for (int i = 0; i < R; ++i) {
    if (quarter == 0) {
      s_ref[wave][16 * i + r16] = sm[i].m;
      s_sum[wave][16 * i + r16] = l[i];
    }
  }
  __syncthreads();  // (also: every wave has read its stage)
  constexpr int kPieces = D / 4;
  const int tid = wave * 64 + lane;
#pragma unroll
  for (int i = 0; i < R; ++i) {
    const int live = min(16, rows - 16 * i);
    if (i > 0) __syncthreads();
    if (r16 < live) {
      const int r = 16 * i + r16;
      const float top = fmaxf(fmaxf(s_ref[0][r], s_ref[1][r]), fmaxf(s_ref[2][r], s_ref[3][r]));
      const float f = factor(sm[i].m, top, cexp);
      f32x4_t* at = reinterpret_cast<f32x4_t*>(stage) + (wave * 16 + r16) * kPieces;
#pragma unroll
      for (int db = 0; db < D / 16; ++db) at[(4 * db + quarter) ^ (r16 & 7)] = acc[i][db] * f;
    }
    __syncthreads();
    if (out) {
      const f32x4_t* in = reinterpret_cast<const f32x4_t*>(stage);
      for (int e = tid; e < live * kPieces; e += kThreads) {
        const int r = e / kPieces, at = r * kPieces + ((e % kPieces) ^ (r & 7));
        f32x4_t sum = in[at];
#pragma unroll
        for (int w = 1; w < 4; ++w) sum += in[w * 16 * kPieces + at];
        *reinterpret_cast<f32x4_t*>(out + (row0 + 16 * i) * D + 4 * e) = sum;
      }
    }
  }
  if (out && tid < min(16 * R, rows)) {
    const float top = fmaxf(fmaxf(s_ref[0][tid], s_ref[1][tid]), fmaxf(s_ref[2][tid], s_ref[3][tid]));
    float sum = 0.0f;
#pragma unroll
    for (int w = 0; w < 4; ++w) sum = fmaf(s_sum[w][tid], factor(s_ref[w][tid], top, cexp), sum);
    out[32 * D + row0 + tid] = top;
    out[32 * D + 32 + row0 + tid] = sum;
  }
  __syncthreads();  // the stages are free again
}

// A wide part, whose waves share blocks of 64 keys. Each wave has 32 rows; it converts all of the keys for itself, from
// registers (lane l has half l / 32 of the rows l % 32 and 32 + l % 32, which the queries follow), and 16 of the values
// (a quarter of row l % 16) for all, through one of two buffers in LDS.
template <class T, int D, bool kPlain>
__device__ __forceinline__ void wide_part(const CacheAttnArgs& a, const Entry& x, const KeptEntry* local, Part& p, unsigned char* stage, float* out, int lane,
                                          int wave) {
  using x8 = typename T::x8;
  constexpr int kTile = kCacheWideBlock * 2 * D;
  const CacheArgs& c = a.c;
  asm("" : "+v"(lane));  // (as above)
  const int l32 = lane & 31, hlf = lane >> 5;
  const int row = lane & 15, quarter = lane >> 4;
  const int nb = (p.end - p.key0 + kCacheWideBlock - 1) / kCacheWideBlock;
  auto key_of = [&](int n) { return p.key0 + n * kCacheWideBlock; };
  // lane n holds where the 16 keys n % 4 of block n / 4 have the head's rows of their page (16 blocks at a time; `without` as
  // above)
  auto heads_at = [&](int n, uint64_t& without) { return head_at<D>(c, p, key_of(n + lane / 4) + 16 * (lane % 4), without); };
  uint64_t without, next_without = 0;
  int64_t heads = heads_at(0, without), next_heads = 0;
  const int in_page = (1 << c.page_shift) - 1;
  const uint32_t v_at = Quarter<D>::code_place(row, quarter), v_scale_at = Quarter<D>::scale_place(row, quarter);
  Half<D> k[2];
  Quarter<D> v;
  auto load_k = [&](int n, int kb) {
    // (the 32 keys may lie in two pages of 16)
    const int at = 4 * (n & 15) + 2 * kb, key = key_of(n) + 32 * kb;
    k[kb].load(c, head_in(c.k_pages, heads, at), key & in_page, head_in(c.k_pages, heads, at + 1), (key + 16) & in_page, l32, hlf);
  };
  auto load_v = [&](int n) {
    v.load(c, head_in(c.v_pages, heads, 4 * (n & 15) + wave), (key_of(n) + 16 * wave) & in_page, v_at, v_scale_at);
  };
  locate_row(a, x, local, l32, p);
  x8 qf[D / 16];
  const uint16_t* q = c.Q + p.token * c.q_stride + p.h * D + (D / 2) * hlf;
#pragma unroll
  for (int s = 0; s < D / 16; ++s) {
    const u32x4_t raw = p.ok ? *reinterpret_cast<const u32x4_t*>(q + 8 * s) : u32x4_t{0u, 0u, 0u, 0u};
    qf[s] = __builtin_bit_cast(x8, raw);
  }
  float slope = kPlain ? 0.0f : slope_of(a.scoring, p.h);
  load_v(0);
  load_k(0, 0);
  load_k(0, 1);
  arrived(qf);
  slope = arrived(slope);
  const float cexp = a.scoring.unit * kLog2e;
  const Frags<D> fr(lane);
  f32x16_t acc[D / 32];
#pragma unroll
  for (int db = 0; db < D / 32; ++db) acc[db] = f32x16_t{};
  RowSoftmax sm;
  const int to = (16 * wave + row) * 2 * D + 16 * ((quarter * (D / 32)) ^ swz<D>(row));
  for (int n = 0; n < nb; ++n) {
    const uint32_t zeros = static_cast<uint32_t>(without >> 4 * (n & 15));
    if ((n & 15) == 8) next_heads = heads_at(n + 8, next_without);
    if ((n & 15) == 15) {
      heads = next_heads;
      without = next_without;
    }
    if (zeros & 15) {
      asm volatile("");  // (as above)
#pragma unroll
      for (int kb = 0; kb < 2; ++kb)
        if (zeros >> (2 * kb + (l32 >> 4)) & 1) k[kb].clear();
      if (zeros >> wave & 1) v.clear();
    }
    unsigned char* vt = stage + (n & 1) * kTile;
    const int key = key_of(n) + 16 * wave + row;
    const float v_scale = key >= p.lo && key < p.end ? v.scale(v_scale_at) : 0.0f;
#pragma unroll
    for (int i = 0; i < D / 32; ++i) *reinterpret_cast<u32x4_t*>(vt + (to ^ 16 * i)) = values<T>(v.codes[i], v_scale);
    load_v(n + 1);
    f32x16_t sc[2] = {f32x16_t{}, f32x16_t{}};
#pragma unroll
    for (int s = 0; s < D / 16; ++s) {
#pragma unroll
      for (int kb = 0; kb < 2; ++kb)
        sc[kb] = T::mfma(__builtin_bit_cast(x8, values<T>(k[kb].codes[s], k[kb].scale(s, hlf))), qf[s], sc[kb]);
    }
    __builtin_amdgcn_sched_barrier(0);
    load_k(n + 1, 0);
    load_k(n + 1, 1);
    finish_scores<2, kPlain>(a, p, slope, key_of(n), hlf, sc);
    x8 pb[4];
    bool moved;
    const float alpha = sm.block<T, 2>(sc, cexp, pb, moved);
    if (moved) {
#pragma unroll
      for (int db = 0; db < D / 32; ++db) acc[db] *= alpha;
    }
    __syncthreads();  // block n's values are there, and everyone is done with those of block n - 1
    // (a quarter of the values is on its way to the registers while the one before is multiplied)
    x8 vf[2][D / 32];
    auto read = [&](int t) {
#pragma unroll
      for (int db = 0; db < D / 32; ++db) vf[t & 1][db] = col_frag<T, D>((const lds_u8_t*)vt, fr, db, 16 * t);
      __builtin_amdgcn_sched_barrier(0);
    };
    read(0);
#pragma unroll
    for (int t = 0; t < 4; ++t) {
      if (t < 3) read(t + 1);
#pragma unroll
      for (int db = 0; db < D / 32; ++db) acc[db] = T::mfma(vf[t & 1][db], pb[t], acc[db]);
      __builtin_amdgcn_sched_barrier(0);
    }
  }
  const float l = sum_halves(sm.l);
  if (out && p.ok) {
#pragma unroll
    for (int db = 0; db < D / 32; ++db)
#pragma unroll
      for (int q = 0; q < 4; ++q)
        *reinterpret_cast<f32x4_t*>(out + l32 * D + 32 * db + 8 * q + 4 * hlf) =
            f32x4_t{acc[db][4 * q], acc[db][4 * q + 1], acc[db][4 * q + 2], acc[db][4 * q + 3]};
    if (hlf == 0) {
      out[32 * D + l32] = sm.m;
      out[32 * D + 32 + l32] = l;
    }
  }
  __syncthreads();  // the buffers are free again
}

// With few rows a sequence (few), the kernel has only the narrow parts of 16 rows, whose registers and LDS
// let more workgroups onto a CU (64 sequences with two 41.6 us, three 39.7; four, which spilled when it was tried, 58); an entry of
// more rows goes through its keys once for each 16 of them, which the runs' units do not count: one sequence of many rows among many of
// few makes its workgroups the last (127 of 2000 keys and a part of 300 tokens on 8000 296 us, as two calls 69 and 71). Otherwise it has
// parts for up to 16, up to 32 and up to 128 rows, that convert their keys once. With short_tasks, sequences are so many
// that each wave may have runs of its own: of all tasks (few, if all of them are small), or, beside groups, of the small ones. A call of
// more rows without groups has none.
template <class T, int D, bool kPlain, bool few, bool short_tasks>
__global__ __launch_bounds__(kThreads, few ? kCache4Few : kCacheGroups) void cache4_attn(CacheAttnArgs a) {
  __shared__ __attribute__((aligned(1024))) unsigned char stage[(few ? 2 : 4) * kCacheBlock * 4 * D];
  __shared__ float s_ref[4][32], s_sum[4][32];
  static_assert(sizeof(stage) >= kCacheGroupBytes, "the groups, before the buffers");
  static_assert(few || sizeof(stage) == 2 * 2 * kCacheWideBlock * 2 * D, "a wide part's buffers");
  static_assert(sizeof(stage) >= 4 * 32 * 2 * D && sizeof(stage) >= 4 * 16 * D * 4, "the narrow waves' values, and results of theirs");
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  constexpr int kCost = short_tasks ? kCache4AloneCost : 0, kMost = D == 128 ? kCache4AloneBlocks : 2 * kCache4AloneBlocks;
  cache_run<kCost, kMost, few ? 0 : kCache4OtherUnits>(a, stage, [&](const Entry& x, const KeptEntry* local, Part& p, int64_t place, bool wide, bool alone) {
    if (short_tasks && alone) {
      narrow_part<T, D, kPlain, 1, 2, true>(a, x, local, p, 0, stage, s_ref, s_sum, part_at<D>(a, place), lane, wave);
    } else if constexpr (few) {
      const int first = p.tile;
      for (int r = first * kCacheTileRows; r < min(x.rows, first * kCacheTileRows + kCacheWideRows); r += 16) {
        p.tile = r / kCacheTileRows;
        narrow_part<T, D, kPlain, 1, 2, false>(a, x, local, p, r % kCacheTileRows, stage, s_ref, s_sum, part_at<D>(a, place + p.tile - first), lane, wave);
      }
    } else if (wide) {
      p.tile += wave;
      wide_part<T, D, kPlain>(a, x, local, p, stage, part_at<D>(a, place + wave), lane, wave);
    } else if (x.rows <= 16) {
      narrow_part<T, D, kPlain, 1, 4, false>(a, x, local, p, 0, stage, s_ref, s_sum, part_at<D>(a, place), lane, wave);
    } else {
      narrow_part<T, D, kPlain, 2, 2, false>(a, x, local, p, 0, stage, s_ref, s_sum, part_at<D>(a, place), lane, wave);
    }
  });
}

template <class T, int D>
hipError_t append(const AppendArgs& a, hipStream_t s) {
  hipLaunchKernelGGL((cache4_append<T, D>), dim3(a.c.tokens), dim3(kThreads), 0, s, a);
  return hipGetLastError();
}

template <class T, int D>
hipError_t read(const ReadArgs& a, hipStream_t s) {
  hipLaunchKernelGGL((cache4_read<T, D>), dim3((a.c.tokens + kReadRows - 1) / kReadRows * (a.c.Hkv / a.heads)), dim3(kThreads), 0, s, a);
  return hipGetLastError();
}

template <class T, int D, bool few, bool short_tasks>
hipError_t attend(const CacheAttnArgs& a, hipStream_t s) {
  const dim3 grid(a.head_workers * a.c.Hkv);
  if (a.scoring.plain())
    hipLaunchKernelGGL((cache4_attn<T, D, true, few, short_tasks>), grid, dim3(kThreads), 0, s, a);
  else
    hipLaunchKernelGGL((cache4_attn<T, D, false, few, short_tasks>), grid, dim3(kThreads), 0, s, a);
  return hipGetLastError();
}

template <class T, int D>
hipError_t attend(const CacheAttnArgs& a, bool few, hipStream_t s) {
  const bool many = enough_to_run_alone(a.c.batch, a.head_workers);
  if (few) return many ? attend<T, D, true, true>(a, s) : attend<T, D, true, false>(a, s);
  return many && a.n_groups > 0 ? attend<T, D, false, true>(a, s) : attend<T, D, false, false>(a, s);
}

}  // namespace

hipError_t launch_cache4_append(const AppendArgs& a, bool f16, int head_dim, hipStream_t s) {
  if (head_dim == 128) return f16 ? append<F16, 128>(a, s) : append<Bf16, 128>(a, s);
  return f16 ? append<F16, 64>(a, s) : append<Bf16, 64>(a, s);
}

hipError_t launch_cache4_read(const ReadArgs& a, bool f16, int head_dim, hipStream_t s) {
  if (head_dim == 128) return f16 ? read<F16, 128>(a, s) : read<Bf16, 128>(a, s);
  return f16 ? read<F16, 64>(a, s) : read<Bf16, 64>(a, s);
}

hipError_t launch_cache4_attn(const CacheAttnArgs& a, bool f16, int head_dim, hipStream_t s) {
  const bool few = cache4_few(a.c.tokens, a.c.H, a.c.Hkv, a.c.batch, a.n_groups);
  hipError_t e = head_dim == 128 ? (f16 ? attend<F16, 128>(a, few, s) : attend<Bf16, 128>(a, few, s))
                                 : (f16 ? attend<F16, 64>(a, few, s) : attend<Bf16, 64>(a, few, s));
  return e != hipSuccess ? e : launch_cache_merge(a, f16, head_dim, s);
}

}  // namespace csg
