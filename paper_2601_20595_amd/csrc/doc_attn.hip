// Attention over packed documents, and its gradient, for gfx950 (CDNA4).
//
// Rows (queries) and keys of document t are rows q_ptr[t] .. q_ptr[t+1] - 1 and k_ptr[t] ..
// k_ptr[t+1] - 1. Row i of a document stands at its key p = i + keys - rows (the last row at
// the last key). It sees key j of its document if the mask is not causal, or j <= p, or
// j < prefix[t]: always the first hi(i) keys, and hi grows with i, so a tile of rows walks
// the blocks of keys below its last row's hi, and only blocks above its first row's hi look
// at the mask at all. With s the scores (scaled, capped, less the distance bias),
//   lse_i = log sum_j exp(s_ij),  P_ij = exp(s_ij - lse_i),  o_i = sum_j P_ij v_j,
//   D_i = do_i . o_i,  dS_ij = P_ij (do_i . v_j - D_i) (1 - tanh^2),
//   dQ_i = scale sum_j dS_ij k_j,  dK_j = scale sum_i dS_ij q_i,  dV_j = sum_i P_ij do_i.
//
// Tiles never hold rows of two documents, so no document's values reach another's results.
// A tile of rows is 128 or 64 (row, head) pairs, a wave for 32 rows of a head; where heads share
// keys, 2 or 4 of them share the tile: then it spans fewer rows, which leaves less of it unused
// on short documents and computes fewer masked pairs. The tiles of a launch are bounded by
// the host, which does not know the documents: document t's first tile is q_ptr[t] / rows a
// tile + t, which leaves room for its last, part-filled one; a workgroup without rows ends.
#include <hip/hip_runtime.h>

#include <numeric>

#include "attn_tile.hpp"
#include "doc_attn.hpp"

namespace csg {
namespace {

using namespace tile;

constexpr int kThreads = 256;
static_assert(kDocTileRows == 32 * (kThreads / 64), "one wave per 32 rows");

// A document and the part of it that a tile holds.
struct Place {
  int q0, q_len, k0, k_len, prefix;
  int first;  // the tile's first row (key) in the document
  bool any;
};

// The document of tile `slot` of `step` rows each; `by_keys`: the tile holds keys.
__device__ __forceinline__ Place find_place(const DocAttnArgs& a, int slot, int step, bool by_keys) {
  Place p;
  const int32_t* ptr = by_keys ? a.k_ptr : a.q_ptr;
  const int rows = by_keys ? a.k_rows : a.q_rows;
  const int d = last_below(a.n_docs, [&](int i) { return clamped(ptr[i], 0, rows) / step + i <= slot; });
  p.q0 = clamped(a.q_ptr[d], 0, a.q_rows);
  p.q_len = clamped(a.q_ptr[d + 1], p.q0, a.q_rows) - p.q0;
  p.k0 = clamped(a.k_ptr[d], 0, a.k_rows);
  p.k_len = clamped(a.k_ptr[d + 1], p.k0, a.k_rows) - p.k0;
  p.prefix = a.prefix ? clamped(a.prefix[d], 0, p.k_len) : 0;
  const int t = slot - ((by_keys ? p.k0 : p.q0) / step + d);
  p.any = t >= 0 && static_cast<int64_t>(t) * step < (by_keys ? p.k_len : p.q_len);
  p.first = p.any ? t * step : 0;
  return p;
}

// Keys that row i of the document sees.
__device__ __forceinline__ int visible(const DocAttnArgs& a, const Place& p, int i) {
  return a.causal ? clamped(max(p.prefix, i + p.k_len - p.q_len + 1), 0, p.k_len) : p.k_len;
}

// How the waves of a workgroup share a tile of rows: kWaves of 32 (row, head) pairs each, and
// kTeams of them, which take turns at the blocks of kKeys keys and add up their sums at the end.
template <int W, int N, int K>
struct Shape {
  static constexpr int kWaves = W, kTeams = N, kKeys = K, kThreads = 64 * W * N;
};
using Whole = Shape<4, 1, 64>;
using Halves = Shape<4, 2, 64>;
using Quarters = Shape<2, 4, 32>;

// This wave's share, one of kWaves, of the loads of kRows rows (fewer at the end: rows past `rows`
// read zero) of one head into a tile at LDS byte `lds`. src: the head's part of the first row.
template <int D, int kRows = kDocBlock, int kWaves = 4>
__device__ __forceinline__ void load_tile(const uint16_t* src, int64_t stride, int rows, uint32_t lds, int wave,
                                          const LoadLane<D>& ll) {
  const int n = rows < kRows ? rows : kRows;
  const __amdgpu_buffer_rsrc_t rs = make_rsrc(src, n > 0 ? static_cast<int>(((n - 1) * stride + D) * 2) : 0);
  constexpr int kPer = kRows / kLoadRows<D> / kWaves;
  const int stride2 = static_cast<int>(2 * stride);
#pragma unroll
  for (int q = 0; q < kPer; ++q) {
    const int i = wave * kPer + q;
    constexpr int kTurns = 16 / kLoadRows<D>;
    // (where every wave starts at a multiple of 16 rows, the turn of the pieces depends on q alone)
    const int turn = swz<D>(kLoadRows<D> * ((kPer % kTurns == 0 ? q : i) % kTurns));
    const int voff = (kLoadRows<D> * i + ll.row) * stride2 + 16 * (ll.piece ^ turn);
    load_to_lds(rs, __builtin_amdgcn_readfirstlane(lds + 1024u * i), voff);
  }
}

// A wave's 32 rows of one head as second operand: lane row `row`, zero if it is not `ok`.
template <class T, int D>
__device__ __forceinline__ void load_rows(const uint16_t* head, int64_t stride, int row, bool ok, int hlf,
                                          typename T::x8 (&f)[D / 16]) {
  const uint16_t* p = head + (ok ? row : 0) * stride + 8 * hlf;
#pragma unroll
  for (int s = 0; s < D / 16; ++s) {
    const u32x4_t raw = ok ? *reinterpret_cast<const u32x4_t*>(p + 16 * s) : u32x4_t{0u, 0u, 0u, 0u};
    f[s] = __builtin_bit_cast(typename T::x8, raw);
  }
}

// A result transposed (lane: one row, 16 elements per 32 in runs of four) times f, rounded.
template <class T, int D>
__device__ __forceinline__ void store_rows(uint16_t* head, int64_t stride, int row, int hlf, const f32x16_t (&acc)[D / 32],
                                           float f) {
  uint16_t* p = head + row * stride + 4 * hlf;
#pragma unroll
  for (int db = 0; db < D / 32; ++db)
#pragma unroll
    for (int b = 0; b < 4; ++b) {
      const f32x4_t v{acc[db][4 * b] * f, acc[db][4 * b + 1] * f, acc[db][4 * b + 2] * f, acc[db][4 * b + 3] * f};
      *reinterpret_cast<u32x2_t*>(p + 32 * db + 8 * b) = __builtin_bit_cast(u32x2_t, __builtin_convertvector(v, typename T::x4));
    }
}

// Sums of teams 1 .. to team 0: 16 bytes a lane side by side, a wave's after the other's.
template <int D>
__device__ __forceinline__ void put_sums(f32x4_t* to, const f32x16_t (&acc)[D / 32]) {
#pragma unroll
  for (int k = 0; k < D / 8; ++k)
    to[64 * k] = f32x4_t{acc[k / 4][4 * (k % 4)], acc[k / 4][4 * (k % 4) + 1], acc[k / 4][4 * (k % 4) + 2], acc[k / 4][4 * (k % 4) + 3]};
}
template <int D>
__device__ __forceinline__ void add_sums(const f32x4_t* from, f32x16_t (&acc)[D / 32], float f, float g) {
#pragma unroll
  for (int k = 0; k < D / 8; ++k) {
    const f32x4_t v = from[64 * k];
#pragma unroll
    for (int e = 0; e < 4; ++e) acc[k / 4][4 * (k % 4) + e] = fmaf(acc[k / 4][4 * (k % 4) + e], f, v[e] * g);
  }
}

// ---- forward -----------------------------------------------------------------------------
// One pass over the keys, which go by DMA into two buffers that the tile's waves share. A wave
// computes keys x rows, so that a row's scores, maximum and sum stay in two lanes and the rounded
// weights already are the operand of values x weights: nothing but keys and values passes LDS.
// Long documents are bound by the SIMDs' issue: per block of 64 keys, 32 products and some 200
// vector instructions of the softmax. 8192 causal rows, 32 heads on 8 of 128: 521 us, 1.06 PFLOP/s of
// visible pairs; matrix instructions take 52 % of the SIMDs' cycles, vector ones 45 %, LDS 26 %,
// without a bank conflict, at 1.95 GHz. Priorities around the products and blocks cut into halves of
// 32 keys (3 % slower) did no better; products of the next block during the softmax spill.
// Capped scores of few long documents are bound by tanh on the longest one's tiles (83 us, 5
// documents of up to 2446 keys, 16 heads on 2).
template <class T, int D, bool kPlain, class S>
__global__ __launch_bounds__(S::kThreads, 2) void doc_forward(DocAttnArgs a) {
  constexpr int kTeams = S::kTeams, kKeys = S::kKeys, kTile = kKeys * D * 2;
  __shared__ __attribute__((aligned(1024))) unsigned char stage[2 * kTeams * 2 * kTile];
  const int lane = threadIdx.x & 63, any_wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wave = any_wave % S::kWaves, team = any_wave / S::kWaves;
  const int l32 = lane & 31, hlf = lane >> 5;
  const int span = 32 * S::kWaves / a.tile_heads, groups = a.H / a.tile_heads;
  // a die runs every 8th workgroup: with the head fastest, it keeps to few key/value heads;
  // the last rows of a causal document, which see the most keys, come first
  const int hg = blockIdx.x % groups;
  const Place p = find_place(a, gridDim.x / groups - 1 - blockIdx.x / groups, span, false);
  if (!p.any) return;
  const int G = a.H / a.Hkv, per_kv = G / a.tile_heads;
  const int kvh = hg / per_kv;
  const int h = kvh * G + (hg - kvh * per_kv) * a.tile_heads + wave % a.tile_heads;
  const int first = p.first + wave / a.tile_heads * 32;
  const int row = first + l32;
  const bool ok = row < p.q_len;
  const int hi = visible(a, p, min(row, p.q_len - 1));
  const int wave_lo = visible(a, p, min(first, p.q_len - 1));  // seen by every row of the wave
  const int nb = (visible(a, p, min(p.first + span, p.q_len) - 1) + kKeys - 1) / kKeys;
  const int wave_nb = first < p.q_len ? (visible(a, p, min(first + 32, p.q_len) - 1) + kKeys - 1) / kKeys : 0;
  const float slope = kPlain ? 0.0f : slope_of(a.scoring, h);
  const int at = row + p.k_len - p.q_len;  // the row's own key

  const LoadLane<D> ll(lane);
  const Frags<D> fr(lane);
  // the team's two buffers of keys, and of values
  const unsigned char* sK = stage + team * 4 * kTile;
  const unsigned char* sV = sK + 2 * kTile;
  const uint32_t sK_addr = lds_address(sK), sV_addr = lds_address(sV);
  const lds_u8_t* sV_lds = (const lds_u8_t*)sV;
  const uint16_t* kh = a.K + p.k0 * a.k_stride + kvh * D;
  const uint16_t* vh = a.V + p.k0 * a.v_stride + kvh * D;
  auto load = [&](int i, int j) {  // block j into buffer i % 2
    load_tile<D, kKeys, S::kWaves>(kh + static_cast<int64_t>(j) * kKeys * a.k_stride, a.k_stride, p.k_len - j * kKeys,
                                   sK_addr + (i & 1) * kTile, wave, ll);
    load_tile<D, kKeys, S::kWaves>(vh + static_cast<int64_t>(j) * kKeys * a.v_stride, a.v_stride, p.k_len - j * kKeys,
                                   sV_addr + (i & 1) * kTile, wave, ll);
  };
  if (team < nb) load(0, team);

  typename T::x8 qf[D / 16];
  load_rows<T, D>(a.Q + p.q0 * a.q_stride + h * D, a.q_stride, row, ok, hlf, qf);
  f32x16_t acc[D / 32];
#pragma unroll
  for (int db = 0; db < D / 32; ++db) acc[db] = f32x16_t{};
  RowSoftmax sm;
  const float c = a.scoring.unit * kLog2e;
  arrived(qf);

  for (int i = 0, j = team; i * kTeams < nb; ++i, j += kTeams) {
    wait_vm<0>();
    __syncthreads();  // the team's block j is there, and everyone is done with the one before
    if (j + kTeams < nb) load(i + 1, j + kTeams);
    if (j >= wave_nb) continue;
    const int buf = (i & 1) * kTile;
    const int key0 = j * kKeys;
    constexpr int kN = kKeys / 32;
    f32x16_t sc[kN];
    __builtin_amdgcn_sched_barrier(0);
    // products of the keys with the wave's rows (lane (l32, hlf) has those of row l32), six reads ahead
#pragma unroll
    for (int kb = 0; kb < kN; ++kb) sc[kb] = f32x16_t{};
#pragma unroll
    for (int s = 0; s < D / 16; ++s)
#pragma unroll
      for (int kb = 0; kb < kN; ++kb) sc[kb] = T::mfma(row_frag<T, D>(sK + buf, fr, s, 32 * kb), qf[s], sc[kb]);
    __builtin_amdgcn_sched_group_barrier(0x100, 6, 0);
#pragma unroll
    for (int i = 0; i < kN * D / 16; ++i) {
      __builtin_amdgcn_sched_group_barrier(0x8, 1, 0);
      __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
    }
    __builtin_amdgcn_sched_barrier(0);
    // the values of the first 16 keys are read ahead of the weights, the others 16 keys ahead
    typename T::x8 vf[2][D / 32];
    auto read_values = [&](int t) {
#pragma unroll
      for (int db = 0; db < D / 32; ++db) vf[t & 1][db] = col_frag<T, D>(sV_lds + buf, fr, db, 16 * t);
    };
    read_values(0);
    if constexpr (!kPlain) {
      cap_scores<kN>(a.scoring, sc);
      bias_scores<kN, -1>(a.scoring, slope, at - key0, hlf, sc);
    }
    if (key0 + kKeys > wave_lo) {
#pragma unroll
      for (int kb = 0; kb < kN; ++kb)
#pragma unroll
        for (int r = 0; r < 16; ++r)
          if (key0 + 32 * kb + result_row(r, hlf) >= hi) sc[kb][r] = -__builtin_inff();
    }
    typename T::x8 pb[2 * kN];
    bool moved;
    const float alpha = sm.block<T, kN>(sc, c, pb, moved);
    if (moved) {
#pragma unroll
      for (int db = 0; db < D / 32; ++db) acc[db] *= alpha;
    }
#pragma unroll
    for (int t = 0; t < 2 * kN; ++t) {
      if (t + 1 < 2 * kN) read_values(t + 1);
#pragma unroll
      for (int db = 0; db < D / 32; ++db) acc[db] = T::mfma(vf[t & 1][db], pb[t], acc[db]);
    }
  }
  if constexpr (kTeams > 1) {
    __shared__ float s_state[kTeams - 1][S::kWaves][2][64];
    static_assert(sizeof(stage) >= (kTeams - 1) * S::kWaves * 64 * (D / 2) * 4, "the teams' sums fit the buffers");
    f32x4_t* sums = reinterpret_cast<f32x4_t*>(stage) + wave * (D / 8) * 64 + lane;
    constexpr int kTeamSums = S::kWaves * (D / 8) * 64;
    __syncthreads();
    if (team > 0) {
      put_sums<D>(sums + (team - 1) * kTeamSums, acc);
      s_state[team - 1][wave][0][lane] = sm.m;
      s_state[team - 1][wave][1][lane] = sm.l;
    }
    __syncthreads();
    if (team > 0) return;
#pragma unroll
    for (int n = 0; n < kTeams - 1; ++n) {
      const float m = s_state[n][wave][0][lane], top = fmaxf(m, sm.m);
      const float f = factor(sm.m, top, c), g = factor(m, top, c);
      sm.m = top;
      sm.l = fmaf(sm.l, f, s_state[n][wave][1][lane] * g);
      add_sums<D>(sums + n * kTeamSums, acc, f, g);
    }
  }
  if (!ok) return;
  const float total = sum_halves(sm.l);
  if (total == 0.0f) {  // nothing visible
#pragma unroll
    for (int db = 0; db < D / 32; ++db) acc[db] = f32x16_t{};
  }
  store_rows<T, D>(a.O + (static_cast<int64_t>(p.q0) * a.H + h) * D, static_cast<int64_t>(a.H) * D, row, hlf, acc,
                   total == 0.0f ? 0.0f : 1.0f / total);
  if (hlf == 0)
    a.LSE[static_cast<int64_t>(h) * a.q_rows + p.q0 + row] = fmaf(log2f(total), kLn2, sm.m * a.scoring.unit);
}

// ---- numbers of the gradients in f16 ----------------------------------------------------------
// Over thousands of keys weights of a row are below f16's smallest normal number, 2^-14, and so are the
// gradients of scores dS that a small gradient of the output gives; there the type loses bits (3000 keys,
// do of 1e-3: dq off by 3.7e-3 of its norm; as below 6e-4, of which its own rounding is most). So weights
// are made 2^14 times as large by the exponent's argument, and dS takes a power of two of each lane's own
// row (key): the lane's largest so far lies below 2^15 with it, and was above 2^10 when it was set, so that
// nothing overflows and what is lost is below 2^-35 of the largest. Sums in fp32 are brought back exactly.
// The look at the largest costs: packed documents of up to 721 rows, heads of 64, queries' gradient 32.1 ->
// 35.5 us, keys' 30.0 -> 31.6; 8191 rows, 32 heads on 8 of 128, 948 -> 1040 and 1085 -> 1131. The factor
// alone costs nothing; the branch stands between a block's scores and its products. Without a branch 36.7
// and 32.7; in one branch with the mask 38.5 and 32.9; the bits of the rounded numbers instead of the
// largest 37.1 and 32.4; one for 64 keys spills; a factor only where it is needed, or the weights' products
// or the next 32 keys' ahead of it, within 1 us of the same.
constexpr float kLog2Shift = 14.0f, kUnshift = 1.0f / 16384.0f;
template <class T>
constexpr float kWeightShift = T::kShortRange ? kLog2Shift : 0.0f;
template <class T>
constexpr float kWeightUnit = T::kShortRange ? kUnshift : 1.0f;

template <class T>
struct Reach {
  uint32_t bits = 227u << 23;  // of the factor, 2^100 until there is anything
  // What the lane's sums are to be multiplied with (1 if its factor stays) in order to take more of x, which
  // is multiplied with the factor.
  template <int N>
  __device__ __forceinline__ void take(f32x16_t& x, f32x16_t (&sums)[N]) {
    if constexpr (T::kShortRange) {
      float m = 0.0f;
#pragma unroll
      for (int r = 0; r < 16; ++r) m = fmaxf(m, fabsf(x[r]));
      m = max_halves(m);
      const bool move = m * __uint_as_float(bits) > 32768.0f;
      if (__builtin_amdgcn_ballot_w64(move) != 0) {
        const uint32_t to = min(264u - (__float_as_uint(m) >> 23), 227u) << 23;  // m becomes 2^10 .. 2^11
        const float f = move ? __uint_as_float(to) * back() : 1.0f;
        bits = move ? to : bits;
#pragma unroll
        for (int k = 0; k < N; ++k) sums[k] *= f;
      }
#pragma unroll
      for (int r = 0; r < 16; ++r) x[r] *= __uint_as_float(bits);
    }
  }
  __device__ __forceinline__ float back() const { return T::kShortRange ? __uint_as_float((254u << 23) - bits) : 1.0f; }
};

// ---- gradient of the queries --------------------------------------------------------------
// The forward's tiles; also leaves each row's statistics to the kernel of the keys' gradient.
// D_i = sum_j P_ij (do_i . v_j) equals do_i . o_i, but for the rounding of o (and of the weights
// that made it), which a row with few large weights cannot afford: there do . v_j - D cancels. With
// it alone, gradients of 20 short documents were off by 3.7e-4 of their norm in fp16, not by 2.9e-4,
// and of sharp scores in bf16 by 4.6e-3. One pass over the keys sums against D' = do_i . o_i:
//   e_i = sum_j P_ij (do_i . v_j - D'_i) = D_i - D'_i,
//   dQ_i / scale = sum_j P_ij (do_i . v_j - D'_i) (1 - tanh^2) k_j - e_i sum_j P_ij (1 - tanh^2) k_j.
// (What multiplies e_i is a sum of rounded weights; e_i itself is of the size of a rounding, so that this
// is of second order. Against the output of more keys than the call's, whose weights do not sum to 1 here, e_i would be
// those keys' part of the sum: then it is 0, and D is D'.)
// For D = 128 the second sum takes the registers of the rows of do, which are read from LDS. 8192 causal
// rows, 32 heads on 8 of 128: 0.88 to 0.92 ms, four products of the pairs at 1.2 PFLOP/s, which is what a
// large matrix product of the library reaches on the card: bound by the matrix instructions and the
// clock that their power leaves. A pass of its own for D took five products and 1.23 ms.
template <class T, int D, bool kPlain, class S>
__global__ __launch_bounds__(S::kThreads, 2) void doc_grad_q(DocAttnArgs a) {
  constexpr int kTeams = S::kTeams, kKeys = S::kKeys, kTile = kKeys * D * 2;
  constexpr bool kRowsInLds = D == 128;
  __shared__ __attribute__((aligned(1024))) unsigned char stage[2 * kTeams * 2 * kTile];
  // by wave, fragment and lane; the teams hold the same
  __shared__ u32x4_t s_rows[kRowsInLds ? S::kWaves * (D / 16) * 64 : 1];
  __shared__ float s_more[kTeams][S::kWaves][64];
  const int lane = threadIdx.x & 63, any_wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wave = any_wave % S::kWaves, team = any_wave / S::kWaves;
  const int l32 = lane & 31, hlf = lane >> 5;
  const int span = 32 * S::kWaves / a.tile_heads, groups = a.H / a.tile_heads;
  const int hg = blockIdx.x % groups;
  const Place p = find_place(a, gridDim.x / groups - 1 - blockIdx.x / groups, span, false);
  if (!p.any) return;
  const int G = a.H / a.Hkv, per_kv = G / a.tile_heads;
  const int kvh = hg / per_kv;
  const int h = kvh * G + (hg - kvh * per_kv) * a.tile_heads + wave % a.tile_heads;
  const int first = p.first + wave / a.tile_heads * 32;
  const int row = first + l32;
  const bool ok = row < p.q_len;
  const int hi = visible(a, p, min(row, p.q_len - 1));
  const int wave_lo = visible(a, p, min(first, p.q_len - 1));
  const int nb = (visible(a, p, min(p.first + span, p.q_len) - 1) + kKeys - 1) / kKeys;
  const int wave_nb = first < p.q_len ? (visible(a, p, min(first + 32, p.q_len) - 1) + kKeys - 1) / kKeys : 0;
  const float slope = kPlain ? 0.0f : slope_of(a.scoring, h);
  const int at = row + p.k_len - p.q_len;

  const LoadLane<D> ll(lane);
  const Frags<D> fr(lane);
  // the team's two buffers of keys, and of values
  const unsigned char* sK = stage + team * 4 * kTile;
  const unsigned char* sV = sK + 2 * kTile;
  const uint32_t sK_addr = lds_address(sK), sV_addr = lds_address(sV);
  const lds_u8_t* sK_lds = (const lds_u8_t*)sK;
  const uint16_t* kh = a.K + p.k0 * a.k_stride + kvh * D;
  const uint16_t* vh = a.V + p.k0 * a.v_stride + kvh * D;
  auto load = [&](int i, int j) {  // block j into buffer i % 2
    load_tile<D, kKeys, S::kWaves>(kh + static_cast<int64_t>(j) * kKeys * a.k_stride, a.k_stride, p.k_len - j * kKeys,
                                   sK_addr + (i & 1) * kTile, wave, ll);
    load_tile<D, kKeys, S::kWaves>(vh + static_cast<int64_t>(j) * kKeys * a.v_stride, a.v_stride, p.k_len - j * kKeys,
                                   sV_addr + (i & 1) * kTile, wave, ll);
  };
  if (team < nb) load(0, team);

  typename T::x8 qf[D / 16], gf[D / 16];
  load_rows<T, D>(a.Q + p.q0 * a.q_stride + h * D, a.q_stride, row, ok, hlf, qf);
  const int64_t o_stride = static_cast<int64_t>(a.H) * D, o_head = p.q0 * o_stride + h * D;
  load_rows<T, D>(a.dO + o_head, o_stride, row, ok, hlf, gf);
  u32x4_t* const my_rows = s_rows + (kRowsInLds ? wave * (D / 16) * 64 + lane : 0);
  if constexpr (kRowsInLds) {
#pragma unroll
    for (int s = 0; s < D / 16; ++s) my_rows[64 * s] = __builtin_bit_cast(u32x4_t, gf[s]);
  }
  const float c = a.scoring.unit * kLog2e;
  float delta = 0.0f, lse2 = 0.0f;
  {
    typename T::x8 of[D / 16];
    load_rows<T, D>(a.O + o_head, o_stride, row, ok, hlf, of);
#pragma unroll
    for (int s = 0; s < D / 16; ++s)
#pragma unroll
      for (int e = 0; e < 8; ++e) delta = fmaf(static_cast<float>(gf[s][e]), static_cast<float>(of[s][e]), delta);
    delta = sum_halves(delta);
    if (ok) {
      const float lse = a.LSE[static_cast<int64_t>(h) * a.q_rows + p.q0 + row];
      // a row that sees nothing: against +inf every weight is 0
      lse2 = lse == -__builtin_inff() ? __builtin_inff() : fmaf(lse, kLog2e, -kWeightShift<T>);
    }
  }
  float more = 0.0f;
  f32x16_t acc[D / 32], keys[D / 32];  // the sums over the keys of the gradient against D', of the weights
#pragma unroll
  for (int db = 0; db < D / 32; ++db) {
    acc[db] = f32x16_t{};
    keys[db] = f32x16_t{};
  }
  Reach<T> reach;
  arrived(qf);
  if constexpr (!kRowsInLds) arrived(gf);
  for (int i = 0, j = team; i * kTeams < nb; ++i, j += kTeams) {
    wait_vm<0>();
    __syncthreads();  // the team's block j is there, and everyone is done with the one before
    if (j + kTeams < nb) load(i + 1, j + kTeams);
    if (j >= wave_nb) continue;
    const int buf = (i & 1) * kTile;
#pragma unroll
    for (int kb = 0; kb < kKeys / 32; ++kb) {
      const int key0 = j * kKeys + 32 * kb;
      f32x16_t sc[1] = {f32x16_t{}}, dp{};
#pragma unroll
      for (int s = 0; s < D / 16; ++s) {
        sc[0] = T::mfma(row_frag<T, D>(sK + buf, fr, s, 32 * kb), qf[s], sc[0]);
        const typename T::x8 g = kRowsInLds ? __builtin_bit_cast(typename T::x8, my_rows[64 * s]) : gf[s];
        dp = T::mfma(row_frag<T, D>(sV + buf, fr, s, 32 * kb), g, dp);
      }
      f32x16_t slip{};
      if constexpr (!kPlain) {
        cap_scores<1>(a.scoring, sc);
#pragma unroll
        for (int r = 0; r < 16; ++r) slip[r] = a.scoring.cap_in != 0.0f ? fmaf(-sc[0][r], sc[0][r], 1.0f) : 1.0f;
        bias_scores<1, -1>(a.scoring, slope, at - key0, hlf, sc);
      }
      f32x16_t w;
#pragma unroll
      for (int r = 0; r < 16; ++r) w[r] = __builtin_amdgcn_exp2f(fmaf(sc[0][r], c, -lse2));
      if (key0 + 32 > wave_lo) {
#pragma unroll
        for (int r = 0; r < 16; ++r)
          if (key0 + result_row(r, hlf) >= hi) w[r] = dp[r] = 0.0f;  // (dp: it may be anything)
      }
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        dp[r] = w[r] * (dp[r] - delta);
        more += dp[r];
        if constexpr (!kPlain) {
          dp[r] *= slip[r];
          w[r] *= slip[r];
        }
      }
      reach.take(dp, acc);
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        const typename T::x8 ds = pack<T>(dp, t), wt = pack<T>(w, t);
#pragma unroll
        for (int db = 0; db < D / 32; ++db) {
          const typename T::x8 kf = col_frag<T, D>(sK_lds + buf, fr, db, 32 * kb + 16 * t);
          acc[db] = T::mfma(kf, ds, acc[db]);
          keys[db] = T::mfma(kf, wt, keys[db]);
        }
      }
    }
  }
  more = sum_halves(more);
  if constexpr (kTeams > 1) {
    s_more[team][wave][lane] = more;
    __syncthreads();
    more = 0.0f;
#pragma unroll
    for (int n = 0; n < kTeams; ++n) more += s_more[n][wave][lane];
  }
  more = a.joined ? 0.0f : more * kWeightUnit<T>;
  if (ok && hlf == 0 && team == 0) {
    const int64_t pitch = a.q_rows;
    float* st = a.stats + h * pitch + p.q0 + row;
    st[0] = lse2;
    st[a.H * pitch] = -(delta + more);
  }
#pragma unroll
  for (int db = 0; db < D / 32; ++db)
#pragma unroll
    for (int r = 0; r < 16; ++r)
      acc[db][r] = fmaf(-more * kWeightUnit<T>, keys[db][r], acc[db][r] * (reach.back() * kWeightUnit<T>));
  if constexpr (kTeams > 1) {
    static_assert(sizeof(stage) >= (kTeams - 1) * S::kWaves * 64 * (D / 2) * 4, "the teams' sums fit the buffers");
    f32x4_t* sums = reinterpret_cast<f32x4_t*>(stage) + wave * (D / 8) * 64 + lane;
    constexpr int kTeamSums = S::kWaves * (D / 8) * 64;
    __syncthreads();
    if (team > 0) put_sums<D>(sums + (team - 1) * kTeamSums, acc);
    __syncthreads();
    if (team > 0) return;
#pragma unroll
    for (int n = 0; n < kTeams - 1; ++n) add_sums<D>(sums + n * kTeamSums, acc, 1.0f, 1.0f);
  }
  if (ok) store_rows<T, D>(a.dQ + p.q0 * a.dq_stride + h * D, a.dq_stride, row, hlf, acc, a.scale);
}

// ---- gradients of the keys and values ------------------------------------------------------
// A tile is 128 keys of one key/value head, 32 a wave, whose gradients stay in registers while
// the rows that see them pass, head by head of the group: a sum over shared heads is no more
// than a longer loop, in a fixed order. For D = 128 the gradients take half of a wave's registers:
// the rows of V are read from LDS, and a second team of waves takes the second half of each step's
// rows, so that a SIMD has two waves although the longest causal tiles are as long as all of a CU's.
// 8192 causal rows, 32 heads on 8 of 128: 1.05 to 1.10 ms, four products of the pairs at 1.0 PFLOP/s, 47 % matrix
// and 24 % vector instructions; both teams
// meet at each step's barrier, and what a wave does between its products is not all hidden. One team,
// fragments read a phase ahead: 1.27; without that 1.73; a team for each gradient, which both need the
// weights, 1.44; tiles of 64 keys with two workgroups a CU 1.41; the second team's sums a step late,
// behind the first team's products, 1.14. Two teams for heads of 64: packed documents of up to 721
// rows 94 instead of 89 us, 4096 rows 135 instead of 155.
template <int D>
constexpr int kKvTeams = D == 128 ? 2 : 1;

template <class T, int D, bool kPlain>
__global__ __launch_bounds__(256 * kKvTeams<D>, 2) void doc_grad_kv(DocAttnArgs a) {
  constexpr int kTile = kDocBlock * D * 2, kTeams = kKvTeams<D>;
  constexpr bool kRowsInLds = D == 128;
  __shared__ __attribute__((aligned(1024))) unsigned char stage[4 * kTile];  // rows of Q, of dO: two steps each
  __shared__ u32x4_t s_rows[kRowsInLds ? 4 * (D / 16) * 64 : 1];  // of V, by wave, fragment and lane; the teams hold the same
  __shared__ __attribute__((aligned(256))) float s_stats[2][2][kDocBlock];  // log-sum-exp, delta
  const int lane = threadIdx.x & 63, any_wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wave = any_wave & 3, team = any_wave >> 2;
  const int l32 = lane & 31, hlf = lane >> 5;
  const int kvh = blockIdx.x % a.Hkv, part = blockIdx.x / a.Hkv % a.row_parts;
  const Place p = find_place(a, blockIdx.x / (a.Hkv * a.row_parts), kDocTileRows, true);  // (the first keys have the most rows)
  if (!p.any) return;
  const int G = a.H / a.Hkv;
  const int shift = p.k_len - p.q_len;
  // the first row that sees key j
  auto first_row = [&](int j) { return a.causal && j >= p.prefix ? max(0, j - shift) : 0; };
  const int first = p.first + wave * 32;
  const int key = first + l32;
  const bool ok = key < p.k_len;
  const int lo = first_row(key);
  const int wave_hi = first_row(first + 31);  // rows from here on see every key of the wave
  const int wave_lo = first < p.k_len ? first_row(first) : p.q_len;  // rows before see none
  const int r0 = min(first_row(p.first), p.q_len);
  const int nb = (p.q_len - r0 + kDocBlock - 1) / kDocBlock;
  // this workgroup's part of all heads' blocks of rows: steps begin .. begin + steps - 1
  const int64_t all_steps = static_cast<int64_t>(nb) * G;
  const int begin = static_cast<int>(all_steps * part / a.row_parts);
  const int steps = static_cast<int>(all_steps * (part + 1) / a.row_parts) - begin;

  const LoadLane<D> ll(lane);
  const Frags<D> fr(lane);
  const unsigned char* const sQ = stage;
  const unsigned char* const sG = stage + 2 * kTile;
  const uint32_t sQ_addr = lds_address(sQ), sG_addr = lds_address(sG), st_addr = lds_address(s_stats);
  const int64_t o_stride = static_cast<int64_t>(a.H) * D;
  const int64_t pitch = a.q_rows;
  const uint16_t* qh = a.Q + p.q0 * a.q_stride + kvh * G * D;
  const uint16_t* gh = a.dO + p.q0 * o_stride + kvh * G * D;
  const int first_g = nb > 0 ? begin / nb : 0, first_j = begin - first_g * nb;
  int load_g = first_g, load_j = first_j;  // the next step to load: block load_j of head load_g
  auto load = [&](int at) {
    const int64_t r = r0 + load_j * kDocBlock;
    const int rows = p.q_len - static_cast<int>(r);
    load_tile<D, kDocBlock, 4 * kTeams>(qh + r * a.q_stride + load_g * D, a.q_stride, rows, sQ_addr + at * kTile, any_wave, ll);
    load_tile<D, kDocBlock, 4 * kTeams>(gh + r * o_stride + load_g * D, o_stride, rows, sG_addr + at * kTile, any_wave, ll);
    if (any_wave < 2) {  // (as loads of the tile, or waiting for them would wait for the tile)
      const float* st = a.stats + (any_wave * a.H + kvh * G + load_g) * pitch + p.q0 + r;
      load_dword_to_lds(make_rsrc(st, 4 * min(kDocBlock, rows)), st_addr + 4 * kDocBlock * (at * 2 + any_wave), 4 * lane);
    }
    if (++load_j == nb) {
      load_j = 0;
      ++load_g;
    }
  };
  if (steps > 0) load(0);

  typename T::x8 kf[D / 16], vf[D / 16];
  load_rows<T, D>(a.K + p.k0 * a.k_stride + kvh * D, a.k_stride, key, ok, hlf, kf);
  load_rows<T, D>(a.V + p.k0 * a.v_stride + kvh * D, a.v_stride, key, ok, hlf, vf);
  u32x4_t* const my_rows = s_rows + (kRowsInLds ? wave * (D / 16) * 64 + lane : 0);
  if constexpr (kRowsInLds) {
#pragma unroll
    for (int s = 0; s < D / 16; ++s) my_rows[64 * s] = __builtin_bit_cast(u32x4_t, vf[s]);
  }
  f32x16_t dk[D / 32], dv[D / 32];
#pragma unroll
  for (int db = 0; db < D / 32; ++db) {
    dk[db] = f32x16_t{};
    dv[db] = f32x16_t{};
  }
  Reach<T> reach;
  const float c = a.scoring.unit * kLog2e;
  arrived(kf);
  if constexpr (!kRowsInLds) arrived(vf);

  auto slope_at = [&](int g) { return kPlain ? 0.0f : arrived(slope_of(a.scoring, kvh * G + g)); };
  float slope = steps > 0 ? slope_at(first_g) : 0.0f;
  for (int i = 0, g = first_g, j = first_j; i < steps; ++i) {
    wait_vm<0>();
    __syncthreads();  // step i is there, and everyone is done with step i - 1
    const int at = i & 1;
    if (i + 1 < steps) load(at ^ 1);
    const unsigned char *tq = sQ + at * kTile, *tg = sG + at * kTile;
#pragma unroll
    for (int n = 0; n < kDocBlock / 32 / kTeams; ++n) {
      const int rb = kTeams == 1 ? n : team;
      const int row0 = r0 + j * kDocBlock + 32 * rb;
      if (row0 + 32 <= wave_lo || row0 >= p.q_len) continue;
      // q . k and do . v - delta of 32 rows and the wave's keys
      f32x16_t x{}, ds;
#pragma unroll
      for (int b = 0; b < 4; ++b) {
        const f32x4_t delta = *reinterpret_cast<const f32x4_t*>(&s_stats[at][1][32 * rb + 8 * b + 4 * hlf]);  // (negative)
#pragma unroll
        for (int r = 0; r < 4; ++r) ds[4 * b + r] = delta[r];
      }
#pragma unroll
      for (int s = 0; s < D / 16; ++s) {
        x = T::mfma(row_frag<T, D>(tq, fr, s, 32 * rb), kf[s], x);
        const typename T::x8 v = kRowsInLds ? __builtin_bit_cast(typename T::x8, my_rows[64 * s]) : vf[s];
        ds = T::mfma(row_frag<T, D>(tg, fr, s, 32 * rb), v, ds);
      }
      // them to weights and gradients of scores
      if constexpr (!kPlain) {
        f32x16_t sc[1] = {x};
        cap_scores<1>(a.scoring, sc);
        if (a.scoring.cap_in != 0.0f) {
#pragma unroll
          for (int r = 0; r < 16; ++r) ds[r] *= fmaf(-sc[0][r], sc[0][r], 1.0f);
        }
        bias_scores<1, 1>(a.scoring, slope, row0 + shift - key, hlf, sc);
        x = sc[0];
      }
#pragma unroll
      for (int b = 0; b < 4; ++b) {
        const f32x4_t lse2 = *reinterpret_cast<const f32x4_t*>(&s_stats[at][0][32 * rb + 8 * b + 4 * hlf]);
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          x[4 * b + r] = __builtin_amdgcn_exp2f(fmaf(x[4 * b + r], c, -lse2[r]));
          ds[4 * b + r] *= x[4 * b + r];
        }
      }
      if (row0 < wave_hi || row0 + 32 > p.q_len) {
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          const int row = row0 + result_row(r, hlf);
          const bool out = row < lo || row >= p.q_len;
          x[r] = out ? 0.0f : x[r];
          ds[r] = out ? 0.0f : ds[r];
        }
      }
      reach.take(ds, dk);
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        const typename T::x8 wt = pack<T>(x, t), dt = pack<T>(ds, t);
#pragma unroll
        for (int db = 0; db < D / 32; ++db) {
          dv[db] = T::mfma(col_frag<T, D>((const lds_u8_t*)tg, fr, db, 32 * rb + 16 * t), wt, dv[db]);
          dk[db] = T::mfma(col_frag<T, D>((const lds_u8_t*)tq, fr, db, 32 * rb + 16 * t), dt, dk[db]);
        }
      }
    }
    if (++j == nb) {
      j = 0;
      if (++g < G) slope = slope_at(g);
    }
  }
  if constexpr (T::kShortRange) {
#pragma unroll
    for (int db = 0; db < D / 32; ++db) {
      dk[db] *= reach.back() * kUnshift;
      dv[db] *= kUnshift;
    }
  }
  // the teams' sums: team 0 finishes those of the keys, team 1 those of the values
  if constexpr (kTeams == 2) {
    static_assert(sizeof(stage) >= 4 * 64 * (D / 2) * 4, "the sums fit the buffers");
    f32x4_t* sums = reinterpret_cast<f32x4_t*>(stage) + wave * (D / 8) * 64 + lane;
    __syncthreads();
    if (team == 1) put_sums<D>(sums, dk);
    __syncthreads();
    if (team == 0) {
      add_sums<D>(sums, dk, 1.0f, 1.0f);
      put_sums<D>(sums, dv);  // (each lane in the places that it has read)
    }
    __syncthreads();
    if (team == 1) add_sums<D>(sums, dv, 1.0f, 1.0f);
  }
  if (!ok) return;
  const bool has_dk = team == 0, has_dv = kTeams == 1 || team == 1;
  if (a.row_parts > 1) {  // for sum_parts
    float* to = a.parts + ((static_cast<int64_t>(part) * a.k_rows + p.k0 + key) * a.Hkv + kvh) * 2 * D + 4 * hlf;
    auto put = [&](float* to, const f32x16_t (&x)[D / 32]) {
#pragma unroll
      for (int db = 0; db < D / 32; ++db)
#pragma unroll
        for (int b = 0; b < 4; ++b)
          *reinterpret_cast<f32x4_t*>(to + 32 * db + 8 * b) = f32x4_t{x[db][4 * b], x[db][4 * b + 1], x[db][4 * b + 2], x[db][4 * b + 3]};
    };
    if (has_dk) put(to, dk);
    if (has_dv) put(to + D, dv);
    return;
  }
  if (has_dk) store_rows<T, D>(a.dK + p.k0 * a.dk_stride + kvh * D, a.dk_stride, key, hlf, dk, a.scale);
  if (has_dv) store_rows<T, D>(a.dV + p.k0 * a.dv_stride + kvh * D, a.dv_stride, key, hlf, dv, 1.0f);
}

// Sums the parts of the keys' and values' gradients, in their order: four elements a thread. Keys
// of no document are left as they are. Bound by the memory (the caches, for as few keys as have
// parts): 2048 keys of 8 heads of 128 in three parts are 50 MB.
template <class T, int D>
__global__ __launch_bounds__(kThreads) void sum_parts(DocAttnArgs a) {
  const int64_t i = static_cast<int64_t>(blockIdx.x) * kThreads + threadIdx.x;
  const int64_t total = static_cast<int64_t>(a.k_rows) * a.Hkv * (2 * D / 4);
  if (i >= total) return;
  const int col = static_cast<int>(i % (2 * D / 4)) * 4;
  const int64_t row = i / (2 * D / 4);
  const int key = static_cast<int>(row / a.Hkv), kvh = static_cast<int>(row - static_cast<int64_t>(key) * a.Hkv);
  // the document of the key
  int lo = 0;
  for (int n = a.n_docs; n > 1;) {
    const int half = n / 2;
    const bool up = a.k_ptr[lo + half] <= key;
    lo = up ? lo + half : lo;
    n = up ? n - half : half;
  }
  if (key < a.k_ptr[lo] || key >= a.k_ptr[lo + 1]) return;
  f32x4_t sum{};
  for (int r = 0; r < a.row_parts; ++r) sum += *reinterpret_cast<const f32x4_t*>(a.parts + r * total * 4 + 4 * i);
  const bool is_v = col >= D;
  if (!is_v) sum *= a.scale;
  uint16_t* to = is_v ? a.dV + key * a.dv_stride + kvh * D + col - D : a.dK + key * a.dk_stride + kvh * D + col;
  *reinterpret_cast<u32x2_t*>(to) = __builtin_bit_cast(u32x2_t, __builtin_convertvector(sum, typename T::x4));
}

// Tiles of rows, at most.
template <class S>
int64_t row_tiles(const DocAttnArgs& a) {
  return (a.q_rows / (32 * S::kWaves / a.tile_heads) + a.n_docs) * static_cast<int64_t>(a.H / a.tile_heads);
}

template <class T, int D, bool kPlain, bool kGradient, class S>
hipError_t launch_rows(DocAttnArgs a, hipStream_t stream) {
  a.tile_heads = std::gcd(a.H / a.Hkv, S::kWaves);
  const dim3 grid(row_tiles<S>(a)), block(S::kThreads);
  if constexpr (kGradient)
    hipLaunchKernelGGL((doc_grad_q<T, D, kPlain, Shape<S::kWaves, S::kTeams, D == 128 ? 32 : S::kKeys>>), grid, block, 0, stream, a);
  else
    hipLaunchKernelGGL((doc_forward<T, D, kPlain, S>), grid, block, 0, stream, a);
  return hipGetLastError();
}

// The shape of the tiles. While there are no more than CUs, the longest tile's way through its keys is
// what a call takes: four teams on half as many rows. Up to two a CU it still is if the documents are
// long, of 1000 keys on the average: two teams (forward with heads of 64, of which a CU holds two such
// workgroups, four teams a little beyond a tile a CU). With more tiles or shorter documents the teams
// would only wait for each other. Whole / halves / quarters, us, forward, documents causal and of one
// length: 32 heads on 8 of 128, 512 rows (136 tiles) 16.2 / 15.5 / 12.9; 1024 (264) 26.0 / 22.3 / 25.6; 2 of
// 1000 (512) 37.0 / 32.9 / 50.5; 2048 (520) 50.2 / 47.4 / 68.1; 4096 (1032) 148 / 153 / 210; 12 heads of 64, 2048 rows
// (204) 33.6 / 24.7 / 18.7, 3000 (288) 46.4 / 32.9 / 28.9, capped 64.0 / 52.1 / 39.0, 4096 (396) 62.7 / 44.3 / 46.3; 32 on
// 8 of 64, 2 of 1000 (512) 25.2 / 22.5 / 26.9; 12 heads of 64, 4 documents of 250 (132) 8.7 / 9.0 / 7.8, 5 of 700
// (384) 17.2 / 20.4 / 17.9, 16 of 250 (564) 13.2 / 16.9 / 17.7; 16 on 4 of 128, capped, 10 of 250 (352) 17.1 /
// 24.6 / 29.9. With the gradient: 16 on 4 of 128, capped, 3000 rows (376) 338 / 289 / 344, 10 of 250 81 / 98 / 117.
template <class T, int D, bool kPlain, bool kGradient>
hipError_t launch_rows(const DocAttnArgs& a, hipStream_t stream) {
  const int64_t tiles = row_tiles<Whole>(a);
  const bool long_docs = a.k_rows >= int64_t{1000} * a.n_docs;
  if (tiles <= a.cus || (!kGradient && D == 64 && long_docs && 4 * tiles <= 5 * static_cast<int64_t>(a.cus)))
    return launch_rows<T, D, kPlain, kGradient, Quarters>(a, stream);
  if (tiles <= 2 * a.cus && long_docs) return launch_rows<T, D, kPlain, kGradient, Halves>(a, stream);
  return launch_rows<T, D, kPlain, kGradient, Whole>(a, stream);
}

template <class T, int D, bool kPlain>
hipError_t forward(const DocAttnArgs& a, hipStream_t stream) {
  return launch_rows<T, D, kPlain, false>(a, stream);
}

template <class T, int D, bool kPlain>
hipError_t grad(const DocAttnArgs& a, hipStream_t stream) {
  hipError_t e = launch_rows<T, D, kPlain, true>(a, stream);
  if (e != hipSuccess) return e;
  const int64_t k_tiles = doc_key_tiles(a.k_rows, a.n_docs) * a.Hkv;
  hipLaunchKernelGGL((doc_grad_kv<T, D, kPlain>), dim3(k_tiles * a.row_parts), dim3(256 * kKvTeams<D>), 0, stream, a);
  e = hipGetLastError();
  if (e != hipSuccess || a.row_parts == 1) return e;
  const int64_t sums = static_cast<int64_t>(a.k_rows) * a.Hkv * (2 * D / 4);
  hipLaunchKernelGGL((sum_parts<T, D>), dim3((sums + kThreads - 1) / kThreads), dim3(kThreads), 0, stream, a);
  return hipGetLastError();
}

template <class T, int D>
hipError_t dispatch(const DocAttnArgs& a, bool gradient, hipStream_t s) {
  if (a.scoring.plain()) return gradient ? grad<T, D, true>(a, s) : forward<T, D, true>(a, s);
  return gradient ? grad<T, D, false>(a, s) : forward<T, D, false>(a, s);
}

hipError_t dispatch(const DocAttnArgs& a, bool f16, int head_dim, bool gradient, hipStream_t s) {
  if (head_dim == 128) return f16 ? dispatch<F16, 128>(a, gradient, s) : dispatch<Bf16, 128>(a, gradient, s);
  return f16 ? dispatch<F16, 64>(a, gradient, s) : dispatch<Bf16, 64>(a, gradient, s);
}

}  // namespace

hipError_t launch_doc_forward(const DocAttnArgs& a, bool f16, int head_dim, hipStream_t stream) {
  return dispatch(a, f16, head_dim, false, stream);
}
hipError_t launch_doc_grad(const DocAttnArgs& a, bool f16, int head_dim, hipStream_t stream) {
  return dispatch(a, f16, head_dim, true, stream);
}

}  // namespace csg
