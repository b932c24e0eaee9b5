// A paged key/value cache for gfx950 (CDNA4): new tokens go in, attention reads it.
//
// Sequence b's keys and values are tokens 0 .. lens[b] - 1; token x lies in page
// table[b][x / page size] at row x % page size, all rows of a head of a page behind each
// other. A call's new tokens q_ptr[b] .. q_ptr[b+1] - 1 are the last of sequence b.
#include <hip/hip_runtime.h>

#include "cache_attn.hpp"
#include "cache_plan.hpp"

namespace csg {
namespace {

using namespace cache;

// ---- new tokens into the cache --------------------------------------------------------------
// A workgroup per token. Pair i of a head (elements i and half + i, or 2 i and 2 i + 1) turns by
// the angle position * inv_freq[i]. The angle is reduced to a fraction of a turn in 64 bits: at
// position 1e6 a 32-bit product is off by 0.06. A thread keeps eight pairs' sines and cosines
// and goes through the heads, 16 elements of each: two loads and two stores of 16 bytes.
// Bound by the memory: 11322 tokens of 64 heads and 2 x 8 of the cache, half of 128 elements rotated,
// 464 MB in 104 us, 4.45 TB/s (a large copy: 4.9). Stores past the caches took 102 us, loads past them
// 108, two heads a turn 104. 64 tokens take 4.6 us, where the host's call takes 8.
template <class T, int D>
__global__ __launch_bounds__(kThreads) void cache_append(AppendArgs a) {
  constexpr int kCols = D / 16, kHeads = kThreads / kCols;
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
  const int col = threadIdx.x % kCols;
  const bool turns = 8 * col < a.half;
  float cs[8], sn[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    cs[e] = 1.0f;
    sn[e] = 0.0f;
    if (turns) {
      const double turn = static_cast<double>(pos) * a.inv_freq[8 * col + e] * 0.15915494309189533577;
      const float part = static_cast<float>(turn - rint(turn));  // the hardware's sine takes turns
      cs[e] = __builtin_amdgcn_cosf(part);
      sn[e] = __builtin_amdgcn_sinf(part);
    }
  }
  const bool split = turns && !a.interleaved;
  const int x0 = split ? 8 * col : 16 * col, x1 = split ? a.half + 8 * col : 16 * col + 8;
  const int n_q = c.Q ? c.H : 0, heads = n_q + 2 * c.Hkv;
  const int page_size = 1 << c.page_shift;
  for (int i = threadIdx.x / kCols; i < heads; i += kHeads) {
    const uint16_t* src;
    uint16_t* dst;
    const bool is_v = i >= n_q + c.Hkv;
    if (i < n_q) {
      src = c.Q + t * c.q_stride + i * D;
      dst = a.q_out + (static_cast<int64_t>(t) * c.H + i) * D;
    } else {
      if (page < 0) break;
      const int h = i - n_q - (is_v ? c.Hkv : 0);
      src = (is_v ? a.V + t * a.v_stride : a.K + t * a.k_stride) + h * D;
      dst = (is_v ? c.v_pages : c.k_pages) +
            ((static_cast<int64_t>(page) * c.Hkv + h) * page_size + (pos & (page_size - 1))) * D;
    }
    if (is_v || !turns) {  // as it is, in any order of the columns
      const u32x4_t y0 = *reinterpret_cast<const u32x4_t*>(src + x0), y1 = *reinterpret_cast<const u32x4_t*>(src + x1);
      *reinterpret_cast<u32x4_t*>(dst + x0) = y0;
      *reinterpret_cast<u32x4_t*>(dst + x1) = y1;
      continue;
    }
    const typename T::x8 y0 = *reinterpret_cast<const typename T::x8*>(src + x0);
    const typename T::x8 y1 = *reinterpret_cast<const typename T::x8*>(src + x1);
    f32x8_t z0, z1;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      if (a.interleaved) {
        const float x = static_cast<float>(e < 4 ? y0[2 * (e & 3)] : y1[2 * (e & 3)]);
        const float y = static_cast<float>(e < 4 ? y0[2 * (e & 3) + 1] : y1[2 * (e & 3) + 1]);
        const float u = fmaf(x, cs[e], -y * sn[e]), v = fmaf(y, cs[e], x * sn[e]);
        if (e < 4) {
          z0[2 * (e & 3)] = u;
          z0[2 * (e & 3) + 1] = v;
        } else {
          z1[2 * (e & 3)] = u;
          z1[2 * (e & 3) + 1] = v;
        }
      } else {
        const float x = static_cast<float>(y0[e]), y = static_cast<float>(y1[e]);
        z0[e] = fmaf(x, cs[e], -y * sn[e]);
        z1[e] = fmaf(y, cs[e], x * sn[e]);
      }
    }
    *reinterpret_cast<typename T::x8*>(dst + x0) = __builtin_convertvector(z0, typename T::x8);
    *reinterpret_cast<typename T::x8*>(dst + x1) = __builtin_convertvector(z1, typename T::x8);
  }
}

// ---- attention over the cache ---------------------------------------------------------------
// Work: entry e < n_groups is the shared keys of a group, for the rows of all its sequences;
// entry n_groups + b is the other keys of sequence b, for its own rows. A row is a new token and
// a head of the key/value head's group, tokens first. Up to 32 rows of an entry are a narrow
// task: the four waves take different blocks of 32 keys for the same rows, each at its own
// pace. More rows make wide tasks of 128, 32 a wave, whose waves share the keys. Every key/value
// head has the same number of workgroups. All tasks' blocks of 32 keys stand in one row (by
// entry, task, block), each task's behind as many empty ones as it costs, and the row is cut into equal
// runs, one a workgroup of the head: every workgroup has the same to do, whatever the lengths
// are. What a workgroup has of a task is a
// part: for each tile of 32 rows, its weights' sums and products against its own reference,
// which cache_merge joins. With the tiles counted through, tile t of run w is in place t + 4 w:
// of two parts one after the other, the second has a later tile, or the next run and at most
// the three tiles before.
// Bound by the memory where keys are many: 2 sequences of over 100000, 918 MB in 160 us and the merge
// 7, 5.4 TB/s; 64 sequences of up to 8000, 483 MB, 94 and 6. With few keys by a chain of latencies
// (bounds, page numbers, keys, products, partial results), 9 us for 900 keys; where 16
// sequences' rows share 8192 keys by what a part costs besides its keys and by 16 MB of partial
// results (36 us and 8; the keys alone would take 27).
// Keys (or values) key .. key + 15, which lie in one page, into LDS; what is behind the part's
// end or before its entry's keys (a sequence need not have its group's tokens in pages of its
// own) reads zero.
template <int D>
__device__ __forceinline__ void load_16(const CacheArgs& c, const uint16_t* pages, const Part& p, int page, int key, uint32_t lds,
                                        const LoadLane<D>& ll) {
  const int rows = page < 0 ? 0 : clamped(p.end - key, 0, 16);
  const int64_t row = ((static_cast<int64_t>(max(page, 0)) * c.Hkv + p.kvh) << c.page_shift) + (key & ((1 << c.page_shift) - 1));
  const __amdgpu_buffer_rsrc_t rs = make_rsrc(pages + row * D, rows * 2 * D);
  if (key < p.lo) {
    const int skip = (p.lo - key) * 2 * D;
#pragma unroll
    for (int i = 0; i < 16 / kLoadRows<D>; ++i) {
      const int at = ll.offset(i, 2 * D);
      load_to_lds(rs, lds + 1024u * i, at < skip ? 1 << 30 : at);
    }
    return;
  }
#pragma unroll
  for (int i = 0; i < 16 / kLoadRows<D>; ++i) load_to_lds(rs, lds + 1024u * i, ll.offset(i, 2 * D));
}

// A narrow part: each wave takes every fourth block, through 16 KiB (D = 128) of LDS of its own:
// the next keys load once the products have read the last, the next values once the sums have.
// Two workgroups a CU keep 128 KiB in flight, and one streams while the other begins or ends
// a part.
template <class T, int D, bool kPlain>
__device__ __forceinline__ void narrow_part(const CacheAttnArgs& a, const Entry& x, const KeptEntry* local, Part& p, unsigned char* stage, float (&s_ref)[4][32],
                                            float (&s_sum)[4][32], float* out, int lane, int wave) {
  constexpr int kTile = kCacheBlock * 2 * D, kLoads = kCacheBlock / kLoadRows<D>;
  const CacheArgs& c = a.c;
  const int l32 = lane & 31, hlf = lane >> 5;
  const LoadLane<D> ll(lane);
  unsigned char* mine = stage + wave * 2 * kTile;
  const uint32_t k_lds = lds_address(mine), v_lds = k_lds + kTile;
  const int count = (p.end - p.key0 + kCacheBlock - 1) / kCacheBlock;
  const int mine_n = count > wave ? (count - wave + 3) / 4 : 0;

  // lane n holds the page of the 16 keys n % 2 of the wave's block n / 2 (32 blocks at a time)
  int pages = -1;
  auto key_of = [&](int n) { return p.key0 + (wave + 4 * n) * kCacheBlock; };
  auto fetch = [&](int n) { pages = page_of(c, p, key_of(n + (lane >> 1)) + 16 * (lane & 1)); };
  auto load = [&](int n, const uint16_t* from, uint32_t lds) {
#pragma unroll
    for (int half = 0; half < 2; ++half)
      load_16<D>(c, from, p, __builtin_amdgcn_readlane(pages, 2 * (n & 31) + half), key_of(n) + 16 * half, lds + half * (kTile / 2), ll);
  };
  if (mine_n > 0) {
    fetch(0);
    load(0, c.k_pages, k_lds);
    load(0, c.v_pages, v_lds);
  }
  locate_row(a, x, local, l32, p);
  typename T::x8 qf[D / 16];
  load_queries<T, D>(a, p, hlf, qf);
  const float slope = kPlain ? 0.0f : slope_of(a.scoring, p.h);
  const float cexp = a.scoring.unit * kLog2e;
  const Frags<D> fr(lane);
  f32x16_t acc[D / 32];
#pragma unroll
  for (int db = 0; db < D / 32; ++db) acc[db] = f32x16_t{};
  RowSoftmax sm;
  arrived(qf);
  for (int n = 0; n < mine_n; ++n) {
    const bool more = n + 1 < mine_n;
    wait_vm<kLoads>();  // the keys are there; the values may be on their way
    f32x16_t sc[1] = {f32x16_t{}};
#pragma unroll
    for (int s = 0; s < D / 16; ++s) sc[0] = T::mfma(row_frag<T, D>(mine, fr, s, 0), qf[s], sc[0]);
    wait_lds();  // the keys have been read
    if (more) {
      if (((n + 1) & 31) == 0) fetch(n + 1);
      load(n + 1, c.k_pages, k_lds);
    }
    finish_scores<1, kPlain>(a, p, slope, key_of(n), hlf, sc);
    typename T::x8 pb[2];
    bool moved;
    const float alpha = sm.block<T, 1>(sc, cexp, pb, moved);
    if (moved) {
#pragma unroll
      for (int db = 0; db < D / 32; ++db) acc[db] *= alpha;
    }
    if (more)
      wait_vm<kLoads>();
    else
      wait_vm<0>();
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int db = 0; db < D / 32; ++db)
        acc[db] = T::mfma(col_frag<T, D>((const lds_u8_t*)(mine + kTile), fr, db, 16 * t), pb[t], acc[db]);
    wait_lds();
    if (more) load(n + 1, c.v_pages, v_lds);
  }

  // the waves' results against their common reference, summed in the order of the waves; the
  // 16-byte pieces of a row are turned by its number, against bank conflicts
  const float l = sum_halves(sm.l);
  if (hlf == 0) {
    s_ref[wave][l32] = sm.m;
    s_sum[wave][l32] = l;
  }
  __syncthreads();  // (also: every wave has read its stage)
  const float top = fmaxf(fmaxf(s_ref[0][l32], s_ref[1][l32]), fmaxf(s_ref[2][l32], s_ref[3][l32]));
  const int live = min(kCacheTileRows, x.rows - p.tile * kCacheTileRows);
  constexpr int kPieces = D / 4;
  if (l32 < live) {
    const float f = factor(sm.m, top, cexp);
    f32x4_t* to = reinterpret_cast<f32x4_t*>(stage) + (wave * 32 + l32) * kPieces;
#pragma unroll
    for (int db = 0; db < D / 32; ++db)
#pragma unroll
      for (int q = 0; q < 4; ++q)
        to[(8 * db + 2 * q + hlf) ^ (l32 & 7)] =
            f32x4_t{acc[db][4 * q] * f, acc[db][4 * q + 1] * f, acc[db][4 * q + 2] * f, acc[db][4 * q + 3] * f};
  }
  __syncthreads();
  if (out) {
    const f32x4_t* in = reinterpret_cast<const f32x4_t*>(stage);
    const int tid = wave * 64 + lane;
    for (int i = tid; i < live * kPieces; i += kThreads) {
      const int row = i / kPieces, at = row * kPieces + ((i % kPieces) ^ (row & 7));
      f32x4_t v = in[at];
#pragma unroll
      for (int k = 1; k < 4; ++k) v += in[k * 32 * kPieces + at];
      *reinterpret_cast<f32x4_t*>(out + 4 * i) = v;
    }
    if (tid < live) {
      float sum = 0.0f;
#pragma unroll
      for (int k = 0; k < 4; ++k) sum = fmaf(s_sum[k][l32], factor(s_ref[k][l32], top, cexp), sum);
      out[32 * D + l32] = top;
      out[32 * D + 32 + l32] = sum;
    }
  }
  __syncthreads();  // the stages are free again
}

// A wide part: blocks of 64 keys in two buffers, which all waves read.
template <class T, int D, bool kPlain>
__device__ __forceinline__ void wide_part(const CacheAttnArgs& a, const Entry& x, const KeptEntry* local, Part& p, unsigned char* stage, float* out, int lane,
                                          int wave) {
  constexpr int kTile = kCacheWideBlock * 2 * D;
  const CacheArgs& c = a.c;
  const int l32 = lane & 31, hlf = lane >> 5;
  const LoadLane<D> ll(lane);
  const uint32_t lds = lds_address(stage) + static_cast<uint32_t>(wave * 16 * 2 * D);
  const int nb = (p.end - p.key0 + kCacheWideBlock - 1) / kCacheWideBlock;
  // a wave brings 16 keys and values of each block; lane n holds the page of those of block n
  // (64 blocks at a time)
  int pages = -1;
  auto fetch = [&](int n) { pages = page_of(c, p, p.key0 + (n + lane) * kCacheWideBlock + 16 * wave); };
  auto load = [&](int n) {
    if (n > 0 && (n & 63) == 0) fetch(n);
    const int page = __builtin_amdgcn_readlane(pages, n & 63), key = p.key0 + n * kCacheWideBlock + 16 * wave;
    const uint32_t to = lds + (n & 1) * 2 * kTile;
    load_16<D>(c, c.k_pages, p, page, key, to, ll);
    load_16<D>(c, c.v_pages, p, page, key, to + kTile, ll);
  };
  fetch(0);
  load(0);
  locate_row(a, x, local, l32, p);
  typename T::x8 qf[D / 16];
  load_queries<T, D>(a, p, hlf, qf);
  const float slope = kPlain ? 0.0f : slope_of(a.scoring, p.h);
  const float cexp = a.scoring.unit * kLog2e;
  const Frags<D> fr(lane);
  f32x16_t acc[D / 32];
#pragma unroll
  for (int db = 0; db < D / 32; ++db) acc[db] = f32x16_t{};
  RowSoftmax sm;
  const bool idle = p.tile * kCacheTileRows >= x.rows;  // no row in this wave
  arrived(qf);
  for (int n = 0; n < nb; ++n) {
    wait_vm<0>();
    __syncthreads();  // block n is there, and everyone is done with block n - 1
    if (n + 1 < nb) load(n + 1);
    if (idle) continue;
    const unsigned char* kt = stage + (n & 1) * 2 * kTile;
    f32x16_t sc[2] = {f32x16_t{}, f32x16_t{}};
#pragma unroll
    for (int s = 0; s < D / 16; ++s)
#pragma unroll
      for (int kb = 0; kb < 2; ++kb) sc[kb] = T::mfma(row_frag<T, D>(kt, fr, s, 32 * kb), qf[s], sc[kb]);
    finish_scores<2, kPlain>(a, p, slope, p.key0 + n * kCacheWideBlock, hlf, sc);
    typename T::x8 pb[4];
    bool moved;
    const float alpha = sm.block<T, 2>(sc, cexp, pb, moved);
    if (moved) {
#pragma unroll
      for (int db = 0; db < D / 32; ++db) acc[db] *= alpha;
    }
#pragma unroll
    for (int t = 0; t < 4; ++t)
#pragma unroll
      for (int db = 0; db < D / 32; ++db)
        acc[db] = T::mfma(col_frag<T, D>((const lds_u8_t*)(kt + kTile), fr, db, 16 * t), pb[t], acc[db]);
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

template <class T, int D, bool kPlain>
__global__ __launch_bounds__(kThreads, 2) void cache_attn(CacheAttnArgs a) {
  __shared__ __attribute__((aligned(1024))) unsigned char stage[4 * 2 * kCacheBlock * 2 * D];
  __shared__ float s_ref[4][32], s_sum[4][32];
  static_assert(sizeof(stage) == 2 * 2 * kCacheWideBlock * 2 * D, "the same memory holds the wide parts' buffers");
  static_assert(sizeof(stage) >= 4 * 32 * D * 4, "and the waves' results");
  static_assert(sizeof(stage) >= kCacheGroupBytes, "and, before, the groups");
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  cache_run<0, 0, 0>(a, stage, [&](const Entry& x, const KeptEntry* local, Part& p, int64_t place, bool wide, bool) {
    if (wide) {
      p.tile += wave;
      wide_part<T, D, kPlain>(a, x, local, p, stage, part_at<D>(a, place + wave), lane, wave);
    } else {
      narrow_part<T, D, kPlain>(a, x, local, p, stage, s_ref, s_sum, part_at<D>(a, place), lane, wave);
    }
  });
}

// The parts of one row of an entry, and what has been loaded of the first 64 of them.
template <int D>
struct RowParts {
  static constexpr int kSide = 256 / D, kAtOnce = 4;
  const unsigned char* base;
  int64_t step;  // bytes from a part to the next
  int count = 0, in_tile;
  float m, l;             // of part `lane`
  f32x4_t in[kAtOnce];    // products of the first parts
  __device__ __forceinline__ const float* part(int q) const { return reinterpret_cast<const float*>(base + q * step); }
  __device__ __forceinline__ void find(const CacheAttnArgs& a, const Plan& plan, const PlanEntry& x, int kvh, int r) {
    if (x.blocks == 0 || r < 0 || r >= x.rows) return;
    const int tile = r / kCacheTileRows;
    in_tile = r % kCacheTileRows;
    const bool wide = x.rows > kCacheTileRows;
    const bool other = x.rows > kCacheAloneRows;
    const int run = other ? plan.run[1] : plan.run[0], shift = other ? plan.shift[1] : plan.shift[0], cost = other ? plan.cost[1] : plan.cost[0];
    // the first block's unit of its task
    const int start = x.before + (wide ? r / kCacheWideRows : 0) * (x.blocks + cost) + cost;
    const int w0 = start / run, w1 = (start + x.blocks - 1) / run;
    const int64_t first = static_cast<int64_t>(kvh) * (plan.tiles + 4 * a.head_workers) + x.tiles + tile + (w0 << shift);
    count = static_cast<int>(min<int64_t>(w1 - w0 + 1, (a.max_parts - first + (1 << shift) - 1) >> shift));
    step = cache_part_bytes(D) << shift;
    base = a.ws + cache_plan_bytes() + first * cache_part_bytes(D);
  }
  // (behind the end of p0 .. p0 + n - 1 the last one again, which weighs 0 there)
  __device__ __forceinline__ void load_products(int p0, int n, int q0, int side, int col) {
#pragma unroll
    for (int q = 0; q < kAtOnce; ++q)
      in[q] = *reinterpret_cast<const f32x4_t*>(part(p0 + min(q0 + kSide * q + side, n - 1)) + in_tile * D + col);
  }
  __device__ __forceinline__ void load(int p0, int lane, int side, int col) {
    m = -__builtin_inff();
    l = 0.0f;
    if (count <= p0) return;
    const int n = min(64, count - p0);
    if (lane < n) {
      m = part(p0 + lane)[32 * D + in_tile];
      l = part(p0 + lane)[32 * D + 32 + in_tile];
    }
    load_products(p0, n, 0, side, col);
  }
};

// One wave joins the parts of one row, as sum_w f_w acc_w / sum_w f_w l_w with f_w = e^(m_w - max m). A
// latency chain of the bounds, the plan, and the references and first products of both entries at once: 3.7 us for a row of some
// parts, 7.5 for 4096 rows, whose parts (16 MB) come from the caches. D / 4 lanes hold
// the row's products of one part, so that 256 / D parts stand side by side in the wave; each of them sums every (256 / D)th part.
template <class T, int D>
__global__ __launch_bounds__(kThreads) void cache_merge(CacheAttnArgs a) {
  constexpr int kSide = RowParts<D>::kSide, kAtOnce = RowParts<D>::kAtOnce;
  const CacheArgs& c = a.c;
  const int lane = threadIdx.x & 63;
  const uint32_t row = blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);  // (at most 2^25 of them)
  const int token = row / static_cast<uint32_t>(c.H), h = row % static_cast<uint32_t>(c.H);
  const Plan plan = *plan_in(a.ws);
  int b;
  if (c.batch < 64) {  // all bounds at once
    const int bound = c.q_ptr[min(lane, c.batch)];
    const uint64_t below = __builtin_amdgcn_ballot_w64(bound <= token);
    if (!(below & 1) || (below >> c.batch & 1)) return;  // (a row of no sequence)
    b = 63 - __builtin_clzll(below & ((1ull << c.batch) - 1));
  } else {
    if (token < first_token(c, 0) || token >= first_token(c, c.batch)) return;
    b = last_below(c.batch, [&](int i) { return c.q_ptr[i] <= token; });
  }
  if (token >= c.tokens) return;
  const int G = c.H / c.Hkv, kvh = h / G;
  const PlanEntry own = entries_in(a.ws)[a.n_groups + b];
  const float cexp = a.scoring.unit * kLog2e;
  const int side = lane / (D / 4), col = 4 * (lane % (D / 4));
  RowParts<D> sets[2];  // its group's keys, its own
  if (own.group >= 0) {
    const PlanEntry x = entries_in(a.ws)[own.group];
    sets[0].find(a, plan, x, kvh, (token - x.token0) * G + (h - kvh * G));
  }
  sets[1].find(a, plan, own, kvh, (token - own.token0) * G + (h - kvh * G));
  sets[0].load(0, lane, side, col);
  sets[1].load(0, lane, side, col);
  f32x4_t acc{};
  float m = -__builtin_inff(), l = 0.0f;
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    RowParts<D>& s = sets[i];
    // 64 parts at a time: their references and sums by the lanes, then their products
    for (int p0 = 0; p0 < s.count; p0 += 64) {
      const int n = min(64, s.count - p0);
      if (p0) s.load(p0, lane, side, col);
      float top = s.m;
#pragma unroll
      for (int d = 1; d < 64; d *= 2) top = fmaxf(top, __shfl_xor(top, d));
      top = fmaxf(top, m);
      const float f = factor(m, top, cexp), pf = factor(s.m, top, cexp);
      float sum = s.l * pf;
#pragma unroll
      for (int d = 1; d < 64; d *= 2) sum += __shfl_xor(sum, d);
      l = fmaf(l, f, sum);
      acc *= f;
      m = top;
      for (int q0 = 0; q0 < n; q0 += kSide * kAtOnce) {
        if (q0) s.load_products(p0, n, q0, side, col);
#pragma unroll
        for (int q = 0; q < kAtOnce; ++q) {
          const int at = q0 + kSide * q + side;
          const float wt = __shfl(pf, min(at, 63));
          if (at < n) acc += s.in[q] * wt;
        }
      }
    }
  }
#pragma unroll
  for (int d = D / 4; d < 64; d *= 2)
#pragma unroll
    for (int k = 0; k < 4; ++k) acc[k] += __shfl_xor(acc[k], d);
  const bool none = l == 0.0f;  // nothing visible (its products may hold what masked keys have)
  const float inv = none ? 0.0f : 1.0f / l;
  if (side == 0) {
    const f32x4_t v = none ? f32x4_t{} : acc * inv;
    *reinterpret_cast<u32x2_t*>(a.O + static_cast<int64_t>(row) * D + col) = __builtin_bit_cast(u32x2_t, __builtin_convertvector(v, typename T::x4));
  }
  if (lane == 0 && a.LSE)
    a.LSE[static_cast<int64_t>(h) * c.tokens + token] =
        none ? -__builtin_inff() : fmaf(log2f(l), kLn2, m * a.scoring.unit);
}

template <class T, int D>
hipError_t append(const AppendArgs& a, hipStream_t s) {
  hipLaunchKernelGGL((cache_append<T, D>), dim3(a.c.tokens), dim3(kThreads), 0, s, a);
  return hipGetLastError();
}

template <class T, int D>
hipError_t merge(const CacheAttnArgs& a, hipStream_t s) {
  const int64_t rows = static_cast<int64_t>(a.c.tokens) * a.c.H;
  hipLaunchKernelGGL((cache_merge<T, D>), dim3((rows + 3) / 4), dim3(kThreads), 0, s, a);
  return hipGetLastError();
}

template <class T, int D, bool kPlain>
hipError_t attend(const CacheAttnArgs& a, hipStream_t s) {
  hipLaunchKernelGGL((cache_attn<T, D, kPlain>), dim3(a.head_workers * a.c.Hkv), dim3(kThreads), 0, s, a);
  hipError_t e = hipGetLastError();
  return e != hipSuccess ? e : merge<T, D>(a, s);
}

template <class T, int D>
hipError_t attend(const CacheAttnArgs& a, hipStream_t s) {
  return a.scoring.plain() ? attend<T, D, true>(a, s) : attend<T, D, false>(a, s);
}

}  // namespace

hipError_t launch_cache_append(const AppendArgs& a, bool f16, int head_dim, hipStream_t s) {
  if (head_dim == 128) return f16 ? append<F16, 128>(a, s) : append<Bf16, 128>(a, s);
  return f16 ? append<F16, 64>(a, s) : append<Bf16, 64>(a, s);
}

hipError_t launch_cache_attn(const CacheAttnArgs& a, bool f16, int head_dim, hipStream_t s) {
  if (head_dim == 128) return f16 ? attend<F16, 128>(a, s) : attend<Bf16, 128>(a, s);
  return f16 ? attend<F16, 64>(a, s) : attend<Bf16, 64>(a, s);
}

hipError_t launch_cache_merge(const CacheAttnArgs& a, bool f16, int head_dim, hipStream_t s) {
  if (head_dim == 128) return f16 ? merge<F16, 128>(a, s) : merge<Bf16, 128>(a, s);
  return f16 ? merge<F16, 64>(a, s) : merge<Bf16, 64>(a, s);
}

}  // namespace csg
