// A paged key/value cache for gfx950 (CDNA4): new tokens go in, attention reads it.
//
// Sequence b's keys and values are tokens 0 .. lens[b] - 1; token x lies in page
// table[b][x / page size] at row x % page size, all rows of a head of a page behind each
// other. A call's new tokens q_ptr[b] .. q_ptr[b+1] - 1 are the last of sequence b.
#include <hip/hip_runtime.h>

#include "attn_tile.hpp"
#include "cache_attn.hpp"

namespace csg {
namespace {

using namespace tile;

constexpr int kThreads = 256;

__device__ __forceinline__ void tell(const CacheArgs& c, int bit) {
  if (c.status) atomicOr(c.status, bit);
}

// Tokens of sequence b in the cache, as far as its row of the page table goes.
__device__ __forceinline__ int length_of(const CacheArgs& c, int b) {
  const int64_t room = static_cast<int64_t>(c.max_pages) << c.page_shift;
  const int n = c.lens[b];
  return n < 0 ? 0 : n > room ? static_cast<int>(room) : n;
}
__device__ __forceinline__ int first_token(const CacheArgs& c, int b) { return clamped(c.q_ptr[b], 0, c.tokens); }

// ---- new tokens into the cache --------------------------------------------------------------
// A workgroup per token. Pair i of a head (elements i and half + i, or 2 i and 2 i + 1) turns by
// the angle position * inv_freq[i]. The angle is reduced to a fraction of a turn in 64 bits: at
// position 1e6 a 32-bit product is off by 0.06. A thread keeps eight pairs' sines and cosines
// and goes through the heads, 16 elements of each: two loads and two stores of 16 bytes.
template <class T, int D>
__global__ __launch_bounds__(kThreads) void cache_append(AppendArgs a) {
  constexpr int kCols = D / 16, kHeads = kThreads / kCols;
  const CacheArgs& c = a.c;
  const int t = blockIdx.x;
  if (t >= first_token(c, c.batch)) return;
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
// a head of the key/value head's group, tokens first; 32 rows make a tile; an entry, a tile and
// a key/value head make a task. A task is its blocks of 32 keys, and all tasks' blocks stand in
// one row (by key/value head, entry, tile, block) that is cut into equal runs, one a workgroup:
// every workgroup reads the same number of keys, whatever the lengths are. What a workgroup has
// of a task is a part: its weights' sums and products against its own reference, which
// cache_merge joins. Task t and workgroup w meet in at most one part, and parts in their order
// never go back in t or w: t + w numbers them.
struct Entry {
  int token0, rows;    // first token, (token, head) rows
  int b0, b1;          // its sequences; the first one's pages are read
  int lo, end;         // keys
  int block0, blocks;  // blocks of keys that hold them
  __device__ __forceinline__ int tiles() const { return (rows + kCacheTileRows - 1) / kCacheTileRows; }
};

// The group of sequence b, -1 if it has none.
__device__ __forceinline__ int group_of(const CacheAttnArgs& a, int b) {
  if (a.n_groups == 0 || b < a.group_ptr[0] || b >= a.group_ptr[a.n_groups]) return -1;
  int lo = 0, n = a.n_groups;
  while (n > 1) {
    const int half = n / 2;
    if (a.group_ptr[lo + half] <= b) {
      lo += half;
      n -= half;
    } else {
      n = half;
    }
  }
  return lo;
}

__device__ __forceinline__ int prefix_of(const CacheAttnArgs& a, int g) {
  const int b = clamped(a.group_ptr[g], 0, a.c.batch);
  return b < a.c.batch ? clamped(a.prefix[g], 0, length_of(a.c, b)) : 0;
}

__device__ __forceinline__ Entry entry_of(const CacheAttnArgs& a, int e) {
  const CacheArgs& c = a.c;
  Entry x;
  if (e < a.n_groups) {
    x.b0 = clamped(a.group_ptr[e], 0, c.batch);
    x.b1 = clamped(a.group_ptr[e + 1], x.b0, c.batch);
    x.lo = 0;
    x.end = x.b1 > x.b0 ? prefix_of(a, e) : 0;
  } else {
    x.b0 = e - a.n_groups;
    x.b1 = x.b0 + 1;
    x.end = length_of(c, x.b0);
    const int g = group_of(a, x.b0);
    x.lo = g < 0 ? 0 : min(prefix_of(a, g), x.end);
  }
  x.token0 = first_token(c, x.b0);
  x.rows = x.b1 > x.b0 ? max(0, first_token(c, x.b1) - x.token0) * (c.H / c.Hkv) : 0;
  x.block0 = x.lo / kCacheBlock;
  x.blocks = x.end > x.lo && x.rows > 0 ? (x.end + kCacheBlock - 1) / kCacheBlock - x.block0 : 0;
  return x;
}

// The plan of a call in the workspace: blocks of one key/value head, tasks of one, blocks a
// workgroup takes; then blocks and tasks before each entry.
struct Plan {
  int64_t* blocks;  // [0]: all, [1]: a run; [2 + e]
  int32_t* tasks;   // [0]: all; [1 + e]
};
__device__ __forceinline__ Plan plan_in(unsigned char* ws) {
  Plan p;
  p.blocks = reinterpret_cast<int64_t*>(ws);
  p.tasks = reinterpret_cast<int32_t*>(ws + 16 + 8 * kMaxCacheEntries);
  return p;
}

// What sums against reference m count against reference top; nothing if they saw no key.
__device__ __forceinline__ float factor(float m, float top, float c) {
  return m == -__builtin_inff() ? 0.0f : __builtin_amdgcn_exp2f((m - top) * c);
}

// A wave reads its own blocks of keys: into its own part of LDS, a block ahead, so that it
// waits for no other wave; their results meet at the part's end.
template <class T, int D, bool kPlain>
__global__ __launch_bounds__(kThreads, 1) void cache_attn(CacheAttnArgs a) {
  constexpr int kRowBytes = 2 * D;
  constexpr int kTile = kCacheBlock * kRowBytes;     // keys or values of a block
  constexpr int kStage = 2 * kTile;
  constexpr int kLoads = kCacheBlock / kLoadRows<D>; // loads of a tile
  constexpr int kHalfLoads = kLoads / 2;             // of 16 rows, which lie in one page
  __shared__ __attribute__((aligned(1024))) unsigned char stage[4 * 2 * kStage];
  __shared__ int64_t s_blocks[kMaxCacheEntries + 1];
  __shared__ int32_t s_tasks[kMaxCacheEntries + 1];
  __shared__ int64_t s_wave_blocks[4];
  __shared__ int32_t s_wave_tasks[4];
  __shared__ float s_ref[4][32], s_sum[4][32];
  static_assert(4 * kTile <= sizeof(stage) / 2, "the waves' results fit the stages");

  const CacheArgs& c = a.c;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int l32 = lane & 31, hlf = lane >> 5;
  const int G = c.H / c.Hkv;
  const int n_entries = a.n_groups + c.batch;

  // blocks and tasks before each entry
  {
    const int per = (n_entries + kThreads - 1) / kThreads;
    int64_t blocks = 0;
    int32_t tasks = 0;
    for (int i = 0; i < per; ++i) {
      const int e = tid * per + i;
      if (e >= n_entries) break;
      const Entry x = entry_of(a, e);
      s_blocks[e] = blocks;  // before the thread's own
      s_tasks[e] = tasks;
      blocks += static_cast<int64_t>(x.tiles()) * x.blocks;
      tasks += x.tiles();
      if (blockIdx.x == 0 && e >= a.n_groups && length_of(c, x.b0) != c.lens[x.b0]) tell(c, kCacheBadLength);
    }
    const int64_t own_blocks = blocks;
    const int32_t own_tasks = tasks;
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
      const int64_t ub = __shfl_up(blocks, d);
      const int32_t ut = __shfl_up(tasks, d);
      if (lane >= d) {
        blocks += ub;
        tasks += ut;
      }
    }
    if (lane == 63) {
      s_wave_blocks[wave] = blocks;
      s_wave_tasks[wave] = tasks;
    }
    __syncthreads();
    blocks -= own_blocks;
    tasks -= own_tasks;
    for (int w = 0; w < wave; ++w) {
      blocks += s_wave_blocks[w];
      tasks += s_wave_tasks[w];
    }
    for (int i = 0; i < per; ++i) {
      const int e = tid * per + i;
      if (e >= n_entries) break;
      s_blocks[e] += blocks;
      s_tasks[e] += tasks;
    }
  }
  const int64_t all = s_wave_blocks[0] + s_wave_blocks[1] + s_wave_blocks[2] + s_wave_blocks[3];
  const int32_t all_tasks = s_wave_tasks[0] + s_wave_tasks[1] + s_wave_tasks[2] + s_wave_tasks[3];
  const int64_t total = all * c.Hkv;
  const int64_t run = max(int64_t{1}, (total + a.workers - 1) / a.workers);
  __syncthreads();
  if (blockIdx.x == 0) {  // for cache_merge
    const Plan p = plan_in(a.ws);
    for (int e = tid; e < n_entries; e += kThreads) {
      p.blocks[2 + e] = s_blocks[e];
      p.tasks[1 + e] = s_tasks[e];
    }
    if (tid == 0) {
      p.blocks[0] = all;
      p.blocks[1] = run;
      p.tasks[0] = all_tasks;
    }
  }

  // a die runs every 8th workgroup: its runs follow each other, so that the tiles of a group,
  // which read the same keys, share its cache
  const int w = a.workers % 8 == 0 ? blockIdx.x % 8 * (a.workers / 8) + blockIdx.x / 8 : blockIdx.x;
  const LoadLane<D> ll(lane);
  const Frags<D> fr(lane);
  unsigned char* mine = stage + wave * 2 * kStage;
  const uint32_t mine_addr = lds_address(mine);
  const float cexp = kPlain ? a.scoring.scale * kLog2e : kLog2e;
  const int page_mask = (1 << c.page_shift) - 1;

  int64_t at = w * run;
  const int64_t stop = min(total, at + run);
  while (at < stop) {
    const int kvh = __builtin_amdgcn_readfirstlane(static_cast<int>(at / all));
    const int64_t in_head = at - kvh * all;
    const int e = last_below(n_entries, [&](int i) { return s_blocks[i] <= in_head; });
    const Entry x = entry_of(a, e);
    const int64_t in_entry = in_head - s_blocks[e];
    const int tile = __builtin_amdgcn_readfirstlane(static_cast<int>(in_entry / x.blocks));
    const int first = __builtin_amdgcn_readfirstlane(static_cast<int>(in_entry - static_cast<int64_t>(tile) * x.blocks));
    const int count = __builtin_amdgcn_readfirstlane(static_cast<int>(min<int64_t>(x.blocks - first, stop - at)));
    const int64_t part = static_cast<int64_t>(kvh) * all_tasks + s_tasks[e] + tile + w;

    // the lane's row: its token, the keys that it sees
    const int r = tile * kCacheTileRows + l32;
    const bool ok = r < x.rows;
    const int token = x.token0 + (ok ? r / G : 0);
    const int h = kvh * G + (ok ? r % G : 0);
    int b = x.b0;
    for (int n = x.b1 - x.b0; n > 1;) {  // the last of the entry's sequences that starts by then
      const int half = n / 2;
      const bool up = c.q_ptr[b + half] <= token;
      b = up ? b + half : b;
      n = up ? n - half : half;
    }
    const int pos = length_of(c, b) - (first_token(c, b + 1) - token);
    const int hi = ok ? min(pos + 1, x.end) : x.end;  // (rows that are none: their queries are 0)
    const float slope = !kPlain && a.scoring.slopes ? a.scoring.slopes[h] : 0.0f;
    typename T::x8 qf[D / 16];
    {
      const uint16_t* q = c.Q + token * c.q_stride + h * D + 8 * hlf;
#pragma unroll
      for (int s = 0; s < D / 16; ++s) {
        const u32x4_t raw = ok ? *reinterpret_cast<const u32x4_t*>(q + 16 * s) : u32x4_t{0u, 0u, 0u, 0u};
        qf[s] = __builtin_bit_cast(typename T::x8, raw);
      }
    }
    // every row sees keys below this
    int all_hi = hi;
#pragma unroll
    for (int d = 1; d < 32; d *= 2) all_hi = min(all_hi, __shfl_xor(all_hi, d));
    all_hi = __builtin_amdgcn_readfirstlane(all_hi);

    f32x16_t acc[D / 32];
#pragma unroll
    for (int db = 0; db < D / 32; ++db) acc[db] = f32x16_t{};
    RowSoftmax sm;

    // The wave's blocks are first + wave, first + wave + 4, ...; lane n holds the page of the
    // 16 keys n % 2 of its block n / 2 (32 blocks at a time): a table entry is there long
    // before its block is asked for.
    const int mine_n = count > wave ? (count - wave + 3) / 4 : 0;
    const int32_t* table = c.table + static_cast<int64_t>(x.b0) * c.max_pages;
    int pages = -1;
    auto fetch_pages = [&](int n) {
      const int key = (x.block0 + first + wave + 4 * (n + (lane >> 1))) * kCacheBlock + 16 * (lane & 1);
      pages = -1;
      if (key < x.end) {
        pages = table[key >> c.page_shift];
        if (pages < 0 || pages >= c.n_pages) {
          tell(c, kCacheBadPage);
          pages = -1;
        }
      }
    };
    auto load = [&](int n) {
      const int key0 = (x.block0 + first + wave + 4 * n) * kCacheBlock;
      const uint32_t lds = mine_addr + (n & 1) * kStage;
#pragma unroll
      for (int half = 0; half < 2; ++half) {
        const int page = __builtin_amdgcn_readlane(pages, 2 * (n & 31) + half);
        const int key = key0 + 16 * half;
        const int rows = page < 0 ? 0 : clamped(x.end - key, 0, 16);  // what is behind reads zero
        const int64_t off = ((static_cast<int64_t>(max(page, 0)) * c.Hkv + kvh) << c.page_shift) + (key & page_mask);
        const __amdgpu_buffer_rsrc_t rk = make_rsrc(c.k_pages + off * D, rows * kRowBytes);
        const __amdgpu_buffer_rsrc_t rv = make_rsrc(c.v_pages + off * D, rows * kRowBytes);
#pragma unroll
        for (int i = 0; i < kHalfLoads; ++i) {
          load_to_lds(rk, lds + 1024u * (half * kHalfLoads + i), ll.offset(i, kRowBytes));
          load_to_lds(rv, lds + kTile + 1024u * (half * kHalfLoads + i), ll.offset(i, kRowBytes));
        }
      }
    };
    if (mine_n > 0) {
      fetch_pages(0);
      load(0);
    }
    for (int n = 0; n < mine_n; ++n) {
      if (n + 1 < mine_n) {
        if (((n + 1) & 31) == 0) fetch_pages(n + 1);
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // block n - 1 has been read from LDS
        load(n + 1);
        wait_vm<2 * kLoads>();
      } else {
        wait_vm<0>();
      }
      const unsigned char* kt = mine + (n & 1) * kStage;
      const lds_u8_t* vt = (const lds_u8_t*)(kt + kTile);
      const int key0 = (x.block0 + first + wave + 4 * n) * kCacheBlock;
      f32x16_t sc[1] = {f32x16_t{}};
#pragma unroll
      for (int s = 0; s < D / 16; ++s) sc[0] = T::mfma(row_frag<T, D>(kt, fr, s, 0), qf[s], sc[0]);
      if constexpr (!kPlain) {
#pragma unroll
        for (int i = 0; i < 16; ++i)
          sc[0][i] = score_of(sc[0][i], a.scoring, slope, pos - (key0 + result_row(i, hlf))).value;
      }
      if (key0 + kCacheBlock > all_hi || key0 < x.lo) {
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          const int key = key0 + result_row(i, hlf);
          if (key >= hi || key < x.lo) sc[0][i] = -__builtin_inff();
        }
      }
      typename T::x8 pb[2];
      bool moved;
      const float alpha = sm.block<T, 1>(sc, cexp, pb, moved);
      if (moved) {
#pragma unroll
        for (int db = 0; db < D / 32; ++db) acc[db] *= alpha;
      }
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int db = 0; db < D / 32; ++db) acc[db] = T::mfma(col_frag<T, D>(vt, fr, db, 16 * t), pb[t], acc[db]);
    }

    // the waves' results against their common reference, in the order of the waves
    const float l = sum_halves(sm.l);
    if (hlf == 0) {
      s_ref[wave][l32] = sm.m;
      s_sum[wave][l32] = l;
    }
    __syncthreads();  // (also: every wave has read its stages)
    const float top = fmaxf(fmaxf(s_ref[0][l32], s_ref[1][l32]), fmaxf(s_ref[2][l32], s_ref[3][l32]));
    {
      const float f = factor(sm.m, top, cexp);
      float* out = reinterpret_cast<float*>(stage) + (wave * 32 + l32) * D;
#pragma unroll
      for (int db = 0; db < D / 32; ++db)
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          const f32x4_t v{acc[db][4 * q] * f, acc[db][4 * q + 1] * f, acc[db][4 * q + 2] * f, acc[db][4 * q + 3] * f};
          *reinterpret_cast<f32x4_t*>(out + 32 * db + 8 * q + 4 * hlf) = v;
        }
    }
    __syncthreads();
    if (part < a.max_parts) {
      float* out = reinterpret_cast<float*>(a.ws + cache_plan_bytes() + part * cache_part_bytes(D));
      const float* in = reinterpret_cast<const float*>(stage);
      for (int i = tid; i < 32 * D / 4; i += kThreads) {
        f32x4_t v = *reinterpret_cast<const f32x4_t*>(in + 4 * i);
#pragma unroll
        for (int k = 1; k < 4; ++k) v += *reinterpret_cast<const f32x4_t*>(in + k * 32 * D + 4 * i);
        *reinterpret_cast<f32x4_t*>(out + 4 * i) = v;
      }
      if (tid < 32) {
        float sum = 0.0f;
#pragma unroll
        for (int k = 0; k < 4; ++k) sum = fmaf(s_sum[k][l32], factor(s_ref[k][l32], top, cexp), sum);
        out[32 * D + l32] = top;
        out[32 * D + 32 + l32] = sum;
      }
    }
    __syncthreads();  // the stages are free again
    at += count;
  }
}

// One wave joins the parts of one row, in order.
template <class T, int D, bool kPlain>
__global__ __launch_bounds__(kThreads) void cache_merge(CacheAttnArgs a) {
  const CacheArgs& c = a.c;
  const int lane = threadIdx.x & 63;
  const int64_t row = static_cast<int64_t>(blockIdx.x) * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int token = static_cast<int>(row / c.H), h = static_cast<int>(row - static_cast<int64_t>(token) * c.H);
  if (token >= first_token(c, c.batch)) return;
  const int G = c.H / c.Hkv, kvh = h / G;
  const int b = last_below(c.batch, [&](int i) { return c.q_ptr[i] <= token; });
  const Plan p = plan_in(a.ws);
  const float cexp = kPlain ? a.scoring.scale * kLog2e : kLog2e;
  const int64_t all = p.blocks[0], run = p.blocks[1];
  const int32_t all_tasks = p.tasks[0];
  constexpr int kPer = D / 64;
  float acc[kPer] = {}, m = -__builtin_inff(), l = 0.0f;
  const int g = group_of(a, b);
  for (int i = 0; i < 2; ++i) {
    const int e = i == 0 ? g : a.n_groups + b;
    if (e < 0) continue;
    const Entry x = entry_of(a, e);
    if (x.blocks == 0 || token < x.token0) continue;
    const int r = (token - x.token0) * G + (h - kvh * G);
    const int tile = r / kCacheTileRows, in_tile = r % kCacheTileRows;
    if (tile >= x.tiles()) continue;
    const int64_t start = kvh * all + p.blocks[2 + e] + static_cast<int64_t>(tile) * x.blocks;
    const int64_t task = static_cast<int64_t>(kvh) * all_tasks + p.tasks[1 + e] + tile;
    for (int64_t w = start / run; w <= (start + x.blocks - 1) / run; ++w) {
      if (task + w >= a.max_parts) break;
      const float* in = reinterpret_cast<const float*>(a.ws + cache_plan_bytes() + (task + w) * cache_part_bytes(D));
      const float pm = in[32 * D + in_tile], pl = in[32 * D + 32 + in_tile];
      const float top = fmaxf(m, pm);
      const float f = factor(m, top, cexp), pf = factor(pm, top, cexp);
      l = fmaf(l, f, pl * pf);
#pragma unroll
      for (int k = 0; k < kPer; ++k) acc[k] = fmaf(acc[k], f, in[in_tile * D + lane * kPer + k] * pf);
      m = top;
    }
  }
  const float inv = l == 0.0f ? 0.0f : 1.0f / l;
  const bool none = l == 0.0f;  // nothing visible (its products may hold what masked keys have)
  const f32x4_t v{none ? 0.0f : acc[0] * inv, none ? 0.0f : acc[kPer - 1] * inv, 0.0f, 0.0f};
  const uint32_t bits = __builtin_bit_cast(u32x2_t, __builtin_convertvector(v, typename T::x4))[0];
  uint16_t* out = a.O + row * D + lane * kPer;
  if constexpr (kPer == 2)
    *reinterpret_cast<uint32_t*>(out) = bits;
  else
    *out = static_cast<uint16_t>(bits);
  if (lane == 0 && a.LSE)
    a.LSE[static_cast<int64_t>(h) * c.tokens + token] =
        none ? -__builtin_inff() : fmaf(log2f(l), kLn2, kPlain ? m * a.scoring.scale : m);
}

template <class T, int D>
hipError_t append(const AppendArgs& a, hipStream_t s) {
  hipLaunchKernelGGL((cache_append<T, D>), dim3(a.c.tokens), dim3(kThreads), 0, s, a);
  return hipGetLastError();
}

template <class T, int D, bool kPlain>
hipError_t attend(const CacheAttnArgs& a, hipStream_t s) {
  hipLaunchKernelGGL((cache_attn<T, D, kPlain>), dim3(a.workers), dim3(kThreads), 0, s, a);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  const int64_t rows = static_cast<int64_t>(a.c.tokens) * a.c.H;
  hipLaunchKernelGGL((cache_merge<T, D, kPlain>), dim3((rows + 3) / 4), dim3(kThreads), 0, s, a);
  return hipGetLastError();
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

}  // namespace csg
