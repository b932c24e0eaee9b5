// The work of attention over a paged cache, whatever its pages hold: entries, tasks and runs, and the
// rows of a part.
#pragma once

#include <hip/hip_runtime.h>

#include "attn_tile.hpp"
#include "cache_attn.hpp"

namespace csg {
namespace cache {

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

struct Entry {
  int token0, rows;    // first token, (token, head) rows
  int b0, b1;          // its sequences; the first one's pages are read
  int lo, end;         // keys
  int own;             // the keys of one sequence, up to its end
  int group;           // its group, -1: none
  int block0, blocks;  // blocks of keys that hold them
  __device__ __forceinline__ void count_blocks() {
    block0 = lo / kCacheBlock;
    blocks = end > lo && rows > 0 ? (end + kCacheBlock - 1) / kCacheBlock - block0 : 0;
  }
  __device__ __forceinline__ int tiles() const { return (rows + kCacheTileRows - 1) / kCacheTileRows; }
  __device__ __forceinline__ bool wide() const { return rows > kCacheTileRows; }
  __device__ __forceinline__ bool small() const { return rows <= kCacheAloneRows; }
  __device__ __forceinline__ int tasks() const { return wide() ? (rows + kCacheWideRows - 1) / kCacheWideRows : 1; }
  // a task's units of work: its blocks, behind what beginning and ending it costs
  __device__ __forceinline__ int span(int cost) const { return blocks > 0 ? cost + blocks : 0; }
};

// What is kept of an entry in LDS.
struct KeptEntry {
  int token0, rows, b0, b1, lo, end;
};

// The groups of a call where they are given.
struct GlobalGroups {
  const CacheAttnArgs& a;
  __device__ __forceinline__ int first(int g) const { return clamped(a.group_ptr[g], 0, a.c.batch); }
  __device__ __forceinline__ int prefix(int g) const {  // no longer than the first sequence
    const int b = first(g);
    return b < a.c.batch ? clamped(a.prefix[g], 0, length_of(a.c, b)) : 0;
  }
};
// The same, copied into LDS.
struct LocalGroups {
  const int32_t* firsts;
  const int32_t* prefixes;
  __device__ __forceinline__ int first(int g) const { return firsts[g]; }
  __device__ __forceinline__ int prefix(int g) const { return prefixes[g]; }
};

// The group of sequence b, -1 if it has none.
template <class Groups>
__device__ __forceinline__ int group_of(const CacheAttnArgs& a, const Groups& groups, int b) {
  if (a.n_groups == 0 || b < groups.first(0) || b >= groups.first(a.n_groups)) return -1;
  int lo = 0, n = a.n_groups;
  while (n > 1) {
    const int half = n / 2;
    if (groups.first(lo + half) <= b) {
      lo += half;
      n -= half;
    } else {
      n = half;
    }
  }
  return lo;
}

template <class Groups>
__device__ __forceinline__ Entry entry_of(const CacheAttnArgs& a, const Groups& groups, int e) {
  const CacheArgs& c = a.c;
  Entry x;
  x.group = -1;
  if (e < a.n_groups) {
    x.own = 0;
    x.b0 = groups.first(e);
    x.b1 = max(x.b0, groups.first(e + 1));
    x.lo = 0;
    x.end = x.b1 > x.b0 ? groups.prefix(e) : 0;
  } else {
    x.own = 1;
    x.b0 = e - a.n_groups;
    x.b1 = x.b0 + 1;
    x.end = length_of(c, x.b0);
    x.group = group_of(a, groups, x.b0);
    x.lo = x.group < 0 ? 0 : min(groups.prefix(x.group), x.end);
  }
  x.token0 = first_token(c, x.b0);
  x.rows = x.b1 > x.b0 ? max(0, first_token(c, x.b1) - x.token0) * (c.H / c.Hkv) : 0;
  x.count_blocks();
  return x;
}

// The plan of a call in the workspace, for cache_merge: an entry's units and tiles before it (of its kind, where
// small and other tasks have runs of their own; the tiles with where the kind's places begin),
// its own blocks, rows and first token; of a sequence, its group's entry too (-1: none).
struct PlanEntry {
  int32_t before, tiles, blocks, rows, token0, group, unused[2];
};
struct Plan {
  int32_t tiles;    // tiles of one key/value head
  // of entries of up to kCacheAloneRows rows, and of more:
  int32_t run[2];    // units of a run
  int32_t shift[2];  // places from a tile's part in one run to that in the next, a task's tiles at most: 1 << shift
  int32_t cost[2];   // units that beginning and ending a task costs
  int32_t unused;
};
__device__ __forceinline__ Plan* plan_in(unsigned char* ws) { return reinterpret_cast<Plan*>(ws); }
__device__ __forceinline__ PlanEntry* entries_in(unsigned char* ws) { return reinterpret_cast<PlanEntry*>(ws + sizeof(Plan)); }
static_assert(sizeof(Plan) + kMaxCacheEntries * sizeof(PlanEntry) <= cache_plan_bytes(), "the plan fits");

// A workgroup's part of a task, and this lane's row of it.
struct Part {
  int kvh, tile;       // key/value head; the wave's tile of 32 rows in the entry
  int key0, end;       // keys of the part (those below the entry's lo are masked)
  int lo;
  const int32_t* table;
  bool ok;             // the lane has a row
  int token, h, pos;   // its token, head, position
  int hi;              // it sees keys below this (lanes without a row, whose queries are 0: all)
  int all_hi;          // every row of the wave sees keys below this
};

// `local`: the sequences' entries, where they are in LDS.
__device__ __forceinline__ void locate_row(const CacheAttnArgs& a, const Entry& x, const KeptEntry* local, int l32, Part& p) {
  const CacheArgs& c = a.c;
  const int G = c.H / c.Hkv;
  const int r = p.tile * kCacheTileRows + l32;
  p.ok = r < x.rows;
  p.token = x.token0 + (p.ok ? r / G : 0);
  p.h = p.kvh * G + (p.ok ? r % G : 0);
  if (x.own) {
    p.pos = x.end - (x.token0 + x.rows / G - p.token);
  } else {
    int b = x.b0;
    for (int n = x.b1 - x.b0; n > 1;) {  // the last of the group's sequences that starts by then
      const int half = n / 2;
      const bool up = (local ? local[b + half].token0 : first_token(c, b + half)) <= p.token;
      b = up ? b + half : b;
      n = up ? n - half : half;
    }
    if (local)
      p.pos = local[b].end - (local[b].token0 + local[b].rows / G - p.token);
    else
      p.pos = length_of(c, b) - (first_token(c, b + 1) - p.token);
  }
  p.hi = p.ok ? min(p.pos + 1, p.end) : p.end;
  int all_hi = p.hi;
#pragma unroll
  for (int d = 1; d < 32; d *= 2) all_hi = min(all_hi, __shfl_xor(all_hi, d));
  p.all_hi = __builtin_amdgcn_readfirstlane(all_hi);
}

template <class T, int D>
__device__ __forceinline__ void load_queries(const CacheAttnArgs& a, const Part& p, int hlf, typename T::x8 (&qf)[D / 16]) {
  const uint16_t* q = a.c.Q + p.token * a.c.q_stride + p.h * D + 8 * hlf;
#pragma unroll
  for (int s = 0; s < D / 16; ++s) {
    const u32x4_t raw = p.ok ? *reinterpret_cast<const u32x4_t*>(q + 16 * s) : u32x4_t{0u, 0u, 0u, 0u};
    qf[s] = __builtin_bit_cast(typename T::x8, raw);
  }
}

// The page of keys key .. key + 15, -1 if it has none to read.
__device__ __forceinline__ int page_of(const CacheArgs& c, const Part& p, int key) {
  if (key >= p.end || key + 16 <= p.lo) return -1;
  const int page = p.table[key >> c.page_shift];
  if (page >= 0 && page < c.n_pages) return page;
  tell(c, kCacheBadPage);
  return -1;
}

// Scores of a block of 32 N keys from its products: cap, bias, mask.
template <int N, bool kPlain>
__device__ __forceinline__ void finish_scores(const CacheAttnArgs& a, const Part& p, float slope, int key0, int hlf, f32x16_t (&sc)[N]) {
  if constexpr (!kPlain) {
    cap_scores<N>(a.scoring, sc);
    bias_scores<N, -1>(a.scoring, slope, p.pos - key0, hlf, sc);
  }
  if (key0 + 32 * N > p.all_hi || key0 < p.lo) {
#pragma unroll
    for (int n = 0; n < N; ++n)
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const int key = key0 + 32 * n + result_row(i, hlf);
        if (key >= p.hi || key < p.lo) sc[n][i] = -__builtin_inff();
      }
  }
}

// Memory of a part's results in place `place`, null if there is none.
template <int D>
__device__ __forceinline__ float* part_at(const CacheAttnArgs& a, int64_t place) {
  return place < a.max_parts ? reinterpret_cast<float*>(a.ws + cache_plan_bytes() + place * cache_part_bytes(D)) : nullptr;
}

// Tasks of a head that are enough for waves with runs of their own.
__host__ __device__ __forceinline__ bool enough_to_run_alone(int tasks, int workers) { return 2 * tasks >= workers; }

// A workgroup's run: its parts, one after the other, through do_part, which all of its threads call with the
// entry, the sequences' entries (locate_row), the part, whose tile is its task's first, that tile's place, and whether the
// task is wide. With kAloneCost > 0 and many tasks of small entries, of up to kAloneBlocks blocks on average, every wave has a run
// of those, and does its parts alone (the last argument): a task then costs kAloneCost units. With other tasks beside
// them the workgroups are divided, another task's unit counting kOtherUnits of a wave's (0: that is not done).
// `stage`: LDS that the parts use (and the groups, before them).
template <int kAloneCost, int kAloneBlocks, int kOtherUnits, class DoPart>
__device__ __forceinline__ void cache_run(const CacheAttnArgs& a, unsigned char* stage, DoPart do_part) {
  __shared__ uint32_t s_wave_units[4], s_wave_tiles[4], s_wave_blocks[4], s_wave_tasks[4];
  __shared__ int s_entry[4], s_first[4], s_tiles[4];
  __shared__ KeptEntry s_entries[kThreads];
  const CacheArgs& c = a.c;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int n_entries = a.n_groups + c.batch;
  // a die runs every 8th workgroup: with the head fastest, it has few heads, and runs that follow
  // each other, whose tasks may read the same keys
  const int kvh = blockIdx.x % c.Hkv;
  int w = blockIdx.x / c.Hkv;
  if (a.head_workers % a.dies == 0) w = w % a.dies * (a.head_workers / a.dies) + w / a.dies;

  int32_t* firsts = reinterpret_cast<int32_t*>(stage);
  const LocalGroups local{firsts, firsts + a.n_groups + 1};
  if (a.n_groups > 0) {
    const GlobalGroups global{a};
    for (int g = tid; g <= a.n_groups; g += kThreads) {
      firsts[g] = global.first(g);
      if (g < a.n_groups) firsts[a.n_groups + 1 + g] = global.prefix(g);
    }
    __syncthreads();
  }
  // Each thread counts some entries; units and tiles before each of them by a scan. Where a thread
  // has one entry, everyone finds it in LDS.
  const int per = (n_entries + kThreads - 1) / kThreads;
  // (With kAloneCost, small entries are counted by themselves: blocks, and tasks and tiles in the halves of a word.)
  uint32_t units = 0, tiles = 0, blocks = 0, tasks = 0;
  Entry mine{};
  for (int i = 0; i < per; ++i) {
    const int e = tid * per + i;
    if (e >= n_entries) break;
    const Entry x = entry_of(a, local, e);
    mine = x;
    if (per == 1) s_entries[e] = {x.token0, x.rows, x.b0, x.b1, x.lo, x.end};
    if (kAloneCost > 0 && x.small()) {
      blocks += x.blocks;
      tasks += (x.blocks > 0 ? 1 : 0) + (x.tiles() << 16);
    } else {
      units += x.tasks() * x.span(a.task_cost);
      tiles += x.tiles();
    }
  }
  uint32_t own_units = units, own_blocks = blocks, own_tasks = tasks;
  const uint32_t own_tiles = tiles;
#pragma unroll
  for (int d = 1; d < 64; d *= 2) {
    const uint32_t uu = __shfl_up(units, d), ut = __shfl_up(tiles, d);
    const uint32_t ub = kAloneCost > 0 ? __shfl_up(blocks, d) : 0, uk = kAloneCost > 0 ? __shfl_up(tasks, d) : 0;
    if (lane >= d) {
      units += uu;
      tiles += ut;
      blocks += ub;
      tasks += uk;
    }
  }
  if (lane == 63) {
    s_wave_units[wave] = units;
    s_wave_tiles[wave] = tiles;
    if constexpr (kAloneCost > 0) {
      s_wave_blocks[wave] = blocks;
      s_wave_tasks[wave] = tasks;
    }
  }
  __syncthreads();
  units -= own_units;
  tiles -= own_tiles;
  blocks -= own_blocks;
  tasks -= own_tasks;
  for (int i = 0; i < wave; ++i) {
    units += s_wave_units[i];
    tiles += s_wave_tiles[i];
    if constexpr (kAloneCost > 0) {
      blocks += s_wave_blocks[i];
      tasks += s_wave_tasks[i];
    }
  }
  auto sum = [](const uint32_t (&of)[4]) { return __builtin_amdgcn_readfirstlane(of[0] + of[1] + of[2] + of[3]); };
  int all_tiles = sum(s_wave_tiles), all_units = sum(s_wave_units);
  // the first `alone` workgroups have runs of small tasks for each wave, the others those of all other tasks
  int alone = 0, all_small = 0, small_tiles = 0;
  if constexpr (kAloneCost > 0) {
    const int all_blocks = sum(s_wave_blocks), all_tasks = sum(s_wave_tasks);
    const int n_tasks = all_tasks & 0xffff;
    small_tiles = all_tasks >> 16;
    const bool pure = kOtherUnits > 0 ? all_units == 0 : all_tiles == 0;
    all_tiles += small_tiles;
    if (enough_to_run_alone(n_tasks, a.head_workers) && all_blocks <= kAloneBlocks * n_tasks &&
        (pure || (kOtherUnits > 0 && a.head_workers > 1))) {
      all_small = all_blocks + kAloneCost * n_tasks;
      alone = a.head_workers;
      if (!pure) {
        const float part = all_small * __builtin_amdgcn_rcpf(static_cast<float>(all_small) + kOtherUnits * static_cast<float>(all_units));
        alone = __builtin_amdgcn_readfirstlane(clamped(static_cast<int>(part * a.head_workers + 0.5f), 1, a.head_workers - 1));
      }
    } else {
      all_units += all_blocks + a.task_cost * n_tasks;
      units += blocks + a.task_cost * (tasks & 0xffff);
      own_units += own_blocks + a.task_cost * (own_tasks & 0xffff);
      tiles += tasks >> 16;
      small_tiles = 0;
    }
  }
  // Bounds that do not ascend may name rows several times, and with them more units than 32 bits count: then
  // there is nothing to do. (As many tiles as the host has reckoned with have no more units than it has.)
  const bool fits = static_cast<uint32_t>(all_tiles) <= a.max_tiles;
  const int others = a.head_workers - alone;
  const bool small = kOtherUnits > 0 ? w < alone : alone > 0;  // (the workgroup's kind of tasks)
  auto run_of = [&](bool is_small) {
    const int all = is_small ? all_small : all_units, runs = is_small ? 4 * alone : others;
    const int units = max(is_small ? kCacheMinRun : a.min_run, (all + runs - 1) / max(1, runs));
    return is_small || kOtherUnits == 0 ? units : units + (units & 1);  // (a wide block is two)
  };
  const int all = fits ? (small ? all_small : all_units) : 0;
  const int run = run_of(small);
  const int first_begin = (small ? 4 * w : w - alone) * run;  // the workgroup's runs: one, or one a wave
  const int other_places = 4 * alone + small_tiles;
  int before = units, own = own_units;
  if constexpr (kAloneCost > 0) {
    if (small) {
      before = blocks + kAloneCost * (tasks & 0xffff);
      own = own_blocks + kAloneCost * (own_tasks & 0xffff);
    }
  }
  // for cache_merge, and the entry where the run begins
  if (blockIdx.x == 0 || (before < first_begin + (small ? 4 : 1) * run && first_begin < before + own)) {
    int units_before = units, tiles_before = tiles;
    int small_before = blocks + kAloneCost * (tasks & 0xffff), small_tiles_before = tasks >> 16;
    for (int i = 0; i < per; ++i) {
      const int e = tid * per + i;
      if (e >= n_entries) break;
      const Entry x = per == 1 ? mine : entry_of(a, local, e);
      const bool is_small = kOtherUnits > 0 ? alone > 0 && x.small() : small;
      const int n = x.tasks() * x.span(is_small ? kAloneCost : a.task_cost);
      const int x_before = is_small ? small_before : units_before, x_tiles = is_small ? small_tiles_before : tiles_before;
      if (is_small == small) {
        for (int k = 0; k < (small ? 4 : 1); ++k) {
          const int begin = first_begin + k * run;
          if (x_before <= begin && begin < x_before + n) {
            s_entry[k] = e;
            s_first[k] = begin - x_before;
            s_tiles[k] = x_tiles;
          }
        }
      }
      if (blockIdx.x == 0) {
        entries_in(a.ws)[e] = {x_before, x_tiles + (is_small ? 0 : other_places), fits ? x.blocks : 0, x.rows, x.token0, x.group, {0, 0}};
        if (x.own && (x.end != c.lens[x.b0] || x.rows / (c.H / c.Hkv) > x.end)) tell(c, kCacheBadLength);
      }
      if (is_small) {
        small_before += n;
        small_tiles_before += x.tiles();
      } else {
        units_before += n;
        tiles_before += x.tiles();
      }
    }
    if (blockIdx.x == 0 && tid == 0) {
      const int small_run = kOtherUnits > 0 && alone ? run_of(true) : run, other_run = kOtherUnits > 0 ? run_of(false) : run;
      *plan_in(a.ws) = {all_tiles, {small_run, other_run}, {alone ? 0 : 2, 2},
                        {alone ? kAloneCost : a.task_cost, a.task_cost}, 0};
      if (!fits) tell(c, kCacheBadLength);
    }
  }
  if (first_begin >= all) return;
  __syncthreads();
  const int mine_k = small ? wave : 0, begin = first_begin + mine_k * run;
  int left = min(run, all - begin);  // (not positive: the wave has no run)
  int e = __builtin_amdgcn_readfirstlane(s_entry[mine_k]), in_entry = __builtin_amdgcn_readfirstlane(s_first[mine_k]);
  int tiles_before = __builtin_amdgcn_readfirstlane(s_tiles[mine_k]);
  const int cost = small ? kAloneCost : a.task_cost;
  const int64_t places = static_cast<int64_t>(kvh) * (all_tiles + 4 * a.head_workers) + 4 * w + mine_k + (small ? 0 : small_tiles);
  const KeptEntry* sequences = per == 1 ? s_entries + a.n_groups : nullptr;
  while (left > 0) {
    Entry x;
    if (per == 1) {
      // (the same in every lane)
      x.token0 = __builtin_amdgcn_readfirstlane(s_entries[e].token0);
      x.rows = __builtin_amdgcn_readfirstlane(s_entries[e].rows);
      x.b0 = __builtin_amdgcn_readfirstlane(s_entries[e].b0);
      x.b1 = __builtin_amdgcn_readfirstlane(s_entries[e].b1);
      x.lo = __builtin_amdgcn_readfirstlane(s_entries[e].lo);
      x.end = __builtin_amdgcn_readfirstlane(s_entries[e].end);
      x.own = e >= a.n_groups;
      x.count_blocks();
    } else {
      x = entry_of(a, GlobalGroups{a}, e);
    }
    const bool other = kOtherUnits > 0 && alone > 0 && x.small() != small;  // (it is of the other workgroups')
    const int n = other ? 0 : x.tasks() * x.span(cost);
    if (in_entry < n) {
      Part p;
      p.kvh = kvh;
      const bool wide = x.wide();
      const int task = wide ? __builtin_amdgcn_readfirstlane(in_entry / x.span(cost)) : 0;
      const int from = in_entry - task * x.span(cost), take = min(x.span(cost) - from, left);
      const int first = max(0, from - cost), count = from + take - cost - first;
      left -= take;
      in_entry += take;
      if (count <= 0) continue;
      p.table = c.table + static_cast<int64_t>(x.b0) * c.max_pages;
      p.lo = x.lo;
      p.key0 = (x.block0 + first) * kCacheBlock;
      p.end = min(x.end, p.key0 + count * kCacheBlock);
      p.tile = wide ? 4 * task : 0;
      do_part(x, sequences, p, places + tiles_before + p.tile, wide, small);
    } else {
      in_entry = 0;
      if (!other) tiles_before += x.tiles();
      ++e;
    }
  }
}

}  // namespace cache
}  // namespace csg
