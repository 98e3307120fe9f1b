// The plan of a window's attention: which requests share a prefix, the order
// of the rows, segments, tiles and the workgroups that take them.  Two
// launches: every page a context needs is checked by a workgroup per request,
// then one workgroup cuts the work (thousands of small steps with a barrier
// between; a step's layers share one plan).

#include <type_traits>

#include "ps_blocks.h"

namespace ps {

namespace {

constexpr int kThreads = 512;
static_assert(kThreads >= kMaxGroups, "a thread for each workgroup of a head");
static_assert(kTallWaves <= 2 * kWideWaves, "tall tiles: half as many workgroups");
constexpr int kWaves = kThreads / 64;

__global__ __launch_bounds__(256) void plan_check_kernel(AttendPlanDev p, BlockWin w, uint32_t* d_flags) {
  const int32_t r = blockIdx.x;
  const BlockReq q = block_req(w, r);
  int bad = !q.ok;
  if (q.ok) {
    const int32_t blocks = (int32_t)(((int64_t)q.ctx + w.bt - 1) / w.bt);
    for (int32_t b = threadIdx.x; b < blocks; b += 256) {
      const int64_t page = w.pages[b < q.pre_len ? q.pre_off + b : q.tail_off + (b - q.pre_len)];
      bad |= page < 0 || page >= w.n_pages;
    }
  }
  bad = __syncthreads_or(bad);
  if (threadIdx.x == 0) {
    p.flags[r] = bad ? PS_R_INVALID : 0u;
    if (d_flags) d_flags[r] = bad ? PS_R_INVALID : 0u;
  }
}

// Inclusive sums over the wave, by row shifts and row broadcasts.
__device__ inline int64_t wave_scan(int64_t x) {
  auto step = [&](auto shift, auto rows) {
    const uint32_t lo = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(uint32_t)x, shift(), rows(), 0xF, false);
    const uint32_t hi = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(x >> 32), shift(), rows(), 0xF, false);
    x += (int64_t)((uint64_t)hi << 32 | lo);
  };
  auto c = [](auto v) { return v; };
  step(c(std::integral_constant<int, 0x111>{}), c(std::integral_constant<int, 0xF>{}));
  step(c(std::integral_constant<int, 0x112>{}), c(std::integral_constant<int, 0xF>{}));
  step(c(std::integral_constant<int, 0x114>{}), c(std::integral_constant<int, 0xF>{}));
  step(c(std::integral_constant<int, 0x118>{}), c(std::integral_constant<int, 0xF>{}));
  step(c(std::integral_constant<int, 0x142>{}), c(std::integral_constant<int, 0xA>{}));  // lanes 15, 47 to the next row
  step(c(std::integral_constant<int, 0x143>{}), c(std::integral_constant<int, 0xC>{}));  // lane 31 to the upper half
  return x;
}

// Exclusive sums over the workgroup of each thread's value; *total to all.
__device__ inline int64_t block_scan(int64_t v, int64_t* total, int64_t* lds) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int64_t x = wave_scan(v);
  __syncthreads();
  if (lane == 63) lds[wave] = x;
  __syncthreads();
  int64_t before = 0, all = 0;
#pragma unroll
  for (int i = 0; i < kWaves; ++i) {
    const int64_t y = lds[i];
    before += i < wave ? y : 0;
    all += y;
  }
  *total = all;
  return before + x - v;
}

// Exclusive scan of value(i) for i in [0, n): store(i, sum before it); returns the sum.
// One pass in rounds of a value per thread, or (many values) a run of them per thread.
template <class V, class S>
__device__ inline int64_t scan_all(int32_t n, int64_t* lds, V value, S store) {
  int64_t total = 0;
  if (n <= 4 * kThreads) {
    int64_t before = 0;
    for (int32_t i0 = 0; i0 < n; i0 += kThreads) {
      const int32_t i = i0 + (int32_t)threadIdx.x;
      const int64_t at = block_scan(i < n ? value(i) : 0, &total, lds);
      if (i < n) store(i, before + at);
      before += total;
    }
    return before;
  }
  const int32_t per = (n + kThreads - 1) / kThreads;
  const int32_t a = min(n, per * (int32_t)threadIdx.x), b = min(n, a + per);
  int64_t sum = 0;
  for (int32_t i = a; i < b; ++i) sum += value(i);
  int64_t at = block_scan(sum, &total, lds);
  for (int32_t i = a; i < b; ++i) {
    const int64_t v = value(i);
    store(i, at);
    at += v;
  }
  return total;
}

// The last of n ascending numbers that is at most u (the first one is).
__device__ inline int32_t last_at_most(const int64_t* v, int32_t n, int64_t u) {
  int32_t a = 0, b = n;
  while (b - a > 1) {
    const int32_t m = (a + b) >> 1;
    if (v[m] <= u) a = m;
    else b = m;
  }
  return a;
}

constexpr int kSmall = 1024;  // requests, up to which the tables lie in shared memory
constexpr int kNear = 1024;   // tiles of a kind, likewise

__device__ inline int64_t units_of(const AttendTile& t) { return (max(0, t.t1 - t.t0) + kUnit - 1) / kUnit; }

// The steps: groups of requests with one prefix; the order of requests (groups
// together) and of their rows; segments; tiles; units and runs; partial results and
// what is to be joined.  Each ends with a barrier, of which the kernel's time is made:
// 12 to 17 us for one request, 25 to 29 us for 128 in 24 groups, 37 us with one key / value
// head, whose 512 workgroups have 2048 waves to be given their runs.
template <bool kFits>
__global__ __launch_bounds__(kThreads) void plan_cut_kernel(AttendPlanDev p, BlockWin w, int32_t ratio,
                                                            uint32_t* d_flags) {
  constexpr int kKeys = kFits ? kSmall : PS_MAX_WINDOW_REQ;
  __shared__ uint32_t keys[kKeys];
  __shared__ uint32_t unsorted[kFits ? kSmall : 1];
  __shared__ int32_t near_table[kFits ? 2 * kSmall : 1], near_least[kFits ? 2 * kSmall : 1];
  __shared__ int32_t near_slot[kFits ? kSmall : 1], near_members[kFits ? kSmall : 1], near_base[kFits ? kSmall : 1];
  __shared__ int64_t near_begin[2][kNear];
  __shared__ int64_t near_run[kMaxGroups * (1 + kWideWaves)];  // first unit of each run, the wide ones' in front
  __shared__ int32_t wide_number[kThreads], wide_units[kThreads];
  __shared__ int64_t sums[kWaves];
  __shared__ int32_t n_todo;
  int32_t* const table = kFits ? near_table : p.table;
  int32_t* const least = kFits ? near_least : p.least;
  int32_t* const slot_of = kFits ? near_slot : p.slot_of;
  int32_t* const members = kFits ? near_members : p.members;
  int32_t* const base = kFits ? near_base : p.base;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int32_t n = w.n_req;

  // Row offsets that do not ascend: nothing is planned.
  int bad = 0;
  for (int32_t r = tid; r < n; r += kThreads) {
    const int32_t lo = w.row_off[r], hi = w.row_off[r + 1];
    bad |= lo < 0 || hi < lo || hi > w.n_rows;
    members[r] = 0;
  }
  for (int32_t i = tid; i <= p.table_mask; i += kThreads) {
    table[i] = 0;
    least[i] = INT32_MAX;
  }
  if (tid == 0) n_todo = 0;
  if (__syncthreads_or(bad)) {
    if (d_flags)
      for (int32_t r = tid; r < n; r += kThreads) d_flags[r] = PS_R_INVALID;
    if (tid == 0) *p.head = AttendHead{w.pages, w.n_rows, p.waves, 0, {}};
    for (int32_t x = tid; x < p.n_runs; x += kThreads) p.runs[x].rounds = p.runs[x].units = 0;
    return;
  }

  // Groups: requests with few rows, all of which see the whole prefix, meet
  // in a hash table by the place and length of their prefix.
  for (int32_t r = tid; r < n; r += kThreads) {
    const BlockReq q = block_req(w, r);
    const int32_t rows = q.hi - q.lo;
    const int64_t pre = (int64_t)q.pre_len * w.bt;
    int32_t at = -1;
    if (p.flags[r] == 0 && rows > 0 && (rows == 1 || (int64_t)rows * ratio <= kShareMaxRows) &&
        pre >= kShareMinTokens && (int64_t)q.ctx - rows + 1 >= pre) {
      uint64_t h = (uint64_t)q.pre_off * 0x9E3779B97F4A7C15ull ^ (uint64_t)q.pre_len * 0xC2B2AE3D27D4EB4Full;
      at = (int32_t)((h ^ h >> 32) & (uint32_t)p.table_mask);
      for (;;) {  // (at most half of the slots are taken)
        const int32_t held = atomicCAS(&table[at], 0, r + 1);
        if (held == 0) break;
        const ps_req d = w.reqs[held - 1];
        if (d.pre_off == q.pre_off && d.pre_len == q.pre_len) break;
        at = (at + 1) & p.table_mask;
      }
      atomicMin(&least[at], r);
    }
    slot_of[r] = at;
  }
  __syncthreads();
  for (int32_t r = tid; r < n; r += kThreads)
    if (slot_of[r] >= 0) atomicAdd(&members[least[slot_of[r]]], 1);
  __syncthreads();

  // The order: by the group's least member, then by request, whatever the
  // order in which the table was filled.
  int grouped = 0;
  auto key_of = [&](int32_t r) {
    const int32_t at = slot_of[r];
    const int32_t first = at >= 0 && members[least[at]] > 1 ? least[at] : r;
    grouped |= first != r;
    return (uint32_t)first << 13 | (uint32_t)r;
  };
  if (kFits) {
    // (a key's place is the number of smaller ones: fewer barriers than a sort's steps)
    for (int32_t r = tid; r < n; r += kThreads) unsorted[r] = key_of(r);
    const bool sort = __syncthreads_or(grouped);
    for (int32_t r = tid; r < n; r += kThreads) {
      const uint32_t key = unsorted[r];
      int32_t at = r;
      if (sort) {
        at = 0;
        for (int32_t i = 0; i < n; ++i) at += unsorted[i] < key;
      }
      keys[at] = key;
    }
  } else {
    int32_t n2 = 64;
    while (n2 < n) n2 <<= 1;
    for (int32_t r = tid; r < n2; r += kThreads) keys[r] = r < n ? key_of(r) : 0xFFFFFFFFu;
    if (__syncthreads_or(grouped))
      for (int32_t k = 2; k <= n2; k <<= 1)
        for (int32_t j = k >> 1; j > 0; j >>= 1) {
          __syncthreads();
          for (int32_t i = tid; i < n2; i += kThreads) {
            const int32_t o = i ^ j;
            if (o > i) {
              const uint32_t x = keys[i], y = keys[o];
              if ((x > y) == ((i & k) == 0)) {
                keys[i] = y;
                keys[o] = x;
              }
            }
          }
        }
  }
  __syncthreads();
  auto rows_of = [&](int32_t i) {
    const int32_t r = keys[i] & 8191u;
    return w.row_off[r + 1] - w.row_off[r];
  };
  scan_all(
      n, sums, [&](int32_t i) { return (int64_t)rows_of(i); }, [&](int32_t i, int64_t at) { base[i] = (int32_t)at; });
  __syncthreads();

  // Segments, and the rows in their order.
  auto write_row = [&](int32_t i, const BlockReq& q, bool ok, int32_t j) {
    const int32_t at = base[i] + j;
    const int64_t lim = (int64_t)q.ctx - (q.hi - q.lo) + j + 1;
    p.row[at] = q.lo + j;
    p.lim[at] = ok && lim > 0 ? (int32_t)lim : 0;
  };
  auto tiles_of = [&](AttendSeg* s) {
    s->wide = (int64_t)s->tokens * ratio > kNarrowRows;
    s->tiles = s->wide ? (int32_t)(((int64_t)s->tokens * ratio + p.wide_rows - 1) / p.wide_rows) : 1;
  };
  for (int32_t i = tid; i < n; i += kThreads) {
    const int32_t r = keys[i] & 8191u, first = keys[i] >> 13;
    const BlockReq q = block_req(w, r);
    const bool ok = p.flags[r] == 0;
    const int32_t rows = q.hi - q.lo;
    const bool shared = slot_of[r] >= 0 && members[first] > 1;
    AttendSeg s{}, none{};
    s.pre_off = q.pre_off;
    s.tail_off = q.tail_off;
    s.pre_len = q.pre_len;
    s.shared = shared;
    const int32_t pre = shared ? q.pre_len * w.bt : 0;
    AttendSeg own = s;
    own.p0 = base[i];
    own.tokens = rows;
    own.t0 = pre;
    own.t1 = ok && rows > 0 ? q.ctx : 0;
    tiles_of(&own);
    if (own.t1 <= own.t0) own.tiles = 0;
    p.segs[2 * i + 1] = own;
    int32_t lead = -1;
    if (shared) {
      // the place of the group's first member: of the keys, the least with this first
      int32_t a = 0, b = i;
      while (a < b) {
        const int32_t m = (a + b) >> 1;
        if ((int32_t)(keys[m] >> 13) < first) a = m + 1;
        else b = m;
      }
      lead = a;
      if (lead == i) {
        const int32_t last = i + members[first] - 1;
        s.p0 = base[i];
        s.tokens = base[last] + rows_of(last) - s.p0;
        s.t1 = pre;
        tiles_of(&s);
        none = s;
      }
    }
    p.segs[2 * i] = none;
    p.lead[i] = lead;
    if (rows <= 8) {
      for (int32_t j = 0; j < rows; ++j) write_row(i, q, ok, j);
    } else {
      p.todo[atomicAdd(&n_todo, 1)] = i;
    }
  }
  __syncthreads();
  for (int32_t k = wave; k < n_todo; k += kWaves) {
    const int32_t i = p.todo[k], r = keys[i] & 8191u;
    const BlockReq q = block_req(w, r);
    const bool ok = p.flags[r] == 0;
    for (int32_t j = lane; j < q.hi - q.lo; j += 64) write_row(i, q, ok, j);
  }

  // Tiles, those of both kinds counted in one sum.
  const int64_t counts = scan_all(
      2 * n, sums,
      [&](int32_t k) { return p.segs[k].wide ? (int64_t)p.segs[k].tiles : (int64_t)p.segs[k].tiles << 32; },
      [&](int32_t k, int64_t at) { p.segs[k].tile0 = p.segs[k].wide ? (int32_t)at : (int32_t)(at >> 32); });
  const int32_t n_tiles[2] = {(int32_t)counts, (int32_t)(counts >> 32)};
  if (tid == 0) n_todo = 0;
  __syncthreads();
  auto write_tile = [&](const AttendSeg& s, int32_t k, int32_t seg) {
    AttendTile t{};
    t.pre_off = s.pre_off;
    t.tail_off = s.tail_off;
    t.pre_len = s.pre_len;
    t.p0 = s.p0;
    t.row0 = k * p.wide_rows;
    t.rows = (int32_t)min((int64_t)s.tokens * ratio - t.row0, (int64_t)(s.wide ? p.wide_rows : kNarrowRows));
    t.t0 = s.t0;
    // (a request's later rows see more: none of the tile's sees more than its last)
    t.t1 = min(s.t1, p.lim[s.p0 + (t.row0 + t.rows - 1) / ratio]);
    t.shared = s.shared;
    t.prefix = !(seg & 1);
    t.pre_tile = -1;
    if (s.shared && !t.prefix) {
      const AttendSeg& l = p.segs[2 * p.lead[seg / 2]];
      t.pre_tile = l.wide ? l.tile0 | kWideBit : l.tile0;
      t.pre_p0 = l.p0;
    }
    p.tiles[s.wide ? 0 : 1][s.tile0 + k] = t;
  };
  for (int32_t k = tid; k < 2 * n; k += kThreads) {
    const AttendSeg s = p.segs[k];
    if (s.tiles <= 4)
      for (int32_t j = 0; j < s.tiles; ++j) write_tile(s, j, k);
    else
      p.todo[atomicAdd(&n_todo, 1)] = k;
  }
  __syncthreads();
  for (int32_t k = wave; k < n_todo; k += kWaves) {
    const int32_t seg = p.todo[k];
    const AttendSeg s = p.segs[seg];
    for (int32_t j = lane; j < s.tiles; j += 64) write_tile(s, j, seg);
  }
  __syncthreads();

  // Units end to end, and who takes them.
  int32_t wide_groups, rounds = 0, runs[2];
  int64_t units[2], wide_cost = 0;  // (units: with those that stand for a tile's start)
  const int32_t start[2] = {kTileUnits, 0};
  int64_t* begin[2];
  auto run_at = [&](int kind) { return near_run + kind * kMaxGroups; };
  for (int kind = 0; kind < 2; ++kind) {
    begin[kind] = n_tiles[kind] <= kNear ? near_begin[kind] : p.begin[kind];
    int64_t mine = 0;
    units[kind] = scan_all(
        n_tiles[kind], sums,
        [&](int32_t k) {
          const AttendTile& t = p.tiles[kind][k];
          const int64_t u = units_of(t);
          mine += u * (kUnitCost + t.rows);
          return u + start[kind];
        },
        [&](int32_t k, int64_t at) { begin[kind][k] = at; });
    if (kind == 0 && n_tiles[0] > 4 * kThreads) mine /= 2;  // (each value was asked for twice)
    if (kind == 0 && n_tiles[0] > 0 && n_tiles[1] > 0) block_scan(mine, &wide_cost, sums);
  }
  {
    int64_t n_wide = units[0] > 0 ? p.groups : 0;
    if (units[0] > 0 && units[1] > 0) {
      // (rounded down: what narrow tiles wait for is latency)
      wide_cost += (int64_t)kWideTileCost * n_tiles[0];
      const int64_t all = wide_cost + kUnitCost * units[1] + (int64_t)kTileCost * n_tiles[1];
      n_wide = max(wide_cost * p.groups / all, (int64_t)1);
      n_wide = min(n_wide, (int64_t)p.groups - 1);
    }
    wide_groups = (int32_t)n_wide;
    runs[0] = (int32_t)min(n_wide, units[0]);
    runs[1] = (int32_t)min((p.groups - n_wide) * p.waves, units[1]);
  }
  __syncthreads();
  // Rounds of whole tiles, as many as leave no workgroup (a thread each) above
  // the average; then `share` units more for each, the most evenly.
  if (wide_groups > 0 && n_tiles[0] >= wide_groups) {
    const int32_t n_wide = wide_groups;
    const bool mine = tid < n_wide;
    int64_t whole = 0, total, share = 0;
    auto tile_at = [&](int32_t i) { return units_of(p.tiles[0][tile_of_round(tid, i, n_wide)]) + kTileUnits; };
    // (each takes as many as it can, in one pass, and gives back what the others cannot.  Rounds taken
    // off one by one, all summed anew, were 16.8 ms for 2047 tiles of each of 128 heads behind one of
    // 400,000 positions)
    const int32_t most = n_tiles[0] / n_wide;
    int32_t can = 0;
    int64_t sum = 0;
    for (int32_t i = 0; mine && i < most; ++i) {
      sum += tile_at(i);
      if (sum * n_wide <= units[0]) {
        can = i + 1;
        whole = sum;
      }
    }
    if (tid == 0) n_todo = most;
    __syncthreads();
    if (mine && can < most) atomicMin(&n_todo, can);
    __syncthreads();
    rounds = n_todo;
    for (int32_t i = rounds; mine && i < can; ++i) whole -= tile_at(i);
    // a level that those below it are filled up to
    int64_t left = units[0], n_below = n_wide;
    bool below = mine;
    for (;;) {
      block_scan(mine && !below ? whole : 0, &total, sums);
      left = units[0] - total;
      const bool out = below && whole * n_below > left;
      block_scan(out ? 1 : 0, &total, sums);
      if (total == 0) break;
      n_below -= total;
      below = below && !out;
    }
    // (left / n_below each, the first left % n_below one more)
    const int64_t rank = block_scan(below ? 1 : 0, &total, sums);
    if (below) share = left / n_below + (rank < left % n_below) - whole;
    const int32_t done = rounds * n_wide;
    const int64_t skip = done < n_tiles[0] ? begin[0][done] : units[0];
    const int64_t at = block_scan(share, &total, sums);
    runs[0] = n_wide;
    if (mine) run_at(0)[tid] = skip + at;
  } else {
    for (int32_t r = tid; r < runs[0]; r += kThreads) {
      run_at(0)[r] = units[0] * r / runs[0];
    }
  }
  // (counting a tile as a unit more made a batch of short contexts no faster, and one of
  // long ones slower: 241 -> 246 us)
  for (int32_t r = tid; r < runs[1]; r += kThreads) run_at(1)[r] = units[1] * r / runs[1];
  __syncthreads();
  // What a wide run has without the tiles' starts; those that have something are numbered.
  auto before = [&](int64_t u) {
    if (u >= units[0]) return units[0] - (int64_t)kTileUnits * n_tiles[0];
    const int32_t k = last_at_most(begin[0], n_tiles[0], u);
    return max(begin[0][k], u - kTileUnits) - (int64_t)kTileUnits * k;
  };
  if (runs[0] > 0) {
    int32_t have = 0;
    if (tid < runs[0])
      have = (int32_t)(before(tid + 1 < runs[0] ? run_at(0)[tid + 1] : units[0]) - before(run_at(0)[tid]));
    int64_t total;
    const int64_t number = block_scan(have > 0, &total, sums);
    wide_units[tid] = have;
    wide_number[tid] = (int32_t)number;
  }
  __syncthreads();
  for (int kind = 0; kind < 2; ++kind) {
    AttendTile* tiles = p.tiles[kind];
    const int32_t whole = kind == 0 ? rounds * wide_groups : 0;
    // (a run that begins at the same unit as the next one is empty and not found)
    auto number_at = [&](int64_t u) {
      const int32_t r = last_at_most(run_at(kind), runs[kind], u);
      return kind == 0 ? wide_number[r] : r;
    };
    for (int32_t k = tid; k < n_tiles[kind]; k += kThreads) {
      const int64_t u = units_of(tiles[k]), b = begin[kind][k] + start[kind];
      int32_t first = 0, pieces = u > 0 ? 1 : 0;
      if (u > 0 && k >= whole) {
        first = number_at(b);
        pieces = number_at(b + u - 1) - first + 1;
      }
      tiles[k].first = first;
      tiles[k].pieces = pieces;
    }
  }
  __syncthreads();
  int64_t slots = 0;
  for (int kind = 0; kind < 2; ++kind) {
    AttendTile* tiles = p.tiles[kind];
    const int64_t before = slots;
    // (kept where there are two pieces or more, or one of a shared segment.  One
    // comparison of a sum: of the same test with && and ||, the compiler dropped the
    // branch that stores the place of a shared tile's only piece.)
    slots += scan_all(
        n_tiles[kind], sums,
        [&](int32_t k) {
          return tiles[k].pieces + tiles[k].shared > 1 ? (int64_t)tiles[k].pieces * tiles[k].rows : (int64_t)0;
        },
        [&](int32_t k, int64_t at) {
          tiles[k].slot = tiles[k].pieces + tiles[k].shared > 1 ? (int32_t)(before + at) : -1;
        });
  }

  // What each wave takes.
  __syncthreads();
  for (int32_t x = tid; x < p.n_runs; x += kThreads) {
    const int32_t g = x / p.waves, kind = g >= wide_groups;
    // (the waves' runs go round the workgroups)
    const int32_t r = kind == 0 ? g : g - wide_groups + x % p.waves * (p.groups - wide_groups);
    AttendRun run{};
    run.kind = kind;
    if (g < p.groups && r < runs[kind]) {
      run.rounds = kind == 0 ? rounds : 0;
      run.stride = wide_groups;
      run.number = kind == 0 ? wide_number[r] : r;
      const int64_t at = run_at(kind)[r];
      run.units = kind == 0 ? wide_units[r] : (int32_t)((r + 1 < runs[1] ? run_at(1)[r + 1] : units[1]) - at);
      if (run.units > 0) {
        run.next = last_at_most(begin[kind], n_tiles[kind], at);
        run.from = max(0, (int32_t)(at - begin[kind][run.next]) - start[kind]);
      }
      if (run.rounds > 0 || run.units > 0) run.tile = p.tiles[kind][run.rounds > 0 ? r : run.next];
    }
    // (of an empty one only what says so)
    if (run.rounds > 0 || run.units > 0) p.runs[x] = run;
    else p.runs[x].rounds = p.runs[x].units = 0;
  }

  // What is to be joined: the rows of own tiles that are kept, with their prefix
  // tiles; of shared segments that end with the prefix, the rows with the prefix
  // alone; of everything else that has no pieces, places of empty rows.
  if (tid == 0) n_todo = 0;
  __syncthreads();
  // (pre_tile, pre_p0: the prefix's first tile and place)
  auto push = [&](int32_t place, int32_t sub, const AttendTile* own, int32_t pre_tile, int32_t pre_p0) {
    AttendJoin x{};
    x.row = p.row[place];
    x.sub = sub;
    x.empty = p.lim[place] <= 0;
    auto part = [&](int i, const AttendTile& t) {
      x.from[i] = t.slot + (place - t.p0) * ratio + sub - t.row0;
      x.count[i] = t.pieces;
      x.step[i] = t.rows;
    };
    if (own) part(0, *own);
    if (pre_tile >= 0) {
      const int32_t k = pre_tile & (kWideBit - 1);
      if (pre_tile & kWideBit) part(1, p.tiles[0][k + ((place - pre_p0) * ratio + sub) / p.wide_rows]);
      else part(1, p.tiles[1][k]);
    }
    p.joins[atomicAdd(&n_todo, 1)] = x;
  };
  for (int kind = 0; kind < 2; ++kind) {
    // a wave per wide tile, 4 lanes per narrow tile
    const int per = kind == 0 ? 64 : 4;
    for (int32_t k = tid / per; k < n_tiles[kind]; k += kThreads / per) {
      const AttendTile t = p.tiles[kind][k];
      if (t.prefix || (t.pieces > 0 && t.slot < 0)) continue;
      for (int32_t r = tid % per; r < t.rows; r += per) {
        const int32_t x = t.row0 + r, at = x / ratio, sub = x - at * ratio;
        if (t.pieces > 0) push(t.p0 + at, sub, &t, t.pre_tile, t.pre_p0);
        else if (sub == 0 || r == 0) push(t.p0 + at, -1, nullptr, -1, 0);
      }
    }
  }
  for (int32_t i = wave; i < n; i += kWaves) {
    const AttendSeg& s = p.segs[2 * i + 1];
    if (s.tiles > 0) continue;
    int32_t pre_tile = -1, pre_p0 = 0;
    if (s.shared) {
      const AttendSeg& l = p.segs[2 * p.lead[i]];
      pre_tile = l.wide ? l.tile0 | kWideBit : l.tile0;
      pre_p0 = l.p0;
    }
    for (int32_t j = lane; j < s.tokens; j += 64)
      if (s.shared)
        for (int32_t sub = 0; sub < ratio; ++sub) push(s.p0 + j, sub, nullptr, pre_tile, pre_p0);
      else
        push(s.p0 + j, -1, nullptr, -1, 0);
  }
  __syncthreads();
  if (tid == 0) *p.head = AttendHead{w.pages, w.n_rows, p.waves, n_todo, {}};
}

}  // namespace

}  // namespace ps

hipError_t ps_launch_attend_plan(const ps::AttendPlanDev& p, const ps::BlockWin& w, int32_t ratio, uint32_t* d_flags,
                                 hipStream_t s) {
  hipLaunchKernelGGL(ps::plan_check_kernel, dim3(w.n_req), dim3(256), 0, s, p, w, d_flags);
  if (p.table_mask < 2 * ps::kSmall)
    hipLaunchKernelGGL(ps::plan_cut_kernel<true>, dim3(1), dim3(ps::kThreads), 0, s, p, w, ratio, d_flags);
  else
    hipLaunchKernelGGL(ps::plan_cut_kernel<false>, dim3(1), dim3(ps::kThreads), 0, s, p, w, ratio, d_flags);
  return hipGetLastError();
}
