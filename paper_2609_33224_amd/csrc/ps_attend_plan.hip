// The plan of a window's attention: which requests share a prefix, the order
// of the rows, segments, tiles and the workgroups that take them.  Two
// launches: every page a context needs is checked by a workgroup per request,
// then one workgroup cuts the work (thousands of small steps with a barrier
// between; a step's layers share one plan).

#include "ps_blocks.h"

namespace ps {

namespace {

constexpr int kThreads = 512;
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

// Exclusive sums over the workgroup of each thread's value; *total to all.
__device__ inline int64_t block_scan(int64_t v, int64_t* total, int64_t* lds) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  int64_t x = v;
  for (int o = 1; o < 64; o <<= 1) {
    const int64_t y = __shfl_up((long long)x, o, 64);
    if (lane >= o) x += y;
  }
  __syncthreads();
  if (lane == 63) lds[wave] = x;
  __syncthreads();
  int64_t before = 0, all = 0;
  for (int i = 0; i < kWaves; ++i) {
    const int64_t y = lds[i];
    before += i < wave ? y : 0;
    all += y;
  }
  *total = all;
  return before + x - v;
}

// Exclusive scan of value(i) for i in [0, n): store(i, sum before it); returns the sum.
template <class V, class S>
__device__ inline int64_t scan_all(int32_t n, int64_t* lds, V value, S store) {
  const int32_t per = (n + kThreads - 1) / kThreads;
  const int32_t a = min(n, per * (int32_t)threadIdx.x), b = min(n, a + per);
  int64_t sum = 0, total;
  for (int32_t i = a; i < b; ++i) sum += value(i);
  int64_t at = block_scan(sum, &total, lds);
  for (int32_t i = a; i < b; ++i) {
    const int64_t v = value(i);
    store(i, at);
    at += v;
  }
  return total;
}

__global__ __launch_bounds__(kThreads) void plan_cut_kernel(AttendPlanDev p, BlockWin w, int32_t ratio,
                                                            uint32_t* d_flags) {
  __shared__ uint32_t keys[PS_MAX_WINDOW_REQ];
  __shared__ int64_t sums[kWaves];
  __shared__ int32_t n_todo;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int32_t n = w.n_req;

  // Row offsets that do not ascend: nothing is planned.
  int bad = 0;
  for (int32_t r = tid; r < n; r += kThreads) {
    const int32_t lo = w.row_off[r], hi = w.row_off[r + 1];
    bad |= lo < 0 || hi < lo || hi > w.n_rows;
  }
  if (__syncthreads_or(bad)) {
    if (d_flags)
      for (int32_t r = tid; r < n; r += kThreads) d_flags[r] = PS_R_INVALID;
    if (tid == 0) *p.head = AttendHead{};
    return;
  }

  // Groups: requests with few rows, all of which see the whole prefix, meet
  // in a hash table by the place and length of their prefix.
  for (int32_t i = tid; i <= p.table_mask; i += kThreads) {
    p.table[i] = 0;
    p.least[i] = INT32_MAX;
  }
  for (int32_t r = tid; r < n; r += kThreads) p.members[r] = 0;
  if (tid == 0) n_todo = 0;
  __syncthreads();
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
        const int32_t held = atomicCAS(&p.table[at], 0, r + 1);
        if (held == 0) break;
        const ps_req d = w.reqs[held - 1];
        if (d.pre_off == q.pre_off && d.pre_len == q.pre_len) break;
        at = (at + 1) & p.table_mask;
      }
      atomicMin(&p.least[at], r);
    }
    p.slot_of[r] = at;
  }
  __syncthreads();
  for (int32_t r = tid; r < n; r += kThreads)
    if (p.slot_of[r] >= 0) atomicAdd(&p.members[p.least[p.slot_of[r]]], 1);
  __syncthreads();

  // The order: by the group's least member, then by request, whatever the
  // order in which the table was filled.
  int32_t n2 = 64;
  while (n2 < n) n2 <<= 1;
  for (int32_t r = tid; r < n2; r += kThreads) {
    uint32_t key = 0xFFFFFFFFu;
    if (r < n) {
      const int32_t at = p.slot_of[r];
      const int32_t first = at >= 0 && p.members[p.least[at]] > 1 ? p.least[at] : r;
      key = (uint32_t)first << 13 | (uint32_t)r;
    }
    keys[r] = key;
  }
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
  __syncthreads();
  scan_all(
      n, sums, [&](int32_t i) { return (int64_t)(w.row_off[(keys[i] & 8191u) + 1] - w.row_off[keys[i] & 8191u]); },
      [&](int32_t i, int64_t at) { p.base[i] = (int32_t)at; });
  __syncthreads();

  // Segments, and the rows in their order.
  auto write_row = [&](int32_t i, const BlockReq& q, bool ok, int32_t j) {
    const int32_t at = p.base[i] + j;
    const int64_t lim = (int64_t)q.ctx - (q.hi - q.lo) + j + 1;
    p.row[at] = q.lo + j;
    p.lim[at] = ok && lim > 0 ? (int32_t)lim : 0;
    p.place[at] = i;
  };
  for (int32_t i = tid; i < n; i += kThreads) {
    const int32_t r = keys[i] & 8191u, first = keys[i] >> 13;
    const BlockReq q = block_req(w, r);
    const bool ok = p.flags[r] == 0;
    const int32_t rows = q.hi - q.lo;
    const bool shared = p.slot_of[r] >= 0 && p.members[first] > 1;
    p.order[i] = r;
    AttendSeg s{};
    s.pre_off = q.pre_off;
    s.tail_off = q.tail_off;
    s.pre_len = q.pre_len;
    s.shared = shared;
    const int32_t pre = shared ? q.pre_len * w.bt : 0;
    AttendSeg own = s;
    own.p0 = p.base[i];
    own.tokens = rows;
    own.t0 = pre;
    own.t1 = ok && rows > 0 ? q.ctx : 0;
    const bool some = own.t1 > own.t0;
    own.wide = (int64_t)rows * ratio > kNarrowRows;
    own.tiles = !some ? 0 : own.wide ? (int32_t)(((int64_t)rows * ratio + kWideRows - 1) / kWideRows) : 1;
    p.segs[2 * i + 1] = own;
    p.segs[2 * i] = AttendSeg{};
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
        const int32_t last = i + p.members[first] - 1, lr = keys[last] & 8191u;
        s.p0 = p.base[i];
        s.tokens = p.base[last] + (w.row_off[lr + 1] - w.row_off[lr]) - s.p0;
        s.t1 = pre;
        s.wide = (int64_t)s.tokens * ratio > kNarrowRows;
        s.tiles = s.wide ? (int32_t)(((int64_t)s.tokens * ratio + kWideRows - 1) / kWideRows) : 1;
        p.segs[2 * i] = s;
      }
    }
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
  __syncthreads();

  // Tiles.
  if (tid == 0) n_todo = 0;
  int32_t n_tiles[2];
  for (int kind = 0; kind < 2; ++kind)
    n_tiles[kind] = (int32_t)scan_all(
        2 * n, sums,
        [&](int32_t k) { return (int64_t)(p.segs[k].wide == (kind == 0) ? p.segs[k].tiles : 0); },
        [&](int32_t k, int64_t at) {
          if (p.segs[k].wide == (kind == 0)) p.segs[k].tile0 = (int32_t)at;
        });
  __syncthreads();
  auto write_tile = [&](const AttendSeg& s, int32_t k, int32_t prefix) {
    AttendTile t{};
    t.pre_off = s.pre_off;
    t.tail_off = s.tail_off;
    t.pre_len = s.pre_len;
    t.p0 = s.p0;
    t.row0 = k * kWideRows;
    t.rows = (int32_t)min((int64_t)s.tokens * ratio - t.row0, (int64_t)(s.wide ? kWideRows : kNarrowRows));
    t.t0 = s.t0;
    // (a request's later rows see more: none of the tile's sees more than its last)
    t.t1 = min(s.t1, p.lim[s.p0 + (t.row0 + t.rows - 1) / ratio]);
    t.shared = s.shared;
    t.prefix = prefix;
    p.tiles[s.wide ? 0 : 1][s.tile0 + k] = t;
  };
  for (int32_t k = tid; k < 2 * n; k += kThreads) {
    const AttendSeg s = p.segs[k];
    if (s.tiles <= 4)
      for (int32_t j = 0; j < s.tiles; ++j) write_tile(s, j, !(k & 1));
    else
      p.todo[atomicAdd(&n_todo, 1)] = k;
  }
  __syncthreads();
  for (int32_t k = wave; k < n_todo; k += kWaves) {
    const AttendSeg s = p.segs[p.todo[k]];
    for (int32_t j = lane; j < s.tiles; j += 64) write_tile(s, j, !(p.todo[k] & 1));
  }
  __syncthreads();

  // Units end to end, who takes them, and the rows of partial results.
  AttendHead h{};
  int64_t units[2];
  auto units_of = [&](const AttendTile& t) { return (int64_t)((max(0, t.t1 - t.t0) + kUnit - 1) / kUnit); };
  for (int kind = 0; kind < 2; ++kind) {
    h.n_tiles[kind] = n_tiles[kind];
    units[kind] = scan_all(
        n_tiles[kind], sums, [&](int32_t k) { return units_of(p.tiles[kind][k]); },
        [&](int32_t k, int64_t at) { p.begin[kind][k] = at; });
  }
  {
    int64_t mine = 0, wide;
    for (int32_t k = tid; k < n_tiles[0]; k += kThreads) mine += units_of(p.tiles[0][k]) * (kUnitCost + p.tiles[0][k].rows);
    block_scan(mine, &wide, sums);
    const int64_t all = wide + kUnitCost * units[1];
    int64_t n_wide = all > 0 ? (wide * p.groups + all / 2) / all : 0;
    if (units[0] > 0) n_wide = max(n_wide, (int64_t)1);
    if (units[1] > 0) n_wide = min(n_wide, (int64_t)p.groups - 1);
    h.wide_groups = h.runs[0] = (int32_t)n_wide;
    h.runs[1] = (int32_t)min((p.groups - n_wide) * kWavesPerGroup, units[1]);
  }
  __syncthreads();
  // Rounds of whole tiles, as many as leave no workgroup (a thread each) above
  // the average; then `share` units more for each, the most evenly.
  int64_t share = 0;
  if (h.wide_groups > 0) {
    const int32_t n_wide = h.wide_groups;
    const bool mine = tid < n_wide;
    int64_t whole = 0, total;
    for (h.rounds = n_tiles[0] / n_wide;; --h.rounds) {
      whole = 0;
      for (int32_t i = 0; mine && i < h.rounds; ++i) whole += units_of(p.tiles[0][tid + i * n_wide]);
      if (!__syncthreads_or(mine && h.rounds > 0 && whole * n_wide > units[0])) break;
    }
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
  }
  int64_t slots = 0;
  for (int kind = 0; kind < 2; ++kind) {
    AttendTile* tiles = p.tiles[kind];
    const int32_t whole = kind == 0 ? h.rounds * h.wide_groups : 0, runs = h.runs[kind];
    const int64_t skip = whole < n_tiles[kind] ? p.begin[kind][whole] : units[kind];
    if (kind == 0) {
      int64_t total;
      const int64_t at = block_scan(share, &total, sums), number = block_scan(share > 0, &total, sums);
      if (tid < runs) {
        p.run_at[0][tid] = skip + at;
        p.runs[0][tid].units = (int32_t)share;
        p.runs[0][tid].number = (int32_t)number;
      }
    } else {
      for (int32_t r = tid; r < runs; r += kThreads) {
        p.run_at[1][r] = units[1] * r / runs;
        p.runs[1][r].units = (int32_t)(units[1] * (r + 1) / runs - units[1] * r / runs);
        p.runs[1][r].number = r;
      }
    }
    __syncthreads();
    for (int32_t r = tid; r < runs; r += kThreads) {
      const int64_t at = p.run_at[kind][r];
      int32_t a = 0, b = n_tiles[kind];  // the last tile that begins at or before `at`
      while (b - a > 1) {
        const int32_t m = (a + b) >> 1;
        if (p.begin[kind][m] <= at) a = m;
        else b = m;
      }
      p.runs[kind][r].tile = a;
      p.runs[kind][r].from = (int32_t)(at - p.begin[kind][a]);
    }
    auto run_of = [&](int64_t u) {  // the last run that begins at or before unit u
      int32_t a = 0, b = runs;
      while (b - a > 1) {
        const int32_t m = (a + b) >> 1;
        if (p.run_at[kind][m] <= u) a = m;
        else b = m;
      }
      return p.runs[kind][a].number;
    };
    for (int32_t k = tid; k < n_tiles[kind]; k += kThreads) {
      const int64_t u = units_of(tiles[k]), b = p.begin[kind][k];
      tiles[k].first = u > 0 && k >= whole ? run_of(b) : 0;
      tiles[k].pieces = u == 0 ? 0 : k < whole ? 1 : run_of(b + u - 1) - tiles[k].first + 1;
    }
    __syncthreads();
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
    __syncthreads();
  }

  // What is to be joined: the rows of own tiles that are kept, with their prefix
  // tiles; of shared segments that end with the prefix, the rows with the prefix
  // alone; of everything else that has no pieces, places of empty rows.
  if (tid == 0) n_todo = 0;
  __syncthreads();
  auto push = [&](int32_t place, int32_t sub, int32_t own) {
    AttendJoin x{place, sub, {own, -1}};
    const int32_t lead = sub < 0 ? -1 : p.lead[p.place[place]];
    if (lead >= 0) {
      const AttendSeg& s = p.segs[2 * lead];
      x.tile[1] = s.wide ? (s.tile0 + ((place - s.p0) * ratio + sub) / kWideRows) | kWideBit : s.tile0;
    }
    p.joins[atomicAdd(&n_todo, 1)] = x;
  };
  for (int kind = 0; kind < 2; ++kind) {
    // a wave per wide tile, a quarter of one per narrow tile
    const int per = kind == 0 ? 64 : 16;
    for (int32_t k = tid / per; k < n_tiles[kind]; k += kThreads / per) {
      const AttendTile t = p.tiles[kind][k];
      if (t.prefix || (t.pieces > 0 && t.slot < 0)) continue;
      for (int32_t r = tid % per; r < t.rows; r += per) {
        const int32_t x = t.row0 + r, at = x / ratio, sub = x - at * ratio;
        if (t.pieces > 0) push(t.p0 + at, sub, kind == 0 ? k | kWideBit : k);
        else if (sub == 0 || r == 0) push(t.p0 + at, -1, -1);
      }
    }
  }
  for (int32_t i = wave; i < n; i += kWaves) {
    const AttendSeg& s = p.segs[2 * i + 1];
    if (s.tiles > 0) continue;
    for (int32_t j = lane; j < s.tokens; j += 64)
      if (s.shared)
        for (int32_t sub = 0; sub < ratio; ++sub) push(s.p0 + j, sub, -1);
      else
        push(s.p0 + j, -1, -1);
  }
  __syncthreads();
  h.n_joins = n_todo;
  if (tid == 0) *p.head = h;
}

}  // namespace

}  // namespace ps

hipError_t ps_launch_attend_plan(const ps::AttendPlanDev& p, const ps::BlockWin& w, int32_t ratio, uint32_t* d_flags,
                                 hipStream_t s) {
  hipLaunchKernelGGL(ps::plan_check_kernel, dim3(w.n_req), dim3(256), 0, s, p, w, d_flags);
  hipLaunchKernelGGL(ps::plan_cut_kernel, dim3(1), dim3(ps::kThreads), 0, s, p, w, ratio, d_flags);
  return hipGetLastError();
}
