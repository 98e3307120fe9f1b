// Internal layout of the block-cache calls (cache write, read back, window
// attention): what their kernels and their host code share.
#pragma once

#include "ps_device.h"

namespace ps {

// A window on the device (ps_kv_window), with the cache's block size.
struct BlockWin {
  const int32_t* pages;
  const ps_req* reqs;
  const int32_t* ctx;
  const int32_t* row_off;
  int64_t pages_len, n_pages;
  int32_t n_req, n_rows;
  int32_t bt;
};

struct BlockCache {
  unsigned char* k;
  unsigned char* v;
  uint8_t* kx;
  uint8_t* vx;
  int64_t page_stride, exp_stride;  // elements
  int64_t n_pages;
  int32_t heads, dim, bt, dtype;
};

struct BlockRows {
  unsigned char* data;
  int64_t row, head;  // strides in elements
  int32_t dtype;
};

// One request of a window, read and checked.
struct BlockReq {
  int64_t pre_off, tail_off;
  int32_t pre_len, tail_len;
  int32_t ctx, lo, hi;
  bool ok;
};

__host__ __device__ inline BlockReq block_req(const BlockWin& w, int32_t r) {
  BlockReq q;
  const ps_req d = w.reqs[r];
  q.pre_off = d.pre_off;
  q.tail_off = d.tail_off;
  q.pre_len = d.pre_len;
  q.tail_len = d.tail_len;
  q.ctx = w.ctx[r];
  q.lo = w.row_off[r];
  q.hi = w.row_off[r + 1];
  q.ok = d.pre_len >= 0 && d.tail_len >= 0 && d.pre_off >= 0 && d.tail_off >= 0 && d.pre_len <= w.pages_len &&
         d.tail_len <= w.pages_len && d.pre_off <= w.pages_len - d.pre_len && d.tail_off <= w.pages_len - d.tail_len &&
         (int64_t)d.pre_len + d.tail_len <= PS_MAX_CHAIN && q.ctx >= 0 &&
         q.ctx <= ((int64_t)d.pre_len + d.tail_len) * w.bt && q.ctx <= PS_MAX_WINDOW_CTX;
  return q;
}

// The request of a row: -1 where it belongs to none.  (Whatever row_off
// holds, the request found is in range and its row range holds the row.)
__host__ __device__ inline int32_t block_row_req(const BlockWin& w, int32_t row) {
  // one row a request: a decode window
  if (row < w.n_req && w.row_off[row] == row && w.row_off[row + 1] == row + 1) return row;
  int32_t a = 0, b = w.n_req;  // the last request that begins at or before the row
  while (b - a > 1) {
    const int32_t m = (a + b) >> 1;
    if (w.row_off[m] <= row) a = m;
    else b = m;
  }
  return w.row_off[a] <= row && row < w.row_off[a + 1] ? a : -1;
}

// Where row `row` of the window, of request r, lies: its page and slot; false where it
// has none.  *has_req: whether a request claims the row.
__host__ __device__ inline bool block_locate(const BlockWin& w, int32_t row, int32_t r, bool* has_req, int64_t* page,
                                             int32_t* slot) {
  *has_req = r >= 0;
  if (r < 0) return false;
  const BlockReq q = block_req(w, r);
  const int64_t pos = (int64_t)q.ctx - q.hi + row;
  if (!q.ok || pos < 0) return false;
  const int32_t b = (int32_t)(pos / w.bt);
  *slot = (int32_t)(pos - (int64_t)b * w.bt);
  *page = w.pages[b < q.pre_len ? q.pre_off + b : q.tail_off + (b - q.pre_len)];
  return *page >= 0 && *page < w.n_pages;
}

// ---- the attention's plan
//
// A segment is a run of a chain's positions [t0, t1) and the window's rows
// that attend over it: a prefix that several requests share with the rows of
// all of them, or what is left of one request's chain with its own rows.  Its
// rows (row of the window x query head of the group, row-major) are cut into
// tiles; a tile is wide (up to kWideRows or kTallRows rows) or narrow (all rows of a segment of
// kNarrowRows at most).  The tiles' positions, in units of kUnit, are laid end
// to end and dealt in runs: the wide ones' to some workgroups of each key / value
// head, the narrow ones' to the waves of the others, so many as the costs say.  Where there
// are more wide tiles than workgroups, these first take whole tiles, in rounds, so that
// neighbours go over the same positions at the same time and find them in the L2 cache;
// what is left makes their shares even.  So a tile may be cut into pieces; pieces and
// shared segments leave partial results, which a second kernel joins.
constexpr int kUnit = 64;
constexpr int kWideRows = 128, kTallRows = 256;  // of a wide tile: which of them, the host says (ps_attend_tall)
constexpr int kNarrowRows = 16;
constexpr int kMaxGroups = 512;                // workgroups per head
constexpr int kWideWaves = 4, kTallWaves = 8;  // of a workgroup, likewise
// Cost of a unit for a workgroup, in rows: of a narrow tile's (1.5 to 1.75 us of e4m3
// with every workgroup at work), and what a wide one's has beside its rows (3.7 us for 128).
constexpr int kUnitCost = 128;
constexpr int kWideTileCost = 256, kTileCost = 160;  // of a tile beside its units: lookups, q, results
// When wide tiles are dealt, each counts as so many units more: what begins and what cuts a
// tile costs about that.  24 prompts of 16 to 1500 tokens: 0: 296 us, 2: 258, 6: 245, 12:
// 250; 128 rows of 4 heads over one prefix alike with all.
constexpr int kTileUnits = 6;

// The tile that workgroup g takes in a round: the rounds go to and fro, since tiles of
// one prompt grow longer.  (4 prompts of 2048 tokens: 315 -> 223 us.)
__host__ __device__ inline int32_t tile_of_round(int32_t g, int32_t round, int32_t n) {
  return round * n + (round & 1 ? n - 1 - g : g);
}

constexpr int kShareMinTokens = 64;  // of a prefix
constexpr int kShareMaxRows = 64;    // of a member (or one row of all its heads)

struct AttendSeg {
  int64_t pre_off, tail_off;  // the chain of one of its requests
  int32_t pre_len;
  int32_t p0, tokens;  // its rows: places p0 .. p0 + tokens of the order
  int32_t t0, t1;
  int32_t tile0, tiles;  // within the list of its kind
  int32_t wide, shared;
};

constexpr int32_t kWideBit = 1 << 30;  // a tile's number: it is a wide one's

struct AttendTile {
  int64_t pre_off, tail_off;
  int32_t pre_len, p0;
  int32_t row0, rows;  // of the segment's rows
  int32_t t0, t1;
  int32_t first;   // number of the first run that takes a piece of it
  int32_t pieces;
  int32_t slot;    // first row of the partial results, `rows` per piece; -1: written out directly
  int32_t shared;  // its rows have another segment
  int32_t prefix;  // it is a shared prefix's
  // of an own tile of a shared segment: the prefix's first tile (| kWideBit) and place
  int32_t pre_tile, pre_p0;
  int32_t pad;
};

// What the second kernel joins for one row of the window and one of the group's query
// heads (sub; -1: all of them, nothing was computed): the rows from[i], from[i] + step[i],
// .. of partial results, count[i] of them, of its own segment and of its prefix.
struct alignas(16) AttendJoin {
  int32_t row, sub;
  int32_t from[2], count[2], step[2];
  int32_t empty;  // the row sees no position
  int32_t pad[3];
};

// What the plan was made for.  An attention that was captured alone runs on whatever plan its memory
// holds when it is replayed: one for other workgroups, for another buffer of pages, behind whose
// end its offsets may lie, or for more rows than this call's buffers have, is not run.
struct AttendHead {
  const int32_t* pages;
  int32_t n_rows;
  int32_t waves;  // AttendPlanDev::waves when the plan was made
  int32_t n_joins;
  int32_t pad[3];
};
__device__ inline bool plan_is_for(const AttendHead& h, const BlockWin& w, int32_t waves) {
  // (one comparison: && would wait for each of its loads in turn)
  return (((uint64_t)h.pages ^ (uint64_t)w.pages) | (uint32_t)(h.waves ^ waves) | (uint32_t)(h.n_rows > w.n_rows)) == 0;
}

// What a wave of a workgroup takes: (wide tiles, all waves the same) `rounds` whole
// tiles, one of each `stride` of them (tile_of_round), then `units` from unit `from` of tile `next` on.
// The first tile's record is here too, so that a wave has one lookup less to wait for.
struct alignas(16) AttendRun {
  AttendTile tile;
  int32_t number;  // of the runs of its kind that have units
  int32_t kind;    // 0: wide, 1: narrow
  int32_t rounds, stride;
  int32_t next, from, units;
  int32_t pad[3];
};

struct AttendPlanDev {
  AttendHead* head;
  uint32_t* flags;    // per request: PS_R_INVALID
  int32_t* table;     // hash slots: request + 1
  int32_t* least;     // per slot: the least request
  int32_t* slot_of;   // per request: its slot, -1 for none
  int32_t* members;   // per request: of the group it leads
  int32_t* base;      // per request in the order of the groups: first of its rows in the row order
  int32_t* lead;      // likewise: the place of its group's first member, -1 unshared
  int32_t* row;       // row order: row of the window
  int32_t* lim;       // positions it sees
  int32_t* todo;      // requests, later segments, with much to write
  AttendSeg* segs;    // 2 per request, in that order: prefix (first members only), own
  AttendTile* tiles[2];
  int64_t* begin[2];  // first unit of each tile
  AttendRun* runs;     // of wave w of workgroup g: waves g + w
  AttendJoin* joins;
  float* part;        // partial results: [head][slot rows][dim], weights as numerators
  float2* part_ml;    // their maxima (times scale * log2 e) and sums
  unsigned char* zeros;  // a row of q of a head
  int32_t table_mask;
  int32_t tile_cap[2];
  int32_t slot_rows;  // per head
  int32_t groups;     // workgroups per head
  int32_t n_runs;     // records of runs, at least groups * waves
  int32_t waves;      // of each
  int32_t wide_rows;  // of a wide tile, at most
};

struct AttendArgs {
  AttendPlanDev plan;
  BlockWin win;
  BlockCache cache;
  BlockRows q, out;
  float* lse;
  float scale;
  int32_t heads, ratio;
  uint32_t bt_mul, bt_shift;  // t / bt = (umulhi(t, bt_mul) + t) >> bt_shift
};

}  // namespace ps

hipError_t ps_launch_kv_write(const ps::BlockCache& c, const ps::BlockWin& w, const ps::BlockRows& k,
                              const ps::BlockRows& v, int32_t num_cus, hipStream_t s);
hipError_t ps_launch_kv_read(const ps::BlockCache& c, const ps::BlockWin& w, const ps::BlockRows& k,
                             const ps::BlockRows& v, int32_t num_cus, hipStream_t s);
hipError_t ps_launch_attend_plan(const ps::AttendPlanDev& p, const ps::BlockWin& w, int32_t ratio, uint32_t* d_flags,
                                 hipStream_t s);
hipError_t ps_launch_attend(const ps::AttendArgs& a, int32_t num_cus, hipStream_t s);
// Resident workgroups of the attention kernel per CU.
int32_t ps_attend_per_cu(int32_t dim, bool tall);
// Whether a window of `rows` rows (x query heads of a group) is cut into tall tiles.
bool ps_attend_tall(int32_t dim, int64_t rows, int32_t n_req);
