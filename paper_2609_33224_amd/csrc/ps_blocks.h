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
         q.ctx <= ((int64_t)d.pre_len + d.tail_len) * w.bt;
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

// Where row `row` of the window lies: its page and slot; false where it has
// none.  *has_req: whether a request claims the row.
__host__ __device__ inline bool block_locate(const BlockWin& w, int32_t row, bool* has_req, int64_t* page,
                                             int32_t* slot) {
  const int32_t r = block_row_req(w, row);
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

// What the attention of one row needs.
struct AttendRow {
  int64_t pre_off, tail_off;
  int32_t pre_len;
  int32_t lim;  // positions it sees; 0: none, -1: a row of no request
};

struct AttendPlanDev {
  AttendRow* rows;
  uint32_t* flags;  // per request, PS_R_INVALID
};

struct AttendArgs {
  AttendPlanDev plan;
  BlockWin win;
  BlockCache cache;
  BlockRows q, out;
  float* lse;
  float scale;
  int32_t heads;
};

}  // namespace ps

hipError_t ps_launch_kv_write(const ps::BlockCache& c, const ps::BlockWin& w, const ps::BlockRows& k,
                              const ps::BlockRows& v, hipStream_t s);
hipError_t ps_launch_kv_read(const ps::BlockCache& c, const ps::BlockWin& w, const ps::BlockRows& k,
                             const ps::BlockRows& v, hipStream_t s);
hipError_t ps_launch_attend_plan(const ps::AttendPlanDev& p, const ps::BlockWin& w, uint32_t* d_flags, hipStream_t s);
hipError_t ps_launch_attend(const ps::AttendArgs& a, hipStream_t s);
