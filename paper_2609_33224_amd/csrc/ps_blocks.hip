// Entry points of the block cache and its attention: argument checks, plan
// memory and launches.

#include <algorithm>
#include <cmath>
#include <new>

#include "ps_blocks.h"
#include "ps_context.h"

struct ps_attend_plan {
  ps_ctx* ctx = nullptr;
  ps_attend_plan* next = nullptr;
  int32_t heads = 0, kv_heads = 0, dim = 0, bt = 0, max_req = 0, max_rows = 0;
  AttendPlanDev dev{};
  bool planned = false;
  BlockWin win{};  // of the last ps_attend_plan_dev
  int32_t ratio() const { return heads / kv_heads; }
};

namespace {

bool aligned16(const void* p) { return ((uintptr_t)p & 15) == 0; }

ps_status check_shape(ps_ctx* c, int32_t kv_heads, int32_t dim, int32_t bt) {
  if (kv_heads < 1 || kv_heads > PS_MAX_KV_HEADS)
    return fail(c, PS_E_RANGE, "n_kv_heads %d outside [1, %d]", kv_heads, PS_MAX_KV_HEADS);
  if (dim < 16 || dim > PS_MAX_HEAD_DIM || dim % 16)
    return fail(c, PS_E_RANGE, "head_dim %d is not a multiple of 16 in [16, %d]", dim, PS_MAX_HEAD_DIM);
  if (bt < 1 || bt > PS_MAX_BLOCK_TOKENS)
    return fail(c, PS_E_RANGE, "block_tokens %d outside [1, %d]", bt, PS_MAX_BLOCK_TOKENS);
  return PS_OK;
}

ps_status check_cache(ps_ctx* c, const ps_kv_cache* k) {
  if (!k) return fail(c, PS_E_INVAL, "cache is NULL");
  ps_status st = check_shape(c, k->n_kv_heads, k->head_dim, k->block_tokens);
  if (st != PS_OK) return st;
  if (k->dtype != PS_T_BF16 && k->dtype != PS_T_F16 && k->dtype != PS_T_E4M3)
    return fail(c, PS_E_INVAL, "unknown cache type %d", k->dtype);
  if (k->n_pages < 0 || k->n_pages > INT32_MAX) return fail(c, PS_E_RANGE, "n_pages outside [0, 2^31)");
  const int64_t slots = (int64_t)k->n_kv_heads * k->block_tokens;
  const int64_t esz = k->dtype == PS_T_E4M3 ? 1 : 2;
  if (k->page_stride < slots * k->head_dim || k->page_stride > (int64_t)1 << 40 || k->page_stride * esz % 16)
    return fail(c, PS_E_INVAL, "page_stride below a page's elements or not a multiple of 16 bytes");
  if (k->n_pages > 0 && (!k->k || !k->v)) return fail(c, PS_E_INVAL, "cache buffer is NULL");
  if (!aligned16(k->k) || !aligned16(k->v)) return fail(c, PS_E_INVAL, "cache buffer is not 16-byte aligned");
  if (k->dtype == PS_T_E4M3) {
    if (k->n_pages > 0 && (!k->k_exp || !k->v_exp)) return fail(c, PS_E_INVAL, "exponent buffer is NULL");
    if (k->exp_page_stride < slots || k->exp_page_stride > (int64_t)1 << 40)
      return fail(c, PS_E_INVAL, "exp_page_stride below a page's rows");
  }
  return PS_OK;
}

ps_status check_window(ps_ctx* c, const ps_kv_window* w) {
  if (!w) return fail(c, PS_E_INVAL, "window is NULL");
  if (w->n_req < 0 || w->pages_len < 0) return fail(c, PS_E_INVAL, "negative n_req or pages_len");
  if (w->n_rows < 0 || w->n_rows > PS_MAX_ROWS)
    return fail(c, PS_E_RANGE, "n_rows %d outside [0, %d]", w->n_rows, PS_MAX_ROWS);
  if (w->n_pages < 0 || w->n_pages > INT32_MAX) return fail(c, PS_E_RANGE, "n_pages outside [0, 2^31)");
  if (w->n_req > 0 && (!w->reqs || !w->ctx_tok || !w->row_off || (w->pages_len > 0 && !w->pages)))
    return fail(c, PS_E_INVAL, "device buffer is NULL");
  return PS_OK;
}

// Whether two of n_rows x heads runs of dim elements share an element: two that are dr rows and dh heads
// apart do where |dr row_stride + dh head_stride| < dim.
bool rows_overlap(const ps_rows& r, int64_t n_rows, int32_t heads, int32_t dim) {
  const int64_t rs = r.row_stride, hs = r.head_stride;
  if ((n_rows > 1 && rs < dim) || (heads > 1 && hs < dim)) return true;
  if (n_rows <= 1 || heads <= 1) return false;
  // a row's heads between its start and the next one's, or a head's rows likewise
  if (rs >= (heads - 1) * hs + dim || hs >= (n_rows - 1) * rs + dim) return false;
  for (int64_t dh = 1; dh < heads; ++dh) {
    const int64_t dr = dh * hs / rs;  // as many rows back, or one more
    if ((dr < n_rows && dh * hs - dr * rs < dim) || (dr + 1 < n_rows && (dr + 1) * rs - dh * hs < dim)) return true;
  }
  return false;
}

// written: n_rows rows of `heads` heads are (none where that is not known yet).
ps_status check_rows(ps_ctx* c, const ps_rows* r, const char* what, bool written, int64_t n_rows, int32_t heads,
                     int32_t dim) {
  if (!r || !r->data) return fail(c, PS_E_INVAL, "%s is NULL", what);
  if (r->dtype != PS_T_BF16 && r->dtype != PS_T_F16) return fail(c, PS_E_INVAL, "%s is not of a 16-bit type", what);
  if (!aligned16(r->data)) return fail(c, PS_E_INVAL, "%s is not 16-byte aligned", what);
  if (r->row_stride % 8 || r->head_stride % 8 || r->row_stride < 0 || r->head_stride < 0 ||
      r->row_stride > (int64_t)1 << 40 || r->head_stride > (int64_t)1 << 40)
    return fail(c, PS_E_INVAL, "strides of %s are not multiples of 8 in [0, 2^40]", what);
  if (written && (r->row_stride < dim || r->head_stride < dim || rows_overlap(*r, n_rows, heads, dim)))
    return fail(c, PS_E_INVAL, "rows of %s overlap", what);
  return PS_OK;
}

BlockWin dev_win(const ps_kv_window& w, int32_t bt) {
  return BlockWin{w.pages, w.reqs, w.ctx_tok, w.row_off, w.pages_len, w.n_pages, w.n_req, w.n_rows, bt};
}

BlockCache dev_cache(const ps_kv_cache& k) {
  return BlockCache{(unsigned char*)k.k, (unsigned char*)k.v, k.k_exp, k.v_exp, k.page_stride, k.exp_page_stride,
                    k.n_pages, k.n_kv_heads, k.head_dim, k.block_tokens, k.dtype};
}

BlockRows dev_rows(const ps_rows& r) {
  return BlockRows{(unsigned char*)r.data, r.row_stride, r.head_stride, r.dtype};
}

ps_status kv_rows(ps_ctx* c, bool write, const ps_kv_cache* cache, const ps_kv_window* w, const ps_rows* k,
                  const ps_rows* v, void* stream) {
  ps_status st;
  if ((st = check_cache(c, cache)) != PS_OK || (st = check_window(c, w)) != PS_OK) return st;
  if (w->n_pages > cache->n_pages) return fail(c, PS_E_INVAL, "the window names more pages than the cache has");
  const bool none = w->n_req == 0 || w->n_rows == 0;
  if (!none) {
    if ((st = check_rows(c, k, "k", !write, w->n_rows, cache->n_kv_heads, cache->head_dim)) != PS_OK ||
        (st = check_rows(c, v, "v", !write, w->n_rows, cache->n_kv_heads, cache->head_dim)) != PS_OK)
      return st;
    if (k->dtype != v->dtype || (cache->dtype != PS_T_E4M3 && k->dtype != cache->dtype))
      return fail(c, PS_E_INVAL, "k, v and the cache differ in type");
  }
  if (!c) return fail(nullptr, PS_E_INVAL, "ctx is NULL");
  if (none) return PS_OK;
  DeviceScope ds(c->device);
  const BlockWin dw = dev_win(*w, cache->block_tokens);
  HIP_TRY(c, (write ? ps_launch_kv_write : ps_launch_kv_read)(dev_cache(*cache), dw, dev_rows(*k), dev_rows(*v),
                                                              c->num_cus, (hipStream_t)stream));
  return PS_OK;
}

// Every buffer of a plan: the pointer and its bytes.
template <class F>
hipError_t each_buffer(ps_attend_plan* p, F f) {
  AttendPlanDev& d = p->dev;
  const size_t n = p->max_req, rows = p->max_rows, part = (size_t)d.slot_rows * p->kv_heads;
  hipError_t e = hipSuccess;
  auto one = [&](auto*& ptr, size_t count) {
    if (e == hipSuccess) e = f(ptr, count * sizeof(*ptr));
  };
  one(d.head, 1);
  one(d.flags, n);
  one(d.table, (size_t)d.table_mask + 1);
  one(d.least, (size_t)d.table_mask + 1);
  one(d.slot_of, n);
  one(d.members, n);
  one(d.base, n);
  one(d.lead, n);
  one(d.row, rows);
  one(d.lim, rows);
  one(d.todo, 2 * n);
  one(d.segs, 2 * n);
  for (int k = 0; k < 2; ++k) {
    one(d.tiles[k], d.tile_cap[k]);
    one(d.begin[k], d.tile_cap[k]);
  }
  // (a row with partial results each, or a place of empty rows: twice where two tiles have some)
  one(d.runs, d.n_runs);
  one(d.joins, (size_t)d.slot_rows + rows + d.tile_cap[0]);
  one(d.part, part * p->dim);
  one(d.part_ml, part);
  one(d.zeros, 2 * PS_MAX_HEAD_DIM);
  return e;
}

void release(ps_attend_plan* p) {
  (void)each_buffer(p, [&](auto*& ptr, size_t) {
    p->ctx->pool.release(ptr);
    return hipSuccess;
  });
}

// The workgroups of a head, and the tiles they take.
void shape_plan(ps_attend_plan* p, int32_t num_cus, bool tall) {
  AttendPlanDev& d = p->dev;
  d.waves = tall ? kTallWaves : kWideWaves;
  d.wide_rows = tall ? kTallRows : kWideRows;
  const int32_t per_cu = ps_attend_per_cu(p->dim, tall);
  // (two at least, of both kinds one; the plan's kernel has a thread for each)
  d.groups = std::min(std::max(num_cus * per_cu / p->kv_heads, 2 * per_cu), per_cu * kMaxGroups / 2);
}

// Sizes that hold whatever window of at most max_req requests and max_rows rows, cut into
// tall tiles or not: those are twice as high, taken by at most half as many workgroups of
// twice as many waves.
void size_plan(ps_attend_plan* p, int32_t num_cus) {
  AttendPlanDev& d = p->dev;
  const int64_t n = p->max_req, rows = (int64_t)p->max_rows * p->ratio();
  int32_t slots = 2;
  while (slots < 2 * n) slots *= 2;
  d.table_mask = slots - 1;
  // a wide tile is full but for the last one of each segment, and a row lies in two segments at most
  d.tile_cap[0] = (int32_t)(2 * n + 2 * rows / kWideRows + 1);
  d.tile_cap[1] = (int32_t)(2 * n + 1);
  shape_plan(p, num_cus, false);
  d.n_runs = d.groups * d.waves;
  // Of partial results: each row of a shared segment once, in both of its segments;
  // and the pieces of tiles that are cut, of which there are fewer than twice
  // as many as workgroups or waves that take them.
  const int64_t shared = std::min(rows, n * std::max(kShareMaxRows, p->ratio()));
  d.slot_rows = (int32_t)std::min<int64_t>(2 * shared + 2 * (int64_t)d.groups * (kWideRows + kWideWaves * kNarrowRows), INT32_MAX);
}

}  // namespace

void ps::free_plans(ps_ctx* c) {
  while (c->plans) {
    ps_attend_plan* p = c->plans;
    c->plans = p->next;
    release(p);
    delete p;
  }
}

extern "C" {

ps_status ps_kv_write_dev(ps_ctx* c, const ps_kv_cache* cache, const ps_kv_window* window, const ps_rows* k,
                          const ps_rows* v, void* hip_stream) {
  return kv_rows(c, true, cache, window, k, v, hip_stream);
}

ps_status ps_kv_read_dev(ps_ctx* c, const ps_kv_cache* cache, const ps_kv_window* window, const ps_rows* k,
                         const ps_rows* v, void* hip_stream) {
  return kv_rows(c, false, cache, window, k, v, hip_stream);
}

ps_status ps_attend_plan_create(ps_ctx* c, int32_t n_heads, int32_t n_kv_heads, int32_t head_dim,
                                int32_t block_tokens, int32_t max_req, int32_t max_rows, ps_attend_plan** out) {
  if (!out) return fail(c, PS_E_INVAL, "out is NULL");
  *out = nullptr;
  ps_status st = check_shape(c, n_kv_heads, head_dim, block_tokens);
  if (st != PS_OK) return st;
  if (n_heads < 1 || n_heads > PS_MAX_HEADS || n_heads % n_kv_heads)
    return fail(c, PS_E_RANGE, "n_heads %d is not a multiple of n_kv_heads in [1, %d]", n_heads, PS_MAX_HEADS);
  if (max_req < 0 || max_req > PS_MAX_WINDOW_REQ)
    return fail(c, PS_E_RANGE, "max_req %d outside [0, %d]", max_req, PS_MAX_WINDOW_REQ);
  if (max_rows < 0 || max_rows > PS_MAX_ROWS)
    return fail(c, PS_E_RANGE, "max_rows %d outside [0, %d]", max_rows, PS_MAX_ROWS);
  if (!c) return fail(nullptr, PS_E_INVAL, "ctx is NULL");
  DeviceScope ds(c->device);
  ps_attend_plan* p = new (std::nothrow) ps_attend_plan();
  if (!p) return fail(c, PS_E_NOMEM, "host allocation failed");
  p->ctx = c;
  p->heads = n_heads;
  p->kv_heads = n_kv_heads;
  p->dim = head_dim;
  p->bt = block_tokens;
  p->max_req = max_req;
  p->max_rows = max_rows;
  size_plan(p, c->num_cus);
  hipError_t e = each_buffer(p, [&](auto*& ptr, size_t bytes) { return c->pool.grow(&ptr, bytes); });
  // (no window's plan: an attention that runs before the first one does nothing)
  if (e == hipSuccess) e = hipMemsetAsync(p->dev.head, 0, sizeof(AttendHead), c->stream);
  if (e == hipSuccess) e = hipMemsetAsync(p->dev.zeros, 0, 2 * PS_MAX_HEAD_DIM, c->stream);
  if (e == hipSuccess) e = hipStreamSynchronize(c->stream);
  if (e != hipSuccess) {
    release(p);
    delete p;
    HIP_TRY(c, e);
  }
  p->next = c->plans;
  c->plans = p;
  *out = p;
  return PS_OK;
}

ps_status ps_attend_plan_destroy(ps_attend_plan* p) {
  if (!p) return PS_OK;
  DeviceScope ds(p->ctx->device);
  // (freeing is refused to a thread that captures, and ends the capture, unless it says that it may)
  hipStreamCaptureMode mode = hipStreamCaptureModeRelaxed;
  const bool relaxed = hipThreadExchangeStreamCaptureMode(&mode) == hipSuccess;
  for (ps_attend_plan** at = &p->ctx->plans; *at; at = &(*at)->next)
    if (*at == p) {
      *at = p->next;
      break;
    }
  release(p);
  if (relaxed) (void)hipThreadExchangeStreamCaptureMode(&mode);
  delete p;
  return PS_OK;
}

ps_status ps_attend_plan_dev(ps_attend_plan* p, const ps_kv_window* window, uint32_t* d_flags, void* hip_stream) {
  ps_ctx* c = p ? p->ctx : nullptr;
  ps_status st = check_window(c, window);
  if (st != PS_OK) return st;
  if (!p) return fail(c, PS_E_INVAL, "plan is NULL");
  if (window->n_req > p->max_req || window->n_rows > p->max_rows)
    return fail(c, PS_E_RANGE, "window of %d requests, %d rows: the plan takes %d, %d", window->n_req, window->n_rows,
                p->max_req, p->max_rows);
  DeviceScope ds(c->device);
  const BlockWin w = dev_win(*window, p->bt);
  p->planned = false;  // (until the launches have succeeded)
  shape_plan(p, c->num_cus, ps_attend_tall(p->dim, (int64_t)w.n_rows * p->ratio(), w.n_req));
  if (w.n_req > 0) HIP_TRY(c, ps_launch_attend_plan(p->dev, w, p->ratio(), d_flags, (hipStream_t)hip_stream));
  p->win = w;
  p->planned = true;
  return PS_OK;
}

ps_status ps_attend_window_dev(ps_attend_plan* p, const ps_kv_cache* cache, const ps_rows* q, const ps_rows* out,
                               float* lse, float scale, void* hip_stream) {
  ps_ctx* c = p ? p->ctx : nullptr;
  ps_status st = check_cache(c, cache);
  if (st != PS_OK) return st;
  if (!std::isfinite(scale * 1.44269504088896341f))  // (it multiplies powers of two)
    return fail(c, PS_E_INVAL, "scale is not finite, or times log2 e it is not");
  const bool none = p && p->planned && (p->win.n_req == 0 || p->win.n_rows == 0);
  if (!none) {
    if ((st = check_rows(c, q, "q", false, 0, 0, cache->head_dim)) != PS_OK ||
        (st = check_rows(c, out, "out", true, p ? p->win.n_rows : 0, p ? p->heads : 0, cache->head_dim)) != PS_OK)
      return st;
    if (q->dtype != out->dtype || (cache->dtype != PS_T_E4M3 && q->dtype != cache->dtype))
      return fail(c, PS_E_INVAL, "q, out and the cache differ in type");
  }
  if (!p) return fail(c, PS_E_INVAL, "plan is NULL");
  if (!p->planned) return fail(c, PS_E_STATE, "ps_attend_plan_dev has not succeeded yet");
  if (cache->n_kv_heads != p->kv_heads || cache->head_dim != p->dim || cache->block_tokens != p->bt)
    return fail(c, PS_E_INVAL, "the plan is for %d heads of %d, blocks of %d", p->kv_heads, p->dim, p->bt);
  if (p->win.n_pages > cache->n_pages) return fail(c, PS_E_INVAL, "the window names more pages than the cache has");
  if (none) return PS_OK;
  DeviceScope ds(c->device);
  AttendArgs a{p->dev, p->win, dev_cache(*cache), dev_rows(*q), dev_rows(*out), lse, scale, p->heads, p->ratio(), 0, 0};
  if (scale == 0) {
    // a q of zeros: the kernel's scale multiplies infinities, where scores are masked
    a.scale = 1;
    a.q.data = p->dev.zeros;
    a.q.row = a.q.head = 0;
  }
  while ((1 << a.bt_shift) < p->bt) ++a.bt_shift;
  a.bt_mul = (uint32_t)(((uint64_t)((1 << a.bt_shift) - p->bt) << 32) / p->bt + 1);
  HIP_TRY(c, ps_launch_attend(a, c->num_cus, (hipStream_t)hip_stream));
  return PS_OK;
}

// For the tests (not in packserve.h): the check of rows that are written.
int32_t ps_test_rows_overlap(const ps_rows* r, int64_t n_rows, int32_t heads, int32_t dim) {
  return rows_overlap(*r, n_rows, heads, dim);
}

// For the tests (not in packserve.h): where the cache calls look for a row, by
// the same code, over a window in host memory.  Returns 0 for a row of no
// request, 1 for a row without a place, 2 and *page, *slot otherwise.
int32_t ps_test_block_locate(const ps_kv_window* w, int32_t block_tokens, int32_t row, int64_t* page, int32_t* slot) {
  bool has = false;
  const BlockWin win = dev_win(*w, block_tokens);
  const bool at = block_locate(win, row, block_row_req(win, row), &has, page, slot);
  return at ? 2 : has ? 1 : 0;
}

}  // extern "C"
