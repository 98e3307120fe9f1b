// Attention of a window's rows over their requests' chains in the block cache.

#include "ps_blocks.h"

namespace ps {

namespace {

// Whether every page that a request's context needs is one of the cache's;
// one workgroup per request.
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

// One workgroup: each row's request and the positions it sees.
__global__ __launch_bounds__(1024) void plan_rows_kernel(AttendPlanDev p, BlockWin w, uint32_t* d_flags) {
  int bad = 0;
  for (int32_t r = threadIdx.x; r < w.n_req; r += 1024) {
    const int32_t lo = w.row_off[r], hi = w.row_off[r + 1];
    bad |= lo < 0 || hi < lo || hi > w.n_rows;
  }
  bad = __syncthreads_or(bad);
  if (bad && d_flags)
    for (int32_t r = threadIdx.x; r < w.n_req; r += 1024) d_flags[r] = PS_R_INVALID;
  for (int32_t row = threadIdx.x; row < w.n_rows; row += 1024) {
    AttendRow o{0, 0, 0, -1};
    const int32_t r = bad || w.n_req == 0 ? -1 : block_row_req(w, row);
    if (r >= 0) {
      const BlockReq q = block_req(w, r);
      o.pre_off = q.pre_off;
      o.tail_off = q.tail_off;
      o.pre_len = q.pre_len;
      const int64_t lim = (int64_t)q.ctx - q.hi + row + 1;
      o.lim = p.flags[r] || lim < 0 ? 0 : (int32_t)lim;
    }
    p.rows[row] = o;
  }
}

template <bool kF16>
__device__ inline float load16(const unsigned char* p, int64_t i) {
  if (kF16) return (float)((const _Float16*)p)[i];
  return __builtin_bit_cast(float, (uint32_t)((const uint16_t*)p)[i] << 16);
}

template <bool kF16>
__device__ inline float round16(float x) {
  if (kF16) return (float)(_Float16)x;
  return (float)(__bf16)x;
}

template <bool kF16, bool kQuant>
__device__ inline float load_cache(const unsigned char* p, const uint8_t* x, int64_t at, int64_t xat) {
  if (!kQuant) return load16<kF16>(p, at);
  const float s = __builtin_bit_cast(float, (uint32_t)x[xat] << 23);
  return round16<kF16>(__builtin_amdgcn_cvt_f32_fp8((int)p[at], 0) * s);
}

// One wave per row and query head: 64 positions at a time, a lane each for
// the scores, then lanes over the head's elements for the weighted sum.
template <bool kF16, bool kQuant>
__global__ __launch_bounds__(256) void attend_kernel(AttendArgs a) {
  const int lane = threadIdx.x & 63;
  const int64_t id = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  const int32_t row = (int32_t)(id / a.heads), h = (int32_t)(id % a.heads);
  if (row >= a.win.n_rows) return;
  const AttendRow m = a.plan.rows[row];
  if (m.lim < 0) return;
  const BlockCache& c = a.cache;
  const int32_t kvh = h / (a.heads / c.heads), D = c.dim;
  const unsigned char* q = a.q.data + 2 * (row * a.q.row + h * a.q.head);
  float acc[4] = {0, 0, 0, 0}, mx = -INFINITY, l = 0;
  for (int32_t t0 = 0; t0 < m.lim; t0 += 64) {
    const int32_t n = min(64, m.lim - t0);
    int64_t at = 0, xat = 0;
    float s = -INFINITY;
    if (lane < n) {
      const int32_t t = t0 + lane, b = t / c.bt;
      const int64_t page = min((uint32_t)c.n_pages - 1u,
                               (uint32_t)a.win.pages[b < m.pre_len ? m.pre_off + b : m.tail_off + (b - m.pre_len)]);
      const int64_t r = (int64_t)kvh * c.bt + (t - b * c.bt);
      at = page * c.page_stride + r * D;
      xat = page * c.exp_stride + r;
      float d = 0;
      for (int e = 0; e < D; ++e) d += load16<kF16>(q, e) * load_cache<kF16, kQuant>(c.k, c.kx, at + e, xat);
      s = d * a.scale;
    }
    float top = s;
    for (int o = 32; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor(top, o, 64));
    const float nm = fmaxf(mx, top), safe = nm == -INFINITY ? 0.0f : nm;
    const float w = expf(s - safe), f = expf(mx - safe);
    float sum = w;
    for (int o = 32; o > 0; o >>= 1) sum += __shfl_xor(sum, o, 64);
    l = l * f + sum;
    mx = nm;
    const float wr = round16<kF16>(w);
    for (int g = 0; g < 4; ++g) acc[g] *= f;
    for (int j = 0; j < n; ++j) {
      const float pw = __shfl(wr, j, 64);
      const int64_t vat = __shfl((long long)at, j, 64), vx = __shfl((long long)xat, j, 64);
      for (int g = 0; g < 4; ++g)
        if (g * 64 + lane < D) acc[g] += pw * load_cache<kF16, kQuant>(c.v, c.vx, vat + g * 64 + lane, vx);
    }
  }
  const float inv = m.lim == 0 ? 0.0f : 1.0f / l;
  for (int g = 0; g < 4; ++g) {
    const int e = g * 64 + lane;
    if (e >= D) continue;
    const int64_t at = row * a.out.row + h * a.out.head + e;
    const float o = m.lim == 0 ? 0.0f : acc[g] * inv;
    if (kF16) ((_Float16*)a.out.data)[at] = (_Float16)o;
    else ((__bf16*)a.out.data)[at] = (__bf16)o;
  }
  if (a.lse && lane == 0) a.lse[(int64_t)row * a.heads + h] = m.lim == 0 ? -INFINITY : mx + logf(l);
}

}  // namespace

}  // namespace ps

hipError_t ps_launch_attend_plan(const ps::AttendPlanDev& p, const ps::BlockWin& w, uint32_t* d_flags, hipStream_t s) {
  if (w.n_req > 0) hipLaunchKernelGGL(ps::plan_check_kernel, dim3(w.n_req), dim3(256), 0, s, p, w, d_flags);
  hipLaunchKernelGGL(ps::plan_rows_kernel, dim3(1), dim3(1024), 0, s, p, w, d_flags);
  return hipGetLastError();
}

hipError_t ps_launch_attend(const ps::AttendArgs& a, hipStream_t s) {
  const dim3 grid((unsigned)(((int64_t)a.win.n_rows * a.heads + 3) / 4)), block(256);
  const bool f16 = a.q.dtype == PS_T_F16, quant = a.cache.dtype == PS_T_E4M3;
  if (f16 && quant) hipLaunchKernelGGL((ps::attend_kernel<true, true>), grid, block, 0, s, a);
  else if (f16) hipLaunchKernelGGL((ps::attend_kernel<true, false>), grid, block, 0, s, a);
  else if (quant) hipLaunchKernelGGL((ps::attend_kernel<false, true>), grid, block, 0, s, a);
  else hipLaunchKernelGGL((ps::attend_kernel<false, false>), grid, block, 0, s, a);
  return hipGetLastError();
}
