// The block cache's rows: quantising them as they are written, and reading
// them back.
//
// One row and head (D elements) is one group of lanes, 8 elements (16 bytes of
// a 16-bit type) each, so a wave takes 64 / (D / 8) of them and every load and
// store is one contiguous run per row and head: 2 D bytes in, D (or 2 D) out.
// Both passes are bound by that traffic, and by launch latency for a few rows.

#include <algorithm>

#include "ps_blocks.h"

namespace ps {

namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

constexpr int kBlock = 256;

// Element j of 8 packed 16-bit values.
template <bool kF16>
__device__ inline float element(const u32x4& x, int j) {
  const uint32_t w = x[j >> 1];
  if (kF16) {
    const uint16_t h = (uint16_t)(j & 1 ? w >> 16 : w);
    return (float)__builtin_bit_cast(_Float16, h);
  }
  return __builtin_bit_cast(float, j & 1 ? w & 0xFFFF0000u : w << 16);
}

// A wave takes `per` rows (kMaxPer at most): a lane each finds where they lie, and the
// wave then moves their units (a head's K or V of a row, LP lanes), several
// steps of 64 lanes at a time, so that the lookups' latency is paid once per wave and several
// loads are in flight.
constexpr int kMaxPer = 8;
constexpr int kWriteAtOnce = 4, kReadAtOnce = 8;  // (the other way round: 93 -> 108 us and 132 -> 146 us)

struct Place {
  int64_t page;
  int32_t slot;
  int32_t state;  // 0: no request's, 1: without a place, 2: in the page
};

struct Unit {
  int64_t at, xat;  // in the cache: first element of the lane, exponent of the row
  int64_t row;
  int32_t head, d, state;
  bool v;
};

// The lane's unit of step `step`; state 0 where there is none.
template <int LP>
__device__ inline Unit unit_of(const BlockCache& c, const Place& mine, int32_t row0, int32_t per, int32_t step) {
  const int lane = threadIdx.x & 63;
  const int32_t id = (step * 64 + lane) / LP, row = id / (2 * c.heads), rest = id - row * 2 * c.heads;
  const int from = row < per ? row : 0;
  Unit u;
  u.state = __shfl(mine.state, from, 64);
  const int64_t page = __shfl((long long)mine.page, from, 64);
  const int32_t slot = __shfl(mine.slot, from, 64);
  u.v = rest >= c.heads;
  u.head = rest - (u.v ? c.heads : 0);
  u.row = row0 + row;
  u.d = (lane % LP) * 8;
  const int32_t r = u.head * c.bt + slot;
  u.at = page * c.page_stride + (int64_t)r * c.dim + u.d;
  u.xat = page * c.exp_stride + r;
  if (row >= per) u.state = 0;
  return u;
}

// The request of row row0 + lane, for the first `per` lanes (block_row_req, by the wave:
// it looks at 64 offsets at a time, so that a window of 4,096 requests takes two
// rounds where a search by halves takes twelve).
__device__ inline int32_t rows_req(const BlockWin& w, int32_t row0, int32_t per) {
  const int lane = threadIdx.x & 63;
  int32_t a = 0, b = w.n_req;  // the last request that begins at or before row0 is in [a, b)
  while (b - a > 64) {
    const int32_t step = (b - a + 63) / 64, at = a + lane * step;
    const uint64_t hit = __ballot(at < b && w.row_off[at] <= row0);
    // (offsets that ascend make it a prefix; any other answer is checked below)
    const int32_t last = hit ? 63 - __builtin_clzll(hit) : 0;
    a += last * step;
    b = min(b, a + step);
  }
  // of 64 requests from there on: how many begin at or before each row
  const int32_t off = a + lane < w.n_req ? w.row_off[a + lane] : INT32_MAX;
  int32_t r = -1;
  for (int32_t i = 0; i < per; ++i) {
    const uint64_t hit = __ballot(a + lane < w.n_req && off <= row0 + i);
    if (lane == i) r = hit >> 63 ? -2 : hit ? a + 63 - __builtin_clzll(hit) : -1;  // -2: maybe a later one
  }
  if (lane >= per || row0 + lane >= w.n_rows) return -1;
  if (r == -2) return block_row_req(w, row0 + lane);
  return r >= 0 && w.row_off[r] <= row0 + lane && row0 + lane < w.row_off[r + 1] ? r : -1;
}

__device__ inline Place place_of(const BlockWin& w, int32_t row0, int32_t per) {
  const int lane = threadIdx.x & 63;
  Place p{0, 0, 0};
  const int32_t r = rows_req(w, row0, per);
  if (lane < per && row0 + lane < w.n_rows) {
    bool has;
    const bool in = block_locate(w, row0 + lane, r, &has, &p.page, &p.slot);
    p.state = in ? 2 : has ? 1 : 0;
    if (!in) {
      p.page = 0;
      p.slot = 0;
    }
  }
  return p;
}

// An e4m3 code is x / 2^e rounded once (to nearest, ties to even), with e the
// least exponent that brings the row's largest magnitude to 448 at most: a
// power of two, so that the scaling itself is exact and reading back is a
// product of 4 significant bits with a power of two.  The exponent comes from
// the bits of that magnitude: 448 = 1.75 * 2^8.
template <int LP, bool kF16, bool kQuant>
__global__ __launch_bounds__(kBlock) void write_kernel(BlockCache c, BlockWin w, BlockRows k, BlockRows v, int32_t per) {
  const int64_t first = ((int64_t)blockIdx.x * (kBlock / 64) + (threadIdx.x >> 6)) * per;
  if (first >= w.n_rows) return;
  const int32_t row0 = (int32_t)first, steps = (per * 2 * c.heads * LP + 63) / 64;
  const Place mine = place_of(w, row0, per);
  for (int32_t s0 = 0; s0 < steps; s0 += kWriteAtOnce) {
    Unit u[kWriteAtOnce];
    u32x4 x[kWriteAtOnce];
#pragma unroll
    for (int i = 0; i < kWriteAtOnce; ++i) {
      u[i] = unit_of<LP>(c, mine, row0, per, s0 + i);
      x[i] = u32x4{0, 0, 0, 0};
      const BlockRows& src = u[i].v ? v : k;
      if (u[i].state == 2 && u[i].d < c.dim)
        x[i] = *(const u32x4*)(src.data + 2 * (u[i].row * src.row + u[i].head * src.head + u[i].d));
    }
#pragma unroll
    for (int i = 0; i < kWriteAtOnce; ++i) {
      const bool put = u[i].state == 2 && u[i].d < c.dim;
      unsigned char* dst = u[i].v ? c.v : c.k;
      if (!kQuant) {
        if (put) *(u32x4*)(dst + 2 * u[i].at) = x[i];
        continue;
      }
      float f[8];
      uint32_t big = 0;
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        f[j] = element<kF16>(x[i], j);
        const uint32_t a = __builtin_bit_cast(uint32_t, f[j]) & 0x7FFFFFFFu;
        big = max(big, a < 0x7F800000u ? a : 0u);
      }
#pragma unroll
      for (int o = LP / 2; o > 0; o >>= 1) big = max(big, (uint32_t)__shfl_xor((int)big, o, 64));
      const int e = max((int)(big >> 23) - 127 - 8 + ((big & 0x7FFFFFu) > 0x600000u ? 1 : 0), -126);
      const float s = __builtin_bit_cast(float, (uint32_t)(127 - e) << 23);
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const float y = f[j] * s;
        f[j] = y > 448.0f ? 448.0f : y < -448.0f ? -448.0f : y;  // (infinities; NaN stays)
      }
      u32x2 o;
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int p = __builtin_amdgcn_cvt_pk_fp8_f32(f[4 * h], f[4 * h + 1], 0, false);
        o[h] = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(f[4 * h + 2], f[4 * h + 3], p, true);
      }
      if (put) {
        *(u32x2*)(dst + u[i].at) = o;
        if (u[i].d == 0) (u[i].v ? c.vx : c.kx)[u[i].xat] = (uint8_t)(e + 127);
      }
    }
  }
}

template <int LP, bool kF16, bool kQuant>
__global__ __launch_bounds__(kBlock) void read_kernel(BlockCache c, BlockWin w, BlockRows k, BlockRows v, int32_t per) {
  const int64_t first = ((int64_t)blockIdx.x * (kBlock / 64) + (threadIdx.x >> 6)) * per;
  if (first >= w.n_rows) return;
  const int32_t row0 = (int32_t)first, steps = (per * 2 * c.heads * LP + 63) / 64;
  const Place mine = place_of(w, row0, per);
  for (int32_t s0 = 0; s0 < steps; s0 += kReadAtOnce) {
    Unit u[kReadAtOnce];
    u32x4 x[kReadAtOnce];
    uint32_t ex[kReadAtOnce];
#pragma unroll
    for (int i = 0; i < kReadAtOnce; ++i) {
      u[i] = unit_of<LP>(c, mine, row0, per, s0 + i);
      x[i] = u32x4{0, 0, 0, 0};
      ex[i] = 127;
      if (u[i].state == 2 && u[i].d < c.dim) {
        const unsigned char* src = u[i].v ? c.v : c.k;
        if (kQuant) {
          const u32x2 y = *(const u32x2*)(src + u[i].at);
          x[i][0] = y[0];
          x[i][1] = y[1];
          ex[i] = (u[i].v ? c.vx : c.kx)[u[i].xat];
        } else {
          x[i] = *(const u32x4*)(src + 2 * u[i].at);
        }
      }
    }
#pragma unroll
    for (int i = 0; i < kReadAtOnce; ++i) {
      u32x4 o = x[i];
      if (kQuant) {
        const float s = __builtin_bit_cast(float, ex[i] << 23);
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const int p = (int)x[i][h];
          if (kF16) {
            o[2 * h] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(p, s, false));
            o[2 * h + 1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(p, s, true));
          } else {
            o[2 * h] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(p, s, false));
            o[2 * h + 1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(p, s, true));
          }
        }
      }
      const BlockRows& dst = u[i].v ? v : k;
      if (u[i].state > 0 && u[i].d < c.dim)
        __builtin_nontemporal_store(o, (u32x4*)(dst.data + 2 * (u[i].row * dst.row + u[i].head * dst.head + u[i].d)));  // (132 -> 124 us)
    }
  }
}

template <int LP>
hipError_t launch(bool write, const BlockCache& c, const BlockWin& w, const BlockRows& k, const BlockRows& v,
                  int32_t num_cus, hipStream_t s) {
  // one row a wave until every CU has 16 waves, then more: their lookups go side by side
  const int32_t per = (int32_t)std::min<int64_t>(kMaxPer, std::max<int64_t>(1, w.n_rows / (16 * num_cus)));
  const int64_t waves = ((int64_t)w.n_rows + per - 1) / per;
  const dim3 grid((unsigned)((waves + kBlock / 64 - 1) / (kBlock / 64))), block(kBlock);
  const bool f16 = k.dtype == PS_T_F16, quant = c.dtype == PS_T_E4M3;
#define PS_ROWS(F, Q)                                                                            \
  do {                                                                                           \
    if (write) hipLaunchKernelGGL((write_kernel<LP, F, Q>), grid, block, 0, s, c, w, k, v, per); \
    else hipLaunchKernelGGL((read_kernel<LP, F, Q>), grid, block, 0, s, c, w, k, v, per);        \
  } while (0)
  if (!quant) PS_ROWS(false, false);  // moved as they are
  else if (f16) PS_ROWS(true, true);
  else PS_ROWS(false, true);
#undef PS_ROWS
  return hipGetLastError();
}

hipError_t rows(bool write, const BlockCache& c, const BlockWin& w, const BlockRows& k, const BlockRows& v,
                int32_t num_cus, hipStream_t s) {
  if (c.dim <= 32) return launch<4>(write, c, w, k, v, num_cus, s);
  if (c.dim <= 64) return launch<8>(write, c, w, k, v, num_cus, s);
  if (c.dim <= 128) return launch<16>(write, c, w, k, v, num_cus, s);
  return launch<32>(write, c, w, k, v, num_cus, s);
}

}  // namespace

}  // namespace ps

hipError_t ps_launch_kv_write(const ps::BlockCache& c, const ps::BlockWin& w, const ps::BlockRows& k,
                              const ps::BlockRows& v, int32_t num_cus, hipStream_t s) {
  return ps::rows(true, c, w, k, v, num_cus, s);
}

hipError_t ps_launch_kv_read(const ps::BlockCache& c, const ps::BlockWin& w, const ps::BlockRows& k,
                             const ps::BlockRows& v, int32_t num_cus, hipStream_t s) {
  return ps::rows(false, c, w, k, v, num_cus, s);
}
