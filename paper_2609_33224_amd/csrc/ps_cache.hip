// The block cache's rows: quantising them as they are written, and reading
// them back.
//
// One row and head (D elements) is one group of lanes, 8 elements (16 bytes of
// a 16-bit type) each, so a wave takes 64 / (D / 8) of them and every load and
// store is one contiguous run per row and head: 2 D bytes in, D (or 2 D) out.
// Both passes are bound by that traffic, and by launch latency for a few rows.

#include "ps_blocks.h"

namespace ps {

namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));

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

// Units of work: (row, K or V, head), the head fastest, LP lanes each.
struct Unit {
  int32_t row, head;
  int which;  // 0: K, 1: V
  int32_t d;  // first element of the lane
};
template <int LP>
__device__ inline bool unit_of(const BlockWin& w, int32_t heads, Unit* u) {
  const int64_t id = ((int64_t)blockIdx.x * kBlock + threadIdx.x) / LP;
  const int64_t per_row = 2 * heads;
  const int64_t row = id / per_row;
  const int32_t rest = (int32_t)(id - row * per_row);
  u->row = (int32_t)row;
  u->which = rest >= heads;
  u->head = rest - u->which * heads;
  u->d = (threadIdx.x % LP) * 8;
  return row < w.n_rows;
}

// An e4m3 code is x / 2^e rounded once (to nearest, ties to even), with e the
// least exponent that brings the row's largest magnitude to 448 at most: a
// power of two, so that the scaling itself is exact and reading back is a
// product of 4 significant bits with a power of two.  The exponent comes from
// the bits of that magnitude: 448 = 1.75 * 2^8.
template <int LP, bool kF16, bool kQuant>
__global__ __launch_bounds__(kBlock) void write_kernel(BlockCache c, BlockWin w, BlockRows k, BlockRows v) {
  Unit u;
  if (!unit_of<LP>(w, c.heads, &u)) return;
  bool has;
  int64_t page;
  int32_t slot;
  if (!block_locate(w, u.row, &has, &page, &slot)) return;  // (the same for all lanes of the unit)
  const BlockRows& src = u.which ? v : k;
  u32x4 x = {0, 0, 0, 0};
  const bool in = u.d < c.dim;
  if (in) x = *(const u32x4*)(src.data + 2 * (u.row * src.row + u.head * src.head + u.d));
  const int64_t at = page * c.page_stride + ((int64_t)u.head * c.bt + slot) * c.dim + u.d;
  unsigned char* dst = u.which ? c.v : c.k;
  if (!kQuant) {
    if (in) *(u32x4*)(dst + 2 * at) = x;
    return;
  }
  float f[8];
  uint32_t big = 0;
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    f[j] = element<kF16>(x, j);
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
    int p = __builtin_amdgcn_cvt_pk_fp8_f32(f[4 * h], f[4 * h + 1], 0, false);
    o[h] = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(f[4 * h + 2], f[4 * h + 3], p, true);
  }
  if (in) *(u32x2*)(dst + at) = o;
  if (u.d == 0) (u.which ? c.vx : c.kx)[page * c.exp_stride + (int64_t)u.head * c.bt + slot] = (uint8_t)(e + 127);
}

template <int LP, bool kF16, bool kQuant>
__global__ __launch_bounds__(kBlock) void read_kernel(BlockCache c, BlockWin w, BlockRows k, BlockRows v) {
  Unit u;
  if (!unit_of<LP>(w, c.heads, &u)) return;
  if (u.d >= c.dim) return;
  bool has;
  int64_t page;
  int32_t slot;
  u32x4 x = {0, 0, 0, 0};
  if (block_locate(w, u.row, &has, &page, &slot)) {
    const int64_t at = page * c.page_stride + ((int64_t)u.head * c.bt + slot) * c.dim + u.d;
    const unsigned char* src = u.which ? c.v : c.k;
    if (!kQuant) {
      x = *(const u32x4*)(src + 2 * at);
    } else {
      const u32x2 p = *(const u32x2*)(src + at);
      const uint32_t ex = (u.which ? c.vx : c.kx)[page * c.exp_stride + (int64_t)u.head * c.bt + slot];
      const float s = __builtin_bit_cast(float, ex << 23);
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        if (kF16) {
          x[2 * h] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8((int)p[h], s, false));
          x[2 * h + 1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8((int)p[h], s, true));
        } else {
          x[2 * h] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((int)p[h], s, false));
          x[2 * h + 1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((int)p[h], s, true));
        }
      }
    }
  }
  const BlockRows& dst = u.which ? v : k;
  if (has) *(u32x4*)(dst.data + 2 * (u.row * dst.row + u.head * dst.head + u.d)) = x;
}

template <int LP>
hipError_t launch(bool write, const BlockCache& c, const BlockWin& w, const BlockRows& k, const BlockRows& v,
                  hipStream_t s) {
  const int64_t lanes = (int64_t)w.n_rows * 2 * c.heads * LP;
  const dim3 grid((unsigned)((lanes + kBlock - 1) / kBlock)), block(kBlock);
  const bool f16 = k.dtype == PS_T_F16, quant = c.dtype == PS_T_E4M3;
#define PS_ROWS(F, Q)                                                                    \
  do {                                                                                   \
    if (write) hipLaunchKernelGGL((write_kernel<LP, F, Q>), grid, block, 0, s, c, w, k, v); \
    else hipLaunchKernelGGL((read_kernel<LP, F, Q>), grid, block, 0, s, c, w, k, v);        \
  } while (0)
  if (!quant) PS_ROWS(false, false);  // moved as they are
  else if (f16) PS_ROWS(true, true);
  else PS_ROWS(false, true);
#undef PS_ROWS
  return hipGetLastError();
}

hipError_t rows(bool write, const BlockCache& c, const BlockWin& w, const BlockRows& k, const BlockRows& v,
                hipStream_t s) {
  if (c.dim <= 32) return launch<4>(write, c, w, k, v, s);
  if (c.dim <= 64) return launch<8>(write, c, w, k, v, s);
  if (c.dim <= 128) return launch<16>(write, c, w, k, v, s);
  return launch<32>(write, c, w, k, v, s);
}

}  // namespace

}  // namespace ps

hipError_t ps_launch_kv_write(const ps::BlockCache& c, const ps::BlockWin& w, const ps::BlockRows& k,
                              const ps::BlockRows& v, hipStream_t s) {
  return ps::rows(true, c, w, k, v, s);
}

hipError_t ps_launch_kv_read(const ps::BlockCache& c, const ps::BlockWin& w, const ps::BlockRows& k,
                             const ps::BlockRows& v, hipStream_t s) {
  return ps::rows(false, c, w, k, v, s);
}
