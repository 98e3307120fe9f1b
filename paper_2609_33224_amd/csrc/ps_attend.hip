// Attention of a window's rows over their requests' chains in the block cache.
//
// One pass over the keys and values with the running maximum and sum of the
// softmax, on the matrix cores: S^T = K Q^T (rows: positions, columns: rows of
// the tile), P = exp2(S c - m c) with c = scale log2 e, O^T += V^T P^T.  In
// this orientation a lane's column is one row of the window in both products, so the
// maximum, the sum and the rescaling are the lane's own, and its weights are
// in the place where the second product takes them: the k index of a matrix
// product may be permuted, and is, so that it names the positions that the lane holds.
//
// A workgroup takes an equal run of the units of its head's wide tiles (AttendPlanDev),
// then each of its waves one of the narrow tiles.
//  - A narrow tile (16 rows at most: the rows of one request that decodes) is
//    bound by the bytes of its keys and values, so each wave takes a run of its
//    own: keys straight from memory into the matrix operand, values through the
//    wave's part of shared memory, where the transposing read turns them.
//  - A wide tile (128 rows: a prefix that many requests share, a prompt) is
//    bound by the matrix cores: 64 positions are staged in shared memory for the four
//    waves, which have 32 rows each.
//  - In windows of long prompts such tiles are tall, 256 rows for eight waves, which
//    take turns with the matrix cores.
// e4m3 values are brought to the 16-bit type with their power of two as they
// are staged (exact but for fp16's range), so one kernel serves both.
//
// Scores, maxima, sums and results are in fp32 throughout.  Two things are rounded to the
// 16-bit type: the weights, since the matrix cores' operands are 16 bits (in two parts they
// would be twice the second product), each by half a step at
// most, 2^-8 of its own size in bf16 and 2^-11 in fp16, so a result by no more than that of
// sum p |v| (the sum that divides them takes them as they were); and the result.  fp16 has
// no such half step below 2^-14, where a weight is off by 2^-25: there all weights are 2^10
// times what they stand for (weight_lift), a row's largest is 2^10 at least, and T small
// ones are off by T 2^-35 max|v| in the result at most.

#include <algorithm>

#include "ps_blocks.h"

namespace ps {

namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef short i16x4 __attribute__((ext_vector_type(4)));

constexpr float kLn2 = 0.693147180559945309f;

// The exponent that weights are lifted by, so that fp16 keeps the bits of small ones (a token that
// takes nearly all of the weight, with a small value, leaves the result to them: 4096 weights of
// 2^-23.4 made it up to 17% too large).  The running maximum that is kept is less by it.
// Weights reach 2^10 where it is the row's, up to 2^raise_by more where it lies below, of fp16's
// 2^16: the rest is for the rounding of score x c, which shifts all weights of a row alike (by less
// than 2^2 for scores below 2^26).  bf16 has fp32's range.
constexpr float weight_lift(bool kF16) { return kF16 ? 10.0f : 0.0f; }
// How far a wide tile's row may outgrow the running maximum before that follows.
constexpr float raise_by(bool kF16) { return kF16 ? 4.0f : 8.0f; }
// A tall tile looks for the maximum where a lane's 32 weights sum up to more: above 32 times the lifted
// largest weight, and no weight that leaves fp16.
constexpr float far_sum(bool kF16) { return kF16 ? 49152.0f : 8192.0f; }

// The logarithm of a sum l of lifted weights under the kept maximum m.
template <bool kF16>
__device__ inline float lse_of(float m, float l) {
  const float lift = weight_lift(kF16);
  return __builtin_fmaf(m + lift, kLn2, __logf(l * __builtin_exp2f(-lift)));
}

template <bool kF16>
__device__ inline f32x4 mfma16(u32x4 a, u32x4 b, f32x4 c) {
  if (kF16)
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}

template <bool kF16>
__device__ inline f32x16 mfma32(u32x4 a, u32x4 b, f32x16 c) {
  if (kF16)
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
  return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}

template <bool kF16>
__device__ inline uint32_t pack(float a, float b) {
  if (kF16) {
    const f16x2 v = {(_Float16)a, (_Float16)b};
    return __builtin_bit_cast(uint32_t, v);
  }
  const bf16x2 v = {(__bf16)a, (__bf16)b};
  return __builtin_bit_cast(uint32_t, v);
}

// Four e4m3 codes to 16 bits, times a power of two.
template <bool kF16>
__device__ inline u32x2 widen(uint32_t x, float s) {
  u32x2 o;
  if (kF16) {
    o[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8((int)x, s, false));
    o[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8((int)x, s, true));
  } else {
    o[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((int)x, s, false));
    o[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((int)x, s, true));
  }
  return o;
}

// Half of 16 codes: 8 values.
template <bool kF16>
__device__ inline u32x4 widen8(uint32_t x, uint32_t y, float s) {
  const u32x2 a = widen<kF16>(x, s), b = widen<kF16>(y, s);
  return u32x4{a[0], a[1], b[0], b[1]};
}

// Sets infinities and NaN among 8 packed 16-bit values to 0; whether there were any.
template <bool kF16>
__device__ inline uint32_t clean8(u32x4& x) {
  constexpr uint32_t lo = kF16 ? 0x7C00u : 0x7F80u, hi = lo << 16;
  uint32_t r = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint32_t out = ((x[i] & lo) == lo ? 0xFFFFu : 0u) | ((x[i] & hi) == hi ? 0xFFFF0000u : 0u);
    r |= out;
    x[i] &= ~out;
  }
  return r;
}

// A lane's number, anew: what is computed from it is not kept in registers from one
// tile to the next.
__device__ inline int fresh(int x) {
  asm volatile("" : "+v"(x));
  return x;
}

// x + y, done here: a rare loop's sums are not put off until all of its loads are in registers.
__device__ inline float added(float x, float y) {
  x += y;
  asm volatile("" : "+v"(x) : : "memory");
  return x;
}

// Four rows' elements to a lane each: of 16 lanes that point to 4 rows of 16
// elements (4 lanes a row, 4 elements a lane), lane i receives column i.
__device__ inline u32x2 read_turned(const unsigned char* p) {
  typedef __attribute__((address_space(3))) i16x4* lds_ptr;
  return __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_ptr)p));
}

__device__ inline float scale_of(uint32_t x) { return __builtin_bit_cast(float, x << 23); }

// A value that is the same for the wave, as a scalar.
__device__ inline int32_t uniform(int32_t x) { return __builtin_amdgcn_readfirstlane(x); }
__device__ inline int64_t uniform(int64_t x) {
  return (int64_t)((uint64_t)(uint32_t)uniform((int32_t)(x >> 32)) << 32 | (uint32_t)uniform((int32_t)x));
}

// The chain of a tile, with what it takes to find a position's bytes.
struct Chain {
  const int32_t* pre;   // the page of block 0 of the prefix segment
  const int32_t* tail;  // the page of the tail's first block, less pre_len
  int32_t pre_len;
};

__device__ inline int32_t block_of(const AttendArgs& a, int32_t t) {
  return (int32_t)((__umulhi((uint32_t)t, a.bt_mul) + (uint32_t)t) >> a.bt_shift);
}

// The page of position t, as it is read: nothing is computed from it here, since
// that would wait for it, and for every load before it.
__device__ inline uint32_t page_of(const AttendArgs& a, const Chain& c, int32_t t) {
  const int32_t b = block_of(a, t);
  return (uint32_t)(b < c.pre_len ? c.pre : c.tail)[b];
}

struct Spot {
  int64_t at;  // first element of the row
  int64_t x;   // its exponent
};
// (A page number was checked when the plan was made; one that has changed since is
// kept inside the cache.)
__device__ inline Spot spot_at(const AttendArgs& a, int32_t head, uint32_t page, uint32_t slot) {
  page = min(page, (uint32_t)a.cache.n_pages - 1u);
  const uint32_t r = (uint32_t)(head * a.win.bt) + slot;  // (r dim < 2^32: the limits of heads, blocks and dim)
  const uint64_t row = r * (uint32_t)a.cache.dim;
  // (a product of 64 bits is three of 32, and strides of pages that need it are rare)
  uint64_t at = (uint64_t)page * (uint32_t)a.cache.page_stride + row, x = (uint64_t)page * (uint32_t)a.cache.exp_stride + r;
  if (a.cache.page_stride >> 32) at += (uint64_t)(page * (uint32_t)(a.cache.page_stride >> 32)) << 32;
  if (a.cache.exp_stride >> 32) x += (uint64_t)(page * (uint32_t)(a.cache.exp_stride >> 32)) << 32;
  return Spot{(int64_t)at, (int64_t)x};
}
__device__ inline Spot spot_of(const AttendArgs& a, int32_t head, uint32_t page, int32_t t) {
  return spot_at(a, head, page, (uint32_t)(t - block_of(a, t) * a.win.bt));
}

// One piece of a tile: positions [ta, tb) for its rows.
struct Piece {
  Chain chain;
  int32_t p0, row0, rows;
  int32_t ta, tb;
  int32_t slot;  // first row of its partial results, -1: the result itself
  int32_t head;
  float c;       // |scale| log2 e, above 0
  uint32_t neg;  // sign bits that turn q where scale is negative
};

// Row r of the tile (of the window's rows in their order x the group's heads).
struct RowAt {
  int32_t place, head;
};
__device__ inline RowAt row_at(const AttendArgs& a, const Piece& p, int32_t r) {
  const int32_t x = p.row0 + r, t = x / a.ratio;
  return RowAt{p.p0 + t, p.head * a.ratio + (x - t * a.ratio)};
}

// Elements d .. d + 3 of position t's value row, infinities and NaN as they
// are and everything else 0.
template <bool kF16, bool kQ8>
__device__ inline f32x4 odd_values(const AttendArgs& a, const Piece& p, int32_t t, int32_t d) {
  const Spot s = spot_of(a, p.head, page_of(a, p.chain, t), t);
  u32x2 x;
  if (kQ8) x = widen<kF16>(*(const uint32_t*)(a.cache.v + s.at + d), scale_of(a.cache.vx[s.x]));
  else x = *(const u32x2*)(a.cache.v + 2 * (s.at + d));
  f32x4 o;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint32_t h = i & 1 ? x[i >> 1] >> 16 : x[i >> 1] & 0xFFFFu;
    const float f = kF16 ? (float)__builtin_bit_cast(_Float16, (uint16_t)h) : __builtin_bit_cast(float, h << 16);
    o[i] = __builtin_isfinite(f) ? 0.0f : f;
  }
  return o;
}

// Eight elements of the row of q that begins at `at`, from element d.
__device__ inline u32x4 load_q(const AttendArgs& a, const Piece& p, int64_t at, bool has, int32_t d) {
  u32x4 x = {0, 0, 0, 0};
  if (has && d < a.cache.dim) {
    x = *(const u32x4*)(a.q.data + 2 * (at + d));
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] ^= p.neg;
  }
  return x;
}

// Four results of a row, from element d: written out, or kept as a partial result.
template <bool kF16>
__device__ inline void put4(const AttendArgs& a, const Piece& p, int32_t r, int32_t d, f32x4 o, float inv) {
  if (d >= a.cache.dim) return;
  if (p.slot >= 0) {
    const int64_t at = (int64_t)p.head * a.plan.slot_rows + p.slot + r;
    *(f32x4*)(a.plan.part + at * a.cache.dim + d) = o;
    return;
  }
  const RowAt w = row_at(a, p, r);
  const u32x2 x = {pack<kF16>(o[0] * inv, o[1] * inv), pack<kF16>(o[2] * inv, o[3] * inv)};
  *(u32x2*)(a.out.data + 2 * ((int64_t)a.plan.row[w.place] * a.out.row + (int64_t)w.head * a.out.head + d)) = x;
}

// A row's maximum (mc: of scores times c, less weight_lift) and sum, likewise; returns what its results are
// multiplied by where they are final.
template <bool kF16>
__device__ inline float put_ml(const AttendArgs& a, const Piece& p, int32_t r, float mc, float l, bool write) {
  if (p.slot >= 0) {
    if (write) a.plan.part_ml[(int64_t)p.head * a.plan.slot_rows + p.slot + r] = float2{mc, l};
    return 1.0f;
  }
  const RowAt w = row_at(a, p, r);
  const bool empty = a.plan.lim[w.place] <= 0;
  if (write && a.lse)
    a.lse[(int64_t)a.plan.row[w.place] * a.heads + w.head] =
        empty ? -INFINITY : lse_of<kF16>(mc, l);
  return empty ? 0.0f : 1.0f / l;
}

// ------------------------------------------------------------------ narrow

// Rows of values in shared memory, in bytes: padded so that the turned reads of 16
// rows (narrow: 32 bytes each) or 8 rows (wide: 64 bytes each) take every bank the
// same number of times; rows of keys so that 8 of them differ in their banks.  Padding
// rather than swizzled chunks: all offsets are then constants of the instructions.
constexpr int narrow_stride(int DP) { return DP * 2 + 32; }
constexpr int value_stride(int DP) { return DP * 2 + 64; }
constexpr int key_stride(int DP) { return DP * 2 + 16; }

// Positions of a narrow step: enough that a wave has 16 KB of a head of 128 in flight.
constexpr int narrow_positions(bool kQ8, int DP) { return kQ8 && DP <= 128 ? 64 : 32; }

// A head of fewer than DP elements is padded (kPad): to those of q come zeros, and to those of its
// keys too, since an infinity of a key times 0 would be NaN.  (A kernel of its own: with the
// selects in it, chunks of full heads took 1.5% longer, 1388 -> 1408 us.)  The least such head:
constexpr int least_dim(int DP) { return DP == 64 ? 16 : DP / 2 + 16; }

template <bool kF16, bool kQ8, int DP, bool kPad>
__device__ void narrow_piece(const AttendArgs& a, const Piece& p, unsigned char* vs) {
  constexpr int kTok = narrow_positions(kQ8, DP);
  constexpr int kH = kTok / 16;                       // rows of positions in the first product
  constexpr int kX = kTok / 32;                       // steps of the second product
  constexpr int kSteps = DP / 32;                     // of the first product
  constexpr int kLoads = kQ8 ? DP / 64 : DP / 32;     // 16-byte loads per lane and 16 positions
  constexpr int kDB = DP / 16;                        // blocks of the second product
  constexpr int kV = narrow_stride(DP);
  static_assert(kNarrowRows == 16, "a row of the tile per column of the products");
  const int lane = fresh(threadIdx.x & 63), col = lane & 15, g = lane >> 4;
  const int D = a.cache.dim;

  f32x4 acc[kDB];
  float m = -INFINITY, l = 0;  // (the maximum of scores times c, less weight_lift)
#pragma unroll
  for (int k = 0; k < kDB; ++k) acc[k] = f32x4{0, 0, 0, 0};

  const int32_t last = p.tb - 1;
  uint32_t page[kH];
  u32x4 kr[kH][kLoads], vr[kH][kLoads];
  uint32_t kx[kH], vx[kH];
  auto pages = [&](int32_t t) {
#pragma unroll
    for (int h = 0; h < kH; ++h) page[h] = page_of(a, p.chain, min(t + 16 * h + col, last));
  };
  auto loads = [&](int32_t t) {
#pragma unroll
    for (int h = 0; h < kH; ++h) {
      const Spot s = spot_of(a, p.head, page[h], min(t + 16 * h + col, last));
#pragma unroll
      for (int i = 0; i < kLoads; ++i) {
        // (where the head has fewer elements than DP, its last ones once more: of keys they
        // become zeros before they are used, of values they make results that nobody reads)
        const int d = kQ8 ? min(64 * i + 16 * g, D - 16) : min(32 * i + 8 * g, D - 8);
        const int64_t at = kQ8 ? s.at + d : 2 * (s.at + d);
        kr[h][i] = *(const u32x4*)(a.cache.k + at);
        vr[h][i] = *(const u32x4*)(a.cache.v + at);
      }
      if (kQ8) {
        kx[h] = a.cache.kx[s.x];
        vx[h] = a.cache.vx[s.x];
      }
    }
  };

  // Pages and rows are asked for together, then keys and values, then q: loads return
  // in order, so that a wait for q's would hold the others back.
  u32x4 q[kSteps];
  pages(p.ta);
  const RowAt qrow = row_at(a, p, min(col, p.rows - 1));
  int32_t lim = a.plan.lim[qrow.place];
  const int64_t qat = a.plan.row[qrow.place] * a.q.row + (int64_t)qrow.head * a.q.head;
  loads(p.ta);
  pages(p.ta + kTok);
  const bool has = col < p.rows;
#pragma unroll
  for (int s = 0; s < kSteps; ++s)
    q[s] = load_q(a, p, qat, has, kQ8 ? 64 * (s >> 1) + 16 * g + 8 * (s & 1) : 32 * s + 8 * g);
  if (!has) lim = INT32_MAX;
  int32_t least = lim;
  for (int o = 8; o > 0; o >>= 1) least = min(least, __shfl_xor(least, o, 64));

  for (int32_t t = p.ta; t < p.tb; t += kTok) {
    // Values into shared memory.  Where a row may not see all of the step's, their
    // infinities and NaN are taken out, since a weight of 0 would not take them
    // away; the rows that see them get them below.
    const bool masked = t + kTok > p.tb || t + kTok > least;  // (the same for the wave)
    uint32_t odd = 0;
#pragma unroll
    for (int h = 0; h < kH; ++h)
#pragma unroll
      for (int i = 0; i < kLoads; ++i) {
        const int row = 16 * h + col;
        if (kQ8) {
          const float s = scale_of(vx[h]);
          u32x4 x = widen8<kF16>(vr[h][i][0], vr[h][i][1], s), y = widen8<kF16>(vr[h][i][2], vr[h][i][3], s);
          if (masked) {
            odd |= clean8<kF16>(x);
            odd |= clean8<kF16>(y);
          }
          *(u32x4*)(vs + row * kV + (8 * i + 2 * g) * 16) = x;
          *(u32x4*)(vs + row * kV + (8 * i + 2 * g + 1) * 16) = y;
        } else {
          if (masked) odd |= clean8<kF16>(vr[h][i]);
          *(u32x4*)(vs + row * kV + (4 * i + g) * 16) = vr[h][i];
        }
      }
    if constexpr (kPad) {
#pragma unroll
      for (int i = 0; i < kLoads; ++i)
        if ((kQ8 ? 64 : 32) * (i + 1) > least_dim(DP) && (kQ8 ? 64 * i + 16 * g : 32 * i + 8 * g) >= D)
#pragma unroll
          for (int h = 0; h < kH; ++h) kr[h][i] = u32x4{0, 0, 0, 0};
    }
    // scores: position 16 h + 4 g + i of the step, row col
    f32x4 s[kH];
#pragma unroll
    for (int h = 0; h < kH; ++h) {
      s[h] = f32x4{0, 0, 0, 0};
#pragma unroll
      for (int st = 0; st < kSteps; ++st) {
        u32x4 ka;
        if (kQ8) {
          const u32x4 x = kr[h][st >> 1];
          ka = st & 1 ? widen8<kF16>(x[2], x[3], scale_of(kx[h])) : widen8<kF16>(x[0], x[1], scale_of(kx[h]));
        } else {
          ka = kr[h][st % kLoads];
        }
        s[h] = mfma16<kF16>(ka, q[st], s[h]);
      }
    }
    // (behind the last step too, its last position over: of loads that depend on a branch
    // the registers are copied behind it, which waits for them)
    loads(t + kTok);
    pages(t + 2 * kTok);
    // (the rows that other lanes wrote)
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");

    if (masked) {
#pragma unroll
      for (int h = 0; h < kH; ++h)
#pragma unroll
        for (int i = 0; i < 4; ++i)
          if (t + 16 * h + 4 * g + i >= min(lim, p.tb)) s[h][i] = -INFINITY;
    }
    float top = s[0][0];
#pragma unroll
    for (int i = 1; i < 4 * kH; ++i) top = fmaxf(top, s[i >> 2][i & 3]);
    top = fmaxf(top, __shfl_xor(top, 16, 64));
    top = fmaxf(top, __shfl_xor(top, 32, 64));
    // (kept as the rounded product that the weights take, so that the factor of a maximum that has
    // not moved is 1: a fused m c - mc is the product's rounding error, the same in every step, and
    // bent the sums of 1024 steps under scores of 100 to 200 by 4e-3)
    const float nm = fmaxf(m, top * p.c - weight_lift(kF16));
    const float mc = nm == -INFINITY ? 0.0f : nm;
    const float f = __builtin_amdgcn_exp2f(m - mc);
    m = nm;
    l *= f;
#pragma unroll
    for (int k = 0; k < kDB; ++k) acc[k] *= f;
    if (masked && __any(odd != 0))
#pragma unroll 1
      for (int32_t o = t; o < min(t + kTok, p.tb); ++o)
#pragma unroll
        for (int k = 0; k < kDB; ++k) {
          const f32x4 x = odd_values<kF16, kQ8>(a, p, o, min(16 * k + fresh(4 * g), D - 4));
#pragma unroll
          for (int i = 0; i < 4; ++i) acc[k][i] = added(acc[k][i], o < lim ? x[i] : 0.0f);
        }
    // lane i of 16: row 4 g + i / 4, elements 16 k + 4 (i % 4) ..
    auto turned = [&](int x, int k) {
      const unsigned char* at = vs + (4 * g + (col >> 2)) * kV + (col & 3) * 8;
      const u32x2 y0 = read_turned(at + 32 * x * kV + 32 * k);
      const u32x2 y1 = read_turned(at + (32 * x + 16) * kV + 32 * k);
      return u32x4{y0[0], y0[1], y1[0], y1[1]};
    };
#pragma unroll
    for (int x = 0; x < kX; ++x) {
      u32x4 va[kDB], pr;
#pragma unroll
      for (int k = 0; DP <= 128 && k < kDB; ++k) va[k] = turned(x, k);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const f32x4& v = s[2 * x + (i >> 1)];
        const float e0 = __builtin_amdgcn_exp2f(__builtin_fmaf(v[(2 * i) & 3], p.c, -mc));
        const float e1 = __builtin_amdgcn_exp2f(__builtin_fmaf(v[(2 * i + 1) & 3], p.c, -mc));
        l += e0 + e1;
        pr[i] = pack<kF16>(e0, e1);
      }
#pragma unroll
      for (int k = 0; k < kDB; ++k) {
        if (DP > 128) va[0] = turned(x, k);  // (no registers to read ahead)
        acc[k] = mfma16<kF16>(va[DP > 128 ? 0 : k], pr, acc[k]);
      }
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  }

  const int at = fresh(lane), d0 = 4 * (at >> 4);
  l += __shfl_xor(l, 16, 64);
  l += __shfl_xor(l, 32, 64);
  const int32_t r = at & 15;
  if (r < p.rows) {
    const float inv = put_ml<kF16>(a, p, r, m, l, d0 == 0);
#pragma unroll
    for (int k = 0; k < kDB; ++k) put4<kF16>(a, p, r, 16 * k + d0, acc[k], inv);
  }
}

// ------------------------------------------------------------------ wide

// Positions of a wide step: 64, or 32 where a row's registers leave no room.
constexpr int wide_positions(int DP) { return DP <= 128 ? 64 : 32; }

// What a thread of a wide or tall tile's workgroup stages: part of one row of a step's
// positions, asked for (pages, then loads) before it is put into shared memory.
template <bool kF16, bool kQ8, int DP, bool kPad, int kTok, int kThreads>
struct Stage {
  static constexpr int kPer = kThreads / kTok;                     // threads that stage a row
  static constexpr int kLoads = (kQ8 ? DP / 16 : DP / 8) / kPer;  // 16-byte loads per thread
  static constexpr int kChunk = kQ8 ? 32 : 16;                     // bytes in shared memory of such a load
  static constexpr int kEach = kQ8 ? 16 : 8;                       // elements
  const int row, sc;  // thread x: row x / kPer, chunks x % kPer + kPer i
  const int32_t last;
  uint32_t page, slot;
  u32x4 kr[kLoads], vr[kLoads];
  uint32_t kx = 0, vx = 0;

  __device__ Stage(const Piece& p, int wave, int lane)
      : row(wave * (64 / kPer) + lane / kPer), sc(lane % kPer), last(p.tb - 1) {}
  __device__ void pages(const AttendArgs& a, const Piece& p, int32_t t) {
    const int32_t at = min(t + row, last), b = block_of(a, at);
    slot = (uint32_t)(at - b * a.win.bt);
    page = (uint32_t)(b < p.chain.pre_len ? p.chain.pre : p.chain.tail)[b];
  }
  __device__ void loads(const AttendArgs& a, const Piece& p) {
    const Spot s = spot_at(a, p.head, page, slot);
    const int D = a.cache.dim;
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
      const int d = kQ8 ? min(16 * (kPer * i + sc), D - 16) : min(8 * (kPer * i + sc), D - 8);  // (as in the narrow kernel)
      const int64_t at = kQ8 ? s.at + d : 2 * (s.at + d);
      kr[i] = *(const u32x4*)(a.cache.k + at);
      vr[i] = *(const u32x4*)(a.cache.v + at);
    }
    if (kQ8) {
      kx = a.cache.kx[s.x];
      vx = a.cache.vx[s.x];
    }
  }
  // Into the step's keys and values; whether values had infinities or NaN, which are
  // taken out of a masked step's (as in the narrow kernel).
  __device__ uint32_t put(unsigned char* keys, unsigned char* values, bool masked, int D) {
    uint32_t odd = 0;
    if constexpr (kPad) {  // (as in the narrow kernel)
#pragma unroll
      for (int i = 0; i < kLoads; ++i)
        if (kEach * kPer * (i + 1) > least_dim(DP) && kEach * (kPer * i + sc) >= D) kr[i] = u32x4{0, 0, 0, 0};
    }
    unsigned char* ks = keys + row * key_stride(DP) + sc * kChunk;
    unsigned char* vs = values + row * value_stride(DP) + sc * kChunk;
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
      const int off = kPer * kChunk * i;
      if (kQ8) {
        const float sk = scale_of(kx), sv = scale_of(vx);
        *(u32x4*)(ks + off) = widen8<kF16>(kr[i][0], kr[i][1], sk);
        *(u32x4*)(ks + off + 16) = widen8<kF16>(kr[i][2], kr[i][3], sk);
        u32x4 x = widen8<kF16>(vr[i][0], vr[i][1], sv), y = widen8<kF16>(vr[i][2], vr[i][3], sv);
        if (masked) {
          odd |= clean8<kF16>(x);
          odd |= clean8<kF16>(y);
        }
        *(u32x4*)(vs + off) = x;
        *(u32x4*)(vs + off + 16) = y;
      } else {
        if (masked) odd |= clean8<kF16>(vr[i]);
        *(u32x4*)(ks + off) = kr[i];
        *(u32x4*)(vs + off) = vr[i];
      }
    }
    return odd;
  }
};

// The larger of a lane's value and that of the lane 32 from it.
__device__ inline float max_of_halves(float x) {
  const uint32_t u = __builtin_bit_cast(uint32_t, x);
  const u32x2 y = __builtin_bit_cast(u32x2, __builtin_amdgcn_permlane32_swap(u, u, false, false));
  const uint32_t own = y[0], other = y[1];  // (a bit cast of y[1] itself reads y[0]: the compiler's)
  return fmaxf(__builtin_bit_cast(float, own), __builtin_bit_cast(float, other));
}

// A wave's scores of 32 kB positions from t, lane: position 32 b + 8 (i / 4) + 4 hb + i % 4:
// those that the row does not see are taken out.
template <int kB>
__device__ inline void mask_scores(f32x16 (&s)[kB], int32_t t, int hb, int32_t end) {
#pragma unroll
  for (int b = 0; b < kB; ++b)
#pragma unroll
    for (int i = 0; i < 16; ++i)
      if (t + 32 * b + 8 * (i >> 2) + 4 * hb + (i & 3) >= end) s[b][i] = -INFINITY;
}

// The largest of a row's scores, times c, less weight_lift.
template <bool kF16, int kB>
__device__ inline float top_of(const f32x16 (&s)[kB], float c) {
  float top = s[0][0];
#pragma unroll
  for (int i = 1; i < 16 * kB; ++i) top = fmaxf(top, s[i >> 4][i & 15]);
  return max_of_halves(top) * c - weight_lift(kF16);
}

// The running maximum (m, of scores times c) of the rows that say so becomes top; the sum and
// the results follow it.  It need not be the row's own: rows say so where that is 2^8 above it
// (fp16: 2^4) or more.  Such weights fit both types and are rounded to as many bits, and of 32
// rows in random order one has a new maximum in most steps, none so large a one.  (Whether a
// row says so depends on the row alone, so its bits do not depend on what lies beside it.)
template <int kDB>
__device__ inline void raise_top(bool up, float top, float& m, float& l, f32x16 (&acc)[kDB]) {
  const float f = up ? __builtin_amdgcn_exp2f(m - top) : 1.0f;
  m = up ? top : m;
  l *= f;
#pragma unroll
  for (int k = 0; k < kDB; ++k) acc[k] *= f;
}

// The infinities and NaN that were taken out of positions [t, end)'s values, to the rows that see them.
template <bool kF16, bool kQ8, int kDB>
__device__ inline void add_odd(const AttendArgs& a, const Piece& p, int32_t t, int32_t end, int hb, int32_t lim,
                               f32x16 (&acc)[kDB]) {
#pragma unroll 1
  for (int32_t o = t; o < end; ++o)
#pragma unroll
    for (int k = 0; k < 4 * kDB; ++k) {
      const f32x4 x = odd_values<kF16, kQ8>(a, p, o, min(8 * k + fresh(4 * hb), a.cache.dim - 4));
#pragma unroll
      for (int i = 0; i < 4; ++i) acc[k >> 2][4 * (k & 3) + i] = added(acc[k >> 2][4 * (k & 3) + i], o < lim ? x[i] : 0.0f);
    }
}

// Weights of a wave's scores 16 x .. 16 x + 15, packed; their sum is added to *sum.
template <bool kF16, int kB>
__device__ inline u32x4 weights(const f32x16 (&s)[kB], int x, float c, float mc, float* sum) {
  u32x4 w;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int at = (x & 1) * 8 + 2 * i;
    const float e0 = __builtin_amdgcn_exp2f(__builtin_fmaf(s[x >> 1][at], c, -mc));
    const float e1 = __builtin_amdgcn_exp2f(__builtin_fmaf(s[x >> 1][at + 1], c, -mc));
    *sum += e0 + e1;
    w[i] = pack<kF16>(e0, e1);
  }
  return w;
}

// The results of a wave's 32 rows from rows0.
template <bool kF16, int kDB>
__device__ inline void put_rows(const AttendArgs& a, const Piece& p, int rows0, int lane, float m, float l,
                                const f32x16 (&acc)[kDB]) {
  const int at = fresh(lane), d0 = 4 * (at >> 5);
  const int32_t r = rows0 + (at & 31);
  if (r >= p.rows) return;
  const float inv = put_ml<kF16>(a, p, r, m, l, d0 == 0);
#pragma unroll
  for (int k = 0; k < kDB; ++k)
#pragma unroll
    for (int i = 0; i < 4; ++i)
      put4<kF16>(a, p, r, 32 * k + 8 * i + d0,
                 f32x4{acc[k][4 * i], acc[k][4 * i + 1], acc[k][4 * i + 2], acc[k][4 * i + 3]}, inv);
}

// Elements 32 k + (lane's column) of 16 positions' values, turned: positions 8 jj + 4 hb ..
__device__ inline u32x4 turned_values(const unsigned char* at, int stride) {
  const u32x2 y0 = read_turned(at), y1 = read_turned(at + 8 * stride);
  return u32x4{y0[0], y0[1], y1[0], y1[1]};
}

// kSplit = 1: each wave has 32 of the 128 rows and all positions of a step; 2: 32 of 64
// rows and half of the positions, the halves' results joined at the end, so that
// tiles of 64 rows keep all four SIMDs at work.
template <bool kF16, bool kQ8, int DP, bool kPad, int kSplit>
__device__ void wide_piece(const AttendArgs& a, const Piece& p, unsigned char* smem, int32_t* odd_at) {
  constexpr int kSteps = DP / 16;
  constexpr int kTok = wide_positions(DP);
  constexpr int kDB = DP / 32;
  constexpr int kK = key_stride(DP), kV = value_stride(DP);
  constexpr int kKeys = kTok * kK, kTile = kTok * (kK + kV);  // bytes of a step's keys; of all
  constexpr int kMine = kTok / kSplit;  // positions of a step that are the wave's
  const int lane = fresh(threadIdx.x & 63), wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int col = lane & 31, hb = lane >> 5;
  const int rows0 = wave / kSplit * 32, off0 = wave % kSplit * kMine;
  const int32_t r = rows0 + col;
  const bool idle = rows0 >= p.rows;

  f32x16 acc[kDB];
#pragma unroll
  for (int k = 0; k < kDB; ++k)
#pragma unroll
    for (int i = 0; i < 16; ++i) acc[k][i] = 0;
  float m = -INFINITY, l = 0;  // (the maximum of scores times c, less weight_lift)

  Stage<kF16, kQ8, DP, kPad, kTok, 256> st(p, wave, lane);
  // (of one request's rows the first sees least; those of a shared prefix see all of it)
  const int32_t least_of_all = min(uniform(a.plan.lim[row_at(a, p, 0).place]), p.tb);
  auto stage = [&](int buf, int32_t t) {
    unsigned char* keys = smem + buf * kTile;
    if (st.put(keys, keys + kKeys, t + kTok > least_of_all, a.cache.dim))
      odd_at[buf] = t;  // (a value left by another piece only costs a look)
  };

  // (the order: as in the narrow kernel)
  st.pages(a, p, p.ta);
  const RowAt qrow = row_at(a, p, min(r, p.rows - 1));
  int32_t lim = a.plan.lim[qrow.place];
  const int64_t qat = a.plan.row[qrow.place] * a.q.row + (int64_t)qrow.head * a.q.head;
  st.loads(a, p);
  st.pages(a, p, p.ta + kTok);
  // (heads above 128: no registers for q, it stays in shared memory)
  u32x4 q[DP <= 128 ? kSteps : 1];
  unsigned char* qs = smem + 2 * kTile + (wave * 32 + col) * kK + hb * 16;
#pragma unroll
  for (int s = 0; s < kSteps; ++s) {
    const u32x4 x = load_q(a, p, qat, r < p.rows, 16 * s + 8 * hb);
    if (DP <= 128) q[s] = x;
    else *(u32x4*)(qs + 32 * s) = x;
  }
  if (r >= p.rows) lim = INT32_MAX;
  int32_t least = lim;
  for (int o = 16; o > 0; o >>= 1) least = min(least, __shfl_xor(least, o, 64));
  stage(0, p.ta);
  __syncthreads();
  int buf = 0;
  for (int32_t t = p.ta; t < p.tb; t += kTok, buf ^= 1) {
    st.loads(a, p);  // (behind the last step too: as in the narrow kernel)
    st.pages(a, p, t + 2 * kTok);
    if (!idle) {
      const unsigned char* ks = smem + buf * kTile + (off0 + col) * kK + hb * 16;
      const unsigned char* vs =
          smem + buf * kTile + kKeys + (off0 + 4 * hb + ((lane & 15) >> 2)) * kV + ((lane >> 4) & 1) * 32 + (lane & 3) * 8;
      // scores: position 32 b + 8 (i / 4) + 4 hb + i % 4 of the tile's
      f32x16 s[kMine / 32];
#pragma unroll
      for (int b = 0; b < kMine / 32; ++b) {
#pragma unroll
        for (int i = 0; i < 16; ++i) s[b][i] = 0;
#pragma unroll
        for (int i = 0; i < kSteps; ++i)
          s[b] = mfma32<kF16>(*(const u32x4*)(ks + 32 * b * kK + 32 * i),
                              DP <= 128 ? q[DP <= 128 ? i : 0] : *(const u32x4*)(qs + 32 * i), s[b]);
      }
      const bool masked = t + kTok > p.tb || t + kTok > least;
      if (masked) mask_scores(s, t + off0, hb, min(lim, p.tb));
      const float top = top_of<kF16>(s, p.c);
      const bool up = top > m + raise_by(kF16);
      if (__any(up)) raise_top(up, top, m, l, acc);
      const float mc = m == -INFINITY ? 0.0f : m;
      // (also for a wave whose rows all see all of the step)
      if (t + kTok > least_of_all && odd_at[buf] == t)
        add_odd<kF16, kQ8>(a, p, t + off0, min(t + off0 + kMine, p.tb), hb, lim, acc);
      auto turned = [&](int x, int k) { return turned_values(vs + 16 * x * kV + 64 * k, kV); };
      // 16 positions at a time: the products of the ones before run beside the
      // exponentials of these.  (Heads above 128: no registers for that.)
      float sum = 0;
      u32x4 pr[kMine / 16];
#pragma unroll
      for (int x = 0; x < kMine / 16; ++x) {
        u32x4 va[kDB];
        if (DP <= 128)
#pragma unroll
          for (int k = 0; k < kDB; ++k) va[k] = turned(x, k);
        pr[x] = weights<kF16>(s, x, p.c, mc, &sum);
        if (DP <= 128)
#pragma unroll
          for (int k = 0; k < kDB; ++k) acc[k] = mfma32<kF16>(va[k], pr[x], acc[k]);
      }
      if (DP > 128)
#pragma unroll
        for (int x = 0; x < kMine / 16; ++x)
#pragma unroll
          for (int k = 0; k < kDB; ++k) acc[k] = mfma32<kF16>(turned(x, k), pr[x], acc[k]);
      l += sum;
    }
    if (t + kTok < p.tb) stage(buf ^ 1, t + kTok);
    __syncthreads();
  }
  l += __shfl_xor(l, 32, 64);
  if (kSplit == 2) {
    // the second half's results to the first half's wave
    float2* ml = (float2*)(smem + 2 * 32 * DP * 4);
    f32x4* os = (f32x4*)(smem + (wave >> 1) * 32 * DP * 4);
    if (wave & 1) {
      if (hb == 0) ml[r] = float2{m, l};
#pragma unroll
      for (int k = 0; k < kDB; ++k)
#pragma unroll
        for (int i = 0; i < 4; ++i)
          os[(4 * k + i) * 64 + lane] =
              f32x4{acc[k][4 * i], acc[k][4 * i + 1], acc[k][4 * i + 2], acc[k][4 * i + 3]};
    }
    __syncthreads();
    if (!(wave & 1)) {
      const float2 x = ml[r];
      const float top = fmaxf(m, x.x), mc = top == -INFINITY ? 0.0f : top;
      const float f = __builtin_amdgcn_exp2f(m - mc);
      const float fx = __builtin_amdgcn_exp2f(x.x - mc);
      l = l * f + x.y * fx;
      m = top;
#pragma unroll
      for (int k = 0; k < kDB; ++k)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const f32x4 o = os[(4 * k + i) * 64 + lane];
#pragma unroll
          for (int e = 0; e < 4; ++e) acc[k][4 * i + e] = acc[k][4 * i + e] * f + o[e] * fx;
        }
    }
    __syncthreads();
    if (wave & 1) return;
  }
  put_rows<kF16>(a, p, rows0, lane, m, l, acc);
}

// ------------------------------------------------------------------ tall

// 256 rows, 8 waves of 32: two to each SIMD, of which one is at its products while the other is
// at its weights.  Waves 4 .. 7 are half a step behind waves 0 .. 3, with a barrier
// between the halves:
//   waves 0 .. 3   weights(t)                       results(t), scores(t + 1)
//   waves 4 .. 7   results(t - 1), scores(t)        weights(t)
// Each half stages its rows of the positions with its weights: waves 0 .. 3 those of step t + 1,
// which they read half a step later, waves 4 .. 7 those of step t + 2.  So scores have
// two buffers of keys and results three of values.  In the products, operands are read
// four products ahead of their use (2100 cycles with the reads where the compiler puts
// them, 1300 so; the weights took 1400 with a maximum looked for in every step, staging 700).
//
// Chunks of 777 to 2048 tokens behind 8192 to 16384, 32 heads over 8: 850 TFLOP/s with the
// wide kernel's tiles, 1060 to 1090 with these, of 1180 that a large matrix product reaches.
constexpr int kTallStep = 64;

template <bool kF16, bool kQ8, int DP, bool kPad>
__device__ void tall_piece(const AttendArgs& a, const Piece& p, unsigned char* smem, int32_t* odd_at) {
  constexpr int kSteps = DP / 16, kTok = kTallStep, kDB = DP / 32;
  constexpr int kK = key_stride(DP), kV = value_stride(DP);
  constexpr int kKeys = kTok * kK, kValues = kTok * kV;
  static_assert(DP == 128 && kTok == 64, "four products of results and of scores at a time");
  const int lane = fresh(threadIdx.x & 63), wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int col = lane & 31, hb = lane >> 5;
  const int rows0 = wave * 32;
  const int32_t r = rows0 + col;
  const bool late = wave >= 4;
  const int ahead = late ? 2 : 1;  // steps that are staged before their scores

  f32x16 acc[kDB];
#pragma unroll
  for (int k = 0; k < kDB; ++k)
#pragma unroll
    for (int i = 0; i < 16; ++i) acc[k][i] = 0;
  float m = -INFINITY, l = 0;  // (the maximum of scores times c, less weight_lift)

  Stage<kF16, kQ8, DP, kPad, kTok, 512> st(p, wave, lane);
  const int32_t least_of_all = min(uniform(a.plan.lim[row_at(a, p, 0).place]), p.tb);  // (as in the wide kernel)
  auto stage = [&](int kb, int vb, int32_t t) {
    if (st.put(smem + kb * kKeys, smem + 2 * kKeys + vb * kValues, t + kTok > least_of_all, a.cache.dim))
      odd_at[vb] = t;
  };
  st.pages(a, p, p.ta);
  const RowAt qrow = row_at(a, p, min(r, p.rows - 1));
  int32_t lim = a.plan.lim[qrow.place];
  const int64_t qat = a.plan.row[qrow.place] * a.q.row + (int64_t)qrow.head * a.q.head;
  st.loads(a, p);
  st.pages(a, p, p.ta + kTok);
  u32x4 q[kSteps];
#pragma unroll
  for (int i = 0; i < kSteps; ++i) q[i] = load_q(a, p, qat, r < p.rows, 16 * i + 8 * hb);
  if (r >= p.rows) lim = INT32_MAX;
  int32_t least = lim;
  for (int o = 16; o > 0; o >>= 1) least = min(least, __shfl_xor(least, o, 64));
  stage(0, 0, p.ta);
  st.loads(a, p);
  st.pages(a, p, p.ta + 2 * kTok);
  if (late) {
    stage(1, 1, p.ta + kTok);  // (behind the last step, its last position over: as in the narrow kernel)
    st.loads(a, p);
    st.pages(a, p, p.ta + 3 * kTok);
  }
  __syncthreads();

  f32x16 s[2];
  u32x4 pr[kTok / 16];
  const unsigned char* ks0 = smem + col * kK + hb * 16;
  const unsigned char* vs0 =
      smem + 2 * kKeys + (4 * hb + ((lane & 15) >> 2)) * kV + ((lane >> 4) & 1) * 32 + (lane & 3) * 8;
  // the four operands of a round of products: values of 16 positions, keys of 64 and 32 elements
  auto values = [&](u32x4 (&x)[4], const unsigned char* vs, int i) {
#pragma unroll
    for (int k = 0; k < 4; ++k) x[k] = turned_values(vs + 16 * i * kV + 64 * k, kV);
  };
  auto keys = [&](u32x4 (&x)[4], const unsigned char* ks, int i) {
#pragma unroll
    for (int k = 0; k < 4; ++k) x[k] = *(const u32x4*)(ks + 32 * (k & 1) * kK + 32 * (2 * i + (k >> 1)));
  };
  auto scores = [&](const u32x4 (&x)[4], int i) {
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      if (i == 0 && k < 2)
#pragma unroll
        for (int e = 0; e < 16; ++e) s[k][e] = 0;
      s[k & 1] = mfma32<kF16>(x[k], q[2 * i + (k >> 1)], s[k & 1]);
    }
  };
  if (late) __syncthreads();  // (half a step behind from here on; the others wait at the end)
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    u32x4 x[4];
    keys(x, ks0, i);
    scores(x, i);
  }
  __syncthreads();
  int kb = 0, vb = 0;
  // (begins with a line of instructions: chunks took 1.5% longer with some places of the loop)
  asm volatile(".p2align 6" ::: "memory");
  for (int32_t t = p.ta; t < p.tb; t += kTok) {
    const bool masked = t + kTok > p.tb || t + kTok > least;
    if (masked) mask_scores(s, t, hb, min(lim, p.tb));
    if (t + kTok > least_of_all && odd_at[vb] == t) {
      // (rows without a maximum take theirs first: their results are multiplied by 0 then)
      const float top = top_of<kF16>(s, p.c);
      raise_top(m == -INFINITY && top > m, top, m, l, acc);
      add_odd<kF16, kQ8>(a, p, t, min(t + kTok, p.tb), hb, lim, acc);
    }
    // Weights from the maximum as it is, which is nearly always near enough.  The row's own is
    // looked for where there is none yet, or where a lane's 32 weights sum up to 2^13 (fp16:
    // 1.5 * 2^15), so that one of them is 2^8 (2^0.5 times the lifted 1) at least and none
    // leaves the type.
    auto all_weights = [&] {
      const float mc = m == -INFINITY ? 0.0f : m;
      float sum = 0;
#pragma unroll
      for (int x = 0; x < kTok / 16; ++x) pr[x] = weights<kF16>(s, x, p.c, mc, &sum);
      return sum;
    };
    float sum = all_weights();
    const uint64_t far = __ballot(sum > far_sum(kF16) || m == -INFINITY);
    if (far) {
      const float top = top_of<kF16>(s, p.c);
      raise_top((far | far >> 32) >> col & 1 && top > m, top, m, l, acc);
      sum = all_weights();
    }
    l += sum;
    {
      const int v2 = vb + ahead;
      stage(kb ^ (ahead & 1), v2 < 3 ? v2 : v2 - 3, t + ahead * kTok);
    }
    st.loads(a, p);
    st.pages(a, p, t + (ahead + 2) * kTok);
    __syncthreads();

    const unsigned char *vs = vs0 + vb * kValues, *ks = ks0 + (kb ^ 1) * kKeys;
    // (behind the last step: scores of keys that were there before, unused)
    u32x4 x[2][4];
    values(x[0], vs, 0);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      if (i < 3) values(x[(i + 1) & 1], vs, i + 1);
      else if (i < 7) keys(x[(i + 1) & 1], ks, i - 3);
      __builtin_amdgcn_sched_barrier(0);
      if (i < 4) {
#pragma unroll
        for (int k = 0; k < 4; ++k) acc[k] = mfma32<kF16>(x[i & 1][k], pr[i], acc[k]);
      } else {
        scores(x[i & 1], i - 4);
      }
      __builtin_amdgcn_sched_barrier(0);
    }
    __syncthreads();
    kb ^= 1;
    vb = vb == 2 ? 0 : vb + 1;
  }
  if (!late) __syncthreads();
  l += __shfl_xor(l, 32, 64);
  put_rows<kF16>(a, p, rows0, lane, m, l, acc);
}

constexpr int shared_bytes(bool kQ8, int DP, bool kTall) {
  const int wide = kTall ? kTallStep * (2 * key_stride(DP) + 3 * value_stride(DP))
                         : 2 * wide_positions(DP) * (key_stride(DP) + value_stride(DP)) +
                               (DP > 128 ? kWideRows * key_stride(DP) : 0);
  const int narrow = (kTall ? kTallWaves : kWideWaves) * narrow_positions(kQ8, DP) * narrow_stride(DP);
  return wide > narrow ? wide : narrow;
}

template <bool kF16, bool kQ8, int DP, bool kTall, bool kPad>
__global__ __launch_bounds__(64 * (kTall ? kTallWaves : kWideWaves), DP <= 128 ? 2 : 1) void attend_kernel(AttendArgs a) {
  constexpr int kWaves = kTall ? kTallWaves : kWideWaves;
  __shared__ __align__(16) unsigned char smem[shared_bytes(kQ8, DP, kTall)];
  __shared__ int32_t odd_at[3];
  if (threadIdx.x < 3) odd_at[threadIdx.x] = -1;
  __syncthreads();
  const int32_t head = blockIdx.x % a.cache.heads, group = blockIdx.x / a.cache.heads;
  const int32_t wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const float c = a.scale * 1.44269504088896341f;
  Piece p;
  p.head = head;
  p.c = fabsf(c);
  p.neg = c < 0 ? 0x80008000u : 0u;
  // (scalars throughout: what is loaded after the first store would be a lane's otherwise)
  const AttendHead plan = *a.plan.head;
  const AttendRun run = a.plan.runs[group * kWaves + wave];
  // (nothing to do rather than a return, behind which the loads of the run would wait)
  const int32_t mine = uniform((int32_t)plan_is_for(plan, a.win, kWaves));
  const int32_t kind = uniform(run.kind), rounds = mine ? uniform(run.rounds) : 0, number = uniform(run.number);
  int32_t next = uniform(run.next), at = uniform(run.from), left = mine ? uniform(run.units) : 0;
  bool first = true;
  for (int32_t round = 0;;) {
    int32_t k, from, most, piece;
    if (round < rounds) {
      k = tile_of_round(group, round++, uniform(run.stride));
      from = piece = 0;
      most = INT32_MAX;
    } else {
      if (left <= 0) break;
      k = next++;
      from = at;
      most = left;
      piece = number;
      at = 0;
    }
    AttendTile t = run.tile;
    if (!first) t = a.plan.tiles[kind][k];
    first = false;
    const int32_t t0 = uniform(t.t0), t1 = uniform(t.t1), slot = uniform(t.slot);
    const int32_t n = min(max(0, (t1 - t0 + kUnit - 1) / kUnit) - from, most);
    if (n <= 0) continue;  // (a tile of no positions)
    p.chain.pre_len = uniform(t.pre_len);
    p.chain.pre = a.win.pages + uniform(t.pre_off);
    p.chain.tail = a.win.pages + (uniform(t.tail_off) - p.chain.pre_len);
    p.p0 = uniform(t.p0);
    p.row0 = uniform(t.row0);
    p.rows = uniform(t.rows);
    p.ta = t0 + from * kUnit;
    p.tb = min(t1, t0 + (from + n) * kUnit);
    p.slot = slot < 0 ? -1 : slot + (piece - uniform(t.first)) * p.rows;
    if constexpr (kTall) {
      if (kind == 0) tall_piece<kF16, kQ8, DP, kPad>(a, p, smem, odd_at);
    } else {
      if (kind == 0 && DP <= 128 && p.rows <= 64) wide_piece<kF16, kQ8, DP, kPad, DP <= 128 ? 2 : 1>(a, p, smem, odd_at);
      else if (kind == 0) wide_piece<kF16, kQ8, DP, kPad, 1>(a, p, smem, odd_at);
    }
    if (kind == 1)
      narrow_piece<kF16, kQ8, DP, kPad>(a, p, smem + wave * narrow_positions(kQ8, DP) * narrow_stride(DP));
    if (most != INT32_MAX) left -= n;
  }
}

// Joins the partial results of the plan's list of rows, for each row and key / value
// head, and writes the rows that nothing was computed for.  Where there are no more rows than
// workgroups (a few long contexts, cut into many pieces), a row is a workgroup's: its
// waves take every fourth run of 64 / LG * kAtOnce pieces; otherwise a wave's.  LG lanes
// hold a row of results, so 64 / LG pieces are read at once, kAtOnce times; their maxima
// and sums come with them, one pass with a running maximum.
template <bool kF16, int LG>
__global__ __launch_bounds__(256) void join_kernel(AttendArgs a) {
  constexpr int kAtOnce = 4, kStep = 64 / LG, kRun = kAtOnce * kStep;
  __shared__ f32x4 rows[3][LG];
  __shared__ float2 mls[4];
  const int lane = threadIdx.x & 63, sub = lane / LG, d = 4 * (lane % LG);
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int32_t D = a.cache.dim;
  const AttendHead plan = *a.plan.head;
  if (!plan_is_for(plan, a.win, a.plan.waves)) return;
  const int64_t n = (int64_t)plan.n_joins * a.cache.heads;
  const bool together = n <= gridDim.x;  // (the same for the grid)
  const int64_t first = together ? blockIdx.x : (int64_t)blockIdx.x * 4 + wave;
  for (int64_t id = first; id < n; id += (int64_t)gridDim.x * (together ? 1 : 4)) {
    const AttendJoin x = a.plan.joins[id / a.cache.heads];
    const int32_t head = (int32_t)(id % a.cache.heads);
    const int64_t row = x.row, slots = (int64_t)head * a.plan.slot_rows;
    const bool writes = !together || wave == 0;
    if (x.sub < 0) {
      for (int32_t h = head * a.ratio; writes && h < (head + 1) * a.ratio; ++h) {
        if (sub == 0 && d < D)
          *(u32x2*)(a.out.data + 2 * (row * a.out.row + (int64_t)h * a.out.head + d)) = u32x2{0, 0};
        if (a.lse && lane == 0) a.lse[row * a.heads + h] = -INFINITY;
      }
      continue;
    }
    const int32_t total = x.count[0] + x.count[1];
    auto slot = [&](int32_t j) {
      const bool own = j < x.count[0];
      return slots + (own ? x.from[0] : x.from[1]) + (int64_t)(own ? j : j - x.count[0]) * (own ? x.step[0] : x.step[1]);
    };
    f32x4 acc = {0, 0, 0, 0};
    float m = -INFINITY, l = 0;  // the lane's, of its every kStep-th piece
    for (int32_t j = together ? wave * kRun : 0; j < total; j += together ? 4 * kRun : kRun) {
      f32x4 o[kAtOnce];
      float2 ml[kAtOnce];
#pragma unroll
      for (int u = 0; u < kAtOnce; ++u) {
        const int32_t at = j + u * kStep + sub;
        o[u] = f32x4{0, 0, 0, 0};
        ml[u] = float2{-INFINITY, 0.0f};
        if (at < total) {
          const int64_t s = slot(at);
          ml[u] = a.plan.part_ml[s];
          if (d < D) o[u] = *(const f32x4*)(a.plan.part + s * D + d);
        }
      }
      float nm = m;
#pragma unroll
      for (int u = 0; u < kAtOnce; ++u) nm = fmaxf(nm, ml[u].x);
      const float mc = nm == -INFINITY ? 0.0f : nm, g = __builtin_amdgcn_exp2f(m - mc);
      m = nm;
      l *= g;
      acc *= g;
#pragma unroll
      for (int u = 0; u < kAtOnce; ++u) {
        const float f = __builtin_amdgcn_exp2f(ml[u].x - mc);
        l = __builtin_fmaf(ml[u].y, f, l);
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[e] = __builtin_fmaf(o[u][e], f, acc[e]);
      }
    }
    float top = m;
#pragma unroll
    for (int o = LG; o < 64; o <<= 1) top = fmaxf(top, __shfl_xor(top, o, 64));
    if (together) {
      if (lane == 0) mls[wave].x = top;
      __syncthreads();
      top = fmaxf(fmaxf(mls[0].x, mls[1].x), fmaxf(mls[2].x, mls[3].x));
    }
    const float f = __builtin_amdgcn_exp2f(m - (top == -INFINITY ? 0.0f : top));
    l *= f;
    acc *= f;
#pragma unroll
    for (int o = LG; o < 64; o <<= 1) {
      l += __shfl_xor(l, o, 64);
#pragma unroll
      for (int e = 0; e < 4; ++e) acc[e] += __shfl_xor(acc[e], o, 64);
    }
    if (together) {
      if (wave > 0 && sub == 0) rows[wave - 1][lane % LG] = acc;
      if (lane == 0) mls[wave].y = l;
      __syncthreads();
      l = mls[0].y + mls[1].y + mls[2].y + mls[3].y;
#pragma unroll
      for (int w = 0; w < 3; ++w) acc += rows[w][lane % LG];
      __syncthreads();
    }
    const int32_t h = head * a.ratio + x.sub;
    const float inv = 1.0f / l;
    if (writes && sub == 0 && d < D) {
      u32x2 w = {0, 0};
      if (!x.empty) w = u32x2{pack<kF16>(acc[0] * inv, acc[1] * inv), pack<kF16>(acc[2] * inv, acc[3] * inv)};
      *(u32x2*)(a.out.data + 2 * (row * a.out.row + (int64_t)h * a.out.head + d)) = w;
    }
    if (writes && a.lse && lane == 0)
      a.lse[row * a.heads + h] = x.empty ? -INFINITY : lse_of<kF16>(top, l);
  }
}

template <bool kF16, bool kQ8, int DP, bool kPad>
void launch(const AttendArgs& a, int32_t num_cus, hipStream_t s) {
  const dim3 grid((unsigned)(a.plan.groups * a.cache.heads));
  const dim3 join((unsigned)std::min<int64_t>((int64_t)a.win.n_rows * a.heads, 8 * num_cus));
  if constexpr (DP == 128) {
    if (a.plan.waves == kTallWaves) {
      hipLaunchKernelGGL((attend_kernel<kF16, kQ8, DP, true, kPad>), grid, dim3(64 * kTallWaves), 0, s, a);
      hipLaunchKernelGGL((join_kernel<kF16, DP / 4>), join, dim3(256), 0, s, a);
      return;
    }
  }
  hipLaunchKernelGGL((attend_kernel<kF16, kQ8, DP, false, kPad>), grid, dim3(64 * kWideWaves), 0, s, a);
  hipLaunchKernelGGL((join_kernel<kF16, DP / 4>), join, dim3(256), 0, s, a);
}

template <bool kF16, bool kQ8, int DP>
void launch_dim(const AttendArgs& a, int32_t num_cus, hipStream_t s) {
  if (a.cache.dim < DP) launch<kF16, kQ8, DP, true>(a, num_cus, s);
  else launch<kF16, kQ8, DP, false>(a, num_cus, s);
}

}  // namespace

}  // namespace ps

int32_t ps_attend_per_cu(int32_t dim, bool tall) { return dim <= 128 && !tall ? 2 : 1; }

// Tall tiles where requests have many rows on the average.  They gain where much lies behind the
// rows and lose a little where nothing does, which only the device knows.  Measured with 32 heads over
// 8 (4 rows a token), e4m3, wide and tall: 8 requests of 700 new tokens behind 16384 1728 and 1451
// us, 4 of 512 702 and 581; 4 of 2048 behind 2048 536 and 461, behind none 222 and 206; 16 of 512
// behind none 101 and 114, 24 of 16 to 1500 244 and 259.  (8 heads over 8: 8 of 512 behind 16384 355 and 296.)
// A mean: requests that decode beside a chunk, and those of no rows that pad a window, bring it down.
constexpr int kTallMin = 1024;
bool ps_attend_tall(int32_t dim, int64_t rows, int32_t n_req) {
  return dim > 64 && dim <= 128 && rows >= (int64_t)kTallMin * n_req;
}

hipError_t ps_launch_attend(const ps::AttendArgs& a, int32_t num_cus, hipStream_t s) {
  const bool f16 = a.q.dtype == PS_T_F16, quant = a.cache.dtype == PS_T_E4M3;
#define PS_DIM(F, Q)                                                       \
  do {                                                                     \
    if (a.cache.dim <= 64) ps::launch_dim<F, Q, 64>(a, num_cus, s);        \
    else if (a.cache.dim <= 128) ps::launch_dim<F, Q, 128>(a, num_cus, s); \
    else ps::launch_dim<F, Q, 256>(a, num_cus, s);                         \
  } while (0)
  if (f16 && quant) PS_DIM(true, true);
  else if (f16) PS_DIM(true, false);
  else if (quant) PS_DIM(false, true);
  else PS_DIM(false, false);
#undef PS_DIM
  return hipGetLastError();
}
