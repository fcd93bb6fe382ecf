// The paged 8-bit cache on the device: layout, rotation, conversion; shared by ag_rotate.hip and the ag_q8_*.hip sources.
#pragma once
#include <atomic>

#include "ag_internal.h"

constexpr int kQ8Block = AG_Q8_BLOCK;  // rows of a block, and of a page
constexpr int kQ8MinExp = -100;        // least exponent of a block's scale: 2^-e and every value of a page stay normal numbers
constexpr float kQ8EmptyMax = -3.40282347e+38f;  // reference maximum before any row (no state that holds a row is below it)

// Device view of an ag_rope; table == nullptr: the vectors arrive turned.
struct ag_rope_dev {
  const float *table;  // [n_rows, D]: cosines, then sines
  const int32_t *pos;  // [n_axes, tokens]
  int n_rows, n_axes;
  int end0, end1;      // pairs [0, end0) turn by axis 0, [end0, end1) by axis 1, the others by axis 2
  int quads;           // end0 and end1 are multiples of 4
  int64_t axis_stride; // tokens
};

// Device view of an ag_q8_cache.
struct ag_q8_dev {
  uint8_t *k, *v;            // [n_pages, 64 D]
  float *k_scale, *v_scale;  // [n_pages]
  uint16_t *k_tail, *v_tail; // [units, 64 D] bf16
  const int32_t *page;       // [units, max_blocks]
  int32_t *len;              // [units]
  int n_pages, max_blocks;
};

// A tile of the attention holds f16 numbers times 2^ek (K) and 2^ev (V): 11 bits instead of the 8 of bf16, in which a turned key would
// lose up to 2^-9 of itself.  That needs rows of like size: where a value is not finite or a row's largest one is below 2^-16 of the
// tile's, the tile is `odd`: it holds bf16, and the attention takes it row by row in 32 bits.
struct q8_tile_info {
  int ek, ev;
  bool odd;
};
constexpr int kQ8TileTop = 14;      // a tile's largest number lies in [2^14, 2^15) ...
constexpr int kQ8TileMinExp = -60;  // ... unless that took a smaller exponent than this (sums of 2^-ev stay in range)
constexpr int kQ8TileSpan = 16;
// Weights are f16 relative to a reference that lies this many bits below the largest one when it is set: those down to 2^-22 of it
// keep their 11 bits, those down to 2^-33 some, and a long cache's many small ones are not lost.
constexpr int kQ8TopBits = 8;

// What ag_q8_fill_kernel leaves for the attention of the same call: the unit's cache as it stood before it.
struct ag_q8_meta {
  int32_t blocks, held, added, pad;  // full blocks, rows of the tail, rows that the call appends
};

// ---- launchers ----
hipError_t ag_launch_rotate(ag_ctx *ctx, hipStream_t s, const void *q, const void *k, ag_dtype dt, int B, int Hq, int Hkv, int L,
                            int D, const ag_rope_dev &rope, void *q_out, void *k_out);

// Appends the tokens whose flag is set (flags == nullptr: all).  words, blk_off: where the flags' masks and prefix counts go (as from
// ag_launch_flag_scan; not used without flags).
// tiles != nullptr: also leaves, for the attention, [units, n_blk] tiles of 64 rows of K (turned) and V -- the tail's rows as they stood, then
// the appended ones -- with what they are to be read with (q8_tile_info), and meta [units].
hipError_t ag_launch_q8_fill(ag_ctx *ctx, hipStream_t s, const void *k, const void *v, const uint8_t *flags, int B, int Hkv, int L, int D,
                             uint64_t *words, int32_t *blk_off, const ag_rope_dev &rope, const ag_q8_dev &cache,
                             uint16_t *tiles, uint32_t *info, ag_q8_meta *meta);
size_t ag_ws_q8_decode_floats(int num_cu, int G, int D);  // records of a step
int64_t ag_q8_decode_cost(int64_t units, int max_blocks);  // the largest number that a step's work list can come to; it counts in 32 bits
hipError_t ag_launch_q8_decode(ag_ctx *ctx, hipStream_t s, const void *q, const void *k_new, const void *v_new, const uint8_t *new_flags,
                               int B, int Hq, int Hkv, int D, const ag_rope_dev &rope, float scale, const ag_q8_dev &cache, void *out, float *rec);

struct ag_q8_prefill_ws {
  uint16_t *tiles;      // what ag_launch_q8_fill leaves
  uint32_t *info;
  ag_q8_meta *meta;
  float *part;          // states of the pieces (n_split > 1)
  int n_qt, n_split;    // query tiles of a unit; pieces a query tile's work may be cut into
};
void ag_q8_prefill_plan(int num_cu, int U, int Hq, int Hkv, int L, int D, int max_blocks, ws_cursor &ws, ag_q8_prefill_ws *w);
// The longest call of fewer query tiles than one of L tokens has (0: there is none).  Of calls with equally many the longest needs most.
int ag_q8_prefill_shorter(int Hq, int Hkv, int L);
hipError_t ag_launch_q8_prefill(ag_ctx *ctx, hipStream_t s, const void *q, const void *k, const void *v, int B, int Hq, int Hkv, int L,
                                int D, const uint64_t *words, const int32_t *blk_off, const ag_rope_dev &rope, float scale,
                                const ag_q8_dev &cache, const ag_q8_prefill_ws &w, void *out);

// Dynamic LDS above the default limit: raised once per device and kernel, to the most that the kernel can need (a limit that
// followed each call could be lowered by one thread under another one's launch).
template <typename K> static inline hipError_t ag_q8_allow_lds(int device, std::atomic<bool> *allowed, K kernel, size_t most) {
  if (allowed[device & 63].load(std::memory_order_relaxed)) return hipSuccess;
  const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void *>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, (int)most);
  if (e == hipSuccess) allowed[device & 63].store(true, std::memory_order_relaxed);
  return e;
}

static inline int ag_q8_fill_blocks(int L) { return (kQ8Block - 1 + L + kQ8Block - 1) / kQ8Block; }  // blocks that tail and tokens can touch

#ifdef __HIPCC__
typedef __attribute__((__vector_size__(8 * sizeof(__bf16)))) __bf16 q8_bf16x8;
typedef __attribute__((__vector_size__(2 * sizeof(__bf16)))) __bf16 q8_bf16x2;
typedef __attribute__((__vector_size__(8 * sizeof(_Float16)))) _Float16 q8_f16x8;
typedef __attribute__((__vector_size__(2 * sizeof(_Float16)))) _Float16 q8_f16x2;
typedef __attribute__((__vector_size__(2 * sizeof(float)))) float q8_f32x2;
typedef __attribute__((__vector_size__(4 * sizeof(float)))) float q8_f32x4;
typedef __attribute__((__vector_size__(16 * sizeof(float)))) float q8_f32x16;
typedef __attribute__((__vector_size__(4 * sizeof(uint32_t)))) uint32_t q8_u32x4;
typedef __attribute__((__vector_size__(2 * sizeof(int16_t)))) int16_t q8_s16x2;
typedef __attribute__((__vector_size__(2 * sizeof(uint16_t)))) uint16_t q8_u16x2;

// Two floats to bf16, round to nearest even, lo in the lower half.
__device__ __forceinline__ uint32_t q8_pack2(float lo, float hi) {
  const q8_f32x2 x = {lo, hi};
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(x, q8_bf16x2));
}
__device__ __forceinline__ float q8_lo(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float q8_hi(uint32_t w) { return __uint_as_float(w & 0xffff0000u); }

// Eight codes (two words) times a power of two as f16: exact, a code has 4 significant bits.
__device__ __forceinline__ q8_f16x8 q8_widen16(uint32_t a, uint32_t b, float scale) {
  const uint4 w = {__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(a, scale, false)),
                   __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(a, scale, true)),
                   __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(b, scale, false)),
                   __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(b, scale, true))};
  return __builtin_bit_cast(q8_f16x8, w);
}
// Four bf16 (two words) times inv = 2^-e (exact) to codes, round to nearest even; what is not finite becomes NaN.
__device__ __forceinline__ uint32_t q8_narrow(uint32_t a, uint32_t b, float inv) {
  auto f = [&](float x) {
    const float y = x * inv;
    return fabsf(y) <= 448.f ? y : __uint_as_float(0x7fc00000u);
  };
  int w = __builtin_amdgcn_cvt_pk_fp8_f32(f(q8_lo(a)), f(q8_hi(a)), 0, false);
  return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(f(q8_lo(b)), f(q8_hi(b)), w, true);
}
// The same for values known to be finite, of which none passes 448 scale = 448 2^e.
__device__ __forceinline__ uint32_t q8_narrow_finite(uint32_t a, uint32_t b, float scale) {
  q8_s16x2 w = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(q8_s16x2{}, __builtin_bit_cast(q8_bf16x2, a), scale, false);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(w, __builtin_bit_cast(q8_bf16x2, b), scale, true);
  return __builtin_bit_cast(uint32_t, w);
}
// The larger of m and the magnitudes (as bits) of the two bf16 of a word; infinities and NaN do not count.
__device__ __forceinline__ uint32_t q8_top(uint32_t m, uint32_t w) {
  const uint32_t a = w & 0x7fffu, b = (w >> 16) & 0x7fffu;
  m = max(m, a < 0x7f80u ? a : 0u);
  return max(m, b < 0x7f80u ? b : 0u);
}
// Exponent of a block whose largest magnitude is the bf16 `top`: the least e >= kQ8MinExp with top 2^-e <= 448 = 1.75 2^8.
__device__ __forceinline__ int q8_exponent(uint32_t top) {
  const int e = (int)(top >> 7) - 127 - ((top & 127u) <= 96u ? 8 : 7);
  return max(kQ8MinExp, e);
}
__device__ __forceinline__ uint32_t q8_tile_word(int ek, int ev, bool odd) { return (uint32_t)(ek + 128) | (uint32_t)(ev + 128) << 8 | (uint32_t)odd << 16; }
__device__ __forceinline__ q8_tile_info q8_tile_of(uint32_t w) { return q8_tile_info{(int)(w & 255) - 128, (int)(w >> 8 & 255) - 128, (w >> 16 & 1) != 0}; }
__device__ __forceinline__ float q8_pow2(int e) { return __uint_as_float((uint32_t)(e + 127) << 23); }

// Where the 16 bytes (codes; 32 bytes in a bf16 tail) of a row's columns 16 x .. or a column's rows lie, in units of 16 values:
//   K: rows 16 a + r, columns 64 c + 16 g ..          -> ((a D / 64 + c) 4 + g) 16 + r
//   V: column 16 f + r, rows 16 i + 4 g + 0..3, i < 4 -> (f 4 + g) 16 + r
// In this order a wave's load of 1 KiB of a page is an A operand of K q^T (V^T p^T), without a trip through LDS.
template <int D> __device__ __forceinline__ int q8_k_at(int t, int c, int g) { return ((((t >> 4) * (D / 64)) + c) * 4 + g) * 16 + (t & 15); }

// ---- rotation ----
struct q8_rows {
  uint32_t r0, r1, r2;  // the table's rows of a token's positions
};
__device__ __forceinline__ uint32_t q8_rope_row(const ag_rope_dev &r, int axis, int64_t token, int32_t *err) {
  const int p = r.pos[axis * r.axis_stride + token];
  if ((uint32_t)p < (uint32_t)r.n_rows) return p;
  atomicOr(err, 2);  // reported, and turned by the nearest row there is
  return p < 0 ? 0 : r.n_rows - 1;
}
__device__ __forceinline__ q8_rows q8_rope_rows(const ag_rope_dev &r, int64_t token, int32_t *err) {
  q8_rows at;
  at.r0 = q8_rope_row(r, 0, token, err);
  at.r1 = r.n_axes > 1 ? q8_rope_row(r, 1, token, err) : at.r0;
  at.r2 = r.n_axes > 2 ? q8_rope_row(r, 2, token, err) : at.r0;
  return at;
}
// Cosines and sines of pairs i .. i + 3 (i a multiple of 4) of a token.
struct q8_angles {
  float4 c, s;
};
__device__ __forceinline__ const float *q8_angle_row(const ag_rope_dev &r, const q8_rows &at, int i, int D) {
  return r.table + (size_t)(i < r.end0 ? at.r0 : (i < r.end1 ? at.r1 : at.r2)) * D;
}
__device__ __forceinline__ q8_angles q8_angles4(const ag_rope_dev &r, const q8_rows &at, int i, int D) {  // (four that turn by one axis)
  const float *a = q8_angle_row(r, at, i, D) + i;
  return q8_angles{*reinterpret_cast<const float4 *>(a), *reinterpret_cast<const float4 *>(a + D / 2)};
}
// One value of a pair: x its own, p the other one; lower: x is the first of the two.  Both products and the sum are rounded by
// themselves (no fused multiply-add): the value does not depend on which half is computed where.
__device__ __forceinline__ float q8_turn(float x, float p, float c, float s, bool lower) {
#pragma clang fp contract(off)
  const float a = x * c, b = p * s;
  return lower ? a - b : a + b;
}
// What products of numbers 2^-e as large are multiplied by: scale 2^e, but neither 0 nor infinite, so that a product of 0 stays 0 and one that
// is infinite an infinity.
__device__ __forceinline__ float q8_unscale(float scale, int e) { return __builtin_amdgcn_fmed3f(ldexpf(scale, e), 1.17549435e-38f, 3.40282347e+38f); }
// The two f16 of a word added to x.
__device__ __forceinline__ float q8_add2(uint32_t w, float x) {
  const q8_f16x2 one = {(_Float16)1.f, (_Float16)1.f};
  return __builtin_amdgcn_fdot2(__builtin_bit_cast(q8_f16x2, w), one, x, false);
}
// Eight values of a vector in 32 bits.
struct q8_eight {
  q8_f32x4 a, b;
  __device__ __forceinline__ uint4 bf16() const { return make_uint4(q8_pack2(a[0], a[1]), q8_pack2(a[2], a[3]), q8_pack2(b[0], b[1]), q8_pack2(b[2], b[3])); }
  __device__ __forceinline__ float top() const {
    return fmaxf(fmaxf(fmaxf(fabsf(a[0]), fabsf(a[1])), fmaxf(fabsf(a[2]), fabsf(a[3]))), fmaxf(fmaxf(fabsf(b[0]), fabsf(b[1])), fmaxf(fabsf(b[2]), fabsf(b[3]))));
  }
  __device__ __forceinline__ q8_f16x8 f16(float scale) const {
    const q8_f32x4 x = a * scale, y = b * scale;
    return __builtin_convertvector(__builtin_shufflevector(x, y, 0, 1, 2, 3, 4, 5, 6, 7), q8_f16x8);
  }
};
__device__ __forceinline__ q8_eight q8_floats(const uint4 &x) {
  return q8_eight{{q8_lo(x.x), q8_hi(x.x), q8_lo(x.y), q8_hi(x.y)}, {q8_lo(x.z), q8_hi(x.z), q8_lo(x.w), q8_hi(x.w)}};
}
// Eight values x of a vector turned, whose partners are p; a: four cosines, their sines, the next four cosines, their sines; lower: they
// are of the vector's first half.
__device__ __forceinline__ q8_eight q8_turn8(const q8_f32x4 (&a)[4], bool lower, const uint4 &x, const uint4 &p) {
  const q8_eight u = q8_floats(x), w = q8_floats(p);
  q8_eight y;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    y.a[i] = q8_turn(u.a[i], w.a[i], a[0][i], a[1][i], lower);
    y.b[i] = q8_turn(u.b[i], w.b[i], a[2][i], a[3][i], lower);
  }
  return y;
}
// Values d .. d + 7 (x) of a vector of D turned, whose partners are p; angles(i): those of pairs i .. i + 3.
template <int D, typename A> __device__ __forceinline__ q8_eight q8_turn8(A &&angles, int d, const uint4 &x, const uint4 &p) {
  const q8_angles e = angles(d & (D / 2 - 1)), f = angles((d & (D / 2 - 1)) + 4);
  const q8_f32x4 a[4] = {{e.c.x, e.c.y, e.c.z, e.c.w}, {e.s.x, e.s.y, e.s.z, e.s.w}, {f.c.x, f.c.y, f.c.z, f.c.w}, {f.s.x, f.s.y, f.s.z, f.s.w}};
  return q8_turn8(a, d < D / 2, x, p);
}
#endif
