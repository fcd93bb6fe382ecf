// One decoding step over the paged 8-bit cache, in one launch: attention of every sequence's new token over the rows its units hold
// and itself, and its append (q and the new key turned on the way).
//
// A step reads every page it attends to once: large steps are bound by HBM, small ones by dependent round trips.  The kernel builds
// its own work list from len[] and hands data between workgroups only where a unit is too long for one.
//   * Work is counted in items of one unit: one for the tail and the new token, then its pages.  A wave takes every NW-th item of its
//     workgroup's segment.
//   * A page holds 64 rows in the order of the matrix operands, so its 16-byte pieces go from memory into registers and there, made
//     f16 (exact, two values an instruction), into S^T = K q^T and O^T = V^T p^T on v_mfma_f32_16x16x32_f16: no LDS, no barrier.  A wave has
//     two pages in flight, 16 to 32 KiB; a piece's registers are asked for again as soon as it is used up.
//   * Queries are f16 times a power of two per row, weights are f16 relative to a reference that is moved only when their sum passes 2^15:
//     11 bits of each, as the codes have 4; row sums add up the rounded weights.  The reference lies 2^-8 below the largest of the page that set it,
//     so weights down to 2^-33 of that count; in the wave that has the tail the tail sets it, and those down to 2^-21 do.  (A weight in three
//     bf16 parts in the columns that G < 16 leaves idle kept 24 bits: 32 sequences of 32 heads 533 us a 4 steps, now 443; output rows are off by 1.7e-3 of
//     their size either way, which the store's rounding gives.)
//   * The workgroup turns its queries and the new key together, into LDS: a lane's own row by itself took 64 lines a load.  The barrier
//     after it waits for LDS alone, and the pages are asked for behind it: ahead of it they held up the small loads.
//   * The tail is a page in bf16; the new token's row is put into it in registers, so that it is one row more.  The wave that has it also
//     stores that row, or, if it is the block's last, the whole block in 8 bits.  Its own score takes what rounding its key to bf16 leaves over
//     as one more product: without, scores of 7 times the usual spread put rows off by 2e-2 of their size, now by 4.6e-3.
//   * 32 sequences of 32 heads over 400 to 4096 rows: 111 us a step, 5.1 TB/s of pages; a chat of 8 heads and hundreds of rows: 10 us, of
//     which the launch and about six dependent round trips are all.
//   * Segments: if the whole step gives every workgroup at most one piece of a unit (a few rounds of its waves), those; if there are more
//     units than workgroups and all are short, one, two or four waves a unit; else all items end to end, in equal ranges.
#include <algorithm>
#include <type_traits>

#include "ag_q8.h"

namespace {

constexpr float kLog2e = 1.4426950408889634f;
// Up to here 8 waves per workgroup and one workgroup per CU: a unit's items are spread over as many waves as the registers allow, and the
// work list is held in them; beyond, 4 waves and two workgroups per CU, so that one streams while the other starts or merges.  A step with 8
// (4) waves: 8 units of 13000 rows 16.3 (25.1) us, 32 of 777 16.6 (17.9), 128 of 8000 37.2 (39.6).
constexpr int kFewUnits = 128;
// Items of a wave up to which a unit is not cut: the meeting of the pieces costs as much as a round (64 units of 2000 rows 16.5 us, with 4
// 19.4).
constexpr int kWholeRounds = 2;
constexpr int kValueBits = 9;     // a page's values in f16 are below 1 (exact: a code has 4 bits, the least is 2^-9), as the tail's are of unit size
// Bits by which a page's reference may lie below the one that a tail has left: its weights are then 2^-4 at most, and those down to 2^-21 of
// the largest count.  (Values of unit size: 5.  Coming down costs a step of few rows 0.5 us of 9.7.)
constexpr float kHighBits = kQ8TopBits + 4;
constexpr int kArriveSplit = 64;  // workgroups from which their arrivals are counted at several addresses
// What a unit costs a workgroup beside its items, in items, where all units are cut into equal ranges: the start of a segment, the tail's two
// bytes a value, the merge.  Without it the ranges that hold the most units end last (a step with 0, 7, 14, 28: 128 units of 8000 rows 41.5,
// 37.5, 35.1, 37.1 us, 256 of 4096 48, 43, 41, 42.5).
constexpr int kUnitCost = 14;
// Items of a wave up to which units are given to teams of waves (1024 units of 300 rows 25.6 us, of 700 32.3; cut into ranges 36.4 and 40.8).
constexpr int kTeamRounds = 6;

struct dec_args {
  const uint16_t *q, *k_new, *v_new;
  const uint8_t *new_flags;
  uint16_t *out;
  ag_q8_dev c;
  ag_rope_dev rope;
  float *rec;        // records [id][G][D + 2]
  int32_t *tickets;  // [U] pieces of a unit that have stored their record; zero between launches
  int32_t *arrived;  // workgroups that have read len[]; zero between launches
  int32_t *err;
  int U, Hkv;
  float qscale;
};

__device__ __forceinline__ void put_pair(float *p, float a, float b) {
  __hip_atomic_store(reinterpret_cast<uint64_t *>(p), (uint64_t)__float_as_uint(a) | ((uint64_t)__float_as_uint(b) << 32),
                     __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_SYSTEM);
}
__device__ __forceinline__ float2 get_pair(const float *p) {
  const uint64_t x = __hip_atomic_load(reinterpret_cast<const uint64_t *>(p), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_SYSTEM);
  return make_float2(__uint_as_float((uint32_t)x), __uint_as_float((uint32_t)(x >> 32)));
}
// Over the wave's lanes (register exchanges: no addresses that live in registers, as lane shuffles have them)
__device__ __forceinline__ uint32_t wave_max(uint32_t x) {
  auto dpp = [](uint32_t y, auto ctrl) { return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)y, decltype(ctrl)::value, 0xf, 0xf, false); };
  x = max(x, dpp(x, std::integral_constant<int, 0xB1>{}));   // quad_perm [1,0,3,2]
  x = max(x, dpp(x, std::integral_constant<int, 0x4E>{}));   // quad_perm [2,3,0,1]
  x = max(x, dpp(x, std::integral_constant<int, 0x141>{}));  // row_half_mirror
  x = max(x, dpp(x, std::integral_constant<int, 0x140>{}));  // row_mirror
  const auto a = __builtin_amdgcn_permlane16_swap(x, x, false, false);
  x = max((uint32_t)a[0], (uint32_t)a[1]);
  const auto b = __builtin_amdgcn_permlane32_swap(x, x, false, false);
  return __builtin_amdgcn_readfirstlane(max((uint32_t)b[0], (uint32_t)b[1]));
}
// Over the four lanes that share lane % 16
__device__ __forceinline__ float kg_max(float x) {
  const auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  x = fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
  const auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return fmaxf(__uint_as_float(b[0]), __uint_as_float(b[1]));
}
__device__ __forceinline__ float kg_sum(float x) {
  const auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  x = __uint_as_float(a[0]) + __uint_as_float(a[1]);
  const auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return __uint_as_float(b[0]) + __uint_as_float(b[1]);
}
// x as bf16 in the lower half of a word, what is left of it as bf16 in the upper one
__device__ __forceinline__ float in_two(float x) {
  const float first = q8_lo(q8_pack2(x, 0.f));
  return __uint_as_float(q8_pack2(first, fabsf(first) < INFINITY ? x - first : 0.f));
}
// x of the lane N columns further (of 16, cyclic)
template <int N> __device__ __forceinline__ float column(float x) {
  return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), 0x120 + (16 - N), 0xf, 0xf, false));
}

template <int D, int G> struct wave_q8 {
  static constexpr int KC = D / 64, KF = 4 * KC, VF = D / 16;
  static constexpr int P = G <= 4 ? 4 : 8;
  static constexpr int SF = D + 4;  // floats per head of the state a wave leaves: max, sum, -, -, o
  q8_f16x8 qf[KC][2];
  int eq;                           // qf: the query times 2^-eq
  q8_f32x4 o[VF];
  float m, l;
  int lane, g, col, head;
  bool second;                      // (columns P and up: what a weight of the tail leaves over)

  __device__ __forceinline__ void init(int lane_) {
    lane = lane_; g = lane >> 4; col = lane & 15; head = col % P; second = col >= P;
    m = kQ8EmptyMax; l = 0.f; eq = 0;
#pragma unroll
    for (int f = 0; f < VF; ++f) o[f] = q8_f32x4{0.f, 0.f, 0.f, 0.f};
  }
  // The query (turned, 32 bits, in LDS) in f16 (11 bits: a turned one in bf16 would shift the scores by 2^-9 of their size), its largest value in
  // [2^14, 2^15)
  __device__ __forceinline__ void query(const float *x) {
    q8_eight y[KC][2];
    float top = 0.f;
#pragma unroll
    for (int c = 0; c < KC; ++c)
#pragma unroll
      for (int s = 0; s < 2; ++s) {
        y[c][s] = eight_at(x, c, s);
        top = fmaxf(top, y[c][s].top());
      }
    top = kg_max(top);
    eq = max(kQ8TileMinExp, min(254, max(1, (int)(__float_as_uint(top) >> 23))) - 127 - kQ8TileTop);
    const float inv = q8_pow2(-eq);
#pragma unroll
    for (int c = 0; c < KC; ++c)
#pragma unroll
      for (int s = 0; s < 2; ++s) qf[c][s] = y[c][s].f16(inv);
  }
  __device__ __forceinline__ q8_eight eight_at(const float *x, int c, int s) const {  // this lane's eight values of a vector
    const q8_f32x4 *p = reinterpret_cast<const q8_f32x4 *>(x + 64 * c + 16 * g + 8 * s);
    return q8_eight{p[0], p[1]};
  }

  // A new reference for the scores (their tile's exponent included): everything so far shrinks to it.
  __device__ __forceinline__ void raise(float m_new) {
    if (__any(m_new != m)) {
      const float alpha = __builtin_amdgcn_exp2f(m - m_new);
      l *= alpha;
#pragma unroll
      for (int f = 0; f < VF; ++f) o[f] *= alpha;
      m = m_new;
    }
  }

  // How far the reference may come down: the state grows by as much, and must not overflow (what is not finite already stays so).
  __device__ __forceinline__ float lower() const {
    float top = 0.f;
#pragma unroll
    for (int f = 0; f < VF; ++f)
#pragma unroll
      for (int r = 0; r < 4; ++r) top = fmaxf(top, fabsf(o[f][r]) < INFINITY ? fabsf(o[f][r]) : 0.f);
    return (float)max(0, min(-kQ8TileMinExp, 127 + 120 - (int)(wave_max(__float_as_uint(top)) >> 23)));
  }

  // A wave's pages: lane x holds the number and the exponents of its page x (of at most 64 at a time); two pages are in flight.
  int ids, ek_v, ev_v;
  // (The same registers hold a tail instead: as long as the two were told apart the compiler kept room for both.)
  q8_u32x4 buf[4 * KF];  // K of two pages, V of two pages; or a tail's K, V
  uint32_t nv[VF / 2];   // this lane's values of the new token, two a register
  __device__ __forceinline__ void numbers(const int32_t *page, int i0, int i1, int step) {
    const int i = i0 + lane * step;
    ids = i < i1 ? page[i] : -1;
  }
  __device__ __forceinline__ void exponents(const ag_q8_dev &c) {
    const bool ok = (uint32_t)ids < (uint32_t)c.n_pages;  // (a number outside the pool: rows that are not there)
    const int id = ok ? ids : 0;
    ek_v = (int)(__float_as_uint(c.k_scale[id]) >> 23) - 127;
    ev_v = (int)(__float_as_uint(c.v_scale[id]) >> 23) - 127;
    ids = ok ? ids : -1;
  }
  template <int AT> __device__ __forceinline__ void load(const uint8_t *pool, int x) {  // every page is read once per step: non-temporal
    const int id = max(0, __builtin_amdgcn_readlane(ids, x));
    const __amdgpu_buffer_rsrc_t rsrc = __builtin_amdgcn_make_buffer_rsrc((void *)(pool + (size_t)id * (kQ8Block * D)), 0, kQ8Block * D, 0x00020000);
#pragma unroll
    for (int f = 0; f < KF; ++f) buf[AT + f] = __builtin_amdgcn_raw_buffer_load_b128(rsrc, lane * 16 + (f & 3) * 1024, f / 4 * 4096, 2);
  }
  __device__ __forceinline__ void first_pages(const ag_q8_dev &c, int n) {
    load<0>(c.k, 0);
    load<2 * KF>(c.v, 0);
    if (n > 1) {
      load<KF>(c.k, 1);
      load<3 * KF>(c.v, 1);
    }
  }
  // Page x of n, which is in buffer B; that buffer's next one is asked for.  The state is kept relative to m, the largest score plus its page's
  // exponent ev of V less kQ8TopBits: a page's weights are 2^(score + ev - m) in f16, its values the codes 2^-kValueBits, its part of the row
  // sum 2^-ev the sum of its weights (as the product takes them: what rounding them changes cancels).
  template <int B> __device__ __forceinline__ void one_page(const ag_q8_dev &c, int x, int n, float qscale, bool &fresh) {
    const bool more = x + 2 < n, now = __builtin_amdgcn_readlane(ids, x) >= 0;
    q8_f32x4 s[4];
#pragma unroll
    for (int a = 0; a < 4; ++a) {
      s[a] = q8_f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int cc = 0; cc < KC; ++cc)
#pragma unroll
        for (int h = 0; h < 2; ++h)
          s[a] = __builtin_amdgcn_mfma_f32_16x16x32_f16(q8_widen16(buf[B * KF + a * KC + cc][2 * h], buf[B * KF + a * KC + cc][2 * h + 1], 1.f), qf[cc][h], s[a], 0, 0, 0);
    }
    if (more) load<B * KF>(c.k, x + 2);
    if (now) {
      const int e = __builtin_amdgcn_readlane(ev_v, x), ev = max(kQ8TileMinExp, e + kValueBits);
      const float f = q8_unscale(qscale, eq + __builtin_amdgcn_readlane(ek_v, x));
      float sum;
      uint32_t w[8];
      auto largest = [&] {
        float mx = s[0][0];
#pragma unroll
        for (int y = 1; y < 16; ++y) mx = fmaxf(mx, s[y >> 2][y & 3]);
        return fmaf(kg_max(mx), f, (float)(ev - kQ8TopBits));
      };
      auto weigh = [&] {
        const float off = (float)ev - m;
        float part[2] = {0.f, 0.f};
#pragma unroll
        for (int y = 0; y < 8; ++y) {
          const q8_f32x2 p = {__builtin_amdgcn_exp2f(fmaf(s[y >> 1][2 * (y & 1)], f, off)), __builtin_amdgcn_exp2f(fmaf(s[y >> 1][2 * (y & 1) + 1], f, off))};
          w[y] = __builtin_bit_cast(uint32_t, __builtin_convertvector(p, q8_f16x2));
          part[y & 1] = q8_add2(w[y], part[y & 1]);
        }
        sum = part[0] + part[1];
      };
      if (fresh) {
        // The wave's first page.  The reference that a tail has left is a score without an exponent: where the values are small it is too high
        // for a page's weights in f16, and comes down (the state is in 32 bits).
        const float mx = largest();
        raise(fmaxf(mx, __builtin_expect(__any(mx < m - kHighBits), 0) ? m - lower() : m));
      }
      fresh = false;
      weigh();
      // no maximum in the common case: only where weights pass 2^15 is the reference moved (for that head alone)
      if (__any(!(sum <= 32768.f))) {
        const float m_new = fmaxf(m, largest());
        raise(kg_max(sum <= 32768.f ? 0.f : 1.f) > 0.f ? m_new : m);
        weigh();
      }
      l += ldexpf(sum, -ev);
      const float scale = q8_pow2(e - ev);
#pragma unroll
      for (int y = 0; y < 8; ++y) w[y] = second ? 0u : w[y];
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const q8_f16x8 pb = __builtin_bit_cast(q8_f16x8, make_uint4(w[4 * h], w[4 * h + 1], w[4 * h + 2], w[4 * h + 3]));
#pragma unroll
        for (int y = 0; y < VF; ++y)
          o[y] = __builtin_amdgcn_mfma_f32_16x16x32_f16(q8_widen16(buf[(2 + B) * KF + y][2 * h], buf[(2 + B) * KF + y][2 * h + 1], scale), pb, o[y], 0, 0, 0);
      }
    }
    if (more) load<(2 + B) * KF>(c.v, x + 2);
  }
  // Pages i0, i0 + step, ... < i1 of a unit; the numbers and exponents of the first 64 are there, and up to two pages are asked for.
  __device__ __forceinline__ void pages(const ag_q8_dev &c, const int32_t *page, int i0, int i1, int step, float qscale) {
    bool fresh = true;
    for (;;) {
      const int n = min(64, (i1 - i0 + step - 1) / step);
      for (int x = 0; x < n; x += 2) {
        one_page<0>(c, x, n, qscale, fresh);
        if (x + 1 < n) one_page<1>(c, x + 1, n, qscale, fresh);
      }
      i0 += 64 * step;
      if (i0 >= i1) break;
      numbers(page, i0, i1, step);
      exponents(c);
      first_pages(c, min(64, (i1 - i0 + step - 1) / step));
    }
  }

  // The tail's n rows and the new token as row n (its turned key in LDS, in_two); `append`: the new row stays.  The rows are bf16
  // of any size, so these products are in bf16: the query and the weights as the sum of two numbers each (the weights' second one
  // in the columns P further, which are idle otherwise).
  __device__ __forceinline__ void fetch_tail(const dec_args &a, int u, int n) {
    const uint16_t *kt = a.c.k_tail + (size_t)u * kQ8Block * D, *vt = a.c.v_tail + (size_t)u * kQ8Block * D;
    // rows that are not there are not read (addresses past the descriptor's end give zeros)
    auto rsrc_of = [](const uint16_t *p) { return __builtin_amdgcn_make_buffer_rsrc((void *)p, 0, kQ8Block * D * 2, 0x00020000); };
    auto load = [](__amdgpu_buffer_rsrc_t rsrc, int at, bool there) {
      return __builtin_amdgcn_raw_buffer_load_b128(rsrc, there ? at : 1 << 24, 0, 0);
    };
    const __amdgpu_buffer_rsrc_t k_rsrc = rsrc_of(kt), v_rsrc = rsrc_of(vt);
#pragma unroll
    for (int x = 0; x < 4; ++x)
#pragma unroll
      for (int c = 0; c < KC; ++c)
#pragma unroll
        for (int s = 0; s < 2; ++s) buf[(x * KC + c) * 2 + s] = load(k_rsrc, ((x * KC + c) * 64 + lane) * 32 + 16 * s, 16 * x + col < n);
#pragma unroll
    for (int f = 0; f < VF; ++f)
#pragma unroll
      for (int i = 0; i < 2; ++i) buf[2 * KF + 2 * f + i] = load(v_rsrc, (f * 64 + lane) * 32 + 16 * i, 32 * i + 4 * g < n);
    const uint16_t *vn = a.v_new + (size_t)u * D;
#pragma unroll
    for (int f = 0; f < VF / 2; ++f) nv[f] = (uint32_t)vn[32 * f + col] | (uint32_t)vn[32 * f + 16 + col] << 16;
  }
  __device__ __forceinline__ void tail(const dec_args &a, int u, int n, int block, bool append, const uint32_t *new_key) {
    uint16_t *kt = a.c.k_tail + (size_t)u * kQ8Block * D, *vt = a.c.v_tail + (size_t)u * kQ8Block * D;
    auto kr = [&](int x, int c, int s) -> q8_u32x4 & { return buf[(x * KC + c) * 2 + s]; };
    auto vr = [&](int f, int i) -> q8_u32x4 & { return buf[2 * KF + 2 * f + i]; };
    q8_u32x4 nk[KC][2], nl[KC][2];  // the new key as it is held, and (in its row's lanes) what that rounding left over: its score is not off by it
#pragma unroll
    for (int c = 0; c < KC; ++c)
#pragma unroll
      for (int s = 0; s < 2; ++s) {
        const q8_u32x4 *p = reinterpret_cast<const q8_u32x4 *>(new_key + 64 * c + 16 * g + 8 * s);
        const q8_u32x4 x[2] = {p[0], p[1]};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const uint32_t even = x[i / 2][2 * (i & 1)], odd = x[i / 2][2 * (i & 1) + 1];
          nk[c][s][i] = __builtin_amdgcn_perm(odd, even, 0x05040100u);
          nl[c][s][i] = col == (n & 15) ? __builtin_amdgcn_perm(odd, even, 0x07060302u) : 0u;
        }
      }
    // the new row joins: row n = 16 (n / 16) + col for K, = 16 i + 4 g + n % 4 for V
#pragma unroll
    for (int x = 0; x < 4; ++x)
      if (16 * x + col == n) {
#pragma unroll
        for (int c = 0; c < KC; ++c)
#pragma unroll
          for (int s = 0; s < 2; ++s) kr(x, c, s) = nk[c][s];
      }
    const bool fills = append && n == kQ8Block - 1;  // the block is full: it goes to its page; else the row joins the tail
    if (append && !fills && col == (n & 15)) {
#pragma unroll
      for (int c = 0; c < KC; ++c)
#pragma unroll
        for (int h = 0; h < 2; ++h) *reinterpret_cast<q8_u32x4 *>(kt + q8_k_at<D>(n, c, g) * 16 + 8 * h) = nk[c][h];
    }
    q8_f32x4 s[4], s_new = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int x = 0; x < 4; ++x) s[x] = q8_f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int c = 0; c < KC; ++c)
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const q8_f16x8 q = qf[c][h];
        const q8_eight y = {{(float)q[0], (float)q[1], (float)q[2], (float)q[3]}, {(float)q[4], (float)q[5], (float)q[6], (float)q[7]}};
        const uint4 hi = y.bf16();
        const q8_eight z = q8_floats(hi);
        const q8_bf16x8 qh = __builtin_bit_cast(q8_bf16x8, hi), ql = __builtin_bit_cast(q8_bf16x8, q8_eight{y.a - z.a, y.b - z.b}.bf16());
#pragma unroll
        for (int x = 0; x < 4; ++x) {
          const q8_bf16x8 k = __builtin_bit_cast(q8_bf16x8, kr(x, c, h));
          s[x] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k, ql, s[x], 0, 0, 0);
          s[x] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k, qh, s[x], 0, 0, 0);
        }
        s_new = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(q8_bf16x8, nl[c][h]), qh, s_new, 0, 0, 0);
      }
    const float f = q8_unscale(a.qscale, eq);
    float mx = -INFINITY;
#pragma unroll
    for (int x = 0; x < 4; ++x)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int row = 16 * x + 4 * g + i;
        s[x][i] = (x == n / 16 ? s[x][i] + s_new[i] : s[x][i]) * f;
        if (row > n) s[x][i] = -INFINITY;
        // the new token: alone its weight is 1 whatever its score is; a score that overflowed to -infinity counts as the least number
        if (row == n) s[x][i] = n == 0 && block == 0 ? 0.f : (s[x][i] < kQ8EmptyMax ? kQ8EmptyMax : s[x][i]);
        mx = fmaxf(mx, s[x][i]);
      }
    auto narrow = [](const q8_u32x4 &x, const q8_u32x4 &y, float inv) {
      return q8_u32x4{q8_narrow(x[0], x[1], inv), q8_narrow(x[2], x[3], inv), q8_narrow(y[0], y[1], inv), q8_narrow(y[2], y[3], inv)};
    };
    auto top4 = [](uint32_t top, const q8_u32x4 &w) { return q8_top(q8_top(q8_top(q8_top(top, w[0]), w[1]), w[2]), w[3]); };
    const int id = fills ? a.c.page[(size_t)u * a.c.max_blocks + block] : 0;
    if (fills) {
      uint32_t top = 0;
#pragma unroll
      for (int x = 0; x < 4; ++x)
#pragma unroll
        for (int c = 0; c < KC; ++c) top = top4(top4(top, kr(x, c, 0)), kr(x, c, 1));
      const int e = q8_exponent(wave_max(top));
      const float inv = q8_pow2(-e);
      q8_u32x4 *to = reinterpret_cast<q8_u32x4 *>(a.c.k + (size_t)id * kQ8Block * D) + lane;
#pragma unroll
      for (int x = 0; x < 4; ++x)
#pragma unroll
        for (int c = 0; c < KC; ++c) to[(x * KC + c) * 64] = narrow(kr(x, c, 0), kr(x, c, 1), inv);
      if (lane == 0) a.c.k_scale[id] = q8_pow2(e);
    }
    raise(fmaxf(m, kg_max(mx)));
    // A weight's first part is the first 16 bits of a number just below it, its second one what is left, rounded: both are positive
    // where the weight is not 0, so that an infinite value comes out with its sign.
    uint32_t w[8];
#pragma unroll
    for (int x = 0; x < 16; x += 2) {
      float p[2];
#pragma unroll
      for (int y = 0; y < 2; ++y) {
        p[y] = __builtin_amdgcn_exp2f(s[x >> 2][(x & 3) + y] - m);
        l += p[y];
        const float first = __uint_as_float(__builtin_elementwise_sub_sat(__float_as_uint(p[y]), 1u) & 0xffff0000u);
        p[y] = second ? p[y] - first : first;
      }
      w[x / 2] = q8_pack2(p[0], p[1]);
    }
    uint32_t old[8], mine[8];  // halves of word y (rows 16 (y / 2) + 4 g + 2 (y % 2) + 0, 1) that are rows before n, and row n
#pragma unroll
    for (int y = 0; y < 8; ++y) {
      const int row = 16 * (y / 2) + 4 * g + 2 * (y & 1);
      old[y] = (row < n ? 0xffffu : 0u) | (row + 1 < n ? 0xffff0000u : 0u);
      mine[y] = (row == n ? 0xffffu : 0u) | (row + 1 == n ? 0xffff0000u : 0u);
    }
#pragma unroll
    for (int f = 0; f < VF; ++f) {
      const uint32_t two = __builtin_amdgcn_perm(nv[f / 2], nv[f / 2], f & 1 ? 0x07060706u : 0x05040504u);
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        q8_u32x4 &v = vr(f, i);
#pragma unroll
        for (int y = 0; y < 4; ++y) v[y] = (v[y] & old[4 * i + y]) | (two & mine[4 * i + y]);
        o[f] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(q8_bf16x8, v),
                                                       __builtin_bit_cast(q8_bf16x8, make_uint4(w[4 * i], w[4 * i + 1], w[4 * i + 2], w[4 * i + 3])), o[f], 0, 0, 0);
      }
    }
    if (append && !fills && g == ((n >> 2) & 3)) {
#pragma unroll
      for (int f = 0; f < VF; ++f) vt[(f * 64 + lane) * 16 + (n >> 4) * 4 + (n & 3)] = (uint16_t)(nv[f / 2] >> (16 * (f & 1)));
    }
    if (fills) {
      uint32_t top = 0;
#pragma unroll
      for (int f = 0; f < VF; ++f) top = top4(top4(top, vr(f, 0)), vr(f, 1));
      const int e = q8_exponent(wave_max(top));
      const float inv = q8_pow2(-e);
      q8_u32x4 *to = reinterpret_cast<q8_u32x4 *>(a.c.v + (size_t)id * kQ8Block * D) + lane;
#pragma unroll
      for (int f = 0; f < VF; ++f) to[f * 64] = narrow(vr(f, 0), vr(f, 1), inv);
      if (lane == 0) a.c.v_scale[id] = q8_pow2(e);
    }
  }
  // The wave's state: per head [max, sum, -, -, o[0 .. D)].
  __device__ __forceinline__ void leave(float *st) {
    l = kg_sum(l);
#pragma unroll
    for (int f = 0; f < VF; ++f) {
      q8_f32x4 x;
#pragma unroll
      for (int r = 0; r < 4; ++r)
        x[r] = o[f][r] + column<P>(o[f][r]);
      if (col < G) *reinterpret_cast<q8_f32x4 *>(st + col * SF + 4 + 16 * f + 4 * g) = x;
    }
    if (col < G && g == 0) {
      st[col * SF] = m;
      st[col * SF + 1] = l;
    }
  }
};

template <int D, int G, int NW>
__global__ __launch_bounds__(64 * NW, 2) void ag_q8_decode_kernel(dec_args a) {
  constexpr int NT = 64 * NW;
  typedef wave_q8<D, G> wave_t;
  constexpr int SF = wave_t::SF;
  constexpr bool kRegs = NW == 8;  // the work list lives in registers
  __shared__ __attribute__((aligned(16))) float s_state[NW][G * SF];
  __shared__ __attribute__((aligned(16))) float s_turned[kRegs ? 1 : NW][(G + 1) * D];  // a team's queries and new key
  extern __shared__ int32_t s_len[];  // [U] rows held; top bit: another one fits
  __shared__ int32_t w_sum[NW][2], s_start[2], s_last, s_order;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int U = a.U, wg = blockIdx.x, grid = gridDim.x;
  const int most = a.c.max_blocks * kQ8Block + kQ8Block - 1;

  // The arguments lie in several cache lines of memory: all are asked for here, not one after the other as the code comes to need them.
  asm volatile("" :: "s"(a.q), "s"(a.out), "s"(a.c.len), "s"(a.c.n_pages), "s"(a.rope.n_rows), "s"(a.U));
  // ---- the work list ----
  auto items_of = [](int n) { return (n & 0x7fffffff) / kQ8Block + 1; };
  int piece = NW;                                       // items of a piece: rounds of the workgroup's waves
  uint32_t piece_inv = (uint32_t)((1ull << 32) / NW);   // ceil(2^32 / piece): x / piece for x piece < 2^32
  auto pieces_of = [&](int t) { return t <= max(kWholeRounds * NW, piece) ? 1 : (int)__umulhi((uint32_t)(t + piece - 1), piece_inv); };
  auto set_rounds = [&](int r) {
    piece = r * NW;
    piece_inv = 0xffffffffu / (uint32_t)piece + 1u;
  };
  auto read_len = [&](int v) {  // rows of unit v, top bit set if another one fits
    const int n = max(0, min(a.c.len[v], most)), at = n / kQ8Block;
    bool room = (n & (kQ8Block - 1)) != kQ8Block - 1;
    if (!room) room = at < a.c.max_blocks && (uint32_t)a.c.page[(size_t)v * a.c.max_blocks + min(at, a.c.max_blocks - 1)] < (uint32_t)a.c.n_pages;
    return n | (room ? (int)0x80000000 : 0);
  };
  // The lengths may only change once every workgroup has read them: each counts its arrival when it has (8 waves: at its end), and the
  // one that arrives last writes them.
  const int groups = !kRegs && grid >= kArriveSplit ? kDecodeArriveGroups : 1;
  auto arrive = [&] {
    s_order = __hip_atomic_fetch_add(a.arrived + (groups == 1 ? 0 : kDecodeArriveStride * (1 + wg % kDecodeArriveGroups)), 1, __ATOMIC_RELAXED,
                                     __HIP_MEMORY_SCOPE_AGENT);
  };
  int sl_r[2] = {0, 0};                                                              // kRegs: this lane's units, lane and 64 + lane
  const int per = (U + NT - 1) / NT, u0 = min(U, tid * per), u1 = min(U, u0 + per);  // else this thread's
  int total = 0, u = 0, sub = 0, team = NW, quota = 1, quota_2 = 1, x = 0;
  bool by_piece = false, by_team = false, idle;
  // Equal ranges.  With two workgroups on a CU the one that came first is served first: 1024 units of up to 4096 rows, all ranges equal, the
  // first halves of the launch ended after 84 us and the others after 94; so those get 8 % more.
  const int half = NW == 8 || grid % 2 ? grid : grid / 2;
  auto set_quotas = [&] {
    quota = quota_2 = (int)((uint32_t)(total + grid - 1) / (uint32_t)grid);
    if (half < grid) {
      quota += quota / 25;
      quota_2 = max(1, (int)((uint32_t)(max(0, total - half * quota) + half - 1) / (uint32_t)half));
    }
  };
  auto range_of = [&](int at) {
    return at < half * quota ? (int)((uint32_t)at / (uint32_t)quota) : half + (int)((uint32_t)(at - half * quota) / (uint32_t)quota_2);
  };
  auto range_at = [&](int r) { return r <= half ? r * quota : half * quota + (r - half) * quota_2; };
  if constexpr (kRegs) {  // (at most kFewUnits units: every wave by itself, without LDS and barriers)
    int t[2] = {0, 0}, cost[2], pre_t[2], pre_p[2] = {0, 0}, p[2] = {0, 0}, pieces = 0, items = 0, sum;
#pragma unroll
    for (int j = 0; j < 2; ++j)
      if (64 * j + lane < U) sl_r[j] = read_len(64 * j + lane);
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      if (64 * j + lane < U) t[j] = items_of(sl_r[j]);
      cost[j] = t[j] ? t[j] + kUnitCost : 0;
      pre_t[j] = total + ag_wave_prefix(cost[j], sum);
      total += sum;
    }
    items = total - U * kUnitCost;
    // pieces of the fewest rounds of the waves for which every piece has a workgroup (sure for the second try)
    int rounds = 1;
    if (items > NW * grid) rounds = (int)((uint32_t)(items + NW * grid - 1) / (uint32_t)(NW * grid));
    for (bool last = false;; last = true) {
      if (rounds > 1) set_rounds(rounds);
      pieces = 0;
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        p[j] = t[j] ? pieces_of(t[j]) : 0;
        pre_p[j] = pieces + ag_wave_prefix(p[j], sum);
        pieces += sum;
      }
      if (pieces <= grid || last || U >= grid) break;
      rounds = max(rounds, (int)((uint32_t)(items + NW * (grid - U) - 1) / (uint32_t)(NW * (grid - U))));
    }
    // ... unless so many units are cut that the remainders of their last pieces weigh more than equal ranges cost
    by_piece = pieces <= grid && (rounds <= 2 || 4 * U <= grid);
    if (!by_piece) set_quotas();
    x = by_piece ? wg : range_at(wg);
    idle = x >= (by_piece ? pieces : total);
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const int from = by_piece ? pre_p[j] : pre_t[j], n = by_piece ? p[j] : cost[j];
      const uint64_t hit = __ballot(from <= x && x < from + n);
      if (hit) {
        const int at = __builtin_ctzll(hit);
        u = 64 * j + at;
        sub = x - __builtin_amdgcn_readlane(from, at);
      }
    }
  } else {
    int my_t = 0, max_t = 0, sum;
    for (int v = u0; v < u1; ++v) {
      const int n = read_len(v);
      s_len[v] = n;
      my_t += items_of(n) + kUnitCost;
      max_t = max(max_t, items_of(n));
    }
    int pre_t = ag_wave_prefix(my_t, sum);
    max_t = (int)wave_max((uint32_t)max_t);
    if (lane == 0) { w_sum[wave][0] = sum; w_sum[wave][1] = max_t; }
    __syncthreads();
    if (tid == 0) arrive();
    max_t = 0;
#pragma unroll
    for (int w = 0; w < NW; ++w) {
      if (w < wave) pre_t += w_sum[w][0];
      total += w_sum[w][0];
      max_t = max(max_t, w_sum[w][1]);
    }
    while (team > 1 && U * team > grid * NW) team /= 2;
    by_team = U * team <= grid * NW && max_t <= kTeamRounds * team;
    if (by_team) {
      u = wg * (NW / team) + wave / team;
      idle = wg * (NW / team) >= U;
    } else {
      team = NW;
      set_quotas();
      x = range_at(wg);
      idle = x >= total;
      if (pre_t <= x && x < pre_t + my_t) {  // exactly one thread, if there is one
        int at = pre_t, v = u0;
        for (;; ++v) {
          const int t = items_of(s_len[v]) + kUnitCost;
          if (x < at + t) break;
          at += t;
        }
        s_start[0] = v;
        s_start[1] = x - at;
      }
      __syncthreads();
      if (!idle) { u = s_start[0]; sub = s_start[1]; }
    }
  }

  const int wt = team == NW ? wave : wave & (team - 1);
  int left = idle || by_piece || by_team ? 0 : min(range_at(wg + 1), total) - x, at = x;
  auto segment = [&]() {
    u = __builtin_amdgcn_readfirstlane(u);
    const bool mine = u < U;
    int sl = 0;
    if constexpr (kRegs) sl = __builtin_amdgcn_readlane(u < 64 ? sl_r[0] : sl_r[1], u & 63);
    else if (mine) sl = __builtin_amdgcn_readfirstlane(s_len[u]);
    const int n = sl & 0x7fffffff, nb = n / kQ8Block, T = nb + 1;
    int t0 = 0, t1 = mine ? T : 0, n_rec = 1, my_rec = 0, rec0 = 0;
    if (by_piece) {
      n_rec = pieces_of(T);
      my_rec = sub;
      rec0 = wg - sub;
      t0 = sub * piece;
      if (n_rec > 1) t1 = min(T, t0 + piece);
    } else if (!by_team) {  // item i of the unit lies at kUnitCost + i of its cost
      const int c0 = sub, c1 = min(T + kUnitCost, c0 + left), first = at - c0;
      left -= c1 - c0;
      at += c1 - c0;
      t0 = max(0, c0 - kUnitCost);
      t1 = max(0, c1 - kUnitCost);
      if (t0 > 0 || t1 < T) {
        const int g0 = range_of(first + kUnitCost), g1 = range_of(first + kUnitCost + T - 1);
        n_rec = g1 - g0 + 1;
        my_rec = wg - g0;
        rec0 = g0;
      }
    }
    if (!by_team && t0 == t1) {  // (the range ends before the unit's first item)
      ++u;
      sub = 0;
      return;
    }
    wave_t wv;
    int own_lane = lane;  // (unknown to the compiler, which would compute all addresses ahead of the loop and keep them in memory)
    asm volatile("" : "+v"(own_lane));
    wv.init(own_lane);
    // item 0 is the tail, item i page i - 1
    const bool has_tail = mine && t0 == 0 && wt == 0;
    const int i0 = t0 + wt - 1 + (t0 + wt == 0 ? team : 0), ip = t1 - 1;
    const int32_t *page = a.c.page + (size_t)u * a.c.max_blocks;
    if (i0 < ip) wv.numbers(page, i0, ip, team);
    int flag = 1;
    if (has_tail) {
      if (a.new_flags) flag = a.new_flags[u];
      wv.fetch_tail(a, u, n & (kQ8Block - 1));
    }
    // the group's queries and the new key, turned, into LDS: a pair of values a thread
    float *turned = s_turned[kRegs ? 0 : wave - wt];
    if (mine && t0 < t1) {
      const int n_vec = t0 == 0 ? G + 1 : G;
      for (int e = own_lane + wt * 64; e < n_vec * (D / 2); e += team * 64) {
        const int vec = e / (D / 2), i = e % (D / 2);
        const uint16_t *x = vec < G ? a.q + ((size_t)u * G + vec) * D : a.k_new + (size_t)u * D;
        const float lo = q8_lo(x[i]), hi = q8_lo(x[D / 2 + i]);
        float c = 1.f, sn = 0.f;
        if (a.rope.table) {
          const int axis = i < a.rope.end0 ? 0 : (i < a.rope.end1 ? 1 : 2);
          const float *row = a.rope.table + (size_t)q8_rope_row(a.rope, axis, u / a.Hkv, a.err) * D + i;
          c = row[0];
          sn = row[D / 2];
        }
        float y = a.rope.table ? q8_turn(lo, hi, c, sn, true) : lo, z = a.rope.table ? q8_turn(hi, lo, c, sn, false) : hi;
        if (vec == G) {  // the new key: bf16, and what that leaves over (half a word each)
          y = in_two(y);
          z = in_two(z);
        }
        turned[vec * D + i] = y;
        turned[vec * D + D / 2 + i] = z;
      }
    }
    if (i0 < ip) {
      wv.exponents(a.c);
    }
    // (The pages are asked for behind this barrier: ahead of it they would stand in the way of the small loads that it waits for.  8 steps of
    // 32 units of up to 13000 rows 169 us with both ahead, 162 with one, 153 with none.)
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    if (i0 < ip || has_tail) {
      const int two = (ip - i0 > team) + 1;
      if (i0 < ip && !has_tail) wv.first_pages(a.c, two);
      wv.query(turned + min(wv.head, G - 1) * D);
      if (has_tail) {
        flag = __builtin_amdgcn_readfirstlane(flag);
        if (flag != 0 && sl >= 0 && lane == 0) atomicOr(a.err, 1);
        wv.tail(a, u, n & (kQ8Block - 1), nb, flag != 0 && sl < 0, reinterpret_cast<const uint32_t *>(turned + G * D));
        if (i0 < ip) wv.first_pages(a.c, two);
      }
      if (i0 < ip) wv.pages(a.c, page, i0, ip, team, a.qscale);
    }
    wv.leave(s_state[wave]);
    __syncthreads();
    // ---- merge the team's waves; thread -> (head, two neighbouring columns) ----
    int e0 = lane;
    asm volatile("" : "+v"(e0));  // (as above)
    e0 += wt * 64;
    auto store_out = [&](int gg, int d, float A0, float A1, float L) {
      const float inv = 1.f / L;
      *reinterpret_cast<uint32_t *>(a.out + ((size_t)u * G + gg) * D + d) = q8_pack2(A0 * inv, A1 * inv);
    };
    auto rec_at = [&](int k) {
      const int id = by_piece ? rec0 + k : 2 * (rec0 + k) + (k == 0 ? 1 : 0);
      return a.rec + (size_t)id * G * (D + 2);
    };
    if (mine)
      for (int e = e0; e < G * D / 2; e += team * 64) {
        const int gg = e / (D / 2), d = 2 * (e - gg * (D / 2));
        float M = kQ8EmptyMax, L = 0.f, A0 = 0.f, A1 = 0.f, ms[NW], ls[NW], o0[NW], o1[NW];
        const int w0 = wave - wt;
#pragma unroll
        for (int w = 0; w < NW; ++w) {
          const float *st = s_state[w0 + (w < team ? w : 0)] + gg * SF;
          ms[w] = w < team ? st[0] : kQ8EmptyMax;
          ls[w] = w < team ? st[1] : 0.f;
          o0[w] = st[4 + d];
          o1[w] = st[5 + d];
        }
#pragma unroll
        for (int w = 0; w < NW; ++w) M = fmaxf(M, ms[w]);
#pragma unroll
        for (int w = 0; w < NW; ++w) {
          const float f = __builtin_amdgcn_exp2f(ms[w] - M);
          const bool any = !(ls[w] == 0.f);  // (a wave without rows)
          L = fmaf(f, ls[w], L);
          A0 = any ? fmaf(f, o0[w], A0) : A0;
          A1 = any ? fmaf(f, o1[w], A1) : A1;
        }
        if (n_rec == 1) {
          store_out(gg, d, A0, A1, L);
        } else {
          float *r = rec_at(my_rec) + gg * (D + 2);
          put_pair(r + d, A0, A1);
          if (d == 0) put_pair(r + D, M, L);
        }
      }
    if (!by_team && n_rec > 1) {
      asm volatile("s_waitcnt vmcnt(0)" ::: "memory");  // this wave's part of the record is in memory
      __syncthreads();
      if (tid == 0) s_last = __hip_atomic_fetch_add(&a.tickets[u], 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == n_rec - 1;
      __syncthreads();
      if (s_last) {  // all pieces are there: they are added in order
        if (tid == 0) a.tickets[u] = 0;
        for (int e = e0; e < G * D / 2; e += NT) {
          const int gg = e / (D / 2), d = 2 * (e - gg * (D / 2));
          float M = kQ8EmptyMax, L = 0.f, A0 = 0.f, A1 = 0.f;
          for (int k0 = 0; k0 < n_rec; k0 += 8) {
            float2 ml[8], o[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) {
              const float *r = rec_at(min(k0 + j, n_rec - 1)) + gg * (D + 2);
              ml[j] = get_pair(r + D);
              o[j] = get_pair(r + d);
            }
            float M_new = M;
#pragma unroll
            for (int j = 0; j < 8; ++j) M_new = fmaxf(M_new, ml[j].x);
            const float keep = __builtin_amdgcn_exp2f(M - M_new);
            M = M_new;
            L *= keep; A0 *= keep; A1 *= keep;
#pragma unroll
            for (int j = 0; j < 8; ++j) {
              if (k0 + j >= n_rec) break;
              const float w = __builtin_amdgcn_exp2f(ml[j].x - M);
              L = fmaf(w, ml[j].y, L);
              A0 = fmaf(w, o[j].x, A0);
              A1 = fmaf(w, o[j].y, A1);
            }
          }
          store_out(gg, d, A0, A1, L);
        }
      }
    }
    ++u;
    sub = 0;
  };
  if (!idle)
    for (;;) {  // (one segment, but where a range covers several units)
      segment();
      if (left <= 0) break;
      __syncthreads();  // the states have been read
    }
  // ---- the last workgroup to arrive counts the appended rows ----
  __syncthreads();
  if (tid == 0) {
    if (kRegs) arrive();
    int last = grid - 1, order = s_order;
    if (groups > 1) {
      const int mine = (grid - wg % kDecodeArriveGroups + kDecodeArriveGroups - 1) / kDecodeArriveGroups;
      order = order == mine - 1 ? __hip_atomic_fetch_add(a.arrived, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) : -1;
      last = kDecodeArriveGroups - 1;
    }
    s_last = order == last;
  }
  __syncthreads();
  if (!s_last) return;
  if constexpr (kRegs) {
    if (wave == 0)
#pragma unroll
      for (int j = 0; j < 2; ++j)
        if (sl_r[j] < 0 && (!a.new_flags || a.new_flags[64 * j + lane] != 0)) a.c.len[64 * j + lane] = (sl_r[j] & 0x7fffffff) + 1;
  } else
  for (int v = tid; v < U; v += NT)
    if (s_len[v] < 0 && (!a.new_flags || a.new_flags[v] != 0)) a.c.len[v] = (s_len[v] & 0x7fffffff) + 1;
  if (tid <= kDecodeArriveGroups) a.arrived[kDecodeArriveStride * tid] = 0;
}

template <int D, int G, int NW>
hipError_t launch_nw(ag_ctx *ctx, hipStream_t s, const dec_args &a) {
  // one workgroup per CU (8 waves) or two (4 waves), and no more than the step can have pieces
  const int64_t most = a.U + (int64_t)a.U * (a.c.max_blocks + 1) / NW;
  const int grid = (int)std::min<int64_t>((8 / NW) * ctx->num_cu, most);
  static std::atomic<bool> allowed[64];
  const hipError_t e = ag_q8_allow_lds(ctx->device, allowed, &ag_q8_decode_kernel<D, G, NW>, (size_t)kDecodeMaxUnits * 4);
  if (e != hipSuccess) return e;
  AG_LAUNCH(ag_time_kernel(ctx, AG_K_Q8_DECODE), (ag_q8_decode_kernel<D, G, NW>), dim3(grid), dim3(64 * NW), NW == 8 ? 0 : (size_t)a.U * 4, s, a);
  return hipGetLastError();
}
template <int D, int G>
hipError_t launch(ag_ctx *ctx, hipStream_t s, const dec_args &a) {
  return a.U <= kFewUnits ? launch_nw<D, G, 8>(ctx, s, a) : launch_nw<D, G, 4>(ctx, s, a);
}
template <int D>
hipError_t launch_g(int G, ag_ctx *ctx, hipStream_t s, const dec_args &a) {
  switch (G) {
    case 1: return launch<D, 1>(ctx, s, a);
    case 2: return launch<D, 2>(ctx, s, a);
    case 4: return launch<D, 4>(ctx, s, a);
    case 8: return launch<D, 8>(ctx, s, a);
  }
  return hipErrorInvalidValue;
}

}  // namespace

// (and what rounding up to whole ranges adds, at most two workgroups a CU)
int64_t ag_q8_decode_cost(int64_t units, int max_blocks) { return units * ((int64_t)max_blocks + 1 + kUnitCost) + (1 << 16); }

size_t ag_ws_q8_decode_floats(int num_cu, int G, int D) { return (size_t)4 * num_cu * G * (D + 2); }

hipError_t ag_launch_q8_decode(ag_ctx *ctx, hipStream_t s, const void *q, const void *k_new, const void *v_new, const uint8_t *new_flags,
                               int B, int Hq, int Hkv, int D, const ag_rope_dev &rope, float scale, const ag_q8_dev &cache, void *out, float *rec) {
  dec_args a;
  a.q = (const uint16_t *)q; a.k_new = (const uint16_t *)k_new; a.v_new = (const uint16_t *)v_new; a.new_flags = new_flags; a.out = (uint16_t *)out;
  a.c = cache; a.rope = rope; a.rec = rec;
  a.tickets = ctx->decode_tickets; a.arrived = ctx->decode_tickets + kDecodeMaxUnits; a.err = ctx->d_err;
  a.U = B * Hkv; a.Hkv = Hkv; a.qscale = scale * kLog2e;
  return D == 128 ? launch_g<128>(Hq / Hkv, ctx, s, a) : launch_g<64>(Hq / Hkv, ctx, s, a);
}
