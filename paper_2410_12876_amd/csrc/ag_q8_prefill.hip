// Attention of many new tokens over the paged 8-bit cache as it stood before the call, and over themselves.
//
// For new token j of a unit the visible rows are: all rows that the cache held, the call's own kept tokens before j, and j itself.
// ag_q8_fill_kernel (launched first) leaves the tail's rows and the kept tokens, turned and packed, as tiles of 64 rows in f16;
// the full blocks of the cache are read as they are.  So the keys of a unit are one sequence of tiles -- its pages, then those --
// of which row j sees the first `bound_j` rows; an evicted token's own key and value, which are in none of them, are what its state starts from
// (and a kept one's that sees nothing else).
//   * A workgroup of 4 waves owns 128 query rows of a unit (token by token, the group's heads of a token side by side) and every wave 32 of
//     them, with a lane owning one column: S^T = K q^T, O^T = V^T p^T on v_mfma_f32_32x32x16_f16, P passes from the first product's
//     accumulators into the second one's operand without leaving the lane.
//   * A tile's 64 rows lie in LDS in the order of the fragments, in two buffers.  A page goes there through registers, its codes made f16
//     (exactly, one instruction for two values) once for the 128 rows; a tile of this call, in that order already, is loaded into LDS
//     directly.  Either way the next tile's loads are in flight while a tile is worked on.
//   * A fragment is read four products before its own, and the two halves' products take turns, so that no product waits for LDS or for the
//     product before it: 765 us in place of 900 for 4096 tokens of 8 heads in 2 groups over 13000 rows, with the pages' numbers and scales
//     looked up 64 tiles at a time (tile by tile they were waited for in every step).  Forming one half's weights between the other half's
//     products, which the compiler can be made to do, gained nothing over this: the second workgroup of the CU fills those gaps already.
//   * Both products are in f16, whose 11 bits keep operands to 2^-12 of themselves (in bf16, 2^-9: an output row's error grew from 1.7e-3
//     to 2.9e-3 of its size, and with scores of 7 times the usual spread a weight was off by a hundredth).  Its narrow range is why queries,
//     tiles and a token's own value carry exponents; tiles of too different values are taken row by row on the vector ALU.
//   * Weights are f16 too, relative to a reference that lies 2^-8 below the largest (score plus exponent) of the tile that set it: down to
//     2^-22 of that they keep 11 bits, down to 2^-33 some.  The row sum adds up the rounded ones, so their rounding cancels where many are
//     alike.  (Against the largest itself and with the unrounded sum, 300000 rows at 2^-25.5 of it put a row off by 1.5e-2 of its size, now by 2.4e-3,
//     which the store's rounding gives.)  Tiles of far smaller values than others add to the row sum in 32 bits (kQ8Span).
//   * No maximum is taken in the common case: weights are formed against the reference as it stands, and only if their sum passes 2^15 is
//     it moved.  The first tile always sets it.
//   * Few items and long caches: the tiles of an item are cut into up to n_split pieces, whose states a second kernel adds up.
#include <algorithm>

#include "ag_q8.h"

namespace {

constexpr float kLog2e = 1.4426950408889634f;
constexpr int kRows = 128;     // query rows of a workgroup
constexpr int kMinTiles = 4;   // tiles of a piece, at least (37 tokens over 777 rows 44.3 us; with 2 43.8, with 6 46, with 8 49.4; over 8000 alike)
constexpr int kMaxSplit = 32;
constexpr int kPageBits = 6;   // a page's values are made as large as those of this call's tiles (codes below 2^9, tiles below 2^15)

struct pf_args {
  const uint16_t *q, *k, *v;
  uint16_t *out;
  const uint64_t *words;
  const int32_t *blk_off;
  const uint16_t *tiles;
  const uint32_t *info;
  const ag_q8_meta *meta;
  ag_q8_dev c;
  ag_rope_dev rope;
  float *part;    // [item][piece][kRows][D + 4]: o, m, l, two of nothing
  int32_t *err;
  int U, Hq, Hkv, L, nw, n_blk, n_qt, n_split;
  float qscale;
};

// Kept tokens of the call before token j, and whether j is appended itself.
__device__ __forceinline__ int rank_of(const pf_args &a, int u, int j, int added, bool &kept) {
  int r = j;
  kept = true;
  if (a.blk_off) {
    const uint64_t w = a.words[(size_t)u * a.nw + (j >> 6)];
    r = a.blk_off[(size_t)u * (a.nw + 1) + (j >> 6)] + __popcll(w & ((1ull << (j & 63)) - 1));
    kept = (w >> (j & 63)) & 1;
  }
  kept = kept && r < added;
  return min(r, added);
}
struct pf_cut {
  int tiles, per, pieces;  // tiles of an item, of a piece; pieces
};
__device__ __forceinline__ pf_cut cut_of(const pf_args &a, const ag_q8_meta &m, int u, int qt, int G) {
  const int last = min(a.L - 1, (qt * kRows + kRows - 1) / G);
  bool kept;
  const int rows = m.held + rank_of(a, u, last, m.added, kept);  // (+ 1 if kept: below)
  pf_cut c;
  c.tiles = m.blocks + (rows + (kept ? 1 : 0) + kQ8Block - 1) / kQ8Block;
  c.per = max(kMinTiles, (c.tiles + a.n_split - 1) / a.n_split);
  c.pieces = max(1, (c.tiles + c.per - 1) / c.per);
  return c;
}

__device__ __forceinline__ float other_half(float x) { return __shfl_xor(x, 32, 64); }
// 2^(d / 2), d <= 0: what is to shrink by 2^d is multiplied by it twice (references of tiles of very different sizes lie further apart than
// a factor can be small).
__device__ __forceinline__ float half_way(float d) { return __builtin_amdgcn_exp2f(0.5f * d); }

template <int D, int G>
__global__ __launch_bounds__(256, 2) void ag_q8_prefill_kernel(pf_args a) {
  constexpr int KC = D / 64, KS = D / 16, DT = D / 32, HALF = kQ8Block * D;  // values of K (V) in a tile
  constexpr int NP = KS;  // 16-byte pieces of a bf16 tile per thread
  extern __shared__ __attribute__((aligned(1024))) uint16_t smem[];  // two tiles: K fragments, V fragments
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int col = lane & 31, h = lane >> 5;
  // block -> (piece, query tile, unit): long query tiles first, units next to each other but each time one further: blocks 8 apart are
  // one XCD's, and a long unit that stayed with its XCD held the launch up (4096 tokens of 8 heads over up to 13000 rows 800 us, so 700; 4 x
  // 600 tokens of 8 heads 152 and 125; the first 4096 of 32 heads 182 and 166), whatever its tiles in that L2 saved.
  int id = blockIdx.x;
  int u = id % a.U;
  id /= a.U;
  u = (u + id) % a.U;
  const int piece = id % a.n_split, qt = a.n_qt - 1 - id / a.n_split;
  const ag_q8_meta meta = a.meta[u];
  const pf_cut cut = cut_of(a, meta, u, qt, G);
  const int t0 = piece * cut.per, t1 = min(cut.tiles, t0 + cut.per);
  if (piece > 0 && t0 >= t1) return;

  // ---- this lane's query row ----
  const int rows = a.L * G, b = u / a.Hkv;
  auto row_of = [&](int c) { return qt * kRows + wave * 32 + c; };
  auto token_of = [&](int row) { return min(row / G, a.L - 1); };
  auto q_of = [&](int row) { return (((size_t)b * a.Hq + (size_t)(u % a.Hkv) * G + row % G) * a.L + token_of(row)) * D; };
  const int j = token_of(row_of(col));
  const size_t k_at = ((size_t)u * a.L + j) * D;
  bool kept;
  const int rank = rank_of(a, u, j, meta.added, kept);
  const bool sole = meta.blocks == 0 && meta.held + rank == 0;  // it sees nothing else
  const int bound = sole ? 0 : meta.held + rank + (kept ? 1 : 0);  // visible rows of those tiles
  // The query in f16 times 2^eq (11 bits; bf16 would lose up to 2^-9 of a turned value, and the scores as much of themselves)
  q8_rows at = {0, 0, 0};
  auto angles = [&](int i) { return q8_angles4(a.rope, at, i, D); };
  if (a.rope.table) at = q8_rope_rows(a.rope, (int64_t)b * a.L + j, a.err);
  auto vector = [&](q8_eight (&y)[KS], const uint16_t *x) {  // this lane's half of a row, turned
    uint4 raw[KS];
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) raw[ks] = *reinterpret_cast<const uint4 *>(x + 16 * ks + 8 * h);
#pragma unroll
    for (int ks = 0; ks < KS; ++ks)
      y[ks] = a.rope.table ? q8_turn8<D>(angles, 16 * ks + 8 * h, raw[ks], raw[ks ^ (KS / 2)]) : q8_floats(raw[ks]);
  };
  q8_f16x8 qx[KS];
  int eq;
  {
    q8_eight y[KS];
    vector(y, a.q + q_of(row_of(col)));
    float top = 0.f;  // (infinities are none of a binade's; NaN is passed over)
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) top = fmaxf(top, y[ks].top());
    top = fmaxf(top, other_half(top));
    eq = max(kQ8TileMinExp, min(254, max(1, (int)(__float_as_uint(top) >> 23))) - 127 - kQ8TileTop);
    const float inv = q8_pow2(-eq);
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) qx[ks] = y[ks].f16(inv);
  }
  float m = kQ8EmptyMax, l = 0.f;
  int ev_top = kQ8PageMinExp;  // the largest exponent that a reference of this wave's rows has been set with
  const bool alone = piece == 0 && (!kept || sole);  // an evicted token sees itself, and so does a kept one that sees nothing else
  q8_f32x16 o[DT];
#pragma unroll
  for (int dt = 0; dt < DT; ++dt)
#pragma unroll
    for (int x = 0; x < 4; ++x) {
      uint2 w = make_uint2(0, 0);
      if (alone) w = *reinterpret_cast<const uint2 *>(a.v + k_at + 32 * dt + 8 * x + 4 * h);
      o[dt][4 * x] = q8_lo(w.x); o[dt][4 * x + 1] = q8_hi(w.x);
      o[dt][4 * x + 2] = q8_lo(w.y); o[dt][4 * x + 3] = q8_hi(w.y);
    }
  if (alone) {
    q8_eight y[KS];
    vector(y, a.k + k_at);
    float s = 0.f, top = 0.f;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks)
#pragma unroll
      for (int i = 0; i < 4; ++i) s = fmaf((float)qx[ks][i], y[ks].a[i], fmaf((float)qx[ks][4 + i], y[ks].b[i], s));
    s = (s + other_half(s)) * q8_unscale(a.qscale, eq);
    // Its value has an exponent as a tile has one: the reference is the score plus that, or the tiles' weights would be as much too small
    // for f16 as the values are small.  (Values that are not finite do not count: other columns are not theirs.)
#pragma unroll
    for (int dt = 0; dt < DT; ++dt)
#pragma unroll
      for (int i = 0; i < 16; ++i) top = fmaxf(top, fabsf(o[dt][i]) < INFINITY ? fabsf(o[dt][i]) : 0.f);
    top = fmaxf(top, other_half(top));
    int e = max(kQ8PageMinExp, max(1, (int)(__float_as_uint(top) >> 23)) - 127 - kQ8TileTop) - kQ8TopBits;
    ev_top = max(ev_top, e + kQ8TopBits);
    // seeing nothing else its weight is 1 whatever its score is; a score that overflowed to -infinity counts as the least number
    if (sole) s = 0.f, e = 0;
    m = (s < kQ8EmptyMax ? kQ8EmptyMax : s) + (float)e;
    const float scale = q8_pow2(-e);
    l = h == 0 ? scale : 0.f;  // (summed over the halves at the end)
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) o[dt] *= scale;
  }
  // rows that every row of the wave sees, and that one of them sees; ev_top over the wave
  int see_all = bound, see_one = bound;
#pragma unroll
  for (int x = 16; x > 0; x >>= 1) {
    see_all = min(see_all, __shfl_xor(see_all, x, 64));
    see_one = max(see_one, __shfl_xor(see_one, x, 64));
    ev_top = max(ev_top, __shfl_xor(ev_top, x, 64));
  }
  see_all = __builtin_amdgcn_readfirstlane(see_all);
  see_one = __builtin_amdgcn_readfirstlane(see_one);
  ev_top = __builtin_amdgcn_readfirstlane(ev_top);

  const int32_t *page = a.c.page + (size_t)u * a.c.max_blocks;
  const uint16_t *tiles = a.tiles + (size_t)u * a.n_blk * 2 * HALF;
  auto rsrc_of = [](const void *p, int bytes) { return __builtin_amdgcn_make_buffer_rsrc((void *)p, 0, bytes, 0x00020000); };
  auto load = [](__amdgpu_buffer_rsrc_t r, int at, int more) { return __builtin_bit_cast(uint4, __builtin_amdgcn_raw_buffer_load_b128(r, at, more, 0)); };
  // Lane x knows tile w_first + x: its page (0: a tile of this call; -1: not there, or odd) and its exponents.  (Read tile by tile, the
  // page's number and then its scales would be waited for in every step.)
  int w_first = t0, w_id = -1, w_ek = 0, w_ev = 0;
  bool any_odd = false, fresh = true;  // fresh: no tile has been taken yet
  auto look_up = [&](int first) {
    const int t = first + lane;
    bool odd = false;
    w_first = first;
    w_id = -1;
    w_ek = w_ev = 0;
    if (t < min(t1, meta.blocks)) {
      const int p = page[t], ps = (uint32_t)p < (uint32_t)a.c.n_pages ? p : 0;  // (a page number outside the pool counts as evicted rows)
      w_id = ps == p ? p : -1;
      w_ek = (int)(__float_as_uint(a.c.k_scale[ps]) >> 23) - 127;
      w_ev = (int)(__float_as_uint(a.c.v_scale[ps]) >> 23) - 127 - kPageBits;
    } else if (t < t1) {
      const q8_tile_info info = q8_tile_of(a.info[(size_t)u * a.n_blk + t - meta.blocks]);
      odd = info.odd;
      w_id = odd ? -1 : 0;
      w_ek = info.ek;
      w_ev = info.ev;
    }
    any_odd |= __any(odd) != 0;
  };
  auto here = [&] {  // (the thread's number, unknown to the compiler: or all addresses below would be kept in registers)
    int x = tid;
    asm volatile("" : "+v"(x));
    return x;
  };
  const uint32_t lds0 = __builtin_amdgcn_readfirstlane((uint32_t)(size_t)(__attribute__((address_space(3))) uint16_t *)smem);
  uint4 rk[KC] = {}, rv[2] = {};  // a thread's pieces of the next page's K and V
  // Tile t: a page into registers, a tile of this call, which lies as LDS wants it, into LDS by itself
  auto request = [&](int t, int buf) {
    const int id = __builtin_amdgcn_readlane(w_id, t - w_first), x = here();
    if (id < 0) return;
    if (t < meta.blocks) {
      const __amdgpu_buffer_rsrc_t pk = rsrc_of(a.c.k + (size_t)id * HALF, HALF), pv = rsrc_of(a.c.v + (size_t)id * HALF, HALF);
#pragma unroll
      for (int i = 0; i < KC; ++i) rk[i] = load(pk, x * 16, i * 4096);
      // rows 16 i + 4 g + 0..3 and 16 i + 4 (g + 2) + 0..3, i < 4, of column 16 f + r: f = x / 32, g = x / 16 % 2, r = x % 16 for thread x
      const int at = ((x >> 5) & (D / 16 - 1)) * 1024 + (x & 31) * 16;
      rv[0] = load(pv, at, 0);
      rv[1] = load(pv, at, 512);
    } else {
      const __amdgpu_buffer_rsrc_t w = rsrc_of(tiles + (size_t)(t - meta.blocks) * 2 * HALF, 4 * HALF);
      const uint32_t base = buf * 4 * HALF + wave * 1024;
#pragma unroll
      for (int i = 0; i < NP; ++i)
        asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, %3 offen lds"
                     :: "s"(lds0 + base + i * 4096), "v"(x * 16), "s"(w), "s"(i * 4096) : "m0", "memory");
    }
  };
  auto stage = [&](int t, int buf) {  // a page from the registers into LDS, widened
    if (t >= meta.blocks) return;
    uint16_t *ks = smem + buf * 2 * HALF, *vs = ks + HALF;
    const int tid = here();
#pragma unroll
    for (int x = 0; x < KC; ++x) {
      const int n = tid + 256 * x, r = n & 15, g = (n >> 4) & 3, c = (n >> 6) % KC, ra = (n >> 6) / KC, tt = 16 * ra + r;
      uint16_t *to = ks + (((tt >> 5) * KS + 4 * c + g) * 64 + (tt & 31)) * 8;
      *reinterpret_cast<q8_f16x8 *>(to) = q8_widen16(rk[x].x, rk[x].y, 1.f);
      *reinterpret_cast<q8_f16x8 *>(to + 32 * 8) = q8_widen16(rk[x].z, rk[x].w, 1.f);
    }
    if (D == 128 || tid < 128) {
      const int e = __builtin_amdgcn_readlane(w_ev, t - w_first);
      const float scale = q8_pow2(e + kPageBits - max(kQ8PageMinExp, e));
      const uint32_t lo[4] = {rv[0].x, rv[0].y, rv[0].z, rv[0].w}, hi[4] = {rv[1].x, rv[1].y, rv[1].z, rv[1].w};
#pragma unroll
      for (int i = 0; i < 4; ++i)
        *reinterpret_cast<q8_f16x8 *>(vs + (((tid >> 6) * 4 + i) * 64 + ((tid >> 4) & 1) * 32 + ((tid >> 5) & 1) * 16 + (tid & 15)) * 8) =
            q8_widen16(lo[i], hi[i], scale);
    }
  };
  if (t0 < t1) {
    look_up(t0);
    request(t0, 0);
    stage(t0, 0);
  }
  for (int t = t0; t < t1; ++t) {
    const int buf = (t - t0) & 1;
    const bool now = __builtin_amdgcn_readlane(w_id, t - w_first) >= 0;
    const int ek = __builtin_amdgcn_readlane(w_ek, t - w_first), e_v = max(kQ8PageMinExp, __builtin_amdgcn_readlane(w_ev, t - w_first));
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");  // (what went to LDS by itself: the compiler does not know of it)
    __syncthreads();
    if (t + 1 < t1) {
      if (t + 1 - w_first >= 64) look_up(t + 1);
      request(t + 1, buf ^ 1);
    }
    const int first = (t - meta.blocks) * kQ8Block;  // the tile's first row among those of the tiles of this call
    if (now && first < see_one) {
      const uint16_t *ks = smem + buf * 2 * HALF + lane * 8, *vs = ks + HALF;
      q8_f32x16 s[2];
#pragma unroll
      for (int x = 0; x < 2; ++x)
#pragma unroll
        for (int i = 0; i < 16; ++i) s[x][i] = 0.f;
#pragma unroll
      for (int kk = 0; kk < KS; ++kk)
#pragma unroll
        for (int x = 0; x < 2; ++x)
          s[x] = __builtin_amdgcn_mfma_f32_32x32x16_f16(*reinterpret_cast<const q8_f16x8 *>(ks + (x * KS + kk) * 512), qx[kk], s[x], 0, 0, 0);
      __builtin_amdgcn_sched_group_barrier(0x100, 4, 0);  // fragments ahead of the products
#pragma unroll
      for (int x = 0; x < 2 * KS; ++x) {
        __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
        if (x + 4 < 2 * KS) __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
      }
      // s[x][i]: row 32 x + 8 (i / 4) + 4 h + i % 4 of the tile.  The state is kept relative to m, the largest score plus its tile's ev less
      // kQ8TopBits: a tile's weights are 2^(score + ev - m), at most 2^15, its values v 2^-ev, and its part of the row sum is 2^-ev the sum of
      // its weights, as the second product takes them: what rounding them changes cancels.  (`apart`: the sum of 2^(score - m).)
      const float f = q8_unscale(a.qscale, eq + ek), ev = (float)e_v;
      if (t >= meta.blocks && first + kQ8Block > see_all) {
        const int b = bound - first - 4 * h;
#pragma unroll
        for (int x = 0; x < 2; ++x)
#pragma unroll
          for (int i = 0; i < 16; ++i)
            if (32 * x + 8 * (i / 4) + i % 4 >= b) s[x][i] = -INFINITY;
      }
      ev_top = max(ev_top, e_v);
      const bool apart = e_v <= ev_top - kQ8Span;
      uint32_t p[2][8];
      float sum = 0.f;
      auto weigh = [&] {
        const float off = ev - m;
        float part[2] = {0.f, 0.f};
#pragma unroll
        for (int x = 0; x < 2; ++x)
#pragma unroll
          for (int i = 0; i < 16; i += 2) {
            const q8_f32x2 w = {__builtin_amdgcn_exp2f(fmaf(s[x][i], f, off)), __builtin_amdgcn_exp2f(fmaf(s[x][i + 1], f, off))};
            p[x][i / 2] = __builtin_bit_cast(uint32_t, __builtin_convertvector(w, q8_f16x2));
            asm volatile("" : "+v"(p[x][i / 2]));  // (packed here: the compiler would carry all 32 weights to the second product)
            part[i / 2 & 1] = q8_add2(p[x][i / 2], part[i / 2 & 1]);
          }
        sum = part[0] + part[1];
      };
      if (!fresh) weigh();
      if (fresh || apart || __any(!(sum <= 32768.f))) {  // no reference yet, or too far below: a new one, and the weights again
        float mx = -INFINITY;
#pragma unroll
        for (int x = 0; x < 2; ++x)
#pragma unroll
          for (int i = 0; i < 16; ++i) mx = fmaxf(mx, s[x][i]);
        mx = fmaf(fmaxf(mx, other_half(mx)), f, ev - (float)kQ8TopBits);
        const float both = fmaxf(sum <= 32768.f ? 0.f : 1.f, other_half(sum <= 32768.f ? 0.f : 1.f));
        const float m_new = fresh || both > 0.f ? fmaxf(m, mx) : m;  // (a row's own reference alone: no row depends on its neighbours)
        const float alpha = half_way(m - m_new);
        l = l * alpha * alpha;
#pragma unroll
        for (int dt = 0; dt < DT; ++dt) o[dt] = o[dt] * alpha * alpha;
        m = m_new;
        fresh = false;
        weigh();
        if (apart) {
#pragma unroll
          for (int x = 0; x < 2; ++x)
#pragma unroll
            for (int i = 0; i < 16; ++i) l += __builtin_amdgcn_exp2f(fmaf(s[x][i], f, -m));
          sum = 0.f;
        }
      }
      l += ldexpf(sum, -e_v);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const q8_f16x8 pb = __builtin_bit_cast(q8_f16x8, make_uint4(p[i >> 1][4 * (i & 1)], p[i >> 1][4 * (i & 1) + 1], p[i >> 1][4 * (i & 1) + 2], p[i >> 1][4 * (i & 1) + 3]));
#pragma unroll
        for (int dt = 0; dt < DT; ++dt)
          o[dt] = __builtin_amdgcn_mfma_f32_32x32x16_f16(*reinterpret_cast<const q8_f16x8 *>(vs + (dt * 4 + i) * 512), pb, o[dt], 0, 0, 0);
      }
      __builtin_amdgcn_sched_group_barrier(0x100, 4, 1);
#pragma unroll
      for (int x = 0; x < 4 * DT; ++x) {
        __builtin_amdgcn_sched_group_barrier(0x008, 1, 1);
        if (x + 4 < 4 * DT) __builtin_amdgcn_sched_group_barrier(0x100, 1, 1);
      }
    }
    if (t + 1 < t1) stage(t + 1, buf ^ 1);
  }
  if (any_odd) {  // rare: tiles with values that are not finite, or of too different sizes; row by row in 32 bits
    const float f = q8_unscale(a.qscale, eq);
    for (int t = max(t0, meta.blocks); t < t1; ++t) {
      const int first = (t - meta.blocks) * kQ8Block;
      if (!q8_tile_of(a.info[(size_t)u * a.n_blk + t - meta.blocks]).odd) continue;
      const uint16_t *tk = tiles + (size_t)(t - meta.blocks) * 2 * HALF, *tv = tk + HALF;
      for (int r = 0; r < kQ8Block && first + r < see_one; ++r) {
        float s = 0.f;
#pragma unroll
        for (int kk = 0; kk < KS; ++kk) {
          const q8_eight y = q8_floats(*reinterpret_cast<const uint4 *>(tk + (((r >> 5) * KS + kk) * 64 + h * 32 + (r & 31)) * 8));
          q8_f16x8 q = qx[kk];
          asm volatile("" : "+v"(q));  // (or the compiler would keep all of the query in 32 bits across the loop)
#pragma unroll
          for (int i = 0; i < 4; ++i) s = fmaf((float)q[i], y.a[i], fmaf((float)q[4 + i], y.b[i], s));
        }
        s = (s + other_half(s)) * f;
        if (first + r < bound) {
          const float m_new = fmaxf(m, s < kQ8EmptyMax ? kQ8EmptyMax : s);
          const float alpha = half_way(m - m_new), w = __builtin_amdgcn_exp2f(s - m_new);
          m = m_new;
          l = l * alpha * alpha + (h == 0 ? w : 0.f);
          // row r: step r / 16, half (r / 4) % 2, element 4 ((r / 8) % 2) + r % 4 of a column's piece
          const uint16_t *vr = tv + ((r >> 4) * 64 + ((r >> 2) & 1) * 32) * 8 + ((r >> 3) & 1) * 4 + (r & 3);
#pragma unroll
          for (int dt = 0; dt < DT; ++dt)
#pragma unroll
            for (int i = 0; i < 16; ++i)
              o[dt][i] = fmaf(o[dt][i] * alpha, alpha, w * __uint_as_float((uint32_t)vr[(dt * 4 * 64 + 8 * (i / 4) + 4 * h + i % 4) * 8] << 16));
        }
      }
    }
  }
  l += other_half(l);
  int end_lane = lane;
  asm volatile("" : "+v"(end_lane));  // (or the addresses below would be kept in registers all the way)
  const int end_row = row_of(end_lane & 31), end_h = end_lane >> 5;
  if (cut.pieces == 1) {
    if (end_row < rows) {
      const float inv = 1.f / l;
      uint16_t *to = a.out + q_of(end_row) + 4 * end_h;
#pragma unroll
      for (int dt = 0; dt < DT; ++dt)
#pragma unroll
        for (int x = 0; x < 4; ++x)
          *reinterpret_cast<uint2 *>(to + 32 * dt + 8 * x) =
              make_uint2(q8_pack2(o[dt][4 * x] * inv, o[dt][4 * x + 1] * inv), q8_pack2(o[dt][4 * x + 2] * inv, o[dt][4 * x + 3] * inv));
    }
    return;
  }
  float *to = a.part + ((((size_t)qt * a.U + u) * a.n_split + piece) * kRows + wave * 32 + (end_lane & 31)) * (D + 4);
#pragma unroll
  for (int dt = 0; dt < DT; ++dt)
#pragma unroll
    for (int x = 0; x < 4; ++x)
      *reinterpret_cast<float4 *>(to + 32 * dt + 8 * x + 4 * end_h) = make_float4(o[dt][4 * x], o[dt][4 * x + 1], o[dt][4 * x + 2], o[dt][4 * x + 3]);
  if (end_h == 0) *reinterpret_cast<float2 *>(to + D) = make_float2(m, l);
}

// Adds up the pieces of the items that were cut: thread = four columns of a query row.
template <int D, int G>
__global__ __launch_bounds__(256) void ag_q8_prefill_merge_kernel(pf_args a) {
  constexpr int TPR = D / 4;
  const int per = 256 / TPR, n_wg = kRows / per;
  int id = blockIdx.x;
  const int part = id % n_wg;
  id /= n_wg;
  const int u = id % a.U, qt = id / a.U;
  const ag_q8_meta meta = a.meta[u];
  const pf_cut cut = cut_of(a, meta, u, qt, G);
  if (cut.pieces == 1) return;
  const int r = part * per + threadIdx.x / TPR, d = (threadIdx.x % TPR) * 4, row = qt * kRows + r;
  if (row >= a.L * G) return;
  const float *from = a.part + (((size_t)qt * a.U + u) * a.n_split * kRows + r) * (D + 4);
  float M = kQ8EmptyMax, L = 0.f;
  for (int p = 0; p < cut.pieces; ++p) M = fmaxf(M, from[(size_t)p * kRows * (D + 4) + D]);
  float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
  for (int p = 0; p < cut.pieces; ++p) {
    const float *f = from + (size_t)p * kRows * (D + 4);
    const float4 x = *reinterpret_cast<const float4 *>(f + d);
    const float2 ml = *reinterpret_cast<const float2 *>(f + D);
    const float w = half_way(ml.x - M);
    L = fmaf(w, ml.y * w, L);
    o.x = fmaf(w, x.x * w, o.x); o.y = fmaf(w, x.y * w, o.y); o.z = fmaf(w, x.z * w, o.z); o.w = fmaf(w, x.w * w, o.w);
  }
  const float inv = 1.f / L;
  const int j = row / G, b = u / a.Hkv;
  *reinterpret_cast<uint2 *>(a.out + (((size_t)b * a.Hq + (size_t)(u % a.Hkv) * G + row % G) * a.L + j) * D + d) =
      make_uint2(q8_pack2(o.x * inv, o.y * inv), q8_pack2(o.z * inv, o.w * inv));
}

// Pieces an item may be cut into, from what the cache can hold at most: so many that the launch fills every CU once (D = 64: twice, of the
// three workgroups that fit).  More pieces balance better, but every one turns the queries again and is added up: 37 tokens of 8 heads in
// groups of 4 over 8000 rows 57 us, with two a CU 66.7, 200 over 5000 75.3 and 71.1, 1500 over 3000 137 and 149, 1024 tokens of 32 heads 68.5
// and 78; head dimension 64, 2 x 900 tokens of 8 heads over 5000 rows 106 us with one, 98.6 with two, 97.6 with four.
int splits(int num_cu, int D, int U, int n_qt, int max_tiles) {
  const int64_t items = (int64_t)U * n_qt;
  const int64_t want = ((D == 128 ? 1 : 2) * num_cu + items - 1) / items;
  return (int)std::max<int64_t>(1, std::min<int64_t>({want, (int64_t)kMaxSplit, (int64_t)(max_tiles + kMinTiles - 1) / kMinTiles}));
}

template <int D, int G>
hipError_t launch(ag_ctx *ctx, hipStream_t s, const pf_args &a) {
  const dim3 grid((unsigned)(a.U * a.n_qt * a.n_split));
  static std::atomic<bool> allowed[64];
  const hipError_t e = ag_q8_allow_lds(ctx->device, allowed, &ag_q8_prefill_kernel<D, G>, 4 * kQ8Block * D * 2);
  if (e != hipSuccess) return e;
  AG_LAUNCH(ag_time_kernel(ctx, AG_K_Q8_PREFILL), (ag_q8_prefill_kernel<D, G>), grid, dim3(256), 4 * kQ8Block * D * 2, s, a);
  if (a.n_split > 1)
    hipLaunchKernelGGL((ag_q8_prefill_merge_kernel<D, G>), dim3((unsigned)(a.U * a.n_qt * (kRows / (256 / (D / 4))))), dim3(256), 0, s, a);
  return hipGetLastError();
}
template <int D>
hipError_t launch_g(int G, ag_ctx *ctx, hipStream_t s, const pf_args &a) {
  switch (G) {
    case 1: return launch<D, 1>(ctx, s, a);
    case 2: return launch<D, 2>(ctx, s, a);
    case 4: return launch<D, 4>(ctx, s, a);
    case 8: return launch<D, 8>(ctx, s, a);
  }
  return hipErrorInvalidValue;
}

}  // namespace

void ag_q8_prefill_plan(int num_cu, int U, int Hq, int Hkv, int L, int D, int max_blocks, ws_cursor &ws, ag_q8_prefill_ws *w) {
  w->tiles = ws.take<uint16_t>((size_t)U * ag_q8_fill_blocks(L) * 2 * kQ8Block * D);
  w->info = ws.take<uint32_t>((size_t)U * ag_q8_fill_blocks(L));
  w->meta = ws.take<ag_q8_meta>(U);
  w->n_qt = (int)(((int64_t)L * (Hq / Hkv) + kRows - 1) / kRows);
  w->n_split = splits(num_cu, D, U, w->n_qt, max_blocks + ag_q8_fill_blocks(L));
  w->part = w->n_split > 1 ? ws.take<float>((size_t)U * w->n_qt * w->n_split * kRows * (D + 4)) : nullptr;
}

int ag_q8_prefill_shorter(int Hq, int Hkv, int L) {
  const int G = Hq / Hkv;
  return (int)((((int64_t)L * G + kRows - 1) / kRows - 1) * kRows / G);
}

hipError_t ag_launch_q8_prefill(ag_ctx *ctx, hipStream_t s, const void *q, const void *k, const void *v, int B, int Hq, int Hkv, int L,
                                int D, const uint64_t *words, const int32_t *blk_off, const ag_rope_dev &rope, float scale,
                                const ag_q8_dev &cache, const ag_q8_prefill_ws &w, void *out) {
  pf_args a;
  a.q = (const uint16_t *)q; a.k = (const uint16_t *)k; a.v = (const uint16_t *)v; a.out = (uint16_t *)out;
  a.words = words; a.blk_off = blk_off; a.tiles = w.tiles; a.info = w.info; a.meta = w.meta; a.c = cache; a.rope = rope;
  a.part = w.part; a.err = ctx->d_err;
  a.U = B * Hkv; a.Hq = Hq; a.Hkv = Hkv; a.L = L; a.nw = ag_nwords(L); a.n_blk = ag_q8_fill_blocks(L); a.n_qt = w.n_qt; a.n_split = w.n_split;
  a.qscale = scale * kLog2e;
  return D == 128 ? launch_g<128>(Hq / Hkv, ctx, s, a) : launch_g<64>(Hq / Hkv, ctx, s, a);
}
