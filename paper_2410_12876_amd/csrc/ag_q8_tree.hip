// A tree of drafted tokens over the paged 8-bit cache, in one launch: every node attends to the rows its unit holds, to the kept nodes above it
// and to itself.
//
// Query rows of a unit are its nodes' heads, r = t G + head; a wave owns 32 of them, a lane one column: S^T = K q^T, O^T = V^T p^T on
// v_mfma_f32_32x32x16.  Bound by the pages' bytes while a unit has few rows, beyond by the matrix instructions and the weights between them.
//   * A page goes from memory into the registers as it lies, and there, made f16 (exact, two values an instruction), into the product: its
//     16-byte pieces are 16 columns of a row (4 x 4 rows of a column) for either half of the wave, in the order in which the query's
//     (the weights') registers are.  No LDS, no barrier between pages; a page's registers are asked for again as soon as they are used up.
//   * A workgroup of 8 waves has RW groups of 32 rows and 8 / RW waves for each, which take every so many-th page; their states are added
//     up in LDS at the end.
//   * Work is one list of (unit, tile of RW groups) end to end, a tile's cost its pages and kUnitCost; a workgroup takes an equal range of it. Tiles
//     that lie in several ranges leave their states as records, the workgroup that comes last adds them up in order.
//   * The tail's rows and the nodes are one sequence of rows behind each other, 64 of them a tile in LDS, in bf16: keys (turned) as the sum of two
//     numbers, queries and weights too, so rows of any size keep 16 bits.  Nodes that a row may not see are masked by the bits of its
//     ancestors, which pointers that double in length find in log2(L) steps.  Rows with infinities or NaN are taken one by one in 32
//     bits, by those who see them.
//   * Queries, page values and page weights are f16 times powers of two, 11 bits of each; the weights' reference lies 2^-kQ8TopBits below the largest
//     of the page that set it and is moved only when weights pass 2^15.  A page's values are as large as f16 holds them unless a page of the
//     same wave has ones 2^kSpan as large: then less, or the weights of such a page (one of zeros, say) would be too small for f16 and its rows
//     missing from the row sum.
#include <algorithm>

#include "ag_q8.h"

namespace {

constexpr float kLog2e = 1.4426950408889634f;
constexpr int kWaves = 8, kThreads = 64 * kWaves;
constexpr int kPageBits = 6;   // a page's values are made as large as 2^15 (codes below 2^9)
constexpr int kSpan = 12;      // a page's values are scaled up at most 2^kSpan more than those of the page with the largest ones ...
constexpr int kLeastExp = -90; // ... and at most 2^90: exact still (codes down to 2^-9, scales to 2^-100), and row sums of 2^18 rows stay in range
constexpr int kUnitCost = 6;   // what a tile costs beside its pages, in pages
constexpr float kLocalBits = 9.f;  // rows that a tree and a tail can have: below 2^9
constexpr int kWords = kQ8TreeMost / 64;
constexpr int kMostRows = 32 * 4;  // rows of a tile, at most

struct tree_args {
  const uint16_t *q, *k, *v;
  const uint8_t *flags;
  const int32_t *parent;
  uint16_t *out;
  ag_q8_dev c;
  ag_rope_dev rope;
  float *rec;        // records [2 grid][RW] of kState bytes
  int32_t *tickets;  // [grid] pieces of the tile that begins in a range that have stored their record; zero between launches
  int32_t *err;
  int U, Hq, Hkv, L, g_log, n_tiles, least;  // least: the smallest range
  float qscale;
};

__device__ __forceinline__ float other_half(float x) { return __shfl_xor(x, 32, 64); }
// x 2^d, d <= 0, in two steps: references of pages of very different sizes lie further apart than a factor can be small
__device__ __forceinline__ float shrink(float x, float half) { return x * half * half; }
// Where values d .. d + 7 of row r lie in fragments of 32 rows (as units of 8 values): step (d / 64, d / 32 % 2, d / 8 % 2), half d / 16 % 2.
// (A 16-byte piece of a page, 16 columns, is a half's part of two steps.)
template <int D> __device__ __forceinline__ int frag_at(int r, int d) {
  const int step = d / 64 * 4 + d / 32 % 2 * 2 + d / 8 % 2;
  return (((r >> 5) * (D / 16) + step) * 2 + d / 16 % 2) * 32 + (r & 31);
}
// The first of the eight columns that half h has in a step.
__device__ __forceinline__ int step_col(int step, int h) { return step / 4 * 64 + step / 2 % 2 * 32 + h * 16 + step % 2 * 8; }

template <int D> struct sizes {
  static constexpr int KS = D / 16, DT = D / 32;
  static constexpr int kTile = kQ8Block * D;             // values of a tile
  static constexpr int kLocal = 3 * kTile * 2;           // bytes of a local tile: keys, what they leave over, values
  static constexpr int kState = DT * 4 * 1024 + 512;     // bytes of a wave's state: 64 lanes' values in fours, then maximum and sum
  static constexpr int kShared = 2 * kLocal > 4 * kState ? 2 * kLocal : 4 * kState;
  static constexpr int lds(int RW) { return kShared + RW * KS * 1024; }
};

template <int D, int RW>
__global__ __launch_bounds__(kThreads, 2) void ag_q8_tree_kernel(tree_args a) {
  constexpr int KC = D / 64, KS = D / 16, DT = D / 32, KW = kWaves / RW;
  typedef sizes<D> S;
  extern __shared__ __attribute__((aligned(1024))) uint8_t smem[];
  uint16_t *s_local = reinterpret_cast<uint16_t *>(smem);  // local tiles, or states
  uint16_t *s_q = reinterpret_cast<uint16_t *>(smem + S::kShared);
  __shared__ int32_t s_eq[32 * RW];
  __shared__ uint64_t s_above[kQ8TreeMost][kWords], s_keep[kWords], s_odd[2];
  __shared__ int32_t s_up[kQ8TreeMost];
  __shared__ int32_t s_sum[kWaves], s_start[2], s_last;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), rg = wave % RW, kg = wave / RW;
  const int wg = blockIdx.x, grid = gridDim.x, G = 1 << a.g_log, rows = a.L << a.g_log;
  const int most = a.c.max_blocks * kQ8Block + kQ8Block - 1;
  auto len_of = [&](int u) { return max(0, min(a.c.len[u], most)); };

  // ---- the work list: this workgroup's range ----
  int total = 0, quota, left, u, off;
  {
    const int tid = threadIdx.x, lane = tid & 63;
    const int per = (a.U + kThreads - 1) / kThreads, u0 = min(a.U, tid * per), u1 = min(a.U, u0 + per);
    int mine = 0, sum;
    for (int v = u0; v < u1; ++v) mine += (len_of(v) / kQ8Block + kUnitCost) * a.n_tiles;
    int before = ag_wave_prefix(mine, sum);
    if (lane == 0) s_sum[wave] = sum;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
      if (w < wave) before += s_sum[w];
      total += s_sum[w];
    }
    quota = max(a.least, (int)((uint32_t)(total + grid - 1) / (uint32_t)grid));
    const int64_t x64 = (int64_t)wg * quota;
    if (x64 >= total) return;
    const int x = (int)x64;
    left = min(quota, total - x);
    if (before <= x && x < before + mine) {
      int at = before, v = u0;
      for (;; ++v) {
        const int cost = (len_of(v) / kQ8Block + kUnitCost) * a.n_tiles;
        if (x < at + cost) break;
        at += cost;
      }
      s_start[0] = v;
      s_start[1] = x - at;
    }
    __syncthreads();
    u = __builtin_amdgcn_readfirstlane(s_start[0]);
    off = __builtin_amdgcn_readfirstlane(s_start[1]);
  }
  int at = wg * quota;  // position in the list

  for (;;) {
    int tid = threadIdx.x;
    asm volatile("" : "+v"(tid));  // (unknown to the compiler: it would keep every address below in registers from one tile to the next)
    const int lane = tid & 63, col = lane & 31, h = lane >> 5;
    const int len = __builtin_amdgcn_readfirstlane(len_of(u)), nb = len / kQ8Block, held = len & (kQ8Block - 1), cost = nb + kUnitCost;
    const int tile = off / cost, sub = off - tile * cost, take = min(cost - sub, left);
    const bool local = sub == 0;
    const int p0 = max(0, sub - kUnitCost), p1 = max(0, sub + take - kUnitCost);  // pages
    const int first = at - sub, g0 = (int)((uint32_t)first / (uint32_t)quota), n_rec = (int)((uint32_t)(first + cost - 1) / (uint32_t)quota) - g0 + 1;
    const int b = u / a.Hkv, row0 = tile * 32 * RW;
    const int my_row = row0 + rg * 32 + col, t = min(my_row >> a.g_log, a.L - 1);
    const bool active = row0 + rg * 32 < rows;  // this wave has rows
    const int32_t *page = a.c.page + (size_t)u * a.c.max_blocks;
    auto q_of = [&](int row) { return (((size_t)b * a.Hq + (size_t)(u % a.Hkv) * G + (row & (G - 1))) * a.L + (row >> a.g_log)) * D; };

    // ---- a wave's pages: lane x holds the number and the exponents of its page x, of at most 64 at a time ----
    int ids = -1, ek_v = 0, ev_v = 0, ev_least = kLeastExp;
    auto look_up = [&](int i0) {
      const int i = i0 + lane * KW, id = i < p1 ? page[i] : -1;
      const bool ok = (uint32_t)id < (uint32_t)a.c.n_pages;  // (a number outside the pool: rows that are not there)
      ids = ok ? id : -1;
      ek_v = (int)(__float_as_uint(a.c.k_scale[ok ? id : 0]) >> 23) - 127;
      ev_v = (int)(__float_as_uint(a.c.v_scale[ok ? id : 0]) >> 23) - 127 - kPageBits;
      int top = ok ? ev_v : -255;
#pragma unroll
      for (int o = 1; o < 64; o <<= 1) top = max(top, __shfl_xor(top, o, 64));
      ev_least = max(ev_least, __builtin_amdgcn_readfirstlane(top) - kSpan);
    };
    const int i0 = p0 + kg;
    if (active && i0 < p1) look_up(i0);

    // ---- the tile's queries, turned, in f16 times 2^eq each, into LDS in the order of the fragments ----
    for (int e = tid; e < 32 * RW * (D / 16); e += kThreads) {
      const int r = e / (D / 16), d = e % (D / 16) * 8, row = row0 + r;
      const bool there = row < rows;
      q8_eight y[2] = {};
      if (there) {
        const uint16_t *x = a.q + q_of(row) + d;
        const uint4 lo = *reinterpret_cast<const uint4 *>(x), hi = *reinterpret_cast<const uint4 *>(x + D / 2);
        if (a.rope.table) {
          const q8_rows turn = q8_rope_rows(a.rope, (int64_t)b * a.L + (row >> a.g_log), a.err);
          auto angles = [&](int i) { return q8_angles4(a.rope, turn, i, D); };
          y[0] = q8_turn8<D>(angles, d, lo, hi);
          y[1] = q8_turn8<D>(angles, d + D / 2, hi, lo);
        } else {
          y[0] = q8_floats(lo);
          y[1] = q8_floats(hi);
        }
      }
      float top = fmaxf(y[0].top(), y[1].top());  // (infinities are none of a binade's; NaN is passed over)
#pragma unroll
      for (int o = 1; o < D / 16; o <<= 1) top = fmaxf(top, __shfl_xor(top, o, 64));
      const int eq = max(kQ8TileMinExp, min(254, max(1, (int)(__float_as_uint(top) >> 23))) - 127 - kQ8TileTop);
      const float inv = q8_pow2(-eq);
      *reinterpret_cast<q8_f16x8 *>(s_q + frag_at<D>(r, d) * 8) = y[0].f16(inv);
      *reinterpret_cast<q8_f16x8 *>(s_q + frag_at<D>(r, d + D / 2) * 8) = y[1].f16(inv);
      if (d == 0) s_eq[r] = eq;
    }

    // ---- local rows: the tail's, then the nodes up to the tile's last one; 64 of them a tile ----
    const int n_nodes = local ? min(((row0 + 32 * RW - 1) >> a.g_log) + 1, a.L) : 0;
    const int n_local = local ? held + n_nodes : 0, n_lt = (n_local + kQ8Block - 1) / kQ8Block;
    const uint16_t *kt = a.c.k_tail + (size_t)u * kQ8Block * D, *vt = a.c.v_tail + (size_t)u * kQ8Block * D;
    const uint16_t *K = a.k + (size_t)u * a.L * D, *V = a.v + (size_t)u * a.L * D;
    auto finite8 = [](uint4 &x) {  // values that are not finite become 0; whether there were any
      uint32_t w[4] = {x.x, x.y, x.z, x.w};
      bool odd = false;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const bool lo = (w[i] & 0x7f80u) == 0x7f80u, hi = (w[i] & 0x7f800000u) == 0x7f800000u;
        odd |= lo || hi;
        w[i] &= (lo ? 0u : 0xffffu) | (hi ? 0u : 0xffff0000u);
      }
      x = make_uint4(w[0], w[1], w[2], w[3]);
      return odd;
    };
    // key row x (a node's turned, or a tail's), values d .. d + 7 and d + D / 2 .. + 7
    auto key_row = [&](int x, int d, q8_eight (&y)[2]) {
      if (x < held) {
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const int dd = d + e * (D / 2);
          y[e] = q8_floats(*reinterpret_cast<const uint4 *>(kt + q8_k_at<D>(x, dd / 64, dd / 16 % 4) * 16 + (d & 8)));
        }
        return;
      }
      const uint16_t *p = K + (size_t)(x - held) * D + d;
      const uint4 lo = *reinterpret_cast<const uint4 *>(p), hi = *reinterpret_cast<const uint4 *>(p + D / 2);
      if (a.rope.table) {
        const q8_rows turn = q8_rope_rows(a.rope, (int64_t)b * a.L + x - held, a.err);
        auto angles = [&](int i) { return q8_angles4(a.rope, turn, i, D); };
        y[0] = q8_turn8<D>(angles, d, lo, hi);
        y[1] = q8_turn8<D>(angles, d + D / 2, hi, lo);
      } else {
        y[0] = q8_floats(lo);
        y[1] = q8_floats(hi);
      }
    };
    auto stage = [&](int lt0) {  // local tiles lt0 and lt0 + 1 into LDS (s_odd is 0 before)
      for (int e = tid; e < 2 * kQ8Block * (D / 16); e += kThreads) {
        const int which = e / (kQ8Block * (D / 16)), r = e / (D / 16) % kQ8Block, d = e % (D / 16) * 8, x = (lt0 + which) * kQ8Block + r;
        if (lt0 + which >= n_lt) break;
        uint16_t *kh = s_local + which * 3 * S::kTile, *kl = kh + S::kTile, *vs = kl + S::kTile;
        q8_eight y[2] = {};
        uint4 vv[2] = {};
        bool odd = false;
        if (x < n_local) {
          key_row(x, d, y);
          if (x >= held) {
#pragma unroll
            for (int i = 0; i < 2; ++i) {
              vv[i] = *reinterpret_cast<const uint4 *>(V + (size_t)(x - held) * D + d + i * (D / 2));
              odd |= finite8(vv[i]);
            }
          } else {
            // a tail's row: its columns' values lie apart (column 16 f + r', row 16 i + 4 g + j: ((4 f + g) 16 + r') 16 + 4 i + j)
            const uint16_t *from = vt + (x >> 2 & 3) * 256 + (x >> 4) * 4 + (x & 3);
#pragma unroll
            for (int i = 0; i < 2; ++i) {
              const int dd = d + i * (D / 2);
              uint32_t w[4];
#pragma unroll
              for (int z = 0; z < 4; ++z)
                w[z] = from[(dd >> 4) * 1024 + ((dd & 15) + 2 * z) * 16] | (uint32_t)from[(dd >> 4) * 1024 + ((dd & 15) + 2 * z + 1) * 16] << 16;
              vv[i] = make_uint4(w[0], w[1], w[2], w[3]);
              odd |= finite8(vv[i]);
            }
          }
        }
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          uint4 hi = y[i].bf16();
          const bool any = finite8(hi);
          const q8_eight z = q8_floats(hi);
          uint4 lo = q8_eight{y[i].a - z.a, y[i].b - z.b}.bf16();
          odd |= any | finite8(lo);
          const int to = frag_at<D>(r, d + i * (D / 2)) * 8;
          *reinterpret_cast<uint4 *>(kh + to) = hi;
          *reinterpret_cast<uint4 *>(kl + to) = lo;
          // row r of column 32 f + c: step r / 16, half r / 4 % 2, element 4 (r / 8 % 2) + r % 4
          const uint32_t w[4] = {vv[i].x, vv[i].y, vv[i].z, vv[i].w};
#pragma unroll
          for (int z8 = 0; z8 < 8; ++z8) {
            const int c = d + i * (D / 2) + z8;
            vs[(((c >> 5) * 4 + (r >> 4)) * 64 + (r >> 2 & 1) * 32 + (c & 31)) * 8 + (r >> 3 & 1) * 4 + (r & 3)] = (uint16_t)(w[z8 / 2] >> (16 * (z8 & 1)));
          }
        }
        if (odd) atomicOr(reinterpret_cast<unsigned long long *>(&s_odd[which]), 1ull << r);
      }
    };
    if (local) {
      if (tid < 2) s_odd[tid] = 0;
      if (tid < kQ8TreeMost) {
        int up = -1;
        bool keep = false;
        if (tid < n_nodes) {
          up = a.parent[(size_t)b * a.L + tid];
          keep = !a.flags || a.flags[(size_t)u * a.L + tid] != 0;
          if (up >= tid) {
            atomicOr(a.err, 4);
            up = -1;
          }
        }
        s_up[tid] = max(-1, up);
#pragma unroll
        for (int w = 0; w < kWords; ++w) s_above[tid][w] = tid >> 6 == w ? 1ull << (tid & 63) : 0;
        const uint64_t kept = __ballot(keep);
        if (lane == 0) s_keep[wave] = kept;
      }
    }
    __syncthreads();
    if (local) {
      stage(0);
      for (int n = 1; n < n_nodes; n *= 2) {  // node t knows the n nodes from itself up; s_up: the next one
        uint64_t more[kWords] = {};
        int up = -1, next = -1;
        if (tid < n_nodes) {
          up = s_up[tid];
          if (up >= 0) {
#pragma unroll
            for (int w = 0; w < kWords; ++w) more[w] = s_above[up][w];
            next = s_up[up];
          }
        }
        __syncthreads();
        if (up >= 0) {
#pragma unroll
          for (int w = 0; w < kWords; ++w) s_above[tid][w] |= more[w];
          s_up[tid] = next;
        }
        __syncthreads();
      }
      if (n_nodes == 1) __syncthreads();
    }

    // ---- the pages ----
    q8_f16x8 qx[KS];
    q8_f32x16 o[DT];
    float m = kQ8EmptyMax, l = 0.f;
#pragma unroll
    for (int i = 0; i < KS; ++i) qx[i] = *reinterpret_cast<const q8_f16x8 *>(s_q + ((rg * KS + i) * 64 + lane) * 8);
    const int eq = s_eq[rg * 32 + col];
#pragma unroll
    for (int dt = 0; dt < DT; ++dt)
#pragma unroll
      for (int i = 0; i < 16; ++i) o[dt][i] = 0.f;
    uint32_t p[2][8];
    if (active && i0 < p1) {
      bool fresh = true;
      q8_u32x4 bk[2][KC][2], bv[DT][2];
      const int k_lane = (col >> 4) * KC * 1024 + h * 256 + (col & 15) * 16, v_lane = (col >> 4) * 1024 + h * 256 + (col & 15) * 16;
      constexpr int kAux = RW == 1 ? 2 : 0;  // (pages that other waves do not read too: non-temporal)
      auto rsrc_of = [&](const uint8_t *pool, int x) {
        const int id = max(0, __builtin_amdgcn_readlane(ids, x));
        return __builtin_amdgcn_make_buffer_rsrc((void *)(pool + (size_t)id * (kQ8Block * D)), 0, kQ8Block * D, 0x00020000);
      };
      auto load_k = [&](int x) {
        const __amdgpu_buffer_rsrc_t r = rsrc_of(a.c.k, x);
#pragma unroll
        for (int y = 0; y < 2; ++y)
#pragma unroll
          for (int c = 0; c < KC; ++c)
#pragma unroll
            for (int j = 0; j < 2; ++j) bk[y][c][j] = __builtin_amdgcn_raw_buffer_load_b128(r, k_lane, y * 2 * KC * 1024 + c * 1024 + j * 512, kAux);
      };
      auto load_v = [&](int x) {
        const __amdgpu_buffer_rsrc_t r = rsrc_of(a.c.v, x);
#pragma unroll
        for (int dt = 0; dt < DT; ++dt)
#pragma unroll
          for (int j = 0; j < 2; ++j) bv[dt][j] = __builtin_amdgcn_raw_buffer_load_b128(r, v_lane, dt * 2048 + j * 512, kAux);
      };
      for (int first_page = i0;;) {
        const int n = min(64, (p1 - first_page + KW - 1) / KW);
        load_k(0);
        load_v(0);
        for (int x = 0; x < n; ++x) {
          const bool now = __builtin_amdgcn_readlane(ids, x) >= 0;
          q8_f32x16 s[2];
#pragma unroll
          for (int y = 0; y < 2; ++y)
#pragma unroll
            for (int i = 0; i < 16; ++i) s[y][i] = 0.f;
#pragma unroll
          for (int c = 0; c < KC; ++c)
#pragma unroll
            for (int j = 0; j < 2; ++j)
#pragma unroll
              for (int e = 0; e < 2; ++e)
#pragma unroll
                for (int y = 0; y < 2; ++y)
                  s[y] = __builtin_amdgcn_mfma_f32_32x32x16_f16(q8_widen16(bk[y][c][j][2 * e], bk[y][c][j][2 * e + 1], 1.f), qx[c * 4 + j * 2 + e], s[y], 0, 0, 0);
          if (x + 1 < n) load_k(x + 1);
          if (now) {
            // s[y][i]: row 32 y + 8 (i / 4) + 4 h + i % 4 of the page.  The state is kept relative to m, the largest score plus its page's
            // exponent ev of V less kQ8TopBits: weights are 2^(score + ev - m) in f16, values v 2^-ev, the page's part of the row sum 2^-ev the sum
            // of its weights as the product takes them.
            const int e = __builtin_amdgcn_readlane(ev_v, x), ev = max(ev_least, e);
            const float f = q8_unscale(a.qscale, eq + __builtin_amdgcn_readlane(ek_v, x));
            float sum = 0.f;
            auto weigh = [&] {
              const float shift = (float)ev - m;
              float part[2] = {0.f, 0.f};
#pragma unroll
              for (int y = 0; y < 2; ++y)
#pragma unroll
                for (int i = 0; i < 16; i += 2) {
                  const q8_f32x2 w = {__builtin_amdgcn_exp2f(fmaf(s[y][i], f, shift)), __builtin_amdgcn_exp2f(fmaf(s[y][i + 1], f, shift))};
                  p[y][i / 2] = __builtin_bit_cast(uint32_t, __builtin_convertvector(w, q8_f16x2));
                  asm volatile("" : "+v"(p[y][i / 2]));  // (packed here: the compiler would carry all 32 weights to the second product)
                  part[i / 2 & 1] = q8_add2(p[y][i / 2], part[i / 2 & 1]);
                }
              sum = part[0] + part[1];
            };
            if (!fresh) weigh();
            if (fresh || __any(!(sum <= 32768.f))) {  // no reference yet, or too far below: a new one, and the weights again
              float mx = -INFINITY;
#pragma unroll
              for (int y = 0; y < 2; ++y)
#pragma unroll
                for (int i = 0; i < 16; ++i) mx = fmaxf(mx, s[y][i]);
              mx = fmaf(fmaxf(mx, other_half(mx)), f, (float)(ev - kQ8TopBits));
              const float over = sum <= 32768.f ? 0.f : 1.f;
              const float m_new = fresh || fmaxf(over, other_half(over)) > 0.f ? fmaxf(m, mx) : m;  // (a row's own reference alone)
              const float alpha = __builtin_amdgcn_exp2f(0.5f * (m - m_new));
              l = shrink(l, alpha);
#pragma unroll
              for (int dt = 0; dt < DT; ++dt) o[dt] = o[dt] * alpha * alpha;
              m = m_new;
              fresh = false;
              weigh();
            }
            l += ldexpf(sum, -ev);
            const float scale = q8_pow2(e + kPageBits - ev);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const q8_f16x8 pb = __builtin_bit_cast(q8_f16x8, make_uint4(p[i >> 1][4 * (i & 1)], p[i >> 1][4 * (i & 1) + 1], p[i >> 1][4 * (i & 1) + 2], p[i >> 1][4 * (i & 1) + 3]));
#pragma unroll
              for (int dt = 0; dt < DT; ++dt)
                o[dt] = __builtin_amdgcn_mfma_f32_32x32x16_f16(q8_widen16(bv[dt][0][i], bv[dt][1][i], scale), pb, o[dt], 0, 0, 0);
            }
          }
          if (x + 1 < n) load_v(x + 1);
        }
        first_page += 64 * KW;
        if (first_page >= p1) break;
        look_up(first_page);
      }
    }

    // ---- the local rows ----
    if (local) {
      const float f = q8_unscale(a.qscale, eq);
      uint64_t see[kWords];  // the nodes that this lane's row sees, itself among them
      bool sole = nb == 0 && held == 0;
#pragma unroll
      for (int w = 0; w < kWords; ++w) {
        const uint64_t own = t >> 6 == w ? 1ull << (t & 63) : 0, others = s_above[t][w] & s_keep[w] & ~own;
        see[w] = own | others;
        sole = sole && others == 0;
      }
      const float above = sole ? 0.f : kLocalBits;  // (alone its weight is exactly 1)
      auto seen = [&](int lt) {  // of local tile lt, as bits: rows before `held`, then nodes
        const int first_row = lt * kQ8Block, n0 = first_row - held;  // node of the tile's row 0 (negative: a row of the tail, in tile 0 alone)
        uint64_t w = n0 < 0 ? (held < 64 ? (1ull << held) - 1 : ~0ull) | see[0] << (-n0) : 0;
        if (n0 >= 0) {
#pragma unroll
          for (int i = 0; i < kWords; ++i) {
            if (i == n0 >> 6) w |= see[i] >> (n0 & 63);
            if (i == (n0 >> 6) + 1 && (n0 & 63) != 0) w |= see[i] << (64 - (n0 & 63));
          }
        }
        return w;
      };
      for (int lt0 = 0; lt0 < n_lt; lt0 += 2) {
        if (lt0 > 0) {
          __syncthreads();
          if (tid < 2) s_odd[tid] = 0;
          __syncthreads();
          stage(lt0);
          __syncthreads();
        }
        for (int which = 0; which < 2; ++which) {
          const int lt = lt0 + which, own = held + t - lt * kQ8Block;  // own: the tile's row that is this lane's own node
          if (lt >= n_lt || !active || lt % KW != KW - 1 - kg) continue;
          const uint64_t all = seen(lt), odd = s_odd[which], bits = all & ~odd;
          if (__any(bits != 0)) {
            const uint16_t *kh = s_local + which * 3 * S::kTile + lane * 8, *kl = kh + S::kTile, *vs = kl + S::kTile;
            q8_f32x16 s[2];
#pragma unroll
            for (int y = 0; y < 2; ++y)
#pragma unroll
              for (int i = 0; i < 16; ++i) s[y][i] = 0.f;
#pragma unroll
            for (int k = 0; k < KS; ++k) {
              q8_f16x8 q = qx[k];
              asm volatile("" : "+v"(q));  // (or the compiler would keep both parts of the query across the loop)
              const q8_eight y = {{(float)q[0], (float)q[1], (float)q[2], (float)q[3]}, {(float)q[4], (float)q[5], (float)q[6], (float)q[7]}};
              const uint4 hi = y.bf16();
              const q8_eight z = q8_floats(hi);
              const q8_bf16x8 qh = __builtin_bit_cast(q8_bf16x8, hi), ql = __builtin_bit_cast(q8_bf16x8, q8_eight{y.a - z.a, y.b - z.b}.bf16());
#pragma unroll
              for (int x = 0; x < 2; ++x) {
                const q8_bf16x8 first_part = *reinterpret_cast<const q8_bf16x8 *>(kh + (x * KS + k) * 512);
                s[x] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(first_part, ql, s[x], 0, 0, 0);
                s[x] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(*reinterpret_cast<const q8_bf16x8 *>(kl + (x * KS + k) * 512), qh, s[x], 0, 0, 0);
                s[x] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(first_part, qh, s[x], 0, 0, 0);
              }
            }
            float mx = -INFINITY;
#pragma unroll
            for (int x = 0; x < 2; ++x) {
              const uint32_t w = (uint32_t)(bits >> (32 * x)) >> (4 * h);
#pragma unroll
              for (int i = 0; i < 16; ++i) {
                const int r = 8 * (i / 4) + i % 4;
                s[x][i] *= f;
                // its own node: alone its weight is 1 whatever its score is; a score that overflowed to -infinity counts as the least number
                if (32 * x + r + 4 * h == own) s[x][i] = sole ? 0.f : (s[x][i] < kQ8EmptyMax ? kQ8EmptyMax : s[x][i]);
                if (!(w >> r & 1)) s[x][i] = -INFINITY;
                mx = fmaxf(mx, s[x][i]);
              }
            }
            // (the weights are bf16: the reference lies above the largest, so that rows of the largest values do not add up to infinity)
            const float m_new = fmaxf(m, fmaxf(mx, other_half(mx)) + above), alpha = __builtin_amdgcn_exp2f(0.5f * (m - m_new));
            l = shrink(l, alpha);
#pragma unroll
            for (int dt = 0; dt < DT; ++dt) o[dt] = o[dt] * alpha * alpha;
            m = m_new;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              uint32_t hi[4], lo[4];
#pragma unroll
              for (int z = 0; z < 4; ++z) {
                const int at_s = 8 * (i & 1) + 2 * z;
                const float w0 = __builtin_amdgcn_exp2f(s[i >> 1][at_s] - m), w1 = __builtin_amdgcn_exp2f(s[i >> 1][at_s + 1] - m);
                l += w0 + w1;
                hi[z] = q8_pack2(w0, w1);
                lo[z] = q8_pack2(w0 - q8_lo(hi[z]), w1 - q8_hi(hi[z]));
              }
              const q8_bf16x8 ph = __builtin_bit_cast(q8_bf16x8, make_uint4(hi[0], hi[1], hi[2], hi[3])), pl = __builtin_bit_cast(q8_bf16x8, make_uint4(lo[0], lo[1], lo[2], lo[3]));
#pragma unroll
              for (int dt = 0; dt < DT; ++dt) {
                const q8_bf16x8 vf = *reinterpret_cast<const q8_bf16x8 *>(vs + (dt * 4 + i) * 512);
                o[dt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf, pl, o[dt], 0, 0, 0);
                o[dt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf, ph, o[dt], 0, 0, 0);
              }
            }
          }
          for (uint64_t left_over = odd; left_over; left_over &= left_over - 1) {  // rare: rows with infinities or NaN, one by one in 32 bits
            const int r = __builtin_ctzll(left_over), x = lt * kQ8Block + r;
            const bool mine = all >> r & 1;
            if (!__any(mine)) continue;
            float s = 0.f;
            for (int k = 0; k < KS; ++k) {
              const int d = step_col(k, h);
              q8_eight y[2];
              key_row(x, d & (D / 2 - 1), y);
              const q8_eight z = d < D / 2 ? y[0] : y[1];
              const q8_f16x8 q = *reinterpret_cast<const q8_f16x8 *>(s_q + ((rg * KS + k) * 64 + lane) * 8);
#pragma unroll
              for (int i = 0; i < 4; ++i) s = fmaf((float)q[i], z.a[i], fmaf((float)q[4 + i], z.b[i], s));
            }
            s = (s + other_half(s)) * f;
            if (r == own) s = sole ? 0.f : (s < kQ8EmptyMax ? kQ8EmptyMax : s);
            if (!mine) continue;
            const float m_new = fmaxf(m, (s < kQ8EmptyMax ? kQ8EmptyMax : s) + above);
            const float alpha = __builtin_amdgcn_exp2f(0.5f * (m - m_new)), w = __builtin_amdgcn_exp2f(s - m_new);
            m = m_new;
            l = shrink(l, alpha) + (h == 0 ? w : 0.f);
#pragma unroll
            for (int dt = 0; dt < DT; ++dt) {
              asm volatile("" ::: "memory");  // (a few loads at a time)
#pragma unroll
              for (int i = 0; i < 16; ++i) {
                const int d = 32 * dt + 8 * (i / 4) + 4 * h + i % 4;
                const uint16_t val = x < held ? vt[((d >> 4) * 4 + (x >> 2 & 3)) * 256 + (d & 15) * 16 + (x >> 4) * 4 + (x & 3)] : V[(size_t)(x - held) * D + d];
                o[dt][i] = shrink(o[dt][i], alpha) + w * __uint_as_float((uint32_t)val << 16);
              }
            }
          }
        }
      }
    }

    // ---- the states of the workgroup's waves, then of the tile's pieces ----
    // (sixteen bytes a lane; records are written through and read past the caches, sc0 and sc1)
    constexpr int kThrough = 17;
    auto join = [&](q8_f32x2 ml, auto &&value) {  // this lane's state and another one of the same row: value(i) its values 4 i .. 4 i + 3
      const float M = fmaxf(m, ml[0]), f1 = __builtin_amdgcn_exp2f(0.5f * (m - M)), f2 = __builtin_amdgcn_exp2f(0.5f * (ml[0] - M));
      m = M;
      l = shrink(l, f1) + shrink(ml[1], f2);
#pragma unroll
      for (int i = 0; i < DT * 4; ++i) {
        const q8_f32x4 x = value(i);
#pragma unroll
        for (int r = 0; r < 4; ++r) o[i / 4][4 * (i % 4) + r] = shrink(o[i / 4][4 * (i % 4) + r], f1) + shrink(x[r], f2);
      }
    };
    auto four = [&](int i) { return q8_f32x4{o[i / 4][4 * (i % 4)], o[i / 4][4 * (i % 4) + 1], o[i / 4][4 * (i % 4) + 2], o[i / 4][4 * (i % 4) + 3]}; };
    int me = lane;
    asm volatile("" : "+v"(me));  // (unknown to the compiler: or the addresses below would be kept in registers all the way)
    auto gather = [&] {  // into the waves with kg = 0
#pragma unroll
      for (int n = KW / 2; n >= 1; n /= 2) {
        __syncthreads();
        uint8_t *st = smem + ((kg >= n ? kg - n : kg) * RW + rg) * S::kState;
        if (kg >= n && kg < 2 * n) {
#pragma unroll
          for (int i = 0; i < DT * 4; ++i) *reinterpret_cast<q8_f32x4 *>(st + i * 1024 + me * 16) = four(i);
          *reinterpret_cast<q8_f32x2 *>(st + DT * 4 * 1024 + me * 8) = q8_f32x2{m, l};
        }
        __syncthreads();
        if (kg < n) join(*reinterpret_cast<const q8_f32x2 *>(st + DT * 4 * 1024 + me * 8), [&](int i) { return *reinterpret_cast<const q8_f32x4 *>(st + i * 1024 + me * 16); });
      }
    };
    auto store = [&] {
      l += other_half(l);
      const int row = row0 + rg * 32 + (me & 31);
      if (kg == 0 && row < rows) {
        const float inv = 1.f / l;
        uint16_t *to = a.out + q_of(row) + 4 * (me >> 5);
#pragma unroll
        for (int dt = 0; dt < DT; ++dt)
#pragma unroll
          for (int x = 0; x < 4; ++x)
            *reinterpret_cast<uint2 *>(to + 32 * dt + 8 * x) =
                make_uint2(q8_pack2(o[dt][4 * x] * inv, o[dt][4 * x + 1] * inv), q8_pack2(o[dt][4 * x + 2] * inv, o[dt][4 * x + 3] * inv));
      }
    };
    gather();
    if (n_rec == 1) {
      store();
    } else {
      auto rec_at = [&](int k) {
        return __builtin_amdgcn_make_buffer_rsrc(a.rec + ((size_t)(2 * (g0 + k) + (k == 0)) * RW + rg) * (S::kState / 4), 0, S::kState, 0x00020000);
      };
      if (kg == 0) {
        const __amdgpu_buffer_rsrc_t to = rec_at(wg - g0);
#pragma unroll
        for (int i = 0; i < DT * 4; ++i) __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(q8_u32x4, four(i)), to, me * 16, i * 1024, kThrough);
        const q8_f32x2 ml = {m, l};
        __builtin_amdgcn_raw_buffer_store_b64(__builtin_bit_cast(q8_u32x2, ml), to, me * 8, DT * 4 * 1024, kThrough);
      }
      asm volatile("s_waitcnt vmcnt(0)" ::: "memory");  // this wave's part of the record is in memory
      __syncthreads();
      if (tid == 0) s_last = __hip_atomic_fetch_add(&a.tickets[g0], 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == n_rec - 1;
      __syncthreads();
      if (s_last) {  // all pieces are there: every wave adds up every so many-th, in order
        if (tid == 0) a.tickets[g0] = 0;
        m = kQ8EmptyMax;
        l = 0.f;
#pragma unroll
        for (int dt = 0; dt < DT; ++dt)
#pragma unroll
          for (int i = 0; i < 16; ++i) o[dt][i] = 0.f;
        for (int k = kg; k < n_rec; k += KW) {
          const __amdgpu_buffer_rsrc_t from = rec_at(k);
          join(__builtin_bit_cast(q8_f32x2, __builtin_amdgcn_raw_buffer_load_b64(from, me * 8, DT * 4 * 1024, kThrough)),
               [&](int i) { return __builtin_bit_cast(q8_f32x4, __builtin_amdgcn_raw_buffer_load_b128(from, me * 16, i * 1024, kThrough)); });
        }
        gather();
        store();
      }
    }
    left -= take;
    at += take;
    if (left <= 0) break;
    off += take;
    if (off >= cost * a.n_tiles) {
      ++u;
      off = 0;
    }
    __syncthreads();  // (LDS is written again)
  }
}

// Groups of 32 rows that a workgroup takes.
int row_groups(int rows) { return rows <= 32 ? 1 : rows <= 64 ? 2 : 4; }
int tiles_of(int rows) { return (rows + kMostRows - 1) / kMostRows; }

template <int D, int RW>
hipError_t launch(ag_ctx *ctx, hipStream_t s, tree_args &a) {
  static std::atomic<bool> allowed[64];
  const hipError_t e = ag_q8_allow_lds(ctx->device, allowed, &ag_q8_tree_kernel<D, RW>, sizes<D>::lds(RW));
  if (e != hipSuccess) return e;
  a.least = kWaves / RW + kUnitCost;
  const int64_t most = ag_q8_tree_cost(a.U, a.L << a.g_log, a.c.max_blocks);
  const int grid = (int)std::min<int64_t>(ctx->num_cu, std::max<int64_t>(1, (most + a.least - 1) / a.least));
  AG_LAUNCH(ag_time_kernel(ctx, AG_K_Q8_TREE), (ag_q8_tree_kernel<D, RW>), dim3(grid), dim3(kThreads), sizes<D>::lds(RW), s, a);
  return hipGetLastError();
}
template <int D>
hipError_t launch_rows(ag_ctx *ctx, hipStream_t s, tree_args &a) {
  switch (row_groups(a.L << a.g_log)) {
    case 1: return launch<D, 1>(ctx, s, a);
    case 2: return launch<D, 2>(ctx, s, a);
    default: return launch<D, 4>(ctx, s, a);
  }
}

}  // namespace

// (and what rounding up to whole ranges adds)
int64_t ag_q8_tree_cost(int64_t units, int rows, int max_blocks) { return units * ((int64_t)max_blocks + kUnitCost) * tiles_of(rows) + (1 << 16); }

size_t ag_ws_q8_tree_floats(int num_cu, int rows, int D) { return (size_t)2 * num_cu * row_groups(rows) * (D / 32 * 4 * 1024 + 512) / 4; }

hipError_t ag_launch_q8_tree(ag_ctx *ctx, hipStream_t s, const void *q, const void *k, const void *v, const uint8_t *flags, const int32_t *parent,
                             int B, int Hq, int Hkv, int L, int D, const ag_rope_dev &rope, float scale, const ag_q8_dev &cache, void *out, float *rec) {
  tree_args a;
  a.q = (const uint16_t *)q; a.k = (const uint16_t *)k; a.v = (const uint16_t *)v; a.flags = flags; a.parent = parent; a.out = (uint16_t *)out;
  a.c = cache; a.rope = rope; a.rec = rec; a.tickets = ctx->decode_tickets; a.err = ctx->d_err;
  a.U = B * Hkv; a.Hq = Hq; a.Hkv = Hkv; a.L = L;
  a.g_log = 0;
  while (Hkv << a.g_log < Hq) ++a.g_log;
  a.n_tiles = tiles_of(L << a.g_log);
  a.least = 0;
  a.qscale = scale * kLog2e;
  return D == 128 ? launch_rows<128>(ctx, s, a) : launch_rows<64>(ctx, s, a);
}
