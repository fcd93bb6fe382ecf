// A tree of drafted tokens over the paged 8-bit cache, in one launch: every node attends to the rows its unit holds, to the kept nodes above it
// and to itself.
//
// Query rows of a unit are its nodes' heads, r = t G + head; a wave owns 32 of them, a lane one column: S^T = K q^T, O^T = V^T p^T on
// v_mfma_f32_32x32x16.  Bound by the pages' bytes while a unit has few rows (32 rows: 0.65 us a page of 16 KiB a CU, 6.5 TB/s; 64: 0.83 us, 5.05 TB/s),
// beyond by the matrix instructions and the conversions and weights between them (128: 1.30 us, 0.82 PFLOP/s).  A short call is a chain of
// round trips: 12 nodes over 777 rows 14.8 us (D = 64: 11.3); 16 x 31 nodes over 4096 rows 40.5 us (28.7), of which the pages take 23, the start 8 and the
// meetings 7.  More units than CUs are rounds of that chain: 512 units of 8 nodes over 400 rows 34 us, 1024 64 (over 1600 rows 89).
//   * A page goes from memory into the registers as it lies, and there, made f16 (exact, two values an instruction), into the product: its
//     16-byte pieces are 16 columns of a row (4 x 4 rows of a column) for either half of the wave, in the order in which the query's
//     (the weights') registers are.  No LDS, no barrier between pages; a page's registers are asked for again as soon as they are used up.
//     (Through LDS, where the groups share one copy: 1.30 against 1.35 us a page then, but with room for fewer local rows 62 against 57 us for
//     4 x 64 nodes over 13000.)
//   * A workgroup of 8 waves, one a CU (two of 4 waves: 50 against 46 us for 16 x 31 nodes), has RW groups of 32 rows and 8 / RW waves for each, which
//     take every so many-th page; their states are added up in LDS at the end.
//   * Every tile (a unit's RW groups) is cut into pieces by its cost, its pages and kUnitCost; a workgroup takes one piece.  (Equal ranges of all tiles
//     end to end balance better, but what lives across that loop cost more: 83 against 57 us for 16 x 31 nodes.)  The pieces of a cut tile leave
//     their states as records, and the one that comes last adds them up in order.
//   * The tail's rows and the nodes are one sequence of rows behind each other, 128 at a time (two tiles of 64) in LDS: keys (turned) in f16 times
//     a power of two for each, values in bf16 and weights as the sum of two bf16, so rows of any size keep 11 and 16 bits.  Nodes that a row may not
//     see are masked by the bits of its ancestors, which pointers that double in length find in log2(L) steps.  Rows with infinities or NaN are
//     taken one by one in 32 bits, by those who see them.  The waves that leave their pages first, the older ones, take them (42 -> 40.5 us).
//   * Queries, page values and page weights are f16 times powers of two: 11 bits of a query and of a weight, all of a value's 4.  The weights'
//     reference lies 2^-kQ8TopBits below the largest of the page that set it and is moved only when weights pass 2^15.  Pages of far smaller values
//     than others add to the row sum in 32 bits (kQ8Span): 32 more exponentials a lane, in such pages alone.
#include <algorithm>

#include "ag_q8.h"

namespace {

constexpr float kLog2e = 1.4426950408889634f;
typedef __attribute__((__vector_size__(4 * sizeof(__bf16)))) __bf16 bf16x4;
constexpr int kWaves = 8, kThreads = 64 * kWaves;
constexpr int kMostUnits = 8 * 64;  // units up to which every wave goes through the list by itself
constexpr int kPageBits = 6;   // a page's values are made as large as 2^15 (codes below 2^9)
constexpr int kUnitCost = 10;   // what a tile costs beside its pages, in pages (16 x 31 nodes over 4096 rows 40.4 us, 4 x 64 over 13000 51.0; 6: 41.4, 51.9; 14: 42.0, 51.7)
constexpr float kLocalBits = 9.f;  // rows that a tree and a tail can have: below 2^9
constexpr int kWords = kQ8TreeMost / 64;

struct tree_args {
  const uint16_t *q, *k, *v;
  const uint8_t *flags;
  const int32_t *parent;
  uint16_t *out;
  ag_q8_dev c;
  ag_rope_dev rope;
  float *rec;        // records [2 places][RW] of kState bytes: only tiles that are cut have any, so those are less than twice as many as places
  int32_t *tickets;  // [2 places] pieces of the tile whose first record that is that have stored theirs; zero between launches
  int32_t *err;
  int U, Hq, Hkv, L, g_log, n_tiles, least, places, slots;  // least: the least cost of a piece; places: workgroups that run at once, slots: for a tile of every unit
  float qscale;
};

__device__ __forceinline__ float other_half(float x) { return __shfl_xor(x, 32, 64); }
// x 2^d, d <= 0, in two steps: references of pages of very different sizes lie further apart than a factor can be small
__device__ __forceinline__ float shrink(float x, float half) { return x * half * half; }
// Eight values of row r of a group of 32 (as units of 8 values): fragment by fragment, in an order of the rows that keeps the eight pieces of a
// row that neighbouring lanes write in different banks.
template <int D> __device__ __forceinline__ int fragment(int group, int step, int half, int r) {
  const int unit = step * 2 + half;
  return (group * (D / 8) + unit) * 32 + (r ^ (unit & 7));
}
// Where values d .. d + 7 of row r lie in fragments of 32 rows (as units of 8 values): step (d / 64, d / 32 % 2, d / 8 % 2), half d / 16 % 2.
// (A 16-byte piece of a page, 16 columns, is a half's part of two steps.)
template <int D> __device__ __forceinline__ int frag_at(int r, int d) {
  const int step = d / 64 * 4 + d / 32 % 2 * 2 + d / 8 % 2;
  return fragment<D>(r >> 5, step, d / 16 % 2, r & 31);
}
// Where the 16-byte piece c of a value row lies: rows of D, their pieces in an order that keeps the four rows of a transposing read, and the rows
// that a wave writes, in different banks.
template <int D> __device__ __forceinline__ int value_at(int r, int c) { return r * D + (c ^ (D == 128 ? (r & 3) << 2 | (r >> 2 & 3) : (r & 3) << 1 | (r >> 2 & 1))) * 8; }
// The first of the eight columns that half h has in a step.
__device__ __forceinline__ int step_col(int step, int h) { return step / 4 * 64 + step / 2 % 2 * 32 + h * 16 + step % 2 * 8; }

// A barrier that waits for LDS alone: loads and stores stay in flight.
__device__ __forceinline__ void barrier() {
  asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
}
// n / d and what is left for 0 <= n < 2^22, 0 < d < 2^22 (an integer division is forty instructions)
struct quotient {
  int q, r;
};
__device__ __forceinline__ quotient divide(int n, int d) {
  int q = (int)((float)n * __builtin_amdgcn_rcpf((float)d)), r = n - q * d;
  if (r < 0) --q, r += d;
  if (r >= d) ++q, r -= d;
  return quotient{q, r};
}

template <int D> struct sizes {
  static constexpr int KS = D / 16, DT = D / 32;
  static constexpr int kTile = kQ8Block * D;          // values of a tile
  static constexpr int kState = DT * 4 * 1024 + 512;  // bytes of a wave's state: 64 lanes' values in fours, then maximum and sum
  static constexpr int lds(int RW) { return std::max(4 * kTile * 2 + RW * KS * 1024, kWaves * kState); }
};

// Positions of a token, and the table's rows of them (apart: so that many are on their way at once).
struct place {
  int32_t p[3];
};
__device__ __forceinline__ place place_of(const ag_rope_dev &r, int64_t token) {
  place x;
  x.p[0] = r.pos[token];
  x.p[1] = r.n_axes > 1 ? r.pos[r.axis_stride + token] : x.p[0];
  x.p[2] = r.n_axes > 2 ? r.pos[2 * r.axis_stride + token] : x.p[0];
  return x;
}
__device__ __forceinline__ q8_rows rows_of(const ag_rope_dev &r, const place &x, int32_t *err) {
  const uint32_t n = r.n_rows;
  if ((uint32_t)x.p[0] >= n || (uint32_t)x.p[1] >= n || (uint32_t)x.p[2] >= n) atomicOr(err, 2);  // reported, and turned by the nearest row
  auto near = [&](int p) { return (uint32_t)min(max(p, 0), r.n_rows - 1); };
  return q8_rows{near(x.p[0]), near(x.p[1]), near(x.p[2])};
}
// Exponent of a row of f16 whose largest magnitude is top (infinities are none of a binade's).
__device__ __forceinline__ int row_exponent(float top) { return max(kQ8TileMinExp, min(254, max(1, (int)(__float_as_uint(top) >> 23))) - 127 - kQ8TileTop); }

template <int D, int RW>
__global__ __launch_bounds__(kThreads, 2) void ag_q8_tree_kernel(tree_args a) {
  constexpr int KC = D / 64, KS = D / 16, DT = D / 32, KW = kWaves / RW, VR = D / 16;  // VR: threads of a row
  typedef sizes<D> S;
  extern __shared__ __attribute__((aligned(1024))) uint8_t smem[];
  uint16_t *s_k = reinterpret_cast<uint16_t *>(smem), *s_v = s_k + 2 * S::kTile, *s_q = s_v + 2 * S::kTile;  // two local tiles, the queries; or states
  __shared__ int32_t s_eq[32 * RW], s_ek[2 * kQ8Block];
  __shared__ uint64_t s_above[kQ8TreeMost][kWords], s_keep[kWords], s_odd[2];
  __shared__ int32_t s_up[kQ8TreeMost];
  __shared__ int32_t s_sum[kWaves][3], s_start[4], s_last;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), rg = wave % RW, kg = wave / RW;
  const int wg = blockIdx.x, G = 1 << a.g_log, rows = a.L << a.g_log;
  const int most = a.c.max_blocks * kQ8Block + kQ8Block - 1;
  auto len_of = [&](int u) { return max(0, min(a.c.len[u], most)); };
  auto cost_of = [&](int len) { return len / kQ8Block + kUnitCost; };

  // ---- the work list: this workgroup's tile, and which of its pieces ----
  // A tile is cut into n = cost / (cost of a piece) pieces, rounded up.  Where there are no more tiles than places for workgroups, the cost of
  // a piece is the least for which every piece has a place; else as much as fills the places once.
  int u = 0, tile, piece, pieces = 1, rec0 = 0;  // rec0: the record of the tile's first piece
  {
    const int tid = threadIdx.x, lane = tid & 63;
    auto n_of = [](int cost, float inv) { return (int)ceilf((float)cost * inv * 0.9999f); };  // (1 for the longest; the same in every wave)
    auto cut = [](int n) { return n > 1 ? n : 0; };
    auto least_of = [&](int total) { return (int)((float)total * ((float)a.n_tiles * 1.0001f) / (float)a.places) + 1; };  // fills the places once
    const int slots = a.slots;
    int off = 0, total = 0, sum;
    bool found = false;
    if (a.U <= kMostUnits) {  // every wave by itself
      constexpr int N = kMostUnits / 64;
      int c[N], longest = 0;
#pragma unroll
      for (int i = 0; i < N; ++i) c[i] = 64 * i + lane < a.U ? cost_of(len_of(64 * i + lane)) : 0;
#pragma unroll
      for (int i = 0; i < N; ++i)
        if (64 * i < a.U) {
          ag_wave_prefix(c[i], sum);
          total += sum;
          longest = max(longest, c[i]);
        }
      int lo = max(a.least, least_of(total));
      if (a.U <= slots) {
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) longest = max(longest, __shfl_xor(longest, o, 64));
        int hi = max(lo, slots > a.U ? min(longest, (int)((float)total / (float)(slots - a.U) * 1.0001f) + 2) : longest);  // (at most total / lo + U pieces)
        while (lo < hi) {
          const int mid = (lo + hi) / 2;
          int n = 0;
#pragma unroll
          for (int i = 0; i < N; ++i)
            if (64 * i < a.U) n += n_of(c[i], 1.f / (float)mid);
          ag_wave_prefix(n, sum);
          if (sum <= slots) hi = mid;
          else lo = mid + 1;
        }
      }
      const float inv = 1.f / (float)lo;
      int before = 0, recs = 0;
#pragma unroll
      for (int i = 0; i < N; ++i)
        if (64 * i < a.U) {
          const int n = n_of(c[i], inv), pre = before + ag_wave_prefix(n * a.n_tiles, sum);
          const uint64_t hit = __ballot(pre <= wg && wg < pre + n * a.n_tiles);
          before += sum;
          const int rec = recs + ag_wave_prefix(cut(n) * a.n_tiles, sum);
          recs += sum;
          if (hit) {
            const int x = __builtin_ctzll(hit);
            found = true;
            u = 64 * i + x;
            pieces = __builtin_amdgcn_readlane(n, x);
            off = wg - __builtin_amdgcn_readlane(pre, x);
            rec0 = __builtin_amdgcn_readlane(rec, x);
          }
        }
    } else {  // more units than places
      const int per = (a.U + kThreads - 1) / kThreads, u0 = min(a.U, tid * per), u1 = min(a.U, u0 + per);
      int mine = 0, recs = 0;
      for (int v = u0; v < u1; ++v) mine += cost_of(len_of(v));
      ag_wave_prefix(mine, sum);
      if (lane == 0) s_sum[wave][0] = sum;
      __syncthreads();
#pragma unroll
      for (int w = 0; w < kWaves; ++w) total += s_sum[w][0];
      const float inv = 1.f / (float)max(a.least, least_of(total));
      mine = 0;
      for (int v = u0; v < u1; ++v) {
        const int n = n_of(cost_of(len_of(v)), inv) * a.n_tiles;
        mine += n;
        recs += n > a.n_tiles ? n : 0;
      }
      int before = ag_wave_prefix(mine, sum);
      if (lane == 0) s_sum[wave][1] = sum;
      int rec = ag_wave_prefix(recs, sum);
      if (lane == 0) s_sum[wave][2] = sum;
      if (tid == 0) s_start[0] = -1;
      __syncthreads();
#pragma unroll
      for (int w = 0; w < kWaves; ++w)
        if (w < wave) {
          before += s_sum[w][1];
          rec += s_sum[w][2];
        }
      if (before <= wg && wg < before + mine) {  // one thread, or none
        for (int v = u0; v < u1; ++v) {
          const int n = n_of(cost_of(len_of(v)), inv);
          if (wg < before + n * a.n_tiles) {
            s_start[0] = v;
            s_start[1] = n;
            s_start[2] = wg - before;
            s_start[3] = rec;
            break;
          }
          before += n * a.n_tiles;
          rec += cut(n) * a.n_tiles;
        }
      }
      __syncthreads();
      u = s_start[0];
      found = u >= 0;
      pieces = s_start[1];
      off = s_start[2];
      rec0 = s_start[3];
    }
    if (!found) return;
    u = __builtin_amdgcn_readfirstlane(u);
    pieces = __builtin_amdgcn_readfirstlane(pieces);
    off = __builtin_amdgcn_readfirstlane(off);
    const quotient of = divide(off, pieces);
    piece = __builtin_amdgcn_readfirstlane(of.r);
    tile = __builtin_amdgcn_readfirstlane(of.q);
    rec0 = __builtin_amdgcn_readfirstlane(rec0) + tile * pieces;
  }

  {
    int tid = threadIdx.x;
    asm volatile("" : "+v"(tid));  // (unknown to the compiler: it would keep every address below in registers all the way)
    const int lane = tid & 63, col = lane & 31, h = lane >> 5;
    const int len = __builtin_amdgcn_readfirstlane(len_of(u)), nb = len / kQ8Block, held = len & (kQ8Block - 1), cost = cost_of(len);
    const int per = (cost + pieces - 1) / pieces, sub = min(piece * per, cost), take = min(per, cost - sub);  // of the tile's cost
    const bool local = sub == 0;
    const int p0 = max(0, sub - kUnitCost), p1 = max(0, sub + take - kUnitCost);  // pages
    const quotient of_u = divide(u, a.Hkv);
    const int b = __builtin_amdgcn_readfirstlane(of_u.q), head = __builtin_amdgcn_readfirstlane(of_u.r), row0 = tile * 32 * RW;
    const bool active = row0 + rg * 32 < rows;  // this wave has rows
    const int32_t *page = a.c.page + (size_t)u * a.c.max_blocks;
    auto q_of = [&](int row) { return (((size_t)b * a.Hq + (size_t)head * G + (row & (G - 1))) * a.L + (row >> a.g_log)) * D; };
    // local rows: the tail's, then the nodes up to the tile's last one; 64 of them a tile
    const int n_nodes = local ? min(((row0 + 32 * RW - 1) >> a.g_log) + 1, a.L) : 0;
    const int n_local = local ? held + n_nodes : 0, n_lt = (n_local + kQ8Block - 1) / kQ8Block;
    const uint16_t *kt = a.c.k_tail + (size_t)u * kQ8Block * D, *vt = a.c.v_tail + (size_t)u * kQ8Block * D;
    const uint16_t *K = a.k + (size_t)u * a.L * D, *V = a.v + (size_t)u * a.L * D;

    // ---- a wave's pages: lane x holds the number and the exponents of its page x, of at most 64 at a time ----
    int ids = -1, ek_v = 0, ev_v = 0;
    const int i0 = p0 + kg;
    auto numbers = [&](int first) {
      const int i = first + lane * KW;
      ids = i < p1 ? page[i] : -1;
    };
    auto exponents = [&] {
      const bool ok = (uint32_t)ids < (uint32_t)a.c.n_pages;  // (a number outside the pool: rows that are not there)
      const int id = ok ? ids : 0;
      ek_v = (int)(__float_as_uint(a.c.k_scale[id]) >> 23) - 127;
      ev_v = (int)(__float_as_uint(a.c.v_scale[id]) >> 23) - 127 - kPageBits;
      ids = ok ? ids : -1;
    };
    if (active && i0 < p1) numbers(i0);

    // ---- the queries and the first local tile: everything that has to be loaded is asked for at once ----
    constexpr int QN = (RW * 32 * VR + kThreads - 1) / kThreads, LN = 2 * kQ8Block * VR / kThreads;  // vectors that a thread has a piece of
    struct piece_of {  // values d .. d + 7 and d + D / 2 .. + 7 of a vector
      uint4 lo, hi;
    };
    auto angles_of = [&](q8_f32x4 (&an)[4], const place &x, int d) {
      const q8_rows r = rows_of(a.rope, x, a.err);
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const q8_angles y = q8_angles4(a.rope, r, d + 4 * i, D);
        an[2 * i] = q8_f32x4{y.c.x, y.c.y, y.c.z, y.c.w};
        an[2 * i + 1] = q8_f32x4{y.s.x, y.s.y, y.s.z, y.s.w};
      }
    };
    auto row_of_item = [](int me, int i) { return (me + i * kThreads) / VR; };
    struct local_rows {
      piece_of k[LN], v[LN];
      place p[LN];
    };
    auto ask_local = [&](local_rows &w, int lt, int me) {  // rows of local tiles lt and lt + 1
      const int d = me % VR * 8;
#pragma unroll
      for (int i = 0; i < LN; ++i) {
        const int x = lt * kQ8Block + row_of_item(me, i), node = min(max(x - held, 0), a.L - 1);
        w.p[i] = a.rope.table ? place_of(a.rope, (int64_t)b * a.L + node) : place{};
        const uint16_t *p = K + (size_t)node * D + d, *v = V + (size_t)node * D + d;
        const bool old = x < held;
        w.k[i].lo = *reinterpret_cast<const uint4 *>(old ? kt + q8_k_at<D>(x, d / 64, d / 16 % 4) * 16 + (d & 8) : p);
        w.k[i].hi = *reinterpret_cast<const uint4 *>(old ? kt + q8_k_at<D>(x, (d + D / 2) / 64, (d + D / 2) / 16 % 4) * 16 + (d & 8) : p + D / 2);
        if (!old) {
          w.v[i].lo = *reinterpret_cast<const uint4 *>(v);
          w.v[i].hi = *reinterpret_cast<const uint4 *>(v + D / 2);
        } else {  // (its columns' values lie apart: column 16 f + r, row 16 i + 4 g + j at ((4 f + g) 16 + r) 16 + 4 i + j)
          const uint16_t *from = vt + (d >> 4) * 1024 + (d & 8) * 16 + (x >> 2 & 3) * 256 + (x >> 4) * 4 + (x & 3), *second = from + D / 32 * 1024;
          uint32_t y[8];
#pragma unroll
          for (int z = 0; z < 4; ++z) {
            y[z] = from[32 * z] | (uint32_t)from[32 * z + 16] << 16;
            y[4 + z] = second[32 * z] | (uint32_t)second[32 * z + 16] << 16;
          }
          w.v[i].lo = make_uint4(y[0], y[1], y[2], y[3]);
          w.v[i].hi = make_uint4(y[4], y[5], y[6], y[7]);
        }
      }
    };
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
    auto turned = [&](q8_eight (&y)[2], const piece_of &x, const q8_f32x4 (&an)[4]) {
      y[0] = q8_turn8(an, true, x.lo, x.hi);
      y[1] = q8_turn8(an, false, x.hi, x.lo);
    };
    auto over_row = [&](float top) {
#pragma unroll
      for (int o = 1; o < VR; o <<= 1) top = fmaxf(top, __shfl_xor(top, o, 64));
      return top;
    };
    auto local_keys = [&](q8_eight (&y)[LN][2], const local_rows &w, const q8_f32x4 (&an)[LN][4], int lt, int me) {  // turned, the nodes'
#pragma unroll
      for (int i = 0; i < LN; ++i) {
        q8_eight z[2];
        turned(z, w.k[i], an[i]);
        const bool old = lt * kQ8Block + row_of_item(me, i) < held;
        const q8_eight x[2] = {q8_floats(w.k[i].lo), q8_floats(w.k[i].hi)};
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          y[i][e].a = old ? x[e].a : z[e].a;
          y[i][e].b = old ? x[e].b : z[e].b;
        }
      }
    };
    auto put_local = [&](q8_eight (&keys)[LN][2], local_rows &rows_in, int lt, int me) {  // what ask_local has asked for, into LDS
      const int d = me % VR * 8;
#pragma unroll
      for (int i = 0; i < LN; ++i) {
        const int r = row_of_item(me, i), x = lt * kQ8Block + r;  // (r < 128)
        const bool there = x < n_local;
        const q8_eight (&y)[2] = keys[i];
        float top = fmaxf(y[0].top(), y[1].top());
        bool odd = !(top < INFINITY);
#pragma unroll
        for (int e = 0; e < 2; ++e)  // (NaN is passed over by maxima)
#pragma unroll
          for (int z = 0; z < 4; ++z) odd |= y[e].a[z] != y[e].a[z] || y[e].b[z] != y[e].b[z];
        top = over_row(odd ? 0.f : top);
        const int ek = row_exponent(top);
        const float inv = odd ? 0.f : q8_pow2(-ek);
        odd |= finite8(rows_in.v[i].lo);
        odd |= finite8(rows_in.v[i].hi);
        if (there) {
          *reinterpret_cast<q8_f16x8 *>(s_k + frag_at<D>(r, d) * 8) = y[0].f16(inv);
          *reinterpret_cast<q8_f16x8 *>(s_k + frag_at<D>(r, d + D / 2) * 8) = y[1].f16(inv);
          if (d == 0) s_ek[r] = ek;
          if (odd) atomicOr(reinterpret_cast<unsigned long long *>(&s_odd[r >> 6]), 1ull << (r & 63));
        }
        // values row by row (rows that are not there: zeros), where the transposing reads find them
        const uint32_t keep = there ? ~0u : 0u;
        const uint4 lo = rows_in.v[i].lo, hi = rows_in.v[i].hi;
        *reinterpret_cast<uint4 *>(s_v + value_at<D>(r, d / 8)) = make_uint4(lo.x & keep, lo.y & keep, lo.z & keep, lo.w & keep);
        *reinterpret_cast<uint4 *>(s_v + value_at<D>(r, (d + D / 2) / 8)) = make_uint4(hi.x & keep, hi.y & keep, hi.z & keep, hi.w & keep);
      }
    };
    {
      const int d = tid % VR * 8;
      piece_of xq[QN];
      place pq[QN];
      local_rows first_rows = {};
      int up = -1;
      bool keep = false;
#pragma unroll
      for (int i = 0; i < QN; ++i) {
        const int row = min(row0 + row_of_item(tid, i), rows - 1);
        pq[i] = a.rope.table ? place_of(a.rope, (int64_t)b * a.L + (row >> a.g_log)) : place{};
        const uint16_t *x = a.q + q_of(row) + d;
        xq[i].lo = *reinterpret_cast<const uint4 *>(x);
        xq[i].hi = *reinterpret_cast<const uint4 *>(x + D / 2);
      }
      if (local) {
        if (tid < n_nodes) {
          up = a.parent[(size_t)b * a.L + tid];
          keep = !a.flags || a.flags[(size_t)u * a.L + tid] != 0;
        }
        ask_local(first_rows, 0, tid);
      }
      if (active && i0 < p1) exponents();
      if (local) {
        if (up >= tid) {
          atomicOr(a.err, 4);
          up = -1;
        }
        const uint64_t kept = __ballot(keep);
        if (tid < kQ8TreeMost) {
          up = max(-1, up);
          s_up[tid] = up;
#pragma unroll
          for (int w = 0; w < kWords; ++w) s_above[tid][w] = tid >> 6 == w ? 1ull << (tid & 63) : 0;
          if (lane == 0) s_keep[wave] = kept;
        }
        if (tid < 2) s_odd[tid] = 0;
      }
      q8_eight yq[QN][2], yk[LN][2];
      if (a.rope.table) {
        q8_f32x4 an[QN][4], ak[LN][4];
#pragma unroll
        for (int i = 0; i < QN; ++i) angles_of(an[i], pq[i], d);
#pragma unroll
        for (int i = 0; i < LN; ++i) angles_of(ak[i], first_rows.p[i], d);  // (without local rows: the table's first)
#pragma unroll
        for (int i = 0; i < QN; ++i) turned(yq[i], xq[i], an[i]);
        local_keys(yk, first_rows, ak, 0, tid);
      } else {
#pragma unroll
        for (int i = 0; i < LN; ++i) {
          yk[i][0] = q8_floats(first_rows.k[i].lo);
          yk[i][1] = q8_floats(first_rows.k[i].hi);
        }
#pragma unroll
        for (int i = 0; i < QN; ++i) {
          yq[i][0] = q8_floats(xq[i].lo);
          yq[i][1] = q8_floats(xq[i].hi);
        }
      }
#pragma unroll
      for (int i = 0; i < QN; ++i) {
        const int r = row_of_item(tid, i);
        const q8_eight (&y)[2] = yq[i];
        const int eq = row_exponent(over_row(fmaxf(y[0].top(), y[1].top())));  // (NaN is passed over)
        const float inv = q8_pow2(-eq);
        if (QN * kThreads == RW * 32 * VR || r < RW * 32) {
          *reinterpret_cast<q8_f16x8 *>(s_q + frag_at<D>(r, d) * 8) = y[0].f16(inv);
          *reinterpret_cast<q8_f16x8 *>(s_q + frag_at<D>(r, d + D / 2) * 8) = y[1].f16(inv);
          if (d == 0) s_eq[r] = eq;
        }
      }
      if (local) {
        barrier();  // (s_odd)
        put_local(yk, first_rows, 0, tid);
        // Node t knows the n nodes from itself up, and the next one: with each step twice as many.
        if (n_nodes <= 64) {  // one wave, in registers
          if (wave == 0) {
            uint64_t mask = 1ull << lane;
            int to = up;
            for (int n = 1; n < n_nodes; n *= 2) {
              const int at = max(to, 0), lo = __shfl((int)(uint32_t)mask, at, 64), hi = __shfl((int)(uint32_t)(mask >> 32), at, 64), next = __shfl(to, at, 64);
              if (to >= 0) {
                mask |= (uint64_t)(uint32_t)hi << 32 | (uint32_t)lo;
                to = next;
              }
            }
            s_above[lane][0] = mask;
          }
        } else {
          for (int n = 1; n < n_nodes; n *= 2) {
            uint64_t more[kWords] = {};
            int to = -1, next = -1;
            if (tid < n_nodes) {
              to = s_up[tid];
              if (to >= 0) {
#pragma unroll
                for (int w = 0; w < kWords; ++w) more[w] = s_above[to][w];
                next = s_up[to];
              }
            }
            barrier();
            if (to >= 0) {
#pragma unroll
              for (int w = 0; w < kWords; ++w) s_above[tid][w] |= more[w];
              s_up[tid] = next;
            }
            barrier();
          }
        }
      }
      barrier();
    }

    // ---- the pages ----
    q8_f16x8 qx[KS];
    q8_f32x16 o[DT];
    float m = kQ8EmptyMax, l = 0.f;
#pragma unroll
    for (int i = 0; i < KS; ++i) qx[i] = *reinterpret_cast<const q8_f16x8 *>(s_q + fragment<D>(rg, i, h, col) * 8);
    const int eq = s_eq[rg * 32 + col];
#pragma unroll
    for (int dt = 0; dt < DT; ++dt)
#pragma unroll
      for (int i = 0; i < 16; ++i) o[dt][i] = 0.f;
    if (active && i0 < p1) {
      bool fresh = true;
      int ev_top = kQ8PageMinExp;  // the largest ev so far
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
        // (pages outside the pool are left out)
        int n = min(64, (p1 - first_page + KW - 1) / KW);
        const uint64_t there = __ballot(ids >= 0);
        if (__popcll(there) != n) {
          n = __popcll(there);
          const int to = ids >= 0 ? __popcll(there & ((1ull << lane) - 1)) : 63;  // (of 64 lanes one is free)
          ids = __builtin_amdgcn_ds_permute(4 * to, ids);
          ek_v = __builtin_amdgcn_ds_permute(4 * to, ek_v);
          ev_v = __builtin_amdgcn_ds_permute(4 * to, ev_v);
        }
        if (n > 0) {
          load_k(0);
          load_v(0);
        }
        for (int x = 0; x < n; ++x) {
          const bool more = x + 1 < n;
          // s[i]: row 32 y + 8 (i / 4) + 4 h + i % 4 of the page.  The state is kept relative to m, the largest score plus its page's
          // exponent ev of V less kQ8TopBits: weights are 2^(score + ev - m) in f16, values v 2^-ev, the page's part of the row sum 2^-ev the sum
          // of its weights as the product takes them (`apart`: the sum of 2^(score - m)).
          const int e = __builtin_amdgcn_readlane(ev_v, x), ev = max(kQ8PageMinExp, e);
          ev_top = max(ev_top, ev);
          const bool apart = ev <= ev_top - kQ8Span;
          const float f = q8_unscale(a.qscale, eq + __builtin_amdgcn_readlane(ek_v, x)), scale = q8_pow2(e + kPageBits - ev);
          q8_f32x16 s[2];
          uint32_t p[2][8];
          float sum = 0.f;
          auto scores = [&](int y) {
#pragma unroll
            for (int i = 0; i < 16; ++i) s[y][i] = 0.f;
#pragma unroll
            for (int c = 0; c < KC; ++c)
#pragma unroll
              for (int j = 0; j < 2; ++j)
#pragma unroll
                for (int z = 0; z < 2; ++z)
                  s[y] = __builtin_amdgcn_mfma_f32_32x32x16_f16(q8_widen16(bk[y][c][j][2 * z], bk[y][c][j][2 * z + 1], 1.f), qx[c * 4 + j * 2 + z], s[y], 0, 0, 0);
          };
          auto weigh = [&](int y) {
            const float shift = (float)ev - m;
            float part[2] = {0.f, 0.f};
#pragma unroll
            for (int i = 0; i < 16; i += 2) {
              const q8_f32x2 w = {__builtin_amdgcn_exp2f(fmaf(s[y][i], f, shift)), __builtin_amdgcn_exp2f(fmaf(s[y][i + 1], f, shift))};
              p[y][i / 2] = __builtin_bit_cast(uint32_t, __builtin_convertvector(w, q8_f16x2));
              part[i / 2 & 1] = q8_add2(p[y][i / 2], part[i / 2 & 1]);
            }
            sum = part[0] + part[1];
          };
          auto raise = [&](int y, bool always) {  // a new reference for the rows whose weights pass 2^15 (a row's own alone), or for all
            float mx = -INFINITY;
#pragma unroll
            for (int i = 0; i < 16; ++i) mx = fmaxf(mx, s[y][i]);
            mx = fmaf(fmaxf(mx, other_half(mx)), f, (float)(ev - kQ8TopBits));
            const float over = sum <= 32768.f ? 0.f : 1.f;
            const float m_new = always || fmaxf(over, other_half(over)) > 0.f ? fmaxf(m, mx) : m;
            const float alpha = __builtin_amdgcn_exp2f(0.5f * (m - m_new));
            l = shrink(l, alpha);
#pragma unroll
            for (int dt = 0; dt < DT; ++dt) o[dt] = o[dt] * alpha * alpha;
            m = m_new;
          };
          auto sum_apart = [&](int y) {
#pragma unroll
            for (int i = 0; i < 16; ++i) l += __builtin_amdgcn_exp2f(fmaf(s[y][i], f, -m));
            sum = 0.f;
          };
          auto values = [&](int y) {
#pragma unroll
            for (int i = 2 * y; i < 2 * y + 2; ++i) {
              const q8_f16x8 pb = __builtin_bit_cast(q8_f16x8, make_uint4(p[y][4 * (i & 1)], p[y][4 * (i & 1) + 1], p[y][4 * (i & 1) + 2], p[y][4 * (i & 1) + 3]));
#pragma unroll
              for (int dt = 0; dt < DT; ++dt)
                o[dt] = __builtin_amdgcn_mfma_f32_32x32x16_f16(q8_widen16(bv[dt][0][i], bv[dt][1][i], scale), pb, o[dt], 0, 0, 0);
            }
          };
          scores(0);
          if (fresh) raise(0, true);
          fresh = false;
          // While the matrix unit has one half's scores (values), the vector unit forms the other half's weights.
          scores(1);
          weigh(0);
          if (more) load_k(x + 1);
          if (apart || __any(!(sum <= 32768.f))) {
            raise(0, false);
            weigh(0);
            if (apart) sum_apart(0);
          }
          l += ldexpf(sum, -ev);
          values(0);
          weigh(1);
          if (apart || __any(!(sum <= 32768.f))) {
            raise(1, false);
            weigh(1);
            if (apart) sum_apart(1);
          }
          l += ldexpf(sum, -ev);
          values(1);
          if (more) load_v(x + 1);
        }
        first_page += 64 * KW;
        if (first_page >= p1) break;
        numbers(first_page);
        exponents();
      }
    }

    // ---- the local rows ----
    if (local) {
      int tid = threadIdx.x;
      asm volatile("" : "+v"(tid));  // (as above)
      const int lane = tid & 63, col = lane & 31, h = lane >> 5, t = min((row0 + rg * 32 + col) >> a.g_log, a.L - 1), eq = s_eq[rg * 32 + col];
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
      for (int half = 0; half < 2 * n_lt; ++half) {  // 32 rows at a time: the group's waves take turns
        if (half > 0 && half % 4 == 0) {
          int me = threadIdx.x;
          asm volatile("" : "+v"(me));  // (as above)
          local_rows next_rows;
          ask_local(next_rows, half / 2, me);
          q8_eight y[LN][2];
          if (a.rope.table) {
            q8_f32x4 an[LN][4];
#pragma unroll
            for (int i = 0; i < LN; ++i) angles_of(an[i], next_rows.p[i], me % VR * 8);
            local_keys(y, next_rows, an, half / 2, me);
          } else {
#pragma unroll
            for (int i = 0; i < LN; ++i) {
              y[i][0] = q8_floats(next_rows.k[i].lo);
              y[i][1] = q8_floats(next_rows.k[i].hi);
            }
          }
          barrier();  // (the tiles before have been read)
          if (tid < 2) s_odd[tid] = 0;
          barrier();
          put_local(y, next_rows, half / 2, me);
          barrier();
        }
        const int lt = half / 2, which = lt & 1, x = half & 1;
        const int own = held + t - lt * kQ8Block;  // the tile's row that is this lane's own node
        const uint64_t all = seen(lt), odd = s_odd[which], bits = all & ~odd;
        const uint32_t half_bits = (uint32_t)(bits >> (32 * x));
        if (active && (KW == 2 ? kg == 0 : half % KW == kg) && __any(half_bits != 0)) {
          const uint16_t *kf = s_k + which * S::kTile + x * KS * 512, *vf = s_v + which * S::kTile + x * 32 * D;
          q8_f32x16 s;
#pragma unroll
          for (int i = 0; i < 16; ++i) s[i] = 0.f;
#pragma unroll
          for (int k = 0; k < KS; ++k)
            s = __builtin_amdgcn_mfma_f32_32x32x16_f16(*reinterpret_cast<const q8_f16x8 *>(kf + fragment<D>(0, k, h, col) * 8),
                                                       *reinterpret_cast<const q8_f16x8 *>(s_q + fragment<D>(rg, k, h, col) * 8), s, 0, 0, 0);
          float mx = -INFINITY;
          const uint32_t w = half_bits >> (4 * h);
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            const int r = 8 * (i / 4) + i % 4;
            s[i] *= q8_unscale(a.qscale, eq + s_ek[64 * which + 32 * x + 4 * h + r]);
            // its own node: alone its weight is 1 whatever its score is; a score that overflowed to -infinity counts as the least number
            if (32 * x + r + 4 * h == own) s[i] = sole ? 0.f : (s[i] < kQ8EmptyMax ? kQ8EmptyMax : s[i]);
            if (!(w >> r & 1)) s[i] = -INFINITY;
            mx = fmaxf(mx, s[i]);
          }
          // (the weights are bf16: the reference lies above the largest, so that rows of the largest values do not add up to infinity)
          const float m_new = fmaxf(m, fmaxf(mx, other_half(mx)) + above), alpha = __builtin_amdgcn_exp2f(0.5f * (m - m_new));
          l = shrink(l, alpha);
#pragma unroll
          for (int dt = 0; dt < DT; ++dt) o[dt] = o[dt] * alpha * alpha;
          m = m_new;
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            uint32_t hi[4], lo[4];
#pragma unroll
            for (int z = 0; z < 4; ++z) {
              const float w0 = __builtin_amdgcn_exp2f(s[8 * i + 2 * z] - m), w1 = __builtin_amdgcn_exp2f(s[8 * i + 2 * z + 1] - m);
              l += w0 + w1;
              hi[z] = q8_pack2(w0, w1);
              lo[z] = q8_pack2(w0 - q8_lo(hi[z]), w1 - q8_hi(hi[z]));
            }
            const q8_bf16x8 ph = __builtin_bit_cast(q8_bf16x8, make_uint4(hi[0], hi[1], hi[2], hi[3])), pl = __builtin_bit_cast(q8_bf16x8, make_uint4(lo[0], lo[1], lo[2], lo[3]));
#pragma unroll
            for (int dt = 0; dt < DT; ++dt) {
              // rows 16 i + 4 h + 0..3 and 8 further of this lane's column: lane x of 16 gives the address of row x / 4, columns 4 (x % 4) ...
              const int r = 4 * h + (lane >> 2 & 3), c = 4 * dt + (lane >> 4 & 1) * 2 + (lane >> 1 & 1);
              auto read = [&](int row) {
                return __builtin_amdgcn_ds_read_tr16_b64_v4bf16((__attribute__((address_space(3))) bf16x4 *)(vf + 16 * i * D + value_at<D>(row, c) + (lane & 1) * 4));
              };
              const q8_bf16x8 v = __builtin_shufflevector(read(r), read(r + 8), 0, 1, 2, 3, 4, 5, 6, 7);
              o[dt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(v, pl, o[dt], 0, 0, 0);
              o[dt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(v, ph, o[dt], 0, 0, 0);
            }
          }
        }
        if (!active || kg != 0 || x != 1) continue;
        for (uint64_t left_over = odd; left_over; left_over &= left_over - 1) {  // rare: rows with infinities or NaN, one by one in 32 bits
          const int r = __builtin_ctzll(left_over), x = lt * kQ8Block + r;
          const bool mine = all >> r & 1;
          if (!__any(mine)) continue;
          float s = 0.f;
          for (int k = 0; k < KS; ++k) {
            const int c = step_col(k, h);
            q8_eight z;
            if (x < held) {
              z = q8_floats(*reinterpret_cast<const uint4 *>(kt + q8_k_at<D>(x, c / 64, c / 16 % 4) * 16 + (c & 8)));
            } else {
              const uint16_t *p = K + (size_t)(x - held) * D;
              const uint4 y = *reinterpret_cast<const uint4 *>(p + c), other = *reinterpret_cast<const uint4 *>(p + (c ^ (D / 2)));
              z = q8_floats(y);
              if (a.rope.table) {
                const q8_rows turn = rows_of(a.rope, place_of(a.rope, (int64_t)b * a.L + x - held), a.err);
                auto angles = [&](int i) { return q8_angles4(a.rope, turn, i, D); };
                z = q8_turn8<D>(angles, c, y, other);
              }
            }
            const q8_f16x8 q = *reinterpret_cast<const q8_f16x8 *>(s_q + fragment<D>(rg, k, h, col) * 8);
#pragma unroll
            for (int i = 0; i < 4; ++i) s = fmaf((float)q[i], z.a[i], fmaf((float)q[4 + i], z.b[i], s));
          }
          s = (s + other_half(s)) * q8_unscale(a.qscale, eq);
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
              const int c = 32 * dt + 8 * (i / 4) + 4 * h + i % 4;
              const uint16_t val = x < held ? vt[((c >> 4) * 4 + (x >> 2 & 3)) * 256 + (c & 15) * 16 + (x >> 4) * 4 + (x & 3)] : V[(size_t)(x - held) * D + c];
              o[dt][i] = shrink(o[dt][i], alpha) + w * __uint_as_float((uint32_t)val << 16);
            }
          }
        }
      }
    }

    // ---- the states of the workgroup's waves, then those of the tile's pieces, are added up: a group's waves share the columns ----
    // (sixteen bytes a lane; records are written through and read past the caches, sc0 and sc1)
    constexpr int kThrough = 17, NP = DT * 4 / KW;  // NP: a wave's share of a state's DT * 4 parts
    int me = threadIdx.x & 63;
    asm volatile("" : "+v"(me));  // (as above)
    barrier();
    {
      uint8_t *to = smem + (kg * RW + rg) * S::kState;
#pragma unroll
      for (int i = 0; i < DT * 4; ++i)
        *reinterpret_cast<q8_f32x4 *>(to + i * 1024 + me * 16) = q8_f32x4{o[i / 4][4 * (i % 4)], o[i / 4][4 * (i % 4) + 1], o[i / 4][4 * (i % 4) + 2], o[i / 4][4 * (i % 4) + 3]};
      *reinterpret_cast<q8_f32x2 *>(to + DT * 4 * 1024 + me * 8) = q8_f32x2{m, l};
    }
    barrier();
    q8_f32x4 acc[NP] = {};
    float top = kQ8EmptyMax, sum = 0.f;
    const int part0 = kg * NP;
    // n states of which z has maximum and sum ml[z] and part j x[z][j]
    auto add = [&](auto &ml, auto &x, int n) {
      float M = top;
#pragma unroll
      for (int z = 0; z < (int)(sizeof(ml) / sizeof(ml[0])); ++z) M = fmaxf(M, z < n ? ml[z][0] : kQ8EmptyMax);
      const float keep = __builtin_amdgcn_exp2f(0.5f * (top - M));
      top = M;
      sum = shrink(sum, keep);
#pragma unroll
      for (int j = 0; j < NP; ++j) acc[j] = acc[j] * keep * keep;
#pragma unroll
      for (int z = 0; z < (int)(sizeof(ml) / sizeof(ml[0])); ++z) {
        if (z >= n) break;
        const float f = __builtin_amdgcn_exp2f(0.5f * (ml[z][0] - M));
        sum += shrink(ml[z][1], f);
#pragma unroll
        for (int j = 0; j < NP; ++j) acc[j] += x[z][j] * f * f;
      }
    };
    {
      q8_f32x2 ml[KW];
      q8_f32x4 x[KW][NP];
#pragma unroll
      for (int z = 0; z < KW; ++z) {
        const uint8_t *from = smem + (z * RW + rg) * S::kState;
        ml[z] = *reinterpret_cast<const q8_f32x2 *>(from + DT * 4 * 1024 + me * 8);
#pragma unroll
        for (int j = 0; j < NP; ++j) x[z][j] = *reinterpret_cast<const q8_f32x4 *>(from + (part0 + j) * 1024 + me * 16);
      }
      add(ml, x, KW);
    }
    auto store = [&] {
      sum += other_half(sum);
      const int row = row0 + rg * 32 + (me & 31);
      if (row < rows) {
        const float inv = 1.f / sum;
        uint16_t *to = a.out + q_of(row) + 4 * (me >> 5) + 8 * part0;
#pragma unroll
        for (int j = 0; j < NP; ++j) *reinterpret_cast<uint2 *>(to + 8 * j) = make_uint2(q8_pack2(acc[j][0] * inv, acc[j][1] * inv), q8_pack2(acc[j][2] * inv, acc[j][3] * inv));
      }
    };
    if (pieces == 1) {
      store();
      return;
    }
    auto rec_at = [&](int k) {
      return __builtin_amdgcn_make_buffer_rsrc(a.rec + ((size_t)(rec0 + k) * RW + rg) * (S::kState / 4), 0, S::kState, 0x00020000);
    };
    {
      const __amdgpu_buffer_rsrc_t to = rec_at(piece);
#pragma unroll
      for (int j = 0; j < NP; ++j) __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(q8_u32x4, acc[j]), to, me * 16, (part0 + j) * 1024, kThrough);
      const q8_f32x2 ml = {top, sum};
      if (kg == 0) __builtin_amdgcn_raw_buffer_store_b64(__builtin_bit_cast(q8_u32x2, ml), to, me * 8, DT * 4 * 1024, kThrough);
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");  // this wave's part of the record is in memory
    __syncthreads();
    if (tid == 0) s_last = __hip_atomic_fetch_add(&a.tickets[rec0], 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == pieces - 1;
    __syncthreads();
    if (!s_last) return;  // all pieces are there: they are added in order, four at a time
    if (tid == 0) a.tickets[rec0] = 0;
    top = kQ8EmptyMax;
    sum = 0.f;
#pragma unroll
    for (int j = 0; j < NP; ++j) acc[j] = q8_f32x4{0.f, 0.f, 0.f, 0.f};
    for (int k = 0; k < pieces; k += 4) {
      q8_f32x2 ml[4];
      q8_f32x4 x[4][NP];
#pragma unroll
      for (int z = 0; z < 4; ++z) {
        const __amdgpu_buffer_rsrc_t from = rec_at(min(k + z, pieces - 1));
        ml[z] = __builtin_bit_cast(q8_f32x2, __builtin_amdgcn_raw_buffer_load_b64(from, me * 8, DT * 4 * 1024, kThrough));
#pragma unroll
        for (int j = 0; j < NP; ++j) x[z][j] = __builtin_bit_cast(q8_f32x4, __builtin_amdgcn_raw_buffer_load_b128(from, me * 16, (part0 + j) * 1024, kThrough));
      }
      add(ml, x, pieces - k);
    }
    store();
  }
}

int tiles_of(int rows, int groups) { return (rows + 32 * groups - 1) / (32 * groups); }
// Groups of 32 rows that a workgroup takes.  More of them share what they load of the pages, fewer have more waves for each group's pages and local
// rows, and less to add up.  So as few as leave a tile for every CU at most, while there are few pages to go through: up to 16 a CU one group (4 x 31
// nodes over 1500 rows, G = 4, 8 heads: 20.3 us with one, 20.8 with two, 24 with four; over 3000 29 / 26 / 28), up to 96 two (over 9000 57 / 39 / 43; 4 x 64
// nodes over 13000 54 with two, 51 with four).  With more tiles than CUs the rest would wait: 32 x 16 nodes over 100 rows 29 / 16.
// The lengths are on the device, so the pages are those that the table has columns for.  A table made for much longer units costs what four groups
// cost short ones: with 500 columns more 4 x 31 nodes over 1500 rows 24 us in place of 19, 64 over 777 22 in place of 17, 12 over 777 17 in place of 15.
int row_groups(int num_cu, int units, int rows, int max_blocks) {
  const int n = tiles_of(rows, 1);
  const int64_t pages = (int64_t)units * n * max_blocks;
  if (n == 1 || ((int64_t)units * n <= num_cu && pages <= 16 * num_cu)) return 1;
  if (n == 2 || ((int64_t)units * tiles_of(rows, 2) <= num_cu && pages <= 96 * num_cu)) return 2;
  return 4;
}

template <int D, int RW>
hipError_t launch(ag_ctx *ctx, hipStream_t s, tree_args &a) {
  static std::atomic<bool> allowed[64];
  const hipError_t e = ag_q8_allow_lds(ctx->device, allowed, &ag_q8_tree_kernel<D, RW>, sizes<D>::lds(RW));
  if (e != hipSuccess) return e;
  a.n_tiles = tiles_of(a.L << a.g_log, RW);
  a.least = 2 * (kWaves / RW) + kUnitCost;
  a.places = ctx->num_cu;
  a.slots = a.places / a.n_tiles;
  const int64_t tiles = (int64_t)a.U * a.n_tiles, most = tiles * ((a.c.max_blocks + kUnitCost + a.least - 1) / a.least);
  const int grid = (int)std::min<int64_t>(tiles <= a.places ? a.places : tiles + a.places, most);
  AG_LAUNCH(ag_time_kernel(ctx, AG_K_Q8_TREE), (ag_q8_tree_kernel<D, RW>), dim3(grid), dim3(kThreads), sizes<D>::lds(RW), s, a);
  return hipGetLastError();
}
template <int D>
hipError_t launch_rows(ag_ctx *ctx, hipStream_t s, tree_args &a) {
  switch (row_groups(ctx->num_cu, a.U, a.L << a.g_log, a.c.max_blocks)) {
    case 1: return launch<D, 1>(ctx, s, a);
    case 2: return launch<D, 2>(ctx, s, a);
    default: return launch<D, 4>(ctx, s, a);
  }
}

}  // namespace

// (with what rounding up adds)
int64_t ag_q8_tree_cost(int64_t units, int rows, int max_blocks) {
  static_assert(kUnitCost <= 16, "the bound is part of the interface");
  return units * ((int64_t)max_blocks + 16) * tiles_of(rows, 1) + (1 << 16);
}

// Two records a workgroup, of as many groups of rows as it may have.
size_t ag_ws_q8_tree_floats(int num_cu, int rows, int D) {
  return (size_t)2 * num_cu * (rows <= 32 ? 1 : rows <= 64 ? 2 : 4) * (D / 32 * 4 * 1024 + 512) / 4;
}

hipError_t ag_launch_q8_tree(ag_ctx *ctx, hipStream_t s, const void *q, const void *k, const void *v, const uint8_t *flags, const int32_t *parent,
                             int B, int Hq, int Hkv, int L, int D, const ag_rope_dev &rope, float scale, const ag_q8_dev &cache, void *out, float *rec) {
  tree_args a;
  a.q = (const uint16_t *)q; a.k = (const uint16_t *)k; a.v = (const uint16_t *)v; a.flags = flags; a.parent = parent; a.out = (uint16_t *)out;
  a.c = cache; a.rope = rope; a.rec = rec; a.tickets = ctx->decode_tickets; a.err = ctx->d_err;
  a.U = B * Hkv; a.Hq = Hq; a.Hkv = Hkv; a.L = L;
  a.g_log = 0;
  while (Hkv << a.g_log < Hq) ++a.g_log;
  a.n_tiles = a.least = a.places = a.slots = 0;
  a.qscale = scale * kLog2e;
  return D == 128 ? launch_rows<128>(ctx, s, a) : launch_rows<64>(ctx, s, a);
}
