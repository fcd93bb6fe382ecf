// Filling the paged 8-bit cache: a call's kept tokens join their units, keys turned on the way.
//
// A unit's new rows follow its tail; rows 64 j .. 64 j + 63 of (tail, new rows) are its block j of this call.  A workgroup takes every
// n-th block of a unit: it finds the block's tokens from the flags' prefix counts, reads their rows of k and v once (a row is 128 or 256
// bytes in one piece), turns k, takes the largest magnitude for the scale and writes the codes in page order; V is transposed
// through LDS.  The block that stays incomplete is written to the tail instead.  Bound by memory: the kept rows in bf16 in, in 8 bits out;
// 516000 kept rows of 128 in 103 us, 4.0 TB/s.
//   * 4 D threads, 16 values each in two pieces that turn by the same angles.  While a block is worked on the next one's rows are on their
//     way, and its angles from the middle of the block on; the barriers wait for LDS alone.  (One workgroup per block, nothing ahead: 160 us.)
//   * Short calls are bound by the latency of the chain flags -> token -> position -> angles and by fetching the code once, so it is one
//     loop, the tail's block included: 333 tokens of 8 heads 15.5 us (18.5 with twice the code).
//   * The first workgroup of a unit reads the old tail and is therefore also the one that writes the new one.
//   * len may change when all workgroups of the unit have read it: they count their arrival, the last one writes it.
//   * The result does not depend on how a row of tokens is cut into calls: a row is rounded to bf16 first, and to 8 bits with its
//     whole block.
#include <algorithm>

#include "ag_q8.h"

namespace {

// Up to here every workgroup counts its unit's flags itself (in flight with the other first loads): 333 tokens of 8 heads 25 us with a
// scan launched before, 18.5 us without.  Beyond, a unit's flags are scanned once.
constexpr int kCountedFlags = 16384;
// Workgroups per CU that a launch has at most: as many as a CU holds.  More of them count the flags again and carry nothing from block to
// block (512 units of 2048 tokens: 101 us, with 4 111); short calls have one per block either way.
constexpr int kFillWg = 2;

struct fill_args {
  const uint16_t *k, *v;
  const uint8_t *flags;    // nullptr: every token is kept
  uint64_t *words;         // the flags' masks and prefix counts: left by a unit's first workgroup, or read (CHUNKS = 0)
  int32_t *blk_off;
  ag_q8_dev c;
  ag_rope_dev rope;
  uint16_t *tiles;
  uint32_t *info;
  ag_q8_meta *meta;
  int32_t *arrived;  // [units] zero between launches
  int32_t *err;
  int Hkv, L, nw, n_blk;
};

// The flags of 16 tokens from t on as bits (those past L: 0).  A row of flags starts at any address.
__device__ __forceinline__ uint32_t flag_bits(const uint8_t *f, int t, int L) {
  uint32_t bits = 0;
  if (t + 16 <= L) {
    uint32_t w[4];
    __builtin_memcpy(w, f + t, 16);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint32_t on = (((w[i] & 0x7f7f7f7fu) + 0x7f7f7f7fu) | w[i]) & 0x80808080u;  // the top bit of every byte that is not 0
      bits |= (on >> 7 & 1) << (4 * i) | (on >> 15 & 1) << (4 * i + 1) | (on >> 23 & 1) << (4 * i + 2) | (on >> 31) << (4 * i + 3);
    }
  } else {
    for (int i = 0; i < L - t; ++i) bits |= (uint32_t)(f[t + i] != 0) << i;
  }
  return bits;
}

// CHUNKS: pieces of 16 flags that a thread reads (the workgroup: all of the unit's); 0: they are taken from words and blk_off.
template <int D, bool TILES, int CHUNKS>
__global__ __launch_bounds__(4 * D, 4) void ag_q8_fill_kernel(fill_args a) {
  constexpr int T = 4 * D, WAVES = T / 64;  // threads: 16 values of a row each
  constexpr int RS = D + 8;                 // values per row of V in LDS (rows 4 apart start 16 banks apart)
  __shared__ __attribute__((aligned(16))) uint16_t s_v[2][kQ8Block * RS];
  __shared__ int32_t s_tok[2][kQ8Block], s_stop, s_sum[WAVES];
  __shared__ struct {
    uint32_t top[2], least[2], odd;  // largest magnitudes of K, V; (TILES) those of their smallest rows; there are infinities or NaN
  } s_of[3];                         // (block x: the one of x % 3)
  const int u = blockIdx.y, wg = blockIdx.x, n_wg = gridDim.x, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  uint16_t *kt = a.c.k_tail + (size_t)u * kQ8Block * D, *vt = a.c.v_tail + (size_t)u * kQ8Block * D;
  const int most = a.c.max_blocks * kQ8Block + kQ8Block - 1;
  const int len0 = max(0, min(a.c.len[u], most));
  // ---- the kept tokens: this thread's flags and how many of the unit's lie before them ----
  uint32_t bits[CHUNKS ? CHUNKS : 1];
  int before = 0, mine = 0;
  if constexpr (CHUNKS > 0) {
    const int t = tid * 16 * CHUNKS;
#pragma unroll
    for (int i = 0; i < CHUNKS; ++i) {
      const int left = a.L - (t + 16 * i);
      bits[i] = a.flags ? (left > 0 ? flag_bits(a.flags + (size_t)u * a.L, t + 16 * i, a.L) : 0u) : (left >= 16 ? 0xffffu : (1u << max(left, 0)) - 1u);
      mine += __popc(bits[i]);
    }
  }
  if (tid == 0) s_stop = 0x7fffffff;
  if (tid < 3) {
    s_of[tid].top[0] = s_of[tid].top[1] = s_of[tid].odd = 0;
    s_of[tid].least[0] = s_of[tid].least[1] = 0x7f80;
  }
  const int held = len0 & (kQ8Block - 1), b0 = len0 / kQ8Block;
  const int32_t *page = a.c.page + (size_t)u * a.c.max_blocks;
  // ---- blocks of this call that may be filled and have no page: the first one ----
  int stop = 0x7fffffff;
  for (int j = tid; j < (held + a.L) / kQ8Block; j += T)
    if (b0 + j >= a.c.max_blocks || (uint32_t)page[min(b0 + j, a.c.max_blocks - 1)] >= (uint32_t)a.c.n_pages) {
      stop = j;
      break;
    }
  // Thread: of the rows, values d .. d + 7 and d + D / 2 .. + 7 of row t, which turn by the same angles; of the columns, rows
  // 16 i + 4 g + 0..3, i < 4, of column col.
  int t, d, g, col;
  auto set = [&](int me) {
    t = me / (D / 16);
    d = me % (D / 16) * 8;
    g = (me >> 4) & 3;
    col = 16 * (me >> 6) + (me & 15);
  };
  set(tid);
  auto d_of = [&](int e) { return d + e * (D / 2); };
  auto k_of = [&](int e) { return q8_k_at<D>(t, d_of(e) / 64, d_of(e) / 16 % 4) * 16 + (d & 8); };
  auto row_of = [&](int y) { return 16 * (y / 2) + 4 * g + 2 * (y & 1); };  // of the column's values 2 y and 2 y + 1, the first one
  if (wg == 0 && held > 0) {  // the tail's values, column by column, to where rows are read and written below
    const uint4 o0 = *reinterpret_cast<const uint4 *>(vt + tid * 16), o1 = *reinterpret_cast<const uint4 *>(vt + tid * 16 + 8);
    const uint32_t ow[8] = {o0.x, o0.y, o0.z, o0.w, o1.x, o1.y, o1.z, o1.w};
#pragma unroll
    for (int y = 0; y < 8; ++y) {
      s_v[0][row_of(y) * RS + col] = (uint16_t)ow[y];
      s_v[0][(row_of(y) + 1) * RS + col] = (uint16_t)(ow[y] >> 16);
    }
  }
  int kept;
  const int32_t *off = nullptr;
  if constexpr (CHUNKS > 0) {
    int sum;
    before = ag_wave_prefix(mine, sum);
    if (lane == 0) s_sum[wave] = sum;
    __syncthreads();
    kept = 0;
#pragma unroll
    for (int w = 0; w < WAVES; ++w) {
      if (w < wave) before += s_sum[w];
      kept += s_sum[w];
    }
    if (wg == 0 && a.words) {
      int r = before;
#pragma unroll
      for (int i = 0; i < CHUNKS; ++i) {
        const int t = tid * 16 * CHUNKS + 16 * i;
        if (t < a.nw * 64) reinterpret_cast<uint16_t *>(a.words + (size_t)u * a.nw)[t / 16] = (uint16_t)bits[i];
        if (t % 64 == 0 && t < a.nw * 64) a.blk_off[(size_t)u * (a.nw + 1) + t / 64] = r;
        r += __popc(bits[i]);
      }
      if (tid == 0) a.blk_off[(size_t)u * (a.nw + 1) + a.nw] = kept;
    }
  } else {
    if (a.flags) off = a.blk_off + (size_t)u * (a.nw + 1);
    kept = off ? off[a.nw] : a.L;
    __syncthreads();
  }
  if (stop < 0x7fffffff) atomicMin(&s_stop, stop);
  int order = 0;
  if (tid == 0) order = __hip_atomic_fetch_add(a.arrived + u, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);  // (len has been read)
  __syncthreads();
  // rows that there is room for: up to the one that would fill the first block without a page
  const int want = (held + kept) / kQ8Block;
  const int add = s_stop < want ? s_stop * kQ8Block + kQ8Block - 1 - held : kept;
  const int total = held + add, full = total / kQ8Block;
  const uint16_t *K = a.k + (size_t)u * a.L * D, *V = a.v + (size_t)u * a.L * D;
  const int n_full = full > wg ? (full - 1 - wg) / n_wg + 1 : 0, n = n_full + (wg == 0 && full * kQ8Block < total ? 1 : 0);
  auto block_of = [&](int x) { return x < n_full ? wg + x * n_wg : full; };
  auto barrier = [] {  // that waits for LDS alone: loads and stores stay in flight
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
  };
  auto tokens = [&](int x) {  // the tokens of its rows, row r0 + i the unit's kept token kk0 + i of this call
    const int kk0 = block_of(x) * kQ8Block - held, hi = min(kk0 + kQ8Block, add);
    int32_t *tok = s_tok[x & 1];
    if constexpr (CHUNKS > 0) {
      if (before < hi && before + mine > kk0) {
        int r = before - kk0;
#pragma unroll
        for (int i = 0; i < CHUNKS; ++i)
          for (uint32_t m = bits[i]; m; m &= m - 1, ++r)
            if (r >= 0 && r < kQ8Block) tok[r] = (tid * CHUNKS + i) * 16 + __builtin_ctz(m);
      }
    } else if (!off) {
      if (tid < kQ8Block) tok[tid] = kk0 + tid;
    } else {
      for (int w = tid; w < a.nw; w += T) {
        int r = off[w] - kk0;
        if (r < kQ8Block && off[w + 1] > kk0)
          for (uint64_t m = a.words[(size_t)u * a.nw + w]; m; m &= m - 1, ++r)
            if (r >= 0 && r < kQ8Block) tok[r] = w * 64 + __builtin_ctzll(m);
      }
    }
  };
  // While a block is worked on, the next one's rows are on their way: first the positions, whose angles are asked for between the
  // block's two halves.
  q8_u32x4 kn[2] = {}, vn[2] = {};
  uint32_t at0 = 0, at1 = 0, at2 = 0;
  q8_f32x4 an[4];
  auto request = [&](int x) {
    const int row = block_of(x) * kQ8Block + t;
    if (row < total) {
      const bool old = row < held;  // (its values of V come from LDS; token 0's are read in their place)
      const int tok = old ? 0 : s_tok[x & 1][t];
      if (!old && a.rope.table) {
        const q8_rows r = q8_rope_rows(a.rope, (int64_t)(u / a.Hkv) * a.L + tok, a.err);
        at0 = r.r0; at1 = r.r1; at2 = r.r2;
      }
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        kn[e] = *reinterpret_cast<const q8_u32x4 *>(old ? kt + k_of(e) : K + (size_t)tok * D + d_of(e));
        vn[e] = *reinterpret_cast<const q8_u32x4 *>(V + (size_t)tok * D + d_of(e));
      }
    }
  };
  auto turn_by = [&] {
    if (a.rope.table) {  // (rows that are not there: by some row of the table)
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const q8_angles y = q8_angles4(a.rope, q8_rows{at0, at1, at2}, d + 4 * i, D);
        an[2 * i] = q8_f32x4{y.c.x, y.c.y, y.c.z, y.c.w};
        an[2 * i + 1] = q8_f32x4{y.s.x, y.s.y, y.s.z, y.s.w};
      }
    }
  };
  if (n > 0) {
    tokens(0);
    if (n > 1) tokens(1);
    barrier();
    request(0);
    if (n > 2) barrier();  // (block 0's list has been read: the first turn of the loop writes block 2's over it)
    turn_by();
  }
#pragma unroll 1
  for (int x = 0; x < n; ++x) {
    int me = tid;
    asm volatile("" : "+v"(me));  // (unknown to the compiler: it would keep every address below in registers)
    set(me);
    const int j = block_of(x), r0 = j * kQ8Block;
    auto &of = s_of[x % 3];
    uint16_t *sv = s_v[x & 1];
    // ---- rows ----
    const bool old = r0 + t < held, there = r0 + t < total && !old;  // (old: only in block 0)
    uint4 kx[2], vx[2];
    q8_eight kf[2];  // (TILES) keys before they are rounded to bf16
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      kx[e] = __builtin_bit_cast(uint4, old || there ? kn[e] : q8_u32x4{});
      vx[e] = __builtin_bit_cast(uint4, there ? vn[e] : q8_u32x4{});
    }
    if (old) {
#pragma unroll
      for (int e = 0; e < 2; ++e) vx[e] = *reinterpret_cast<const uint4 *>(sv + t * RS + d_of(e));
    }
#pragma unroll
    for (int e = 0; e < 2; ++e) kf[e] = q8_floats(kx[e]);
    if (x + 1 < n) request(x + 1);
    if (there && a.rope.table) {
#pragma unroll
      for (int e = 0; e < 2; ++e) kf[e] = q8_turn8(an, e == 0, kx[e], kx[e ^ 1]);
#pragma unroll
      for (int e = 0; e < 2; ++e) kx[e] = kf[e].bf16();
    }
    q8_u16x2 both_k = {0, 0}, both_v = {0, 0};  // the magnitudes' bits
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      const uint32_t w[4] = {kx[e].x, kx[e].y, kx[e].z, kx[e].w}, v[4] = {vx[e].x, vx[e].y, vx[e].z, vx[e].w};
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        both_k = __builtin_elementwise_max(both_k, __builtin_bit_cast(q8_u16x2, w[i] & 0x7fff7fffu));
        both_v = __builtin_elementwise_max(both_v, __builtin_bit_cast(q8_u16x2, v[i] & 0x7fff7fffu));
      }
      if (!old) *reinterpret_cast<uint4 *>(sv + t * RS + d_of(e)) = vx[e];
    }
    uint32_t top_k = max(both_k[0], both_k[1]), top_v = max(both_v[0], both_v[1]);
    if (max(top_k, top_v) >= 0x7f80u) {  // rare: infinities and NaN do not count
      of.odd = 1;
      top_k = top_v = 0;
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        top_k = q8_top(q8_top(q8_top(q8_top(top_k, kx[e].x), kx[e].y), kx[e].z), kx[e].w);
        top_v = q8_top(q8_top(q8_top(q8_top(top_v, vx[e].x), vx[e].y), vx[e].z), vx[e].w);
      }
    }
    if constexpr (TILES) {
#pragma unroll
      for (int o = 1; o < D / 16; o <<= 1) {  // over a row
        top_k = max(top_k, (uint32_t)__shfl_xor((int)top_k, o, 64));
        top_v = max(top_v, (uint32_t)__shfl_xor((int)top_v, o, 64));
      }
      uint32_t least_k = top_k ? top_k : 0x7f80u, least_v = top_v ? top_v : 0x7f80u;
#pragma unroll
      for (int o = D / 16; o <= 32; o <<= 1) {
        top_k = max(top_k, (uint32_t)__shfl_xor((int)top_k, o, 64));
        top_v = max(top_v, (uint32_t)__shfl_xor((int)top_v, o, 64));
        least_k = min(least_k, (uint32_t)__shfl_xor((int)least_k, o, 64));
        least_v = min(least_v, (uint32_t)__shfl_xor((int)least_v, o, 64));
      }
      if (lane == 0) {
        atomicMin(&of.least[0], least_k);
        atomicMin(&of.least[1], least_v);
      }
    } else {
#pragma unroll
      for (int o = 1; o <= 32; o <<= 1) {
        top_k = max(top_k, (uint32_t)__shfl_xor((int)top_k, o, 64));
        top_v = max(top_v, (uint32_t)__shfl_xor((int)top_v, o, 64));
      }
    }
    if (lane == 0) {
      atomicMax(&of.top[0], top_k);
      atomicMax(&of.top[1], top_v);
    }
    if (tid == 0) {
      auto &next = s_of[(x + 1) % 3];  // (last read two blocks ago)
      next.top[0] = next.top[1] = next.odd = 0;
      next.least[0] = next.least[1] = 0x7f80;
    }
    if (x + 2 < n) tokens(x + 2);
    barrier();
    if (x + 1 < n) turn_by();
    // ---- columns ----
    uint32_t vw[8];
#pragma unroll
    for (int y = 0; y < 8; ++y) vw[y] = sv[row_of(y) * RS + col] | (uint32_t)sv[(row_of(y) + 1) * RS + col] << 16;
    const uint32_t block_k = of.top[0], block_v = of.top[1];
    const bool odd = __builtin_amdgcn_readfirstlane(of.odd) != 0;
    if constexpr (TILES) {  // as the attention's tiles lie in LDS (ag_q8_prefill.hip)
      auto binade = [](uint32_t top) { return max((int)(top >> 7), 1) - 127; };
      const bool row_by_row = odd || (block_k && binade(of.least[0]) + kQ8TileSpan < binade(block_k)) ||
                              (block_v && binade(of.least[1]) + kQ8TileSpan < binade(block_v));
      const int ek = max(kQ8TileMinExp, binade(block_k) - kQ8TileTop), ev = max(kQ8TileMinExp, binade(block_v) - kQ8TileTop);
      const float ik = q8_pow2(-ek), iv = q8_pow2(-ev);
      uint16_t *tk = a.tiles + ((size_t)u * a.n_blk + j) * 2 * kQ8Block * D, *tv = tk + kQ8Block * D;
#pragma unroll
      for (int e = 0; e < 2; ++e) {  // row t % 32 of fragment (t / 32, d / 16), half d / 8 % 2
        *reinterpret_cast<uint4 *>(tk + ((((t >> 5) * (D / 16) + d_of(e) / 16) * 2 + (d >> 3 & 1)) * 32 + (t & 31)) * 8) =
            row_by_row ? kx[e] : __builtin_bit_cast(uint4, kf[e].f16(ik));
      }
      auto half2 = [&](uint32_t w) {
        const q8_f32x2 y = {q8_lo(w) * iv, q8_hi(w) * iv};
        return row_by_row ? w : __builtin_bit_cast(uint32_t, __builtin_convertvector(y, q8_f16x2));
      };
#pragma unroll
      for (int i = 0; i < 4; ++i)
        *reinterpret_cast<uint2 *>(tv + (((((col >> 5) * 4 + i) * 2 + (g & 1)) * 32 + (col & 31)) * 8 + (g >> 1) * 4)) =
            make_uint2(half2(vw[2 * i]), half2(vw[2 * i + 1]));
      if (tid == 0) a.info[(size_t)u * a.n_blk + j] = q8_tile_word(ek, ev, row_by_row);
    }
    if (j < full) {  // ---- a page ----
      const int id = page[b0 + j];
      const int ek = q8_exponent(block_k), ev = q8_exponent(block_v);
      uint2 nk[2], nv[2];
      const float sk = q8_pow2(ek), sv = q8_pow2(ev);
      if (!odd) {
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          nk[e] = make_uint2(q8_narrow_finite(kx[e].x, kx[e].y, sk), q8_narrow_finite(kx[e].z, kx[e].w, sk));
          nv[e] = make_uint2(q8_narrow_finite(vw[4 * e], vw[4 * e + 1], sv), q8_narrow_finite(vw[4 * e + 2], vw[4 * e + 3], sv));
        }
      } else {
        const float ik = q8_pow2(-ek), iv = q8_pow2(-ev);
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          nk[e] = make_uint2(q8_narrow(kx[e].x, kx[e].y, ik), q8_narrow(kx[e].z, kx[e].w, ik));
          nv[e] = make_uint2(q8_narrow(vw[4 * e], vw[4 * e + 1], iv), q8_narrow(vw[4 * e + 2], vw[4 * e + 3], iv));
        }
      }
      uint8_t *pk = a.c.k + (size_t)id * kQ8Block * D;
#pragma unroll
      for (int e = 0; e < 2; ++e) *reinterpret_cast<uint2 *>(pk + k_of(e)) = nk[e];
      reinterpret_cast<uint4 *>(a.c.v + (size_t)id * kQ8Block * D)[me] = make_uint4(nv[0].x, nv[0].y, nv[1].x, nv[1].y);
      if (tid == 0) {
        a.c.k_scale[id] = sk;
        a.c.v_scale[id] = sv;
      }
    } else {  // ---- the tail ----
      if (there) {
#pragma unroll
        for (int e = 0; e < 2; ++e) *reinterpret_cast<uint4 *>(kt + k_of(e)) = kx[e];
      }
#pragma unroll
      for (int y = 0; y < 8; ++y) {
        const int row = r0 + row_of(y);
        uint16_t *p = vt + me * 16 + 2 * y;
        if (row >= held && row < total) p[0] = (uint16_t)vw[y];
        if (row + 1 >= held && row + 1 < total) p[1] = (uint16_t)(vw[y] >> 16);
      }
    }
  }
  if (tid == 0) {  // the last workgroup that read len writes it
    if (order == n_wg - 1) {
      a.arrived[u] = 0;
      a.c.len[u] = len0 + add;
      if (add < kept) atomicOr(a.err, 1);
    }
    if (TILES && wg == 0) a.meta[u] = ag_q8_meta{b0, held, add, 0};
  }
}

}  // namespace

hipError_t ag_launch_q8_fill(ag_ctx *ctx, hipStream_t s, const void *k, const void *v, const uint8_t *flags, int B, int Hkv, int L, int D,
                             uint64_t *words, int32_t *blk_off, const ag_rope_dev &rope, const ag_q8_dev &cache,
                             uint16_t *tiles, uint32_t *info, ag_q8_meta *meta) {
  fill_args a;
  a.k = (const uint16_t *)k; a.v = (const uint16_t *)v; a.flags = flags;
  a.words = words; a.blk_off = blk_off; a.c = cache; a.rope = rope;
  a.tiles = tiles; a.info = info; a.meta = meta;
  a.arrived = ctx->decode_tickets; a.err = ctx->d_err;
  a.Hkv = Hkv; a.L = L; a.nw = ag_nwords(L); a.n_blk = ag_q8_fill_blocks(L);
  const dim3 grid(std::min(a.n_blk, std::max(1, kFillWg * ctx->num_cu / (B * Hkv))), B * Hkv), block(4 * D);
  if (flags && L > kCountedFlags) {
    const hipError_t e = ag_launch_flag_scan(ctx, s, flags, B * Hkv, L, words, blk_off, nullptr);
    if (e != hipSuccess) return e;
  }
#define AG_FILL(DD, TT, CC) AG_LAUNCH(ag_time_kernel(ctx, AG_K_Q8_FILL), (ag_q8_fill_kernel<DD, TT, CC>), grid, block, 0, s, a)
#define AG_FILL_C(DD, TT)                                                          \
  do {                                                                             \
    if (L <= 16 * 4 * DD) AG_FILL(DD, TT, 1);                                      \
    else if (L <= kCountedFlags) AG_FILL(DD, TT, kCountedFlags / (16 * 4 * DD));   \
    else AG_FILL(DD, TT, 0);                                                       \
  } while (0)
  if (D == 128 && tiles) AG_FILL_C(128, true);
  else if (D == 128) AG_FILL_C(128, false);
  else if (tiles) AG_FILL_C(64, true);
  else AG_FILL_C(64, false);
#undef AG_FILL_C
#undef AG_FILL
  return hipGetLastError();
}
