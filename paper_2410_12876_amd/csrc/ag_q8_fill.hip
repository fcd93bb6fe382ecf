// Filling the paged 8-bit cache: a call's kept tokens join their units, keys turned on the way.
//
// A unit's new rows follow its tail; rows 64 j .. 64 j + 63 of (tail, new rows) are its block j of this call.  One workgroup makes
// one block: it finds the block's tokens from the flags' prefix counts, reads their rows of k and v once (a row is 128 or 256
// bytes in one piece), turns k, takes the largest magnitude for the scale and writes the codes in page order; V is transposed
// through LDS.  A block that stays incomplete is written to the tail instead.  Bound by memory: the kept rows in bf16 in, in 8 bits out.
//   * The first workgroup of a unit reads the old tail and is therefore also the one that writes the new one.
//   * len may change when all workgroups of the unit have read it: they count their arrival, the last one writes it.
//   * The result does not depend on how a row of tokens is cut into calls: a row is rounded to bf16 first, and to 8 bits with its
//     whole block.
#include "ag_q8.h"

namespace {

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

// Sum over the lanes before this one; total: the wave's sum.
__device__ __forceinline__ int wave_prefix(int x, int &total) {
  int y = x;
  y += __builtin_amdgcn_update_dpp(0, y, 0x111, 0xf, 0xf, false);
  y += __builtin_amdgcn_update_dpp(0, y, 0x112, 0xf, 0xf, false);
  y += __builtin_amdgcn_update_dpp(0, y, 0x114, 0xf, 0xf, false);
  y += __builtin_amdgcn_update_dpp(0, y, 0x118, 0xf, 0xf, false);
  y += __builtin_amdgcn_update_dpp(0, y, 0x142, 0xa, 0xf, false);
  y += __builtin_amdgcn_update_dpp(0, y, 0x143, 0xc, 0xf, false);
  total = __builtin_amdgcn_readlane(y, 63);
  return y - x;
}
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
__global__ __launch_bounds__(256) void ag_q8_fill_kernel(fill_args a) {
  constexpr int KC = D / 64, VF = D / 64;  // K: chunks of 64 columns; V: pieces of 16 columns per wave
  constexpr int RS = D + 8;                // values per row of V in LDS (rows 4 apart start 16 banks apart)
  __shared__ __attribute__((aligned(16))) uint16_t s_v[kQ8Block * RS];
  __shared__ int32_t s_tok[kQ8Block], s_stop, s_order;
  __shared__ uint32_t s_top[2], s_least[2], s_odd;  // largest magnitudes of K, V; (TILES) those of their smallest rows; not finite
  __shared__ int32_t s_sum[4];
  const int u = blockIdx.y, wg = blockIdx.x, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
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
  const int held = len0 & (kQ8Block - 1), b0 = len0 / kQ8Block;
  const int32_t *page = a.c.page + (size_t)u * a.c.max_blocks;
  // ---- blocks of this call that may be filled and have no page: the first one ----
  int stop = 0x7fffffff;
  for (int j = tid; j < (held + a.L) / kQ8Block; j += 256)
    if (b0 + j >= a.c.max_blocks || (uint32_t)page[min(b0 + j, a.c.max_blocks - 1)] >= (uint32_t)a.c.n_pages) {
      stop = j;
      break;
    }
  int kept;
  const int32_t *off = nullptr;
  if constexpr (CHUNKS > 0) {
    int sum;
    before = wave_prefix(mine, sum);
    if (lane == 0) s_sum[wave] = sum;
    __syncthreads();
    kept = 0;
#pragma unroll
    for (int w = 0; w < 4; ++w) {
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
  __syncthreads();
  // rows that there is room for: up to the one that would fill the first block without a page
  const int want = (held + kept) / kQ8Block;
  const int add = s_stop < want ? s_stop * kQ8Block + kQ8Block - 1 - held : kept;
  const int total = held + add, full = total / kQ8Block;
  if (tid == 0) {  // (len has been read)
    s_order = __hip_atomic_fetch_add(a.arrived + u, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    if (s_order == (int)gridDim.x - 1) {
      a.arrived[u] = 0;
      a.c.len[u] = len0 + add;
      if (add < kept) atomicOr(a.err, 1);
    }
    if (TILES && wg == 0) a.meta[u] = ag_q8_meta{b0, held, add, 0};
  }
  const uint16_t *K = a.k + (size_t)u * a.L * D, *V = a.v + (size_t)u * a.L * D;
  uint16_t *kt = a.c.k_tail + (size_t)u * kQ8Block * D, *vt = a.c.v_tail + (size_t)u * kQ8Block * D;

  auto block = [&](int j) {
    // ---- its tokens ----
    const int r0 = j * kQ8Block, kk0 = r0 - held;  // row r0 + i is the unit's kept token kk0 + i of this call
    if (tid < kQ8Block) s_tok[tid] = -1;
    if (tid < 2) { s_top[tid] = 0; s_least[tid] = 0x7f80; }
    if (tid == 0) s_odd = 0;
    if (r0 < held) {  // the tail's values, column by column, to where rows are read and written below
#pragma unroll
      for (int x = 0; x < VF; ++x) {
        const int f = VF * wave + x, gg = lane >> 4;
        const uint4 o0 = *reinterpret_cast<const uint4 *>(vt + (f * 64 + lane) * 16), o1 = *reinterpret_cast<const uint4 *>(vt + (f * 64 + lane) * 16 + 8);
        const uint32_t ow[8] = {o0.x, o0.y, o0.z, o0.w, o1.x, o1.y, o1.z, o1.w};
#pragma unroll
        for (int y = 0; y < 8; ++y) {
          const int row = 16 * (y / 2) + 4 * gg + 2 * (y & 1);
          s_v[row * RS + 16 * f + (lane & 15)] = (uint16_t)ow[y];
          s_v[(row + 1) * RS + 16 * f + (lane & 15)] = (uint16_t)(ow[y] >> 16);
        }
      }
    }
    __syncthreads();
    const int hi = min(kk0 + kQ8Block, add);
    if constexpr (CHUNKS > 0) {
      int r = before;
      if (r < hi && r + mine > kk0) {
#pragma unroll
        for (int i = 0; i < CHUNKS; ++i)
#pragma unroll
          for (int x = 0; x < 16; ++x)
            if (bits[i] >> x & 1) {
              if (r >= kk0 && r < hi) s_tok[r - kk0] = (tid * CHUNKS + i) * 16 + x;
              ++r;
            }
      }
    } else if (!off) {
      if (tid < kQ8Block && kk0 + tid >= 0 && kk0 + tid < hi) s_tok[tid] = kk0 + tid;
    } else {
      for (int w = tid; w < a.nw; w += 256) {
        int r = off[w];
        if (r < hi && off[w + 1] > kk0) {
          for (uint64_t m = a.words[(size_t)u * a.nw + w]; m; m &= m - 1, ++r)
            if (r >= kk0 && r < hi) s_tok[r - kk0] = w * 64 + __builtin_ctzll(m);
        }
      }
    }
    __syncthreads();
    // ---- rows: thread (row 16 wave + lane % 16, columns 64 c + 16 g ..) ----
    const int t = 16 * wave + (lane & 15), g = lane >> 4;
    const bool old = r0 + t < held;  // (only in block 0)
    const int tok = s_tok[t];
    uint4 kx[KC][2], vx[KC][2];
    q8_eight kf[KC][2];  // (TILES) keys before they are rounded to bf16
#pragma unroll
    for (int c = 0; c < KC; ++c)
#pragma unroll
      for (int s = 0; s < 2; ++s) {
        kx[c][s] = vx[c][s] = make_uint4(0, 0, 0, 0);
        const int d = 64 * c + 16 * g + 8 * s;
        if (old) {
          kx[c][s] = *reinterpret_cast<const uint4 *>(kt + q8_k_at<D>(t, c, g) * 16 + 8 * s);
          vx[c][s] = *reinterpret_cast<const uint4 *>(s_v + t * RS + d);
        } else if (tok >= 0) {
          kx[c][s] = *reinterpret_cast<const uint4 *>(K + (size_t)tok * D + d);
          vx[c][s] = *reinterpret_cast<const uint4 *>(V + (size_t)tok * D + d);
        }
        kf[c][s] = q8_floats(kx[c][s]);
      }
    if (!old && tok >= 0 && a.rope.table) {
      const q8_rows at = q8_rope_rows(a.rope, (int64_t)(u / a.Hkv) * a.L + tok, a.err);
#pragma unroll
      for (int c = 0; c < KC; ++c)
#pragma unroll
        for (int s = 0; s < 2; ++s) {
          const int d = 64 * c + 16 * g + 8 * s;
          uint4 p;
          if constexpr (KC == 2) p = kx[c ^ 1][s];
          else p = *reinterpret_cast<const uint4 *>(K + (size_t)tok * D + (d ^ (D / 2)));
          kf[c][s] = q8_turn8<D>([&](int i) { return q8_angles4(a.rope, at, i, D); }, d, kx[c][s], p);
        }
#pragma unroll
      for (int c = 0; c < KC; ++c)
#pragma unroll
        for (int s = 0; s < 2; ++s) kx[c][s] = kf[c][s].bf16();
    }
    uint32_t top_k = 0, top_v = 0, odd = 0;
#pragma unroll
    for (int c = 0; c < KC; ++c)
#pragma unroll
      for (int s = 0; s < 2; ++s) {
        const uint32_t w[4] = {kx[c][s].x, kx[c][s].y, kx[c][s].z, kx[c][s].w}, x[4] = {vx[c][s].x, vx[c][s].y, vx[c][s].z, vx[c][s].w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          top_k = q8_top(top_k, w[i]);
          top_v = q8_top(top_v, x[i]);
          if (TILES) odd |= (uint32_t)((x[i] & 0x7f80u) == 0x7f80u) | (uint32_t)((x[i] & 0x7f800000u) == 0x7f800000u) |
                            (uint32_t)((w[i] & 0x7f80u) == 0x7f80u) | (uint32_t)((w[i] & 0x7f800000u) == 0x7f800000u);
        }
        if (!old) *reinterpret_cast<uint4 *>(s_v + t * RS + 64 * c + 16 * g + 8 * s) = vx[c][s];
      }
    auto over = [](uint32_t x, int from, int to, auto &&f) {  // over lanes `from`, 2 from, .. to apart
      for (int o = from; o <= to; o <<= 1) x = f(x, (uint32_t)__shfl_xor((int)x, o, 64));
      return x;
    };
    auto larger = [](uint32_t x, uint32_t y) { return max(x, y); };
    auto smaller = [](uint32_t x, uint32_t y) { return min(x, y); };
    if constexpr (TILES) {
      const uint32_t row_k = over(top_k, 16, 32, larger), row_v = over(top_v, 16, 32, larger);  // (a row's four threads)
      const uint32_t least_k = over(row_k ? row_k : 0x7f80u, 1, 8, smaller), least_v = over(row_v ? row_v : 0x7f80u, 1, 8, smaller);
      if (odd) s_odd = 1;
      if (lane == 0) {
        atomicMin(&s_least[0], least_k);
        atomicMin(&s_least[1], least_v);
      }
    }
    top_k = over(top_k, 1, 32, larger);
    top_v = over(top_v, 1, 32, larger);
    if (lane == 0) {
      atomicMax(&s_top[0], top_k);
      atomicMax(&s_top[1], top_v);
    }
    __syncthreads();
    // ---- columns: thread (column 16 f + lane % 16, rows 16 i + 4 g + 0..3), f = VF wave .. ----
    uint32_t vw[VF][8];
#pragma unroll
    for (int x = 0; x < VF; ++x)
#pragma unroll
      for (int y = 0; y < 8; ++y) {
        const int row = 16 * (y / 2) + 4 * g + 2 * (y & 1);
        vw[x][y] = s_v[row * RS + 16 * (VF * wave + x) + (lane & 15)] | (uint32_t)s_v[(row + 1) * RS + 16 * (VF * wave + x) + (lane & 15)] << 16;
      }
    if constexpr (TILES) {  // as the attention's tiles lie in LDS (ag_q8_prefill.hip)
      auto binade = [](uint32_t top) { return max((int)(top >> 7), 1) - 127; };
      const bool row_by_row = s_odd != 0 || (s_top[0] && binade(s_least[0]) + kQ8TileSpan < binade(s_top[0])) ||
                              (s_top[1] && binade(s_least[1]) + kQ8TileSpan < binade(s_top[1]));
      const int ek = max(kQ8TileMinExp, binade(s_top[0]) - kQ8TileTop), ev = max(kQ8TileMinExp, binade(s_top[1]) - kQ8TileTop);
      const float ik = q8_pow2(-ek), iv = q8_pow2(-ev);
      uint16_t *tk = a.tiles + ((size_t)u * a.n_blk + j) * 2 * kQ8Block * D, *tv = tk + kQ8Block * D;
#pragma unroll
      for (int c = 0; c < KC; ++c)
#pragma unroll
        for (int s = 0; s < 2; ++s)
          *reinterpret_cast<uint4 *>(tk + ((((t >> 5) * (D / 16) + 4 * c + g) * 2 + s) * 32 + (t & 31)) * 8) =
              row_by_row ? kx[c][s] : __builtin_bit_cast(uint4, kf[c][s].f16(ik));
      auto half2 = [&](uint32_t w) {
        const q8_f32x2 x = {q8_lo(w) * iv, q8_hi(w) * iv};
        return row_by_row ? w : __builtin_bit_cast(uint32_t, __builtin_convertvector(x, q8_f16x2));
      };
#pragma unroll
      for (int x = 0; x < VF; ++x) {
        const int f = VF * wave + x;
#pragma unroll
        for (int i = 0; i < 4; ++i)
          *reinterpret_cast<uint2 *>(tv + (((((f >> 1) * 4 + i) * 2 + (g & 1)) * 32 + (f & 1) * 16 + (lane & 15)) * 8 + (g >> 1) * 4)) =
              make_uint2(half2(vw[x][2 * i]), half2(vw[x][2 * i + 1]));
      }
      if (tid == 0) a.info[(size_t)u * a.n_blk + j] = q8_tile_word(ek, ev, row_by_row);
    }
    if (j < full) {  // ---- a page ----
      const int id = page[b0 + j];
      const int ek = q8_exponent(s_top[0]), ev = q8_exponent(s_top[1]);
      const float ik = q8_pow2(-ek), iv = q8_pow2(-ev);
      uint4 *pk = reinterpret_cast<uint4 *>(a.c.k + (size_t)id * kQ8Block * D), *pv = reinterpret_cast<uint4 *>(a.c.v + (size_t)id * kQ8Block * D);
#pragma unroll
      for (int c = 0; c < KC; ++c)
        pk[q8_k_at<D>(t, c, g)] = make_uint4(q8_narrow(kx[c][0].x, kx[c][0].y, ik), q8_narrow(kx[c][0].z, kx[c][0].w, ik),
                                             q8_narrow(kx[c][1].x, kx[c][1].y, ik), q8_narrow(kx[c][1].z, kx[c][1].w, ik));
#pragma unroll
      for (int x = 0; x < VF; ++x)
        pv[(VF * wave + x) * 64 + lane] = make_uint4(q8_narrow(vw[x][0], vw[x][1], iv), q8_narrow(vw[x][2], vw[x][3], iv),
                                                     q8_narrow(vw[x][4], vw[x][5], iv), q8_narrow(vw[x][6], vw[x][7], iv));
      if (tid == 0) {
        a.c.k_scale[id] = q8_pow2(ek);
        a.c.v_scale[id] = q8_pow2(ev);
      }
    } else {  // ---- the tail ----
      if (!old && r0 + t < total) {
#pragma unroll
        for (int c = 0; c < KC; ++c)
#pragma unroll
          for (int s = 0; s < 2; ++s) *reinterpret_cast<uint4 *>(kt + q8_k_at<D>(t, c, g) * 16 + 8 * s) = kx[c][s];
      }
#pragma unroll
      for (int x = 0; x < VF; ++x)
#pragma unroll
        for (int y = 0; y < 8; ++y) {
          const int row = 16 * (y / 2) + 4 * g + 2 * (y & 1);
          uint16_t *p = vt + ((VF * wave + x) * 64 + lane) * 16 + 2 * y;
          if (r0 + row >= held && r0 + row < total) p[0] = (uint16_t)vw[x][y];
          if (r0 + row + 1 >= held && r0 + row + 1 < total) p[1] = (uint16_t)(vw[x][y] >> 16);
        }
    }
    __syncthreads();  // (LDS is free again, the old tail has been read)
  };
  if (wg < full || wg == 0) {
    if (wg * kQ8Block < total) block(wg);
    if (wg == 0 && full > 0 && full * kQ8Block < total) block(full);
  }
}

}  // namespace

// Up to here every workgroup counts the unit's flags itself (at most 64 a thread, in flight with the other first loads): 333 tokens of 8
// heads 25 us with a scan launched before, XX without.  Beyond, a unit's flags are scanned once.
int ag_q8_fill_flags() { return 4 * 16 * 256; }

hipError_t ag_launch_q8_fill(ag_ctx *ctx, hipStream_t s, const void *k, const void *v, const uint8_t *flags, int B, int Hkv, int L, int D,
                             uint64_t *words, int32_t *blk_off, const ag_rope_dev &rope, const ag_q8_dev &cache,
                             uint16_t *tiles, uint32_t *info, ag_q8_meta *meta) {
  fill_args a;
  a.k = (const uint16_t *)k; a.v = (const uint16_t *)v; a.flags = flags;
  a.words = words; a.blk_off = blk_off; a.c = cache; a.rope = rope;
  a.tiles = tiles; a.info = info; a.meta = meta;
  a.arrived = ctx->decode_tickets; a.err = ctx->d_err;
  a.Hkv = Hkv; a.L = L; a.nw = ag_nwords(L); a.n_blk = ag_q8_fill_blocks(L);
  const dim3 grid(a.n_blk, B * Hkv), block(256);
  if (flags && L > ag_q8_fill_flags()) {
    const hipError_t e = ag_launch_flag_scan(ctx, s, flags, B * Hkv, L, words, blk_off, nullptr);
    if (e != hipSuccess) return e;
  }
#define AG_FILL(DD, TT, CC) AG_LAUNCH(ag_time_kernel(ctx, AG_K_Q8_FILL), (ag_q8_fill_kernel<DD, TT, CC>), grid, block, 0, s, a)
#define AG_FILL_C(DD, TT)                       \
  do {                                          \
    if (L <= 4096) AG_FILL(DD, TT, 1);          \
    else if (L <= 16384) AG_FILL(DD, TT, 4);    \
    else AG_FILL(DD, TT, 0);                    \
  } while (0)
  if (D == 128 && tiles) AG_FILL_C(128, true);
  else if (D == 128) AG_FILL_C(128, false);
  else if (tiles) AG_FILL_C(64, true);
  else AG_FILL_C(64, false);
#undef AG_FILL_C
#undef AG_FILL
  return hipGetLastError();
}
