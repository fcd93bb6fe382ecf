// Rotary positions: q and k of a layer turned in one launch, by one to three position axes.
//   pair i of a vector (values i and i + D/2), angle row p = pos[axis(i)][token]:  y_i = x_i cos - x_(i+D/2) sin,
//   y_(i+D/2) = x_(i+D/2) cos + x_i sin; products and sum rounded one by one in 32 bits, then once to the type.
// Bound by memory: 2 (Hq + Hkv) tokens D values in and out.  A thread owns 16 bytes of a vector and the 16 bytes of their partners
// for several heads of one token, so that the angles (as many bytes as two bf16 vectors) are read once for all of those.
// 4096 tokens x 64 heads of 128 in bf16: 26.4 to 27 us, 5.0 to 5.2 TB/s; 2 x 2900 tokens x 40 heads of 64 in fp32, three axes: 24.6 us.
#include "ag_q8.h"

namespace {

// Heads whose loads are in flight together (1, 2, 4, 8: 27.2, 26.9, 27.0, 26.6 us in bf16, 24.0, 24.6, 25.0, 27.2 in fp32 at the sizes above).
constexpr int kHeadsAtOnce = 2;

template <typename T> __device__ __forceinline__ void unpack(const uint4 &x, float *f) {
  const uint32_t w[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if constexpr (sizeof(T) == 2) {
      f[2 * i] = q8_lo(w[i]);
      f[2 * i + 1] = q8_hi(w[i]);
    } else {
      f[i] = __uint_as_float(w[i]);
    }
  }
}
template <typename T> __device__ __forceinline__ uint4 pack(const float *f) {
  if constexpr (sizeof(T) == 2) return make_uint4(q8_pack2(f[0], f[1]), q8_pack2(f[2], f[3]), q8_pack2(f[4], f[5]), q8_pack2(f[6], f[7]));
  return make_uint4(__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3]));
}

// grid (chunks of 256 (token, piece) pairs, groups of `heads` heads).  q and q_out (k and k_out) may be the same memory.
template <typename T>
__global__ __launch_bounds__(256) void ag_rotate_kernel(const T *q, const T *k, T *q_out, T *k_out, int tokens, int Hq, int Hkv, int L,
                                                        int D, int heads, ag_rope_dev rope, int32_t *err) {
  constexpr int E = 16 / sizeof(T);  // values of a piece
  const int pieces = D / 2 / E;
  const int64_t id = (int64_t)blockIdx.x * 256 + threadIdx.x;
  const int n = (int)(id / pieces), i = (int)(id - (int64_t)n * pieces) * E;
  if (n >= tokens) return;
  const int b = n / L, t = n - b * L;
  const q8_rows at = q8_rope_rows(rope, n, err);
  float c[E], s[E];
#pragma unroll
  for (int j = 0; j < E; j += 4) {
    if (rope.quads) {
      const q8_angles e = q8_angles4(rope, at, i + j, D);
      c[j] = e.c.x; c[j + 1] = e.c.y; c[j + 2] = e.c.z; c[j + 3] = e.c.w;
      s[j] = e.s.x; s[j + 1] = e.s.y; s[j + 2] = e.s.z; s[j + 3] = e.s.w;
    } else {
#pragma unroll
      for (int x = j; x < j + 4; ++x) {
        const float *row = q8_angle_row(rope, at, i + x, D) + i + x;
        c[x] = row[0];
        s[x] = row[D / 2];
      }
    }
  }
  const int h0 = blockIdx.y * heads, h1 = min(h0 + heads, Hq + Hkv);
  for (int h = h0; h < h1; h += kHeadsAtOnce) {
    uint4 lo[kHeadsAtOnce], hi[kHeadsAtOnce];
    auto place = [&](int j) { return (((size_t)(j < Hq ? b * Hq + j : b * Hkv + j - Hq)) * L + t) * D + i; };
#pragma unroll
    for (int x = 0; x < kHeadsAtOnce; ++x) {
      const int j = min(h + x, h1 - 1);
      const T *p = (j < Hq ? q : k) + place(j);
      lo[x] = *reinterpret_cast<const uint4 *>(p);
      hi[x] = *reinterpret_cast<const uint4 *>(p + D / 2);
    }
#pragma unroll
    for (int x = 0; x < kHeadsAtOnce; ++x) {
      if (h + x >= h1) break;
      float u[E], w[E], y[E], z[E];
      unpack<T>(lo[x], u);
      unpack<T>(hi[x], w);
#pragma unroll
      for (int j = 0; j < E; ++j) {
        y[j] = q8_turn(u[j], w[j], c[j], s[j], true);
        z[j] = q8_turn(w[j], u[j], c[j], s[j], false);
      }
      T *p = (h + x < Hq ? q_out : k_out) + place(h + x);
      *reinterpret_cast<uint4 *>(p) = pack<T>(y);
      *reinterpret_cast<uint4 *>(p + D / 2) = pack<T>(z);
    }
  }
}

}  // namespace

hipError_t ag_launch_rotate(ag_ctx *ctx, hipStream_t s, const void *q, const void *k, ag_dtype dt, int B, int Hq, int Hkv, int L,
                            int D, const ag_rope_dev &rope, void *q_out, void *k_out) {
  const int tokens = B * L, E = dt == AG_BF16 ? 8 : 4, H = Hq + Hkv;
  const int64_t wgs = ((int64_t)tokens * (D / 2 / E) + 255) / 256;
  // heads of a thread: as many as leave every CU 8 workgroups, at most 16 (with 1 a CU: 27.2 us for 26.4, fp32 25.4 for 24.1)
  int heads = 16;
  while (heads > 1 && wgs * ((H + heads - 1) / heads) < 8 * ctx->num_cu) heads /= 2;
  const dim3 grid((unsigned)wgs, (H + heads - 1) / heads);
  if (dt == AG_BF16)
    AG_LAUNCH(ag_time_kernel(ctx, AG_K_ROTATE), ag_rotate_kernel<uint16_t>, grid, dim3(256), 0, s, (const uint16_t *)q, (const uint16_t *)k,
              (uint16_t *)q_out, (uint16_t *)k_out, tokens, Hq, Hkv, L, D, heads, rope, ctx->d_err);
  else
    AG_LAUNCH(ag_time_kernel(ctx, AG_K_ROTATE), ag_rotate_kernel<float>, grid, dim3(256), 0, s, (const float *)q, (const float *)k,
              (float *)q_out, (float *)k_out, tokens, Hq, Hkv, L, D, heads, rope, ctx->d_err);
  return hipGetLastError();
}
