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

// Which vector of q (of k, from head Hq on) head j of token t of sequence b is: 64 bits, 2^31 of 16 values are 64 GiB.
__device__ __forceinline__ size_t vector_at(int b, int t, int j, int Hq, int Hkv, int L) {
  return (j < Hq ? (size_t)b * Hq + j : (size_t)b * Hkv + (j - Hq)) * L + t;
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
    auto place = [&](int j) { return vector_at(b, t, j, Hq, Hkv, L) * D + i; };
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

// Every head's vector normalised by its root mean square and turned, y = turn(x r w), in one pass.  Bound by memory as the rotation is: 4096 tokens of
// 64 heads (136 MB) 29.7 us, 4.6 TB/s; one token each of 32 sequences 5.1 us, the launch.
// A vector's pieces are `lanes` (a power of two) neighbouring lanes': the squares of a piece and of its partner are added up in a lane, then
// over the group.  Sums are in 32 bits; where one passes their range (values from 2^60 on) the vector is taken 2^-70 as large.
template <typename T>
__global__ __launch_bounds__(256) void ag_norm_rotate_kernel(const T *q, const T *k, T *q_out, T *k_out, const T *q_weight, const T *k_weight,
                                                             float eps, int tokens, int Hq, int Hkv, int L, int D, int lanes_log, int heads,
                                                             ag_rope_dev rope, int32_t *err) {
  constexpr int E = 16 / sizeof(T);  // values of a piece
  constexpr float kSmall = 8.470329473e-22f;  // 2^-70
  const int lanes = 1 << lanes_log;
  const int64_t id = (int64_t)blockIdx.x * 256 + threadIdx.x;
  const int64_t token = id >> lanes_log;
  const int piece = (int)id & (lanes - 1), i = piece * E;
  const bool there = token < tokens && i < D / 2;  // (the other lanes take part in the sums)
  const int n = there ? (int)token : 0, at_i = there ? i : 0;
  const int b = n / L, t = n - b * L;
  float c[E], s[E];
  if (rope.table) {
    const q8_rows at = q8_rope_rows(rope, n, err);
#pragma unroll
    for (int j = 0; j < E; j += 4) {
      if (rope.quads) {
        const q8_angles e = q8_angles4(rope, at, at_i + j, D);
        c[j] = e.c.x; c[j + 1] = e.c.y; c[j + 2] = e.c.z; c[j + 3] = e.c.w;
        s[j] = e.s.x; s[j + 1] = e.s.y; s[j + 2] = e.s.z; s[j + 3] = e.s.w;
      } else {
#pragma unroll
        for (int x = j; x < j + 4; ++x) {
          const float *row = q8_angle_row(rope, at, at_i + x, D) + at_i + x;
          c[x] = row[0];
          s[x] = row[D / 2];
        }
      }
    }
  }
  const float inv_d = 1.f / (float)D;
  const int h0 = blockIdx.y * heads, h1 = min(h0 + heads, Hq + Hkv);
  for (int h = h0; h < h1; h += kHeadsAtOnce) {
    uint4 lo[kHeadsAtOnce], hi[kHeadsAtOnce];
    auto place = [&](int j) { return vector_at(b, t, j, Hq, Hkv, L) * D + at_i; };
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
      const T *weight = (h + x < Hq ? q_weight : k_weight) + at_i;
      float u[E], w[E], gu[E], gw[E], y[E], z[E];
      unpack<T>(lo[x], u);
      unpack<T>(hi[x], w);
      unpack<T>(*reinterpret_cast<const uint4 *>(weight), gu);
      unpack<T>(*reinterpret_cast<const uint4 *>(weight + D / 2), gw);
      auto squares = [&] {
        float sum = 0.f;
#pragma unroll
        for (int j = 0; j < E; ++j) sum = fmaf(u[j], u[j], fmaf(w[j], w[j], sum));
        if (!there) sum = 0.f;
        for (int o = 1; o < lanes; o <<= 1) sum += __shfl_xor(sum, o, 64);
        return sum * inv_d;
      };
      const float mean = squares();
      float r = 1.f / sqrtf(mean + eps);
      if (__builtin_expect(__any(!(mean < INFINITY)), 0)) {  // (a group's lanes have one sum)
        const float f = mean < INFINITY ? 1.f : kSmall;
#pragma unroll
        for (int j = 0; j < E; ++j) u[j] *= f, w[j] *= f;
        const float small = squares();
        r = mean < INFINITY ? r : 1.f / sqrtf(small + eps * kSmall * kSmall);
      }
#pragma unroll
      for (int j = 0; j < E; ++j) {
#pragma clang fp contract(off)
        const float a = u[j] * r * gu[j], e = w[j] * r * gw[j];
        y[j] = rope.table ? q8_turn(a, e, c[j], s[j], true) : a;
        z[j] = rope.table ? q8_turn(e, a, c[j], s[j], false) : e;
      }
      if (!there) continue;
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

hipError_t ag_launch_norm_rotate(ag_ctx *ctx, hipStream_t s, const void *q, const void *k, ag_dtype dt, int B, int Hq, int Hkv, int L,
                                 int D, const void *q_weight, const void *k_weight, float eps, const ag_rope_dev &rope, void *q_out, void *k_out) {
  const int tokens = B * L, E = dt == AG_BF16 ? 8 : 4, H = Hq + Hkv;
  int lanes_log = 0;
  while ((1 << lanes_log) < D / 2 / E) ++lanes_log;  // at most 64: D <= 512
  const int64_t wgs = (((int64_t)tokens << lanes_log) + 255) / 256;
  int heads = 16;  // as for the rotation
  while (heads > 1 && wgs * ((H + heads - 1) / heads) < 8 * ctx->num_cu) heads /= 2;
  const dim3 grid((unsigned)wgs, (H + heads - 1) / heads);
  if (dt == AG_BF16)
    AG_LAUNCH(ag_time_kernel(ctx, AG_K_NORM_ROTATE), ag_norm_rotate_kernel<uint16_t>, grid, dim3(256), 0, s, (const uint16_t *)q, (const uint16_t *)k,
              (uint16_t *)q_out, (uint16_t *)k_out, (const uint16_t *)q_weight, (const uint16_t *)k_weight, eps, tokens, Hq, Hkv, L, D, lanes_log,
              heads, rope, ctx->d_err);
  else
    AG_LAUNCH(ag_time_kernel(ctx, AG_K_NORM_ROTATE), ag_norm_rotate_kernel<float>, grid, dim3(256), 0, s, (const float *)q, (const float *)k,
              (float *)q_out, (float *)k_out, (const float *)q_weight, (const float *)k_weight, eps, tokens, Hq, Hkv, L, D, lanes_log, heads, rope,
              ctx->d_err);
  return hipGetLastError();
}
