// A pool of pages that several caches share: pages counted by the table entries that name them, handed out, shared, given back, moved together.
//
// Everything is decided by the counts and the tables as they stand before a launch, in the order of page, unit and block numbers, so the
// result does not depend on timing; counts change by integer atomics, whose order does not matter.
//   * ag_q8_fork_kernel, one launch: a workgroup per unit copies the tails (2 x 128 D bytes in and out; what bounds a large fork is that
//     copy, 1024 units 10 us, a small one the chain parent -> length -> table -> count, 3.5 us) and counts the entries.
//   * Who gets which page needs the free pages' ranks.  ag_q8_list_kernel lists, for every 4096 pages, those in use and then the free ones, and counts; the
//     second launch finds the chunk of a rank by a search over the counts' prefix sums.  (Taking both from the counts themselves would make
//     one launch read what another one of its workgroups changes.  For small pools there is a launch that does not.)
//   * ag_q8_move_kernel: source i is the i-th page in use behind N, destination i the i-th free page before it, so no page is both.  Bound by memory:
//     5600 pages (184 MB) 29 us.
#include <algorithm>

#include "ag_q8.h"

namespace {

constexpr int kListThreads = 1024;
constexpr int kThreads = 256;
constexpr int kUnitsAWg = kThreads / 64;  // a wave per unit

// Over a workgroup of N waves: exclusive prefix sum and total.  Two barriers.
template <int N> __device__ __forceinline__ int wg_prefix(int x, int &total, int32_t *sums) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  int sum, at = ag_wave_prefix(x, sum);
  __syncthreads();
  if (lane == 0) sums[wave] = sum;
  __syncthreads();
  total = 0;
#pragma unroll
  for (int w = 0; w < N; ++w) {
    if (w < wave) at += sums[w];
    total += sums[w];
  }
  return at;
}

struct blocks {
  int first, end, table;  // blocks that are to have pages; the table's
};
__device__ __forceinline__ blocks wanted(const ag_q8_dev &c, int u, int rows) {
  const int most = c.max_blocks * kQ8Block + kQ8Block - 1, n = max(0, min(c.len[u], most));
  const int end = (int)(((int64_t)n + rows) / kQ8Block);
  return blocks{n / kQ8Block, min(end, c.max_blocks), end};
}

// Workgroups [0, chunks): the chunk's pages listed, those in use first; the others (rows >= 0): the pages that their units want.
__global__ __launch_bounds__(kListThreads) void ag_q8_list_kernel(ag_q8_dev c, const int32_t *page, const int32_t *ref, int chunks, int U, int rows,
                                                                   ag_q8_pool_ws w, int32_t *err) {
  __shared__ int32_t sums[kListThreads / 64];
  const int tid = threadIdx.x, lane = tid & 63;
  if ((int)blockIdx.x >= chunks) {
    const int u = ((int)blockIdx.x - chunks) * (kListThreads / 64) + (tid >> 6);
    if (u >= U) return;
    const blocks b = wanted(c, u, rows);
    int n = 0;
    for (int j = b.first + lane; j < b.end; j += 64) n += (uint32_t)page[(size_t)u * c.max_blocks + j] >= (uint32_t)c.n_pages;
    int total;
    ag_wave_prefix(n, total);
    if (lane == 0) {
      w.need[u] = total;
      if (b.table > c.max_blocks) atomicOr(err, 1);
    }
    return;
  }
  const int chunk = blockIdx.x, first = chunk * kQ8PageChunk, p = first + 4 * tid, here = min(kQ8PageChunk, c.n_pages - first);
  int r[4];
  int n_used = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    r[i] = p + i < c.n_pages ? ref[p + i] : 0;
    n_used += r[i] != 0;
  }
  int total, at = wg_prefix<kListThreads / 64>(n_used, total, sums);
  int32_t *list = w.list + (size_t)first;
#pragma unroll
  for (int i = 0; i < 4; ++i)
    if (p + i < c.n_pages) {
      if (r[i] != 0) list[at++] = p + i;
      else list[total + (4 * tid + i - at)] = p + i;
    }
  if (tid == 0) w.count[chunk] = here - total;
}

// s_pre[i] = free pages before chunk i, i <= chunks.
template <int N> __device__ __forceinline__ void free_before(const int32_t *count, int chunks, int32_t *s_pre, int32_t *sums) {
  int before = 0;
  for (int i0 = 0; i0 < chunks; i0 += 64 * N) {
    const int i = i0 + (int)threadIdx.x;
    int total;
    const int at = wg_prefix<N>(i < chunks ? count[i] : 0, total, sums);
    if (i < chunks) s_pre[i] = before + at;
    before += total;
  }
  if (threadIdx.x == 0) s_pre[chunks] = before;
  __syncthreads();
}
// The chunk that holds element k, of those of which before(i) are ahead of chunk i: the last one with before(i) <= k.
template <typename F> __device__ __forceinline__ int chunk_of(F &&before, int chunks, int k) {
  int lo = 0, hi = chunks - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) / 2;
    if (before(mid) <= k) lo = mid;
    else hi = mid - 1;
  }
  return lo;
}
__device__ __forceinline__ int free_page(const ag_q8_pool_ws &w, const int32_t *s_pre, int chunks, int n_pages, int k) {
  const int i = chunk_of([&](int x) { return s_pre[x]; }, chunks, k), here = min(kQ8PageChunk, n_pages - i * kQ8PageChunk);
  return w.list[(size_t)i * kQ8PageChunk + here - (s_pre[i + 1] - s_pre[i]) + k - s_pre[i]];
}
__device__ __forceinline__ int used_page(const ag_q8_pool_ws &w, const int32_t *s_pre, int chunks, int k) {
  auto before = [&](int x) { return x * kQ8PageChunk - s_pre[x]; };
  const int i = chunk_of(before, chunks, k);
  return w.list[(size_t)i * kQ8PageChunk + k - before(i)];
}

// A wave per unit: the blocks without a page take the free pages from the unit's rank on.
__global__ __launch_bounds__(kThreads) void ag_q8_reserve_kernel(ag_q8_dev c, int32_t *page, int32_t *ref, int chunks, int U, int rows,
                                                                  ag_q8_pool_ws w, int32_t *err) {
  extern __shared__ int32_t s_pre[];  // [chunks + 1]
  __shared__ int32_t sums[kUnitsAWg];
  const int tid = threadIdx.x, lane = tid & 63, u0 = blockIdx.x * kUnitsAWg, u = u0 + (tid >> 6);
  int before = 0, total;
  for (int i = tid; i < u0; i += kThreads) before += w.need[i];
  wg_prefix<kUnitsAWg>(before, total, sums);
  free_before<kUnitsAWg>(w.count, chunks, s_pre, sums);
  if (u >= U) return;
  int rank = total;
  for (int i = u0; i < u; ++i) rank += w.need[i];
  if (w.need[u] == 0) return;
  const int there = s_pre[chunks];
  const blocks b = wanted(c, u, rows);
  bool out = false;
  for (int j0 = b.first; j0 < b.end; j0 += 64) {
    const int j = j0 + lane;
    int32_t *entry = page + (size_t)u * c.max_blocks + j;
    const bool mine = j < b.end && (uint32_t)*entry >= (uint32_t)c.n_pages;
    int n, k = rank + ag_wave_prefix(mine, n);
    if (mine && k < there) {
      const int p = free_page(w, s_pre, chunks, c.n_pages, k);
      *entry = p;
      ref[p] = 1;
    }
    out |= mine && k >= there;
    rank += n;
  }
  if (out) atomicOr(err, 1);
}

// The same in one launch, by one workgroup, for a small pool, units of which a thread takes one each, and few blocks: 500 pages and 32 units 3.1 us
// (in two launches 2.2 + 3.8), 8000 pages and 1024 units 7.2 (3.8 + 4.3, and 2 to 3 between them).  More pages or blocks are better off in two: 24800
// pages took one workgroup 14 us (4.5 + 4.7), 256 units that want 16 blocks each 9.1 (5.2).
constexpr int kSmallPages = 8 * kListThreads, kSmallBlocks = 4;
__global__ __launch_bounds__(kListThreads) void ag_q8_reserve_small_kernel(ag_q8_dev c, int32_t *page, int32_t *ref, int U, int rows, int32_t *err) {
  constexpr int WAVES = kListThreads / 64, N = kSmallPages / kListThreads;
  __shared__ uint16_t s_free[kSmallPages];
  __shared__ int32_t s_count[N * WAVES], sums[WAVES], s_there;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  // this thread's unit: the blocks that want a page
  blocks b{0, 0, 0};
  if (tid < U) b = wanted(c, tid, rows);
  int32_t *entries = page + (size_t)min(tid, U - 1) * c.max_blocks;
  uint32_t missing = 0;  // bit j: block b.first + j
#pragma unroll
  for (int j = 0; j < kSmallBlocks; ++j)
    if (b.first + j < b.end) missing |= (uint32_t)((uint32_t)entries[b.first + j] >= (uint32_t)c.n_pages) << j;
  // the free pages, kListThreads at a time
  uint32_t mine = 0;
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const int p = i * kListThreads + tid;
    if (i * kListThreads < c.n_pages && p < c.n_pages && ref[p] == 0) mine |= 1u << i;
  }
  int32_t n_free[N];
#pragma unroll
  for (int i = 0; i < N; ++i) {
    n_free[i] = __popcll(__ballot(mine >> i & 1));
    if (lane == 0) s_count[i * WAVES + wave] = n_free[i];
  }
  __syncthreads();
  int total, count = tid < N * WAVES ? s_count[tid] : 0;
  const int before = wg_prefix<WAVES>(count, total, sums);
  if (tid < N * WAVES) s_count[tid] = before;
  if (tid == 0) s_there = total;
  int rank_total, rank = wg_prefix<WAVES>(__popc(missing), rank_total, sums);  // (its barriers are s_count's too)
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const uint64_t all = __ballot(mine >> i & 1);
    if (mine >> i & 1) s_free[s_count[i * WAVES + wave] + __popcll(all & ((1ull << lane) - 1))] = (uint16_t)(i * kListThreads + tid);
  }
  __syncthreads();
  bool out = b.table > c.max_blocks;
  for (; missing; missing &= missing - 1, ++rank) {
    if (rank < s_there) {
      const int p = s_free[rank];
      entries[b.first + __builtin_ctz(missing)] = p;
      ref[p] = 1;
    } else {
      out = true;
    }
  }
  if (out) atomicOr(err, 1);
}

template <int D>
__global__ __launch_bounds__(kThreads) void ag_q8_fork_kernel(ag_q8_dev src, int src_B, const int32_t *parent, ag_q8_dev dst, int32_t *page, int Hkv, int32_t *ref) {
  constexpr int N = kQ8Block * D * 2 / 16 / kThreads;  // 16-byte pieces of a tail per thread
  const int u = blockIdx.x, tid = threadIdx.x, b = u / Hkv, from = parent[b];
  const bool some = (uint32_t)from < (uint32_t)src_B;
  const int v = some ? from * Hkv + u % Hkv : 0;
  q8_u32x4 k[N], x[N];
  if (some) {
    const q8_u32x4 *sk = reinterpret_cast<const q8_u32x4 *>(src.k_tail + (size_t)v * kQ8Block * D) + tid;
    const q8_u32x4 *sv = reinterpret_cast<const q8_u32x4 *>(src.v_tail + (size_t)v * kQ8Block * D) + tid;
#pragma unroll
    for (int i = 0; i < N; ++i) k[i] = sk[i * kThreads];
#pragma unroll
    for (int i = 0; i < N; ++i) x[i] = sv[i * kThreads];
  }
  const int most = src.max_blocks * kQ8Block + kQ8Block - 1, n = some ? max(0, min(src.len[v], most)) : 0, full = n / kQ8Block;
  for (int j = tid; j < dst.max_blocks; j += kThreads) {
    int32_t *entry = page + (size_t)u * dst.max_blocks + j;
    const int old = *entry;
    int now = -1;
    if (j < full) {
      now = src.page[(size_t)v * src.max_blocks + j];
      if ((uint32_t)now >= (uint32_t)dst.n_pages) now = -1;
    }
    if (now != old) {
      if ((uint32_t)old < (uint32_t)dst.n_pages) atomicSub(ref + old, 1);
      if (now >= 0) atomicAdd(ref + now, 1);
      *entry = now;
    }
  }
  if (tid == 0) dst.len[u] = n;
  if (!some) return;
  q8_u32x4 *dk = reinterpret_cast<q8_u32x4 *>(dst.k_tail + (size_t)u * kQ8Block * D) + tid;
  q8_u32x4 *dv = reinterpret_cast<q8_u32x4 *>(dst.v_tail + (size_t)u * kQ8Block * D) + tid;
#pragma unroll
  for (int i = 0; i < N; ++i) dk[i * kThreads] = k[i];
#pragma unroll
  for (int i = 0; i < N; ++i) dv[i * kThreads] = x[i];
}

__global__ __launch_bounds__(kThreads) void ag_q8_release_kernel(ag_q8_dev c, int32_t *page, int Hkv, int32_t *ref, const uint8_t *which) {
  const int u = blockIdx.x;
  if (which && which[u / Hkv] == 0) return;
  for (int j = threadIdx.x; j < c.max_blocks; j += kThreads) {
    int32_t *entry = page + (size_t)u * c.max_blocks + j;
    const int p = *entry;
    if ((uint32_t)p < (uint32_t)c.n_pages) atomicSub(ref + p, 1);
    *entry = -1;
  }
  if (threadIdx.x == 0) c.len[u] = 0;
}

// A workgroup copies page p's codes to page `to`.
template <int D> __device__ __forceinline__ void copy_page(const ag_q8_dev &c, size_t p, size_t to) {
  constexpr int P = kQ8Block * D / 16 / kThreads;  // 16-byte pieces of a page per thread
  const int tid = threadIdx.x;
  q8_u32x4 a[P], b[P];
  const q8_u32x4 *pk = reinterpret_cast<const q8_u32x4 *>(c.k + p * kQ8Block * D) + tid, *pv = reinterpret_cast<const q8_u32x4 *>(c.v + p * kQ8Block * D) + tid;
#pragma unroll
  for (int i = 0; i < P; ++i) a[i] = pk[i * kThreads];
#pragma unroll
  for (int i = 0; i < P; ++i) b[i] = pv[i * kThreads];
  q8_u32x4 *tk = reinterpret_cast<q8_u32x4 *>(c.k + to * kQ8Block * D) + tid, *tv = reinterpret_cast<q8_u32x4 *>(c.v + to * kQ8Block * D) + tid;
#pragma unroll
  for (int i = 0; i < P; ++i) tk[i * kThreads] = a[i];
#pragma unroll
  for (int i = 0; i < P; ++i) tv[i * kThreads] = b[i];
}

// Every workgroup takes every n-th of the pages that move, and of the pages whose new number is to be written down.
template <int D>
__global__ __launch_bounds__(kThreads) void ag_q8_move_kernel(ag_q8_dev c, int32_t *ref, int32_t *moved, int32_t *used, int chunks, ag_q8_pool_ws w) {
  extern __shared__ int32_t s_pre[];
  __shared__ int32_t sums[kThreads / 64];
  const int tid = threadIdx.x;
  free_before<kThreads / 64>(w.count, chunks, s_pre, sums);
  const int N = c.n_pages - s_pre[chunks];  // pages in use
  // free pages before N: those of the chunks ahead of N's, and of its own list those below N
  int holes = 0;
  if (N < c.n_pages) {
    const int i = N / kQ8PageChunk, here = min(kQ8PageChunk, c.n_pages - i * kQ8PageChunk), n = s_pre[i + 1] - s_pre[i];
    const int32_t *list = w.list + (size_t)i * kQ8PageChunk + here - n;
    int lo = 0, hi = n;  // the first one that is not below N
    while (lo < hi) {
      const int mid = (lo + hi) / 2;
      if (list[mid] < N) lo = mid + 1;
      else hi = mid;
    }
    holes = s_pre[i] + lo;
  }
  if (blockIdx.x == 0 && tid == 0) used[0] = N;
  for (int64_t x = (int64_t)blockIdx.x * kThreads + tid; x < c.n_pages; x += (int64_t)gridDim.x * kThreads) {
    const int i = (int)x / kQ8PageChunk, at = (int)x % kQ8PageChunk, here = min(kQ8PageChunk, c.n_pages - i * kQ8PageChunk);
    const int p = w.list[x], n_used = here - (s_pre[i + 1] - s_pre[i]);
    if (at >= n_used) {
      moved[p] = -1;
    } else if (p < N) {
      moved[p] = p;
    } else {
      const int k = i * kQ8PageChunk - s_pre[i] + at - (N - holes), to = free_page(w, s_pre, chunks, c.n_pages, k);
      moved[p] = to;
      ref[to] = ref[p];
      ref[p] = 0;
      c.k_scale[to] = c.k_scale[p];
      c.v_scale[to] = c.v_scale[p];
    }
  }
  for (int k = blockIdx.x; k < holes; k += gridDim.x)
    copy_page<D>(c, used_page(w, s_pre, chunks, N - holes + k), free_page(w, s_pre, chunks, c.n_pages, k));
}

// The same in one launch for a small pool: every workgroup finds the pages that move by itself, from counts that nobody writes before all have
// read them: the workgroup that comes last writes the new ones.  500 pages, half in use, 7.5 us (in two launches 11.5), 2000 10.5 (13); 4000 16.5 (14).  More
// workgroups copy faster but arrive one after the other: 512 of them 8.7 us and 14.4.
constexpr int kSmallMove = 2048, kSmallMoveWgs = 64;
template <int D>
__global__ __launch_bounds__(kThreads) void ag_q8_move_small_kernel(ag_q8_dev c, int32_t *ref, int32_t *moved, int32_t *used, int32_t *ticket) {
  constexpr int T = kSmallMove / kThreads, WAVES = kThreads / 64;
  __shared__ uint16_t s_from[kSmallMove / 2], s_to[kSmallMove / 2];
  __shared__ int32_t sums[WAVES], s_last;
  const int tid = threadIdx.x, per = (c.n_pages + kThreads - 1) / kThreads;  // a thread has `per` pages behind each other
  const int p0 = tid * per, p1 = min(c.n_pages, p0 + per);
  uint32_t in_use = 0;
#pragma unroll
  for (int i = 0; i < T; ++i)
    if (p0 + i < p1 && ref[p0 + i] != 0) in_use |= 1u << i;
  int N, holes, at = wg_prefix<WAVES>(__popc(in_use), N, sums);
  const int below = max(0, min(p1, N) - p0);  // pages of the thread before N
  const uint32_t there = p1 > p0 ? (1u << (p1 - p0)) - 1 : 0, ahead = (1u << below) - 1;
  uint32_t to = ~in_use & there & ahead, from = in_use & ~ahead;
  int k_to = wg_prefix<WAVES>(__popc(to), holes, sums), unused, k_from = wg_prefix<WAVES>(__popc(from), unused, sums);
  for (; to; to &= to - 1) s_to[k_to++] = (uint16_t)(p0 + __builtin_ctz(to));
  for (; from; from &= from - 1) s_from[k_from++] = (uint16_t)(p0 + __builtin_ctz(from));
  __syncthreads();
  for (int k = blockIdx.x; k < holes; k += gridDim.x) copy_page<D>(c, s_from[k], s_to[k]);
  if (tid == 0) s_last = __hip_atomic_fetch_add(ticket, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == (int)gridDim.x - 1;
  __syncthreads();
  if (!s_last) return;
  if (tid == 0) {
    ticket[0] = 0;
    used[0] = N;
  }
  for (int i = 0; p0 + i < p1; ++i)
    if (p0 + i < N || !(in_use >> i & 1)) moved[p0 + i] = in_use >> i & 1 ? p0 + i : -1;
  for (int k = tid; k < holes; k += kThreads) {
    const int a = s_from[k], b = s_to[k];
    moved[a] = b;
    ref[b] = ref[a];
    ref[a] = 0;
    c.k_scale[b] = c.k_scale[a];
    c.v_scale[b] = c.v_scale[a];
  }
}

__global__ __launch_bounds__(kThreads) void ag_q8_remap_kernel(int32_t *page, int64_t n, int n_pages, const int32_t *moved) {
  for (int64_t i = (int64_t)blockIdx.x * kThreads + threadIdx.x; i < n; i += (int64_t)gridDim.x * kThreads) {
    const int p = page[i];
    if ((uint32_t)p < (uint32_t)n_pages) page[i] = moved[p];
  }
}

hipError_t launch_list(ag_ctx *ctx, hipStream_t s, const ag_q8_dev &c, const int32_t *page, const int32_t *ref, int U, int rows, const ag_q8_pool_ws &w) {
  const int chunks = ag_q8_page_chunks(c.n_pages), per = kListThreads / 64;
  AG_LAUNCH(ag_time_kernel(ctx, AG_K_Q8_PAGES), ag_q8_list_kernel, dim3(chunks + (U + per - 1) / per), dim3(kListThreads), 0, s, c, page, ref, chunks, U,
            rows, w, ctx->d_err);
  return hipGetLastError();
}

}  // namespace

hipError_t ag_launch_q8_reserve(ag_ctx *ctx, hipStream_t s, int units, const ag_q8_dev &c, int32_t *page, int32_t *ref, int rows, const ag_q8_pool_ws &w) {
  // (len / 64 to (len + rows) / 64 - 1: at most rows / 64 + 1 blocks)
  if (c.n_pages <= kSmallPages && units <= kListThreads && rows / kQ8Block + 1 <= kSmallBlocks) {
    AG_LAUNCH(ag_time_kernel(ctx, AG_K_Q8_PAGES), ag_q8_reserve_small_kernel, dim3(1), dim3(kListThreads), 0, s, c, page, ref, units, rows, ctx->d_err);
    return hipGetLastError();
  }
  const hipError_t e = launch_list(ctx, s, c, page, ref, units, rows, w);
  if (e != hipSuccess) return e;
  const int chunks = ag_q8_page_chunks(c.n_pages);
  AG_LAUNCH(ag_time_kernel(ctx, AG_K_Q8_PAGES), ag_q8_reserve_kernel, dim3((units + kUnitsAWg - 1) / kUnitsAWg), dim3(kThreads), (size_t)(chunks + 1) * 4, s,
            c, page, ref, chunks, units, rows, w, ctx->d_err);
  return hipGetLastError();
}

hipError_t ag_launch_q8_fork(ag_ctx *ctx, hipStream_t s, const ag_q8_dev &src, int src_B, const int32_t *parent, const ag_q8_dev &dst, int32_t *dst_page,
                             int B, int Hkv, int D, int32_t *ref) {
  const dim3 grid(B * Hkv);
  if (D == 128) AG_LAUNCH(ag_time_kernel(ctx, AG_K_Q8_FORK), ag_q8_fork_kernel<128>, grid, dim3(kThreads), 0, s, src, src_B, parent, dst, dst_page, Hkv, ref);
  else AG_LAUNCH(ag_time_kernel(ctx, AG_K_Q8_FORK), ag_q8_fork_kernel<64>, grid, dim3(kThreads), 0, s, src, src_B, parent, dst, dst_page, Hkv, ref);
  return hipGetLastError();
}

hipError_t ag_launch_q8_release(ag_ctx *ctx, hipStream_t s, int B, int Hkv, const ag_q8_dev &c, int32_t *page, int32_t *ref, const uint8_t *which) {
  AG_LAUNCH(ag_time_kernel(ctx, AG_K_Q8_PAGES), ag_q8_release_kernel, dim3(B * Hkv), dim3(kThreads), 0, s, c, page, Hkv, ref, which);
  return hipGetLastError();
}

hipError_t ag_launch_q8_compact_pages(ag_ctx *ctx, hipStream_t s, const ag_q8_dev &c, int D, int32_t *ref, int32_t *moved, int32_t *used,
                                      const ag_q8_pool_ws &w) {
  if (c.n_pages <= kSmallMove) {
    const dim3 wgs(std::max(1, std::min(c.n_pages / 2, kSmallMoveWgs)));
    if (D == 128) AG_LAUNCH(ag_time_kernel(ctx, AG_K_Q8_PAGES), ag_q8_move_small_kernel<128>, wgs, dim3(kThreads), 0, s, c, ref, moved, used, ctx->decode_tickets);
    else AG_LAUNCH(ag_time_kernel(ctx, AG_K_Q8_PAGES), ag_q8_move_small_kernel<64>, wgs, dim3(kThreads), 0, s, c, ref, moved, used, ctx->decode_tickets);
    return hipGetLastError();
  }
  const hipError_t e = launch_list(ctx, s, c, nullptr, ref, 0, 0, w);
  if (e != hipSuccess) return e;
  const int chunks = ag_q8_page_chunks(c.n_pages), grid = std::min(c.n_pages, 8 * ctx->num_cu);
  const size_t lds = (size_t)(chunks + 1) * 4;
  if (D == 128) AG_LAUNCH(ag_time_kernel(ctx, AG_K_Q8_PAGES), ag_q8_move_kernel<128>, dim3(grid), dim3(kThreads), lds, s, c, ref, moved, used, chunks, w);
  else AG_LAUNCH(ag_time_kernel(ctx, AG_K_Q8_PAGES), ag_q8_move_kernel<64>, dim3(grid), dim3(kThreads), lds, s, c, ref, moved, used, chunks, w);
  return hipGetLastError();
}

hipError_t ag_launch_q8_remap(ag_ctx *ctx, hipStream_t s, int units, const ag_q8_dev &c, int32_t *page, const int32_t *moved) {
  const int64_t n = (int64_t)units * c.max_blocks;
  const int grid = (int)std::min<int64_t>((n + kThreads - 1) / kThreads, 8 * ctx->num_cu);
  AG_LAUNCH(ag_time_kernel(ctx, AG_K_Q8_PAGES), ag_q8_remap_kernel, dim3(grid), dim3(kThreads), 0, s, page, n, c.n_pages, moved);
  return hipGetLastError();
}
