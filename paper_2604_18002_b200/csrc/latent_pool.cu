// ngc_pool_update and ngc_latent_write: the pages of a common pool and the rows of new tokens.
//
// The books (page table, used map, lengths) of one list are the work of one CTA: every step depends on the one before
// (what eviction returns can be handed out again), and all of it is a few reads per sequence and one byte per page of the
// pool.  Warps take sequences for the eviction; sums over sequences and over the used map give every new page its rank,
// and the page of rank r finds its sequence by bisection, so the free pages are never listed.  Only the slot map is as
// long as the tokens: a cluster of CTAs per list shares it, the others wait for the books at the cluster's barrier and
// read the first CTA's sums from its shared memory.  Bound by latency: a chain of dependent reads (lengths -> table row ->
// used map -> table -> slots).
#include <cooperative_groups.h>

#include "latent_pool.cuh"
#include "ptx.cuh"

namespace cg = cooperative_groups;

namespace ngc {
namespace {

constexpr int kThreads = 1024;
constexpr int kWarps = kThreads / 32;
constexpr int kMaxB = 8192;

struct PoolParams {
  int32_t* table;              // [B][G][cap]
  uint8_t* used;               // [G][n_pages]
  int32_t* lens;               // [B][G]
  const int32_t* kept;         // [B][G][k_max] or null
  const int32_t* budget;
  const int32_t* n_new;
  int32_t* slots;              // [G][n_slots]
  int32_t* first;              // [B+1]
  int32_t* dev_status;
  int B, G, cap, n_pages, page, page_shift, k_max, n_slots;
};

// Inclusive sum over the CTA's threads; `total` gets the sum of all.  Two barriers.
__device__ __forceinline__ int block_scan(int v, int* warp_sums, int& total) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int u = __shfl_up_sync(0xffffffffu, v, o);
    if (lane >= o) v += u;
  }
  if (lane == 31) warp_sums[warp] = v;
  __syncthreads();
  int w = warp_sums[lane];
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int u = __shfl_up_sync(0xffffffffu, w, o);
    if (lane >= o) w += u;
  }
  total = __shfl_sync(0xffffffffu, w, 31);
  const int before = __shfl_sync(0xffffffffu, w, (warp + 31) & 31);
  __syncthreads();
  return v + (warp > 0 ? before : 0);
}

// Last b with sum[b] <= x, for 0 <= x < sum[B] (sequences without a share never are the answer).
__device__ __forceinline__ int find_seq(const int* sum, int B, int x) {
  int lo = 0, hi = B;                                  // sum[lo] <= x < sum[hi]
  while (hi - lo > 1) {
    const int m = (lo + hi) >> 1;
    if (sum[m] <= x) lo = m; else hi = m;
  }
  return lo;
}

// The used map of one list, 16 pages per call: bit i of the answer is set where page at + i is free.
__device__ __forceinline__ uint32_t free_mask(const uint8_t* used, int at, int n_pages, bool wide) {
  uint32_t m = 0;
  if (wide && at + 16 <= n_pages) {
    const uint4 v = *reinterpret_cast<const uint4*>(used + at);
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 16; ++i) m |= ((w[i >> 2] >> (8 * (i & 3))) & 0xffu) == 0 ? 1u << i : 0u;
  } else {
    for (int i = 0; i < 16 && at + i < n_pages; ++i) m |= used[at + i] == 0 ? 1u << i : 0u;
  }
  return m;
}

// What sequence b keeps, gives back and needs; one warp.  Returns to lane 0 the length it goes on from (-1: it does not
// grow), and the pages it needs.
__device__ __forceinline__ void settle_sequence(const PoolParams& p, int gi, int b, int first_token, int& len_out, int& need_out, int& have_out) {
  const int lane = threadIdx.x & 31;
  const int64_t list = (int64_t)b * p.G + gi;
  int32_t* row = p.table + list * p.cap;
  uint8_t* used = p.used + (int64_t)gi * p.n_pages;
  int len = p.lens[list];
  const int n_new = p.n_new[b];
  const int budget = p.kept ? p.budget[b] : -1;
  len_out = -1;
  need_out = 0;
  have_out = 0;
  if (len < 0 || len > p.cap * p.page || n_new < -1 || budget < -1 || budget > p.k_max) {
    if (lane == 0) set_dev_status(p.dev_status, NGC_DEV_BAD_COUNTS);
    return;
  }
  int have = (len + p.page - 1) >> p.page_shift;
  const bool evict = budget >= 0, leave = n_new < 0;
  bool bad_page = false, bad_kept = budget > have;
  const int32_t* kept = p.kept + (evict ? list * p.k_max : 0);
  if (evict || leave)                                  // (growth alone needs nothing of the old entries but the last page's, below)
    for (int j = lane; j < have; j += 32) bad_page = bad_page || (uint32_t)row[j] >= (uint32_t)p.n_pages;
  if (evict && !bad_kept)
    for (int j = lane; j < budget; j += 32) {
      const int u = kept[j], prev = j > 0 ? kept[j - 1] : -1;
      bad_kept = bad_kept || u <= prev || u >= have;
    }
  if (__any_sync(0xffffffffu, bad_page || bad_kept)) {
    bad_page = __any_sync(0xffffffffu, bad_page);
    if (lane == 0) set_dev_status(p.dev_status, bad_page ? NGC_DEV_BAD_PAGE : NGC_DEV_BAD_KEPT);
    return;
  }
  if (evict || leave) {
    for (int j = lane; j < have; j += 32) used[row[j]] = 0;
    __syncwarp();
    if (leave) {
      for (int j = lane; j < have; j += 32) row[j] = -1;
      len = have = 0;
    } else {
      // in place: entry j comes from kept[j] >= j, and a step of 32 entries reads its sources before it writes
      const int last = budget > 0 ? kept[budget - 1] : -1;
      for (int j0 = 0; j0 < budget; j0 += 32) {
        const int j = j0 + lane;
        const int pg = j < budget ? row[kept[j]] : 0;
        __syncwarp();
        if (j < budget) { row[j] = pg; used[pg] = 1; }
        __syncwarp();
      }
      for (int j = budget + lane; j < have; j += 32) row[j] = -1;
      len = budget * p.page - (last == have - 1 ? have * p.page - len : 0);
      if (budget == 0) len = 0;
      have = budget;
    }
    if (lane == 0) p.lens[list] = len;
  }
  const int grow = max(n_new, 0);
  if (grow > p.n_slots - first_token) {
    if (lane == 0) set_dev_status(p.dev_status, NGC_DEV_BAD_COUNTS);
    return;
  }
  if (grow > p.cap * p.page - len) {
    if (lane == 0) set_dev_status(p.dev_status, NGC_DEV_STRIP_FULL);
    return;
  }
  // the tokens that still fit the last page go where its entry says
  if (grow > 0 && (len & (p.page - 1)) != 0 && (uint32_t)row[have - 1] >= (uint32_t)p.n_pages) {
    if (lane == 0) set_dev_status(p.dev_status, NGC_DEV_BAD_PAGE);
    return;
  }
  len_out = len;
  have_out = have;
  need_out = ((len + grow + p.page - 1) >> p.page_shift) - have;
}

__global__ void __launch_bounds__(kThreads) pool_update_kernel(PoolParams p) {
  extern __shared__ int sh[];
  __shared__ int warp_sums[32];
  int* first = sh;                                     // [B+1] new tokens of the sequences before
  int* need = first + p.B + 1;                         // [B+1] pages ...
  int* from = need + p.B + 1;                          // [B] length a sequence grows from, -1: it does not
  cg::cluster_group cluster = cg::this_cluster();
  const int rank = (int)cluster.block_rank(), n_ranks = (int)cluster.num_blocks();
  const int gi = blockIdx.y;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;

  ptx::grid_dep_wait();
  // new tokens of the sequences before, failing ones included: the same in every list
  int run = 0;
  for (int b0 = 0; b0 < p.B; b0 += kThreads) {
    const int b = b0 + tid;
    const int n = b < p.B ? max(p.n_new[b], 0) : 0;
    int total;
    const int incl = block_scan(n, warp_sums, total);
    if (b < p.B) first[b + 1] = run + incl;
    run += total;
  }
  if (tid == 0) first[0] = 0;
  __syncthreads();
  if (gi == 0 && rank == 0)
    for (int b = tid; b <= p.B; b += kThreads) p.first[b] = first[b];

  if (rank == 0) {
    uint8_t* used = p.used + (int64_t)gi * p.n_pages;
    for (int b = warp; b < p.B; b += kWarps) {
      int len, n, have;
      settle_sequence(p, gi, b, first[b], len, n, have);
      if (lane == 0) { from[b] = len; need[b + 1] = n; }
    }
    __syncthreads();
    run = 0;
    for (int b0 = 0; b0 < p.B; b0 += kThreads) {
      const int b = b0 + tid;
      const int n = b < p.B ? need[b + 1] : 0;
      int total;
      const int incl = block_scan(n, warp_sums, total);
      if (b < p.B) need[b + 1] = run + incl;
      run += total;
    }
    if (tid == 0) need[0] = 0;
    const int wanted = run;
    const bool wide = ((uintptr_t)used & 15) == 0;
    __syncthreads();
    // how many pages are free; sequences beyond the last that fits do not grow
    int limit = wanted;
    if (wanted > 0) {
      int mine = 0, n_free;
      for (int at = 16 * tid; at < p.n_pages; at += 16 * kThreads) mine += __popc(free_mask(used, at, p.n_pages, wide));
      block_scan(mine, warp_sums, n_free);
      if (n_free < wanted) {
        int best = 0;
        for (int b = tid; b < p.B; b += kThreads) {
          if (need[b + 1] <= n_free) best = max(best, need[b + 1]);
          else if (need[b + 1] > need[b]) { from[b] = -1; set_dev_status(p.dev_status, NGC_DEV_POOL_FULL); }
        }
        if (tid == 0) warp_sums[0] = 0;
        __syncthreads();
        atomicMax(&warp_sums[0], best);
        __syncthreads();
        limit = warp_sums[0];
        __syncthreads();
      }
    }
    run = 0;
    for (int at0 = 0; run < limit && at0 < p.n_pages; at0 += 16 * kThreads) {
      const int at = at0 + 16 * tid;
      uint32_t m = at < p.n_pages ? free_mask(used, at, p.n_pages, wide) : 0u;
      int total;
      const int n = __popc(m);
      int r = run + block_scan(n, warp_sums, total) - n;
      for (; m != 0 && r < limit; m &= m - 1, ++r) {
        const int pg = at + __ffs(m) - 1;
        const int b = find_seq(need, p.B, r);
        const int entry = ((from[b] + p.page - 1) >> p.page_shift) + r - need[b];
        if (NGC_IN_BOUNDS(p.dev_status, from[b] >= 0 && entry >= 0 && entry < p.cap)) {
          p.table[((int64_t)b * p.G + gi) * p.cap + entry] = pg;
          used[pg] = 1;
        }
      }
      run += total;
    }
    for (int b = tid; b < p.B; b += kThreads)
      if (from[b] >= 0 && first[b + 1] > first[b]) p.lens[(int64_t)b * p.G + gi] = from[b] + first[b + 1] - first[b];
  }
  cluster.sync();                                      // the books are done, and visible to the whole cluster
  if (rank != 0) {
    const int* far = cluster.map_shared_rank(from, 0);
    for (int b = tid; b < p.B; b += kThreads) from[b] = far[b];
  }
  __syncthreads();
  const int total = min(first[p.B], p.n_slots);
  int32_t* slots = p.slots + (int64_t)gi * p.n_slots;
  for (int i = rank * kThreads + tid; i < p.n_slots; i += n_ranks * kThreads) {
    int slot = -1;
    if (i < total) {
      const int b = find_seq(first, p.B, i);
      if (from[b] >= 0) {
        const int pos = from[b] + i - first[b];
        if (NGC_IN_BOUNDS(p.dev_status, (pos >> p.page_shift) < p.cap))
          slot = (p.table[((int64_t)b * p.G + gi) * p.cap + (pos >> p.page_shift)] << p.page_shift) + (pos & (p.page - 1));
      }
    }
    slots[i] = slot;
  }
  cluster.sync();                                      // the first CTA's shared memory stays until all have read it
}

// One warp per row: a row of 512 + 64 channels is 72 pieces of 16 bytes.  Bound by HBM.
__global__ void __launch_bounds__(256) latent_write_kernel(uint4* rows, const int32_t* slots, const uint4* latent, const uint4* rope, int n_slots,
                                                           int lists, int lat16, int rope16, int layer_begin, int64_t rows_per_layer,
                                                           int32_t* dev_status) {
  const int lane = threadIdx.x & 31;
  const int l = layer_begin + blockIdx.y;
  const int gi = list_of(lists, l, 0, 1);
  ptx::grid_dep_wait();
  for (int64_t i = (int64_t)blockIdx.x * 8 + (threadIdx.x >> 5); i < n_slots; i += (int64_t)gridDim.x * 8) {
    const int slot = slots[(int64_t)gi * n_slots + i];
    if (slot < 0 || slot >= rows_per_layer) {
      if (slot != -1 && lane == 0) set_dev_status(dev_status, NGC_DEV_BAD_SLOT);
      continue;
    }
    uint4* dst = rows + ((int64_t)l * rows_per_layer + slot) * (lat16 + rope16);
    const uint4* a = latent + ((int64_t)l * n_slots + i) * lat16;
    const uint4* r = rope + ((int64_t)l * n_slots + i) * rope16;
    for (int c = lane; c < lat16 + rope16; c += 32) dst[c] = c < lat16 ? a[c] : r[c - lat16];
  }
}

}  // namespace
}  // namespace ngc

extern "C" int ngc_pool_update(ngc_latent_pool* c, const int32_t* kept_sorted, const int32_t* budget, int k_max, const int32_t* n_new,
                               int32_t* slots, int n_slots, int32_t* first, int32_t* dev_status, ngc_stream stream) {
  using namespace ngc;
  NGC_API_RANGE("ngc_pool_update");
  if (!valid_latent_pool(c) || !n_new || !slots || n_slots < 1 || !first || (kept_sorted == nullptr) != (budget == nullptr) ||
      (kept_sorted && k_max < 1))
    return NGC_ERR_INVALID_ARG;
  if (c->B > kMaxB) return NGC_ERR_UNSUPPORTED;
  PoolParams p;
  p.table = c->page_table; p.used = c->page_used; p.lens = c->lens;
  p.kept = kept_sorted; p.budget = budget; p.n_new = n_new; p.slots = slots; p.first = first; p.dev_status = dev_status;
  p.B = c->B; p.G = lists_G(c->lists, c->L, 1); p.cap = c->pages_cap; p.n_pages = c->n_pages;
  p.page = c->page; p.page_shift = c->page == 32 ? 5 : 6; p.k_max = kept_sorted ? k_max : 0; p.n_slots = n_slots;
  if (p.G > 65535) return NGC_ERR_UNSUPPORTED;
  static PerDeviceOnce once;
  const int rc = once.run([] {
    return cudaFuncSetAttribute(pool_update_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (3 * kMaxB + 2) * 4);
  });
  if (rc != NGC_OK) return rc;
  unsigned cluster = 1;
  while (cluster < 8 && n_slots > (int)cluster * 4 * kThreads) cluster *= 2;
  NGC_CUDA_TRY(launch_pdl_cluster(pool_update_kernel, dim3(cluster, p.G), dim3(kThreads), cluster, (3 * (size_t)p.B + 2) * 4, stream, p));
  return launch_status();
}

extern "C" int ngc_latent_write(ngc_latent_pool* c, const int32_t* slots, int n_slots, const void* latent, const void* rope,
                                int layer_begin, int layer_end, int32_t* dev_status, ngc_stream stream) {
  using namespace ngc;
  NGC_API_RANGE("ngc_latent_write");
  if (!valid_latent_pool(c) || !slots || n_slots < 1 || !latent || !rope || layer_begin < 0 || layer_begin >= layer_end || layer_end > c->L ||
      !aligned16(c->rows) || !aligned16(latent) || !aligned16(rope))
    return NGC_ERR_INVALID_ARG;
  if (c->dtype != NGC_BF16 || !built_latent_dims(c->d_latent, c->d_rope) || layer_end - layer_begin > 65535) return NGC_ERR_UNSUPPORTED;
  const int64_t blocks = ((int64_t)n_slots + 7) / 8;
  const dim3 grid((unsigned)(blocks < 148 * 8 ? blocks : 148 * 8), layer_end - layer_begin);
  NGC_CUDA_TRY(launch_pdl(latent_write_kernel, grid, dim3(256), 0, stream, (uint4*)c->rows, slots, (const uint4*)latent, (const uint4*)rope,
                          n_slots, c->lists, c->d_latent / 8, c->d_rope / 8, layer_begin, (int64_t)c->n_pages * c->page, dev_status));
  return launch_status();
}
