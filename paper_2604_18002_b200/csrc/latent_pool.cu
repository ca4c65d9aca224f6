// ngc_pool_update and ngc_latent_write: the pages of a common pool and the rows of new tokens.
//
// The books (page table, used map, lengths) of one list are the work of one cluster of CTAs: every step depends on the one
// before (what eviction returns can be handed out again), and all of it is a few reads per sequence and one byte per page of the
// pool.  Sequences are dealt out to the threads of the cluster, those that evict or leave to its warps; what they find lies in
// the first CTA's shared memory.  There sums over sequences and over the map give every new page its rank, and the page of rank r
// finds its sequence by bisection.  The slot map is shared by the cluster again, or, for many tokens, a kernel of its own.
// Bound by latency, a chain of dependent reads (lengths -> table row -> map -> table -> slots) and the barriers between them, and
// by one SM's instructions where all sequences evict: 256 threads per CTA, because barriers of 1024 took longer than the work (64
// growing sequences of one list: 10 -> 8 us), and up to eight CTAs per list (a round of 64 sequences on 28 lists: 20 -> 17 us; 256
// prompts, 281 thousand tokens on 28 lists: 73 -> 19 us and 21 for the slots' kernel, which writes 31 MB at 1.5 TB/s).
#include <cooperative_groups.h>

#include "latent_pool.cuh"
#include "ptx.cuh"

namespace cg = cooperative_groups;

namespace ngc {
namespace {

constexpr int kThreads = 256;
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
  int split;                   // the slots are left to a kernel of their own
};

// Inclusive sum over the CTA's threads; `total` gets the sum of all.  Two barriers.  Sums stop at kMost, so counts that are no
// counts cannot wrap around and pass for small ones: what lies behind them has no slot.
constexpr int kMost = 0x3fffffff;
__device__ __forceinline__ int add(int a, int b) { return min(a + b, kMost); }                 // of 0 .. kMost
__device__ __forceinline__ int block_scan(int v, int* warp_sums, int& total) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int u = __shfl_up_sync(0xffffffffu, v, o);
    if (lane >= o) v = add(v, u);
  }
  if (lane == 31) warp_sums[warp] = v;
  __syncthreads();
  int before = 0;
  total = 0;
#pragma unroll
  for (int w = 0; w < kWarps; ++w) {
    const int u = warp_sums[w];
    before = add(before, w < warp ? u : 0);
    total = add(total, u);
  }
  __syncthreads();
  return add(v, before);
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

// What a sequence goes on from: the length it grows from (-1: it does not grow), the pages it needs.
struct Settled { int len, need; };

// The part that both ways share: may the sequence grow from `len` tokens?  `last_page`: the entry of its last page, where that has room.
__device__ __forceinline__ Settled settle_growth(const PoolParams& p, int len, int n_new, int last_page) {
  const int grow = max(n_new, 0), have = (len + p.page - 1) >> p.page_shift;
  if (grow > p.cap * p.page - len) {
    set_dev_status(p.dev_status, NGC_DEV_STRIP_FULL);
    return {-1, 0};
  }
  if (grow > 0 && (len & (p.page - 1)) != 0 && (uint32_t)last_page >= (uint32_t)p.n_pages) {
    set_dev_status(p.dev_status, NGC_DEV_BAD_PAGE);
    return {-1, 0};
  }
  return {len, ((len + grow + p.page - 1) >> p.page_shift) - have};
}

// A sequence that evicts or leaves; one warp.  `rows` holds the table row of up to kRowMax pages while it is rewritten.
constexpr int kRowMax = 512;
__device__ Settled settle_eviction(const PoolParams& p, int gi, int b, int* rows, uint8_t* used) {
  const int lane = threadIdx.x & 31;
  const int64_t list = (int64_t)b * p.G + gi;
  int32_t* row = p.table + list * p.cap;
  const int len = p.lens[list], n_new = p.n_new[b], budget = p.kept ? p.budget[b] : -1;
  const int have = (len + p.page - 1) >> p.page_shift, keep = max(budget, 0);
  const int32_t* kept = p.kept + (budget > 0 ? list * p.k_max : 0);
  bool bad_page = false, bad_kept = keep > have;
  const bool small = have <= kRowMax;
  for (int j = lane; j < have; j += 32) {
    const int pg = row[j];
    bad_page = bad_page || (uint32_t)pg >= (uint32_t)p.n_pages;
    if (small) rows[j] = pg;
  }
  if (!bad_kept)
    for (int j = lane; j < keep; j += 32) {
      const int u = kept[j], prev = j > 0 ? kept[j - 1] : -1;
      bad_kept = bad_kept || u <= prev || u >= have;
    }
  bad_page = __any_sync(0xffffffffu, bad_page);
  if (__any_sync(0xffffffffu, bad_kept) || bad_page) {
    if (lane == 0) set_dev_status(p.dev_status, bad_page ? NGC_DEV_BAD_PAGE : NGC_DEV_BAD_KEPT);
    return {-1, 0};
  }
  const int stay = n_new < 0 ? 0 : keep;                 // pages that stay
  const int last_unit = stay > 0 ? kept[stay - 1] : -1;
  int last_page = -1;
  if (small) {
    for (int j = lane; j < have; j += 32) used[rows[j]] = 0;
    __syncwarp();
    for (int j = lane; j < stay; j += 32) {
      const int pg = rows[kept[j]];
      row[j] = pg;
      used[pg] = 1;
    }
    if (stay > 0) last_page = rows[last_unit];
    __syncwarp();
  } else {
    for (int j = lane; j < have; j += 32) used[row[j]] = 0;
    if (stay > 0) last_page = row[last_unit];
    __syncwarp();
    // in place: entry j comes from kept[j] >= j, and a step of 32 entries reads its sources before it writes
    for (int j0 = 0; j0 < stay; j0 += 32) {
      const int j = j0 + lane;
      const int pg = j < stay ? row[kept[j]] : 0;
      __syncwarp();
      if (j < stay) { row[j] = pg; used[pg] = 1; }
      __syncwarp();
    }
  }
  for (int j = stay + lane; j < have; j += 32) row[j] = -1;
  const int left = stay == 0 ? 0 : stay * p.page - (last_unit == have - 1 ? have * p.page - len : 0);
  Settled s = {-1, 0};
  if (lane == 0) {
    p.lens[list] = left;
    s = settle_growth(p, left, n_new, last_page);
  }
  return s;
}

// Who grows where pages are short: in order of sequences each that fits beside those before it, so that one too large does not keep
// the pages from the others.  need[b + 1] are the sums of the pages wanted, and become those of the pages granted.  One warp, 32
// sequences at a time: what is more than all that is left is refused at once, then the first of the others that does not fit, until all do.
__device__ void grant_growth(const PoolParams& p, int* need, int* from, int n_free) {
  const int lane = threadIdx.x & 31;
  int wanted = 0, granted = 0;                         // of the sequences before these 32
  for (int b0 = 0; b0 < p.B; b0 += 32) {
    const int b = b0 + lane, sum = need[min(b, p.B - 1) + 1];
    int before = __shfl_up_sync(0xffffffffu, sum, 1);
    if (lane == 0) before = wanted;
    wanted = __shfl_sync(0xffffffffu, sum, 31);
    const int mine = b < p.B ? sum - before : 0;
    bool refused = mine > n_free - granted;
    for (;;) {
      int incl = refused ? 0 : mine;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) { const int v = __shfl_up_sync(0xffffffffu, incl, o); if (lane >= o) incl += v; }
      const uint32_t over = __ballot_sync(0xffffffffu, !refused && mine > 0 && incl > n_free - granted);
      if (over == 0) {
        if (b < p.B) need[b + 1] = granted + incl;
        granted += __shfl_sync(0xffffffffu, incl, 31);
        break;
      }
      const int first = __ffs(over) - 1, left = n_free - granted - __shfl_sync(0xffffffffu, incl - mine, first);
      refused = refused || (lane >= first && mine > left);
    }
    if (refused) { from[b] = -1; set_dev_status(p.dev_status, NGC_DEV_POOL_FULL); }
  }
}

// Slot of position pos (-1: none) of sequence b.
__device__ __forceinline__ int slot_of(const PoolParams& p, int gi, int b, int pos) {
  if (pos < 0 || !NGC_IN_BOUNDS(p.dev_status, (pos >> p.page_shift) < p.cap)) return -1;
  return (p.table[((int64_t)b * p.G + gi) * p.cap + (pos >> p.page_shift)] << p.page_shift) + (pos & (p.page - 1));
}

__global__ void __launch_bounds__(kThreads) pool_update_kernel(PoolParams p) {
  extern __shared__ int sh[];
  __shared__ int warp_sums[kWarps];
  __shared__ int rows[kWarps][kRowMax];
  __shared__ uint16_t list[16 * kThreads];
  __shared__ int n_waiting;
  int* first = sh;                                     // [B+1] new tokens of the sequences before
  int* need = first + p.B + 1;                         // [B+1] pages ...
  int* from = need + p.B + 1;                          // [B] length a sequence grows from, -1: it does not
  int* waiting = from + p.B;                           // [B / ranks] sequences of this CTA that evict or leave
  cg::cluster_group cluster = cg::this_cluster();
  const int rank = (int)cluster.block_rank(), n_ranks = (int)cluster.num_blocks();
  const int gi = blockIdx.y;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  uint8_t* const used = p.used + (int64_t)gi * p.n_pages;
  const bool wide = ((uintptr_t)used & 15) == 0;

  ptx::grid_dep_launch();
  ptx::grid_dep_wait();
  if (tid == 0) n_waiting = 0;
  // new tokens of the sequences before, failing ones included: the same in every list
  int run = 0;
  for (int b0 = 0; b0 < p.B; b0 += kThreads) {
    const int b = b0 + tid;
    const int n = b < p.B ? min(max(p.n_new[b], 0), kMost) : 0;
    int total;
    const int incl = block_scan(n, warp_sums, total);
    if (b < p.B) first[b + 1] = add(run, incl);
    run = add(run, total);
  }
  if (tid == 0) first[0] = 0;
  if (n_ranks > 1) cluster.sync(); else __syncthreads();               // (all CTAs have begun: the first's shared memory is there)
  int* const need0 = n_ranks > 1 ? cluster.map_shared_rank(need, 0) : need;
  int* const from0 = n_ranks > 1 ? cluster.map_shared_rank(from, 0) : from;
  if (gi == 0 && rank == 0)
    for (int b = tid; b <= p.B; b += kThreads) p.first[b] = first[b];
  // sequences that only grow, a thread each; the others are left to the warps
  for (int b = rank + n_ranks * tid; b < p.B; b += n_ranks * kThreads) {
    const int64_t list = (int64_t)b * p.G + gi;
    const int n_new = p.n_new[b], len = p.lens[list], budget = p.kept ? p.budget[b] : -1;
    Settled s = {-1, 0};
    // (new tokens without slots count as no counts, before anything of the sequence is changed)
    if (len < 0 || len > p.cap * p.page || n_new < -1 || n_new > max(p.n_slots - first[b], 0) || budget < -1 || budget > p.k_max) {
      set_dev_status(p.dev_status, NGC_DEV_BAD_COUNTS);
    } else if (budget >= 0 || n_new < 0) {
      waiting[atomicAdd(&n_waiting, 1)] = b;
      continue;
    } else {
      const int have = (len + p.page - 1) >> p.page_shift;
      const int last_page = n_new > 0 && (len & (p.page - 1)) != 0 ? p.table[list * p.cap + have - 1] : 0;
      s = settle_growth(p, len, n_new, last_page);
    }
    from0[b] = s.len;
    need0[b + 1] = s.need;
  }
  __syncthreads();
  for (int i = warp; i < n_waiting; i += kWarps) {
    const int b = waiting[i];
    const Settled s = settle_eviction(p, gi, b, rows[warp], used);
    if (lane == 0) { from0[b] = s.len; need0[b + 1] = s.need; }
  }
  if (n_ranks > 1) cluster.sync(); else __syncthreads();
  if (rank == 0) {
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
    __syncthreads();
    if (wanted > 0) {
      // how many pages are free; where they are too few, not all sequences grow
      int limit = wanted, here = 0, n_free;
      uint32_t m = 0;                                  // of this thread's last 16 pages: all it has, in a pool of up to 4096
      for (int at = 16 * tid; at < p.n_pages; at += 16 * kThreads) here += __popc(m = free_mask(used, at, p.n_pages, wide));
      block_scan(here, warp_sums, n_free);
      if (n_free < wanted) {
        if (warp == 0) grant_growth(p, need, from, n_free);
        __syncthreads();
        limit = need[p.B];
      }
      run = 0;
      for (int at0 = 0; run < limit && at0 < p.n_pages; at0 += 16 * kThreads) {
        const int at = at0 + 16 * tid;
        if (p.n_pages > 16 * kThreads) m = at < p.n_pages ? free_mask(used, at, p.n_pages, wide) : 0u;
        int total, rk = block_scan(__popc(m), warp_sums, total) - __popc(m);
        for (; m != 0; m &= m - 1, ++rk) list[rk] = (uint16_t)(16 * tid + __ffs(m) - 1);      // the free pages of this step, in order
        __syncthreads();
        for (int k = tid; k < min(total, limit - run); k += kThreads) {
          const int pg = at0 + list[k], b = find_seq(need, p.B, run + k);
          const int entry = ((from[b] + p.page - 1) >> p.page_shift) + run + k - need[b];
          if (NGC_IN_BOUNDS(p.dev_status, from[b] >= 0 && entry >= 0 && entry < p.cap)) {
            p.table[((int64_t)b * p.G + gi) * p.cap + entry] = pg;
            used[pg] = 1;
          }
        }
        run += total;
        __syncthreads();
      }
    }
    for (int b = tid; b < p.B; b += kThreads)
      if (from[b] >= 0 && first[b + 1] > first[b]) p.lens[(int64_t)b * p.G + gi] = from[b] + first[b + 1] - first[b];
  }
  if (n_ranks > 1) {
    cluster.sync();                                    // the books are done, and visible to the whole cluster
    if (rank != 0)
      for (int b = tid; b < p.B; b += kThreads) from[b] = from0[b];
    cluster.sync();                                    // (the first CTA's shared memory stays until all have read it)
  }
  int32_t* slots = p.slots + (int64_t)gi * p.n_slots;
  if (p.split) {                                       // many: only each sequence's first, for the second kernel
    for (int b = rank * kThreads + tid; b < p.B; b += n_ranks * kThreads)
      if (first[b + 1] > first[b] && first[b] < p.n_slots) slots[first[b]] = slot_of(p, gi, b, from[b]);
    return;
  }
  for (int i = rank * kThreads + tid; i < p.n_slots; i += n_ranks * kThreads) {
    int slot = -1;
    if (i < first[p.B]) {
      const int b = find_seq(first, p.B, i);
      slot = slot_of(p, gi, b, from[b] < 0 ? -1 : from[b] + i - first[b]);
    }
    slots[i] = slot;
  }
}

// The slots of many tokens: a warp takes kRun tokens, looks for the first one's sequence and goes on from there.  The first token of
// every sequence has its slot already, -1 if the sequence did not grow.  Bound by latency, a chain of reads per warp (numbers of the
// tokens, first slot, length, table entry): four tokens per lane in one store took 23 us instead of 21, longer runs 25 to 27.
constexpr int kRun = 512;
__global__ void __launch_bounds__(kThreads) pool_slots_kernel(PoolParams p) {
  extern __shared__ int first[];
  ptx::grid_dep_launch();
  ptx::grid_dep_wait();
  const int gi = blockIdx.y, lane = threadIdx.x & 31;
  for (int b = threadIdx.x; b <= p.B; b += kThreads) first[b] = p.first[b];
  __syncthreads();
  int32_t* slots = p.slots + (int64_t)gi * p.n_slots;
  const int total = min(first[p.B], p.n_slots), mask = p.page - 1;
  const int64_t base = ((int64_t)blockIdx.x * kWarps + (threadIdx.x >> 5)) * kRun;
  if (base >= p.n_slots) return;
  // (what belongs to the sequence is kept from token to token)
  int b = base < total ? find_seq(first, p.B, (int)base) : 0, end = first[b], start = 0;
  if (base < total) --b;                                 // (the first token takes the step to its sequence)
  bool grew = false;
  const int32_t* row = p.table;
  int low[kRun / 32], entry[kRun / 32];                  // place in the page, page (-1: no slot)
#pragma unroll
  for (int k = 0; k < kRun / 32; ++k) {
    const int64_t i = base + 32 * k + lane;
    low[k] = 0;
    entry[k] = -1;
    if (i < total) {
      if ((int)i >= end) {
        do end = first[++b + 1]; while ((int)i >= end);
        const int64_t list = (int64_t)b * p.G + gi;
        grew = slots[first[b]] >= 0;
        start = p.lens[list] - end;
        row = p.table + list * p.cap;
      }
      const int pos = start + (int)i;
      low[k] = pos & mask;
      if (grew && NGC_IN_BOUNDS(p.dev_status, (pos >> p.page_shift) < p.cap)) entry[k] = row[pos >> p.page_shift];
    }
  }
#pragma unroll
  for (int k = 0; k < kRun / 32; ++k) {
    const int64_t i = base + 32 * k + lane;
    if (i < p.n_slots) slots[i] = entry[k] < 0 ? -1 : (entry[k] << p.page_shift) + low[k];
  }
}

// One warp per row: a row of 512 + 64 channels is 72 pieces of 16 bytes.  Bound by HBM: 32 thousand rows on 8 layers, 592 MB in and out, in
// 100 us (5.9 TB/s); 64 rows take 4.5 us, a launch and two dependent reads.
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
  if (c->B > kMaxB || n_slots > kMost) return NGC_ERR_UNSUPPORTED;
  PoolParams p;
  p.table = c->page_table; p.used = c->page_used; p.lens = c->lens;
  p.kept = kept_sorted; p.budget = budget; p.n_new = n_new; p.slots = slots; p.first = first; p.dev_status = dev_status;
  p.B = c->B; p.G = lists_G(c->lists, c->L, 1); p.cap = c->pages_cap; p.n_pages = c->n_pages;
  p.page = c->page; p.page_shift = c->page == 32 ? 5 : 6; p.k_max = kept_sorted ? k_max : 0; p.n_slots = n_slots;
  if (p.G > 65535) return NGC_ERR_UNSUPPORTED;
  // A cluster per list where there is work for it, evictions or many sequences; as many CTAs as are resident at once.
  unsigned cluster = 1;
  if (kept_sorted || p.B > kThreads)
    while (cluster < 8 && 2 * cluster * p.G <= 2 * 148) cluster *= 2;
  p.split = n_slots > 4 * kThreads * (int)cluster;     // (four tokens per thread: 281 thousand tokens on 28 layers, 73 us without)
  const size_t smem = (size_t)(2 * (p.B + 1) + p.B + (p.B + (int)cluster - 1) / (int)cluster) * 4;      // first, need, from, waiting
  static PerDeviceOnce once;
  const int rc = once.run([] {
    cudaError_t e = cudaFuncSetAttribute(pool_update_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (4 * kMaxB + 16) * 4);
    return e == cudaSuccess ? cudaFuncSetAttribute(pool_slots_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (kMaxB + 1) * 4) : e;
  });
  if (rc != NGC_OK) return rc;
  NGC_CUDA_TRY(launch_pdl_cluster(pool_update_kernel, dim3(cluster, p.G), dim3(kThreads), cluster, smem, stream, p));
  if (p.split)
    NGC_CUDA_TRY(launch_pdl(pool_slots_kernel, dim3((unsigned)(((int64_t)n_slots + kWarps * kRun - 1) / (kWarps * kRun)), p.G), dim3(kThreads),
                            (size_t)(p.B + 1) * 4, stream, p));
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
