// Row moves around a draft: ngc_commit_draft appends the K/V rows of the accepted nodes, ngc_fork_kv
// copies a prefilled sequence to the sequences of its group.  Contiguous and paged caches.
//
// Both only move whole rows: HBM-bound for large batches, launch latency for small ones.
#include <cooperative_groups.h>

#include "ngc_common.cuh"
#include "ptx.cuh"

namespace ngc {
namespace {

namespace cg = cooperative_groups;

constexpr int kMoveThreads = 256;

struct MoveParams {
  uint4* k;
  uint4* v;
  const int64_t* seq_off;
  int32_t* lens;
  const int32_t* page_table;    // null: contiguous
  int32_t* dev_status;
  int64_t rows;                 // per plane
  int L, B, Hkv, row_vecs, page, pages_cap, lists, G, lens_lists;
  const uint4* tree_k;          // commit
  const uint4* tree_v;
  const int32_t* path;
  const int32_t* n_path;
  int N;
  const int32_t* src_of;        // fork
};

__device__ __forceinline__ int64_t move_capacity(const MoveParams& p, int b) {
  return p.page_table ? (int64_t)p.pages_cap * p.page : p.seq_off[b + 1] - p.seq_off[b];
}
__device__ __forceinline__ int move_len(const MoveParams& p, int b, int l, int h) {
  return p.lens[len_index(p.lens_lists, p.L, p.Hkv, b, l, h)];
}
// Plane row of position t of strip (b, l, h); the page entries in question have been checked.
__device__ __forceinline__ int64_t move_row(const MoveParams& p, int b, int l, int h, int t) {
  if (!p.page_table) return p.seq_off[b] + t;
  const int32_t* row = p.page_table + ((int64_t)b * p.G + list_of(p.lists, l, h, p.Hkv)) * p.pages_cap;
  return ((int64_t)b * p.pages_cap + row[t / p.page]) * p.page + t % p.page;
}
// Whether an entry [lo, hi) of a list's table row is no page.
__device__ __forceinline__ bool pages_bad(const MoveParams& p, int b, int gi, int lo, int hi) {
  const int32_t* row = p.page_table + ((int64_t)b * p.G + gi) * p.pages_cap;
  bool bad = false;
  for (int j = lo; j < hi; ++j) bad |= (uint32_t)row[j] >= (uint32_t)p.pages_cap;
  return bad;
}
// Length of list gi of b as the tables count lists (a length per sequence serves all of its lists).
__device__ __forceinline__ int list_len(const MoveParams& p, int b, int gi, int n_lens) {
  return p.lens[(int64_t)b * n_lens + (n_lens == 1 ? 0 : gi)];
}

// ---------------------------------------------------------------- commit

// A cluster of CTAs per sequence.  All of them check the path and the room (every list, since a sequence is committed
// whole or not at all), copy their share of the rows, and meet at a cluster barrier: behind it nobody reads the lengths
// any more and the first CTA writes the new ones.  One launch: for a single rollout the call is all latency (28 layers x 2
// heads, 4 of 8 nodes: 4.5 us).  256 sequences, 7 of 16 nodes, pages of 32: 25 us, 103 MB; three rounds of dependent loads
// (lengths, table entries, rows) stand before the stores.
constexpr int kMoveVecs = 2;                    // vectors of K, and of V, a thread has in flight
__global__ void __launch_bounds__(kMoveThreads) commit_kernel(MoveParams p) {
  const cg::cluster_group cluster = cg::this_cluster();
  __shared__ int s_path[NGC_TREE_MAX_NODES];
  __shared__ int s_wrong;
  const int ctas = (int)cluster.num_blocks(), rank = (int)cluster.block_rank();
  const int b = blockIdx.x / ctas, tid = threadIdx.x;
  ptx::grid_dep_wait();
  ptx::grid_dep_launch();
  // path, lengths and path length in one round of loads, the pages in a second
  const int n_lens = lists_G(p.lens_lists, p.L, p.Hkv), lists = p.page_table ? p.G : n_lens;
  int n = p.n_path[b], x = 0, before = -1, len = tid < lists ? list_len(p, b, tid, n_lens) : 0;
  if (tid < p.N) {
    x = p.path[(int64_t)b * p.N + tid];
    if (tid > 0) before = p.path[(int64_t)b * p.N + tid - 1];
  }
  const int64_t cap = move_capacity(p, b);
  bool bad = n < 0 || n > p.N;
  if (bad) n = 0;
  if (tid < n) {
    bad = x <= before || x < 0 || x >= p.N;
    s_path[tid] = x;
  }
  bool full = false, bad_page = false;
  for (int gi = tid; gi < lists; gi += kMoveThreads) {
    if (gi != tid) len = list_len(p, b, gi, n_lens);
    if (len < 0 || (int64_t)len + n > cap) full = true;
    else if (p.page_table && n > 0) bad_page = bad_page || pages_bad(p, b, gi, len / p.page, (len + n - 1) / p.page + 1);
  }
  if (tid == 0) s_wrong = 0;
  __syncthreads();
  if (bad || full || bad_page) atomicOr(&s_wrong, (bad ? 1 : 0) | (full ? 2 : 0) | (bad_page ? 4 : 0));
  __syncthreads();
  const int wrong = s_wrong;
  const int status = wrong & 1 ? NGC_DEV_BAD_TREE : wrong & 2 ? NGC_DEV_STRIP_FULL : wrong & 4 ? NGC_DEV_BAD_PAGE : NGC_DEV_OK;
  if (status != NGC_DEV_OK) {
    if (tid == 0) set_dev_status(p.dev_status, status);
    n = 0;
  }
  // rows of the sequence: (plane, row of the path), K and V of each; a thread per 16-byte piece
  const uint32_t piece = tid & (p.row_vecs - 1), per_round = kMoveThreads / p.row_vecs;        // (row_vecs: 8, 16 or 32)
  const uint32_t total = (uint32_t)(p.L * p.Hkv) * n;
  for (uint32_t i0 = rank * per_round + tid / p.row_vecs; i0 < total; i0 += ctas * per_round * kMoveVecs) {
    uint4 xk[kMoveVecs], xv[kMoveVecs];
    int64_t to[kMoveVecs];
#pragma unroll
    for (int e = 0; e < kMoveVecs; ++e) {
      const uint32_t i = i0 + e * ctas * per_round;
      to[e] = -1;
      if (i >= total) continue;
      const uint32_t plane = i / (uint32_t)n, j = i - plane * n, l = plane / (uint32_t)p.Hkv, h = plane - l * p.Hkv;
      const int64_t from = ((((int64_t)l * p.B + b) * p.Hkv + h) * p.N + s_path[j]) * p.row_vecs + piece;
      xk[e] = p.tree_k[from];
      xv[e] = p.tree_v[from];
      const int64_t row = move_row(p, b, l, h, move_len(p, b, l, h) + (int)j);
      if (NGC_IN_BOUNDS(p.dev_status, row >= 0 && row < p.rows)) to[e] = ((int64_t)plane * p.rows + row) * p.row_vecs + piece;
    }
#pragma unroll
    for (int e = 0; e < kMoveVecs; ++e)
      if (to[e] >= 0) {
        p.k[to[e]] = xk[e];
        p.v[to[e]] = xv[e];
      }
  }
  cluster.sync();
  if (rank == 0 && n > 0)
    for (int gi = tid; gi < n_lens; gi += kMoveThreads) p.lens[(int64_t)b * n_lens + gi] += n;
}

// ---------------------------------------------------------------- fork

// Barrier of `threads` threads of the CTA (whole warps).
__device__ __forceinline__ void named_barrier(int id, int threads) {
  asm volatile("bar.sync %0, %1;" ::"r"(id), "r"(threads) : "memory");
}

// A source strip is read once for all of its copies: bulk copies bring up to 64 KB of it into shared memory, from where
// bulk stores write it to every destination (a lane per destination).  No data passes through registers, and a CTA
// of one busy warp keeps 64 KB in flight.  grid.x = (strip, chunk of its rows), chunks beyond the grid's follow in turns;
// grid.y deals the destinations out, so that one prompt's group alone fills the GPU.  Bound by DRAM writes: 4 prompts of 900
// to 1100 tokens to 16 sequences each, 28 layers x 2 heads, 1.8 GB: 330 us, 5.5 TB/s; a prompt of 350 to 8, paged: 19 us.
constexpr int kForkThreads = 128;
constexpr int kForkQuarter = 16384, kForkChunk = 4 * kForkQuarter;     // bytes
constexpr int kForkMaxB = 65536;

__global__ void __launch_bounds__(kForkThreads) fork_kernel(MoveParams p, int n_chunks) {
  extern __shared__ __align__(128) uint8_t stage[];                    // [4][kForkQuarter]
  __shared__ uint32_t is_source[kForkMaxB / 32];
  __shared__ uint64_t full[4];
  __shared__ int dst[kForkThreads], bad_dst[kForkThreads], n_dst;
  const int tid = threadIdx.x, lane = tid & 31;
  const int strip = blockIdx.x / n_chunks, chunk0 = blockIdx.x % n_chunks, isv = strip & 1, plane = strip >> 1;
  const int l = plane / p.Hkv, h = plane % p.Hkv, own_list = p.page_table ? list_of(p.lists, l, h, p.Hkv) : 0;
  const bool reports = blockIdx.x == 0 && blockIdx.y == 0, sets_lens = blockIdx.x == 0;
  const int n_lens = lists_G(p.lens_lists, p.L, p.Hkv);
  const int row_bytes = p.row_vecs * 16, chunk_rows = kForkChunk / row_bytes, quarter_rows = kForkQuarter / row_bytes;
  uint8_t* const buf = (uint8_t*)(isv ? p.v : p.k) + (int64_t)plane * p.rows * row_bytes;
  if (tid == 0) {
    for (int i = 0; i < 4; ++i) ptx::mbar_init(&full[i], 1);
    ptx::fence_barrier_init();
  }
  for (int i = tid; i < (p.B + 31) / 32; i += kForkThreads) is_source[i] = 0;
  ptx::grid_dep_wait();
  ptx::grid_dep_launch();
  __syncthreads();
  for (int b = tid; b < p.B; b += kForkThreads) {
    const int s = p.src_of[b];
    if (s == -1 || s == b) continue;
    if (s < 0 || s >= p.B || (p.src_of[s] != -1 && p.src_of[s] != s)) {
      if (reports) set_dev_status(p.dev_status, NGC_DEV_BAD_SOURCE);
    } else {
      atomicOr(&is_source[s >> 5], 1u << (s & 31));
    }
  }
  __syncthreads();
  int turn = 0;                                 // chunks that went through the stage so far (phase of its barriers)
  bool ok = true;
  for (int word = 0; word < (p.B + 31) / 32; ++word)
    for (uint32_t bits = is_source[word]; bits; bits &= bits - 1) {
      const int s = 32 * word + __ffs(bits) - 1;
      // the source's lengths, and its pages of this strip's list
      const int64_t cap_s = move_capacity(p, s);
      const int lists = p.page_table ? p.G : n_lens;
      bool wrong = false;
      for (int gi = tid; gi < lists; gi += kForkThreads) {
        const int len = list_len(p, s, gi, n_lens);
        wrong = wrong || len < 0 || len > cap_s;
      }
      if (__syncthreads_or(wrong)) {
        if (reports && tid == 0) set_dev_status(p.dev_status, NGC_DEV_BAD_COUNTS);
        continue;
      }
      const int len = move_len(p, s, l, h);
      const int32_t* from = p.page_table ? p.page_table + ((int64_t)s * p.G + own_list) * p.pages_cap : nullptr;
      const int pages = p.page_table ? (len + p.page - 1) / p.page : 0;
      for (int j = tid; j < pages; j += kForkThreads) wrong = wrong || from[j] < 0 || from[j] >= p.pages_cap;
      const bool bad_source_page = __syncthreads_or(wrong);
      for (int b0 = 0; b0 < p.B; b0 += kForkThreads) {
        // destinations among the next sequences: a thread each
        const int b = b0 + tid;
        if (tid == 0) n_dst = 0;
        __syncthreads();
        if (b < p.B && b != s && p.src_of[b] == s && (s + b) % gridDim.y == blockIdx.y) {
          const int64_t cap_b = move_capacity(p, b);
          bool small = false, bad_page = bad_source_page;
          for (int gi = 0; gi < n_lens; ++gi) small |= list_len(p, s, gi, n_lens) > cap_b;
          const int32_t* to = p.page_table ? p.page_table + ((int64_t)b * p.G + own_list) * p.pages_cap : nullptr;
          if (!small)
            for (int j = 0; j < pages; ++j) bad_page |= (uint32_t)to[j] >= (uint32_t)p.pages_cap;
          if (small || bad_page) set_dev_status(p.dev_status, small ? NGC_DEV_STRIP_FULL : NGC_DEV_BAD_PAGE);
          else dst[atomicAdd(&n_dst, 1)] = b;
        }
        __syncthreads();
        const int n = n_dst;
        if (tid < 32 && n > 0) {
          for (int r0 = chunk0 * chunk_rows; ok && r0 < len; r0 += n_chunks * chunk_rows) {
            ptx::bulk_wait_read<0>();           // this lane's stores have read the stage
            __syncwarp();
            const int rows = min(chunk_rows, len - r0);
            if (lane == 0) {
              for (int i = 0; i * quarter_rows < rows; ++i) {
                const int m = min(quarter_rows, rows - i * quarter_rows);
                ptx::mbar_expect_tx(&full[i], (uint32_t)(m * row_bytes));
                const int step = p.page_table ? p.page : m;
                for (int r = 0; r < m; r += step) {
                  const int t = r0 + i * quarter_rows + r;
                  const int64_t row = p.page_table ? ((int64_t)s * p.pages_cap + from[t / p.page]) * p.page : p.seq_off[s] + t;
                  ptx::bulk_load(stage + i * kForkQuarter + r * row_bytes, buf + row * row_bytes, (uint32_t)(min(step, m - r) * row_bytes), &full[i]);
                }
              }
            }
            __syncwarp();
            for (int i = 0; i * quarter_rows < rows; ++i) {
              // (phases are counted per quarter: a short chunk does not use them all)
              const int m = min(quarter_rows, rows - i * quarter_rows);
              ok = __all_sync(0xffffffffu, ptx::mbar_wait_bounded(&full[i], (turn >> (8 * i)) & 1));
              if (!ok) {                        // giving up: no copy may be in flight when the CTA ends
                for (int j = i + 1; j * quarter_rows < rows; ++j) ptx::mbar_wait_bounded(&full[j], (turn >> (8 * j)) & 1);
                break;
              }
              for (int d = lane; d < n; d += 32) {
                const int b2 = dst[d];
                const int32_t* to = p.page_table ? p.page_table + ((int64_t)b2 * p.G + own_list) * p.pages_cap : nullptr;
                const int step = p.page_table ? p.page : m;
                for (int r = 0; r < m; r += step) {
                  const int t = r0 + i * quarter_rows + r;
                  const int64_t row = p.page_table ? ((int64_t)b2 * p.pages_cap + to[t / p.page]) * p.page : p.seq_off[b2] + t;
                  if (NGC_IN_BOUNDS(p.dev_status, row >= 0 && row + min(step, m - r) <= p.rows))
                    ptx::bulk_store(buf + row * row_bytes, stage + i * kForkQuarter + r * row_bytes, (uint32_t)(min(step, m - r) * row_bytes));
                }
              }
              ptx::bulk_commit();
              turn ^= 1 << (8 * i);
            }
            if (!ok && lane == 0) set_dev_status(p.dev_status, NGC_DEV_TIMEOUT);
          }
        } else if (tid >= 32 && sets_lens) {
          // meanwhile the other warps set the lengths of those whose lists all have good pages; nobody reads a destination's
          // lengths (a source is no destination)
          const int t = tid - 32, threads = kForkThreads - 32;
          for (int d = t; d < n; d += threads) bad_dst[d] = 0;
          named_barrier(1, threads);
          if (p.page_table) {
            const uint32_t entries = (uint32_t)p.G * p.pages_cap;
            for (uint32_t j = t; j < entries; j += threads) {
              const uint32_t gi = j / (uint32_t)p.pages_cap;
              if ((int)(j - gi * p.pages_cap) >= (list_len(p, s, gi, n_lens) + p.page - 1) / p.page) continue;
              const bool bad_source = (uint32_t)p.page_table[(int64_t)s * entries + j] >= (uint32_t)p.pages_cap;
#pragma unroll 4
              for (int d = 0; d < n; ++d)
                if (bad_source | ((uint32_t)p.page_table[(int64_t)dst[d] * entries + j] >= (uint32_t)p.pages_cap)) bad_dst[d] = 1;
            }
            named_barrier(1, threads);
          }
          for (int i = t; i < n * n_lens; i += threads) {
            const int d = i / n_lens, gi = i % n_lens;
            if (!bad_dst[d]) p.lens[(int64_t)dst[d] * n_lens + gi] = p.lens[(int64_t)s * n_lens + gi];
            else if (gi == 0) set_dev_status(p.dev_status, NGC_DEV_BAD_PAGE);
          }
        }
        __syncthreads();                        // the list may change
      }
    }
  if (tid < 32) ptx::bulk_wait<0>();            // every store has been written
}

// ---------------------------------------------------------------- host side

MoveParams move_params(const ngc_cache* c, const PagedView& pv, int32_t* dev_status) {
  MoveParams p = {};
  p.k = (uint4*)c->k; p.v = (uint4*)c->v; p.seq_off = c->seq_off; p.lens = c->lens; p.dev_status = dev_status;
  p.rows = c->rows; p.L = c->L; p.B = c->B; p.Hkv = c->Hkv; p.row_vecs = c->d * elt_bytes(c->dtype) / 16;
  p.page_table = pv.table; p.page = pv.page; p.pages_cap = pv.pages_cap; p.lists = pv.lists;
  p.G = lists_G(pv.lists, c->L, c->Hkv); p.lens_lists = c->lens_lists;
  return p;
}

int commit_impl(const ngc_cache* c, const PagedView& pv, const void* tree_k, const void* tree_v, const int32_t* path,
                const int32_t* n_path, int N, int32_t* dev_status, cudaStream_t stream) {
  if (!tree_k || !tree_v || !path || !n_path || N < 1) return NGC_ERR_INVALID_ARG;
  if ((((uintptr_t)tree_k | (uintptr_t)tree_v | (uintptr_t)c->k | (uintptr_t)c->v) & 15) != 0) return NGC_ERR_INVALID_ARG;
  if (N > NGC_TREE_MAX_NODES) return NGC_ERR_UNSUPPORTED;
  MoveParams p = move_params(c, pv, dev_status);
  p.tree_k = (const uint4*)tree_k; p.tree_v = (const uint4*)tree_v; p.path = path; p.n_path = n_path; p.N = N;
  // CTAs per sequence: at most 8, no more than a round of vectors would occupy if every node were accepted, nor than
  // about one round of CTAs in all (each of them repeats the checks)
  const int64_t most = (int64_t)c->L * c->Hkv * N * p.row_vecs;
  unsigned cluster = 1;
  while (cluster < 8 && most > (int64_t)cluster * kMoveThreads * kMoveVecs && (int64_t)c->B * cluster * 2 <= 4 * 148) cluster *= 2;
  if ((int64_t)c->B * cluster > 0x7fffffffLL || most > 0x7fffffffLL) return NGC_ERR_UNSUPPORTED;
  NGC_CUDA_TRY(launch_pdl_cluster(commit_kernel, dim3((unsigned)c->B * cluster), dim3(kMoveThreads), cluster, 0, stream, p));
  return NGC_OK;
}

int fork_impl(const ngc_cache* c, const PagedView& pv, const int32_t* src_of, int32_t* dev_status, cudaStream_t stream) {
  if (!src_of) return NGC_ERR_INVALID_ARG;
  if ((((uintptr_t)c->k | (uintptr_t)c->v) & 15) != 0) return NGC_ERR_INVALID_ARG;
  MoveParams p = move_params(c, pv, dev_status);
  p.src_of = src_of;
  if (c->B > kForkMaxB) return NGC_ERR_UNSUPPORTED;
  static PerDeviceOnce attr_once;
  const int rc = attr_once.run([] { return cudaFuncSetAttribute(fork_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kForkChunk); });
  if (rc != NGC_OK) return rc;
  // one round of CTAs (three fit an SM; two rounds: 348 us instead of 333 us for four prompts to sixteen rollouts each),
  // first over the rows of the strips, then over the destinations
  const int64_t strips = (int64_t)c->L * c->Hkv * 2, want = 3 * 148;
  const int64_t most_chunks = ((int64_t)c->max_len * p.row_vecs * 16 + kForkChunk - 1) / kForkChunk;
  int64_t chunks = (want + strips - 1) / strips;
  if (chunks > most_chunks) chunks = most_chunks;
  if (chunks < 1) chunks = 1;
  int64_t deals = (want + strips * chunks - 1) / (strips * chunks);
  if (deals > c->B) deals = c->B;
  if (strips * chunks > 0x7fffffffLL) return NGC_ERR_UNSUPPORTED;
  NGC_CUDA_TRY(launch_pdl(fork_kernel, dim3((unsigned)(strips * chunks), (unsigned)deals), dim3(kForkThreads), kForkChunk, stream, p, (int)chunks));
  return NGC_OK;
}

}  // namespace
}  // namespace ngc

extern "C" int ngc_commit_draft(ngc_cache* c, const void* tree_k, const void* tree_v, const int32_t* path, const int32_t* n_path,
                                int N, int32_t* dev_status, ngc_stream stream) {
  NGC_API_RANGE("ngc_commit_draft");
  using namespace ngc;
  if (!valid_cache(c)) return NGC_ERR_INVALID_ARG;
  const PagedView none = {nullptr, 0, 0, NGC_LISTS_SHARED};
  return commit_impl(c, none, tree_k, tree_v, path, n_path, N, dev_status, (cudaStream_t)stream);
}

extern "C" int ngc_commit_draft_paged(ngc_paged_cache* pc, const void* tree_k, const void* tree_v, const int32_t* path,
                                      const int32_t* n_path, int N, int32_t* dev_status, ngc_stream stream) {
  NGC_API_RANGE("ngc_commit_draft_paged");
  using namespace ngc;
  ngc_cache c;
  if (!paged_as_cache(pc, &c)) return NGC_ERR_INVALID_ARG;
  if (c.dtype != NGC_BF16 || c.d != 128) return NGC_ERR_UNSUPPORTED;
  const PagedView pv = {pc->page_table, pc->page, pc->pages_cap, pc->lists};
  return commit_impl(&c, pv, tree_k, tree_v, path, n_path, N, dev_status, (cudaStream_t)stream);
}

extern "C" int ngc_fork_kv(ngc_cache* c, const int32_t* src_of, int32_t* dev_status, ngc_stream stream) {
  NGC_API_RANGE("ngc_fork_kv");
  using namespace ngc;
  if (!valid_cache(c)) return NGC_ERR_INVALID_ARG;
  const PagedView none = {nullptr, 0, 0, NGC_LISTS_SHARED};
  return fork_impl(c, none, src_of, dev_status, (cudaStream_t)stream);
}

extern "C" int ngc_fork_pages(ngc_paged_cache* pc, const int32_t* src_of, int32_t* dev_status, ngc_stream stream) {
  NGC_API_RANGE("ngc_fork_pages");
  using namespace ngc;
  ngc_cache c;
  if (!paged_as_cache(pc, &c)) return NGC_ERR_INVALID_ARG;
  if (c.dtype != NGC_BF16 || c.d != 128) return NGC_ERR_UNSUPPORTED;
  const PagedView pv = {pc->page_table, pc->page, pc->pages_cap, pc->lists};
  return fork_impl(&c, pv, src_of, dev_status, (cudaStream_t)stream);
}
