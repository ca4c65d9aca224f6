// Row moves around a draft: ngc_commit_draft appends the K/V rows of the accepted nodes, ngc_fork_kv
// copies a prefilled sequence to the sequences of its group.  Contiguous and paged caches.
//
// Both only move 16-byte vectors: HBM-bound for large batches, launch latency for small ones.
#include "ngc_common.cuh"
#include "ptx.cuh"

namespace ngc {
namespace {

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
// Whether pages [lo, hi) of every list of b are pages; all threads take part, each checks its share.
__device__ __forceinline__ bool pages_bad(const MoveParams& p, int b, int gi, int lo, int hi) {
  const int32_t* row = p.page_table + ((int64_t)b * p.G + gi) * p.pages_cap;
  for (int j = lo; j < hi; ++j)
    if (row[j] < 0 || row[j] >= p.pages_cap) return true;
  return false;
}
// Length of list gi of b as the tables count lists (a length per sequence serves all of its lists).
__device__ __forceinline__ int list_len(const MoveParams& p, int b, int gi, int n_lens) {
  return p.lens[(int64_t)b * n_lens + (n_lens == 1 ? 0 : gi)];
}

// ---------------------------------------------------------------- commit

__global__ void __launch_bounds__(kMoveThreads) commit_rows_kernel(MoveParams p) {
  const int b = blockIdx.y, tid = threadIdx.x;
  ptx::grid_dep_wait();
  ptx::grid_dep_launch();
  const int n = p.n_path[b];
  const int32_t* path = p.path + (int64_t)b * p.N;
  int status = NGC_DEV_OK;
  if (n < 0 || n > p.N) status = NGC_DEV_BAD_TREE;
  else
    for (int j = tid; j < n; j += kMoveThreads)
      if (path[j] < (j ? path[j - 1] + 1 : 0) || path[j] >= p.N) status = NGC_DEV_BAD_TREE;
  if (__syncthreads_or(status != NGC_DEV_OK)) status = NGC_DEV_BAD_TREE;
  const int n_lens = lists_G(p.lens_lists, p.L, p.Hkv);
  if (status == NGC_DEV_OK) {
    const int64_t cap = move_capacity(p, b);
    bool full = false, bad_page = false;
    const int lists = p.page_table ? p.G : n_lens;
    for (int gi = tid; gi < lists; gi += kMoveThreads) {
      const int len = list_len(p, b, gi, n_lens);
      if (len < 0 || (int64_t)len + n > cap) full = true;
      else if (p.page_table && n > 0) bad_page = bad_page || pages_bad(p, b, gi, len / p.page, (len + n - 1) / p.page + 1);
    }
    if (__syncthreads_or(full)) status = NGC_DEV_STRIP_FULL;
    else if (__syncthreads_or(bad_page)) status = NGC_DEV_BAD_PAGE;
  }
  if (status != NGC_DEV_OK) {
    if (tid == 0) set_dev_status(p.dev_status, status);
    return;
  }
  // vectors of the sequence: (plane, K or V, row of the path, piece)
  const int per_row = p.row_vecs, per_half = n * per_row;
  const int64_t total = (int64_t)p.L * p.Hkv * 2 * per_half;
  for (int64_t i = (int64_t)blockIdx.x * kMoveThreads + tid; i < total; i += (int64_t)gridDim.x * kMoveThreads) {
    const int half = (int)(i / per_half), rest = (int)(i % per_half), j = rest / per_row, c = rest % per_row;
    const int plane = half >> 1, l = plane / p.Hkv, h = plane % p.Hkv;
    const uint4* src = (half & 1 ? p.tree_v : p.tree_k) + ((((int64_t)l * p.B + b) * p.Hkv + h) * p.N + path[j]) * per_row + c;
    const int64_t row = move_row(p, b, l, h, move_len(p, b, l, h) + j);
    if (NGC_IN_BOUNDS(p.dev_status, row >= 0 && row < p.rows))
      (half & 1 ? p.v : p.k)[((int64_t)plane * p.rows + row) * per_row + c] = *src;
  }
}

// Lengths of the sequences that were committed: the same checks, one warp per sequence.
__global__ void __launch_bounds__(kMoveThreads) commit_lens_kernel(MoveParams p) {
  ptx::grid_dep_launch();
  ptx::grid_dep_wait();          // every CTA of the copy has read the lengths
  const int b = blockIdx.x * (kMoveThreads / 32) + (threadIdx.x >> 5), lane = threadIdx.x & 31;
  if (b >= p.B) return;
  const int n = p.n_path[b];
  const int32_t* path = p.path + (int64_t)b * p.N;
  bool bad = n < 0 || n > p.N;
  if (!bad)
    for (int j = lane; j < n; j += 32) bad = bad || path[j] < (j ? path[j - 1] + 1 : 0) || path[j] >= p.N;
  if (__any_sync(0xffffffffu, bad)) return;
  const int n_lens = lists_G(p.lens_lists, p.L, p.Hkv), lists = p.page_table ? p.G : n_lens;
  const int64_t cap = move_capacity(p, b);
  for (int gi = lane; gi < lists; gi += 32) {
    const int len = list_len(p, b, gi, n_lens);
    if (len < 0 || (int64_t)len + n > cap) bad = true;
    else if (p.page_table && n > 0) bad = bad || pages_bad(p, b, gi, len / p.page, (len + n - 1) / p.page + 1);
  }
  if (__any_sync(0xffffffffu, bad)) return;
  for (int gi = lane; gi < n_lens; gi += 32) p.lens[(int64_t)b * n_lens + gi] += n;
}

// ---------------------------------------------------------------- fork

// One CTA per (destination, plane, K or V); destinations vary fastest, so that the copies of one source strip run
// side by side and read it from L2.
__global__ void __launch_bounds__(kMoveThreads) fork_rows_kernel(MoveParams p) {
  const int tid = threadIdx.x;
  const int b = blockIdx.x % p.B, strip = blockIdx.x / p.B, isv = strip & 1, plane = strip >> 1;
  const int l = plane / p.Hkv, h = plane % p.Hkv;
  ptx::grid_dep_wait();
  ptx::grid_dep_launch();
  const int s = p.src_of[b];
  if (s == -1 || s == b) return;
  int status = NGC_DEV_OK;
  if (s < 0 || s >= p.B || (p.src_of[s] != -1 && p.src_of[s] != s)) status = NGC_DEV_BAD_SOURCE;
  const int n_lens = lists_G(p.lens_lists, p.L, p.Hkv);
  if (status == NGC_DEV_OK) {
    const int64_t cap_s = move_capacity(p, s), cap_b = move_capacity(p, b);
    bool counts = false, full = false, bad_page = false;
    const int lists = p.page_table ? p.G : n_lens;
    for (int gi = tid; gi < lists; gi += kMoveThreads) {
      const int len = list_len(p, s, gi, n_lens);
      if (len < 0 || len > cap_s) counts = true;
      else if (len > cap_b) full = true;
      else if (p.page_table) {
        const int pages = (len + p.page - 1) / p.page;
        bad_page = bad_page || pages_bad(p, s, gi, 0, pages) || pages_bad(p, b, gi, 0, pages);
      }
    }
    if (__syncthreads_or(counts)) status = NGC_DEV_BAD_COUNTS;
    else if (__syncthreads_or(full)) status = NGC_DEV_STRIP_FULL;
    else if (__syncthreads_or(bad_page)) status = NGC_DEV_BAD_PAGE;
  }
  if (status != NGC_DEV_OK) {
    if (tid == 0) set_dev_status(p.dev_status, status);
    return;
  }
  const int len = move_len(p, s, l, h);
  uint4* buf = (isv ? p.v : p.k) + (int64_t)plane * p.rows * p.row_vecs;
  for (int i = tid; i < len * p.row_vecs; i += kMoveThreads) {
    const int t = i / p.row_vecs, c = i % p.row_vecs;
    const int64_t from = move_row(p, s, l, h, t), to = move_row(p, b, l, h, t);
    if (NGC_IN_BOUNDS(p.dev_status, from >= 0 && from < p.rows && to >= 0 && to < p.rows))
      buf[to * p.row_vecs + c] = buf[from * p.row_vecs + c];
  }
  // nobody reads a destination's lengths (a source is no destination)
  if (strip == 0)
    for (int gi = tid; gi < n_lens; gi += kMoveThreads) p.lens[(int64_t)b * n_lens + gi] = p.lens[(int64_t)s * n_lens + gi];
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
  if (c->B > 65535) return NGC_ERR_UNSUPPORTED;
  const int64_t most = (int64_t)c->L * c->Hkv * 2 * N * p.row_vecs;
  int64_t per_seq = (most + kMoveThreads * 4 - 1) / (kMoveThreads * 4);
  if (per_seq > 16) per_seq = 16;
  NGC_CUDA_TRY(launch_pdl(commit_rows_kernel, dim3((unsigned)per_seq, (unsigned)c->B), dim3(kMoveThreads), 0, stream, p));
  NGC_CUDA_TRY(launch_pdl(commit_lens_kernel, dim3((unsigned)((c->B + 7) / 8)), dim3(kMoveThreads), 0, stream, p));
  return NGC_OK;
}

int fork_impl(const ngc_cache* c, const PagedView& pv, const int32_t* src_of, int32_t* dev_status, cudaStream_t stream) {
  if (!src_of) return NGC_ERR_INVALID_ARG;
  if ((((uintptr_t)c->k | (uintptr_t)c->v) & 15) != 0) return NGC_ERR_INVALID_ARG;
  MoveParams p = move_params(c, pv, dev_status);
  p.src_of = src_of;
  const int64_t grid = (int64_t)c->B * c->L * c->Hkv * 2;
  if (grid > 0x7fffffffLL) return NGC_ERR_UNSUPPORTED;
  NGC_CUDA_TRY(launch_pdl(fork_rows_kernel, dim3((unsigned)grid), dim3(kMoveThreads), 0, stream, p));
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
