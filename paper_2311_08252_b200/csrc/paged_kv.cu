// Pages of a KV cache: rows written into them and compacted (rest_paged_kv_write,
// rest_paged_kv_commit), contexts forked (rest_pages_fork, rest_pages_copy), grown and trimmed
// (rest_pages_reserve, rest_pages_release).  Not in the paper, which never describes the cache.
//
// Row l of context b sits in page table[b][l / page], row l % page of it.  refs[p] counts the
// contexts that hold page p; a page is free iff its count is 0.  There is no list of free pages:
// pages are handed out lowest number first, to contexts in order, so every result is fixed by
// the inputs whatever the scheduling, and releasing a page is one integer decrement.
//
// All of these move bytes and compute nothing: the bound is HBM for the row and page copies
// (every byte read once and written once, 16 bytes per access, four accesses of a thread in
// flight) and the launch for the tables, whose kernels are one block (or one block per context).
// Measured (B200; a copy runs at 6536 GB/s): 128 contexts x 64 rows x 32 KV heads written and committed 44 us
// (4.9 TB/s), 1 context 7 us (two launches); 64 contexts forked into 7 each, 128-row pages copied, room and
// release 70 to 85 us (6.6 to 5.5 TB/s).  A pool's counts are read by one block: reserve and release
// of 64 contexts 15 us for 2^14 pages, 99 us for 2^17, 567 us for 2^20.
#include <cuda_runtime.h>
#include <stdint.h>

#include "common.cuh"
#include "paged_pool.cuh"
#include "rest.h"

namespace {

using namespace rest_pool;

constexpr int kMaxDepth = REST_MAX_M;

// ------------------------------------------------------------------------------------ rows
// One warp per 2 KB of one new K or V row (four 16-byte vectors per lane, all loaded before the
// first store): a row of many heads is spread over several warps, so that a single stream's few
// rows still occupy many SMs.
constexpr int kWriteWarps = 8, kWriteVecs = 128;

__global__ void __launch_bounds__(kWriteWarps * 32)
rest_paged_kv_write_kernel(Pool c, const uint4* __restrict__ k_new, const uint4* __restrict__ v_new, int64_t n_b,
                           int64_t n_n, int64_t n_h, const int32_t* __restrict__ kv_len,
                           const int32_t* __restrict__ n_nodes, int64_t units, int N, int chunks, int row_vecs,
                           int dv_log) {
  grid_wait();
  const int lane = threadIdx.x & 31;
  const int64_t unit = (int64_t)blockIdx.x * kWriteWarps + (threadIdx.x >> 5);
  if (unit >= units) return;
  const int chunk = (int)(unit % chunks);
  const int64_t rest_ = unit / chunks;
  const int which = (int)(rest_ & 1);
  const int i = (int)((rest_ >> 1) % N);
  const int b = (int)((rest_ >> 1) / N);
  if (n_nodes && i >= n_nodes[b]) return;
  const int64_t to = row_offset(c, b, kv_len[b] + i);
  if (kv_len[b] < 0 || to < 0) return;
  const uint4* src = (which ? v_new : k_new) + b * n_b + i * n_n;
  uint4* dst = (which ? c.v : c.k) + to;
  uint4 x[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const int e = chunk * kWriteVecs + j * 32 + lane;
    if (e < row_vecs) x[j] = __ldcs(src + (e >> dv_log) * n_h + (e & ((1 << dv_log) - 1)));
  }
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const int e = chunk * kWriteVecs + j * 32 + lane;
    if (e < row_vecs) dst[(e >> dv_log) * c.s_head + (e & ((1 << dv_log) - 1))] = x[j];
  }
}

// One block per context.  A thread owns one 16-byte column of one (head, K or V) and holds that
// column of every accepted row in registers before it writes the first: a slot may be the source
// of one path position and the target of another, and all such conflicts then lie inside one
// thread's program order.  Where rows sit is worked out once per block, by one thread per row.
// One block per context also lets the new length be written into the very array that the old
// one is read from.
constexpr int kCommitThreads = 512;

__global__ void __launch_bounds__(kCommitThreads)
rest_paged_kv_commit_kernel(Pool c, const int32_t* kv_len, const int32_t* __restrict__ accept_nodes,
                            const int32_t* __restrict__ accept_len, int H_kv, int N, int max_depth, int dv_log,
                            int32_t* new_kv_len) {
  grid_wait();
  __shared__ int64_t s_from[kMaxDepth], s_to[kMaxDepth];
  const int b = blockIdx.x;
  const int L = *reinterpret_cast<const volatile int32_t*>(kv_len + b);
  int len = accept_len[b];
  len = len < 0 ? 0 : (len > max_depth ? max_depth : len);
  if (threadIdx.x < kMaxDepth) {
    int64_t from = -1, to = -1;
    if ((int)threadIdx.x < len && L >= 0) {
      int nd = accept_nodes[(int64_t)b * max_depth + threadIdx.x];
      nd = nd < 0 ? 0 : (nd >= N ? N - 1 : nd);
      from = row_offset(c, b, L + nd);
      to = row_offset(c, b, L + (int)threadIdx.x);
      if (from == to) from = -1;                     // already in place
    }
    s_from[threadIdx.x] = to < 0 ? -1 : from;
    s_to[threadIdx.x] = to;
  }
  __syncthreads();
  const int vecs = (2 * H_kv) << dv_log;
  for (int e = threadIdx.x; e < vecs; e += kCommitThreads) {
    const int h = e >> (dv_log + 1);
    const int within = e & ((1 << dv_log) - 1);
    uint4* base = (((e >> dv_log) & 1) ? c.v : c.k) + h * c.s_head + within;
    uint4 x[kMaxDepth];
#pragma unroll
    for (int i = 0; i < kMaxDepth; ++i)
      if (i < len && s_from[i] >= 0) x[i] = base[s_from[i]];
#pragma unroll
    for (int i = 0; i < kMaxDepth; ++i)
      if (i < len && s_from[i] >= 0) base[s_to[i]] = x[i];
  }
  if (new_kv_len && threadIdx.x == 0) new_kv_len[b] = L + len;   // every read of L is behind the barrier
}

// ----------------------------------------------------------------------------------- pages
// One block per 16 KB of one page of K or V (256 threads, four vectors each).
constexpr int kCopyThreads = 256, kCopyVecs = 1024;

__global__ void __launch_bounds__(kCopyThreads)
rest_pages_copy_kernel(Pool c, const int32_t* __restrict__ src, const int32_t* __restrict__ dst, int chunks,
                       int vecs, int dv_log) {
  grid_wait();
  const int pair = blockIdx.x / chunks, chunk = blockIdx.x % chunks;
  const int a = src[pair], z = dst[pair];
  if (a < 0 || a >= c.P || z < 0 || z >= c.P || a == z) return;
  uint4* base = blockIdx.y ? c.v : c.k;
  int64_t at[4];
  uint4 x[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const int e = chunk * kCopyVecs + j * kCopyThreads + threadIdx.x;
    const int row = (e >> dv_log) & ((1 << c.page_log) - 1), h = e >> (dv_log + c.page_log);
    at[j] = h * c.s_head + row * c.s_row + (e & ((1 << dv_log) - 1));
    if (e < vecs) x[j] = base[a * c.s_page + at[j]];
  }
#pragma unroll
  for (int j = 0; j < 4; ++j)
    if (chunk * kCopyVecs + j * kCopyThreads + (int)threadIdx.x < vecs) base[z * c.s_page + at[j]] = x[j];
}

// ---------------------------------------------------------------------------------- tables
constexpr int kPlanThreads = 1024;

// Exclusive prefix sum of x over the block's 1024 threads; `total` receives the sum.
__device__ __forceinline__ int block_scan(int x, int& total, int* s_warp) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  int inc = x;
#pragma unroll
  for (int d = 1; d < 32; d <<= 1) {
    const int y = __shfl_up_sync(0xFFFFFFFFu, inc, d);
    if (lane >= d) inc += y;
  }
  __syncthreads();                       // s_warp may still be read from the call before
  if (lane == 31) s_warp[warp] = inc;
  __syncthreads();
  if (warp == 0) {
    int w = s_warp[lane];
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
      const int y = __shfl_up_sync(0xFFFFFFFFu, w, d);
      if (lane >= d) w += y;
    }
    s_warp[lane] = w;
  }
  __syncthreads();
  total = s_warp[31];
  return inc - x + (warp ? s_warp[warp - 1] : 0);
}

// Calls take(rank, page) for the free pages in ascending order, ranks below `limit` only; every
// thread owns one run of pages, so ranks follow page numbers.  Returns how many pages are free.
template <typename F>
__device__ __forceinline__ int for_free_pages(const int32_t* refs, int P, int limit, int* s_warp, F take) {
  const int per = (P + kPlanThreads - 1) / kPlanThreads;
  const int64_t lo64 = (int64_t)threadIdx.x * per;
  const int lo = (int)(lo64 < P ? lo64 : P), hi = P - lo < per ? P : lo + per;
  int mine = 0;
#pragma unroll 8
  for (int p = lo; p < hi; ++p) mine += refs[p] == 0;
  int total;
  int rank = block_scan(mine, total, s_warp);
  const int end = rank + mine;
  if (limit > total) limit = total;
  for (int p = lo; p < hi && rank < end && rank < limit; ++p)
    if (refs[p] == 0) take(rank++, p, total);
  return total;
}

__global__ void __launch_bounds__(kPlanThreads)
rest_pages_fork_plan_kernel(const int32_t* __restrict__ parents, const int32_t* __restrict__ children, int F,
                            int32_t* refs, int P, const int32_t* __restrict__ table, int64_t table_stride,
                            int table_cols, int32_t* n_pages, int32_t* kv_len, int B, int page_log,
                            int32_t* __restrict__ copy_src, int32_t* __restrict__ copy_dst,
                            int32_t* __restrict__ status) {
  grid_wait();
  __shared__ int s_child[kPlanThreads], s_page[kPlanThreads], s_warp[32];
  const int f = threadIdx.x;
  const int ch = f < F ? children[f] : -1, pa = f < F ? parents[f] : -1;
  s_child[f] = ch;
  __syncthreads();
  int st = REST_CTX_OK, L = 0, full = 0, part = 0;
  if (f < F) {
    if (ch < 0 || ch >= B || pa < 0 || pa >= B || pa == ch || n_pages[ch] != 0) st = REST_CTX_BAD_PAGES;
    for (int o = 0; o < f; ++o)
      if (s_child[o] == ch) st = REST_CTX_BAD_PAGES;      // the same child twice: the first call's wins
    if (st == REST_CTX_OK) {                              // an empty parent leaves an empty child
      L = kv_len[pa];
      full = L >> page_log;
      part = (L & ((1 << page_log) - 1)) != 0;
      if (L < 0 || full + part > n_pages[pa] || full + part > table_cols) { st = REST_CTX_BAD_PAGES; part = 0; }
    }
  }
  int need;
  const int off = block_scan(part, need, s_warp);
  const int have = for_free_pages(refs, P, need, s_warp, [&](int rank, int p, int) { s_page[rank] = p; });
  __syncthreads();
  if (part && off >= have) st = REST_CTX_NO_PAGES;
  if (f < F) {
    int a = -1, z = -1;
    if (st == REST_CTX_OK) {
      if (part) {
        a = table[pa * table_stride + full];
        z = s_page[off];
        if (a < 0 || a >= P) a = -1;                       // nothing to copy; the child's page is its own all the same
        refs[z] = 1;
      }
      n_pages[ch] = full + part;
      kv_len[ch] = L;
    }
    copy_src[f] = a;
    copy_dst[f] = z;
    status[f] = st;
  }
}

// Tables of the forked contexts: one block per fork.
__global__ void __launch_bounds__(128)
rest_pages_fork_tables_kernel(const int32_t* __restrict__ parents, const int32_t* __restrict__ children,
                              int32_t* refs, int P, int32_t* table, int64_t table_stride, int table_cols,
                              const int32_t* __restrict__ kv_len, int page_log, const int32_t* __restrict__ copy_dst,
                              const int32_t* __restrict__ status) {
  grid_wait();
  const int f = blockIdx.x;
  if (status[f] != REST_CTX_OK) return;
  const int ch = children[f], full = kv_len[ch] >> page_log, own = copy_dst[f];
  const int32_t* from = table + parents[f] * table_stride;
  int32_t* to = table + ch * table_stride;
  for (int col = threadIdx.x; col < table_cols; col += 128) {
    int p = -1;
    if (col < full) {
      p = from[col];
      if (p >= 0 && p < P) atomicAdd(refs + p, 1); else p = -1;
    } else if (col == full) {
      p = own;
    }
    to[col] = p;
  }
}

// Contexts' first ranks sit in shared memory; the page of rank r goes to the context whose range
// holds r (found by bisection), if all of that context's pages can be had.
__global__ void __launch_bounds__(kPlanThreads)
rest_pages_reserve_kernel(int32_t* refs, int P, int32_t* table, int64_t table_stride, int table_cols,
                          int32_t* n_pages, const int32_t* __restrict__ need_len, int B, int page_log,
                          int32_t* __restrict__ status) {
  grid_wait();
  extern __shared__ int s_first[];                     // [B + 1]
  __shared__ int s_warp[32];
  const int tid = threadIdx.x;
  auto wanted = [&](int b, int& st) {                  // pages context b asks for
    const int len = need_len[b], have = n_pages[b];
    st = REST_CTX_OK;
    const int64_t want = len <= 0 ? 0 : ((int64_t)len + (1 << page_log) - 1) >> page_log;
    if (have < 0 || have > table_cols || want > table_cols) { st = REST_CTX_BAD_PAGES; return 0; }
    return want > have ? (int)want - have : 0;
  };
  int total = 0;
  for (int base = 0; base < B; base += kPlanThreads) {
    int st, sum;
    const int need = base + tid < B ? wanted(base + tid, st) : 0;
    // a sum beyond the pool's size only has to stay beyond it
    const int capped = need > P ? P + 1 : need;
    const int off = block_scan(capped, sum, s_warp);
    if (base + tid < B) {
      const int64_t first = (int64_t)total + off;
      s_first[base + tid] = first > P + 1 ? P + 1 : (int)first;
    }
    const int64_t t = (int64_t)total + sum;
    total = t > P + 1 ? P + 1 : (int)t;
  }
  if (tid == 0) s_first[B] = total;
  __syncthreads();
  const int have = for_free_pages(refs, P, total, s_warp, [&](int rank, int p, int free_pages) {
    int lo = 0, hi = B;                                // last b with s_first[b] <= rank
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if (s_first[mid] <= rank) lo = mid; else hi = mid;
    }
    if (s_first[lo + 1] <= free_pages) {
      table[lo * table_stride + n_pages[lo] + rank - s_first[lo]] = p;
      refs[p] = 1;
    }
  });
  __syncthreads();
  for (int b = tid; b < B; b += kPlanThreads) {
    int st;
    const int need = wanted(b, st);
    if (st == REST_CTX_OK && need > 0) {
      if (s_first[b + 1] <= have) n_pages[b] += need; else st = REST_CTX_NO_PAGES;
    }
    status[b] = st;
  }
}

__global__ void __launch_bounds__(128)
rest_pages_release_kernel(int32_t* refs, int P, int32_t* table, int64_t table_stride, int table_cols,
                          int32_t* n_pages, const int32_t* __restrict__ keep_len, int page_log, int window,
                          int sinks) {
  grid_wait();
  const int b = blockIdx.x;
  const int keep = keep_len[b];
  if (keep < 0) return;                                // this context stays as it is
  int have = n_pages[b];
  have = have < 0 ? 0 : (have > table_cols ? table_cols : have);
  const int kept = (int)(((int64_t)keep + (1 << page_log) - 1) >> page_log);
  int32_t* row = table + b * table_stride;
  for (int col = threadIdx.x; col < have; col += 128) {
    const int64_t first = (int64_t)col << page_log, last = first + (1 << page_log) - 1;
    const bool behind = window > 0 && first >= sinks && last <= (int64_t)keep - window;
    if (col < kept && !behind) continue;
    const int p = row[col];
    row[col] = -1;
    if (p >= 0 && p < P && atomicSub(refs + p, 1) <= 0) atomicAdd(refs + p, 1);   // never below 0
  }
  __syncthreads();
  if (threadIdx.x == 0 && kept < have) n_pages[b] = kept;
}

}  // namespace

extern "C" rest_status rest_paged_kv_write(void* d_k_pages, void* d_v_pages, const int64_t* page_strides, int32_t P,
                                           int32_t page, const int32_t* d_table, int64_t table_stride,
                                           int32_t table_cols, const int32_t* d_kv_len, const void* d_k_new,
                                           const void* d_v_new, const int64_t* new_strides, const int32_t* d_n_nodes,
                                           int32_t B, int32_t H_kv, int32_t N, int32_t D, void* stream) {
  if (B < 0 || H_kv < 1 || N < 0 || !new_strides) return REST_INVALID_ARG;
  if (B == 0 || N == 0) return REST_OK;
  if (!d_kv_len || !d_k_new || !d_v_new || !table_ok(d_table, table_stride, table_cols)) return REST_INVALID_ARG;
  Pool c;
  if (rest_status st = fill_pool(c, d_k_pages, d_v_pages, page_strides, d_table, table_stride, table_cols, P, H_kv, page, D))
    return st;
  if (!stride_ok(new_strides, 3) || !aligned16(d_k_new, d_v_new)) return REST_INVALID_ARG;
  const int row_vecs = H_kv * D / 8, chunks = (row_vecs + kWriteVecs - 1) / kWriteVecs;
  const int64_t units = (int64_t)B * N * 2 * chunks, blocks = (units + kWriteWarps - 1) / kWriteWarps;
  if (blocks > 0x7FFFFFFFll) return REST_UNSUPPORTED;
  REST_CUDA_TRY(launch(rest_paged_kv_write_kernel, dim3((unsigned)blocks), kWriteWarps * 32, 0, stream, c,
                       static_cast<const uint4*>(d_k_new), static_cast<const uint4*>(d_v_new), new_strides[0] / 8,
                       new_strides[1] / 8, new_strides[2] / 8, d_kv_len, d_n_nodes, units, (int)N, chunks, row_vecs,
                       log2_of(D / 8)));
  return REST_OK;
}

extern "C" rest_status rest_paged_kv_commit(void* d_k_pages, void* d_v_pages, const int64_t* page_strides, int32_t P,
                                            int32_t page, const int32_t* d_table, int64_t table_stride,
                                            int32_t table_cols, const int32_t* d_kv_len,
                                            const int32_t* d_accept_nodes, const int32_t* d_accept_len, int32_t B,
                                            int32_t H_kv, int32_t N, int32_t D, int32_t max_depth,
                                            int32_t* d_new_kv_len, void* stream) {
  if (B < 0 || H_kv < 1 || N < 1 || max_depth < 1) return REST_INVALID_ARG;
  if (B == 0) return REST_OK;
  if (!d_kv_len || !d_accept_nodes || !d_accept_len || !table_ok(d_table, table_stride, table_cols))
    return REST_INVALID_ARG;
  if (max_depth > kMaxDepth) return REST_UNSUPPORTED;
  Pool c;
  if (rest_status st = fill_pool(c, d_k_pages, d_v_pages, page_strides, d_table, table_stride, table_cols, P, H_kv, page, D))
    return st;
  REST_CUDA_TRY(launch(rest_paged_kv_commit_kernel, dim3((unsigned)B), kCommitThreads, 0, stream, c, d_kv_len,
                       d_accept_nodes, d_accept_len, (int)H_kv, (int)N, (int)max_depth, log2_of(D / 8),
                       d_new_kv_len));
  return REST_OK;
}

extern "C" rest_status rest_pages_copy(void* d_k_pages, void* d_v_pages, const int64_t* page_strides, int32_t P,
                                       int32_t page, int32_t H_kv, int32_t D, const int32_t* d_src,
                                       const int32_t* d_dst, int32_t n, void* stream) {
  if (n < 0 || H_kv < 1) return REST_INVALID_ARG;
  if (n == 0) return REST_OK;
  if (!d_src || !d_dst) return REST_INVALID_ARG;
  Pool c;
  if (rest_status st = fill_pool(c, d_k_pages, d_v_pages, page_strides, nullptr, 0, 0, P, H_kv, page, D)) return st;
  const int64_t vecs = (int64_t)H_kv * page * (D / 8), chunks = (vecs + kCopyVecs - 1) / kCopyVecs;
  if (vecs > (1 << 30) || chunks * n > 0x7FFFFFFFll) return REST_UNSUPPORTED;
  REST_CUDA_TRY(launch(rest_pages_copy_kernel, dim3((unsigned)(chunks * n), 2), kCopyThreads, 0, stream, c, d_src, d_dst,
                       (int)chunks, (int)vecs, log2_of(D / 8)));
  return REST_OK;
}

extern "C" rest_status rest_pages_fork(int32_t* d_refs, int32_t P, int32_t* d_table, int64_t table_stride,
                                       int32_t table_cols, int32_t* d_n_pages, int32_t* d_kv_len, int32_t B,
                                       int32_t page, const int32_t* d_parents, const int32_t* d_children, int32_t F,
                                       int32_t* d_copy_src, int32_t* d_copy_dst, int32_t* d_status, void* stream) {
  if (F < 0 || B < 1 || P < 1) return REST_INVALID_ARG;
  if (F == 0) return REST_OK;
  if (!d_refs || !d_n_pages || !d_kv_len || !d_parents || !d_children || !d_copy_src || !d_copy_dst || !d_status ||
      !table_ok(d_table, table_stride, table_cols))
    return REST_INVALID_ARG;
  if (!page_ok(page) || F > REST_MAX_FORKS || P > REST_MAX_PAGES) return REST_UNSUPPORTED;
  REST_CUDA_TRY(launch(rest_pages_fork_plan_kernel, dim3(1), kPlanThreads, 0, stream, d_parents, d_children, (int)F,
                       d_refs, (int)P, static_cast<const int32_t*>(d_table), table_stride, (int)table_cols, d_n_pages,
                       d_kv_len, (int)B, log2_of(page), d_copy_src, d_copy_dst, d_status));
  REST_CUDA_TRY(launch(rest_pages_fork_tables_kernel, dim3((unsigned)F), 128, 0, stream, d_parents, d_children, d_refs,
                       (int)P, d_table, table_stride, (int)table_cols, static_cast<const int32_t*>(d_kv_len),
                       log2_of(page), static_cast<const int32_t*>(d_copy_dst),
                       static_cast<const int32_t*>(d_status)));
  return REST_OK;
}

extern "C" rest_status rest_pages_reserve(int32_t* d_refs, int32_t P, int32_t* d_table, int64_t table_stride,
                                          int32_t table_cols, int32_t* d_n_pages, const int32_t* d_need_len, int32_t B,
                                          int32_t page, int32_t* d_status, void* stream) {
  if (B < 0 || P < 1) return REST_INVALID_ARG;
  if (B == 0) return REST_OK;
  if (!d_refs || !d_n_pages || !d_need_len || !d_status || !table_ok(d_table, table_stride, table_cols))
    return REST_INVALID_ARG;
  if (!page_ok(page) || B > REST_MAX_PAGED_CONTEXTS || P > REST_MAX_PAGES) return REST_UNSUPPORTED;
  REST_CUDA_TRY(launch(rest_pages_reserve_kernel, dim3(1), kPlanThreads, sizeof(int) * ((size_t)B + 1), stream, d_refs,
                       (int)P, d_table, table_stride, (int)table_cols, d_n_pages, d_need_len, (int)B, log2_of(page),
                       d_status));
  return REST_OK;
}

extern "C" rest_status rest_pages_release(int32_t* d_refs, int32_t P, int32_t* d_table, int64_t table_stride,
                                          int32_t table_cols, int32_t* d_n_pages, const int32_t* d_keep_len, int32_t B,
                                          int32_t page, int32_t window, int32_t sinks, void* stream) {
  if (B < 0 || P < 1 || window < 0 || sinks < 0) return REST_INVALID_ARG;
  if (B == 0) return REST_OK;
  if (!d_refs || !d_n_pages || !d_keep_len || !table_ok(d_table, table_stride, table_cols)) return REST_INVALID_ARG;
  if (!page_ok(page)) return REST_UNSUPPORTED;
  REST_CUDA_TRY(launch(rest_pages_release_kernel, dim3((unsigned)B), 128, 0, stream, d_refs, (int)P, d_table,
                       table_stride, (int)table_cols, d_n_pages, d_keep_len, log2_of(page), (int)window, (int)sinks));
  return REST_OK;
}
