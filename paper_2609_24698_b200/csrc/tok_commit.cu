// token_commit: rows of new tokens (a chain, or the accepted path of a tree) into the token cache, then L += count.
//
// A copy: bound by HBM, by latency for the few rows of a tree.  Where a sequence has at most 64 rows to give, one CTA copies them
// and moves L itself: one launch.  With more, CTAs share the rows and a second kernel moves L when all of them have read it.
#include "tok_common.cuh"

namespace tsv {

namespace {

constexpr int kCommitThreads = 256;
constexpr int kCommitBytes = 65536;      // shared memory of a CTA where several share a sequence: up to 64 rows of all planes

struct CommitArgs {
  tsv_tok_shape s;
  tsv_tok_cache c;
  tsv_tok_batch bt;
  const void *k, *v;
  int64_t k_bytes, v_bytes;              // of a packed row's stride
  const int32_t *path, *count;
  int32_t path_ld, row_vecs;             // 16-byte vectors of a row
  int32_t unit_rows;                     // rows of a CTA where several share a sequence
  uint32_t tries;                        // of a wait for copies
  int32_t* status;
};

// What sequence b gives, by the whole CTA alike: its count, 0 if it is flagged.  All rows of the sequence are looked over by every
// CTA that takes part of them, so that either all of them are written or none.
__device__ __forceinline__ int commit_count(const CommitArgs& a, int b, int n, int L, int* s_bad) {
  const int cnt = a.count ? __ldg(a.count + b) : n;
  if (threadIdx.x == 0) {
    int st = 0;
    if (cnt < 0 || cnt > n || (a.path && cnt > a.path_ld)) st |= TSV_ST_NODES;
    if (L < 0 || (int64_t)L + n > a.s.max_L) st |= TSV_ST_LENGTH;
    *s_bad = st;
  }
  __syncthreads();
  if (!*s_bad) {
    int st = 0;
    if (a.path)
      for (int i = threadIdx.x; i < cnt; i += kCommitThreads) {
        const int node = __ldg(a.path + (size_t)b * a.path_ld + i);
        if (node < 0 || node >= n) st |= TSV_ST_NODES;
      }
    if (a.c.page_table && cnt > 0)
      for (int lp = L / a.c.page_tokens + threadIdx.x; lp <= (L + cnt - 1) / a.c.page_tokens; lp += kCommitThreads)
        if (tok_cache_row(a.c, a.s.window, a.s.n_sink, b, min(lp * a.c.page_tokens + a.c.page_tokens - 1, L + cnt - 1)) < 0) st |= TSV_ST_PAGE;
    if (st) atomicOr(s_bad, st);
    __syncthreads();
  }
  const int st = *s_bad;
  __syncthreads();
  if (st) {
    if (threadIdx.x == 0) atomicOr(a.status + b, st);
    return 0;
  }
  return cnt;
}

// Where pair t of the rows from i0 on (row and plane) comes from and goes to; nothing where a ring's slot gets a later row.
__device__ __forceinline__ void commit_pair(const CommitArgs& a, const TokUnit& u, int L, int cnt, int i0, int planes, int t, const void*& src, void*& dst) {
  const int plane = planes == 2 ? t & 1 : 0, i = i0 + (planes == 2 ? t >> 1 : t);
  if (!a.c.page_table && L + i >= a.s.n_sink && i < cnt - a.s.window) return;
  const int node = a.path ? __ldg(a.path + (size_t)u.b * a.path_ld + i) : i;
  const int64_t row = tok_cache_row(a.c, a.s.window, a.s.n_sink, u.b, L + i);
  src = reinterpret_cast<const char*>(plane ? a.v : a.k) + (u.row0 + node) * (plane ? a.v_bytes : a.k_bytes);
  dst = reinterpret_cast<char*>(plane ? a.c.v : a.c.k) + row * a.row_vecs * 16;
}

// Rows i0 .. i1 - 1 of what the sequence gives.  A warp takes every eighth of the (row, plane) pairs, 32 of them at a time: a lane
// looks up where one goes, then the warp copies one after the other, two under way at a time.
__device__ __forceinline__ void commit_rows(const CommitArgs& a, const TokUnit& u, int L, int cnt, int i0, int i1) {
  constexpr int W = kCommitThreads / 32;
  const int rv = a.row_vecs, planes = a.v ? 2 : 1, warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int pairs = (i1 - i0) * planes;
  for (int t0 = warp; t0 < pairs; t0 += 32 * W) {
    const int t = t0 + lane * W;
    unsigned long long src = 0, dst = 0;
    if (t < pairs) {
      const void* s = nullptr;
      void* d = nullptr;
      commit_pair(a, u, L, cnt, i0, planes, t, s, d);
      src = reinterpret_cast<unsigned long long>(s); dst = reinterpret_cast<unsigned long long>(d);
    }
    const int here = min(32, (pairs - t0 + W - 1) / W);
    for (int k = 0; k < here; k += 2) {
      const uint4* from[2];
      uint4* to[2];
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        from[e] = reinterpret_cast<const uint4*>(__shfl_sync(0xffffffffu, src, (k + e) & 31));
        to[e] = reinterpret_cast<uint4*>(__shfl_sync(0xffffffffu, dst, (k + e) & 31));
        if (k + e >= here) to[e] = nullptr;
      }
      for (int v0 = lane; v0 < rv; v0 += 128) {
        uint4 x[2][4];
#pragma unroll
        for (int e = 0; e < 2; ++e)
#pragma unroll
          for (int j = 0; j < 4; ++j) if (to[e] && v0 + 32 * j < rv) x[e][j] = __ldg(from[e] + v0 + 32 * j);
#pragma unroll
        for (int e = 0; e < 2; ++e)
#pragma unroll
          for (int j = 0; j < 4; ++j) if (to[e] && v0 + 32 * j < rv) to[e][v0 + 32 * j] = x[e][j];
      }
    }
  }
}

__global__ void __launch_bounds__(kCommitThreads) commit_seq_kernel(const CommitArgs a) {
  __shared__ int s_bad;
  TokUnit u;
  u.b = blockIdx.x; u.unit = 0;
  const int flags = a.status[u.b];                        // (read by every thread ahead of the first barrier, written behind it)
  u.n = tok_count(a.s, a.bt, u.b, nullptr, u.row0);
  if (u.n < 0 && threadIdx.x == 0) atomicOr(a.status + u.b, TSV_ST_NODES);
  if (u.n < 0) return;
  const int L = a.c.L[u.b];
  if (__syncthreads_or(flags)) return;
  const int cnt = commit_count(a, u.b, u.n, L, &s_bad);
  commit_rows(a, u, L, cnt, 0, cnt);
  if (threadIdx.x == 0 && cnt) a.c.L[u.b] = L + cnt;      // (every thread has read L before a barrier of commit_count)
}

// The rows of a unit through shared memory by bulk copies, a row and plane per thread: all of the CTA's loads are under way at once, then
// all of its stores.  (Through registers, a warp per row: 262 MB 62 us instead of 57.)
__global__ void __launch_bounds__(kCommitThreads) commit_rows_kernel(const CommitArgs a) {
  extern __shared__ __align__(128) unsigned char stage[];
  __shared__ __align__(8) uint64_t bar;
  __shared__ int s_bad, s_found;
  __shared__ TokUnit s_u;
  const uint32_t bar_at = (uint32_t)__cvta_generic_to_shared(&bar), at = (uint32_t)__cvta_generic_to_shared(stage);
  const int tid = threadIdx.x, planes = a.v ? 2 : 1, bytes = a.row_vecs * 16;
  if (tid < 32) {
    TokUnit u;
    const bool f = find_unit(a.s, a.bt, a.c.L, 1, a.unit_rows, blockIdx.x, a.status, u);
    if (tid == 0) {
      s_found = f && a.status[u.b] == 0; s_u = u;
      bulk_bar_init(bar_at, 1);
      asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
      asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    }
  }
  __syncthreads();
  if (!s_found) return;
  const TokUnit u = s_u;
  const int L = u.L, cnt = commit_count(a, u.b, u.n, L, &s_bad);
  const int i0 = u.unit * a.unit_rows, pairs = max(0, min(cnt, i0 + a.unit_rows) - i0) * planes;
  const void* src = nullptr;
  void* dst = nullptr;
  if (tid < pairs) commit_pair(a, u, L, cnt, i0, planes, tid, src, dst);
  const int copies = __syncthreads_count(src != nullptr);
  if (!copies) return;
  if (tid == 0) bulk_expect(bar_at, (uint32_t)copies * bytes);
  __syncthreads();
  if (src) bulk_load(at + tid * bytes, src, bytes, bar_at);
  if (src) {
    if (bulk_bar_wait(bar_at, 0, a.tries)) {
      bulk_store(dst, at + tid * bytes, bytes);
    } else {
      atomicOr(a.status + u.b, TSV_ST_INTERNAL);
      bulk_bar_wait(bar_at, 0, kBulkTries);               // (no copy is under way into shared memory when this CTA gives it up)
    }
    bulk_commit();
    bulk_wait();
  }
}

// Rows too wide for that: a row per CTA, through registers.
__global__ void __launch_bounds__(kCommitThreads) commit_wide_kernel(const CommitArgs a) {
  __shared__ int s_bad, s_found;
  __shared__ TokUnit s_u;
  if (threadIdx.x < 32) {
    TokUnit u;
    const bool f = find_unit(a.s, a.bt, a.c.L, 1, 1, blockIdx.x, a.status, u);
    if (threadIdx.x == 0) { s_found = f && a.status[u.b] == 0; s_u = u; }
  }
  __syncthreads();
  if (!s_found) return;
  const TokUnit u = s_u;
  const int L = u.L, cnt = commit_count(a, u.b, u.n, L, &s_bad);
  if (u.unit < cnt) commit_rows(a, u, L, cnt, u.unit, u.unit + 1);
}

__global__ void commit_lengths_kernel(const CommitArgs a) {
  const int b = blockIdx.x * blockDim.x + threadIdx.x;
  if (b >= a.s.B || a.status[b]) return;
  const int n = __ldg(a.bt.n + b), cnt = a.count ? __ldg(a.count + b) : n, L = a.c.L[b];
  int st = 0;
  if (n == 0) st = (cnt != 0 ? TSV_ST_NODES : 0) | (L < 0 || L > a.s.max_L ? TSV_ST_LENGTH : 0);      // (no CTA has looked at a sequence without tokens)
  if (st) atomicOr(a.status + b, st);
  else a.c.L[b] = L + cnt;
}

}  // namespace

int launch_token_commit(const tsv_tok_shape& s, const tsv_tok_cache& c, const tsv_tok_batch& bt, const tsv_tok_rows& in, const int32_t* path, int path_ld,
                        const int32_t* count, int32_t* status, cudaStream_t st) {
  const int es = s.dtype == TSV_BF16 ? 2 : 4;
  CommitArgs a = {s, c, bt, in.k, in.v, in.k_ld * es, in.v_ld * es, path, count, path_ld, s.Hk * s.d * es / 16, 0, wait_tries(kBulkTries), status};
  if (s.max_n <= 64) {
    TSV_PREP(commit_seq_kernel);
    commit_seq_kernel<<<s.B, kCommitThreads, 0, st>>>(a);
    count_launch();
  } else {
    const int row = a.row_vecs * 16 * (c.v ? 2 : 1);        // (at most 256 heads x 512 x 4 bytes x 2: too large for shared memory)
    if (row > 4 * kCommitBytes / 2) a.unit_rows = 0;
    else a.unit_rows = row >= kCommitBytes ? 1 : kCommitBytes / row > 64 ? 64 : kCommitBytes / row;
    const int64_t units = tok_units_bound(s, bt.rows, 1, a.unit_rows ? a.unit_rows : 1);
    if (units > 0x7fffffff) return TSV_ERR_LIMIT;
    TSV_PREP(commit_rows_kernel);
    TSV_PREP(commit_wide_kernel);
    TSV_PREP(commit_lengths_kernel);
    if (a.unit_rows) {
      const int smem = a.unit_rows * row;
      if (!ensure_smem((const void*)commit_rows_kernel, smem)) return TSV_ERR_CUDA;
      commit_rows_kernel<<<(unsigned)units, kCommitThreads, smem, st>>>(a);
    } else {
      commit_wide_kernel<<<(unsigned)units, kCommitThreads, 0, st>>>(a);
    }
    commit_lengths_kernel<<<(s.B + 127) / 128, 128, 0, st>>>(a);
    count_launch(2);
  }
  return cudaGetLastError() == cudaSuccess ? TSV_OK : TSV_ERR_CUDA;
}

}  // namespace tsv
