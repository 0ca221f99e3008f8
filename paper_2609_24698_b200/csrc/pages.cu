// Pages of a paged pool: pages_assign, pages_free, pages_fork, pages_compact.
//
// Who holds what is decided by one CTA (the lists are short and each step needs the counts of the one before); the contents move in
// a kernel over all SMs, 16 KiB of one page of one plane at a time, through shared memory by bulk copies (six under way per CTA): a copy,
// bound by HBM, or by launches and latency for few pages.
// Pages are counted in the order of their numbers, so every result is the same whatever the order of execution: the only atomics
// are on whole numbers.
#include "tok_common.cuh"

namespace tsv {

namespace {

constexpr int kPlanThreads = 1024;
constexpr int kPlanWarps = kPlanThreads / 32;
constexpr int kScan = 16;                          // pages of a lane per round of a scan
constexpr int kCopyThreads = 256;
constexpr int kChunk = 16384;                      // bytes of a work item of the copy kernel
constexpr int kStages = 6, kStoreLag = 3;          // chunks of a CTA in shared memory; loads ahead of the stores
constexpr int kCopyCtas = 2;                       // CTAs per SM
constexpr int kArrays = 128;                       // planes and row arrays of a launch

struct Pool {
  int32_t *table, *ref;
  int32_t slots, max_pages, n_pages, page_tokens;
};
// Workspace: {pairs, used pages}, pairs of pages to copy, pairs of slots whose rows to copy, free pages / new numbers
struct Work {
  int32_t* head;
  int2 *pages, *rows;
  int32_t* list;
};
__host__ __device__ inline size_t pairs_room(int n_pages) { return n_pages / 2 + 1 > TSV_MAX_PAGE_LIST ? n_pages / 2 + 1 : TSV_MAX_PAGE_LIST; }
inline Work work_of(char* ws, int n_pages) {
  Work w;
  w.head = reinterpret_cast<int32_t*>(ws);
  w.pages = reinterpret_cast<int2*>(ws + 256);
  w.rows = w.pages + pairs_room(n_pages);
  w.list = reinterpret_cast<int32_t*>(w.rows + TSV_MAX_PAGE_LIST);
  return w;
}

// The sum over the warps before this one of a number that a warp's lanes have alike; the sum of all in s_warp[kPlanWarps].  By the whole CTA.
__device__ __forceinline__ int warps_before(int mine, int* s_warp /* [kPlanWarps + 1] */) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  __syncthreads();
  if (lane == 0) s_warp[warp] = mine;
  __syncthreads();
  if (warp == 0) {
    const int v = s_warp[lane];
    int x = v;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int y = __shfl_up_sync(0xffffffffu, x, o);
      if (lane >= o) x += y;
    }
    s_warp[lane] = x - v;
    if (lane == 31) s_warp[kPlanWarps] = x;
  }
  __syncthreads();
  return s_warp[warp];
}

// Goes over pages p0 .. p1 - 1 in rounds of kPlanThreads * kScan and calls emit(page, rank) for those with `want(page)`, rank counted from
// the lowest; stops behind the round that reaches `enough`.  Returns their number (of the rounds gone over).  By the whole CTA.
template <typename Want, typename Emit>
__device__ __forceinline__ int scan_pages(int p0, int p1, int enough, int* s_warp /* [kPlanWarps + 1] */, Want want, Emit emit) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  int total = 0;
  for (int64_t base = p0; base < p1 && total < enough; base += kPlanThreads * kScan) {
    const int64_t at = base + (int64_t)warp * 32 * kScan + lane;
    unsigned hit[kScan];
    int mine = 0;
#pragma unroll
    for (int k = 0; k < kScan; ++k) hit[k] = at + 32 * k < p1 && want((int)(at + 32 * k)) ? 1u : 0u;
#pragma unroll
    for (int k = 0; k < kScan; ++k) { hit[k] = __ballot_sync(0xffffffffu, hit[k]); mine += __popc(hit[k]); }
    int rank = total + warps_before(mine, s_warp);
#pragma unroll
    for (int k = 0; k < kScan; ++k) {
      if (hit[k] >> lane & 1u) emit((int)(at + 32 * k), rank + __popc(hit[k] & ((1u << lane) - 1u)));
      rank += __popc(hit[k]);
    }
    total += s_warp[kPlanWarps];
  }
  __syncthreads();
  return total;
}

struct ListCtl {
  int need[TSV_MAX_PAGE_LIST];        // fresh pages an entry wants; later the rank of its first one, -1: it gets none
  int key[TSV_MAX_PAGE_LIST];         // the slot an entry writes (-1: none)
  int other[TSV_MAX_PAGE_LIST];       // the slot it copies
  int warp[kPlanWarps + 1];
  int total;
};

// Is the slot that entry i writes written by an earlier entry, or copied by any?
__device__ __forceinline__ bool clash(const ListCtl& c, int i, int n, bool sources) {
  const int k = c.key[i];
  bool hit = false;
  for (int j = 0; j < n; ++j) hit |= (j < i && c.key[j] == k) || (sources && c.other[j] == k);
  return hit;
}

// Entries in order take their pages out of `left`; an entry for which too few are left takes none.  By thread 0.
__device__ __forceinline__ void grant(ListCtl& c, int n, int left, int32_t* status) {
  int at = 0;
  for (int i = 0; i < n; ++i) {
    const int want = c.need[i];
    if (want < 0) continue;
    if (want > left - at) { c.need[i] = -1; atomicOr(status + i, TSV_ST_POOL); continue; }
    c.need[i] = at;
    at += want;
  }
}

// pages_assign (FORK = false) and pages_fork: what entry i wants is counted by a warp, then the free pages are listed, then the entries
// get theirs.
template <bool FORK>
__global__ void __launch_bounds__(kPlanThreads) list_kernel(const Pool p, const int n, const int32_t* src, const int32_t* dst, const int32_t* first,
                                                            const int32_t* last, const int32_t* L, const Work w, int32_t* status) {
  __shared__ ListCtl c;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  if (tid < n) {
    const int k = dst[tid], o = FORK ? src[tid] : -1;
    c.key[tid] = k >= 0 && k < p.slots ? k : -1;        // (what a refused entry names counts against the others all the same)
    c.other[tid] = o >= 0 && o < p.slots ? o : -1;
    c.need[tid] = 0;
  }
  if (tid == 0) c.total = 0;
  __syncthreads();
  bool bad = false;
  if (tid < n) bad = c.key[tid] < 0 || (FORK && c.other[tid] < 0) || clash(c, tid, n, FORK);
  if (bad) c.need[tid] = -1;
  __syncthreads();
  for (int i = warp; i < n; i += kPlanWarps) {
    if (c.need[i] < 0) continue;                        // (warp-uniform)
    const int32_t* to = p.table + (size_t)c.key[i] * p.max_pages;
    int want = 0;
    bool wrong = false;
    if (FORK) {
      const int32_t* from = p.table + (size_t)c.other[i] * p.max_pages;
      const int len = L[c.other[i]], whole = len / p.page_tokens;
      wrong = len < 0 || (int64_t)len > (int64_t)p.max_pages * p.page_tokens;
      for (int lp = lane; lp < p.max_pages; lp += 32) {
        const int pg = from[lp];
        wrong |= to[lp] != -1 || pg < -1 || pg >= p.n_pages || (pg >= 0 && p.ref[pg] < 1);
        want += pg >= 0 && lp >= whole;
      }
    } else {
      const int f = first[i], l = last[i];
      wrong = f < 0 || l > p.max_pages || f > l;
      if (!wrong) for (int lp = f + lane; lp < l; lp += 32) want += to[lp] < 0;
    }
    for (int o = 16; o; o >>= 1) want += __shfl_xor_sync(0xffffffffu, want, o);
    wrong = __any_sync(0xffffffffu, wrong);
    if (lane == 0) {
      c.need[i] = wrong ? -1 : want;
      if (!wrong) atomicAdd(&c.total, want);
    }
  }
  __syncthreads();
  if (tid < n && c.need[tid] < 0) atomicOr(status + tid, TSV_ST_PAGE);
  const int wanted = c.total;
  // (every want is asked of the same list: none that is refused changes another's pages)
  const int found = wanted ? scan_pages(0, p.n_pages, wanted, c.warp, [&](int pg) { return p.ref[pg] == 0; },
                                        [&](int pg, int rank) { if (rank < wanted) w.list[rank] = pg; }) : 0;
  if (tid == 0) {
    grant(c, n, min(found, wanted), status);
    if (FORK) w.head[0] = n;
  }
  __syncthreads();
  for (int i = warp; i < n; i += kPlanWarps) {
    int at = c.need[i];
    if (FORK && lane == 0) { w.pages[i] = make_int2(-1, -1); w.rows[i] = at < 0 ? make_int2(-1, -1) : make_int2(c.other[i], c.key[i]); }
    __syncwarp();
    if (at < 0) continue;
    int32_t* to = p.table + (size_t)c.key[i] * p.max_pages;
    const int32_t* from = FORK ? p.table + (size_t)c.other[i] * p.max_pages : nullptr;
    const int len = FORK ? L[c.other[i]] : 0, whole = FORK ? len / p.page_tokens : 0;
    const int f = FORK ? 0 : first[i], l = FORK ? p.max_pages : last[i];
    for (int base = f; base < l; base += 32) {
      const int lp = base + lane;
      const int pg = FORK && lp < l ? from[lp] : -1;
      const bool fresh = lp < l && (FORK ? pg >= 0 && lp >= whole : to[lp] < 0);
      const unsigned m = __ballot_sync(0xffffffffu, fresh);
      if (fresh) {
        const int mine = w.list[at + __popc(m & ((1u << lane) - 1u))];
        to[lp] = mine;
        p.ref[mine] = 1;
        if (FORK && lp == whole && len % p.page_tokens) w.pages[i] = make_int2(pg, mine);
      } else if (pg >= 0) {
        to[lp] = pg;
        atomicAdd(p.ref + pg, 1);
      }
      at += __popc(m);
    }
  }
}

// A warp per entry.  A table word is taken by an exchange, so that of two entries with the same page of a slot one gives it up.
__global__ void __launch_bounds__(kCopyThreads) free_kernel(const Pool p, const int n, const int32_t* slot, const int32_t* first, const int32_t* last,
                                                            int32_t* status) {
  const int i = (blockIdx.x * kCopyThreads + threadIdx.x) >> 5, lane = threadIdx.x & 31;
  if (i >= n) return;
  const int k = slot[i], f = first[i], l = last[i];
  bool wrong = k < 0 || k >= p.slots || f < 0 || l > p.max_pages || f > l;
  if (!wrong)
    for (int lp = f + lane; lp < l; lp += 32) {
      const int pg = atomicExch(p.table + (size_t)k * p.max_pages + lp, -1);
      if (pg == -1) continue;
      if (pg < 0 || pg >= p.n_pages) { wrong = true; continue; }
      if (atomicSub(p.ref + pg, 1) < 1) { atomicAdd(p.ref + pg, 1); wrong = true; }    // (nobody held it)
    }
  if (wrong) atomicOr(status + i, TSV_ST_PAGE);
}

__global__ void __launch_bounds__(kPlanThreads) compact_kernel(const Pool p, const Work w, int32_t* n_used) {
  __shared__ int s_warp[kPlanWarps + 1];
  int used, moves;
  if (p.n_pages <= kPlanThreads * kScan) {                // the counts stay in registers (three scans of them: a call of few pages 27.6 us instead of 23.5)
    const int lane = threadIdx.x & 31, at = (threadIdx.x >> 5) * 32 * kScan + lane;
    unsigned held = 0;
    int mine = 0;
#pragma unroll
    for (int k = 0; k < kScan; ++k) held |= (at + 32 * k < p.n_pages && p.ref[at + 32 * k] != 0 ? 1u : 0u) << k;
#pragma unroll
    for (int k = 0; k < kScan; ++k) mine += __popc(__ballot_sync(0xffffffffu, held >> k & 1u));
    warps_before(mine, s_warp);
    used = s_warp[kPlanWarps];
    unsigned hole[kScan], far[kScan];
    mine = 0;                                             // holes below, pages beyond: 16 bits each (at most 8192 of each)
#pragma unroll
    for (int k = 0; k < kScan; ++k) {
      const int pg = at + 32 * k;
      hole[k] = __ballot_sync(0xffffffffu, pg < used && !(held >> k & 1u));
      far[k] = __ballot_sync(0xffffffffu, pg >= used && (held >> k & 1u));
      mine += __popc(hole[k]) + (__popc(far[k]) << 16);
    }
    int rank = warps_before(mine, s_warp);
    moves = s_warp[kPlanWarps] & 0xffff;
#pragma unroll
    for (int k = 0; k < kScan; ++k) {
      const int pg = at + 32 * k;
      const unsigned below = (1u << lane) - 1u;
      if (hole[k] >> lane & 1u) w.pages[(rank & 0xffff) + __popc(hole[k] & below)].y = pg;
      if (far[k] >> lane & 1u) w.pages[(rank >> 16) + __popc(far[k] & below)].x = pg;
      if (pg >= used && pg < p.n_pages) w.list[pg] = pg;
      rank += __popc(hole[k]) + (__popc(far[k]) << 16);
    }
    __syncthreads();
  } else {
    used = scan_pages(0, p.n_pages, p.n_pages + 1, s_warp, [&](int pg) { return p.ref[pg] != 0; }, [](int, int) {});
    scan_pages(0, used, p.n_pages + 1, s_warp, [&](int pg) { return p.ref[pg] == 0; }, [&](int pg, int rank) { w.pages[rank].y = pg; });
    moves = scan_pages(used, p.n_pages, p.n_pages + 1, s_warp, [&](int pg) { w.list[pg] = pg; return p.ref[pg] != 0; },
                       [&](int pg, int rank) { w.pages[rank].x = pg; });
  }
  for (int i = threadIdx.x; i < moves; i += kPlanThreads) {
    const int2 m = w.pages[i];
    w.list[m.x] = m.y;
    p.ref[m.y] = p.ref[m.x];
    p.ref[m.x] = 0;
  }
  if (threadIdx.x == 0) { w.head[0] = moves; w.head[1] = used; *n_used = used; }
}

struct CopyArgs {
  char* base[kArrays];
  int64_t bytes[kArrays];
  int32_t chunk0[kArrays + 1];      // work items of the arrays before
  int32_t n, n_planes;              // arrays of this launch; the first n_planes of them are planes
  Work w;
  Pool p;
  int32_t compact;                  // `failed` is n_used, else status
  int32_t renumber;                 // the table's words become the new numbers (compact)
  int32_t* failed;                  // where a copy that never came is told of
  int32_t n_failed;
  uint32_t tries;                   // of a wait for a copy
};

// Thread 0 moves the planes' chunks: a load into the next stage once the store out of it has been read, a store three chunks behind the
// loads.  The other warps copy the row arrays, which may be of 4-byte alignment, and renumber the table.
// (Loads and stores through registers, 8 vectors of a thread: 289 MB of scattered pages 124 us instead of 111.)
__global__ void __launch_bounds__(kCopyThreads) copy_kernel(const __grid_constant__ CopyArgs a) {
  extern __shared__ __align__(128) unsigned char stage[];
  __shared__ __align__(8) uint64_t bars[kStages];
  const int tid = threadIdx.x, pairs = a.w.head[0];
  const int planes = min(a.n, a.n_planes), per_plane = a.chunk0[planes], per_row = a.chunk0[a.n] - per_plane;
  if (tid == 0) {
    const uint32_t at = (uint32_t)__cvta_generic_to_shared(stage), bar = (uint32_t)__cvta_generic_to_shared(bars);
    for (int i = 0; i < kStages; ++i) bulk_bar_init(bar + 8 * i, 1);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    const int64_t items = (int64_t)pairs * per_plane;
    char* to[kStages];
    uint32_t size[kStages];
    int64_t item = blockIdx.x;
    int loaded = 0, stored = 0;                            // chunks so far
    bool fail = false;
    // one round of the stages, unrolled: what a stage is for stays in registers
    while (!fail && (item < items || stored < loaded)) {
#pragma unroll
      for (int st = 0; st < kStages; ++st) {
        if (!fail && item < items && loaded - stored <= kStoreLag && loaded % kStages == st) {
          const int i = (int)(item / per_plane), c = (int)(item - (int64_t)i * per_plane);
          int lo = 0, hi = planes;                         // the plane of this chunk
          while (hi - lo > 1) { const int mid = (lo + hi) >> 1; if (a.chunk0[mid] <= c) lo = mid; else hi = mid; }
          const int2 pr = a.w.pages[i];
          const int64_t bytes = a.bytes[lo], off = (int64_t)(c - a.chunk0[lo]) * kChunk;
          item += gridDim.x;
          size[st] = pr.x < 0 ? 0 : (uint32_t)(bytes - off < kChunk ? bytes - off : kChunk);
          to[st] = a.base[lo] + pr.y * bytes + off;
          bulk_wait_read<kStages - kStoreLag - 1>();       // (the store out of this stage has been read)
          bulk_expect(bar + 8 * st, size[st]);
          if (size[st]) bulk_load(at + st * kChunk, a.base[lo] + pr.x * bytes + off, size[st], bar + 8 * st);
          ++loaded;
        }
        const int sst = (st + kStages - kStoreLag) % kStages;      // (the store that is due behind this load)
        if (!fail && stored < loaded && stored % kStages == sst && (loaded - stored > kStoreLag || item >= items)) {
          fail = !bulk_bar_wait(bar + 8 * sst, (stored / kStages) & 1, a.tries);
          if (!fail) {
            if (size[sst]) bulk_store(to[sst], at + sst * kChunk, size[sst]);
            bulk_commit();
            ++stored;
          }
        }
      }
    }
    bulk_wait();
    if (fail) {                                            // (an internal error)
      for (int i = 0; i < a.n_failed; ++i) { if (a.compact) a.failed[i] = -1; else atomicOr(a.failed + i, TSV_ST_INTERNAL); }
      // (no load is under way into shared memory when this CTA gives it up)
      for (; stored < loaded; ++stored) bulk_bar_wait(bar + 8 * (stored % kStages), (stored / kStages) & 1, kBulkTries);
    }
  } else if (tid >= 32) {
    const int t = tid - 32, n = kCopyThreads - 32;
    const int64_t items = (int64_t)pairs * per_row;
    for (int64_t item = blockIdx.x; item < items; item += gridDim.x) {
      const int i = (int)(item / per_row), c = per_plane + (int)(item - (int64_t)i * per_row);
      int lo = planes, hi = a.n;
      while (hi - lo > 1) { const int mid = (lo + hi) >> 1; if (a.chunk0[mid] <= c) lo = mid; else hi = mid; }
      const int2 pr = a.w.rows[i];
      if (pr.x < 0) continue;
      const int64_t bytes = a.bytes[lo], off = (int64_t)(c - a.chunk0[lo]) * kChunk;
      const char* src = a.base[lo] + pr.x * bytes + off;
      char* dst = a.base[lo] + pr.y * bytes + off;
      const int left = (int)(bytes - off < kChunk ? bytes - off : kChunk);
      if ((((uintptr_t)src | (uintptr_t)dst | (uintptr_t)left) & 15) == 0)
        for (int k = t * 16; k < left; k += n * 16) *reinterpret_cast<uint4*>(dst + k) = *reinterpret_cast<const uint4*>(src + k);
      else
        for (int k = t * 4; k < left; k += n * 4) *reinterpret_cast<uint32_t*>(dst + k) = *reinterpret_cast<const uint32_t*>(src + k);
    }
    if (a.renumber) {
      const int used = a.w.head[1];
      const int64_t words = (int64_t)a.p.slots * a.p.max_pages;
      for (int64_t i = (int64_t)blockIdx.x * n + t; i < words; i += (int64_t)gridDim.x * n) {
        const int pg = a.p.table[i];
        if (pg >= used && pg < a.p.n_pages) a.p.table[i] = a.w.list[pg];
      }
    }
  }
}

Pool pool_of(const tsv_page_pool& p) { return {p.page_table, p.ref, p.slots, p.max_pages, p.n_pages, p.page_tokens}; }

int launch_copies(const tsv_page_pool& p, const Work& w, bool rows, int64_t most_pairs, bool renumber, int32_t* failed, int n_failed, cudaStream_t st) {
  const int total = p.n_planes + (rows ? p.n_rows : 0);
  TSV_PREP(copy_kernel);
  if (!ensure_smem((const void*)copy_kernel, kStages * kChunk)) return TSV_ERR_CUDA;
  for (int at = 0; at < total || (at == 0 && renumber); at += kArrays) {
    CopyArgs a;
    a.n = total - at < kArrays ? total - at : kArrays;
    a.n_planes = p.n_planes - at < 0 ? 0 : p.n_planes - at;
    a.w = w; a.p = pool_of(p);
    a.compact = renumber;
    a.renumber = renumber && at == 0;
    a.failed = failed; a.n_failed = n_failed;
    a.tries = wait_tries(kBulkTries);
    int64_t chunks = 0;
    for (int i = 0; i < a.n; ++i) {
      const tsv_page_array& x = at + i < p.n_planes ? p.planes[at + i] : p.rows[at + i - p.n_planes];
      a.base[i] = reinterpret_cast<char*>(x.base); a.bytes[i] = x.bytes; a.chunk0[i] = (int32_t)chunks;
      chunks += (x.bytes + kChunk - 1) / kChunk;
    }
    a.chunk0[a.n] = (int32_t)chunks;                        // (at most 2^16 of each array: check_pool)
    int64_t grid = most_pairs * chunks;
    if (renumber && grid < 32) grid = 32;
    if (grid > 148 * kCopyCtas) grid = 148 * kCopyCtas;
    if (grid < 1) grid = 1;
    copy_kernel<<<(unsigned)grid, kCopyThreads, kStages * kChunk, st>>>(a);
    count_launch();
  }
  return cudaGetLastError() == cudaSuccess ? TSV_OK : TSV_ERR_CUDA;
}

}  // namespace

size_t pages_workspace(const tsv_page_pool& p) {
  return 256 + (pairs_room(p.n_pages) + TSV_MAX_PAGE_LIST) * sizeof(int2) + ((size_t)p.n_pages * sizeof(int32_t) + 255) / 256 * 256;
}

int launch_pages_assign(const tsv_page_pool& p, int n, const int32_t* slot, const int32_t* first, const int32_t* last, char* ws, int32_t* status,
                        cudaStream_t st) {
  TSV_PREP(list_kernel<false>);
  list_kernel<false><<<1, kPlanThreads, 0, st>>>(pool_of(p), n, nullptr, slot, first, last, nullptr, work_of(ws, p.n_pages), status);
  count_launch();
  return cudaGetLastError() == cudaSuccess ? TSV_OK : TSV_ERR_CUDA;
}

int launch_pages_free(const tsv_page_pool& p, int n, const int32_t* slot, const int32_t* first, const int32_t* last, int32_t* status, cudaStream_t st) {
  TSV_PREP(free_kernel);
  free_kernel<<<(n * 32 + kCopyThreads - 1) / kCopyThreads, kCopyThreads, 0, st>>>(pool_of(p), n, slot, first, last, status);
  count_launch();
  return cudaGetLastError() == cudaSuccess ? TSV_OK : TSV_ERR_CUDA;
}

int launch_pages_fork(const tsv_page_pool& p, int n, const int32_t* src, const int32_t* dst, const int32_t* L, char* ws, int32_t* status, cudaStream_t st) {
  const Work w = work_of(ws, p.n_pages);
  TSV_PREP(list_kernel<true>);
  list_kernel<true><<<1, kPlanThreads, 0, st>>>(pool_of(p), n, src, dst, nullptr, nullptr, L, w, status);
  count_launch();
  return launch_copies(p, w, true, n, false, status, n, st);
}

int launch_pages_compact(const tsv_page_pool& p, int32_t* n_used, char* ws, cudaStream_t st) {
  const Work w = work_of(ws, p.n_pages);
  TSV_PREP(compact_kernel);
  compact_kernel<<<1, kPlanThreads, 0, st>>>(pool_of(p), w, n_used);
  count_launch();
  return launch_copies(p, w, false, p.n_pages / 2, true, n_used, 1, st);
}

}  // namespace tsv
