// Shared pieces of the token-level operators (qk_norm_rope, window_sink_attn, token_commit): the packed batch of new tokens,
// its draft trees, and the rows of the token cache.
#pragma once
#include "kernels.h"

namespace tsv {

// A piece of a sequence's new tokens: unit `unit` of `per` rows out of n[b] * rows_per_token, found by its number over the batch.
struct TokUnit {
  int b, unit, n, L;
  int64_t row0;
};

// New tokens of a sequence; -1 (flagged, where `status` is given) if its rows are not inside the packed arrays.
__device__ __forceinline__ int tok_count(const tsv_tok_shape& s, const tsv_tok_batch& bt, int b, int32_t* status, int64_t& row0) {
  const int n = __ldg(bt.n + b);
  row0 = __ldg(bt.row0 + b);
  if (n < 0 || n > s.max_n || row0 < 0 || row0 > bt.rows - n) {     // (row0 + n may pass 64 bits)
    if (status) atomicOr(status + b, TSV_ST_NODES);
    return -1;
  }
  return n;
}

// Warp-collective: which sequence unit number `item` belongs to (units of `per` rows, `rpt` rows per token); false behind the last.
// 64 sequences are requested at a time, their lengths (L_all) with them: the loads are what this costs.  (A prefix array made once would
// take another launch.)
__device__ __forceinline__ bool find_unit(const tsv_tok_shape& s, const tsv_tok_batch& bt, const int32_t* L_all, int rpt, int per, int64_t item, int32_t* status, TokUnit& u) {
  const int lane = threadIdx.x & 31;
  int64_t before = 0;
  for (int base = 0; base < s.B; base += 64) {
    int n[2], L[2];
    int64_t row0[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      n[h] = 0; row0[h] = 0; L[h] = 0;
      const int b = base + 32 * h + lane;
      if (b < s.B) { L[h] = L_all[b]; n[h] = max(0, tok_count(s, bt, b, status, row0[h])); }
    }
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int64_t units = ((int64_t)n[h] * rpt + per - 1) / per;
      int64_t x = units;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const int64_t y = __shfl_up_sync(0xffffffffu, x, o);
        if (lane >= o) x += y;
      }
      const unsigned hit = __ballot_sync(0xffffffffu, before + x > item);
      if (hit) {
        const int src = __ffs(hit) - 1;
        u.b = base + 32 * h + src;
        u.unit = (int)(item - before - __shfl_sync(0xffffffffu, x - units, src));
        u.n = __shfl_sync(0xffffffffu, n[h], src);
        u.L = __shfl_sync(0xffffffffu, L[h], src);
        u.row0 = __shfl_sync(0xffffffffu, row0[h], src);
        return true;
      }
      before += __shfl_sync(0xffffffffu, x, 31);
    }
  }
  return false;
}
// Units that a batch of `rows` packed rows can have at most.
inline int64_t tok_units_bound(const tsv_tok_shape& s, int64_t rows, int64_t rpt, int64_t per) {
  const int64_t by_rows = (rows * rpt + per - 1) / per + s.B, by_n = (int64_t)s.B * (((int64_t)s.max_n * rpt + per - 1) / per);
  return by_rows < by_n ? by_rows : by_n < 1 ? 1 : by_n;
}

// Facts of a draft tree for the lanes of one warp: lane i has node i's depth and the mask of its ancestors (itself included).
// Returns status bits (warp-uniform); a chain needs none of this.
__device__ __forceinline__ int tok_tree(const tsv_tok_batch& bt, const TokUnit& u, int& depth, uint32_t& anc) {
  const int lane = threadIdx.x & 31;
  depth = 0; anc = 0;
  if (u.n > TSV_MAX_D) return TSV_ST_PARENT;
  const int p = lane < u.n ? __ldg(bt.parent + u.row0 + lane) : -1;
  const bool bad = lane < u.n && (lane == 0 ? p != -1 : p < 0 || p >= lane);
  if (__any_sync(0xffffffffu, bad)) return TSV_ST_PARENT;
  int cur = p;
  if (lane < u.n) anc = 1u << lane;
  while (__any_sync(0xffffffffu, cur >= 0)) {             // (parents come before their children: this ends within n steps)
    if (cur >= 0) { anc |= 1u << cur; ++depth; }
    const int up = __shfl_sync(0xffffffffu, p, cur & 31);
    if (cur >= 0) cur = up;
  }
  return TSV_OK;
}

// Row of the token cache that holds position pos of sequence b; -1: no such page.  (Page sizes are powers of two nearly always, and a
// ring's turn is a subtraction where the position is less than a window beyond: a division is some forty instructions.)
__device__ __forceinline__ int64_t tok_cache_row(const tsv_tok_cache& c, int window, int n_sink, int b, int pos) {
  if (!c.page_table) {
    if (pos < n_sink) return (int64_t)b * ((int64_t)n_sink + window) + pos;
    int at = pos - n_sink;
    if (at >= window) { at -= window; if (at >= window) at %= window; }
    return (int64_t)b * ((int64_t)n_sink + window) + n_sink + at;
  }
  const int P = c.page_tokens;
  const bool pow2 = (P & (P - 1)) == 0;
  const int sh = 31 - __clz(P), lp = pow2 ? pos >> sh : pos / P, in = pow2 ? pos & (P - 1) : pos - lp * P;
  if (lp >= c.max_pages) return -1;
  const int page = __ldg(c.page_table + (size_t)b * c.max_pages + lp);
  const int64_t row = (int64_t)page * P + in;
  return page < 0 || row >= c.rows ? -1 : row;
}

// Asynchronous copies of whole 16-byte multiples through shared memory, without registers: global -> shared counted on an mbarrier, and
// back in groups.
__device__ __forceinline__ void bulk_load(uint32_t dst, const void* src, uint32_t bytes, uint32_t bar) {
  asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(dst), "l"(src), "r"(bytes), "r"(bar) : "memory");
}
__device__ __forceinline__ void bulk_store(void* dst, uint32_t src, uint32_t bytes) {
  asm volatile("cp.async.bulk.global.shared::cta.bulk_group [%0], [%1], %2;" ::"l"(dst), "r"(src), "r"(bytes) : "memory");
}
__device__ __forceinline__ void bulk_commit() { asm volatile("cp.async.bulk.commit_group;" ::: "memory"); }
template <int N> __device__ __forceinline__ void bulk_wait_read() { asm volatile("cp.async.bulk.wait_group.read %0;" ::"n"(N) : "memory"); }
__device__ __forceinline__ void bulk_wait() { asm volatile("cp.async.bulk.wait_group 0;" ::: "memory"); }
__device__ __forceinline__ void bulk_expect(uint32_t bar, uint32_t bytes) {
  asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(bytes) : "memory");
}
__device__ __forceinline__ void bulk_bar_init(uint32_t bar, uint32_t count) { asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(bar), "r"(count)); }
constexpr uint32_t kBulkTries = 1u << 14;      // of up to 4 us
__device__ __forceinline__ bool bulk_bar_wait(uint32_t bar, uint32_t parity, uint32_t tries) {
#pragma unroll 1
  for (uint32_t it = 0; it < tries; ++it) {
    uint32_t ok;
    asm volatile("{\n\t.reg .pred p;\n\tmbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2, %3;\n\tselp.b32 %0, 1, 0, p;\n\t}"
                 : "=r"(ok) : "r"(bar), "r"(parity), "r"(4000u) : "memory");
    if (ok) return true;
  }
  return false;
}

}  // namespace tsv
