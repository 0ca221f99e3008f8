// Shared pieces of the window_sink_attn kernels: the key list of a tile of query rows, its masks, the rows behind it, and the
// exact recomputation of single rows.
//
// The rows of one sequence and key head are ordered token by token, the G = H / Hk query heads of a token next to each other: row r
// is token r / G, head hk * G + r % G.  A tile is a range of them, and its keys are a LIST: sinks 0 .. ns - 1, then the positions
// lo .. (those of them that are new tokens' come from the call's rows), in a tree then its nodes.  Every key of the list is
// visible to some query of the sequence; which query sees which is the mask's.
#pragma once
#include "tok_common.cuh"

namespace tsv {

struct AttnArgs {
  tsv_tok_shape s;
  tsv_tok_cache c;
  tsv_tok_batch bt;
  tsv_tok_rows in;
  void* out;
  float* po;                // partial outputs [row tiles][splits][rows of a tile][d], their {max, sum} behind them
  float2* pml;
  int32_t G;                // H / Hk
  int32_t nsplit;           // shares that a tile's keys are cut into
  int32_t cluster;          // the shares are a cluster's CTAs, which join them (16-row tiles), and not partial outputs
  float scale2;             // softmax scale * log2(e): scores in powers of two
  int32_t* status;
};

// The tensor-core path (tok_attn_tc.cu).  `units`: tiles over all sequences (a bound), of tc_tile rows; tc_halves CTAs share one's columns.
int launch_attn_tc(const AttnArgs& a, int64_t units, cudaStream_t st);
inline int tc_tile(int d) { return d > 128 ? 128 : 256; }
inline int tc_halves(int d) { return d > 256 ? 2 : 1; }

struct TileList {
  int b, n, L, G;
  int64_t row0;
  int hk, r0, nr;           // key head; first row and rows of the tile
  int ns, lo, nc, nk;       // sinks, first position of the window part, keys that are positions, keys
  int p0, p1;               // positions of the tile's first and last token (chain)
  int ok;                   // 0: no such tile, 1: a tile, 2: its rows are zero
};

// What a row of the list is: a row of the cache (>= 0), a new row (-2 - row), or nothing (-1: a missing page).
__device__ __forceinline__ int64_t list_row(const AttnArgs& a, const TileList& t, int kk) {
  if (kk >= t.nc) return -2 - (t.row0 + kk - t.nc);
  const int pos = kk < t.ns ? kk : t.lo + kk - t.ns;
  if (pos >= t.L) return -2 - (t.row0 + pos - t.L);
  return tok_cache_row(a.c, a.s.window, a.s.n_sink, t.b, pos);
}
template <typename T>
__device__ __forceinline__ const T* row_ptr(const AttnArgs& a, int hk, int64_t code, bool value) {
  const bool v = value && a.c.v;
  if (code >= 0) return reinterpret_cast<const T*>(v ? a.c.v : a.c.k) + (code * a.s.Hk + hk) * a.s.d;
  return reinterpret_cast<const T*>(v ? a.in.v : a.in.k) + (-2 - code) * (v ? a.in.v_ld : a.in.k_ld) + (size_t)hk * a.s.d;
}

// Does the query at position p (in a tree: with ancestors anc) see key kk of the list?
__device__ __forceinline__ bool list_sees(const AttnArgs& a, const TileList& t, const int* depth, int p, uint32_t anc, int kk) {
  int pos = kk < t.ns ? kk : t.lo + kk - t.ns;
  if (kk >= t.nc) {
    const int j = kk - t.nc;
    if (!(anc >> j & 1u)) return false;
    pos = t.L + depth[j];
  }
  return pos <= p && (pos > p - a.s.window || pos < a.s.n_sink);
}

// The tile that item number `item` (units of `per` rows, over all sequences) of key head hk is; by one warp, lane 0's result counts.
// depth, anc: shared, TSV_MAX_D each, filled for trees.
__device__ __forceinline__ TileList make_list(const AttnArgs& a, int64_t item, int hk, int per, int* depth, uint32_t* anc) {
  TileList t;
  TokUnit u;
  t.ok = 0;
  if (!find_unit(a.s, a.bt, a.c.L, a.G, per, item, a.status, u)) return t;
  const int lane = threadIdx.x & 31;
  t.b = u.b; t.n = u.n; t.row0 = u.row0; t.G = a.G; t.hk = hk;
  t.L = u.L;
  t.r0 = u.unit * per;
  t.nr = (int)min((int64_t)per, (int64_t)u.n * a.G - t.r0);
  int st = t.L < 0 || (int64_t)t.L + u.n > a.s.max_L ? TSV_ST_LENGTH : 0;
  if (a.bt.parent) {
    int dep;
    uint32_t an;
    st |= tok_tree(a.bt, u, dep, an);
    depth[lane] = dep; anc[lane] = an;
  }
  t.ok = st ? 2 : 1;
  if (st) { if (lane == 0) atomicOr(a.status + u.b, st); return t; }
  const int t0 = t.r0 / a.G, t1 = (t.r0 + t.nr - 1) / a.G;
  t.p0 = t.L + t0; t.p1 = t.L + t1;
  t.lo = max(0, (a.bt.parent ? t.L : t.p0) - a.s.window + 1);
  t.ns = min(a.s.n_sink, t.lo);
  t.nc = t.ns + (a.bt.parent ? t.L : t.p1 + 1) - t.lo;
  t.nk = t.nc + (a.bt.parent ? t.n : 0);
  return t;
}

// The kernels multiply the values of unseen keys by an exact zero, which is not enough where a value is infinite or NaN.  So a tile with
// a result that is not finite is computed a second time, with such values taken as zero: then what a row does not see has no
// influence on its bits.  Rows that DO see something not finite, and those whose sums are beyond the range although their result is not
// (values near the largest, in the first sum by the weights of up to 2^10 of the tensor-core path), are then computed by the definition:
//
// One row, by one warp: keys k0 .. k1 - 1 of the list, what the row does not see skipped altogether.  Returns whether a score or a
// value that it sees is not finite.  m in units of log2; o[i]: dims lane + 32 i, with weights that add up to one, which no sum of finite
// values leaves the range by; l: the sum of weights at the maximum m, NEGATIVE as a mark that o is divided by it.  Where nothing is seen m is
// -inf, l and o zero.  Where every score seen is -inf, the weights are 0 / 0 if these are all keys of the row (l NaN); in a share of them the
// others decide the weights of these, zero, which leave what is not finite NaN (m -inf, l -1, o the values times zero).
__device__ __forceinline__ bool is_finite(float x) { return fabsf(x) < INFINITY; }
template <typename T>
__device__ __noinline__ bool exact_row(const AttnArgs& a, const TileList& t, const int* depth, const T* q, int p, uint32_t anc, int k0, int k1,
                                       float& m, float& l, float* o) {
  const int lane = threadIdx.x & 31, d = a.s.d;
  m = -INFINITY; l = 0.f;
  bool nan = false, saw = false, any = false;
#pragma unroll
  for (int i = 0; i < 16; ++i) o[i] = 0.f;
  float inv = 0.f;
  for (int pass = 0; pass < 2; ++pass) {
    for (int kk = k0; kk < k1; ++kk) {
      if (!list_sees(a, t, depth, p, anc, kk)) continue;
      const int64_t code = list_row(a, t, kk);
      if (code == -1) continue;
      const T* k = row_ptr<T>(a, t.hk, code, false);
      float x = 0.f;
      for (int e = lane; e < d; e += 32) x = fmaf(to_f(q[e]), to_f(k[e]), x);
      x = warp_sum(x) * a.scale2;
      if (pass == 0) {
        any = true; nan |= isnan(x); saw |= !is_finite(x);
        const float to = fmaxf(m, x);
        if (to != -INFINITY) l = l * exp2f(m - to) + exp2f(x - to);
        m = to;
        continue;
      }
      const float w = m == -INFINITY ? 0.f : exp2f(x - m) * inv;
      const T* v = row_ptr<T>(a, t.hk, code, true);
#pragma unroll
      for (int i = 0; i < 16; ++i)
        if (lane + 32 * i < d) {
          const float y = to_f(v[lane + 32 * i]);
          saw |= !is_finite(y);
          o[i] = fmaf(w, y, o[i]);
        }
    }
    inv = 1.f / l;
  }
  if (m == -INFINITY && any) l = a.nsplit == 1 ? NAN : 1.f;
  l = nan ? NAN : -l;
  return __any_sync(0xffffffffu, saw);
}
// 16 bytes in shared memory, infinities and NaN taken as zero.
__device__ __forceinline__ uint32_t finite_word(uint32_t w, bf16) {
  if ((w & 0x7F80u) == 0x7F80u) w &= 0xFFFF0000u;
  if ((w & 0x7F800000u) == 0x7F800000u) w &= 0xFFFFu;
  return w;
}
__device__ __forceinline__ uint32_t finite_word(uint32_t w, float) { return (w & 0x7F800000u) == 0x7F800000u ? 0u : w; }
template <typename T>
__device__ __forceinline__ void make_finite(void* p) {
  uint4 v = *reinterpret_cast<uint4*>(p);
  v.x = finite_word(v.x, T()); v.y = finite_word(v.y, T()); v.z = finite_word(v.z, T()); v.w = finite_word(v.w, T());
  *reinterpret_cast<uint4*>(p) = v;
}

}  // namespace tsv
