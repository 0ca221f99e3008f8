// window_sink_attn: attention of packed new tokens over their sinks, their window and each other.
//
//   out = sum_j softmax_j(scale q.k_j) v_j,   j <= p and (j > p - window or j < n_sink); in a tree new tokens see ancestors only
//
// Kernels here: attn_mma_kernel (bf16, few rows per sequence: 16 query rows, mma.sync), attn_fp32_kernel (fp32: 16 query rows, FMAs), and
// attn_join_kernel, which joins the partial outputs of tiles whose keys were split over CTAs.  Calls with more rows: tok_attn_tc.cu.
#include <algorithm>

#include "tok_attn.cuh"
#include "tc_common.cuh"

namespace tsv {

namespace {

using tc::cp16;
using tc::cp_commit;
using tc::cp_wait;
using tc::ex2;
using tc::smem_u32;

constexpr int kRows = 16;             // query rows of a tile
constexpr int kThreads = 128;

// Keys of this share: a multiple of 16, the same number for every share.
__device__ __forceinline__ void split_range(const AttnArgs& a, const TileList& t, int& k0, int& k1) {
  const int per = ((t.nk + a.nsplit - 1) / a.nsplit + 15) & ~15;
  k0 = min(t.nk, (int)blockIdx.z * per);
  k1 = min(t.nk, k0 + per);
}
__device__ __forceinline__ size_t part_index(const AttnArgs& a) {      // of this CTA's first partial row
  return (((size_t)blockIdx.x * gridDim.y + blockIdx.y) * a.nsplit + blockIdx.z) * kRows;
}
template <typename T>
__device__ __forceinline__ T* out_row(const AttnArgs& a, const TileList& t, int r) {
  const int g = t.r0 + r;
  return reinterpret_cast<T*>(a.out) + ((t.row0 + g / t.G) * a.s.H + (size_t)t.hk * t.G + g % t.G) * a.s.d;
}
template <typename T>
__device__ __forceinline__ const T* query_row(const AttnArgs& a, const TileList& t, int r) {
  const int g = t.r0 + r;
  return reinterpret_cast<const T*>(a.in.q) + (t.row0 + g / t.G) * a.in.q_ld + ((size_t)t.hk * t.G + g % t.G) * a.s.d;
}
template <typename T>
__device__ __forceinline__ void zero_rows(const AttnArgs& a, const TileList& t) {
  float z[Vec<T>::N];
#pragma unroll
  for (int e = 0; e < Vec<T>::N; ++e) z[e] = 0.f;
  const int nv = a.s.d / Vec<T>::N;
  for (int i = threadIdx.x; i < t.nr * nv; i += blockDim.x) st16(out_row<T>(a, t, i / nv) + (i % nv) * Vec<T>::N, z);
}
// Position and ancestors of row r.
__device__ __forceinline__ void row_facts(const AttnArgs& a, const TileList& t, const int* depth, const uint32_t* anc, int r, int& p, uint32_t& an) {
  const int tok = (t.r0 + r) / t.G;
  p = t.L + (a.bt.parent ? depth[tok] : tok);
  an = a.bt.parent ? anc[tok] : 0;
}
__device__ __forceinline__ void cluster_sync() {
  asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
  asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
}
__device__ __forceinline__ uint32_t at_rank(uint32_t saddr, uint32_t rank) {
  uint32_t r;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(saddr), "r"(rank));
  return r;
}
__device__ __forceinline__ float2 ld_rank2(uint32_t addr) {
  float2 v;
  asm volatile("ld.shared::cluster.v2.f32 {%0, %1}, [%2];" : "=f"(v.x), "=f"(v.y) : "r"(addr) : "memory");
  return v;
}
__device__ __forceinline__ float4 ld_rank4(uint32_t addr) {
  float4 v;
  asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(addr) : "memory");
  return v;
}

// What both kernels keep of a tile, and its share of the result: sum of weights and of weighted values at the maximum m.
struct TileCtl {
  float2 ml[kRows];
  int depth[TSV_MAX_D];
  uint32_t anc[TSV_MAX_D];
  int pos[kRows];
  uint32_t row_anc[kRows];
  TileList t;
  uint32_t bad[2];                    // rows with a result that is not finite, after the first pass and after the second
};

// The tile of this CTA; false (alike in all CTAs of a cluster) where there is nothing to attend to.
template <typename T>
__device__ __forceinline__ bool begin_tile(const AttnArgs& a, TileCtl& sm) {
  if (threadIdx.x < 32) {
    const TileList t = make_list(a, blockIdx.x, blockIdx.y, kRows, sm.depth, sm.anc);
    if (threadIdx.x == 0) { sm.t = t; sm.bad[0] = sm.bad[1] = 0; }
  }
  __syncthreads();
  const TileList& t = sm.t;
  if (t.ok != 1) {
    if (t.ok == 2 && (a.nsplit == 1 || (a.cluster && blockIdx.z == 0))) zero_rows<T>(a, t);
    return false;
  }
  if (threadIdx.x < kRows) {
    int p = 0;
    uint32_t an = 0;
    if ((int)threadIdx.x < t.nr) row_facts(a, t, sm.depth, sm.anc, threadIdx.x, p, an);
    sm.pos[threadIdx.x] = p; sm.row_anc[threadIdx.x] = an;
  }
  return true;
}

// From o [16][ld] and sm.ml in shared memory, written by this CTA before, to the output: through the partial outputs, or at once, the
// shares of a cluster's CTAs joined in order.  Rows of sm.bad[0] that see something not finite, and those of sm.bad[1], are computed by
// definition first.
__device__ __forceinline__ bool all_finite(const float4& x) { return is_finite(x.x) && is_finite(x.y) && is_finite(x.z) && is_finite(x.w); }
// Four values joined from a cluster's shares with weights that add up to one: what is finite stays so.  Out of line, for shares of which one is
// divided by its sum (l < 0), or whose plain sum is not finite.
__device__ __noinline__ float4 join_again(float m, int shares, uint32_t ml_at, uint32_t o_at) {
  float4 y = make_float4(0.f, 0.f, 0.f, 0.f);
  float l = 0.f;
  for (int pass = 0; pass < 2; ++pass)
    for (int s = 0; s < shares; ++s) {
      const float2 ml = ld_rank2(at_rank(ml_at, s));
      if (ml.x == -INFINITY && ml.y == 0.f) continue;
      float w = exp2f(ml.x - m);
      if (pass == 0) { l = fmaf(fabsf(ml.y), w, l); continue; }
      const float4 v = ld_rank4(at_rank(o_at, s));
      w = w / l * (ml.y < 0.f ? -ml.y : 1.f);
      y.x = fmaf(v.x, w, y.x); y.y = fmaf(v.y, w, y.y); y.z = fmaf(v.z, w, y.z); y.w = fmaf(v.w, w, y.w);
    }
  return y;
}
// The same of partial outputs in memory: the shares' o at po, `stride` floats apart, their {m, l} in the lanes (h: share lane + 32 h).
__device__ __noinline__ float4 join_parts_again(const float* po, size_t stride, bool live, int shares, float w0, float w1, float l0, float l1) {
  float4 y = make_float4(0.f, 0.f, 0.f, 0.f);
  float l = 0.f;
  for (int pass = 0; pass < 2; ++pass)
    for (int s = 0; s < shares; ++s) {
      float w = __shfl_sync(0xffffffffu, s < 32 ? w0 : w1, s & 31);
      const float ls = __shfl_sync(0xffffffffu, s < 32 ? l0 : l1, s & 31);
      if (w == -1.f) continue;
      if (pass == 0) { l = fmaf(fabsf(ls), w, l); continue; }
      if (!live) continue;
      const float4 v = *reinterpret_cast<const float4*>(po + s * stride);
      w = w / l * (ls < 0.f ? -ls : 1.f);
      y.x = fmaf(v.x, w, y.x); y.y = fmaf(v.y, w, y.y); y.z = fmaf(v.z, w, y.z); y.w = fmaf(v.w, w, y.w);
    }
  return y;
}
template <typename T>
__device__ __forceinline__ void end_tile(const AttnArgs& a, TileCtl& sm, float* o, int ld, int k0, int k1) {
  const TileList& t = sm.t;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, d = a.s.d;
  __syncthreads();
  if (sm.bad[0]) {
    for (int r = warp; r < t.nr; r += kThreads / 32) {
      if (!(sm.bad[0] >> r & 1u)) continue;
      float m, l, x[16];
      if (!exact_row<T>(a, t, sm.depth, query_row<T>(a, t, r), sm.pos[r], sm.row_anc[r], k0, k1, m, l, x) && !(sm.bad[1] >> r & 1u)) continue;
#pragma unroll
      for (int i = 0; i < 16; ++i) if (lane + 32 * i < d) o[r * ld + lane + 32 * i] = x[i];
      if (lane == 0) sm.ml[r] = make_float2(m, l);
    }
    __syncthreads();
  }
  const int nv = d / 4;
  if (a.nsplit > 1 && !a.cluster) {
    const size_t at = part_index(a);
    for (int i = tid; i < t.nr * nv; i += kThreads) {
      const int r = i / nv, c = i % nv * 4;
      *reinterpret_cast<float4*>(a.po + (at + r) * d + c) = *reinterpret_cast<const float4*>(o + r * ld + c);
    }
    if (tid < t.nr) a.pml[at + tid] = sm.ml[tid];
    return;
  }
  const int shares = a.nsplit;
  if (shares > 1) cluster_sync();                         // every CTA's share is there
  const uint32_t o_at = smem_u32(o), ml_at = smem_u32(sm.ml);
  for (int i = tid + kThreads * (shares > 1 ? (int)blockIdx.z : 0); i < t.nr * nv; i += kThreads * shares) {
    const int r = i / nv, c = i % nv * 4;
    float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
    float l = 0.f;
    if (shares == 1) {
      x = *reinterpret_cast<const float4*>(o + r * ld + c);
      l = sm.ml[r].y < 0.f ? 1.f : sm.ml[r].y;
    } else {
      float2 ml[8];
      float4 v[8];
      float m = -INFINITY, least = 0.f;
#pragma unroll
      for (int s = 0; s < 8; ++s)
        if (s < shares) {
          ml[s] = ld_rank2(at_rank(ml_at + r * 8, s));
          v[s] = ld_rank4(at_rank(o_at + (r * ld + c) * 4, s));
          m = fmaxf(m, ml[s].x);
        }
#pragma unroll
      for (int s = 0; s < 8; ++s)
        if (s < shares && !(ml[s].x == -INFINITY && ml[s].y == 0.f)) {           // (else nothing seen)
          const float w = exp2f(ml[s].x - m);
          l = fmaf(ml[s].y, w, l);
          least = fminf(least, ml[s].y);
          x.x = fmaf(v[s].x, w, x.x); x.y = fmaf(v[s].y, w, x.y); x.z = fmaf(v[s].z, w, x.z); x.w = fmaf(v[s].w, w, x.w);
        }
      if (least < 0.f || (!all_finite(x) && l > 0.f && is_finite(l))) {
        const float4 y = join_again(m, shares, ml_at + r * 8, o_at + (r * ld + c) * 4);
        if (least < 0.f || all_finite(y)) { x = y; l = 1.f; }
      }
    }
    const float inv = 1.f / l;
    T* out = out_row<T>(a, t, r) + c;
    if (sizeof(T) == 4) {
      *reinterpret_cast<float4*>(out) = make_float4(x.x * inv, x.y * inv, x.z * inv, x.w * inv);
    } else {
      __nv_bfloat162 h[2] = {__floats2bfloat162_rn(x.x * inv, x.y * inv), __floats2bfloat162_rn(x.z * inv, x.w * inv)};
      *reinterpret_cast<uint2*>(out) = *reinterpret_cast<const uint2*>(h);
    }
  }
  if (shares > 1) cluster_sync();                         // nobody's share is read any more
}

__device__ __forceinline__ void ldsm4(uint32_t* r, uint32_t addr) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0, %1, %2, %3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr));
}
__device__ __forceinline__ void ldsm2(uint32_t* r, uint32_t addr) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x2.shared.b16 {%0, %1}, [%2];" : "=r"(r[0]), "=r"(r[1]) : "r"(addr));
}
__device__ __forceinline__ void ldsm4t(uint32_t* r, uint32_t addr) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr));
}
__device__ __forceinline__ void mma16816(float* c, const uint32_t* a, const uint32_t* b) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
               : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b[0]), "r"(b[1]));
}
__device__ __forceinline__ uint32_t pack2(float x, float y) {
  __nv_bfloat162 h = __floats2bfloat162_rn(x, y);
  return *reinterpret_cast<uint32_t*>(&h);
}

// ---------------------------------------------------------------- bf16, 16 rows
// Four warps, blocks of KB keys.  d <= 128: a quarter of a block's keys is a warp's own from the scores to the output (16 rows x 128 columns
// are 64 registers), with its own maxima and sums; the warps are joined at the end, and a block has one barrier.  (Through shared memory, as
// below: 8 sequences of 32 heads on 8 x 128, 32 k keys, 366 us instead of 277, at that step.)  Beyond, where one warp's registers do not hold all of d:
// each computes the scores of a quarter of the keys, the row maxima go through shared memory, then each adds the whole block's P V to
// its quarter of the output columns.  P is rounded to bf16 for the product (half a step, at most 2^-8 of a weight; the sum of the weights is of
// the unrounded ones); scores, maxima, sums and the output are fp32.  Rows of K and V come by 16-byte asynchronous copies, ST - 1 blocks
// ahead of the arithmetic (a window of 32 k tokens streams from HBM: that much has to be under way), through the page table or from the
// new rows, whose addresses are worked out a block before their copies: 16-byte chunks of a row are stored at chunk ^ (row & 7), which
// keeps every ldmatrix free of bank conflicts.  DP: d rounded up to 64, 128, 256 or 512, the rest zero.
template <int DP, bool SHARED>
struct MmaCfg {
  static constexpr int KB = DP <= 128 ? 64 : 32;
  static constexpr int ST = DP == 64 ? 4 : DP == 128 ? (SHARED ? 4 : 3) : DP == 256 ? (SHARED ? 4 : 3) : SHARED ? 4 : 2;
};
template <int DP, bool SHARED>
struct MmaSmem {
  static constexpr int KB = MmaCfg<DP, SHARED>::KB, ST = MmaCfg<DP, SHARED>::ST;
  alignas(16) bf16 q[kRows * DP];
  bf16 k[ST][KB * DP];                // (and the output at the end)
  bf16 v[SHARED ? 1 : ST][SHARED ? 8 : KB * DP];
  bf16 p[kRows * KB];
  const bf16* row[ST + 1][SHARED ? 1 : 2][KB];      // where a block's rows begin (nullptr: nothing there)
  float red[4][kRows], sum[4][kRows];
  TileCtl c;
  int missing[ST + 1][2];             // a key of the block has no page (32 keys each)
};

// (Shared memory leaves one to three CTAs an SM, so a thread may have more than the 128 registers at which the compiler stops by itself, and
// spills: single tokens of 8 sequences, 32 heads on 8 x 128, 32 k keys, warm 236 us; 218 with as many as it wants.)
template <int DP, bool SHARED>
__global__ void __launch_bounds__(kThreads, 1) attn_mma_kernel(const AttnArgs a) {
  extern __shared__ __align__(16) unsigned char smem_raw[];
  typedef MmaSmem<DP, SHARED> Sm;
  Sm& sm = *reinterpret_cast<Sm*>(smem_raw);
  constexpr int KB = Sm::KB, ST = Sm::ST;
  constexpr int CH = DP / 8, KW = KB / 4, NT = KW / 8;    // 16-byte chunks of a row; keys of a warp, in tiles of 8
  constexpr bool OWN = DP <= 128;                         // a warp's keys are its own to the end
  constexpr int CW = OWN ? DP : DP / 4, CT = CW / 8;      // output columns of a warp, in tiles of 8
  static_assert(sizeof(float) * kRows * DP * (OWN ? 4 : 1) <= sizeof(sm.k), "the output lies in the blocks' place");
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  if (!begin_tile<bf16>(a, sm.c)) return;
  const TileList& t = sm.c.t;
  int k0, k1;
  split_range(a, t, k0, k1);
  const int nb = (k1 - k0 + KB - 1) / KB;
  auto find = [&](int j) {                                // the rows behind block j
    if (tid >= KB || j >= nb) return;
    const int kk = k0 + j * KB + tid, slot = j % (ST + 1);
    int64_t code = -1;
    if (kk < k1) {
      code = list_row(a, t, kk);
      if (code == -1) atomicOr(a.status + t.b, TSV_ST_PAGE);
    }
    const bool none = __any_sync(0xffffffffu, kk < k1 && code == -1);
    if (lane == 0) sm.missing[slot][warp] = none;
    sm.row[slot][0][tid] = code == -1 ? nullptr : row_ptr<bf16>(a, t.hk, code, false);
    if (!SHARED) sm.row[slot][SHARED ? 0 : 1][tid] = code == -1 ? nullptr : row_ptr<bf16>(a, t.hk, code, true);
  };
  const int dch = a.s.d / 8;
  auto load = [&](int j) {
    if (j < nb) {
      const int slot = j % (ST + 1);
      const uint32_t ks = smem_u32(sm.k[j % ST]), vs = smem_u32(sm.v[SHARED ? 0 : j % ST]);
#pragma unroll 4
      for (int i = tid; i < KB * CH; i += kThreads) {
        const int r = i / CH, c = i % CH;
        const bf16* kp = sm.row[slot][0][r];
        const bool live = kp && c < dch;
        const uint32_t at = (uint32_t)(r * CH + (c ^ (r & 7))) * 16;
        cp16(ks + at, live ? (const void*)(kp + c * 8) : a.in.k, live);
        if (!SHARED) {
          const bf16* vp = sm.row[slot][SHARED ? 0 : 1][r];
          cp16(vs + at, live ? (const void*)(vp + c * 8) : a.in.k, live);
        }
      }
    }
    cp_commit();                                          // (a group per block, empty ones behind the last)
  };
  const uint32_t qs = smem_u32(sm.q);
  for (int i = tid; i < kRows * CH; i += kThreads) {
    const int r = i / CH, c = i % CH;
    const bool live = r < t.nr && c < dch;
    cp16(qs + (uint32_t)(r * CH + (c ^ (r & 7))) * 16, live ? (const void*)(query_row<bf16>(a, t, r) + c * 8) : a.in.q, live);
  }
  const int g = lane >> 2, tc = lane & 3;
  const uint32_t ps = smem_u32(sm.p);
  for (int pass = 0; pass < 2; ++pass) {                  // (the second one only where a result is not finite)
  for (int j = 0; j < ST; ++j) find(j);
  __syncthreads();                                        // (the rows' facts too)
  for (int j = 0; j + 1 < ST; ++j) load(j);
  int rp[2];
  uint32_t ra[2];
#pragma unroll
  for (int h = 0; h < 2; ++h) { rp[h] = sm.c.pos[g + 8 * h]; ra[h] = sm.c.row_anc[g + 8 * h]; }
  // Positions of the window part that every row sees.
  int seen0 = 0, seen1 = -1;
  {
    const int p0 = __reduce_min_sync(0xffffffffu, lane < t.nr ? sm.c.pos[lane & (kRows - 1)] : 0x7fffffff), p1 = __reduce_max_sync(0xffffffffu, lane < t.nr ? sm.c.pos[lane & (kRows - 1)] : 0);
    seen0 = max(t.lo, p1 - a.s.window + 1);
    seen1 = min(t.lo + t.nc - t.ns - 1, p0);
  }
  float m[2] = {-INFINITY, -INFINITY}, l[2] = {0.f, 0.f};
  float o[CT][4];
#pragma unroll
  for (int i = 0; i < CT; ++i)
#pragma unroll
    for (int e = 0; e < 4; ++e) o[i][e] = 0.f;
  for (int j = 0; j < nb; ++j) {
    const int st = j % ST, slot = j % (ST + 1);
    cp_wait<ST - 2>();
    if (pass)                                             // (what this thread has copied)
      for (int i = tid; i < KB * CH; i += kThreads) make_finite<bf16>((SHARED ? sm.k[st] : sm.v[SHARED ? 0 : st]) + (i / CH * CH + (i % CH ^ (i / CH & 7))) * 8);
    __syncthreads();                                      // block j is here; everyone is done with block j - 1
    load(j + ST - 1);
    find(j + ST);
    const uint32_t ks = smem_u32(sm.k[st]), vs = SHARED ? ks : smem_u32(sm.v[SHARED ? 0 : st]);
    // scores of this warp's keys
    float s[NT][4];
#pragma unroll
    for (int i = 0; i < NT; ++i)
#pragma unroll
      for (int e = 0; e < 4; ++e) s[i][e] = 0.f;
#pragma unroll 8
    for (int kk = 0; kk < DP / 16; ++kk) {
      uint32_t af[4];
      { const int r = (lane & 7) + ((lane >> 3) & 1) * 8, c = 2 * kk + (lane >> 4);
        ldsm4(af, qs + (uint32_t)(r * CH + (c ^ (r & 7))) * 16); }
      if (NT == 2) {
        uint32_t bf[4];
        const int r = warp * KW + (lane & 7) + (lane >> 4) * 8, c = 2 * kk + ((lane >> 3) & 1);
        ldsm4(bf, ks + (uint32_t)(r * CH + (c ^ (r & 7))) * 16);
        mma16816(s[0], af, bf);
        mma16816(s[NT - 1], af, bf + 2);
      } else {
        uint32_t bf[2];
        const int r = warp * KW + (lane & 7), c = 2 * kk + ((lane >> 3) & 1);
        ldsm2(bf, ks + (uint32_t)(r * CH + (c ^ (r & 7))) * 16);
        mma16816(s[0], af, bf);
      }
    }
    // masks, row maxima over the block
    const bool missing = sm.missing[slot][0] || (KB > 32 && sm.missing[slot][1]);
    float mx[2] = {-INFINITY, -INFINITY};
    const int kk0 = k0 + j * KB + warp * KW, at0 = t.lo + kk0 - t.ns;
    const bool whole = !missing && kk0 >= t.ns && kk0 + KW <= k1 && at0 >= seen0 && at0 + KW - 1 <= seen1;
    if (whole) {
#pragma unroll
      for (int i = 0; i < NT; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) { s[i][e] *= a.scale2; mx[e >> 1] = fmaxf(mx[e >> 1], s[i][e]); }
    } else {
#pragma unroll
    for (int i = 0; i < NT; ++i)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int h = e >> 1, key = warp * KW + i * 8 + 2 * tc + (e & 1), kk = k0 + j * KB + key;
        bool see = kk < k1 && list_sees(a, t, sm.c.depth, rp[h], ra[h], kk);
        if (missing && see) see = sm.row[slot][0][key] != nullptr;
        s[i][e] = see ? s[i][e] * a.scale2 : -INFINITY;
        mx[h] = fmaxf(mx[h], s[i][e]);
      }
    }
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      mx[h] = fmaxf(mx[h], __shfl_xor_sync(0xffffffffu, mx[h], 1));
      mx[h] = fmaxf(mx[h], __shfl_xor_sync(0xffffffffu, mx[h], 2));
    }
    if (OWN) {
      float alpha[2], ref[2];
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const float mn = fmaxf(m[h], mx[h]);
        ref[h] = mn == -INFINITY ? 0.f : mn;
        alpha[h] = ex2(m[h] - ref[h]);
        m[h] = mn;
        l[h] *= alpha[h];
      }
      if (__any_sync(0xffffffffu, alpha[0] != 1.f || alpha[1] != 1.f)) {
#pragma unroll
        for (int i = 0; i < CT; ++i)
#pragma unroll
          for (int e = 0; e < 4; ++e) o[i][e] *= alpha[e >> 1];
      }
      uint32_t af[4];                                     // (the scores' places in the registers are those of the product's operand)
#pragma unroll
      for (int i = 0; i < 2; ++i) {
#pragma unroll
        for (int e = 0; e < 4; ++e) { float& x = s[i % NT][e]; x = ex2(x - ref[e >> 1]); l[e >> 1] += x; }
        af[2 * i] = pack2(s[i % NT][0], s[i % NT][1]);
        af[2 * i + 1] = pack2(s[i % NT][2], s[i % NT][3]);
      }
#pragma unroll
      for (int i = 0; i < CT; i += 2) {
        uint32_t bf[4];
        const int r = warp * KW + (lane & 7) + ((lane >> 3) & 1) * 8, c = i + (lane >> 4);
        ldsm4t(bf, vs + (uint32_t)(r * CH + (c ^ (r & 7))) * 16);
        mma16816(o[i], af, bf);
        mma16816(o[i + 1], af, bf + 2);
      }
      continue;
    }
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      if (tc == 0) sm.red[warp][g + 8 * h] = mx[h];
    }
    __syncthreads();
    float alpha[2], ref[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      float mn = m[h];
#pragma unroll
      for (int w = 0; w < 4; ++w) mn = fmaxf(mn, sm.red[w][g + 8 * h]);
      ref[h] = mn == -INFINITY ? 0.f : mn;
      alpha[h] = ex2(m[h] - ref[h]);
      m[h] = mn;
      l[h] *= alpha[h];
    }
#pragma unroll
    for (int i = 0; i < NT; ++i) {
#pragma unroll
      for (int e = 0; e < 4; ++e) { s[i][e] = ex2(s[i][e] - ref[e >> 1]); l[e >> 1] += s[i][e]; }
      const int key = warp * KW + i * 8;                  // P: chunk of 8 keys, stored like the rows of K
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int r = g + 8 * h, c = key / 8;
        *reinterpret_cast<uint32_t*>(reinterpret_cast<char*>(sm.p) + (r * (KB / 8) + (c ^ (r & (KB / 8 - 1)))) * 16 + tc * 4) = pack2(s[i][2 * h], s[i][2 * h + 1]);
      }
    }
#pragma unroll
    for (int i = 0; i < CT; ++i)
#pragma unroll
      for (int e = 0; e < 4; ++e) o[i][e] *= alpha[e >> 1];
    __syncthreads();
    // P V, this warp's columns
#pragma unroll
    for (int kk = 0; kk < KB / 16; ++kk) {
      uint32_t af[4];
      { const int r = (lane & 7) + ((lane >> 3) & 1) * 8, c = 2 * kk + (lane >> 4);
        ldsm4(af, ps + (uint32_t)(r * (KB / 8) + (c ^ (r & (KB / 8 - 1)))) * 16); }
#pragma unroll
      for (int i = 0; i < CT; i += 2) {
        uint32_t bf[4];
        const int r = kk * 16 + (lane & 7) + ((lane >> 3) & 1) * 8, c = (warp * CW) / 8 + i + (lane >> 4);
        ldsm4t(bf, vs + (uint32_t)(r * CH + (c ^ (r & 7))) * 16);
        mma16816(o[i], af, bf);
        mma16816(o[i + 1], af, bf + 2);
      }
    }
  }
  // sums over the row's lanes and warps
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    l[h] += __shfl_xor_sync(0xffffffffu, l[h], 1);
    l[h] += __shfl_xor_sync(0xffffffffu, l[h], 2);
    if (OWN && tc == 0) sm.red[warp][g + 8 * h] = m[h];
    if (tc == 0) sm.sum[warp][g + 8 * h] = l[h];
  }
  cp_wait<0>();
  __syncthreads();                                        // (and everyone is done with the blocks)
  float* os = reinterpret_cast<float*>(sm.k);
  if (OWN) {
    // the warps' shares at the rows' maxima, then added up in order
    float part[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int r = g + 8 * h;
      float mn = -INFINITY;
#pragma unroll
      for (int w = 0; w < 4; ++w) mn = fmaxf(mn, sm.red[w][r]);
      const float to = mn == -INFINITY ? 0.f : mn;
      part[h] = ex2(m[h] - to);
      l[h] = 0.f;
#pragma unroll
      for (int w = 0; w < 4; ++w) l[h] = fmaf(sm.sum[w][r], ex2(sm.red[w][r] - to), l[h]);
      m[h] = mn;
      if (warp == 0 && tc == 0) sm.c.ml[r] = make_float2(m[h], l[h]);
      const bool bad = !is_finite(l[h]) || (m[h] == -INFINITY && a.nsplit == 1);
      if (bad && r < t.nr) atomicOr(sm.c.bad + pass, 1u << r);
#pragma unroll
      for (int i = 0; i < CT; ++i) *reinterpret_cast<float2*>(os + (warp * kRows + r) * DP + i * 8 + 2 * tc) = make_float2(o[i][2 * h] * part[h], o[i][2 * h + 1] * part[h]);
    }
    __syncthreads();
    for (int i = tid; i < kRows * DP / 4; i += kThreads) {
      float4 x = *reinterpret_cast<const float4*>(os + 4 * i);
#pragma unroll
      for (int w = 1; w < 4; ++w) {
        const float4 y = *reinterpret_cast<const float4*>(os + w * kRows * DP + 4 * i);
        x.x += y.x; x.y += y.y; x.z += y.z; x.w += y.w;
      }
      const int r = 4 * i / DP;
      if (r < t.nr && !all_finite(x)) atomicOr(sm.c.bad + pass, 1u << r);
      *reinterpret_cast<float4*>(os + 4 * i) = x;
    }
  } else
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const int r = g + 8 * h;
    l[h] = sm.sum[0][r] + sm.sum[1][r] + sm.sum[2][r] + sm.sum[3][r];
    // (nothing of this share seen: {-inf, 0} and zeros; without shares every row sees its own key)
    bool bad = !is_finite(l[h]) || (m[h] == -INFINITY && a.nsplit == 1);
#pragma unroll
    for (int i = 0; i < CT; ++i) {
      bad |= !is_finite(o[i][2 * h]) || !is_finite(o[i][2 * h + 1]);
      *reinterpret_cast<float2*>(os + r * DP + warp * CW + i * 8 + 2 * tc) = make_float2(o[i][2 * h], o[i][2 * h + 1]);
    }
    if (bad && r < t.nr) atomicOr(sm.c.bad + pass, 1u << r);
    if (warp == 0 && tc == 0) sm.c.ml[r] = make_float2(m[h], l[h]);
  }
  __syncthreads();
  if (!sm.c.bad[0]) break;
  }
  end_tile<bf16>(a, sm.c, reinterpret_cast<float*>(sm.k), DP, k0, k1);
}

// ---------------------------------------------------------------- fp32, 16 rows
// The numerics type: FMAs in fp32.  Blocks of 32 keys in shared memory (rows padded by 16 bytes: a quarter-warp's loads of eight rows hit
// eight different bank groups), the next one's copies under the arithmetic of the current one where two fit; a thread computes the
// scores of one key for four rows, then owns every 128th column of all 16 rows.
constexpr int kKeys32 = 32;

struct F32Ctl {
  float p[kRows][kKeys32 + 4], alpha[kRows], m[kRows], l[kRows];
  int64_t code[2][kKeys32];
  TileCtl c;
};
__host__ __device__ inline int f32_ctl() { return (int)((sizeof(F32Ctl) + 15) & ~(size_t)15); }
inline int f32_block(const AttnArgs& a) { return 4 * (a.c.v ? 2 : 1) * kKeys32 * (a.s.d + 4); }

template <int NC>       // columns of a thread
__global__ void __launch_bounds__(kThreads) attn_fp32_kernel(const AttnArgs a, const int buffers) {
  extern __shared__ __align__(16) unsigned char smem_raw[];
  F32Ctl& sm = *reinterpret_cast<F32Ctl*>(smem_raw);
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, d = a.s.d, ld = d + 4;
  float* q = reinterpret_cast<float*>(smem_raw + f32_ctl());      // (and the output at the end)
  float* blocks = q + kRows * d;
  const int bstride = (a.c.v ? 2 : 1) * kKeys32 * ld;
  if (!begin_tile<float>(a, sm.c)) return;
  const TileList& t = sm.c.t;
  int k0, k1;
  split_range(a, t, k0, k1);
  const int nv = d / 4, nb = (k1 - k0 + kKeys32 - 1) / kKeys32;
  for (int i = tid; i < kRows * nv; i += kThreads) {
    const int r = i / nv, c = i % nv;
    cp16(smem_u32(q + r * d + c * 4), r < t.nr ? (const void*)(query_row<float>(a, t, r) + c * 4) : a.in.q, r < t.nr);
  }
  auto codes = [&](int j) {
    if (tid >= kKeys32 || j >= nb) return;
    const int kk = k0 + j * kKeys32 + tid;
    int64_t code = -1;
    if (kk < k1) {
      code = list_row(a, t, kk);
      if (code == -1) atomicOr(a.status + t.b, TSV_ST_PAGE);
    }
    sm.code[j & 1][tid] = code;
  };
  auto load = [&](int j) {
    if (j < nb) {
      float* ks = blocks + (buffers > 1 ? (j & 1) * bstride : 0);
      for (int i = tid; i < kKeys32 * nv; i += kThreads) {
        const int r = i / nv, c = i % nv;
        const int64_t code = sm.code[j & 1][r];
        cp16(smem_u32(ks + r * ld + c * 4), code != -1 ? (const void*)(row_ptr<float>(a, t.hk, code, false) + c * 4) : a.in.k, code != -1);
        if (a.c.v) cp16(smem_u32(ks + (kKeys32 + r) * ld + c * 4), code != -1 ? (const void*)(row_ptr<float>(a, t.hk, code, true) + c * 4) : a.in.k, code != -1);
      }
    }
    cp_commit();
  };
  for (int pass = 0; pass < 2; ++pass) {                  // (the second one only where a result is not finite)
  float o[NC][kRows];
#pragma unroll
  for (int c = 0; c < NC; ++c)
#pragma unroll
    for (int r = 0; r < kRows; ++r) o[c][r] = 0.f;
  if (tid < kRows) { sm.m[tid] = -INFINITY; sm.l[tid] = 0.f; }
  codes(0);
  __syncthreads();
  load(0);
  codes(1);
  for (int j = 0; j < nb; ++j) {
    const int kb = k0 + j * kKeys32;
    const float* ks = blocks + (buffers > 1 ? (j & 1) * bstride : 0);
    const float* vs = a.c.v ? ks + kKeys32 * ld : ks;
    __syncthreads();                                      // (block j + 1's rows; everyone is done with block j - 1)
    if (buffers > 1) { load(j + 1); cp_wait<1>(); } else cp_wait<0>();
    if (pass)                                             // (what this thread has copied)
      for (int i = tid; i < kKeys32 * nv; i += kThreads) make_finite<float>(const_cast<float*>(vs) + i / nv * ld + i % nv * 4);
    __syncthreads();
    // scores: key `lane`, rows 4 warp ..
    float s[4] = {0.f, 0.f, 0.f, 0.f};
    for (int c = 0; c < nv; ++c) {
      const float4 kv = *reinterpret_cast<const float4*>(ks + lane * ld + c * 4);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float4 qv = *reinterpret_cast<const float4*>(q + (4 * warp + i) * d + c * 4);
        s[i] = fmaf(kv.x, qv.x, fmaf(kv.y, qv.y, fmaf(kv.z, qv.z, fmaf(kv.w, qv.w, s[i]))));
      }
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int r = 4 * warp + i;
      const bool see = kb + lane < k1 && sm.code[j & 1][lane] != -1 && list_sees(a, t, sm.c.depth, sm.c.pos[r], sm.c.row_anc[r], kb + lane);
      s[i] = see ? s[i] * a.scale2 : -INFINITY;
      float mx = s[i];
#pragma unroll
      for (int x = 16; x; x >>= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, x));
      const float mo = sm.m[r], mn = fmaxf(mo, mx), ref = mn == -INFINITY ? 0.f : mn;
      const float w = exp2f(s[i] - ref), al = exp2f(mo - ref);
      const float sum = warp_sum(w);
      sm.p[r][lane] = w;
      __syncwarp();
      if (lane == 0) { sm.alpha[r] = al; sm.m[r] = mn; sm.l[r] = sm.l[r] * al + sum; }
    }
    __syncthreads();
    codes(j + 2);                                         // (in the place of block j's)
#pragma unroll
    for (int r = 0; r < kRows; ++r) {
      const float al = sm.alpha[r];
#pragma unroll
      for (int c = 0; c < NC; ++c) o[c][r] *= al;
    }
    for (int k = 0; k < kKeys32; k += 4) {
      float v[NC][4];
#pragma unroll
      for (int c = 0; c < NC; ++c)
#pragma unroll
        for (int i = 0; i < 4; ++i) v[c][i] = tid + c * kThreads < d ? vs[(k + i) * ld + tid + c * kThreads] : 0.f;
#pragma unroll
      for (int r = 0; r < kRows; ++r) {
        const float4 p = *reinterpret_cast<const float4*>(&sm.p[r][k]);
#pragma unroll
        for (int c = 0; c < NC; ++c) o[c][r] = fmaf(p.x, v[c][0], fmaf(p.y, v[c][1], fmaf(p.z, v[c][2], fmaf(p.w, v[c][3], o[c][r]))));
      }
    }
    if (buffers == 1) { __syncthreads(); load(j + 1); }
  }
  cp_wait<0>();
  __syncthreads();
  const bool again = pass == 0;
#pragma unroll
  for (int r = 0; r < kRows; ++r) {
    if (r >= t.nr) break;
    const float l = sm.l[r];
    bool bad = !is_finite(l) || (sm.m[r] == -INFINITY && a.nsplit == 1);
#pragma unroll
    for (int c = 0; c < NC; ++c) bad |= !is_finite(o[c][r]);
    if (tid == 0) sm.c.ml[r] = make_float2(sm.m[r], l);
    if (bad) atomicOr(sm.c.bad + pass, 1u << r);
  }
  __syncthreads();
  if (!sm.c.bad[0] || !again) {                              // (Q's place: it is not read any more)
#pragma unroll
    for (int r = 0; r < kRows; ++r)
#pragma unroll
      for (int c = 0; c < NC; ++c) if (tid + c * kThreads < d) q[r * d + tid + c * kThreads] = o[c][r];
    break;
  }
  }
  end_tile<float>(a, sm.c, q, d, k0, k1);
}

// ---------------------------------------------------------------- partial outputs
// out = sum_s 2^(m_s - m) O_s / sum_s 2^(m_s - m) l_s, shares in order.  A warp per row and 128 columns: its lanes fetch the shares' {m, l}
// at once (at most 64 shares), then eight shares' values are under way at a time.
template <typename T>
__global__ void __launch_bounds__(kThreads) attn_join_kernel(const AttnArgs a, const int per) {
  __shared__ TileList s_t;
  __shared__ int depth[TSV_MAX_D];
  __shared__ uint32_t anc[TSV_MAX_D];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, d = a.s.d, chunks = (d + 127) / 128;
  if (warp == 0) {
    const TileList t = make_list(a, blockIdx.x, blockIdx.y, per, depth, anc);
    if (lane == 0) s_t = t;
  }
  __syncthreads();
  const TileList& t = s_t;
  if (t.ok == 2 && blockIdx.z == 0) zero_rows<T>(a, t);
  if (t.ok != 1) return;
  for (int i = warp + (kThreads / 32) * blockIdx.z; i < t.nr * chunks; i += (kThreads / 32) * gridDim.z) {
    const int r = i / chunks, col = (i % chunks * 32 + lane) * 4;
    const size_t base = (((size_t)blockIdx.x * gridDim.y + blockIdx.y) * a.nsplit) * per + r;
    float2 ml[2];
    float m = -INFINITY;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      ml[h] = make_float2(-INFINITY, 0.f);
      if (lane + 32 * h < a.nsplit) ml[h] = a.pml[base + (size_t)(lane + 32 * h) * per];
      m = fmaxf(m, ml[h].x);
    }
#pragma unroll
    for (int o = 16; o; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
    float w[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) w[h] = ml[h].x == -INFINITY && ml[h].y == 0.f ? -1.f : exp2f(ml[h].x - m);      // (-1: nothing seen)
    float l = 0.f;
    float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
    for (int s0 = 0; s0 < a.nsplit; s0 += 8) {
      float4 v[8];
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        v[k] = make_float4(0.f, 0.f, 0.f, 0.f);
        if (s0 + k < a.nsplit && col < d) v[k] = *reinterpret_cast<const float4*>(a.po + (base + (size_t)(s0 + k) * per) * d + col);
      }
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        const float ws = __shfl_sync(0xffffffffu, s0 + k < 32 ? w[0] : w[1], (s0 + k) & 31), ls = __shfl_sync(0xffffffffu, s0 + k < 32 ? ml[0].y : ml[1].y, (s0 + k) & 31);
        if (s0 + k >= a.nsplit || ws == -1.f) continue;
        l = fmaf(ls, ws, l);
        x.x = fmaf(v[k].x, ws, x.x); x.y = fmaf(v[k].y, ws, x.y); x.z = fmaf(v[k].z, ws, x.z); x.w = fmaf(v[k].w, ws, x.w);
      }
    }
    const bool divided = ml[0].y < 0.f || ml[1].y < 0.f;
    if (__any_sync(0xffffffffu, divided || !all_finite(x))) {      // (nearly never; then by all lanes alike)
      const bool must = __any_sync(0xffffffffu, divided);
      const float4 y = join_parts_again(a.po + base * d + col, (size_t)per * d, col < d, a.nsplit, w[0], w[1], ml[0].y, ml[1].y);
      if (must || (!all_finite(x) && l > 0.f && is_finite(l) && all_finite(y))) { x = y; l = 1.f; }
    }
    if (col < d) {
      T* out = out_row<T>(a, t, r) + col;
      out[0] = from_f<T>(x.x / l); out[1] = from_f<T>(x.y / l); out[2] = from_f<T>(x.z / l); out[3] = from_f<T>(x.w / l);
    }
  }
}

// A grid of tiles, key heads and shares; the shares of a tile a cluster where its CTAs join them.
template <typename... P, typename... A>
int launch_tiles(void (*kernel)(P...), const AttnArgs& a, dim3 grid, int smem, cudaStream_t st, A... args) {
  if (!ensure_smem((const void*)kernel, smem)) return TSV_ERR_CUDA;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = grid; cfg.blockDim = dim3(kThreads); cfg.dynamicSmemBytes = smem; cfg.stream = st;
  cudaLaunchAttribute at[1];
  at[0].id = cudaLaunchAttributeClusterDimension;
  at[0].val.clusterDim.x = at[0].val.clusterDim.y = 1;
  at[0].val.clusterDim.z = a.cluster ? a.nsplit : 1;
  cfg.attrs = at; cfg.numAttrs = 1;
  if (cudaLaunchKernelEx(&cfg, kernel, args...) != cudaSuccess) return TSV_ERR_CUDA;
  count_launch();
  return TSV_OK;
}

template <int DP, bool SHARED>
int mma_launch(const AttnArgs& a, dim3 grid, cudaStream_t st) {
  TSV_PREP((attn_mma_kernel<DP, SHARED>));
  return launch_tiles(attn_mma_kernel<DP, SHARED>, a, grid, (int)sizeof(MmaSmem<DP, SHARED>), st, a);
}

template <int NC>
int fp32_launch(const AttnArgs& a, dim3 grid, cudaStream_t st) {
  TSV_PREP(attn_fp32_kernel<NC>);
  const int one = f32_ctl() + 4 * kRows * a.s.d, buffers = one + 2 * f32_block(a) <= 227 * 1024 ? 2 : 1;
  return launch_tiles(attn_fp32_kernel<NC>, a, grid, one + buffers * f32_block(a), st, a, buffers);
}

size_t up256(size_t x) { return (x + 255) & ~(size_t)255; }

struct AttnPlan {
  bool tc;                // 128-row tiles on the tensor cores
  int per;                // query rows of a tile
  int64_t tiles;          // tiles over all sequences (bound)
  int nsplit, cluster;
  size_t off_pml;
};

// bf16 in tiles of 128 rows where a sequence may have more rows for a key head than one tile of 16.  us, tiles of 128 / of 16 rows, 32 heads
// on 8 of 128: 64 sequences, window 1024: 16 rows 80 / 99, 32 rows 81 / 205, 64 rows 82 / 315; 4 sequences, window 128: 16 / 16, 15 / 17,
// 16 / 21; 8 heads of 64, 64 sequences, window 1024: 74 / 70, 76 / 119, 82 / 168.  Single tokens (1 to 256 sequences, windows of 128 to
// 32 k): d = 64 and 128 shared 17 / 15 to 97 / 72, the larger ones of 32 on 8 x 128 and of d above 128 the other way about, 135 / 160.
// Above d = 128 also where there are 64 tiles and more, or lists of 16 k keys: 16 heads x 512, 256 sequences, window 128 42 / 55, 64 of 2048
// 81 / 91, one of 32 k 56 / 60, but eight of 2048 38 / 34; 8 heads on 8 x 256, 64 of 2048 201 / 296, eight of 32 k 364 / 932; the worst found
// was 2 heads x 512 with values of their own, eight of 32 k 216 / 185.  (Cold, and before the kernel of tiles of 16
// had all its registers, which took up to a seventh off its times.)
int64_t keys_of(const tsv_tok_shape& s) {                 // of a list, at most
  const int64_t reach = std::min<int64_t>((int64_t)s.window + s.max_n, s.max_L);
  return reach + std::min<int64_t>(s.n_sink, s.max_L);
}
bool takes_tc(const tsv_tok_shape& s) {
  if (s.dtype != TSV_BF16) return false;
  return (int64_t)s.max_n * (s.H / s.Hk) > kRows || (s.d > 128 && ((int64_t)s.B * s.Hk >= 64 || keys_of(s) >= 16384));
}

// Tiles and CTAs that splitting the keys aims at: those that run at a time.
int slots_of(const tsv_tok_shape& s) { return takes_tc(s) ? 148 / tc_halves(s.d) : s.d <= 128 ? 2 * 148 : 148; }

// Keys are split where the tiles alone would leave SMs without work.  Tiles of 16 rows: into shares of 32 keys and more, up to eight as a
// cluster's CTAs, which join them; into more, of 512 keys and more, through partial outputs.  (8 sequences of 8 key heads x 128, 32 k keys:
// 9 shares, nearly two rounds of CTAs, 229 us; 8 at most, 238.)
AttnPlan plan_of(const tsv_tok_shape& s, int64_t rows) {
  AttnPlan p;
  p.tc = takes_tc(s);
  p.per = p.tc ? tc_tile(s.d) : kRows;
  p.tiles = tok_units_bound(s, rows, s.H / s.Hk, p.per);
  const int64_t ctas = p.tiles * s.Hk;
  const int64_t keys = keys_of(s);
  p.cluster = 0;
  if (p.tc) {                                             // 512 keys and more, and no more CTAs than run at a time
    const int64_t ns = std::min(slots_of(s) / ctas, (keys + 511) / 512);
    p.nsplit = (int)std::max<int64_t>(1, std::min<int64_t>(ns, 64));
  } else {
    // The time in keys: rounds of CTAs, of a share and what a CTA takes without keys; more than eight shares, which another kernel joins.
    int64_t best = INT64_MAX;
    for (int ns = 1; ns <= 64; ++ns) {
      const int64_t share = ((keys + ns - 1) / ns + 15) & ~15, all = ctas * ns;
      if (ns > 1 && ((ns - 1) * (ns > 8 ? 512 : 32) >= keys || (ns > 8 && all > 2 * slots_of(s)))) break;
      const int64_t time = (all + slots_of(s) - 1) / slots_of(s) * (share + 128) + (ns > 8 ? 200 : 0);
      if (time < best) { best = time; p.nsplit = ns; }
    }
    p.cluster = p.nsplit > 1 && p.nsplit <= 8;
  }
  p.off_pml = up256((size_t)2 * slots_of(s) * p.per * s.d * sizeof(float));
  return p;
}

}  // namespace

// The most that any number of rows takes: keys are split while there are fewer tiles than slots_of, into less than twice as many.
size_t tok_attn_workspace(const tsv_tok_shape& s, int64_t rows) {
  const AttnPlan p = plan_of(s, rows);
  return p.off_pml + up256((size_t)2 * slots_of(s) * p.per * sizeof(float2));
}

int launch_tok_attn(const tsv_tok_shape& s, const tsv_tok_cache& c, const tsv_tok_batch& bt, const tsv_tok_rows& in, void* out, char* ws, int32_t* status,
                    cudaStream_t st) {
  const AttnPlan p = plan_of(s, bt.rows);
  if (p.tiles > 0x7fffffff) return TSV_ERR_LIMIT;
  AttnArgs a;
  a.s = s; a.c = c; a.bt = bt; a.in = in; a.out = out;
  a.po = reinterpret_cast<float*>(ws);
  a.pml = reinterpret_cast<float2*>(ws + p.off_pml);
  a.G = s.H / s.Hk;
  a.nsplit = p.nsplit;
  a.cluster = p.cluster;
  a.scale2 = s.sm_scale * 1.4426950408889634f;
  a.status = status;
  const dim3 grid((unsigned)p.tiles, s.Hk, p.nsplit);
  int r;
  if (p.tc) {
    r = launch_attn_tc(a, p.tiles, st);
  } else if (s.dtype == TSV_FP32) {
    r = s.d <= 128 ? fp32_launch<1>(a, grid, st) : s.d <= 256 ? fp32_launch<2>(a, grid, st) : fp32_launch<4>(a, grid, st);
  } else if (!c.v) {
    r = s.d <= 64 ? mma_launch<64, true>(a, grid, st) : s.d <= 128 ? mma_launch<128, true>(a, grid, st)
      : s.d <= 256 ? mma_launch<256, true>(a, grid, st) : mma_launch<512, true>(a, grid, st);
  } else {
    r = s.d <= 64 ? mma_launch<64, false>(a, grid, st) : s.d <= 128 ? mma_launch<128, false>(a, grid, st)
      : s.d <= 256 ? mma_launch<256, false>(a, grid, st) : mma_launch<512, false>(a, grid, st);
  }
  if (r) return r;
  if (p.nsplit > 1 && !p.cluster) {
    const dim3 jg((unsigned)p.tiles, s.Hk, (p.per * ((s.d + 127) / 128) + 3) / 4);
    if (s.dtype == TSV_FP32) attn_join_kernel<float><<<jg, kThreads, 0, st>>>(a, p.per);
    else attn_join_kernel<bf16><<<jg, kThreads, 0, st>>>(a, p.per);
    count_launch();
  }
  return cudaGetLastError() == cudaSuccess ? TSV_OK : TSV_ERR_CUDA;
}

}  // namespace tsv
