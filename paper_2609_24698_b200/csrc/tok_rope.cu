// qk_norm_rope: per head of every new token's queries and keys an RMS norm with weights, then the position rotation of
// some of its dims, in one pass over the vectors.
//
//   y = x / sqrt(sum x^2 / d + eps) * w;   (a, b) -> (a cos t - b sin t, a sin t + b cos t),   t = position * inv_freq[i]
//
// Bound by HBM (each vector is read and written once; 8 FLOP per element), by latency for a handful of tokens.
// A CTA takes TPI tokens and a share of their heads.  Its threads first make the cosines and sines of these tokens in shared
// memory (the angle is the same for every head: rot / 2 values per token against (H + Hk) * d elements); then a group of lanes
// owns a head, and a lane the SAME dims of every head its warp walks over, both members of each pair among them: weights and
// angles stay in registers, the rotation needs no exchange, and the only reduction is the sum of squares over the group.
#include "tok_common.cuh"

namespace tsv {

namespace {

constexpr int kRopeThreads = 256;
constexpr int kRopeWarps = kRopeThreads / 32;

struct RopeArgs {
  tsv_tok_shape s;
  tsv_tok_batch bt;
  const int32_t* L;
  const void *q, *k;
  void *q_out, *k_out;
  int64_t q_ld, k_ld, ldq, ldk;
  const float *wq, *wk, *inv_freq;
  float eps;
  int32_t rot, first, pairs;
  int32_t tpi;             // tokens of a CTA: 1, 2, 4 or 8
  int32_t group;           // lanes of a head: a power of two
  int32_t* status;
};

// The angle is exact as a product of a 30-bit and a 24-bit number in fp64; whole turns are taken off there too (what is left has
// an error of some 2^-53 of the turns, 2^-25 at positions of 2^30), and only the rest of at most half a turn goes on in fp32.
__device__ __forceinline__ float2 cos_sin(int pos, float freq) {
  double turns = (double)pos * (double)freq * 0.15915494309189533576888;
  turns -= rint(turns);
  float s, c;
  sincospif(2.f * (float)turns, &s, &c);
  return make_float2(c, s);
}

// UPL: pairs of 16-byte vectors a lane owns (2 for fp32 heads of more than 256 dims)
template <typename T, int UPL>
__global__ void __launch_bounds__(kRopeThreads) rope_kernel(const RopeArgs a) {
  constexpr int VE = Vec<T>::N, AHEAD = UPL == 1 ? 4 : 2;
  extern __shared__ float2 cs_tab[];                       // [tpi][rot / 2]
  __shared__ int s_ok, s_pos[8];
  __shared__ TokUnit s_u;
  const tsv_tok_shape& s = a.s;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, half = a.rot / 2;
  if (warp == 0) {
    TokUnit u;
    int ok = 0;                                            // 0: nothing to do, 1: rows, 2: zeros
    if (find_unit(s, a.bt, a.L, 1, a.tpi, blockIdx.x, a.status, u)) {
      const int L = u.L;
      int st = L < 0 || (int64_t)L + u.n > s.max_L ? TSV_ST_LENGTH : 0, depth = 0;
      uint32_t anc;
      if (a.bt.parent) st |= tok_tree(a.bt, u, depth, anc);
      ok = st ? 2 : 1;
      if (st && lane == 0) atomicOr(a.status + u.b, st);
      const int i = u.unit * a.tpi + lane;
      const int at = a.bt.parent && !st ? __shfl_sync(0xffffffffu, depth, i & 31) : i;
      if (lane < a.tpi) s_pos[lane] = L + at;
    }
    if (lane == 0) { s_ok = ok; s_u = u; }
  }
  __syncthreads();
  const int ok = s_ok;
  if (!ok) return;
  const TokUnit u = s_u;
  const int t0 = u.unit * a.tpi, nt = min(a.tpi, u.n - t0);
  if (ok == 1) {
    for (int i = tid; i < nt * half; i += kRopeThreads) cs_tab[i] = cos_sin(s_pos[i / half], __ldg(a.inv_freq + i % half));
    __syncthreads();
  }
  // warps of a token: a share of its heads each, with gridDim.y
  const int wpt = kRopeWarps / a.tpi, tok = warp / wpt;
  if (tok >= nt) return;
  const int64_t row = u.row0 + t0 + tok;
  const int part = blockIdx.y * wpt + warp % wpt, parts = gridDim.y * wpt;
  const int hpw = 32 / a.group, gl = lane % a.group, gi = lane / a.group;
  const int nv = s.d / VE, hu = half / VE, fv = a.first / VE;
  // the vectors of this lane, and the angles of their pairs
  int vec[UPL][2];
  float2 cs[UPL][VE];
  bool turn[UPL];
#pragma unroll
  for (int p = 0; p < UPL; ++p) {
    const int un = gl + p * a.group;
    if (a.pairs || un >= hu) {
      const int j = 2 * (a.pairs ? un : un - hu), skip = a.pairs ? 0 : 2 * hu;
      vec[p][0] = a.pairs || j < fv ? j : j + skip;
      vec[p][1] = a.pairs || j + 1 < fv ? j + 1 : j + 1 + skip;
    } else {
      vec[p][0] = fv + un; vec[p][1] = fv + hu + un;
    }
#pragma unroll
    for (int h = 0; h < 2; ++h) if (vec[p][h] >= nv) vec[p][h] = -1;
    turn[p] = false;
#pragma unroll
    for (int e = 0; e < VE; ++e) cs[p][e] = make_float2(1.f, 0.f);
    if (ok == 1) {
      const float2* tab = cs_tab + tok * half;
      if (!a.pairs && un < hu) {
        turn[p] = true;
#pragma unroll
        for (int e = 0; e < VE; ++e) cs[p][e] = tab[un * VE + e];
      } else if (a.pairs) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const int e0 = vec[p][h] * VE - a.first;
          if (vec[p][h] >= 0 && e0 >= 0 && e0 < a.rot) {
            turn[p] = true;
#pragma unroll
            for (int e = 0; e < VE / 2; ++e) cs[p][h * (VE / 2) + e] = tab[e0 / 2 + e];
          }
        }
      }
    }
  }
  const float inv_d = 1.f / (float)s.d;
#pragma unroll 1
  for (int which = 0; which < 2; ++which) {
    const T* in = reinterpret_cast<const T*>(which ? a.k : a.q);
    if (!in) continue;
    in += row * (which ? a.k_ld : a.q_ld);
    T* out = reinterpret_cast<T*>(which ? a.k_out : a.q_out) + row * (which ? a.ldk : a.ldq);
    const float* w = which ? a.wk : a.wq;
    const int heads = which ? s.Hk : s.H;
    float wt[UPL][2 * VE];
#pragma unroll
    for (int p = 0; p < UPL; ++p)
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int e = 0; e < VE; ++e) wt[p][h * VE + e] = w && vec[p][h] >= 0 ? __ldg(w + vec[p][h] * VE + e) : 1.f;
    // (the last part first: keys have few heads, and the parts of a token that get none of the queries' rest take them)
    const int first = (which ? parts - 1 - part : part) * hpw;
    // four heads' loads of a lane at a time: a warp has few heads to walk over, and their latency is what it waits for
    const int step = parts * hpw;
#pragma unroll 1
    for (int h0 = first; h0 < heads; h0 += AHEAD * step) {
      uint4 raw[AHEAD][UPL][2];
#pragma unroll
      for (int u = 0; u < AHEAD; ++u)
#pragma unroll
        for (int p = 0; p < UPL; ++p)
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            const int head = h0 + u * step + gi;
            raw[u][p][h] = make_uint4(0, 0, 0, 0);
            if (head < heads && vec[p][h] >= 0 && ok == 1) raw[u][p][h] = *reinterpret_cast<const uint4*>(in + (size_t)head * s.d + vec[p][h] * VE);
          }
#pragma unroll
      for (int u = 0; u < AHEAD; ++u) {
        const int head = h0 + u * step + gi;
        const bool live = head < heads;
        float x[UPL][2 * VE];
        float ss = 0.f;
#pragma unroll
        for (int p = 0; p < UPL; ++p) {
#pragma unroll
          for (int h = 0; h < 2; ++h) ld16(reinterpret_cast<const T*>(&raw[u][p][h]), x[p] + h * VE);
#pragma unroll
          for (int e = 0; e < 2 * VE; ++e) ss = fmaf(x[p][e], x[p][e], ss);
        }
        for (int o = a.group >> 1; o; o >>= 1) ss += __shfl_xor_sync(0xffffffffu, ss, o);
        const float r = 1.f / sqrtf(fmaf(ss, inv_d, a.eps));
#pragma unroll
        for (int p = 0; p < UPL; ++p) {
          float y[2 * VE];
#pragma unroll
          for (int e = 0; e < 2 * VE; ++e) y[e] = ok == 1 ? x[p][e] * r * wt[p][e] : 0.f;
          if (turn[p]) {
            if (a.pairs) {
#pragma unroll
              for (int e = 0; e < VE; ++e) {
                const float ya = y[2 * e], yb = y[2 * e + 1];
                y[2 * e] = ya * cs[p][e].x - yb * cs[p][e].y;
                y[2 * e + 1] = ya * cs[p][e].y + yb * cs[p][e].x;
              }
            } else {
#pragma unroll
              for (int e = 0; e < VE; ++e) {
                const float ya = y[e], yb = y[VE + e];
                y[e] = ya * cs[p][e].x - yb * cs[p][e].y;
                y[VE + e] = ya * cs[p][e].y + yb * cs[p][e].x;
              }
            }
          }
#pragma unroll
          for (int h = 0; h < 2; ++h)
            if (live && vec[p][h] >= 0) st16(out + (size_t)head * s.d + vec[p][h] * VE, y + h * VE);
        }
      }
    }
  }
}

template <typename T, int UPL>
int rope_launch(const RopeArgs& a, dim3 grid, int smem, cudaStream_t st) {
  TSV_PREP((rope_kernel<T, UPL>));
  rope_kernel<T, UPL><<<grid, kRopeThreads, smem, st>>>(a);
  count_launch();
  return cudaGetLastError() == cudaSuccess ? TSV_OK : TSV_ERR_CUDA;
}

}  // namespace

int launch_rope(const tsv_tok_shape& s, const int32_t* L, const tsv_tok_batch& bt, const tsv_tok_rows& in, const float* wq, const float* wk, float eps,
                const float* inv_freq, int rot, int first, int pairs, void* q_out, int64_t ldq, void* k_out, int64_t ldk, int32_t* status,
                cudaStream_t st) {
  RopeArgs a = {s, bt, L, in.q, in.k, q_out, k_out, in.q_ld, in.k_ld, ldq, ldk, wq, wk, inv_freq, eps, rot, first, pairs, 1, 1, status};
  const int ve = s.dtype == TSV_BF16 ? 8 : 4, units = (s.d / ve + 1) / 2;
  while (a.group < units && a.group < 32) a.group *= 2;
  // Tokens of a CTA: one per warp (8) where that leaves two CTAs for every SM, fewer below; then shares of the heads, down to one
  // head per warp, until there are as many.
  const int64_t rows = bt.rows < (int64_t)s.B * s.max_n ? bt.rows : (int64_t)s.B * s.max_n;
  while (a.tpi < 8 && rows / (2 * a.tpi) >= 2 * 148) a.tpi *= 2;
  const int64_t units_all = tok_units_bound(s, bt.rows, 1, a.tpi);
  if (units_all > 0x7fffffff) return TSV_ERR_LIMIT;
  const int wpt = kRopeWarps / a.tpi, hpw = 32 / a.group;
  int gy = 1;
  while (gy < 64 && rows / a.tpi * gy < 2 * 148 && gy * wpt * hpw < s.H) gy *= 2;
  const dim3 grid((unsigned)units_all, gy);
  const int smem = a.tpi * (rot / 2) * (int)sizeof(float2);
  if (s.dtype == TSV_BF16) return rope_launch<bf16, 1>(a, grid, smem, st);
  return units > 32 ? rope_launch<float, 2>(a, grid, smem, st) : rope_launch<float, 1>(a, grid, smem, st);
}

}  // namespace tsv
