// qk_norm_rope: per head of every new token's queries and keys an RMS norm with weights, then the position rotation of
// some of its dims, in one pass over the vectors.
//
//   y = x / sqrt(sum x^2 / d + eps) * w;   (a, b) -> (a cos t - b sin t, a sin t + b cos t),   t = position * inv_freq[i]
//
// Bound by HBM (each vector is read and written once; 8 FLOP per element), by latency for a handful of tokens.
// A warp takes some tokens, one after the other, and a share of their heads.  Its lanes first make the token's cosines and sines in shared
// memory (the angle is the same for every head: rot / 2 values per token against (H + Hk) * d elements); then a group of lanes
// owns a head, and a lane the SAME dims of every head its warp walks over, both members of each pair among them: weights and
// angles stay in registers (their products), the rotation needs no exchange, and the only reduction is the sum of squares over the group.
// Arithmetic goes two values at a time (fma.rn.f32x2): with one the instructions took as long as the bytes.
#include <type_traits>

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
  int32_t tokens, parts;   // tokens of a warp, one after the other; warps that share a token's heads
  int32_t group;           // lanes of a head: a power of two
  int32_t* status;
};

// The angle in turns is made in fp64: a rounding of the product of a 30-bit and a 24-bit number, one of 1 / (2 pi) and one of the product with
// it, at most 3 x 2^-53 of the turns (position 2^30, frequency 1: 2^27.3 turns, 2^-24 of a turn).  Whole turns are taken off there too,
// and only the rest of at most half a turn goes on in fp32.
__device__ __forceinline__ float2 cos_sin(int pos, float freq) {
  double turns = (double)pos * (double)freq * 0.15915494309189533576888;
  turns -= rint(turns);
  float s, c;
  sincospif(2.f * (float)turns, &s, &c);
  return make_float2(c, s);
}

// Two fp32 at a time.
__device__ __forceinline__ uint64_t pair2(float x, float y) {
  uint64_t r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(x), "f"(y));
  return r;
}
__device__ __forceinline__ float2 unpair(uint64_t v) {
  float2 r;
  asm("mov.b64 {%0, %1}, %2;" : "=f"(r.x), "=f"(r.y) : "l"(v));
  return r;
}
__device__ __forceinline__ uint64_t fma2(uint64_t a, uint64_t b, uint64_t c) {
  uint64_t r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
  return r;
}
__device__ __forceinline__ uint64_t mul2(uint64_t a, uint64_t b) {
  uint64_t r;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}

// Means of squares beyond these (squares that fp32 does not hold, or as zero) are taken again of the vector times a power of two that brings
// its largest value, or the square root of eps, to 1 .. 4: the norm does not depend on it.  (0, an infinity and NaN stay as they are.)
__device__ __forceinline__ bool in_range(float mean) {      // 2^-100 .. 2^120, in one comparison
  return (uint32_t)(__float_as_int(mean) - (27 << 23)) < 220u << 23;
}
__device__ __forceinline__ float scale_of(float x) {
  if (!(x > 0.f && x < INFINITY)) return 1.f;
  const int e = (__float_as_int(x) >> 23) - 127;
  return __int_as_float((127 - min(max(e, -126), 126)) << 23);
}

// A unit: two 16-byte vectors of a head, their members as pairs (a, b) two at a time.  PAIRS: neighbours; else member i of one vector and of
// the other.
template <typename T, bool PAIRS> struct Unit;
template <bool PAIRS> struct Unit<bf16, PAIRS> {
  static __device__ __forceinline__ void split(const uint4 (&v)[2], uint64_t (&a)[4], uint64_t (&b)[4]) {
    const uint32_t w[8] = {v[0].x, v[0].y, v[0].z, v[0].w, v[1].x, v[1].y, v[1].z, v[1].w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint32_t p = PAIRS ? w[2 * i] : w[i], q = PAIRS ? w[2 * i + 1] : w[4 + i];
      const float pl = __uint_as_float(p << 16), ph = __uint_as_float(p & 0xFFFF0000u), ql = __uint_as_float(q << 16), qh = __uint_as_float(q & 0xFFFF0000u);
      a[i] = PAIRS ? pair2(pl, ql) : pair2(pl, ph);
      b[i] = PAIRS ? pair2(ph, qh) : pair2(ql, qh);
    }
  }
  static __device__ __forceinline__ void join(const uint64_t (&a)[4], const uint64_t (&b)[4], uint4 (&v)[2]) {
    uint32_t w[8];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float2 x = unpair(a[i]), y = unpair(b[i]);
      const __nv_bfloat162 p = PAIRS ? __floats2bfloat162_rn(x.x, y.x) : __floats2bfloat162_rn(x.x, x.y), q = PAIRS ? __floats2bfloat162_rn(x.y, y.y) : __floats2bfloat162_rn(y.x, y.y);
      w[PAIRS ? 2 * i : i] = *reinterpret_cast<const uint32_t*>(&p);
      w[PAIRS ? 2 * i + 1 : 4 + i] = *reinterpret_cast<const uint32_t*>(&q);
    }
    v[0] = make_uint4(w[0], w[1], w[2], w[3]);
    v[1] = make_uint4(w[4], w[5], w[6], w[7]);
  }
};
template <bool PAIRS> struct Unit<float, PAIRS> {
  static __device__ __forceinline__ void split(const uint4 (&v)[2], uint64_t (&a)[2], uint64_t (&b)[2]) {
    const float w[8] = {__uint_as_float(v[0].x), __uint_as_float(v[0].y), __uint_as_float(v[0].z), __uint_as_float(v[0].w),
                        __uint_as_float(v[1].x), __uint_as_float(v[1].y), __uint_as_float(v[1].z), __uint_as_float(v[1].w)};
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      a[i] = PAIRS ? pair2(w[4 * i], w[4 * i + 2]) : pair2(w[2 * i], w[2 * i + 1]);
      b[i] = PAIRS ? pair2(w[4 * i + 1], w[4 * i + 3]) : pair2(w[4 + 2 * i], w[5 + 2 * i]);
    }
  }
  static __device__ __forceinline__ void join(const uint64_t (&a)[2], const uint64_t (&b)[2], uint4 (&v)[2]) {
    float w[8];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const float2 x = unpair(a[i]), y = unpair(b[i]);
      if (PAIRS) { w[4 * i] = x.x; w[4 * i + 1] = y.x; w[4 * i + 2] = x.y; w[4 * i + 3] = y.y; }
      else { w[2 * i] = x.x; w[2 * i + 1] = x.y; w[4 + 2 * i] = y.x; w[5 + 2 * i] = y.y; }
    }
    v[0] = make_uint4(__float_as_uint(w[0]), __float_as_uint(w[1]), __float_as_uint(w[2]), __float_as_uint(w[3]));
    v[1] = make_uint4(__float_as_uint(w[4]), __float_as_uint(w[5]), __float_as_uint(w[6]), __float_as_uint(w[7]));
  }
};

// UPL: units a lane owns (2 for fp32 heads of more than 256 dims)
template <typename T, int UPL, bool PAIRS>
__global__ void __launch_bounds__(kRopeThreads, UPL == 1 ? 2 : 1) rope_kernel(const RopeArgs a) {
  constexpr int VE = Vec<T>::N, NP = VE / 2, AHEAD = 2;      // NP: pairs of pairs of a unit
  extern __shared__ float2 cs_all[];                       // [warps][rot / 2]
  const tsv_tok_shape& s = a.s;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, half = a.rot / 2;
  float2* cs_tab = cs_all + warp * half;
  // the vectors of this lane
  const int hpw = 32 / a.group, gl = lane % a.group, gi = lane / a.group;
  const int nv = s.d / VE, hu = half / VE, fv = a.first / VE;
  int vec[UPL][2];
  bool turn[UPL][2];
#pragma unroll
  for (int p = 0; p < UPL; ++p) {
    const int un = gl + p * a.group;
    if (PAIRS || un >= hu) {
      const int j = 2 * (PAIRS ? un : un - hu), skip = PAIRS ? 0 : 2 * hu;
      vec[p][0] = PAIRS || j < fv ? j : j + skip;
      vec[p][1] = PAIRS || j + 1 < fv ? j + 1 : j + 1 + skip;
    } else {
      vec[p][0] = fv + un; vec[p][1] = fv + hu + un;
    }
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      if (vec[p][h] >= nv) vec[p][h] = -1;
      turn[p][h] = PAIRS ? vec[p][h] >= fv && vec[p][h] < fv + 2 * hu : un < hu;
    }
  }
  const float inv_d = 1.f / (float)s.d;
  // this warp's tokens (numbered over all sequences), and its share of their heads
  const int parts = a.parts, w0 = blockIdx.x * kRopeWarps + warp, part = w0 % parts, step = parts * hpw;
  const int64_t tok0 = (int64_t)(w0 / parts) * a.tokens;
  TokUnit u;
  int ok = 0, depth = 0, left = 0;                         // ok: 1 rows, 2 zeros; tokens of the sequence that are left
  uint4 raw[AHEAD][UPL][2];
#pragma unroll 1
  for (int64_t t = tok0; t < tok0 + a.tokens; ++t) {
    if (left == 0) {
      // (the last warp of all looks at every sequence: it finds those that are flagged)
      if (!find_unit(s, a.bt, a.L, 1, 1, t, a.status, u)) break;
      left = u.n - u.unit;
      int st = u.L < 0 || (int64_t)u.L + u.n > s.max_L ? TSV_ST_LENGTH : 0;
      uint32_t anc;
      if (a.bt.parent) st |= tok_tree(a.bt, u, depth, anc);
      ok = st ? 2 : 1;
      if (st && lane == 0) atomicOr(a.status + u.b, st);
    }
    const int64_t row = u.row0 + u.unit;
    const int pos = u.L + (a.bt.parent && ok == 1 ? __shfl_sync(0xffffffffu, depth, u.unit & 31) : u.unit);
    ++u.unit; --left;
    // AHEAD heads' loads of a lane at a time: a warp has few heads to walk over, and their latency is what it waits for
    auto fetch = [&](const T* in, int h0, int heads) {
#pragma unroll
      for (int e = 0; e < AHEAD; ++e)
#pragma unroll
        for (int p = 0; p < UPL; ++p)
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            const int head = h0 + e * step + gi;
            raw[e][p][h] = make_uint4(0, 0, 0, 0);
            if (head < heads && vec[p][h] >= 0 && ok == 1) raw[e][p][h] = *reinterpret_cast<const uint4*>(in + (size_t)head * s.d + vec[p][h] * VE);
          }
    };
    const bool early = a.q && part * hpw < s.H;            // the first of them under the angles' arithmetic
    if (early) fetch(reinterpret_cast<const T*>(a.q) + row * a.q_ld, part * hpw, s.H);
    if (ok == 1) {
      __syncwarp();                                        // (the token before is done with the table)
      for (int i = lane; i < half; i += 32) cs_tab[i] = cos_sin(pos, __ldg(a.inv_freq + i));
      __syncwarp();
    }
#pragma unroll 1
    for (int which = 0; which < 2; ++which) {
      const T* in = reinterpret_cast<const T*>(which ? a.k : a.q);
      if (!in) continue;
      in += row * (which ? a.k_ld : a.q_ld);
      T* out = reinterpret_cast<T*>(which ? a.k_out : a.q_out) + row * (which ? a.ldk : a.ldq);
      const float* w = which ? a.wk : a.wq;
      const int heads = which ? s.Hk : s.H;
      // (the last part first: keys have few heads, and the parts of a token that get none of the queries' rest take them)
      const int first = (which ? parts - 1 - part : part) * hpw;
      if (first >= heads) continue;
      // weights times cosines and sines: a' = a (wa c) - b (wb s), b' = a (wa s) + b (wb c)
      uint64_t ac[UPL][NP], as[UPL][NP], bc[UPL][NP], bs[UPL][NP];
#pragma unroll
      for (int p = 0; p < UPL; ++p) {
        float wt[2][VE];
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
          for (int e = 0; e < VE; ++e) wt[h][e] = w && ok == 1 && vec[p][h] >= 0 ? __ldg(w + vec[p][h] * VE + e) : 1.f;
#pragma unroll
        for (int i = 0; i < NP; ++i) {
          float wa[2], wb[2];
          float2 c[2];
#pragma unroll
          for (int x = 0; x < 2; ++x) {
            const int h = PAIRS ? i / (NP / 2) : 0, e = PAIRS ? 2 * (i % (NP / 2)) + x : 2 * i + x;      // PAIRS: pair e of vector h; else pair e
            wa[x] = PAIRS ? wt[h][2 * e] : wt[0][e];
            wb[x] = PAIRS ? wt[h][2 * e + 1] : wt[1][e];
            c[x] = make_float2(1.f, 0.f);
            if (turn[p][h] && ok == 1) c[x] = cs_tab[PAIRS ? (vec[p][h] - fv) * (VE / 2) + e : (gl + p * a.group) * VE + e];
          }
          ac[p][i] = pair2(wa[0] * c[0].x, wa[1] * c[1].x); as[p][i] = pair2(wa[0] * c[0].y, wa[1] * c[1].y);
          bc[p][i] = pair2(wb[0] * c[0].x, wb[1] * c[1].x); bs[p][i] = pair2(-wb[0] * c[0].y, -wb[1] * c[1].y);
        }
      }
      // 32 heads of a lane, a bit each in `later` for those that are to be done once more (the outputs may be the inputs' places: what has been
      // written cannot be looked at again)
      uint32_t later = 0;
      auto walk = [&](auto slow, int from) {
        constexpr bool SLOW = decltype(slow)::value;
        uint32_t bit = 1;
#pragma unroll 1
        for (int h0 = from; h0 < heads && bit; h0 += AHEAD * step, bit <<= AHEAD) {
          if (SLOW || !(early && which == 0 && h0 == first)) fetch(in, h0, heads);
#pragma unroll
          for (int e = 0; e < AHEAD; ++e) {
            const int head = h0 + e * step + gi;
            uint64_t xa[UPL][NP], xb[UPL][NP], s2 = 0, s3 = 0;
#pragma unroll
            for (int p = 0; p < UPL; ++p) {
              Unit<T, PAIRS>::split(raw[e][p], xa[p], xb[p]);
#pragma unroll
              for (int i = 0; i < NP; ++i) { s2 = fma2(xa[p][i], xa[p][i], s2); s3 = fma2(xb[p][i], xb[p][i], s3); }
            }
            const float2 sa = unpair(s2), sb = unpair(s3);
            float ss = (sa.x + sa.y) + (sb.x + sb.y);
            for (int o = a.group >> 1; o; o >>= 1) ss += __shfl_xor_sync(0xffffffffu, ss, o);
            float mean = fmaf(ss, inv_d, a.eps);
            const bool far = SLOW ? (later & bit << e) != 0 : !in_range(mean);
            if (!SLOW && far) later |= bit << e;
            if (SLOW) {
              float mx = 0.f, s1 = 0.f;
#pragma unroll
              for (int p = 0; p < UPL; ++p)
#pragma unroll
                for (int i = 0; i < NP; ++i) {
                  const float2 u = unpair(xa[p][i]), v = unpair(xb[p][i]);
                  mx = fmaxf(fmaxf(mx, fmaxf(fabsf(u.x), fabsf(u.y))), fmaxf(fabsf(v.x), fabsf(v.y)));
                }
              for (int o = a.group >> 1; o; o >>= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, o));
              const float by = scale_of(fmaxf(mx, sqrtf(a.eps)));
              const uint64_t by2 = pair2(by, by);
#pragma unroll
              for (int p = 0; p < UPL; ++p)
#pragma unroll
                for (int i = 0; i < NP; ++i) {
                  xa[p][i] = mul2(xa[p][i], by2); xb[p][i] = mul2(xb[p][i], by2);
                  const float2 u = unpair(xa[p][i]), v = unpair(xb[p][i]);
                  s1 = fmaf(u.x, u.x, fmaf(u.y, u.y, fmaf(v.x, v.x, fmaf(v.y, v.y, s1))));
                }
              for (int o = a.group >> 1; o; o >>= 1) s1 += __shfl_xor_sync(0xffffffffu, s1, o);
              mean = fmaf(s1, inv_d, a.eps * by * by);
            }
            const float r = ok == 1 ? rsqrtf(mean) : 0.f;    // (2 units in the last place)
            const uint64_t r2 = pair2(r, r);
#pragma unroll
            for (int p = 0; p < UPL; ++p) {
              uint64_t ya[NP], yb[NP];
#pragma unroll
              for (int i = 0; i < NP; ++i) {
                if (turn[p][PAIRS ? i / (NP / 2) : 0]) {
                  ya[i] = mul2(fma2(xa[p][i], ac[p][i], mul2(xb[p][i], bs[p][i])), r2);
                  yb[i] = mul2(fma2(xa[p][i], as[p][i], mul2(xb[p][i], bc[p][i])), r2);
                } else {
                  ya[i] = mul2(mul2(xa[p][i], ac[p][i]), r2);
                  yb[i] = mul2(mul2(xb[p][i], bc[p][i]), r2);
                }
              }
              uint4 v[2];
              Unit<T, PAIRS>::join(ya, yb, v);
#pragma unroll
              for (int h = 0; h < 2; ++h)
                if (head < heads && vec[p][h] >= 0 && far == SLOW) *reinterpret_cast<uint4*>(out + (size_t)head * s.d + vec[p][h] * VE) = v[h];
            }
          }
        }
      };
#pragma unroll 1
      for (int from = first; from < heads; from += 32 * step, later = 0) {
        walk(std::false_type(), from);
        if (__any_sync(0xffffffffu, later != 0)) walk(std::true_type(), from);      // (nearly never)
      }
    }
  }
}

template <typename T, int UPL, bool PAIRS>
int rope_launch(const RopeArgs& a, dim3 grid, int smem, cudaStream_t st) {
  TSV_PREP((rope_kernel<T, UPL, PAIRS>));
  rope_kernel<T, UPL, PAIRS><<<grid, kRopeThreads, smem, st>>>(a);
  count_launch();
  return cudaGetLastError() == cudaSuccess ? TSV_OK : TSV_ERR_CUDA;
}
template <typename T, int UPL>
int rope_launch(const RopeArgs& a, dim3 grid, int smem, cudaStream_t st) {
  return a.pairs ? rope_launch<T, UPL, true>(a, grid, smem, st) : rope_launch<T, UPL, false>(a, grid, smem, st);
}

}  // namespace

int launch_rope(const tsv_tok_shape& s, const int32_t* L, const tsv_tok_batch& bt, const tsv_tok_rows& in, const float* wq, const float* wk, float eps,
                const float* inv_freq, int rot, int first, int pairs, void* q_out, int64_t ldq, void* k_out, int64_t ldk, int32_t* status,
                cudaStream_t st) {
  RopeArgs a = {s, bt, L, in.q, in.k, q_out, k_out, in.q_ld, in.k_ld, ldq, ldk, wq, wk, inv_freq, eps, rot, first, pairs, 1, 1, 1, status};
  const int ve = s.dtype == TSV_BF16 ? 8 : 4, units = (s.d / ve + 1) / 2;
  while (a.group < units && a.group < 32) a.group *= 2;
  // Two CTAs of 8 warps per SM, every warp with the same number of tokens, one after the other; where there are fewer tokens than warps,
  // several share the heads of one, down to one pass over the lanes each.  (CTAs of 2 tokens, each with its own search for its sequence
  // and its own table of angles: 164 us for 17 k tokens of 40 heads x 128; of 16: 78.)
  const int64_t rows = bt.rows < (int64_t)s.B * s.max_n ? bt.rows : (int64_t)s.B * s.max_n, warps = 2 * 148 * kRopeWarps;
  const int hpw = 32 / a.group, most = (s.H + hpw - 1) / hpw;
  while (a.parts < most && rows * a.parts * 2 <= warps) a.parts *= 2;
  const int64_t share = (rows * a.parts + warps - 1) / warps;
  a.tokens = (int32_t)(share < 1 ? 1 : share);
  const int64_t chunks = rows / a.tokens + 1;               // (one behind the last token: it looks at every sequence; no more than about `warps`)
  const dim3 grid((unsigned)((chunks * a.parts + kRopeWarps - 1) / kRopeWarps));
  const int smem = kRopeWarps * (rot / 2) * (int)sizeof(float2);
  if (s.dtype == TSV_BF16) return rope_launch<bf16, 1>(a, grid, smem, st);
  return units > 32 ? rope_launch<float, 2>(a, grid, smem, st) : rope_launch<float, 1>(a, grid, smem, st);
}

}  // namespace tsv
