// window_sink_attn on the tensor cores (tcgen05), bf16: tiles of 128 query rows of one sequence and key head, two at a time up to d = 128.
//
// A persistent CTA per SM walks over work items (one or two tiles, key head, columns, share of the keys), warps by role:
//   warps 0-3    softmax of the first tile, a row per thread
//   warps 4-7    softmax of the second tile; where there is one tile, its epilogue, under the next item's scores and softmax
//   warp 8       issues S = Q K^T, as far ahead as buffers allow, into the next item too
//   warp 9       finds the items ahead of the others: tile, keys, tree
//   warps 10-13  copy blocks of K and V into shared memory: two warps K, two V, or all four where K is V (a wait for a barrier's phase is
//                only good for a thread that sees all of them).  Rows come by 16-byte asynchronous copies: from pages, a ring or the call's
//                own tensors, any of them with strides of their own, which no tensor map describes; a barrier counts a block's copies as
//                they land, and the thread that issues the products orders them before its reads (fence.proxy.async)
//   warp 14      Q, by TMA where the heads of a key head fill a box evenly, else like K and V
//   warp 15      issues O += P V, P as the A operand straight from tensor memory
//
// K and V live in panels of a block's rows x 64 columns (128-byte swizzle): K row-major is the K-major operand of S, and the same layout
// read MN-major the operand of P V, so that where the keys are the values one copy serves both products.  Two tiles share a block of K
// and V: copies (half of the shared-memory traffic of a tile) and their instructions per product halve, and one tile's softmax runs
// under the other's products.
//
// Tensor memory: O, and beside it at most 256 columns of S: two blocks' scores for each tile (four at d = 512), so that the next block's are
// there when a softmax is done.  P (bf16) overlays the S it came from.  (Two tiles with one buffer of 128 columns each, scores after the
// P V of the block before: 16 heads x 64 125 us instead of 117.)
//
// d = 512: Q of a tile (128 KiB) leaves no room for blocks of keys ahead, and tensor memory none for S beside all of O (512 columns).  So
// an item belongs to the two CTAs of a cluster, each with half of the columns of Q, K, V and O: it multiplies its halves of Q and K, sends
// its part of S to the other through distributed shared memory, adds what comes from there, and both do the same softmax.  Nothing is
// read or multiplied twice, Q fits twice (the next tile's comes under this one's work) and so do three blocks of 48 keys.  Prompts of 64
// heads x 512: 654 us (cold; 649 to 667 in a long run); with all of Q and K in both CTAs, which was the form before, 755 with blocks of
// 48 keys and 828 of 64.
//
// Softmax: S is read once, in slabs of 64 keys (48 at d = 512).  The row's reference is its first maximum, rounded up to a whole power of
// two; it moves where a later slab exceeds it by more than 2^10 (bf16 and fp32 have the range for weights above one), and then what is
// there of P, the sum and O are multiplied by a power of two, exactly.  Nearly never after the first slab.
// P is rounded to bf16 for the product (half a step, at most 2^-8 of a weight); scores, sums and O are fp32.
//
// What bounds it (prompts of 32 heads on 8 x 128, window 1024, 17 k tokens: 549 us cold, 585 to 595 at the clocks of a long run; 36 % of the
// tensor pipe's cycles, 38 % of the special function units'): a tile's softmax of 64 keys takes 2.2 k cycles, a third of it the exponentials, which two warps of a scheduler share
// the unit for, the rest latencies of dependent instructions; the products of both tiles 1.6 k (K = 16 of P V from tensor memory costs
// 103 cycles for 128 columns, of S from shared memory 50 up to 64 keys).  At d = 512 a block's softmax and exchange (2.5 k cycles for 48 keys,
// of which 0.5 wait for the other CTA).  Figures of two forms are those of the step that they belong to, cold.
#include <cuda.h>
#include <cudaTypedefs.h>

#include "tc_common.cuh"
#include "tok_attn.cuh"

namespace tsv {

namespace {

using namespace tc;

constexpr int kTile = 128;            // query rows of a tile
constexpr int kMmaWarp = 8, kListWarp = 9, kCopyWarps = 5, kOutWarp = 15, kWarps = 16;
constexpr int kPanel = 16384;
constexpr int kItems = 3;             // items found ahead
constexpr float kGap = 10.f;          // log2 units by which a maximum may exceed the row's reference
constexpr int kCtl = 3 * 1024;            // bytes in front of the panels (a multiple of 1024)
// Polls of up to 4 us before a wait gives up: a role may wait for a whole item, and that may be millions of keys, or rows computed one by one.
// A warp whose wait has given up starts nothing more that runs by itself (copies, products, words for the other CTA), takes no item and gives
// none out, and goes to the end, where what is under way is waited for before the memory is given up.
constexpr uint32_t kWaitLimit = WAIT_LIMIT << 8;
constexpr uint32_t kDrain = WAIT_LIMIT;     // those at the end

template <int N> struct Int { static constexpr int value = N; };

template <int DP, bool SHARED>
struct Cfg {
  static constexpr int PAIR = DP == 512 ? 2 : 1;             // CTAs of an item, 256 columns each
  static constexpr int NT = DP <= 128 ? 2 : 1;               // tiles of an item
  static constexpr int OC = DP / PAIR;                       // columns of a CTA
  static constexpr int NP = OC / 64;                         // panels of them: copied, announced and multiplied together
  static constexpr int KP = SHARED ? 0 : NP;                 // panels of K where V has its own
  static constexpr int QB = PAIR == 2 ? 2 : NT;              // tiles of Q in shared memory
  static constexpr int BN = PAIR == 2 ? 48 : DP == 256 && SHARED ? 128 : 64;            // keys of a block
  static constexpr int SL = BN < 64 ? BN : 64;               // columns of a slab of S
  static constexpr int PB = BN * 128;                        // bytes of a panel of keys
  static constexpr int NKB = KP == 0 ? 0 : DP == 512 ? 1 : DP == 256 ? 2 : 4;          // buffers of a block's K
  static constexpr int NVB = DP <= 128 ? 4 : DP == 512 && SHARED ? 3 : 2;   // of its V
  static constexpr int SB = (NT == 1 && PAIR == 1 ? 2 : 4) / NT, SW = 2 * kTile / (NT * SB);     // a tile's buffers of S, their columns
  static constexpr int TEAM = KP ? 2 : 4;                    // warps that copy a block of K or V
  static constexpr int RW = BN % (32 * TEAM) ? BN / TEAM : 32;       // rows that a warp copies at a time
  static constexpr int XB = PAIR == 2 ? kTile * BN * 4 : 0;  // the other CTA's part of S
  static constexpr int SMEM = kCtl + QB * NP * kPanel + (NKB + NVB) * NP * PB + XB;
};

// An item: tile, output columns, keys.  mode: 0 the first time; of those that left a mark then, 1 as before (which rows are not finite?)
// and 2 with values that are not finite taken as zero.
struct Item {
  TileList t;
  int unit, split, k0, k1, nb, nt, mode, li;
  int missing;                        // a page of the list is not there
  int depth[TSV_MAX_D];
  uint32_t anc[TSV_MAX_D];
};

struct TcCtl {
  uint64_t fullQ[2], emptyQ[2];               // by buffer
  uint64_t fullK[4], emptyK[4];
  uint64_t fullV[4], emptyV[4];
  uint64_t s_full[4], p_ready[4], s_free[4], o_full[2], o_free[2];
  uint64_t stat_full, stat_free;              // one tile: reference and sum of its rows, for the epilogue
  uint64_t x_full[4], x_free[4];              // a warp's rows of the other CTA's part of S: there; taken there, of this one's
  uint64_t bad_full[2][4];                    // the other CTA's word of `bad`, by turns
  uint64_t drained[2];                        // at the end: all products are done
  uint32_t bad[2][4];                         // rows with a result that is not finite there, a bit each
  uint64_t item_full[kItems], item_free[kItems];
  uint32_t tmem_base;
  uint32_t failed;                            // a pair: a wait has given up in one of the CTAs
  uint32_t redo[32];                  // items with a result that is not finite, a bit each
  float2 stat[kTile];
  Item item[kItems];
};
static_assert(sizeof(TcCtl) <= kCtl, "control block overflow");

__device__ __forceinline__ void bar_init(uint64_t* b, int count) {
  asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(smem_u32(b)), "r"(count));
}
__device__ __forceinline__ void bar_arrive(uint64_t* b) {
  asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(smem_u32(b)) : "memory");
}
// A first look in line, then tries to the limit in a function: a wait is in the code of some thirty places.  A test is back sooner than a try
// that may suspend, a try leaves the other warps more; pairs of CTAs, whose softmax hardly ever finds a phase incomplete, take the test
// (prompts of 64 heads x 512: 672 against 691 us; 32 heads x 128 the other way about, 565 and 540).
__device__ __noinline__ bool bar_wait_on(uint32_t addr, uint32_t parity, uint32_t tries) {
#pragma unroll 1
  for (uint32_t it = 0; it < tries; ++it) {
    uint32_t ok;
    asm volatile("{\n\t.reg .pred p;\n\tmbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2, %3;\n\tselp.b32 %0, 1, 0, p;\n\t}"
                 : "=r"(ok) : "r"(addr), "r"(parity), "r"(SUSPEND_NS) : "memory");
    if (ok) return true;
  }
  return false;
}
template <bool TEST>
__device__ __forceinline__ bool bar_wait(uint64_t* bar, uint32_t parity, uint32_t tries) {
  const uint32_t addr = smem_u32(bar);
  uint32_t ok;
  if (TEST)
    asm volatile("{\n\t.reg .pred p;\n\tmbarrier.test_wait.parity.shared::cta.b64 p, [%1], %2;\n\tselp.b32 %0, 1, 0, p;\n\t}" : "=r"(ok) : "r"(addr), "r"(parity) : "memory");
  else
    asm volatile("{\n\t.reg .pred p;\n\tmbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2, %3;\n\tselp.b32 %0, 1, 0, p;\n\t}"
                 : "=r"(ok) : "r"(addr), "r"(parity), "r"(SUSPEND_NS) : "memory");
  return ok || bar_wait_on(addr, parity, tries);
}
// The same for what the other CTA of a pair sends: its words are ordered before their arrival (release) at the scope of the cluster, so that is the
// scope of the wait.
__device__ __noinline__ bool bar_wait_pair_on(uint32_t addr, uint32_t parity, uint32_t tries) {
#pragma unroll 1
  for (uint32_t it = 0; it < tries; ++it) {
    uint32_t ok;
    asm volatile("{\n\t.reg .pred p;\n\tmbarrier.try_wait.parity.acquire.cluster.shared::cta.b64 p, [%1], %2, %3;\n\tselp.b32 %0, 1, 0, p;\n\t}"
                 : "=r"(ok) : "r"(addr), "r"(parity), "r"(SUSPEND_NS) : "memory");
    if (ok) return true;
  }
  return false;
}
__device__ __forceinline__ bool bar_wait_pair(uint64_t* bar, uint32_t parity, uint32_t tries) {
  const uint32_t addr = smem_u32(bar);
  uint32_t ok;
  asm volatile("{\n\t.reg .pred p;\n\tmbarrier.test_wait.parity.acquire.cluster.shared::cta.b64 p, [%1], %2;\n\tselp.b32 %0, 1, 0, p;\n\t}" : "=r"(ok) : "r"(addr), "r"(parity) : "memory");
  return ok || bar_wait_pair_on(addr, parity, tries);
}
__device__ __forceinline__ uint32_t other_cta(const void* p, uint32_t rank) {
  uint32_t r;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(smem_u32(p)), "r"(rank));
  return r;
}
__device__ __forceinline__ void pair_sync() {
  asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
  asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
}
// An arrival of this thread when its copies so far have landed.
__device__ __forceinline__ void bar_arrive_copied(uint64_t* b) {
  asm volatile("cp.async.mbarrier.arrive.noinc.shared::cta.b64 [%0];" ::"r"(smem_u32(b)) : "memory");
}
__device__ __forceinline__ void fence_proxy() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }
__device__ __forceinline__ uint32_t uniform(uint32_t x) { return __shfl_sync(0xffffffffu, x, 0); }
__device__ __forceinline__ bool elect_one() {
  uint32_t r;
  asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.b32 %0, 1, 0, p;\n\t}" : "=r"(r));
  return r != 0;
}
// High word of the descriptors here (make_desc): 1024 bytes from eight rows to the next, descriptor version 1, 128-byte swizzle.  The low
// one: address / 16, and the distance of 64-column panels / 16 where that counts.
constexpr uint32_t kDescHi = 1024 >> 4 | 1u << 14 | 2u << 29;
// (a CTA of a cluster has its rank in the address's upper bits)
__device__ __forceinline__ uint32_t desc_lo(uint32_t addr, uint32_t far) { return (addr >> 4 & 0x3fff) | far << 16; }

// The products with the descriptors' low words apart: the high ones never change, and each word goes to a uniform register of its own
// for every product.
__device__ __forceinline__ void mma_ss2(uint32_t d_tmem, uint32_t a_lo, uint32_t a_hi, uint32_t b_lo, uint32_t b_hi, uint32_t idesc, uint32_t acc) {
  asm volatile("{\n\t.reg .pred p;\n\t.reg .b64 a, b;\n\tsetp.ne.b32 p, %6, 0;\n\tmov.b64 a, {%1, %2};\n\tmov.b64 b, {%3, %4};\n\t"
               "tcgen05.mma.cta_group::1.kind::f16 [%0], a, b, %5, p;\n\t}"
               ::"r"(d_tmem), "r"(a_lo), "r"(a_hi), "r"(b_lo), "r"(b_hi), "r"(idesc), "r"(acc) : "memory");
}
__device__ __forceinline__ void mma_ts2(uint32_t d_tmem, uint32_t a_tmem, uint32_t b_lo, uint32_t b_hi, uint32_t idesc, uint32_t acc) {
  asm volatile("{\n\t.reg .pred p;\n\t.reg .b64 b;\n\tsetp.ne.b32 p, %5, 0;\n\tmov.b64 b, {%2, %3};\n\t"
               "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], b, %4, p;\n\t}"
               ::"r"(d_tmem), "r"(a_tmem), "r"(b_lo), "r"(b_hi), "r"(idesc), "r"(acc) : "memory");
}
// Bits [lo, hi) of a word, any lo and hi.
__device__ __forceinline__ uint32_t bits(int lo, int hi) {
  lo = max(lo, 0); hi = min(hi, 32);
  return lo >= hi ? 0u : (0xffffffffu << lo) & (0xffffffffu >> (32 - hi));
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
__device__ __forceinline__ uint64_t add2(uint64_t a, uint64_t b) {
  uint64_t r;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
__device__ __forceinline__ uint64_t mul2(uint64_t a, uint64_t b) {
  uint64_t r;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
// 32 bytes at a 32-byte boundary
__device__ __forceinline__ void store32(void* p, const uint32_t* r) {
  asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(p), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]) : "memory");
}

// 2^x for a whole x <= 0, exactly (below the smallest normal number: 0).
__device__ __forceinline__ float power_of_two(float x) {
  const int e = (int)fmaxf(x, -127.f) + 127;
  return __int_as_float(max(e, 0) << 23);
}

__device__ __forceinline__ void tmem_ld16_nowait(uint32_t taddr, uint32_t* r) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]),
        "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
      : "r"(taddr));
}
__device__ __forceinline__ void tmem_regs_ready16(uint32_t* r) {
  asm volatile("" : "+r"(r[0]), "+r"(r[1]), "+r"(r[2]), "+r"(r[3]), "+r"(r[4]), "+r"(r[5]), "+r"(r[6]), "+r"(r[7]), "+r"(r[8]), "+r"(r[9]), "+r"(r[10]), "+r"(r[11]), "+r"(r[12]), "+r"(r[13]), "+r"(r[14]), "+r"(r[15]) :: "memory");
}

struct TcArgs {
  alignas(64) CUtensorMap q;    // [rows][H][d]; a box is 128 rows of a tile (G heads of 128 / G tokens, or 128 heads of one) x 64 columns
  AttnArgs a;
  int32_t items;
  int32_t q_box;                // the queries come by it
  uint32_t tries;               // of a wait
};
__device__ __forceinline__ void tma_box3(uint32_t dst, const CUtensorMap* map, int x, int y, int z, uint32_t bar) {
  asm volatile("cp.async.bulk.tensor.3d.shared::cta.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];"
               ::"r"(dst), "l"(reinterpret_cast<uint64_t>(map)), "r"(x), "r"(y), "r"(z), "r"(bar) : "memory");
}

// What is rare stays out of the loops' code.

// Of keys c0 .. (bits of m) those that have a page.
__device__ __noinline__ uint32_t have_pages(const AttnArgs& a, const TileList& t, int c0, uint32_t m) {
  for (uint32_t x = m; x; x &= x - 1) {
    const int i = __ffs(x) - 1;
    if (list_row(a, t, c0 + i) == -1) m &= ~(1u << i);
  }
  return m;
}
// Multiplies the first `words` words (a multiple of 16) of P at p_col, and `cols` columns of O, by f (a power of two).
__device__ __noinline__ void rescale(uint32_t p_col, int words, uint32_t o_col, int cols, float f) {
  asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory");
#pragma unroll 1
  for (int v = 0; v < words; v += 16) {
    uint32_t r[16];
    tmem_ld16(p_col + v, r);
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      const float2 pv = __bfloat1622float2(*reinterpret_cast<const __nv_bfloat162*>(&r[e]));
      const __nv_bfloat162 h = __floats2bfloat162_rn(pv.x * f, pv.y * f);
      r[e] = *reinterpret_cast<const uint32_t*>(&h);
    }
    tmem_st16(p_col + v, r);
  }
#pragma unroll 1
  for (int v = 0; v < cols; v += 16) {
    uint32_t r[16];
    tmem_ld16(o_col + v, r);
#pragma unroll
    for (int e = 0; e < 16; ++e) r[e] = __float_as_uint(__uint_as_float(r[e]) * f);
    tmem_st16(o_col + v, r);
  }
  asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory");
}
// Columns c0 .. c1 - 1 of row r of an item (r0: in its sequence and key head) by definition, if the row sees something not finite or is
// `still` not finite without what it does not see; part: the row's place among partial outputs.  By a warp.
__device__ __noinline__ void exact_output(const AttnArgs& a, const TileList& t, const int* depth, int gr, int p, uint32_t an, int k0, int k1, int c0, int c1,
                                          size_t part, bool still) {
  const int lane = threadIdx.x & 31;
  const int64_t tok = t.row0 + gr / a.G;
  const size_t head = (size_t)t.hk * a.G + gr % a.G;
  float m, l, o[16];
  if (!exact_row<bf16>(a, t, depth, reinterpret_cast<const bf16*>(a.in.q) + tok * a.in.q_ld + head * a.s.d, p, an, k0, k1, m, l, o) && !still) return;
  bf16* out = reinterpret_cast<bf16*>(a.out) + (tok * a.s.H + head) * a.s.d;
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    const int col = lane + 32 * i;
    if (col < c0 || col >= c1) continue;
    if (a.nsplit > 1) a.po[part * a.s.d + col] = o[i]; else out[col] = from_f<bf16>(l < 0.f ? o[i] : o[i] / l);
  }
  if (a.nsplit > 1 && c0 == 0 && lane == 0) a.pml[part] = make_float2(m, l);
}

template <int DP, bool SHARED>
__global__ void __launch_bounds__(32 * kWarps, 1) attn_tc_kernel(const __grid_constant__ TcArgs g) {
  typedef Cfg<DP, SHARED> C;
  constexpr int NT = C::NT;
  extern __shared__ __align__(1024) unsigned char smem_raw[];
  const AttnArgs& a = g.a;
  TcCtl& sm = *reinterpret_cast<TcCtl*>(smem_raw);
  const uint32_t base = smem_u32(smem_raw) + kCtl;
  const uint32_t q_at = base, k_at = q_at + C::QB * C::NP * kPanel, v_at = k_at + C::NKB * C::NP * C::PB, x_at = v_at + C::NVB * C::NP * C::PB;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int rank = C::PAIR == 2 ? (int)(blockIdx.x & 1) : 0, col0 = rank * C::OC;      // its columns: from col0 on
  constexpr uint32_t FULL = 0xffffffffu;
  int fail = (smem_u32(smem_raw) & 1023u) ? 1 : 0;             // (swizzled panels need a 1024-byte aligned base)
  if (tid == 0) {
    for (int i = 0; i < kItems; ++i) { bar_init(&sm.item_full[i], 1); bar_init(&sm.item_free[i], kWarps - 1); }
    for (int i = 0; i < 4; ++i) { bar_init(&sm.fullV[i], 32 * C::TEAM); bar_init(&sm.fullK[i], 32 * C::TEAM); bar_init(&sm.emptyK[i], 1); bar_init(&sm.emptyV[i], 1); bar_init(&sm.s_full[i], 1); bar_init(&sm.p_ready[i], kTile); bar_init(&sm.s_free[i], 1); bar_init(&sm.x_full[i], 1); bar_init(&sm.x_free[i], 1); bar_init(&sm.bad_full[0][i], 1); bar_init(&sm.bad_full[1][i], 1); }
    for (int i = 0; i < 2; ++i) { bar_init(&sm.fullQ[i], g.q_box ? 1 : 32); bar_init(&sm.emptyQ[i], 1); bar_init(&sm.o_full[i], 1); bar_init(&sm.o_free[i], kTile); bar_init(&sm.drained[i], 1); }
    bar_init(&sm.stat_full, kTile); bar_init(&sm.stat_free, kTile);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (tid < 32) sm.redo[tid] = 0;
  if (tid == 32) sm.failed = 0;
  if (warp == kMmaWarp) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(smem_u32(&sm.tmem_base)) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  auto all_sync = [&]() { __syncwarp(); if (C::PAIR == 2) pair_sync(); else __syncthreads(); };
  fence_before();
  all_sync();                                                   // (a pair: each has its barriers before the other reaches for them)
  fence_after();
  const uint32_t tm = sm.tmem_base, s_col = tm, o_col = tm + 2 * kTile;

  auto wait = [&](uint64_t* b, uint32_t parity) { if (!fail && !bar_wait<C::PAIR == 2>(b, parity, g.tries)) fail = 1; };
  // After the first round: whether there is a second (alike in all threads of a CTA or a pair).
  auto marks = [&](int i) {
    uint32_t m = sm.redo[i & 31];
    if (C::PAIR == 2) {
      uint32_t v;
      asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(v) : "r"(other_cta(&sm.redo[i & 31], rank ^ 1)) : "memory");
      m |= v;
    }
    return m;
  };
  auto again = [&]() {
    all_sync();
    uint32_t any = 0;
    for (int i = 0; i < 32; ++i) any |= marks(i);
    return any != 0;
  };
  // Calls body(item) for this CTA's items, as the list warp finds them, until it marks the end; then, where one has left a mark, for those.
  auto walk = [&](auto&& body) {
    uint32_t slot = 0, parity = 0;
#pragma unroll 1
    for (int round = 0; round < 2; ++round) {
#pragma unroll 1
      for (bool end = false; !end;) {
        wait(&sm.item_full[slot], parity);
        fail = __any_sync(0xffffffffu, fail);
        if (fail) break;                                   // (without its item a role has nothing to go by)
        const Item& w = sm.item[slot];
        end = w.t.ok == 0;
        if (!end) body(w);
        __syncwarp();
        if (lane == 0) bar_arrive(&sm.item_free[slot]);
        if (++slot == kItems) { slot = 0; parity ^= 1; }
      }
      if (round == 0 && !again()) break;
    }
  };

  if (warp == kListWarp) {
    // ------------------------------------------------------------------ items
    uint32_t c = 0;
#pragma unroll 1
    for (int round = 0; round < 2; ++round) {
      int li = 0;
      int idx = blockIdx.x / C::PAIR;
#pragma unroll 1
      for (bool more = true; more; idx += gridDim.x / C::PAIR, ++li) {
        if (idx < g.items && round && !(marks(li >> 5) >> (li & 31) & 1u)) continue;
        const int i2 = idx / a.s.Hk, hk = idx - i2 * a.s.Hk, unit = i2 / a.nsplit, split = i2 - unit * a.nsplit;
#pragma unroll 1
        for (int mode = round; more && mode <= 2 * round; ++mode, ++c) {
          wait(&sm.item_free[c % kItems], (c / kItems & 1) ^ 1);
          fail = __any_sync(0xffffffffu, fail);
          if (fail) { more = false; break; }               // (the others may still be at the item in that place)
          Item& w = sm.item[c % kItems];
          TileList t;
          t.ok = 0;
          if (idx < g.items) t = make_list(a, unit, hk, NT * kTile, w.depth, w.anc);
          more = t.ok != 0;
          int k0 = 0, k1 = 0, nb = 0;
          bool missing = false;
          if (t.ok == 1) {
            const int blocks = (t.nk + C::BN - 1) / C::BN, per = (blocks + a.nsplit - 1) / a.nsplit;
            k0 = min(t.nk, split * per * C::BN);
            k1 = min(t.nk, k0 + per * C::BN);
            nb = (k1 - k0 + C::BN - 1) / C::BN;
            if (a.c.page_table) {                          // the last position of the list in each of its pages
              const int P = a.c.page_tokens, s1 = min(t.ns, t.L) - 1, w1 = min(t.L, t.lo + (t.nc - t.ns)) - 1;
              for (int lp = lane; s1 >= 0 && lp <= s1 / P; lp += 32) missing |= tok_cache_row(a.c, a.s.window, a.s.n_sink, t.b, min(s1, lp * P + P - 1)) < 0;
              for (int lp = t.lo / P + lane; w1 >= t.lo && lp <= w1 / P; lp += 32) missing |= tok_cache_row(a.c, a.s.window, a.s.n_sink, t.b, min(w1, lp * P + P - 1)) < 0;
            }
          }
          missing = __any_sync(0xffffffffu, missing);
          // The queries into L2, two items before they are copied: those copies all come at once, when Q is free, and left to them HBM would
          // idle in between.
          if (nb && mode == 0 && rank == 0) {
            const int t0 = t.r0 / a.G, t1 = (t.r0 + t.nr - 1) / a.G;
            for (int tok = t0 + lane; tok <= t1; tok += 32)
              asm volatile("cp.async.bulk.prefetch.L2.global [%0], %1;" ::"l"(reinterpret_cast<const bf16*>(a.in.q) + (t.row0 + tok) * a.in.q_ld + (size_t)hk * a.G * a.s.d), "r"(a.G * a.s.d * 2) : "memory");
          }
          if (lane == 0) {
            w.t = t; w.unit = unit; w.split = split; w.k0 = k0; w.k1 = k1; w.nb = nb; w.nt = t.ok && t.nr > kTile ? 2 : 1; w.mode = mode; w.li = li; w.missing = missing;
            if (missing && rank == 0) atomicOr(a.status + t.b, TSV_ST_PAGE);
          }
          __syncwarp();
          if (lane == 0) bar_arrive(&sm.item_full[c % kItems]);
        }
      }
      if (round == 0 && (!again() || fail)) break;
    }
  } else if (warp > kListWarp && warp < kOutWarp) {
    // ------------------------------------------------------------------ producers
    // Four rows x 128 bytes go with an instruction; a lane knows where the rows lane, lane + 32, .. of the warp's share begin.
    const int chunk = lane & 7, sub = lane >> 3, dch = a.s.d / 8, me = warp - kListWarp - 1;
    const char* none = reinterpret_cast<const char*>(a.in.q);
    // Rows r0 .. r0 + n.value - 1 of this CTA's columns; at: where row r0 + lane begins (0: nothing there)
    auto copy_rows = [&](auto n, uint32_t to, uint32_t stride, int r0, unsigned long long at) {
      const int pan0 = rank * C::NP;
#pragma unroll
      for (int i = 0; i < decltype(n)::value / 4; ++i) {
        const unsigned long long b = __shfl_sync(0xffffffffu, at, 4 * i + sub);
        const int r = r0 + 4 * i + sub;
        const uint32_t dst = to + r * 128 + ((chunk ^ (r & 7)) << 4);
        const char* src = reinterpret_cast<const char*>(b) + (pan0 * 8 + chunk) * 16;
#pragma unroll
        for (int p = 0; p < C::NP; ++p) {
          const bool live = b && (pan0 + p) * 8 + chunk < dch;
          cp16(dst + p * stride, live ? src + p * 128 : none, live);
        }
      }
    };
    if (me == kCopyWarps - 1) {
      uint32_t par = 3, qb = 0, used = 0, last = 3;        // a bit per buffer; used: it has been filled, last: that phase's parity
      walk([&](const Item& w) {
        if (w.nb == 0) return;
        if (C::PAIR == 1) { wait(&sm.emptyQ[0], par & 1); par ^= 1u; }
#pragma unroll 1
        for (int tile = 0; tile < w.nt; ++tile) {
          const int r0 = w.t.r0 + tile * kTile, hk = w.t.hk;
          if (C::PAIR == 1) qb = tile; else { wait(&sm.emptyQ[qb], par >> qb & 1); par ^= 1u << qb; }
          fail = __any_sync(FULL, fail);
          if (fail) return;
          used |= 1u << qb; last ^= 1u << qb;
          const uint32_t to = q_at + qb * C::NP * kPanel;
          if (g.q_box) {
            if (lane == 0) {
              const uint32_t bar = smem_u32(sm.fullQ + qb);
              asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(C::NP * kPanel) : "memory");
              for (int p = 0; p < C::NP; ++p) tma_box3(to + p * kPanel, &g.q, (rank * C::NP + p) * 64, hk * a.G + r0 % a.G, (int)(w.t.row0 + r0 / a.G), bar);
            }
            __syncwarp();
          } else {
#pragma unroll 1
            for (int x = 0; x < kTile; x += 32) {
              const int gr = r0 + x + lane;
              unsigned long long at = 0;
              if (gr - w.t.r0 < w.t.nr) at = reinterpret_cast<unsigned long long>(reinterpret_cast<const bf16*>(a.in.q) + (w.t.row0 + gr / a.G) * a.in.q_ld + ((size_t)hk * a.G + gr % a.G) * a.s.d);
              copy_rows(Int<32>{}, to, kPanel, x, at);
            }
            bar_arrive_copied(sm.fullQ + qb);
          }
          if (C::PAIR == 2) qb ^= 1;
        }
      });
      // (whoever has failed, no copy is under way at the end, and no product: nearly always they are done long before)
      for (int i = 0; i < 2; ++i) if (used >> i & 1u) bar_wait_on(smem_u32(&sm.fullQ[i]), last >> i & 1u, kDrain);
    } else {
      const bool is_v = !C::KP || me >= C::TEAM;
      const int r0 = C::RW * (me % C::TEAM);               // of a block's rows, and every RW TEAM rows on
      uint64_t* full = is_v ? sm.fullV : sm.fullK;
      uint64_t* room = is_v ? sm.emptyV : sm.emptyK;
      const uint32_t base_at = is_v ? v_at : k_at;
      const int nbuf = is_v ? C::NVB : C::NKB;
      uint32_t par = 0xffffffffu;                          // a bit per buffer
      int buf = 0;
      walk([&](const Item& w) {
        const int nb = w.nb;
        if (nb == 0) return;
        const int hk = w.t.hk;
        constexpr int X = C::BN / (C::RW * C::TEAM), STEP = C::RW * C::TEAM;
        unsigned long long at[X];
        auto find = [&](int j) {                           // where this lane's rows of block j begin
#pragma unroll
          for (int x = 0; x < X; ++x) {
            const int r = r0 + STEP * x + lane, kk = w.k0 + j * C::BN + r;
            at[x] = 0;
            if (lane < C::RW && kk < w.k1) {
              const int64_t code = list_row(a, w.t, kk);
              if (code != -1) at[x] = reinterpret_cast<unsigned long long>(row_ptr<bf16>(a, hk, code, is_v));
            }
          }
        };
        find(0);
#pragma unroll 1
        for (int j = 0; j < nb; ++j) {
          const int rows16 = (min(C::BN, w.k1 - w.k0 - j * C::BN) + 15) & ~15;
          const uint32_t to = base_at + buf * C::NP * C::PB;
          wait(&room[buf], par >> buf & 1);
#pragma unroll
          for (int x = 0; x < X; ++x)
            if (r0 + STEP * x < rows16) copy_rows(Int<C::RW>{}, to, C::PB, r0 + STEP * x, at[x]);
          if (w.mode == 2 && is_v) {                       // (what this thread has copied)
            cp_commit();
            cp_wait<0>();
            for (int p = 0; p < C::NP; ++p)
              for (int x = 0; x < X; ++x)
                for (int r = r0 + STEP * x + sub, e = 0; e < C::RW / 4 && r0 + STEP * x < rows16; ++e, r += 4)
                  make_finite<bf16>(smem_raw + (to + p * C::PB + r * 128 + ((chunk ^ (r & 7)) << 4) - smem_u32(smem_raw)));
            bar_arrive(&full[buf]);
          } else {
            bar_arrive_copied(&full[buf]);
          }
          par ^= 1u << buf;
          buf = buf + 1 == nbuf ? 0 : buf + 1;
          if (j + 1 < nb) find(j + 1);
        }
      });
    }
    cp_commit();
    cp_wait<0>();
  } else if (warp == kMmaWarp || warp == kOutWarp) {
    // ------------------------------------------------------------------ products (issued by one thread of a converged warp)
    const uint32_t idesc_v = make_idesc(C::OC, 1);
    const bool one = elect_one();
    // the next S buffer of each tile, in a byte of its own (an item of one tile does not use the other's)
    auto next = [&](uint32_t x, int t) { return (x >> 8 * t & 255u) + 1 == C::SB ? x & ~(255u << 8 * t) : x + (1u << 8 * t); };
    // S buffer xs = Q (buffer qb) K^T (buffer kb, of K or V), `keys` of them
    auto scores = [&](int xs, int qb, int kb, int keys, bool go) {
      fence_proxy();
      fence_after();
      // (values that the compiler knows to be the warp's: they go through uniform registers, one instruction each for a product)
      const uint32_t qd = uniform(desc_lo(q_at + qb * C::NP * kPanel, 1)), kd = uniform(desc_lo((C::KP ? k_at : v_at) + kb * C::NP * C::PB, 1));
      const uint32_t to = uniform(s_col + xs * C::SW), id = uniform(make_idesc((min(C::BN, keys) + 15) & ~15, 0));
      if (go) {
#pragma unroll
        for (int i = 0; i < 4 * C::NP; ++i)
          mma_ss2(to, qd + (i >> 2) * (kPanel >> 4) + 2 * (i & 3), kDescHi, kd + (i >> 2) * (C::PB >> 4) + 2 * (i & 3), kDescHi, id, i != 0);
      }
    };
    // O of tile t (+)= P (S buffer xo) V (buffer vo)
    auto output = [&](int t, int xo, int vo, int keys, int acc, bool go) {
      fence_proxy();
      fence_after();
      const uint32_t vd = uniform(desc_lo(v_at + vo * C::NP * C::PB, C::PB >> 4)), pc = uniform(s_col + xo * C::SW), oc = uniform(o_col + t * C::OC);
      const uint32_t left = uniform(keys), more = uniform(acc);
      if (go) {
#pragma unroll
        for (int k = 0; k < C::BN / 16; ++k) {
          if (16 * k >= (int)left) break;
          mma_ts2(oc, pc + 8 * k, vd + k * (2048 >> 4), kDescHi, idesc_v, k ? 1u : more);
        }
      }
    };
    if (warp == kMmaWarp) {
      // Scores, as far ahead as buffers allow, into the next item too
      constexpr int NB = C::KP ? C::NKB : C::NVB;
      uint64_t* full = C::KP ? sm.fullK : sm.fullV;
      uint32_t par_q = 0, par_k = 0, par_s = 0xfu;         // parities: a bit per buffer
      uint32_t x = 0;
      int kb = 0, qx = 0;                                  // next buffer of K, of a pair's Q
      walk([&](const Item& w) {
        const int nb = w.nb, nt = NT == 2 ? w.nt : 1, k_all = w.k1 - w.k0;
        if (nb == 0) return;
#pragma unroll 1
        for (int j = 0; j < nb; ++j) {
          wait(&full[kb], par_k >> kb & 1);
          par_k ^= 1u << kb;
#pragma unroll 1
          for (int t = 0; t < nt; ++t) {
            const int xs = t * C::SB + (int)(x >> 8 * t & 255u), qb = C::PAIR == 2 ? qx : t;
            if (j == 0) { wait(&sm.fullQ[qb], par_q >> qb & 1); par_q ^= 1u << qb; }
            wait(&sm.s_free[xs], par_s >> xs & 1);
            par_s ^= 1u << xs;
            fail = __any_sync(0xffffffffu, fail);
            const bool go = one && !fail;
            scores(xs, qb, kb, k_all - j * C::BN, go);
            if (go) {
              if (C::KP && t == nt - 1) mma_commit(&sm.emptyK[kb]);
              mma_commit(&sm.s_full[xs]);
              if (j == nb - 1 && t == nt - 1) mma_commit(&sm.emptyQ[C::PAIR == 2 ? qb : 0]);
            }
            __syncwarp();
            x = next(x, t);
          }
          kb = kb + 1 == NB ? 0 : kb + 1;
        }
        qx ^= 1;
      });
    } else {
      // Outputs
      uint32_t par_v = 0, par_p = 0, par_o = 3, x = 0;
      int vb = 0;
      walk([&](const Item& w) {
        const int nb = w.nb, nt = NT == 2 ? w.nt : 1, k_all = w.k1 - w.k0;
#pragma unroll 1
        for (int j = 0; j < nb; ++j) {
          wait(&sm.fullV[vb], par_v >> vb & 1);
          par_v ^= 1u << vb;
#pragma unroll 1
          for (int t = 0; t < nt; ++t) {
            const int xo = t * C::SB + (int)(x >> 8 * t & 255u);
            if (j == 0) { wait(&sm.o_free[t], par_o >> t & 1); par_o ^= 1u << t; }
            wait(&sm.p_ready[xo], par_p >> xo & 1);
            par_p ^= 1u << xo;
            fail = __any_sync(0xffffffffu, fail);
            const bool go = one && !fail;
            output(t, xo, vb, k_all - j * C::BN, j, go);
            if (go) {
              if (t == nt - 1) mma_commit(&sm.emptyV[vb]);
              mma_commit(&sm.s_free[xo]);
              if (j == nb - 1) mma_commit(&sm.o_full[t]);
            }
            __syncwarp();
            x = next(x, t);
          }
          vb = vb + 1 == C::NVB ? 0 : vb + 1;
        }
      });
    }
    uint64_t* done = &sm.drained[warp == kOutWarp];
    if (one) mma_commit(done);
    __syncwarp();
    bar_wait_on(smem_u32(done), 0, kDrain);
  } else {
    // ------------------------------------------------------------------ softmax and epilogue
    const int grp = warp >> 2, q4 = warp & 3;              // (a warp reaches the 32 lanes of tensor memory of its number modulo 4)
    const uint32_t lane_at = (uint32_t)(q4 * 32) << 16;
    const int tile = NT == 2 ? grp : 0, row = q4 * 32 + lane;
    auto out_at = [&](const TileList& t, int r) {          // (r: within the item)
      const int gr = t.r0 + r;
      return reinterpret_cast<bf16*>(a.out) + ((t.row0 + gr / a.G) * a.s.H + (size_t)t.hk * a.G + gr % a.G) * a.s.d;
    };
    auto part_at = [&](const Item& w, int r) { return ((size_t)(w.unit * a.s.Hk + w.t.hk) * a.nsplit + w.split) * (NT * kTile) + r; };
    auto position = [&](const Item& w, int r, uint32_t& an) {      // of row r; its ancestors
      const int tok = (w.t.r0 + min(r, w.t.nr - 1)) / a.G;
      an = a.bt.parent ? w.anc[tok] : 0;
      return w.t.L + (a.bt.parent ? w.depth[tok] : tok);
    };
    // Rows without keys: zeros of a flagged sequence, or an empty share of split keys.
    auto no_keys = [&](const Item& w) {
      const int r = tile * kTile + row;
      if (w.mode || r >= w.t.nr) return;
      if (w.t.ok == 2) {                                   // (with the keys split: the join's)
        uint4* o = reinterpret_cast<uint4*>(out_at(w.t, r));
        if (a.nsplit == 1)
          for (int c = col0 / 8; c < min(a.s.d, col0 + C::OC) / 8; ++c) o[c] = make_uint4(0, 0, 0, 0);
      } else if (col0 == 0) {
        a.pml[part_at(w, r)] = make_float2(-INFINITY, 0.f);
      }
    };
    // O out of tensor memory; its rows' reference and sum are ref and sum.  bad: of mode 1, for mode 2.
    bool bad = false;
    uint32_t turn = 0;
    // A row that is bad in one CTA of a pair is so in both: its columns are to come from the same scores.
    auto bad_in_pair = [&](bool odd) {
      const uint32_t mine = __ballot_sync(FULL, odd), k = turn & 1;
      if (lane == 0) {
        asm volatile("st.shared::cluster.u32 [%0], %1;" ::"r"(other_cta(&sm.bad[k][q4], rank ^ 1)), "r"(mine) : "memory");
        asm volatile("mbarrier.arrive.release.cluster.shared::cluster.b64 _, [%0];" ::"r"(other_cta(&sm.bad_full[k][q4], rank ^ 1)) : "memory");
      }
      if (!fail && !bar_wait_pair_on(smem_u32(&sm.bad_full[k][q4]), turn >> 1 & 1, g.tries)) fail = 1;
      ++turn;
      return ((mine | *(volatile uint32_t*)&sm.bad[k][q4]) >> lane & 1u) != 0;
    };
    auto epilogue = [&](const Item& w, float ref, float sum) {
      const TileList& t = w.t;
      const int mode = w.mode, rt = tile * kTile, r0 = rt + q4 * 32;
      // (mode 2 writes the marked rows only: the others' results of the first round are right)
      const bool live = rt + row < t.nr, put = live && (mode == 0 || (mode == 2 && bad));
      const uint32_t ocol = o_col + tile * C::OC + lane_at;
      bool odd = !is_finite(sum) || (ref == -INFINITY && a.nsplit == 1);
      if (a.nsplit > 1) {
        const size_t part = part_at(w, rt + row);
        float* po = a.po + part * a.s.d + col0;
        float nz = 0.f;                                    // 0 x each value: NaN where one is not finite
#pragma unroll 1
        for (int c = 0; c < C::OC; c += 32) {
          uint32_t r[32];
          tmem_ld32(ocol + c, r);
#pragma unroll
          for (int e = 0; e < 32; e += 4) {
#pragma unroll
            for (int i = 0; i < 4; ++i) nz = fmaf(__uint_as_float(r[e + i]), 0.f, nz);
            if (put && col0 + c + e < a.s.d) *reinterpret_cast<uint4*>(po + c + e) = make_uint4(r[e], r[e + 1], r[e + 2], r[e + 3]);
          }
        }
        odd |= !(nz == 0.f);
        if (put && col0 == 0) a.pml[part] = make_float2(ref, sum);
      } else {
        // a row per lane, 32 bytes of it at a time: whole sectors, no exchanges between lanes
        const float inv = 1.f / sum;
        const uint64_t inv2 = pair2(inv, inv);
        bf16* o = out_at(t, min(rt + row, t.nr - 1)) + col0;
        const bool wide = (((uintptr_t)a.out | (uintptr_t)(a.s.d * 2)) & 31) == 0;
        const __nv_bfloat162 zero2 = __floats2bfloat162_rn(0.f, 0.f);
        __nv_bfloat162 nz[2] = {zero2, zero2};             // 0 x each value: NaN where one is not finite
#pragma unroll 1
        for (int c = 0; c < C::OC; c += 32) {
          uint32_t r[32];
          tmem_ld32(ocol + c, r);
#pragma unroll
          for (int e = 0; e < 32; e += 2) {
            const float2 x = unpair(mul2(pair2(__uint_as_float(r[e]), __uint_as_float(r[e + 1])), inv2));
            const __nv_bfloat162 v = __floats2bfloat162_rn(x.x, x.y);
            nz[(e >> 1) & 1] = __hfma2(v, zero2, nz[(e >> 1) & 1]);
            r[e >> 1] = *reinterpret_cast<const uint32_t*>(&v);
          }
          const int left = a.s.d - col0 - c;     // columns that there are
          if (put && wide) {
            if (left >= 16) store32(o + c, r);
            if (left >= 32) store32(o + c + 16, r + 8);
          } else if (put) {
#pragma unroll
            for (int e = 0; e < 4; ++e)
              if (8 * e < left) *reinterpret_cast<uint4*>(o + c + 8 * e) = make_uint4(r[4 * e], r[4 * e + 1], r[4 * e + 2], r[4 * e + 3]);
          }
        }
        const float2 za = __bfloat1622float2(nz[0]), zb = __bfloat1622float2(nz[1]);
        odd |= !(za.x == 0.f && za.y == 0.f && zb.x == 0.f && zb.y == 0.f);
      }
      fence_before();
      bar_arrive(&sm.o_free[tile]);
      odd = odd && live;
      if (mode == 0 && odd) atomicOr(&sm.redo[(w.li >> 5) & 31], 1u << (w.li & 31));
      if (mode == 1) bad = C::PAIR == 2 ? bad_in_pair(odd) : odd;
      if (mode == 2) {
        uint32_t an;
        const int p = position(w, rt + row, an);
        const uint32_t still = __ballot_sync(FULL, C::PAIR == 2 ? bad_in_pair(odd) : odd);
        __syncwarp();                                      // (a row's own lane has written it before: the warp's stores come behind those)
        for (uint32_t todo = __ballot_sync(FULL, bad); todo; todo &= todo - 1) {
          const int x = __ffs(todo) - 1;
          exact_output(a, t, w.depth, t.r0 + r0 + x, __shfl_sync(FULL, p, x), __shfl_sync(FULL, an, x), w.k0, w.k1, col0,
                       min(a.s.d, col0 + C::OC), part_at(w, r0 + x), still >> x & 1u);
        }
      }
    };
    if (NT == 1 && grp == 1) {
      // ---------------------------------------------------------------- epilogue of the one tile
      uint32_t n = 0;
      walk([&](const Item& w) {
        if (w.nb == 0) { no_keys(w); return; }
        wait(&sm.stat_full, n & 1);
        const float2 st = sm.stat[row];
        bar_arrive(&sm.stat_free);
        wait(&sm.o_full[0], n & 1);
        ++n;
        fence_after();
        epilogue(w, st.x, st.y);
      });
    } else {
      // ---------------------------------------------------------------- softmax
      uint32_t cS = 0, par_s = 0, n = 0;                   // blocks so far, parities of s_full; items
      // O holds the blocks before this one.
      auto wait_o = [&]() {
        wait(&sm.s_free[tile * C::SB + (cS - 1) % C::SB], (cS - 1) / C::SB & 1);
        fence_after();
      };
      // A pair: this row's part of the scores goes to the other CTA, and that one's part is added (the sum is the same bits in both).
      uint32_t sv[C::SL], par_x = 0;
      const uint32_t x_mine = x_at + row * 16, x_to = C::PAIR == 2 ? other_cta(smem_raw + (x_mine - smem_u32(smem_raw)), rank ^ 1) : 0;
      const uint32_t x_full_to = C::PAIR == 2 ? other_cta(&sm.x_full[q4], rank ^ 1) : 0, x_free_to = C::PAIR == 2 ? other_cta(&sm.x_free[q4], rank ^ 1) : 0;
      auto load = [&](uint32_t col) {                      // (to be followed by a wait and `loaded`)
        tmem_ld32_nowait(col, sv);
        if (C::SL == 64) tmem_ld32_nowait(col + 32, sv + 32); else tmem_ld16_nowait(col + 32, sv + 32);
      };
      auto loaded = [&]() {
        asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
        tmem_regs_ready(sv);
        if (C::SL == 64) tmem_regs_ready(sv + 32); else tmem_regs_ready16(sv + 32);
      };
      auto send = [&](int x) {                             // the scores of buffer x, which stay in sv
        wait(&sm.s_full[x], par_s >> x & 1);
        par_s ^= 1u << x;
        fence_after();
        load(s_col + x * C::SW + lane_at);
        wait(&sm.x_free[q4], par_x ^ 1);
        if (lane == 0 && !fail) asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(smem_u32(&sm.x_full[q4])), "r"(32 * C::SL * 4) : "memory");
        loaded();
        if (fail) return;
#pragma unroll
        for (int e = 0; e < C::SL; e += 4)
          asm volatile("st.async.weak.shared::cluster.mbarrier::complete_tx::bytes.v4.b32 [%0], {%1, %2, %3, %4}, [%5];"
                       ::"r"(x_to + e * (kTile * 4)), "r"(sv[e]), "r"(sv[e + 1]), "r"(sv[e + 2]), "r"(sv[e + 3]), "r"(x_full_to) : "memory");
      };
      auto receive = [&]() {
        if (!fail && !bar_wait_pair(&sm.x_full[q4], par_x, g.tries)) fail = 1;
#pragma unroll
        for (int h = 0; h < C::SL; h += 24) {
          float v[24];
#pragma unroll
          for (int e = 0; e < 24; e += 4)
            asm volatile("ld.shared.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(v[e]), "=f"(v[e + 1]), "=f"(v[e + 2]), "=f"(v[e + 3]) : "r"(x_mine + (h + e) * (kTile * 4)) : "memory");
#pragma unroll
          for (int e = 0; e < 24; e += 2) {
            const float2 y = unpair(add2(pair2(__uint_as_float(sv[(h + e) % C::SL]), __uint_as_float(sv[(h + e + 1) % C::SL])), pair2(v[e], v[e + 1])));
            sv[(h + e) % C::SL] = __float_as_uint(y.x); sv[(h + e + 1) % C::SL] = __float_as_uint(y.y);
          }
        }
        // (the sums are made before anything that follows, so the loads are done by then: see `taken`)
        tmem_regs_ready(sv);
        tmem_regs_ready16(sv + 32 % C::SL);
        par_x ^= 1;
      };
      // What was received has been read by the whole warp: the other CTA may send again.  The arrival is relaxed, and what orders the lanes'
      // loads before it is a dependency, not the memory model's release: every value that was loaded has been added to a sum (receive), which a
      // load that is still open would have held up, and lane 0 arrives after the warp has come together behind that.  (Nothing that this warp
      // writes is handed over here.  With a release, which waits for all of the thread's accesses, the scores on their way to the other CTA
      // among them: 8 x 2000 tokens 886 us instead of 793.)
      auto taken = [&]() {
        __syncwarp();
        if (lane == 0) asm volatile("mbarrier.arrive.relaxed.cluster.shared::cluster.b64 _, [%0];" ::"r"(x_free_to) : "memory");
      };
      walk([&](const Item& w) {
        const TileList& t = w.t;
        if (w.nb == 0) { if (NT == 2) no_keys(w); return; }
        if (tile * kTile >= t.nr) return;
        // what this row sees of the list: positions kmin .. kmax and those below ksink, nodes
        const bool tree = a.bt.parent != nullptr, missing = w.missing != 0;
        uint32_t an;
        const int p = position(w, tile * kTile + row, an), nb = w.nb, k0 = w.k0, k1 = w.k1, nc = t.nc;
        const int shift = t.ns - t.lo;                     // index of a position of the window part, less the position
        const int kmin = max(0, p - a.s.window + 1 + shift), kmax = tree ? nc - 1 : p + shift;
        const int ksink = min(max(t.ns, min(a.s.n_sink, t.nk) + shift), kmax + 1);
        uint32_t nodes = 0;
        if (tree)
          for (int j = 0; j < t.n; ++j)
            if ((an >> j & 1u) && (t.L + w.depth[j] > p - a.s.window || t.L + w.depth[j] < a.s.n_sink)) nodes |= 1u << j;
        // keys that every row of the warp sees
        const int all0 = __reduce_max_sync(FULL, kmin), all1 = min(min(__reduce_min_sync(FULL, kmax) + 1, nc), k1);
        float ref = -INFINITY;
        uint64_t l2[4] = {0, 0, 0, 0};                     // (four sums of two)
        const uint64_t scale2 = pair2(a.scale2, a.scale2);
        if (C::PAIR == 2) send(cS % C::SB);
#pragma unroll 1
        for (int j = 0; j < nb; ++j) {
          const int x = tile * C::SB + (int)(cS % C::SB), c0 = k0 + j * C::BN, slabs = (min(C::BN, k1 - c0) + C::SL - 1) / C::SL;
          const uint32_t scol = s_col + x * C::SW + lane_at;
          if (C::PAIR == 1) {
            wait(&sm.s_full[x], par_s >> x & 1);
            par_s ^= 1u << x;
            fence_after();
          }
#pragma unroll 1
          for (int i = 0; i < slabs; ++i) {
            const int c = c0 + C::SL * i;
            if (C::PAIR == 1) load(scol + C::SL * i);
            uint32_t vis[2];
            bool whole[2];
#pragma unroll
            for (int v = 0; v < 2; ++v) {
              const int wide = v ? C::SL - 32 : 32, cv = c + 32 * v, x = nc - cv;
              const uint32_t every = FULL >> (32 - wide);
              whole[v] = !missing && cv >= all0 && cv + wide <= all1;
              vis[v] = every;
              if (!whole[v]) {
                vis[v] = bits(kmin - cv, min(kmax + 1, nc) - cv) | bits(-cv, min(ksink, nc) - cv);
                if (tree && x < 32 && x > -32) vis[v] |= x >= 0 ? nodes << x : nodes >> -x;
                vis[v] &= bits(0, min(wide, k1 - cv));
                if (missing) vis[v] = have_pages(a, t, cv, vis[v]);
                whole[v] = __all_sync(FULL, vis[v] == every);
              }
            }
            if (C::PAIR == 1) loaded(); else receive();
#pragma unroll
            for (int v = 0; v < 2; ++v) {
              if (whole[v]) continue;
#pragma unroll
              for (int e = 0; e < (v ? C::SL - 32 : 32); ++e) if (!(vis[v] >> e & 1u)) sv[32 * v + e] = 0xff800000u;
            }
            float m8[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) m8[e] = fmaxf(fmaxf(__uint_as_float(sv[e]), __uint_as_float(sv[e + 8])), __uint_as_float(sv[e + 16]));
#pragma unroll
            for (int e = 24; e < C::SL - 8; e += 16)
#pragma unroll
              for (int x = 0; x < 8; ++x) m8[x] = fmaxf(fmaxf(m8[x], __uint_as_float(sv[e + x])), __uint_as_float(sv[e + 8 + x]));
#pragma unroll
            for (int x = 0; x < 8; ++x) m8[x] = fmaxf(m8[x], __uint_as_float(sv[C::SL - 8 + x]));
            const float mx = fmaxf(fmaxf(fmaxf(m8[0], m8[1]), fmaxf(m8[2], m8[3])), fmaxf(fmaxf(m8[4], m8[5]), fmaxf(m8[6], m8[7]))) * a.scale2;
            const bool up = mx > ref + kGap || (ref == -INFINITY && mx > ref);
            const bool any_up = __any_sync(FULL, up);
            if (C::PAIR == 2) taken();
            if (any_up) {                                  // (alike in the warp: accesses to tensor memory are the whole warp's)
              const float to = up ? ceilf(mx) : ref, f = up && ref != -INFINITY ? power_of_two(ref - to) : 1.f;
              ref = to;
              if (__any_sync(FULL, f != 1.f)) {
                const uint64_t f2 = pair2(f, f);
#pragma unroll
                for (int x = 0; x < 4; ++x) l2[x] = fma2(l2[x], f2, 0);
                if (j) wait_o();
                rescale(scol, C::SL / 2 * i, o_col + tile * C::OC + lane_at, j ? C::OC : 0, f);
              }
            }
            const float neg = ref == -INFINITY ? 0.f : -ref;
            const uint64_t neg2 = pair2(neg, neg);
#pragma unroll
            for (int e = 0; e < C::SL; e += 2) {
              const float2 y = unpair(fma2(pair2(__uint_as_float(sv[e]), __uint_as_float(sv[e + 1])), scale2, neg2));
              const float p0 = ex2(y.x), p1 = ex2(y.y);
              l2[(e >> 1) & 3] = add2(l2[(e >> 1) & 3], pair2(p0, p1));
              const __nv_bfloat162 h = __floats2bfloat162_rn(p0, p1);
              sv[e >> 1] = *reinterpret_cast<const uint32_t*>(&h);
            }
            tmem_st16(scol + C::SL / 2 * i, sv);
            tmem_st16(scol + C::SL / 2 * i + 16, sv + 16);     // (48: its last eight words lie behind P)
          }
          asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory");
          fence_before();
          bar_arrive(&sm.p_ready[x]);
          ++cS;
          if (C::PAIR == 2 && j + 1 < nb) send(cS % C::SB);
        }
        const float2 la = unpair(add2(l2[0], l2[1])), lb = unpair(add2(l2[2], l2[3]));
        const float sum = (la.x + la.y) + (lb.x + lb.y);
        if (NT == 1) {
          wait(&sm.stat_free, (n & 1) ^ 1);
          sm.stat[row] = make_float2(ref, sum);
          bar_arrive(&sm.stat_full);
          ++n;
        } else {
          wait(&sm.o_full[tile], n & 1);
          ++n;
          fence_after();
          epilogue(w, ref, sum);
        }
      });
    }
  }
  if (__any_sync(FULL, fail)) {                                  // an internal error: every sequence is flagged
    for (int b = lane; b < a.s.B; b += 32) atomicOr(a.status + b, TSV_ST_INTERNAL);
    if (C::PAIR == 2 && lane == 0) {
      *(volatile uint32_t*)&sm.failed = 1;
      asm volatile("st.shared::cluster.u32 [%0], %1;" ::"r"(other_cta(&sm.failed, rank ^ 1)), "r"(1) : "memory");
    }
  }
  fence_before();
  all_sync();                                                   // (a pair: nobody reaches for the other's memory any more)
  // Scores that the other CTA has sent, which nobody may have waited for, land within microseconds.
  if (C::PAIR == 2 && *(volatile uint32_t*)&sm.failed)
    for (int i = 0; i < 1000; ++i) __nanosleep(1000);
  if (warp == kMmaWarp) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, 512;" ::"r"(tm) : "memory");
}

bool query_map(CUtensorMap* m, const AttnArgs& a) {
  static PFN_cuTensorMapEncodeTiled fn = nullptr;
  if (!fn) {
    void* p = nullptr;
    cudaDriverEntryPointQueryResult q;
    if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &p, cudaEnableDefault, &q) == cudaSuccess && q == cudaDriverEntryPointSuccess)
      fn = reinterpret_cast<PFN_cuTensorMapEncodeTiled>(p);
  }
  if (!fn || a.bt.rows < 1) return false;
  const cuuint64_t dim[3] = {(cuuint64_t)a.s.d, (cuuint64_t)a.s.H, (cuuint64_t)a.bt.rows};
  const cuuint64_t stride[2] = {(cuuint64_t)a.s.d * 2, (cuuint64_t)a.in.q_ld * 2};
  const cuuint32_t box[3] = {64u, (cuuint32_t)(a.G < 128 ? a.G : 128), (cuuint32_t)(a.G < 128 ? 128 / a.G : 1)}, one[3] = {1, 1, 1};
  return fn(m, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, const_cast<void*>(a.in.q), dim, stride, box, one, CU_TENSOR_MAP_INTERLEAVE_NONE,
            CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <int DP, bool SHARED>
int tc_launch(const AttnArgs& a, int64_t units, cudaStream_t st) {
  typedef Cfg<DP, SHARED> C;
  TcArgs g;
  g.a = a;
  g.tries = wait_tries(kWaitLimit);
  // (heads that do not fill a box of 128 rows evenly, or rows beyond a tensor map's: by the copying warps' own loads)
  g.q_box = (128 % a.G == 0 || a.G % 128 == 0) && a.bt.rows < (int64_t)1 << 31 && a.in.q_ld < (int64_t)1 << 38 && query_map(&g.q, a);
  const int64_t items = units * a.s.Hk * a.nsplit;
  if (items > 0x7fffffff - 148) return TSV_ERR_LIMIT;
  g.items = (int32_t)items;
  if (!ensure_smem((const void*)attn_tc_kernel<DP, SHARED>, C::SMEM)) return TSV_ERR_CUDA;
  TSV_PREP((attn_tc_kernel<DP, SHARED>));
  const int most = 148 / C::PAIR, grid = g.items < most ? g.items : most;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(grid * C::PAIR));
  cfg.blockDim = dim3(32 * kWarps);
  cfg.dynamicSmemBytes = C::SMEM;
  cfg.stream = st;
  cudaLaunchAttribute at[1];
  at[0].id = cudaLaunchAttributeClusterDimension;
  at[0].val.clusterDim.x = C::PAIR;
  at[0].val.clusterDim.y = at[0].val.clusterDim.z = 1;
  cfg.attrs = at;
  cfg.numAttrs = C::PAIR == 2;
  if (cudaLaunchKernelEx(&cfg, attn_tc_kernel<DP, SHARED>, g) != cudaSuccess) return TSV_ERR_CUDA;
  count_launch();
  return TSV_OK;
}

}  // namespace

int launch_attn_tc(const AttnArgs& a, int64_t units, cudaStream_t st) {
  const int d = a.s.d;
  if (!a.c.v)
    return d <= 64 ? tc_launch<64, true>(a, units, st) : d <= 128 ? tc_launch<128, true>(a, units, st)
         : d <= 256 ? tc_launch<256, true>(a, units, st) : tc_launch<512, true>(a, units, st);
  return d <= 64 ? tc_launch<64, false>(a, units, st) : d <= 128 ? tc_launch<128, false>(a, units, st)
       : d <= 256 ? tc_launch<256, false>(a, units, st) : tc_launch<512, false>(a, units, st);
}

}  // namespace tsv
