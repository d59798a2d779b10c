// Attention of one new token per row over a paged cache: the kernel, compiled per head dimension.
//
// Mathematics.  For up to 8 query heads of one kv head (16 with two products) and a tile of 16
// positions: S^T = K Q^T, the running maximum m and sum l of exp2(S scale log2 e - m), O^T = O^T exp2(m_old - m) +
// V^T P^T.  O, m and l are additive over any cut of the positions once brought to a common maximum, which is all that
// the split over the length needs.
//
// What bounds it.  K and V are read once: 2 G flops per byte (G query heads per kv head, 16-bit cache), far
// below the ~260 of this GPU's tensor cores, so HBM decides and the kernel is built to keep copies in flight:
//   * one CTA per SM; two producer warps walk the CTA's share of all positions of all rows and fill a ring of up to
//     ~200 KB of 32 KB stages by TMA (4-D tensor map over the pool: dim, position, kv head, page; boxes of up to a
//     page, of 16 positions where a row ends), so both layouts cost the same; page ids are looked up 32 at a time, one
//     window ahead; they never wait for the arithmetic until the ring is full.  (One producer warp with 16-position
//     boxes took 1.2 us per stage whatever its bytes: 64 rows of up to 16384 positions 562 us, now 322.)
//   * the share is cut by positions, not by rows: row lengths are read on the device, every CTA sums them up and takes
//     the same number of units (stages; a row's start and end count as 3/4 of one), so ragged batches and one long row
//     load all SMs alike;
//   * a consumer warp takes one piece of 16 positions at a time, 32 or 64 where a row of the cache is 128 bytes or less
//     (mma.sync m16n8k16).  Positions (dims) are the 16 rows of a product and heads its 8 columns: K and V come from the
//     swizzled stage by ldmatrix as they lie there, no row is wasted on G <= 8 heads, and 8 heads x 128 dims of O take 32
//     registers.  P is used as two terms, P - round(P) in a second product: 16 (bf16) or 22 (fp16) bits of it count.
//     tcgen05.mma would need P, a few hundred numbers, written to shared memory and results fetched from tensor memory
//     for every piece; the legacy pipe is 14 to 25 % busy here;
//   * epilogue warps add the consumers' (m, l, O) up at the end of a row, while the consumers go on with the next row.  They are
//     latency-bound: four of them beside ten consumers (two beside twelve: 512 rows x 100, 32/8 heads 72 us, now 57; 64 rows
//     x 16384 329, now 322; with one term of an 8-bit weight, 64 x 4096, 32/8 102, then 99, but 96 x 8192, 64/8 140.5, then 141.4).
//     Rows that lie inside a CTA are written at once; of a row that is cut every CTA leaves (m, l, O) of its piece and
//     k_paged_join adds them up in the order of the CTAs: bits depend on the lengths alone, no atomics.
//   * few rows are latency: each (row, kv head) gets a cluster of CTAs that add their pieces up through distributed
//     shared memory; rows of few units are not cut at all (launch(), cost_of()).
//
// Measured (us in short replays, of the measured copy rate 6451 GB/s): 64 rows x 1..16384 GQA 32/8 x 128 bf16 321
// (100 %); 96 rows x 17..8192 64/8 8-bit 148 (85 %: the widening to fp16 and two terms of a weight keep the warps busy); 1 row x 131071
// 64/8 fp16 90 (92 %: 6 us are start and join); 32 rows x 129..1025 32/32 bf16 56 (84 %: 9 us are start and join); 1 row x 513 32/32 7.2;
// 4 rows x 513..545 64/8 fp32 8.5 (latency).  In a loop of a second the GPU's power cap makes the first 331 to 359 and the second 157 to
// 164.  Few rows over a table with room for 8192 positions or more are cut and joined instead of shared by clusters: 11.1 and 13.9.
// Short rows pay about 1 us per row and kv head for their ends: 128 rows x 200, 64/8 27 (63 %), 128 x 64 15.9 (37 %; pages of 64).
//
// fp32 queries (bf16 cache): q and P are three bf16 terms by truncation (8 + 8 + 8 bits: exact), sums of products short
// chains (error of fp32 outputs against 64 bits 1e-7 .. 3e-7).  8-bit cache: the
// stored numbers are widened to fp16 (exact), bf16 queries are scaled by a power of two per head so that fp16 holds
// them (down to 2^-31 of the head's largest).  Where P is fp16, it is exp2(.. + 15): 2^-29 of the largest stays a normal number.
//
// Every wait is bounded (d3_paged_set_wait_ns); when one runs out the CTA stores D3_ETIMEOUT, stops issuing, lets its copies land and ends.  (A
// cluster's hardware barriers are met by every thread on every path, so they end when those waits have.)
#pragma once

#include <cuda.h>
#include <cuda_fp16.h>

#include <atomic>
#include <type_traits>

#include "d3_paged.cuh"

namespace d3 {
namespace paged_attn {

constexpr int kTile = 16;             // positions of a product's rows, and of the smallest TMA box
constexpr int kProducers = 2;         // warps that issue copies, stage by stage in turn
constexpr int kFewRows = 128;         // rows that a producer warp sums up by itself
constexpr int kMaxStages = 12;
constexpr int kItems = 4;              // items between the consumers and the epilogue at most
constexpr int kSmemMost = 224 * 1024; // of 227 KB
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

template <int CACHE> struct CacheBytes { static constexpr int v = CACHE == D3_E4M3 ? 1 : 2; };
template <int X> struct QBytes { static constexpr int v = X == D3_FP32 ? 4 : 2; };

__device__ __forceinline__ uint32_t smem_u32(const void *p) { return (uint32_t)__cvta_generic_to_shared(p); }
__device__ __forceinline__ uint64_t now_ns() {
  uint64_t t;
  asm volatile("mov.u64 %0, %globaltimer;" : "=l"(t));
  return t;
}
__device__ __forceinline__ void mb_init(uint32_t bar, uint32_t count) {
  asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(bar), "r"(count) : "memory");
}
__device__ __forceinline__ void mb_arrive(uint32_t bar) {
  asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ void mb_arrive_tx(uint32_t bar, uint32_t bytes) {
  asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(bytes) : "memory");
}
__device__ __forceinline__ bool mb_try(uint32_t bar, uint32_t parity) {
  uint32_t ok;
  asm volatile(
      "{\n\t.reg .pred p;\n\tmbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n\tselp.u32 %0, 1, 0, p;\n\t}"
      : "=r"(ok) : "r"(bar), "r"(parity) : "memory");
  return ok != 0;
}
// Bounded wait; false once it, or another wait of the CTA, has run out.
__device__ __forceinline__ bool mb_try_cluster(uint32_t bar, uint32_t parity);
template <bool CLUSTER = false>
__device__ __forceinline__ bool mb_wait(uint32_t bar, uint32_t parity, volatile int *abort_flag, unsigned long long wait_ns,
                                        bool check_abort = true) {
  if (CLUSTER ? mb_try_cluster(bar, parity) : mb_try(bar, parity)) return true;
  const uint64_t t0 = now_ns();
  for (uint32_t it = 1;; ++it) {
    if (CLUSTER ? mb_try_cluster(bar, parity) : mb_try(bar, parity)) return true;
    if ((it & 31u) == 0u) {
      if (check_abort && *abort_flag) return false;
      if (now_ns() - t0 > wait_ns) break;
    }
  }
  *abort_flag = 1;
  return false;
}
// ---- thread-block clusters: an address of another CTA's shared memory, stores and arrivals there
__device__ __forceinline__ uint32_t in_cta(uint32_t addr, uint32_t rank) {
  uint32_t r;
  asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(addr), "r"(rank));
  return r;
}
template <int V>
__device__ __forceinline__ void store_there(uint32_t addr, const float (&v)[V]) {
  if constexpr (V == 4) asm volatile("st.shared::cluster.v4.f32 [%0], {%1,%2,%3,%4};" ::"r"(addr), "f"(v[0]), "f"(v[1]), "f"(v[2]), "f"(v[3]) : "memory");
  else if constexpr (V == 2) asm volatile("st.shared::cluster.v2.f32 [%0], {%1,%2};" ::"r"(addr), "f"(v[0]), "f"(v[1]) : "memory");
  else asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(addr), "f"(v[0]) : "memory");
}
__device__ __forceinline__ void arrive_there(uint32_t bar) {
  asm volatile("mbarrier.arrive.release.cluster.shared::cluster.b64 _, [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ void cluster_arrive() { asm volatile("barrier.cluster.arrive.release;" ::: "memory"); }
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait.acquire;" ::: "memory"); }
__device__ __forceinline__ bool mb_try_cluster(uint32_t bar, uint32_t parity) {
  uint32_t ok;
  asm volatile(
      "{\n\t.reg .pred p;\n\tmbarrier.try_wait.parity.acquire.cluster.shared::cta.b64 p, [%1], %2;\n\tselp.u32 %0, 1, 0, p;\n\t}"
      : "=r"(ok) : "r"(bar), "r"(parity) : "memory");
  return ok != 0;
}
__device__ __forceinline__ void tma_box(uint32_t dst, const CUtensorMap *map, int dim, int pos, int head, int page, uint32_t bar) {
  asm volatile(
      "cp.async.bulk.tensor.4d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4, %5}], [%6];"
      ::"r"(dst), "l"(reinterpret_cast<uint64_t>(map)), "r"(dim), "r"(pos), "r"(head), "r"(page), "r"(bar)
      : "memory");
}
__device__ __forceinline__ void bulk_copy(uint32_t dst, const void *src, uint32_t bytes, uint32_t bar) {
  asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];"
               ::"r"(dst), "l"(src), "r"(bytes), "r"(bar) : "memory");
}
__device__ __forceinline__ void ldsm4(uint32_t (&r)[4], uint32_t addr) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr));
}
// transpose of an 8 x 8 matrix of 16-bit numbers held by the warp
__device__ __forceinline__ uint32_t transpose8(uint32_t v) {
  uint32_t r;
  asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(v));
  return r;
}
__device__ __forceinline__ void ldsm4t(uint32_t (&r)[4], uint32_t addr) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr));
}
template <bool F16>
__device__ __forceinline__ void mma(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  if (F16)   // (not volatile: a function of its registers, free to be scheduled between the loads)
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
  else
    asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ float exp2_fast(float x) {   // 2^x to 2^-22 relative; 0 for -inf
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
template <bool F16>
__device__ __forceinline__ uint32_t pack(float lo, float hi) {
  uint32_t r;
  if (F16) asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  else asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  return r;
}
template <bool F16>
__device__ __forceinline__ void unpack(uint32_t r, float &lo, float &hi) {
  if (F16) {
    const float2 v = __half22float2(*reinterpret_cast<const __half2 *>(&r));
    lo = v.x; hi = v.y;
  } else {
    lo = __uint_as_float(r << 16);
    hi = __uint_as_float(r & 0xffff0000u);
  }
}
// two e4m3 numbers (low 16 bits of v) as two fp16 numbers, exactly
__device__ __forceinline__ uint32_t widen(uint32_t v) {
  uint32_t r;
  const unsigned short h = (unsigned short)v;
  asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(r) : "h"(h));
  return r;
}
// x, y by truncation to their upper 16 bits, packed; and what is left of them
__device__ __forceinline__ uint32_t cut(float &x, float &y) {
  const uint32_t a = __float_as_uint(x) & 0xffff0000u, b = __float_as_uint(y) & 0xffff0000u;
  x -= __uint_as_float(a);
  y -= __uint_as_float(b);
  return (a >> 16) | b;
}

// x / y, without a 64-bit division where 32 bits do
__device__ __forceinline__ long long divide(long long x, int y) {
  return x < (1ll << 32) ? (long long)((uint32_t)x / (uint32_t)y) : x / y;
}
// How `total` cost is dealt out to n CTAs: the first `more` of them get each + 1, the others each.
struct Shares {
  long long each;
  int more;
  __device__ __forceinline__ Shares() {}
  __device__ __forceinline__ Shares(long long total, int n) {
    each = divide(total, n);
    more = (int)(total - each * n);
  }
  __device__ __forceinline__ long long start(int i) const { return each * i + min(i, more); }
  __device__ __forceinline__ int holder(long long x) const {   // the CTA that x belongs to
    const long long edge = (each + 1) * more;
    if (x < edge) return (int)(x / (each + 1));
    return (int)(more + (x - edge) / each);
  }
};
// Cost of an item (the pass over a row's positions for one tile of heads): kUnitCost per unit and kItemCost for its query
// fragments and its sums.  The unit i of an item that starts at cost S belongs to the CTA that holds S + lead +
// step * i.  With few units per CTA only units count, so that no CTA is left without one.  Where items stay whole
// (no join) step and lead are 0, and with no more items than CTAs only items count.
constexpr int kUnitShift = 2, kUnitCost = 1 << kUnitShift, kItemCost = 3;
struct Cost {
  int unit, item, lead, step;
  __device__ __forceinline__ long long of(int units) const { return (long long)unit * units + item; }
  __device__ __forceinline__ long long first_unit(long long past) const {   // the first one at or behind S + lead + past
    return past <= 0 ? 0 : step == 0 ? 0x7fffffff : step == 1 ? past : (past + kUnitCost - 1) >> kUnitShift;
  }
};

enum { STAGE_FIRST = 1, STAGE_LAST = 2, STAGE_FINAL = 4 };   // of the item within this CTA; of the CTA
// an item lies in this CTA / started before it / starts in it and goes on; no item at all
enum { OUT_WHOLE = 0, OUT_HEAD = 1, OUT_TAIL = 2, OUT_NONE = 3 };

// V neighbouring dims of a result, times f, rounded once
template <int X, int V>
__device__ __forceinline__ void write_out(const PagedAttnArgs &a, long long at, const float (&o)[V], float f) {
  if constexpr (X == D3_FP32) {
    float *p = static_cast<float *>(a.out) + at;
    if (V == 4 && a.out_wide) { *reinterpret_cast<float4 *>(p) = make_float4(o[0] * f, o[1 % V] * f, o[2 % V] * f, o[3 % V] * f); return; }
    if (V == 2 && a.out_wide) { *reinterpret_cast<float2 *>(p) = make_float2(o[0] * f, o[1 % V] * f); return; }
#pragma unroll
    for (int e = 0; e < V; ++e) p[e] = o[e] * f;
  } else {
    uint16_t *p = static_cast<uint16_t *>(a.out) + at;
    uint32_t w[(V + 1) / 2];
#pragma unroll
    for (int e = 0; e < V; e += 2) w[e / 2] = pack<X == D3_FP16>(o[e] * f, V > 1 ? o[(e + 1) % V] * f : 0.f);
    if (V == 4 && a.out_wide) { *reinterpret_cast<uint2 *>(p) = make_uint2(w[0], w[V / 2 - 1 < 0 ? 0 : V / 2 - 1]); return; }
    if (V == 2 && a.out_wide) { *reinterpret_cast<uint32_t *>(p) = w[0]; return; }
#pragma unroll
    for (int e = 0; e < V; ++e) p[e] = (uint16_t)(w[e / 2] >> (16 * (e & 1)));
  }
}

// What the producers tell the consumers about a stage (one 16-byte load).
struct __align__(16) StageInfo {
  int row;
  uint32_t heads;       // the tile's first query head | kv head << 16
  uint32_t bits;        // positions in the stage (0 .. 256) | STAGE_* << 9 | OUT_* << 12 | heads of the tile << 14 | (cluster) CTAs it lies in << 19
  uint32_t tiles;       // which tiles hold positions
};
// What the consumers tell the epilogue warps about an item.
struct __align__(16) ItemInfo {
  int row;
  uint32_t heads;       // as above
  uint32_t bits;        // OUT_* | last of the CTA << 2 | heads << 3 | first warp with a piece of it << 8 | such warps << 16 | (cluster) CTAs << 24
};

template <int DH, int CACHE, int X, int MT>
struct Cfg {
  static constexpr int kEs = CacheBytes<CACHE>::v;
  static constexpr int kRow = DH * kEs;                      // bytes of a cache row
  static constexpr int kBox = kRow < 128 ? kRow : 128;       // bytes of a box row = swizzle width
  static constexpr int kBoxes = kRow / kBox;                 // boxes per piece of K (or V)
  static constexpr int kHeads = X == D3_FP32 ? 8 : 8 * MT;   // query heads of a tile
  static constexpr int kUnit = unit_positions(DH, kEs);      // positions of a stage (of up to 32 KB)
  static constexpr int kPT = kRow > 128 ? 1 : kRow > 64 ? 2 : 4;   // tiles of a piece, i.e. of a warp's trip (32 fragment registers)
  static constexpr int kHalfBytes = kUnit * kRow;            // K (or V) of a stage
  static constexpr int kQRow = DH * QBytes<X>::v + 16;       // a query head in shared memory (padded: no bank conflicts)
  static constexpr int kQBytes = kHeads * kQRow;
  static constexpr int kStageBytes = 2 * kHalfBytes;
  // Registers are dealt out to four warps at a time: 16 warps of 128 (which 32 accumulator and 16 query registers fit
  // into), or 12 of 168 for 16 heads or three-term queries.
  static constexpr int kEpilogue = MT == 1 ? 4 : 2;
  static constexpr int kWarps = MT == 1 ? 14 - kEpilogue : 8;      // consumers
  static constexpr int kClusterWarps = MT == 1 ? 12 : 8;           // consumers of a cluster's CTA (three units are one turn)
  static constexpr int kThreads = 32 * (kWarps + kProducers + kEpilogue);
  static constexpr int kHeadFloats = DH + 4;                 // of a head's sums in shared memory (padded: no bank conflicts)
  static constexpr bool kF16 = CACHE != D3_BF16;
  static constexpr int kTiles = X == D3_FP32 ? 1 : MT;       // 8-head tiles
  // Terms of P.  The sums use P unrounded, so what is left of it is an error of the result: 2^-16 with two bf16 numbers, 2^-22 with
  // two fp16 ones.  (One fp16 number under a bf16 result, 2^-11, makes 96 rows x 8192 of 8 bits 141 us instead of 148; results
  // then differ from fp32 arithmetic's by 5.7e-4 of their size, not 5.8e-5, and where values nearly cancel by far more than their rounding.)
  static constexpr int kQTerms = X == D3_FP32 ? 3 : 1, kPTerms = X == D3_FP32 ? 3 : 2;
};

template <int DH, int CACHE, int X, int MT>
__global__ void __launch_bounds__(Cfg<DH, CACHE, X, MT>::kThreads, 1)
k_paged_attention(const __grid_constant__ CUtensorMap map_k, const __grid_constant__ CUtensorMap map_v,
                  const __grid_constant__ CUtensorMap map_k16, const __grid_constant__ CUtensorMap map_v16,
                  const __grid_constant__ PagedAttnArgs a) {
  using C = Cfg<DH, CACHE, X, MT>;
  constexpr int kUnit = C::kUnit;
  constexpr int KK = DH / 16, KT = C::kTiles, TQ = C::kQTerms, TP = C::kPTerms, PT = C::kPT;
  constexpr bool F16 = C::kF16;
  extern __shared__ unsigned char s_dyn[];
  __shared__ __align__(8) uint64_t s_full[kMaxStages], s_empty[kMaxStages], s_sums_full[kItems], s_sums_free[kItems], s_own[C::kWarps],
      s_joined[C::kWarps + C::kEpilogue];
  __shared__ StageInfo s_info[kMaxStages];
  __shared__ float s_m[C::kWarps + C::kEpilogue][C::kHeads], s_l[C::kWarps + C::kEpilogue][C::kHeads];
  __shared__ ItemInfo s_item[kItems];
  __shared__ long long s_sum[32];
  __shared__ int s_abort, s_start_row;   // (start: the first row's, where all threads look for it)
  __shared__ long long s_start_before;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int HG = a.hkv * a.tiles_per_head;
  const int CL = a.cluster, rank = CL ? (int)blockIdx.x % CL : 0;   // CTAs of a cluster (0: none), which share an item
  const int NW = CL ? C::kClusterWarps : C::kWarps;   // consumers: a cluster's CTA has one item, and no epilogue beside it
  const int S = a.n_stages;
  const uint32_t ring = (smem_u32(s_dyn) + 1023u) & ~1023u;
  unsigned char *ring_p = s_dyn + (ring - smem_u32(s_dyn));
  unsigned char *q_slots = ring_p + (size_t)S * C::kStageBytes;
  float *s_o = reinterpret_cast<float *>(q_slots + (size_t)S * C::kQBytes);   // [warp][head][kHeadFloats]
  float *s_j = s_o + (size_t)NW * a.heads_per_tile * C::kHeadFloats;   // cluster: [CTA][head][kHeadFloats], (m, l) behind the sums

  if (warp == 0) {
    // Drills (d3_paged_stall_next) are in the barriers alone: they expect one arrival more than there will be, so none of them
    // ends a phase.  (As tests in the loops of producers and consumers drills cost 64 rows x 16384 2.5 %.)
    const int drill = blockIdx.x == (CL ? 1u : 0u) ? a.stall : 0, extra = drill == D3_STALL_SUMS ? 1 : 0;
    if (lane < S) {
      mb_init(smem_u32(&s_full[lane]), drill == D3_STALL_COPIES ? 2 : 1);
      mb_init(smem_u32(&s_empty[lane]), NW + extra);
    }
    if (lane < C::kWarps + C::kEpilogue && CL) mb_init(smem_u32(&s_joined[lane]), CL - 1);
    if (lane < C::kWarps && !CL) mb_init(smem_u32(&s_own[lane]), C::kEpilogue);
    if (lane >= 32 - kItems) {
      mb_init(smem_u32(&s_sums_full[lane & (kItems - 1)]), NW + extra);
      mb_init(smem_u32(&s_sums_free[lane & (kItems - 1)]), C::kEpilogue);
    }
    if (lane == 31) {
      s_abort = 0;
      s_start_row = a.n_rows;
      s_start_before = 0;
    }
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == C::kWarps + C::kEpilogue && lane < 4) {
    const CUtensorMap *m = lane == 0 ? &map_k : lane == 1 ? &map_v : lane == 2 ? &map_k16 : &map_v16;
    asm volatile("prefetch.tensormap [%0];" ::"l"(reinterpret_cast<uint64_t>(m)) : "memory");
  }

  // ---- the rows' unit counts, summed over all rows by every CTA: up to 128 rows by each producer warp for itself, more of
  // them by all threads
  auto as_row = [&](int r, bool &bad) -> int {   // table row, -1 = padding
    if (r >= 0 && r < a.table_rows) return r;
    if (r != -1) bad = true;
    return -1;
  };
  auto as_length = [&](int c, bool &bad) -> int {
    if (c < 0 || c > ((long long)a.table_width << a.page_shift)) { bad = true; return 0; }
    return c;
  };
  auto row_of = [&](int b, bool &bad) -> int { return a.rows ? as_row(a.rows[b], bad) : b; };
  auto length_of = [&](int b, bool &bad) -> int { return as_length(a.context[b], bad); };
  auto units_of = [&](int len) -> int { return len > 0 ? (len + kUnit - 1) / kUnit : 1; };   // a row without context still gets its zeros
  const bool few = a.few;
  long long units = 0;   // of all rows, for one tile of heads
  int live_rows = 0;
  bool whole = a.whole;   // no item is cut between CTAs
  auto cost_of = [&](long long n) -> Cost {
    if (whole) return (long long)live_rows * HG <= gridDim.x ? Cost{0, 1, 0, 0} : Cost{kUnitCost, kItemCost, 0, 0};
    return n * HG >= 4ll * gridDim.x ? Cost{kUnitCost, kItemCost, kItemCost, kUnitCost} : Cost{1, 0, 0, 1};
  };
  if (!few && !CL) {
    pdl_wait();
    pdl_trigger();
    const int per = (a.n_rows + C::kThreads - 1) / C::kThreads;
    long long mine = 0;
    bool bad = false;
    int mine_rows = 0;
    for (int i = 0; i < per; ++i) {
      const int b = tid * per + i;
      if (b < a.n_rows) {
        bool strange = false, unused = false;
        if (row_of(b, strange) >= 0) { mine += units_of(length_of(b, strange)); ++mine_rows; }
        else length_of(b, unused);   // (padding may hold anything)
        bad = bad || strange;
      }
    }
    if (bad && blockIdx.x == 0 && a.status) *a.status = D3_EINVAL;
    // units in the upper, rows in the lower bits of one sum
    long long inc = (mine << 17) | mine_rows;
    const long long own_sum = inc;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
      const long long u = __shfl_up_sync(0xffffffffu, inc, d);
      if (lane >= d) inc += u;
    }
    if (lane == 31) s_sum[warp] = inc;
    __syncthreads();
    long long before = inc - own_sum, all = 0;
    for (int w = 0; w < C::kThreads / 32; ++w) {
      const long long v = s_sum[w];
      if (w < warp) before += v;
      all += v;
    }
    units = all >> 17;
    live_rows = (int)(all & 0x1ffff);
    const Cost cost = cost_of(units);
    const int n_cta = (int)min((whole ? live_rows : units) * HG, (long long)gridDim.x);
    if ((int)blockIdx.x < n_cta) {
      const Shares sh((units * cost.unit + (long long)live_rows * cost.item) * HG, n_cta);
      const long long x0 = sh.start(blockIdx.x);
      long long p = ((before >> 17) * cost.unit + (before & 0x1ffff) * cost.item) * HG;
      if (x0 >= p && x0 < p + (mine * cost.unit + (long long)mine_rows * cost.item) * HG) {
        for (int i = 0; i < per; ++i) {   // the first row is the one whose range of the costs holds x0
          const int b = tid * per + i;
          bool dummy = false;
          if (b < a.n_rows && row_of(b, dummy) >= 0) {
            const long long n = cost.of(units_of(length_of(b, dummy))) * HG;
            if (x0 < p + n) { s_start_row = b; s_start_before = p; break; }
            p += n;
          }
        }
      }
    }
  }
  __syncthreads();   // the barriers, and the first row where it was looked for
  if (CL) cluster_arrive();

  auto produce = [&]() {
    // ------------------------------------------------------------ producers
    const int me = warp - C::kWarps - C::kEpilogue;
    bool dummy = false;
    int row, trow, len;
    // few rows: their table rows and lengths stay in registers, row lane * per + i in entry i
    constexpr int kPer = kFewRows / 32;
    const int per = (a.n_rows + 31) / 32;
    int r_[kPer], c_[kPer], at_lane = 0, at_entry = 0;
    auto kept = [&](const int (&v)[kPer]) -> int {
      int x = v[0];
#pragma unroll
      for (int i = 1; i < kPer; ++i) x = at_entry == i ? v[i] : x;
      return __shfl_sync(0xffffffffu, x, at_lane);
    };
    int few_units = 0, few_rows = 0, few_longest = 0;   // of this lane
    if (CL) {
      pdl_wait();
      pdl_trigger();
    } else if (few) {
      pdl_wait();
      pdl_trigger();
      bool bad = false;
#pragma unroll
      for (int i = 0; i < kPer; ++i) {   // (all loads before the first use)
        const int b = lane * per + i;
        const bool there = i < per && b < a.n_rows;
        c_[i] = there ? a.context[b] : 0;
        r_[i] = !there ? -1 : a.rows ? a.rows[b] : b;
      }
#pragma unroll
      for (int i = 0; i < kPer; ++i) {
        if (i < per && lane * per + i < a.n_rows) {
          bool strange = false;
          c_[i] = as_length(c_[i], strange);
          r_[i] = as_row(r_[i], bad);
          if (r_[i] >= 0) { few_units += units_of(c_[i]); few_longest = max(few_longest, units_of(c_[i])); ++few_rows; bad = bad || strange; }
        }
      }
      if (bad && blockIdx.x == 0 && a.status) *a.status = D3_EINVAL;
      units = __reduce_add_sync(0xffffffffu, few_units);
      live_rows = __reduce_add_sync(0xffffffffu, few_rows);
      // Items stay whole where that makes the busiest CTA at most 8 units longer than an even share: a unit takes 0.5 us, the
      // sums of a cut item and their join about 4 (4 rows of 2048 positions, 32 heads: 25.4 us whole, 30.0 cut).
      const long long items = (long long)live_rows * HG, even = units * HG;
      const int longest = __reduce_max_sync(0xffffffffu, few_longest);
      whole = whole || (items <= gridDim.x ? longest * (long long)gridDim.x <= even + 8ll * gridDim.x : longest <= 8);
    }
    const int n_cta = (int)min((whole ? live_rows : units) * HG, (long long)gridDim.x);   // every one of them has work
    auto idle = [&]() {   // a stage that sends the other warps home
      if (me == 0 && lane == 0) {
        if (!a.whole && !CL) a.join[blockIdx.x] = make_int4(0, 0, 0, 0);
        s_info[0] = StageInfo{0, 0u, (uint32_t)((STAGE_LAST | STAGE_FINAL) << 9 | OUT_NONE << 12), 0u};
        mb_arrive(smem_u32(&s_full[0]));
      }
    };
    if (!CL && (int)blockIdx.x >= n_cta) { idle(); return; }
    const Cost cost = CL ? Cost{1, 0, 0, 1} : cost_of(units);
    Shares sh;
    long long x0, x1, item;   // this CTA's costs; where its first item starts
    int nu, tile, unit, lies_in = 1;
    const int32_t *pages = a.table;
    auto fetch = [&](int base) -> int { return base + lane < a.table_width ? __ldg(pages + base + lane) : -1; };
    // page ids of the row, one per lane: 32 aligned pages in `win`, the next 32 in `win_next`.  A unit is at most 16
    // aligned pages and never straddles a window.
    int win0 = -1, win = 0, win_next = 0;
    if (CL) {   // a cluster per item, its CTAs take equal runs of the units
      const int index = (int)blockIdx.x / CL;
      bool bad = false;
      row = index / HG;
      tile = index - row * HG;
      // the length and the first page ids are asked for together
      const int c = a.context[row];
      trow = row_of(row, bad);
      pages = a.table + (long long)max(trow, 0) * a.table_stride;
      win = fetch(0);
      win_next = fetch(32);
      len = trow >= 0 ? as_length(c, bad) : 0;
      if (bad && rank == 0 && tile == 0 && a.status) *a.status = D3_EINVAL;
      nu = units_of(len);
      lies_in = min(nu, CL);
      const int each = nu / CL, more = nu - each * CL;
      x0 = each * rank + min(rank, more);
      x1 = x0 + each + (rank < more ? 1 : 0);
      if (trow < 0 || x0 == x1) { idle(); return; }
      item = 0;
      unit = (int)x0;
      if ((unit * kUnit) >> a.page_shift < 32) win0 = 0;
    } else if (few) {   // all of it in 32 bits
      const int total = ((int)units * cost.unit + live_rows * cost.item) * HG, each = (int)((unsigned)total / (unsigned)n_cta);
      sh.each = each; sh.more = total - each * n_cta;
      const int x = each * (int)blockIdx.x + min((int)blockIdx.x, sh.more);
      x0 = x;
      x1 = x + each + ((int)blockIdx.x < sh.more ? 1 : 0);
      const int mine = (few_units * cost.unit + few_rows * cost.item) * HG;
      int inc = mine;
#pragma unroll
      for (int d = 1; d < 32; d <<= 1) {
        const int u = __shfl_up_sync(0xffffffffu, inc, d);
        if (lane >= d) inc += u;
      }
      int p = inc - mine, entry = 0;
      at_lane = __ffs(__ballot_sync(0xffffffffu, x >= p && x < inc)) - 1;
#pragma unroll
      for (int i = 0; i + 1 < kPer; ++i) {
        const int n = r_[i] >= 0 ? (cost.unit * units_of(c_[i]) + cost.item) * HG : 0;
        if (entry == i && x >= p + n) { p += n; entry = i + 1; }
      }
      at_entry = __shfl_sync(0xffffffffu, entry, at_lane);
      const int start_before = __shfl_sync(0xffffffffu, p, at_lane);
      row = at_lane * per + at_entry;
      trow = kept(r_);
      len = kept(c_);
      nu = units_of(len);
      const int one = cost.unit * nu + cost.item, at = x - start_before;
      tile = (int)((unsigned)at / (unsigned)one);
      item = start_before + tile * one;
      unit = (int)cost.first_unit(at - tile * one - cost.lead);
    } else {
      sh = Shares((units * cost.unit + (long long)live_rows * cost.item) * HG, n_cta);
      x0 = sh.start(blockIdx.x);
      x1 = sh.start(blockIdx.x + 1);
      row = min(s_start_row, a.n_rows - 1);   // (these bounds matter when somebody else changes the lengths during the call)
      trow = max(row_of(row, dummy), 0);
      len = length_of(row, dummy);
      nu = units_of(len);
      const long long at = x0 - s_start_before, one = cost.of(nu);   // s_start_before: cost of the rows before
      tile = (int)min(max(one < (1ll << 31) ? divide(at, (int)one) : at / one, 0ll), (long long)HG - 1);
      item = s_start_before + tile * one;
      unit = (int)min(cost.first_unit(x0 - item - cost.lead), 0x7fffffffll);
    }
    const bool behind = unit >= nu;   // no unit of that item is this CTA's: begin with the next one
    int kvh = tile, sub = 0;
    if (a.tiles_per_head > 1) { kvh = tile / a.tiles_per_head; sub = tile % a.tiles_per_head; }
    if (!CL) pages = a.table + (long long)trow * a.table_stride;
    const int box_rows = min(1 << a.page_shift, kUnit), page_mask = (1 << a.page_shift) - 1;
    const int full_boxes = kUnit / box_rows, full_shift = 31 - __clz(full_boxes);
    int s = 0, issued = 0;
    uint32_t parity = 1;
    bool first = true, ok = true;
    auto next_item = [&]() {   // next tile of the row, or next row
      unit = 0;
      item += cost.of(nu);
      if (win0 > 0) win0 = -1;   // (a row's first window serves its next tile too)
      ++tile;
      if (++sub == a.tiles_per_head) { sub = 0; ++kvh; }
      if (tile == HG) {
        tile = kvh = 0;
        win0 = -1;
        do {
          ++row;
          if (++at_entry == per) { at_entry = 0; ++at_lane; }
          trow = row >= a.n_rows ? 0 : few ? kept(r_) : row_of(row, dummy);
        } while (trow < 0);
        len = row >= a.n_rows ? 0 : few ? kept(c_) : length_of(row, dummy);
        row = min(row, a.n_rows - 1);   // (behind the last row only when somebody else changes the lengths during the call)
        nu = units_of(len);
        pages = a.table + (long long)trow * a.table_stride;
      }
    };
    if (behind) next_item();
    long long at = item + cost.lead + (long long)cost.step * unit;   // of the unit
    if (at >= x1) { idle(); return; }   // whole items: none starts in this CTA's share
    int cut_row = -1, cut_head = 0, cut_kvh = 0, cut_nh = 0;         // the item that goes on in the next CTA, if it starts here
    long long cut_last = 0;
    for (int k = 0; at < x1; ++k) {
      const bool ends = unit + 1 == nu;
      const long long next = ends ? item + cost.of(nu) + cost.lead : at + cost.step;
      const bool last = ends || next >= x1, final = next >= x1;
      const int nh = min(a.heads_per_tile, a.group - sub * a.heads_per_tile), head = kvh * a.group + sub * a.heads_per_tile;
      const bool whole_start = item + cost.lead >= x0;      // its unit 0 is this CTA's
      if (last && !ends && whole_start) {
        cut_row = row; cut_head = head; cut_kvh = kvh; cut_nh = nh;
        cut_last = item + cost.lead + (long long)cost.step * (nu - 1);
      }
      if ((k & (kProducers - 1)) == me) {
        const int p0 = unit * kUnit, n = max(0, min(kUnit, len - p0));   // n = 0 only for a row without context
        const int pg0 = p0 >> a.page_shift;
        if (n > 0) {
          if (win0 < 0) { win0 = pg0 & ~31; win = fetch(win0); win_next = fetch(win0 + 32); }
          else if (pg0 >= win0 + 32) {
            // (a unit is 16 pages at most, and the other producer takes every second one: never past the next window)
            win0 += 32; win = win_next; win_next = fetch(win0 + 32);
          }
        }
        // which tiles are there: lane p looks at tile p
        const int id_p = __shfl_sync(0xffffffffu, win, ((p0 + lane * kTile) >> a.page_shift) & 31);
        const bool inside = lane * kTile < n, good = id_p >= 0 && id_p < a.n_pages;
        const unsigned tiles = __ballot_sync(0xffffffffu, inside && good);
        if (inside && !good && a.status) *a.status = D3_EINVAL;
        // this lane's copy: box of positions, K or V, 128-byte column.  Whole units go in boxes of up to a page, the
        // last unit of a row in boxes of 16 positions (nothing is fetched behind the tile the row ends in).
        const bool whole = n == kUnit;
        const int bs = whole ? full_shift : (kUnit == 64 ? 2 : kUnit == 128 ? 3 : 4);
        const int box = lane & ((1 << bs) - 1), is_v = (lane >> bs) & 1, col = lane >> (bs + 1);
        const int off = box * (kUnit >> bs), pos = p0 + off;
        const int id = __shfl_sync(0xffffffffu, win, (pos >> a.page_shift) & 31);
        const bool want = col < C::kBoxes && off < n && id >= 0 && id < a.n_pages;
        if (!mb_wait(smem_u32(&s_empty[s]), parity, &s_abort, a.wait_ns)) ok = false;
        ok = __all_sync(0xffffffffu, ok);
        if (!ok) break;
        const uint32_t full = smem_u32(&s_full[s]);
        if (lane == 0) {
          const int kind = !last || (ends && whole_start) ? OUT_WHOLE : !ends && whole_start ? OUT_TAIL : OUT_HEAD;
          const int flags = (first ? STAGE_FIRST : 0) | (last ? STAGE_LAST : 0) | (final ? STAGE_FINAL : 0);
          s_info[s] = StageInfo{row, (uint32_t)head | (uint32_t)kvh << 16,
                                (uint32_t)n | (uint32_t)flags << 9 | (uint32_t)kind << 12 | (uint32_t)nh << 14 | (uint32_t)lies_in << 19, tiles};
          mb_arrive_tx(full, (uint32_t)__popc(tiles) * 2u * kTile * C::kRow + (first ? (uint32_t)(nh * DH * QBytes<X>::v) : 0u));
        }
        __syncwarp();
        if (want) {
          const uint32_t dst = ring + s * C::kStageBytes + is_v * C::kHalfBytes + col * (kUnit * C::kBox) + off * C::kBox;
          const CUtensorMap *map = whole ? (is_v ? &map_v : &map_k) : (is_v ? &map_v16 : &map_k16);
          tma_box(dst, map, col * (C::kBox / C::kEs), pos & page_mask, kvh, id, full);
        }
        if (first && lane < nh) {
          bulk_copy(smem_u32(q_slots) + s * C::kQBytes + lane * C::kQRow,
                    static_cast<const char *>(a.q) + (row * a.q_row_stride + (head + lane) * a.q_head_stride) * QBytes<X>::v,
                    DH * QBytes<X>::v, full);
        }
      }
      issued = k + 1;
      first = last;
      if (++s == S) { s = 0; parity ^= 1u; }
      ++unit;
      if (ends && !final) next_item();
      at = next;
    }
    if (me == 0 && lane == 0) {
      // an item that starts here and goes on: what the joining kernel adds up
      int4 join = make_int4(0, 0, 0, 0);
      if (ok && cut_row >= 0 && !CL) join = make_int4(min(sh.holder(cut_last), n_cta - 1) - (int)blockIdx.x + 1, cut_row, cut_head, cut_kvh | cut_nh << 16);
      if (!a.whole && !CL) a.join[blockIdx.x] = join;
    }
    // Copies in flight end by themselves: wait for them before the shared memory goes, also where the consumers are already gone
    // (a wait ran out; or somebody else changed the lengths during the call and the two producers saw different ones).
    const unsigned long long drain = a.wait_ns > kDrainFloorNs ? a.wait_ns : kDrainFloorNs;
    for (int k = max(0, issued - S); k < issued; ++k)
      if ((k & (kProducers - 1)) == me && !mb_wait(smem_u32(&s_full[k % S]), (uint32_t)((k / S) & 1), &s_abort, drain, false)) ok = false;
    if (!ok && lane == 0 && a.status) *a.status = D3_ETIMEOUT;
  };

  bool met = false;   // this thread has seen the whole cluster started
  auto epilogue = [&](int i0) {
    // ------------------------------------------------------------ epilogue: a head per warp, DH / 32 dims per lane.  The
    // consumers have nothing left to do at a CTA's last item and help there (4 rows x 545, 8 heads a tile: 9.7 us without, 8.6 with).
    constexpr int V = DH / 32;
    constexpr int kMany = C::kEpilogue == 4 ? 2 : 4;   // heads of a warp at a time
    const bool helps = CL || warp < NW;
    auto gave_up = [&]() { if (lane == 0 && a.status) *a.status = D3_ETIMEOUT; };
    for (int it = i0;; ++it) {
      const int at = it & (kItems - 1), me = CL ? warp : helps ? warp + C::kEpilogue : (warp - C::kWarps + it) & (C::kEpilogue - 1);   // (single heads in turn)
      if (!__all_sync(0xffffffffu, mb_wait(smem_u32(&s_sums_full[at]), (uint32_t)(it / kItems) & 1u, &s_abort, a.wait_ns))) { gave_up(); break; }
      const ItemInfo item = s_item[at];
      const int kind = item.bits & 3, nh = (item.bits >> 3) & 31, first_warp = (item.bits >> 8) & 255, warps = (item.bits >> 16) & 255;
      const int workers = item.bits & 4 ? C::kWarps + C::kEpilogue : C::kEpilogue;
      if (CL && kind != OUT_WHOLE && rank > 0) { cluster_wait(); met = true; }   // the first CTA's barriers are there
      if (kind == OUT_NONE) {
        if (CL && rank > 0 && lane == 0) arrive_there(in_cta(smem_u32(&s_joined[me]), 0));
        break;
      }
      int from = first_warp + min(lane, warps - 1);   // lane k: the k-th warp that had a piece of the item
      if (from >= NW) from -= NW;
      const float vs = a.v_scale ? __ldg(a.v_scale + (item.heads >> 16)) : 1.f;
      auto finish = [&](int h, const float (&o)[V], float m, float l) {
        const float f = l == 0.f ? 0.f : vs / l;
        write_out<X, V>(a, item.row * a.out_row_stride + (long long)((item.heads & 0xffffu) + h) * a.out_head_stride + lane * V, o, f);
        if (lane == 0 && a.lse)
          a.lse[(long long)item.row * a.hq + (item.heads & 0xffffu) + h] = l == 0.f ? -INFINITY : (m + (log2f(l) - (F16 ? 15.f : 0.f))) * kLn2;
      };
      // HB heads at a time, in independent chains: this is all latency
      auto heads = [&](auto hb, int h0) {
        constexpr int HB = decltype(hb)::value;
        float M[HB], L[HB], c[HB], o[HB][V];
#pragma unroll
        for (int i = 0; i < HB; ++i) {
          const int h = min(h0 + i * workers, nh - 1);
          L[i] = lane < warps ? s_l[from][h] : 0.f;
          c[i] = lane < warps ? s_m[from][h] : -INFINITY;
          M[i] = c[i];
        }
#pragma unroll
        for (int d = 8; d; d >>= 1)
#pragma unroll
          for (int i = 0; i < HB; ++i) M[i] = fmaxf(M[i], __shfl_xor_sync(0xffffffffu, M[i], d));
#pragma unroll
        for (int i = 0; i < HB; ++i) {
          c[i] = exp2_fast(c[i] - (M[i] == -INFINITY ? 0.f : M[i]));   // 0 beyond the warps that had pieces
          L[i] *= c[i];
#pragma unroll
          for (int e = 0; e < V; ++e) o[i][e] = 0.f;
        }
#pragma unroll
        for (int d = 8; d; d >>= 1)
#pragma unroll
          for (int i = 0; i < HB; ++i) L[i] += __shfl_xor_sync(0xffffffffu, L[i], d);
        // groups of the warps; what is past the last one counts as that one with factor 0
        constexpr int GR = HB == 1 ? 4 : 2;
        for (int k = 0; k < warps; k += GR) {
#pragma unroll
          for (int j = 0; j < GR; ++j) {
            const int w = __shfl_sync(0xffffffffu, from, k + j);
#pragma unroll
            for (int i = 0; i < HB; ++i) {
              const int h = min(h0 + i * workers, nh - 1);
              const float cw = __shfl_sync(0xffffffffu, c[i], k + j);
              const float *src = s_o + (w * a.heads_per_tile + h) * C::kHeadFloats + lane * V;
              float x[V];
              if constexpr (V == 4) { const float4 v = *reinterpret_cast<const float4 *>(src); x[0] = v.x; x[1] = v.y; x[2] = v.z; x[3] = v.w; }
              else if constexpr (V == 2) { const float2 v = *reinterpret_cast<const float2 *>(src); x[0] = v.x; x[1] = v.y; }
              else x[0] = *src;
#pragma unroll
              for (int e = 0; e < V; ++e) o[i][e] += cw * x[e];
            }
          }
        }
#pragma unroll
        for (int i = 0; i < HB; ++i) {
          const int h = h0 + i * workers;
          if (h >= nh) break;
          const float l = __shfl_sync(0xffffffffu, L[i], 0), m = __shfl_sync(0xffffffffu, M[i], 0);
          if (kind == OUT_WHOLE) {
            finish(h, o[i], m, l);
          } else if (CL) {   // to the cluster's first CTA
            float *dst = s_j + ((size_t)rank * a.heads_per_tile + h) * C::kHeadFloats;
            const uint32_t there = in_cta(smem_u32(dst), 0);
            store_there<V>(there + 4 * lane * V, o[i]);
            if (lane == 0) {
              const float ml[2] = {m, l};
              store_there<2>(there + 4 * DH, ml);
            }
          } else {
            const size_t part = (size_t)(2 * blockIdx.x + (kind == OUT_TAIL ? 1 : 0)) * 16 + h;
#pragma unroll
            for (int e = 0; e < V; ++e) a.part_o[part * DH + lane * V + e] = o[i][e];
            if (lane == 0) { a.part_ml[2 * part] = m; a.part_ml[2 * part + 1] = l; }
          }
        }
      };
      if (nh <= workers) { if (me < nh) heads(std::integral_constant<int, 1>(), me); }
      else for (int h0 = me; h0 < nh; h0 += kMany * workers) heads(std::integral_constant<int, kMany>(), h0);
      __syncwarp();
      if (!helps) {
        if (lane == 0) mb_arrive(smem_u32(&s_sums_free[at]));
        if (lane < warps) mb_arrive(smem_u32(&s_own[from]));
      }
      if (CL && kind != OUT_WHOLE) {
        if (rank > 0) {
          if (lane == 0) arrive_there(in_cta(smem_u32(&s_joined[me]), 0));
        } else {
          // ---- the item's first CTA: the pieces of all, in their order
          const int pieces = item.bits >> 24;
          if (!__all_sync(0xffffffffu, mb_wait<true>(smem_u32(&s_joined[me]), 0, &s_abort, a.wait_ns))) { gave_up(); break; }
          const int stride = a.heads_per_tile * C::kHeadFloats;
          auto join = [&](auto hb, int h0) {
            constexpr int HB = decltype(hb)::value;
            float M[HB], L[HB], c[HB], o[HB][V];
            const float *all[HB];
#pragma unroll
            for (int i = 0; i < HB; ++i) {
              all[i] = s_j + min(h0 + i * workers, nh - 1) * C::kHeadFloats;
              const float2 ml = *reinterpret_cast<const float2 *>(all[i] + min(lane, pieces - 1) * stride + DH);
              c[i] = M[i] = lane < pieces ? ml.x : -INFINITY;
              L[i] = ml.y;
#pragma unroll
              for (int e = 0; e < V; ++e) o[i][e] = 0.f;
            }
#pragma unroll
            for (int d = 8; d; d >>= 1)
#pragma unroll
              for (int i = 0; i < HB; ++i) M[i] = fmaxf(M[i], __shfl_xor_sync(0xffffffffu, M[i], d));
#pragma unroll
            for (int i = 0; i < HB; ++i) {
              c[i] = exp2_fast(c[i] - (M[i] == -INFINITY ? 0.f : M[i]));   // 0 beyond the pieces
              L[i] = lane < pieces ? L[i] * c[i] : 0.f;
            }
#pragma unroll
            for (int d = 8; d; d >>= 1)
#pragma unroll
              for (int i = 0; i < HB; ++i) L[i] += __shfl_xor_sync(0xffffffffu, L[i], d);
            for (int k = 0; k < pieces; k += 2) {
#pragma unroll
              for (int j = 0; j < 2; ++j)
#pragma unroll
                for (int i = 0; i < HB; ++i) {
                  const float ck = __shfl_sync(0xffffffffu, c[i], k + j);
                  const float *src = all[i] + min(k + j, pieces - 1) * stride + lane * V;
                  float x[V];
                  if constexpr (V == 4) { const float4 v = *reinterpret_cast<const float4 *>(src); x[0] = v.x; x[1] = v.y; x[2] = v.z; x[3] = v.w; }
                  else if constexpr (V == 2) { const float2 v = *reinterpret_cast<const float2 *>(src); x[0] = v.x; x[1] = v.y; }
                  else x[0] = *src;
#pragma unroll
                  for (int e = 0; e < V; ++e) o[i][e] += ck * x[e];
                }
            }
#pragma unroll
            for (int i = 0; i < HB; ++i)
              if (h0 + i * workers < nh)
                finish(h0 + i * workers, o[i], __shfl_sync(0xffffffffu, M[i], 0), __shfl_sync(0xffffffffu, L[i], 0));
          };
          if (nh <= workers) { if (me < nh) join(std::integral_constant<int, 1>(), me); }
          else for (int h0 = me; h0 < nh; h0 += kMany * workers) join(std::integral_constant<int, kMany>(), h0);
        }
      }
      if (item.bits & 4) break;
    }
  };

  // -------------------------------------------------------------- consumers
  auto consume = [&]() -> int {   // how many items ended here; 0 when a wait ran out
  // Fragments (g = lane / 4, t = lane % 4).  Scores: A = K (rows = positions), B = Q^T (column g = head), result: positions
  // g, g + 8 of heads 2t, 2t + 1.  Sums: A = V^T (rows = dims), B = P^T, result: dims g, g + 8 of heads 2t, 2t + 1.
  const int g = lane >> 2, t = lane & 3, mat = lane >> 3;
  // 16-bit cache: row and 16-byte chunk of this lane's ldmatrix row; 8-bit: the same for two chunks of 16 dims
  constexpr int kPerRow = C::kBox / 16;
  const int k_row = (lane & 7) + 8 * (mat & 1), k_chunk = mat >> 1;                      // K: (0-7), (8-15), then the next chunk
  const int v_row = CACHE == D3_E4M3 ? k_row : (lane & 7) + 8 * (mat >> 1);              // V: 16-bit: dims first, then positions
  const int v_chunk = CACHE == D3_E4M3 ? k_chunk : mat & 1;
  auto lane_part = [](int r, int c) -> uint32_t {   // of an address; the swizzle XORs the chunk with the row's 128-byte line
    return (uint32_t)(r * C::kBox + ((c ^ (((r * C::kBox) >> 7) & (kPerRow - 1))) << 4));
  };
  const uint32_t k_lane = lane_part(k_row, k_chunk), v_lane = lane_part(v_row, v_chunk);
  uint32_t qb[KT][TQ][KK][2];
  float o[KT][KK][4], mx[KT][2], sum[KT][2], mul[KT][2];
#pragma unroll
  for (int i = 0; i < KT; ++i) {
#pragma unroll
    for (int e = 0; e < 2; ++e) { mx[i][e] = -INFINITY; sum[i][e] = 0.f; mul[i][e] = 0.f; }
#pragma unroll
    for (int n = 0; n < KK; ++n) o[i][n][0] = o[i][n][1] = o[i][n][2] = o[i][n][3] = 0.f;
  }
  int piece_turn = 0;       // pieces of the CTA so far, mod NW: whose turn it is
  int items = 0, uses = 0;   // that ended; that this warp had a part of
  bool ok = true;
  int first_warp = 0, item_pieces = 0;   // of the running item: whose its first piece was, and how many there were
  int s = 0;
  uint32_t parity = 0;
  for (bool more = true; more;) {
    if (!mb_wait(smem_u32(&s_full[s]), parity, &s_abort, a.wait_ns)) ok = false;
    ok = __all_sync(0xffffffffu, ok);
    if (!ok) break;
    const StageInfo info = s_info[s];
    const uint32_t flags = info.bits >> 9;
    const int n = info.bits & 511;
    more = !(flags & STAGE_FINAL);
    if (flags & STAGE_FIRST) {
      // ---- this thread's fragments of Q, and what a raw score is multiplied by
      const int nh = (info.bits >> 14) & 31;
      first_warp = piece_turn; item_pieces = 0;
      const float ks = a.k_scale ? __ldg(a.k_scale + (info.heads >> 16)) : 1.f;
#pragma unroll
      for (int i = 0; i < KT; ++i) {
        const int h = g + 8 * i;
        const bool live = h < nh;
        const unsigned char *qp = q_slots + s * C::kQBytes + (live ? h : 0) * C::kQRow;
        float factor = a.scale * kLog2e * ks;
        if constexpr (X == D3_FP32) {
#pragma unroll
          for (int kk = 0; kk < KK; ++kk)
#pragma unroll
            for (int j = 0; j < 2; ++j) {
              const float2 v = *reinterpret_cast<const float2 *>(qp + (16 * kk + 8 * j + 2 * t) * 4);
              float x = live ? v.x : 0.f, y = live ? v.y : 0.f;
#pragma unroll
              for (int q = 0; q < TQ; ++q) qb[i][q][kk][j] = cut(x, y);
            }
        } else {
          // the pairs: dims 16kk + 2t, +8 (16-bit cache); 16kk + 4t, +2 (8-bit cache, whose four bytes of a
          // fragment register are four neighbouring dims)
          constexpr int kA = CACHE == D3_E4M3 ? 4 : 2, kB = CACHE == D3_E4M3 ? 2 : 8;
#pragma unroll
          for (int kk = 0; kk < KK; ++kk)
#pragma unroll
            for (int j = 0; j < 2; ++j) {
              const uint32_t v = *reinterpret_cast<const uint32_t *>(qp + (16 * kk + kB * j + kA * t) * 2);
              qb[i][0][kk][j] = live ? v : 0u;
            }
          if constexpr (CACHE == D3_E4M3 && X == D3_BF16) {
            // To fp16: the head's largest |q| is brought to [2^14, 2^15) by a power of two, so that the 8 bits of a number stay
            // whole down to 2^-31 of the largest (fp16's step below its normal numbers is 2^-24); a smaller one is off by 2^-39 of it
            // at most.  The products' sums stay below 128 * 448 * 2^15.
            float top = 0.f;
#pragma unroll
            for (int kk = 0; kk < KK; ++kk)
#pragma unroll
              for (int j = 0; j < 2; ++j) {
                float x, y;
                unpack<false>(qb[i][0][kk][j], x, y);
                top = fmaxf(top, fmaxf(fabsf(x), fabsf(y)));
              }
            top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 1));
            top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 2));
            // (both powers are normal numbers; a head of numbers below 2^-112, the subnormal ones among them, takes the largest)
            const int e = top < INFINITY ? min(14 - ((int)(__float_as_uint(top) >> 23) - 127), 126) : 0;
            const float down = __uint_as_float((uint32_t)(127 + e) << 23), up = __uint_as_float((uint32_t)(127 - e) << 23);
            factor *= up;
#pragma unroll
            for (int kk = 0; kk < KK; ++kk)
#pragma unroll
              for (int j = 0; j < 2; ++j) {
                float x, y;
                unpack<false>(qb[i][0][kk][j], x, y);
                qb[i][0][kk][j] = pack<true>(x * down, y * down);
              }
          }
        }
        mul[i][0] = __shfl_sync(0xffffffffu, factor, 8 * t);       // of heads 2t and 2t + 1
        mul[i][1] = __shfl_sync(0xffffffffu, factor, 8 * t + 4);
      }
    }
    const int n_pieces = (n + PT * kTile - 1) / (PT * kTile);
    item_pieces += n_pieces;
    // pieces go round the warps
    int p = warp - piece_turn;
    if (p < 0) p += NW;
    piece_turn += n_pieces;
    if (piece_turn >= NW) piece_turn -= NW;
    if (p < n_pieces) {   // (a stage has 4 pieces at most)
      // positions of each tile of the piece; none where its page id was out of range
      int valid[PT];
#pragma unroll
      for (int j = 0; j < PT; ++j)
        valid[j] = (info.tiles >> (p * PT + j)) & 1 ? min(kTile, n - (p * PT + j) * kTile) : 0;
      int there = 0;
#pragma unroll
      for (int j = 0; j < PT; ++j) there += valid[j];
      const bool partial = there < PT * kTile;
      const uint32_t kbase = ring + s * C::kStageBytes + p * (PT * kTile * C::kBox) + k_lane;
      const uint32_t vbase = ring + s * C::kStageBytes + C::kHalfBytes + p * (PT * kTile * C::kBox) + v_lane;
      // 16-byte chunk c (even) of tile j past the lane's own: an XOR inside the 128-byte line, the next column behind it
      auto chunk = [&](uint32_t base, int j, int c) -> uint32_t {
        return (base ^ ((c % kPerRow) << 4)) + (c / kPerRow) * (kUnit * C::kBox) + j * (kTile * C::kBox);
      };
      // all fragments of K are asked for before the first product, those of V before the softmax
      constexpr int NF = CACHE == D3_E4M3 ? KK / 2 : KK;   // ldmatrix per tile and operand
      uint32_t kf[PT][NF][4], vf[PT][NF][4];
#pragma unroll
      for (int j = 0; j < PT; ++j)
#pragma unroll
        for (int c = 0; c < NF; ++c) ldsm4(kf[j][c], chunk(kbase, j, 2 * c));
      // Chains of products that a score is summed in: two where a warp has only one at a time to work on; with three terms the
      // largest has two and the others have their own, because the tensor cores' sums lose a little with every product of
      // a chain (error of fp32 outputs against 64 bits at 5000 positions 1.2e-6 with one chain).
      constexpr int NC = TQ == 3 ? 3 : PT * KT == 1 ? 2 : 1;
      float sc[PT][KT][NC][4];
#pragma unroll
      for (int j = 0; j < PT; ++j)
#pragma unroll
        for (int i = 0; i < KT; ++i)
#pragma unroll
          for (int c = 0; c < NC; ++c) sc[j][i][c][0] = sc[j][i][c][1] = sc[j][i][c][2] = sc[j][i][c][3] = 0.f;
#pragma unroll
      for (int kk = 0; kk < KK; ++kk)
#pragma unroll
        for (int j = 0; j < PT; ++j) {
          uint32_t f[4];
          if constexpr (CACHE != D3_E4M3) {
            f[0] = kf[j][kk][0]; f[1] = kf[j][kk][1]; f[2] = kf[j][kk][2]; f[3] = kf[j][kk][3];
          } else {   // chunk kk of positions 0-7 and of 8-15: four dims 4t.. of position g
            const uint32_t x = kf[j][kk / 2][2 * (kk & 1)], y = kf[j][kk / 2][2 * (kk & 1) + 1];
            f[0] = widen(x); f[1] = widen(y); f[2] = widen(x >> 16); f[3] = widen(y >> 16);
          }
#pragma unroll
          for (int i = 0; i < KT; ++i)
#pragma unroll
            for (int q = TQ - 1; q >= 0; --q)
              mma<F16>(sc[j][i][NC == 3 ? (q == 0 ? kk & 1 : 2) : kk % NC], f, qb[i][q][kk][0], qb[i][q][kk][1]);
        }
#pragma unroll
      for (int j = 0; j < PT; ++j)
#pragma unroll
        for (int c = 0; c < NF; ++c) ldsm4t(vf[j][c], chunk(vbase, j, 2 * c));
      // ---- softmax of the piece: [0] head 2t, [1] head 2t + 1 of position g; [2], [3] of position g + 8 (of each tile)
      uint32_t pb[PT][KT][TP][2];
#pragma unroll
      for (int i = 0; i < KT; ++i) {
        float v[PT][4], cm[2] = {-INFINITY, -INFINITY};
#pragma unroll
        for (int j = 0; j < PT; ++j) {
#pragma unroll
          for (int e = 0; e < 4; ++e) v[j][e] = (NC == 3 ? sc[j][i][2 % NC][e] + (sc[j][i][0][e] + sc[j][i][1 % NC][e])
                                                               : NC == 2 ? sc[j][i][0][e] + sc[j][i][NC - 1][e] : sc[j][i][0][e]) * mul[i][e & 1];
          if (partial) {
            if (g >= valid[j]) v[j][0] = v[j][1] = -INFINITY;
            if (g + 8 >= valid[j]) v[j][2] = v[j][3] = -INFINITY;
          }
          cm[0] = fmaxf(cm[0], fmaxf(v[j][0], v[j][2]));
          cm[1] = fmaxf(cm[1], fmaxf(v[j][1], v[j][3]));
        }
#pragma unroll
        for (int d = 4; d < 32; d <<= 1) {
          cm[0] = fmaxf(cm[0], __shfl_xor_sync(0xffffffffu, cm[0], d));
          cm[1] = fmaxf(cm[1], __shfl_xor_sync(0xffffffffu, cm[1], d));
        }
        if (__any_sync(0xffffffffu, cm[0] > mx[i][0] || cm[1] > mx[i][1])) {   // a new maximum: rescale (by 0 at the first piece)
          const float m0 = fmaxf(mx[i][0], cm[0]), m1 = fmaxf(mx[i][1], cm[1]);
          const float c0 = m0 > mx[i][0] ? exp2_fast(mx[i][0] - m0) : 1.f, c1 = m1 > mx[i][1] ? exp2_fast(mx[i][1] - m1) : 1.f;
          mx[i][0] = m0; mx[i][1] = m1;
          sum[i][0] *= c0; sum[i][1] *= c1;
#pragma unroll
          for (int n = 0; n < KK; ++n) { o[i][n][0] *= c0; o[i][n][1] *= c1; o[i][n][2] *= c0; o[i][n][3] *= c1; }
        }
        float ref[2];
#pragma unroll
        for (int e = 0; e < 2; ++e) ref[e] = mx[i][e] == -INFINITY ? 0.f : (F16 ? mx[i][e] - 15.f : mx[i][e]);
#pragma unroll
        for (int j = 0; j < PT; ++j) {
          float pr[4];
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            pr[e] = exp2_fast(v[j][e] - ref[e & 1]);
            sum[i][e & 1] += pr[e];
          }
          // P^T fragments: positions 2t, 2t + 1 (+ 8) of head g, the transpose of what this thread holds
#pragma unroll
          for (int r = 0; r < 2; ++r) {
            float x = pr[2 * r], y = pr[2 * r + 1];
            if constexpr (TP == 3) {
#pragma unroll
              for (int q = 0; q < 3; ++q) pb[j][i][q][r] = transpose8(cut(x, y));
            } else {
              const uint32_t hi = pack<F16>(x, y);
              pb[j][i][0][r] = transpose8(hi);
              if constexpr (TP == 2) {
                float hx, hy;
                unpack<F16>(hi, hx, hy);
                pb[j][i][TP - 1][r] = transpose8(pack<F16>(x - hx, y - hy));
              }
            }
          }
        }
      }
      // ---- O^T += V^T P^T.  What the page holds behind the row's end must not reach a product (0 x NaN is NaN).
#pragma unroll
      for (int j = 0; j < PT; ++j) {
        uint32_t keep0 = 0xffffffffu, keep1 = 0xffffffffu;
        if (partial) {
          keep0 = (2 * t < valid[j] ? 0xffffu : 0u) | (2 * t + 1 < valid[j] ? 0xffff0000u : 0u);
          keep1 = (2 * t + 8 < valid[j] ? 0xffffu : 0u) | (2 * t + 9 < valid[j] ? 0xffff0000u : 0u);
        }
#pragma unroll
        for (int n = 0; n < KK; ++n) {
          uint32_t f[4];
          if constexpr (CACHE != D3_E4M3) {   // dims 16n.. / +8 of positions 0-7, then of 8-15
            f[0] = vf[j][n][0]; f[1] = vf[j][n][1]; f[2] = vf[j][n][2]; f[3] = vf[j][n][3];
          } else {
            // chunk n of positions 0-7 and of 8-15: positions 2t, 2t + 1 of dims 2g, 2g + 1.  Even dims make rows
            // 0-7 of the product, odd ones rows 8-15
            const uint32_t lo = __byte_perm(vf[j][n / 2][2 * (n & 1)], 0, 0x3120), hi = __byte_perm(vf[j][n / 2][2 * (n & 1) + 1], 0, 0x3120);
            f[0] = widen(lo); f[1] = widen(lo >> 16); f[2] = widen(hi); f[3] = widen(hi >> 16);
          }
          if (partial) { f[0] &= keep0; f[1] &= keep0; f[2] &= keep1; f[3] &= keep1; }
#pragma unroll
          for (int i = 0; i < KT; ++i) {
            if constexpr (TP == 3) {   // fp32 results: every piece's products in a chain of their own
              float d[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
              for (int q = TP - 1; q >= 0; --q) mma<F16>(d, f, pb[j][i][q][0], pb[j][i][q][1]);
#pragma unroll
              for (int e = 0; e < 4; ++e) o[i][n][e] += d[e];
            } else {
#pragma unroll
              for (int q = TP - 1; q >= 0; --q) mma<F16>(o[i][n], f, pb[j][i][q][0], pb[j][i][q][1]);
            }
          }
        }
      }
    }
    __syncwarp();
    if (lane == 0) mb_arrive(smem_u32(&s_empty[s]));
    if (++s == S) { s = 0; parity ^= 1u; }

    if (flags & STAGE_LAST) {
      // ---- the item's end in this CTA: this warp's sums to shared memory, for the epilogue warps to add up
      const int warps = min(item_pieces, NW), turn = warp - first_warp + (warp < first_warp ? NW : 0);
      // Room in the ring of items, and this warp's sums of the last item that it had a part of are taken: short items lie in
      // different warps, and none waits for the one before it (128 rows of 64 positions, 64 / 8 heads: 20.2 us with one set for
      // all, 18.3 so, 14.8 with four epilogue warps as well).
      const int slot = items & (kItems - 1);
      if (items >= kItems && !mb_wait(smem_u32(&s_sums_free[slot]), (uint32_t)(items / kItems - 1) & 1u, &s_abort, a.wait_ns)) ok = false;
      if (turn < warps && uses > 0 && !mb_wait(smem_u32(&s_own[warp]), (uint32_t)(uses - 1) & 1u, &s_abort, a.wait_ns)) ok = false;
      ok = __all_sync(0xffffffffu, ok);
      if (!ok) break;
      if (turn < warps) {
        ++uses;
#pragma unroll
        for (int i = 0; i < KT; ++i) {
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            const int h = 2 * t + e + 8 * i;
            float l = sum[i][e];
#pragma unroll
            for (int d = 4; d < 32; d <<= 1) l += __shfl_xor_sync(0xffffffffu, l, d);
            if (h < a.heads_per_tile) {
              float *dst = s_o + (warp * a.heads_per_tile + h) * C::kHeadFloats;
#pragma unroll
              for (int n = 0; n < KK; ++n) {
                if constexpr (CACHE == D3_E4M3) {
                  *reinterpret_cast<float2 *>(dst + 16 * n + 2 * g) = make_float2(o[i][n][e], o[i][n][2 + e]);
                } else {
                  dst[16 * n + g] = o[i][n][e];
                  dst[16 * n + 8 + g] = o[i][n][2 + e];
                }
              }
              if (g == 0) { s_m[warp][h] = mx[i][e]; s_l[warp][h] = l; }
            }
            mx[i][e] = -INFINITY; sum[i][e] = 0.f;
          }
#pragma unroll
          for (int n = 0; n < KK; ++n) o[i][n][0] = o[i][n][1] = o[i][n][2] = o[i][n][3] = 0.f;
        }
      }
      if (warp == 0 && lane == 0)
        s_item[slot] = ItemInfo{info.row, info.heads,
                          ((flags >> 3) & 3) | (more ? 0u : 4u) | ((info.bits >> 14) & 31) << 3 | (uint32_t)first_warp << 8 | (uint32_t)warps << 16 |
                              ((info.bits >> 19) & 31) << 24};
      __syncwarp();
      if (lane == 0) mb_arrive(smem_u32(&s_sums_full[slot]));
      ++items;
    }
  }
  if (!ok && lane == 0 && a.status) *a.status = D3_ETIMEOUT;
  return ok ? items : 0;
  };

  if (warp >= C::kWarps + C::kEpilogue) {
    produce();
  } else {
    pdl_wait();   // (before the first wait with a limit, which the kernel before this one must not use up)
    const int items = warp < NW ? consume() : 1;
    if (items > 0) epilogue(items - 1);
  }
  if (CL) {   // no CTA of the cluster leaves while another may still write to it (every wait before this one is bounded)
    if (!met) cluster_wait();
    cluster_arrive();
    cluster_wait();
  }
}

// Joins the pieces of the item that starts in CTA blockIdx.x and goes on behind it.  Parts: this CTA's second slot, then the
// first slots of the CTAs that follow, in that order.  16 warps: 16 / heads of them share a head's parts, a lane
// has DH / 32 neighbouring dims; the last sum runs over those warps in order.
constexpr int kJoinWarps = 16;
template <int DH, int X, bool F16>
__global__ void __launch_bounds__(32 * kJoinWarps) k_paged_join(const __grid_constant__ PagedAttnArgs a) {
  constexpr int V = DH / 32;
  __shared__ float s_o[kJoinWarps][DH], s_l[kJoinWarps], s_m[kJoinWarps];
  pdl_wait();
  pdl_trigger();
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int share_of = kJoinWarps / a.heads_per_tile, h = warp / share_of, first = warp % share_of;
  auto part = [&](int k) -> size_t { return (size_t)(k == 0 ? 2 * blockIdx.x + 1 : 2 * (blockIdx.x + k)) * 16 + h; };
  auto sums_of = [&](int k, float (&x)[V]) {
    const float *src = a.part_o + part(k) * DH + lane * V;
    if constexpr (V == 4) { const float4 v = *reinterpret_cast<const float4 *>(src); x[0] = v.x; x[1] = v.y; x[2] = v.z; x[3] = v.w; }
    else if constexpr (V == 2) { const float2 v = *reinterpret_cast<const float2 *>(src); x[0] = v.x; x[1] = v.y; }
    else x[0] = *src;
  };
  // one round trip: the first 32 (m, l) and the sums of the first two parts are asked for together with the job; what
  // of them is not a part of it is not used
  float2 next_ml = make_float2(-INFINITY, 0.f);
  float early[2][V];
  if (h < a.heads_per_tile) {
    const int mine0 = first + lane * share_of;
    if (blockIdx.x + mine0 < gridDim.x) next_ml = *reinterpret_cast<const float2 *>(a.part_ml + 2 * part(mine0));
#pragma unroll
    for (int i = 0; i < 2; ++i)
      if (blockIdx.x + first + i * share_of < gridDim.x) sums_of(first + i * share_of, early[i]);
  }
  const int4 job = a.join[blockIdx.x];
  if (job.x == 0) return;
  const int parts = job.x, row = job.y, kvh = job.w & 0xffff, nh = job.w >> 16;
  const bool busy = h < nh;
  float M = -INFINITY, L = 0.f, o[V];
#pragma unroll
  for (int e = 0; e < V; ++e) o[e] = 0.f;
  if (busy) {
    // 32 parts at a time: their (m, l), then their sums, 8 loads in flight
    for (int k0 = first; k0 < parts; k0 += 32 * share_of) {
      const int mine = k0 + lane * share_of;
      float2 ml = make_float2(-INFINITY, 0.f);
      if (mine < parts) ml = k0 == first ? next_ml : *reinterpret_cast<const float2 *>(a.part_ml + 2 * part(mine));
      float m = ml.x;
#pragma unroll
      for (int d = 16; d; d >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, d));
      m = fmaxf(m, M);
      const float ref = m == -INFINITY ? 0.f : m;
      const float keep = M == -INFINITY ? 0.f : exp2_fast(M - ref);
      M = m;
      const float c = ml.y != 0.f ? exp2_fast(ml.x - ref) : 0.f;
      float l = ml.y != 0.f ? ml.y * c : 0.f;
#pragma unroll
      for (int d = 16; d; d >>= 1) l += __shfl_xor_sync(0xffffffffu, l, d);
      L = L * keep + l;
#pragma unroll
      for (int e = 0; e < V; ++e) o[e] *= keep;
      const unsigned there = __ballot_sync(0xffffffffu, ml.y != 0.f);
      const int n = min(32, (parts - k0 + share_of - 1) / share_of);
      auto take = [&](int i, const float (&x)[V]) {
        const float ci = __shfl_sync(0xffffffffu, c, i);
#pragma unroll
        for (int e = 0; e < V; ++e) o[e] += (there >> i & 1) ? ci * x[e] : 0.f;
      };
      int i = 0;
      if (k0 == first) {
        take(0, early[0]);
        if (n > 1) take(1, early[1]);
        i = 2;
      }
#pragma unroll 8
      for (; i < n; ++i) {
        float x[V];
        sums_of(k0 + i * share_of, x);
        take(i, x);
      }
    }
  }
#pragma unroll
  for (int e = 0; e < V; ++e) s_o[warp][lane * V + e] = o[e];
  if (lane == 0) { s_m[warp] = M; s_l[warp] = L; }
  __syncthreads();
  if (!busy || first != 0) return;
  float top = -INFINITY;
  for (int w = 0; w < share_of; ++w) top = fmaxf(top, s_m[warp + w]);
  const float ref = top == -INFINITY ? 0.f : top;
  L = 0.f;
#pragma unroll
  for (int e = 0; e < V; ++e) o[e] = 0.f;
  for (int w = 0; w < share_of; ++w) {
    const float l = s_l[warp + w];
    if (l == 0.f) continue;
    const float c = exp2_fast(s_m[warp + w] - ref);
    L += l * c;
#pragma unroll
    for (int e = 0; e < V; ++e) o[e] += s_o[warp + w][lane * V + e] * c;
  }
  const float f = L == 0.f ? 0.f : (a.v_scale ? __ldg(a.v_scale + kvh) : 1.f) / L;
  const long long head = job.z + h;
  write_out<X, V>(a, row * a.out_row_stride + head * a.out_head_stride + lane * V, o, f);
  if (lane == 0 && a.lse) a.lse[(long long)row * a.hq + head] = L == 0.f ? -INFINITY : (top + (log2f(L) - (F16 ? 15.f : 0.f))) * kLn2;
}

// ---------------------------------------------------------------- launch
// What is known of a kernel on a device: the SMs (0: not asked yet) and how many clusters of 2 .. 16 CTAs run at once.
struct Device {
  std::atomic<int> sms, clusters[17];
};

template <int DH, int CACHE, int X, int MT>
int launch(const PoolMaps &m, PagedAttnArgs a, cudaStream_t st) {
  using C = Cfg<DH, CACHE, X, MT>;
  auto kernel = k_paged_attention<DH, CACHE, X, MT>;
  const int head_bytes = a.heads_per_tile * C::kHeadFloats * (int)sizeof(float);   // a set of sums
  auto stages_beside = [&](int sets) {
    const int n = (kSmemMost - 1024 - sets * head_bytes) / (C::kStageBytes + C::kQBytes);
    return n < kMaxStages ? n : kMaxStages;
  };
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return -1;
  static Device devices[64];
  Device &d = devices[dev];
  int n = d.sms.load(std::memory_order_acquire);
  if (n == 0) {
    if (cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess || n < 1) return -1;
    if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmemMost) != cudaSuccess ||
        cudaFuncSetAttribute(kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1) != cudaSuccess)
      return -1;
    for (int cl = 2; cl <= 16; ++cl) {
      cudaLaunchConfig_t cfg;
      memset(&cfg, 0, sizeof(cfg));
      cfg.gridDim = dim3(cl);
      cfg.blockDim = dim3(C::kThreads);
      cfg.dynamicSmemBytes = kSmemMost;
      cudaLaunchAttribute attr;
      attr.id = cudaLaunchAttributeClusterDimension;
      attr.val.clusterDim.x = cl; attr.val.clusterDim.y = 1; attr.val.clusterDim.z = 1;
      cfg.attrs = &attr;
      cfg.numAttrs = 1;
      int most = 0;
      if (cudaOccupancyMaxActiveClusters(&most, kernel, &cfg) != cudaSuccess) { cudaGetLastError(); most = 0; }
      d.clusters[cl].store(most, std::memory_order_relaxed);   // (the same numbers, if two threads are here)
    }
    if (n > kFusedMaxCtas) n = kFusedMaxCtas;
    d.sms.store(n, std::memory_order_release);
  }
  const long long most = (((long long)a.table_width << a.page_shift) + C::kUnit - 1) / C::kUnit;   // units a row can have
  const long long items = (long long)a.n_rows * a.hkv * a.tiles_per_head;
  // Few items: a cluster of CTAs for each, as many as run at once, whose first CTA gets the others' sums through
  // distributed shared memory; no sums over all rows at the start, no join (which costs 4.5 us).  A unit takes a CTA 0.5 us;
  // rows may take 24 units a CTA at most (whatever the table has room for counts): clusters leave some SMs out, and rows
  // of different lengths would leave clusters idle.  Under 5 units a row stays whole (1 row, 32 kv heads of 128, bf16,
  // whole or cut / cluster: 128 positions 5.3 / 5.7 us, 512 8.1 / 7.0, 2048 13.8 / 10.3; 1 row, 8 kv heads: 512 8.8 / 7.0,
  // 2048 10.8 / 9.2).
  constexpr int kWide = DH / 32 * QBytes<X>::v;   // bytes of the dims a lane writes
  a.out_wide = (uintptr_t)a.out % kWide == 0 && a.out_row_stride * QBytes<X>::v % kWide == 0 && a.out_head_stride * QBytes<X>::v % kWide == 0;
  a.cluster = 0;
  if (most >= 5) {
    int cl = (int)(most < 16 ? most : 16);
    while (cl >= 2 && (items > d.clusters[cl].load(std::memory_order_relaxed) || stages_beside(C::kClusterWarps + cl) < 3)) --cl;
    const long long longest = cl >= 2 ? (most + cl - 1) / cl : 0;
    if (cl >= 2 && longest <= 24 && longest <= items * most / n + 9) a.cluster = cl;
  }
  // (All of this is for tables no wider than the lengths need: the host knows no other bound of them.)
  // Otherwise items stay whole whatever the lengths, and no join is launched, where the table has room for 10 units a row at
  // most: the busiest CTA is at most one row longer than an even share (40 kv heads, 8 rows of 512 positions: 20.9 us whole,
  // 22.7 cut); 16 units where every item has a CTA for itself (32 kv heads, 4 rows of 768: 13.1 us without the join, 15.9 with it).
  a.whole = !a.cluster && most <= (items <= n ? 16 : 10);
  const int sets = a.cluster ? C::kClusterWarps + a.cluster : C::kWarps;
  a.n_stages = stages_beside(sets);
  if (a.n_stages < 2) return -1;
  const size_t smem = 1024 + (size_t)a.n_stages * (C::kStageBytes + C::kQBytes) + (size_t)sets * head_bytes;
  // few enough rows for a warp, and all costs within 32 bits whatever the lengths are
  const double capacity = ((double)a.table_width * (1 << a.page_shift) / C::kUnit + 1) * kUnitCost + kItemCost;
  a.few = a.n_rows <= kFewRows && a.n_rows * capacity * a.hkv * a.tiles_per_head < 1.0e9 ? 1 : 0;
  auto map = [](const TMap &t) -> const CUtensorMap & { return *reinterpret_cast<const CUtensorMap *>(&t); };
  if (a.cluster) {
    cudaLaunchConfig_t cfg;
    memset(&cfg, 0, sizeof(cfg));
    cfg.gridDim = dim3((unsigned)(items * a.cluster));
    cfg.blockDim = dim3(C::kThreads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = st;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = a.cluster; attr[1].val.clusterDim.y = 1; attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 2;
    return cudaLaunchKernelEx(&cfg, kernel, map(m.k), map(m.v), map(m.k16), map(m.v16), a) == cudaSuccess ? 0 : -1;
  }
  if (launch_pdl(kernel, dim3(n), dim3(C::kThreads), smem, st, map(m.k), map(m.v), map(m.k16), map(m.v16), a) != cudaSuccess) return -1;
  if (!a.whole)
    if (launch_pdl(k_paged_join<DH, X, C::kF16>, dim3(n), dim3(32 * kJoinWarps), 0, st, a) != cudaSuccess) return -1;
  return 0;
}

template <int DH>
int launch_types(const PoolMaps &m, const PagedAttnArgs &a, int x, cudaStream_t st) {
  const int cache = m.of.dtype;
  const bool wide = a.heads_per_tile > 8;
  if (cache == D3_BF16 && x == D3_FP32) return launch<DH, D3_BF16, D3_FP32, 2>(m, a, st);
  if (cache == D3_BF16) return wide ? launch<DH, D3_BF16, D3_BF16, 2>(m, a, st) : launch<DH, D3_BF16, D3_BF16, 1>(m, a, st);
  if (cache == D3_FP16) return wide ? launch<DH, D3_FP16, D3_FP16, 2>(m, a, st) : launch<DH, D3_FP16, D3_FP16, 1>(m, a, st);
  if (x == D3_BF16) return wide ? launch<DH, D3_E4M3, D3_BF16, 2>(m, a, st) : launch<DH, D3_E4M3, D3_BF16, 1>(m, a, st);
  return wide ? launch<DH, D3_E4M3, D3_FP16, 2>(m, a, st) : launch<DH, D3_E4M3, D3_FP16, 1>(m, a, st);
}

}  // namespace paged_attn
}  // namespace d3
