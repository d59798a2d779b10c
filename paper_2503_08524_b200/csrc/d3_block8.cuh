// Shared by the 8-bit block operators: host-side checks, numbers of every type, and the PTX of the tensor-core products.
#pragma once

#include <cuda.h>   // CUtensorMap and its enums; the encoder is fetched at run time
#include <cuda_fp16.h>
#include <cuda_fp8.h>

#include "d3_internal.cuh"

namespace d3 {

constexpr int kScaleBlock = 128;                 // numbers that share a scale
constexpr float kE4m3Max = 448.f;
constexpr float kLeastTop = 7.888609e-31f;       // 2^-100: a block's largest number counts as this at least
constexpr uint32_t kTryNs = 50;                  // a try of a wait that fails takes 40 to 80 ns
constexpr uint32_t kWaitTries = 40000000u;       // bound of every device-side wait: about two seconds
constexpr uint32_t kDrainTries = 40000u;         // the least that copies and products in flight are waited for: about two milliseconds

// ------------------------------------------------------------------ host
inline int type_bytes(int dtype) { return dtype == D3_FP32 ? 4 : dtype == D3_E4M3 ? 1 : 2; }
inline bool wide_type(int dtype) { return dtype == D3_BF16 || dtype == D3_FP16 || dtype == D3_FP32; }
inline bool on_bytes(const void *p, int bytes) { return ((uintptr_t)p & (uintptr_t)(bytes - 1)) == 0; }
// Rows of `width` bytes, `stride` bytes apart.
struct RowSet {
  const void *p;
  int64_t n, stride, width;
};
// The rows of a set that is written do not overlap one another.
inline bool rows_distinct(const RowSet &s) { return s.n <= 1 || s.stride >= s.width; }
// Two sets have a byte in common, as far as can be told without looking at every row: rows of one stride exactly (columns of one
// buffer may be written while others are read), others by the memory between their first and last bytes.
inline bool rows_common(const RowSet &a, const RowSet &b) {
  if (!a.p || !b.p || a.n < 1 || b.n < 1 || a.width < 1 || b.width < 1) return false;
  const int64_t a0 = (int64_t)(uintptr_t)a.p, b0 = (int64_t)(uintptr_t)b.p;
  const int64_t a1 = a0 + (a.n - 1) * a.stride + a.width, b1 = b0 + (b.n - 1) * b.stride + b.width;
  if (a0 >= b1 || b0 >= a1) return false;
  const int64_t stride = a.n > 1 ? a.stride : b.stride;
  if ((a.n > 1 && b.n > 1 && a.stride != b.stride) || stride < a.width || stride < b.width) return true;
  // row i of a and row j of b: the distance of their starts is delta + (j - i) * stride; only the two multiples next to -delta can meet
  const int64_t delta = b0 - a0;
  int64_t q = delta / stride;
  if (q * stride > delta) --q;
  for (int t = 0; t < 2; ++t, ++q) {
    const int64_t off = delta - q * stride;       // start of b's row i - ... relative to a's row that is q rows on
    if (q > -b.n && q < a.n && off < a.width && -off < b.width) return true;
  }
  return false;
}
inline bool same_rows(const RowSet &a, const RowSet &b) { return a.p == b.p && a.width == b.width && (a.n <= 1 || a.stride == b.stride); }

// What d3_weight8_map writes.
struct Weight8Map {
  TMap map;                  // (k, row), boxes of 128 bytes x 128 rows, 128-byte swizzle, zeros outside
  d3_weight8 of;             // the matrix it was made for (map and scales left out)
};
static_assert(sizeof(Weight8Map) <= D3_WEIGHT8_MAP_BYTES, "room for the map");
// tensor map of [rows][k] bytes with `stride` bytes between rows; false when the driver refuses or has no encoder
bool encode_rows8(TMap *out, const void *base, int rows, int k, int64_t stride, int box_rows);
// tensor map of results [rows][n] of a type: boxes of 128 bytes x 128 rows in the 128-byte swizzle
bool encode_results8(TMap *out, void *base, int rows, int n, int dtype, int64_t stride);
bool have_encoder8();

// A product as the kernels see it.
struct Mm8Args {
  int n_rows, n, k, n_kb;            // n_kb: blocks of 128 along k
  const float *a_scale;
  long long a_scale_stride;
  const float *w_scale[2];           // [ceil(n / 128)][n_kb]
  void *out;
  long long out_stride;
  int out_dtype;
  float *scale;
  long long scale_stride;
  int32_t *status;
  uint32_t wait_tries;
  int stall;                         // drill: the first CTA's copies seem never to land
};
// each enqueues one kernel; cudaSuccess or what the launch said (w1: the second matrix of the gated form)
struct FewPlan { int rows, split; };   // rows of a CTA, CTAs that share the k of a tile
cudaError_t launch_mm8_few(const TMap &w0, const TMap *w1, const void *a, int64_t a_stride, const Mm8Args &p, const FewPlan &plan, cudaStream_t st);
cudaError_t launch_mm8_many(const TMap &w0, const TMap *w1, const void *a, int64_t a_stride, const Mm8Args &p, cudaStream_t st);
// estimates of what the kernels take, in us; `plan`: the best way of the kernel for few rows
float plan_mm8_few(const Mm8Args &p, int mats, FewPlan &plan);
float estimate_mm8_many(const Mm8Args &p, int mats);

// ------------------------------------------------------------------ device
#ifdef __CUDACC__
__device__ __forceinline__ float half_lo(uint32_t w) { return __half2float(__ushort_as_half((unsigned short)(w & 0xffffu))); }
__device__ __forceinline__ float half_hi(uint32_t w) { return __half2float(__ushort_as_half((unsigned short)(w >> 16))); }
// 8 consecutive numbers as floats (16-byte aligned)
__device__ __forceinline__ void load8(const void *base, long long at, int dtype, float (&v)[8]) {
  if (dtype == D3_FP32) {
    const float4 *p = reinterpret_cast<const float4 *>(static_cast<const float *>(base) + at);
    const float4 a = p[0], b = p[1];
    v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w; v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
    return;
  }
  const uint4 u = *reinterpret_cast<const uint4 *>(static_cast<const char *>(base) + 2 * at);
  const uint32_t w[4] = {u.x, u.y, u.z, u.w};
  if (dtype == D3_BF16) {
#pragma unroll
    for (int i = 0; i < 4; ++i) { v[2 * i] = __uint_as_float(w[i] << 16); v[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u); }
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) { v[2 * i] = half_lo(w[i]); v[2 * i + 1] = half_hi(w[i]); }
  }
}
// two floats in a 32-bit word, rounded to nearest even
__device__ __forceinline__ uint32_t pack2(float a, float b, int dtype) {
  uint32_t r;
  if (dtype == D3_BF16) asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(b), "f"(a));
  else asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(b), "f"(a));
  return r;
}
__device__ __forceinline__ void store8(void *base, long long at, int dtype, const float (&v)[8]) {
  if (dtype == D3_FP32) {
    float4 *p = reinterpret_cast<float4 *>(static_cast<float *>(base) + at);
    p[0] = make_float4(v[0], v[1], v[2], v[3]);
    p[1] = make_float4(v[4], v[5], v[6], v[7]);
    return;
  }
  *reinterpret_cast<uint4 *>(static_cast<char *>(base) + 2 * at) =
      make_uint4(pack2(v[0], v[1], dtype), pack2(v[2], v[3], dtype), pack2(v[4], v[5], dtype), pack2(v[6], v[7], dtype));
}
__device__ __forceinline__ void store1(void *base, long long at, int dtype, float v) {
  if (dtype == D3_FP32) static_cast<float *>(base)[at] = v;
  else if (dtype == D3_BF16) static_cast<bf16 *>(base)[at] = __float2bfloat16_rn(v);
  else static_cast<__half *>(base)[at] = __float2half_rn(v);
}
__device__ __forceinline__ float load1(const void *base, long long at, int dtype) {
  if (dtype == D3_FP32) return static_cast<const float *>(base)[at];
  if (dtype == D3_BF16) return __bfloat162float(static_cast<const bf16 *>(base)[at]);
  return __half2float(static_cast<const __half *>(base)[at]);
}
// four floats in 8 bits each (saturating: only a NaN, or the rounding of a quotient, is beyond 448 after the division by the scale)
__device__ __forceinline__ uint32_t pack_e4m3(float a, float b, float c, float d) {
  uint16_t lo, hi;
  asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(lo) : "f"(b), "f"(a));
  asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(hi) : "f"(d), "f"(c));
  return (uint32_t)lo | ((uint32_t)hi << 16);
}
// the larger one, NaN if either is
__device__ __forceinline__ float max_nan(float a, float b) {
  float r;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
  return r;
}
__device__ __forceinline__ uint32_t smem_at(const void *p) { return (uint32_t)__cvta_generic_to_shared(p); }
__device__ __forceinline__ void mbar_init(uint32_t bar, uint32_t count) {
  asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(bar), "r"(count) : "memory");
}
__device__ __forceinline__ void mbar_expect(uint32_t bar, uint32_t bytes) {
  asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(bytes) : "memory");
}
__device__ __forceinline__ void mbar_arrive(uint32_t bar) {
  asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ bool mbar_try(uint32_t bar, uint32_t parity) {
  uint32_t ok;
  asm volatile("{\n\t.reg .pred p;\n\tmbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n\tselp.u32 %0, 1, 0, p;\n\t}"
               : "=r"(ok) : "r"(bar), "r"(parity) : "memory");
  return ok;
}
// Bounded wait for a barrier's phase; false when the limit ran out (the CTA's flag is then set) or, with `leave`, when another
// wait of the CTA did.  The limit is a count of tries: one takes 40 to 80 ns where it fails, and a look at a clock in this
// loop costs the few warps that drive the tensor core more than it tells.
__device__ __forceinline__ bool mbar_wait(uint32_t bar, uint32_t parity, volatile int *gave_up, uint32_t tries, bool leave = true) {
  for (uint32_t n = 0;; ++n) {
    if (mbar_try(bar, parity)) return true;
    if ((n & 255u) == 255u && ((leave && *gave_up) || n >= tries)) break;
  }
  *gave_up = 1;
  return false;
}
// Barriers that the lanes of a warp have to reach together.  Loops of unlike lengths or a branch of one lane may have left them apart.
__device__ __forceinline__ void group_sync(int barrier, int threads) {
  __syncwarp();
  asm volatile("bar.sync %0, %1;" ::"r"(barrier), "r"(threads) : "memory");
}
__device__ __forceinline__ void cluster_arrive() {
  __syncwarp();
  asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
}
__device__ __forceinline__ void cluster_wait() {
  __syncwarp();
  asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
}
__device__ __forceinline__ void cluster_sync() {
  cluster_arrive();
  cluster_wait();
}
// one lane of a converged warp, the same one every time
__device__ __forceinline__ bool elect_one() {
  uint32_t r;
  asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(r));
  return r;
}
// 4 bytes to shared memory without waiting
__device__ __forceinline__ void copy4(uint32_t to, const void *from) {
  asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(to), "l"(from) : "memory");
}
__device__ __forceinline__ void tma_rows8(uint32_t dst, const void *map, int x, int y, uint32_t bar) {
  asm volatile("cp.async.bulk.tensor.2d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];"
               ::"r"(dst), "l"(reinterpret_cast<uint64_t>(map)), "r"(x), "r"(y), "r"(bar) : "memory");
}
// Shared-memory descriptor of rows of 128 bytes in the 128-byte swizzle, k contiguous: groups of 8 rows are 1024 bytes apart.
__device__ __forceinline__ uint64_t desc_rows8(uint32_t at) {
  return (uint64_t)((at & 0x3ffffu) >> 4) | ((uint64_t)1 << 16) | ((uint64_t)(1024 >> 4) << 32) | ((uint64_t)1 << 46) | ((uint64_t)2 << 61);
}
// Instruction descriptor: e4m3 x e4m3 -> fp32, both operands k-contiguous, M x N.
__host__ __device__ constexpr uint32_t idesc_e4m3(int M, int N) {
  return (1u << 4) | ((uint32_t)(N >> 3) << 17) | ((uint32_t)(M >> 4) << 24);
}
__device__ __forceinline__ void tc_fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tc_fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tc_mma_e4m3(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t add) {
  asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\ttcgen05.mma.cta_group::1.kind::f8f6f4 [%0], %1, %2, %3, p;\n\t}"
               ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(add) : "memory");
}
// one arrival once everything that this thread has given the tensor core so far is done
__device__ __forceinline__ void tc_commit(uint32_t bar) {
  asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
}
// two floats in a register pair, multiplied and added by one instruction
__device__ __forceinline__ uint64_t two_of(uint32_t low, uint32_t high) {
  uint64_t r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "r"(low), "r"(high));
  return r;
}
__device__ __forceinline__ void fma_two(uint64_t &acc, uint64_t a, uint64_t b) { asm("fma.rn.f32x2 %0, %1, %2, %0;" : "+l"(acc) : "l"(a), "l"(b)); }
__device__ __forceinline__ float low_of(uint64_t v) { return __uint_as_float((uint32_t)v); }
__device__ __forceinline__ float high_of(uint64_t v) { return __uint_as_float((uint32_t)(v >> 32)); }
// Scale of a block whose largest absolute value is `top`, and what quotients by it are made of.
struct BlockScale {
  float scale, inverse, divisor;
};
__device__ __forceinline__ BlockScale block_scale(float top) {
  BlockScale b;
  top = max_nan(top, kLeastTop);
  constexpr float kPart = 1.f / kE4m3Max;              // (top / 448, rounded as the quotients below are; every top's is the division's)
  const float q = top * kPart, s = fmaf(fmaf(-q, kE4m3Max, top), kPart, q);
  const bool infinite = top == INFINITY;
  b.scale = infinite ? top : s;
  b.inverse = __frcp_rn(b.scale);                      // (2^-109 <= scale < 2^120: normal numbers both)
  b.divisor = infinite ? 0.f : s;                      // (beside an infinity finite numbers become 0, not 0 * inf)
  return b;
}
// Blocks whose remainders would fall below the smallest number are divided 2^64 times larger: this says so of a scale and sets it up,
// the numbers are the caller's to multiply.
constexpr float kLift = 0x1p64f;
__device__ __forceinline__ bool lift(BlockScale &b) {
  if (!(b.scale < 0x1p-90f)) return false;
  b.inverse *= 1.f / kLift;
  b.divisor *= kLift;
  return true;
}
// Two numbers divided by their block's scale, as fp32 division rounds it: v * inverse with the remainder's share put back
// (Markstein's division: correct where the inverse is the rounded reciprocal; checked for every divisor next to each border between two
// codes of 8 bits, where with an inverse that is 2^-23 off some numbers get the other code).  The remainder is exact, so its rounding
// downwards says nothing but that one of nothing is -0, which leaves a quotient of -0 as it is.
__device__ __forceinline__ uint64_t quotient_two(float v0, float v1, const BlockScale &b) {
  const uint64_t v = two_of(__float_as_uint(v0), __float_as_uint(v1)), i = two_of(__float_as_uint(b.inverse), __float_as_uint(b.inverse)),
                 d = two_of(__float_as_uint(-b.divisor), __float_as_uint(-b.divisor));
  uint64_t q, r;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(q) : "l"(v), "l"(i));
  asm("fma.rm.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(q), "l"(d), "l"(v));
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(q) : "l"(r), "l"(i), "l"(q));
  return q;
}
// four numbers of a block in 8 bits
__device__ __forceinline__ uint32_t quantize4(float v0, float v1, float v2, float v3, const BlockScale &b) {
  const uint64_t lo = quotient_two(v0, v1, b), hi = quotient_two(v2, v3, b);
  return pack_e4m3(low_of(lo), high_of(lo), low_of(hi), high_of(hi));
}

// 16, 32 or 64 accumulator columns of this thread's lane, to be read behind tc_ld_wait only
__device__ __forceinline__ void tc_ld(uint32_t at, uint32_t (&r)[16]) {
  asm volatile("tcgen05.ld.sync.aligned.32x32b.x16.b32 "
               "{%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]),
                 "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
               : "r"(at) : "memory");
}
__device__ __forceinline__ void tc_ld(uint32_t at, uint32_t (&r)[32]) {
  asm volatile("tcgen05.ld.sync.aligned.32x32b.x32.b32 "
               "{%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,"
               "%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]),
                 "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]), "=r"(r[17]), "=r"(r[18]), "=r"(r[19]),
                 "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]),
                 "=r"(r[30]), "=r"(r[31])
               : "r"(at) : "memory");
}
__device__ __forceinline__ void tc_ld(uint32_t at, uint32_t (&r)[64]) {
  asm volatile("tcgen05.ld.sync.aligned.32x32b.x64.b32 "
               "{%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,"
               "%22,%23,%24,%25,%26,%27,%28,%29,%30,%31,%32,%33,%34,%35,%36,%37,%38,%39,%40,%41,%42,%43,"
               "%44,%45,%46,%47,%48,%49,%50,%51,%52,%53,%54,%55,%56,%57,%58,%59,%60,%61,%62,%63}, [%64];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]),
                 "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]), "=r"(r[17]), "=r"(r[18]), "=r"(r[19]),
                 "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]),
                 "=r"(r[30]), "=r"(r[31]), "=r"(r[32]), "=r"(r[33]), "=r"(r[34]), "=r"(r[35]), "=r"(r[36]), "=r"(r[37]), "=r"(r[38]), "=r"(r[39]),
                 "=r"(r[40]), "=r"(r[41]), "=r"(r[42]), "=r"(r[43]), "=r"(r[44]), "=r"(r[45]), "=r"(r[46]), "=r"(r[47]), "=r"(r[48]), "=r"(r[49]),
                 "=r"(r[50]), "=r"(r[51]), "=r"(r[52]), "=r"(r[53]), "=r"(r[54]), "=r"(r[55]), "=r"(r[56]), "=r"(r[57]), "=r"(r[58]), "=r"(r[59]),
                 "=r"(r[60]), "=r"(r[61]), "=r"(r[62]), "=r"(r[63])
               : "r"(at) : "memory");
}
// waits for the loads so far; nothing may read their registers earlier, which naming them here says
__device__ __forceinline__ void tc_ld_wait(uint32_t (&r)[16]) {
  asm volatile("tcgen05.wait::ld.sync.aligned;"
               : "+r"(r[0]), "+r"(r[1]), "+r"(r[2]), "+r"(r[3]), "+r"(r[4]), "+r"(r[5]), "+r"(r[6]), "+r"(r[7]), "+r"(r[8]), "+r"(r[9]),
                 "+r"(r[10]), "+r"(r[11]), "+r"(r[12]), "+r"(r[13]), "+r"(r[14]), "+r"(r[15])
               :: "memory");
}
__device__ __forceinline__ void tc_ld_wait(uint32_t (&r)[32]) {
  asm volatile("tcgen05.wait::ld.sync.aligned;"
               : "+r"(r[0]), "+r"(r[1]), "+r"(r[2]), "+r"(r[3]), "+r"(r[4]), "+r"(r[5]), "+r"(r[6]), "+r"(r[7]), "+r"(r[8]), "+r"(r[9]),
                 "+r"(r[10]), "+r"(r[11]), "+r"(r[12]), "+r"(r[13]), "+r"(r[14]), "+r"(r[15]), "+r"(r[16]), "+r"(r[17]), "+r"(r[18]), "+r"(r[19]),
                 "+r"(r[20]), "+r"(r[21]), "+r"(r[22]), "+r"(r[23]), "+r"(r[24]), "+r"(r[25]), "+r"(r[26]), "+r"(r[27]), "+r"(r[28]), "+r"(r[29]),
                 "+r"(r[30]), "+r"(r[31])
               :: "memory");
}
__device__ __forceinline__ void tc_ld_wait(uint32_t (&r)[64]) {
  asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
#pragma unroll
  for (int i = 0; i < 64; i += 8)
    asm volatile("" : "+r"(r[i]), "+r"(r[i + 1]), "+r"(r[i + 2]), "+r"(r[i + 3]), "+r"(r[i + 4]), "+r"(r[i + 5]), "+r"(r[i + 6]), "+r"(r[i + 7]) :: "memory");
}
// silu(g) * u = g / (1 + exp(-g)) * u, with 2^x and 1/x of the special function unit.  2^x is as good as its argument: the product
// -g log2(e) is rounded, by up to 2^-18 where |g| is 88, and log2(e) itself is 2^-26 off in 32 bits, so what both left out, which
// fused multiply-adds give, is put back by 2^(hi + lo) = 2^hi (1 + lo ln 2).  From 1 + exp(-g) = 2^126 on the reciprocal is below the normal
// numbers, where the unit gives 0, so far out a quarter of both sides is divided.  An exp(-g) that is infinite (g below -88.72) gives 0.
__device__ __forceinline__ float gate_of(float g, float u) {
  constexpr float kLog2e = 1.44269504f, kRest = 1.925963e-8f;    // log2(e) = 1.44269502162933 in 32 bits + 0.00000001925963
  const float hi = g * -kLog2e, lo = fmaf(g, -kRest, fmaf(g, -kLog2e, -hi)), part = hi > 100.f ? 0.25f : 1.f;
  float t, r;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(t) : "f"(hi));
  if (fabsf(hi) < 128.f) t = fmaf(t, lo * 0.693147181f, t);      // (beyond, t is 0 or infinite, and lo may be NaN)
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(fmaf(t, part, part)));
  return g * part * r * u;
}
#endif

}  // namespace d3
