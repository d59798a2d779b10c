// Paged key-value operators: block tables and slot maps, append, and the C ABI of the three calls.
#include <cuda.h>   // CUtensorMap and its enums; the encoder is fetched at run time
#include <cuda_fp16.h>
#include <cuda_fp8.h>
#include <math.h>

#include <atomic>
#include <type_traits>

#include "d3_paged.cuh"

namespace d3 {

namespace {

// ------------------------------------------------------------------ plan
// Latency decides: the whole plan is one launch.  Every CTA reads the R lengths and keeps the three running sums
// (tokens, pages needed, pages given back) of all requests in shared memory; after that the CTAs share page and token
// entries between them and need nothing of one another: a page that is taken is looked up by its rank in
// (old stack ++ pages given back), so nothing waits for the stack or the table to be written, and what is written is
// never what another CTA reads.  Only where the new lengths replace the old ones in place must no CTA read them any
// more when they are written: with several CTAs a second launch, of one CTA, then writes the lengths
// (192 prompts in place: 8.4 us; as one cluster of eight CTAs with a barrier 20.8).
constexpr int kPlanMaxThreads = 1024;
constexpr int kPlanMaxPer = D3_MAX_REQUESTS / kPlanMaxThreads;   // requests of one thread

struct PlanArgs {
  int R, page_shift, n_pages, width, T;
  long long table_stride;
  const int32_t *cached, *added;
  int32_t *table, *free_pages;
  const int32_t *n_free;
  int32_t *cached_out, *n_free_out, *first;
  long long *slots;
  int32_t *row, *context, *status;
  int maps, lengths;   // what this launch writes: pages, maps and `first`; cached_out and n_free_out
};

// the request whose half-open range [sum[b], sum[b + 1]) holds x  (sum[0] = 0 <= x < sum[R])
__device__ __forceinline__ int owner(const int *sum, int R, int x) {
  int lo = 0, hi = R;          // sum[lo] <= x < sum[hi]
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (sum[mid] <= x) lo = mid; else hi = mid;
  }
  return lo;
}

// S: type of the sums (32 bits where no sum of R entries of at most max_tokens or n_pages can leave them)
template <typename S>
__global__ void __launch_bounds__(kPlanMaxThreads) k_page_plan(const __grid_constant__ PlanArgs a) {
  extern __shared__ int s_plan[];
  int *s_first = s_plan, *s_need = s_first + (a.R + 1), *s_back = s_need + (a.R + 1), *s_cached = s_back + (a.R + 1);
  __shared__ S s_warp[3][32];
  __shared__ int s_bad;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, threads = blockDim.x;
  const int page_mask = (1 << a.page_shift) - 1;
  const long long max_len = (long long)a.width << a.page_shift;
  if (tid == 0) s_bad = 0;
  pdl_wait();
  pdl_trigger();
  __syncthreads();

  const int n_free = *a.n_free;
  const int per = (a.R + threads - 1) / threads;
  S sum[3] = {0, 0, 0};                       // this thread's tokens, pages needed, pages given back
  int c_[kPlanMaxPer], add_[kPlanMaxPer], need_[kPlanMaxPer], back_[kPlanMaxPer];
  int bad = (n_free < 0 || n_free > a.n_pages) ? 2 : 0;
#pragma unroll
  for (int i = 0; i < kPlanMaxPer; ++i) {
    const int b = tid * per + i;
    c_[i] = add_[i] = need_[i] = back_[i] = 0;
    if (i < per && b < a.R) {
      const int c = a.cached[b], n = a.added[b];
      const long long grown = (long long)c + (n > 0 ? n : 0);
      const int have = (int)(((long long)c + page_mask) >> a.page_shift);
      if (c < 0 || c > max_len || (n < 0 && have > a.n_pages)) { bad |= 2; }
      else if (grown > max_len || n > a.T) { bad |= 1; }
      else {
        c_[i] = c;
        if (n < 0) back_[i] = have;
        else {
          add_[i] = n;
          need_[i] = (int)((grown + page_mask) >> a.page_shift) - have;
        }
      }
      sum[0] += add_[i]; sum[1] += need_[i]; sum[2] += back_[i];
    }
  }
  if (bad) atomicOr(&s_bad, bad);
  S inc[3] = {sum[0], sum[1], sum[2]};
#pragma unroll
  for (int d = 1; d < 32; d <<= 1) {
#pragma unroll
    for (int k = 0; k < 3; ++k) {
      const S u = __shfl_up_sync(0xffffffffu, inc[k], d);
      if (lane >= d) inc[k] += u;
    }
  }
  if (lane == 31) { s_warp[0][warp] = inc[0]; s_warp[1][warp] = inc[1]; s_warp[2][warp] = inc[2]; }
  __syncthreads();
  S total[3], before[3];
#pragma unroll
  for (int k = 0; k < 3; ++k) total[k] = lane < threads / 32 ? s_warp[k][lane] : 0;   // one value per warp
#pragma unroll
  for (int k = 0; k < 3; ++k) before[k] = total[k];
#pragma unroll
  for (int d = 1; d < 32; d <<= 1) {
#pragma unroll
    for (int k = 0; k < 3; ++k) {
      const S u = __shfl_up_sync(0xffffffffu, total[k], d);
      if (lane >= d) total[k] += u;
    }
  }
#pragma unroll
  for (int k = 0; k < 3; ++k) {
    before[k] = __shfl_sync(0xffffffffu, total[k] - before[k], warp) + inc[k] - sum[k];
    total[k] = __shfl_sync(0xffffffffu, total[k], 31);
  }
  bad = s_bad;
  if ((long long)n_free + total[2] > a.n_pages) bad |= 2;      // more pages than there are came back
  if (total[0] > a.T || total[1] > (long long)n_free + total[2]) bad |= 1;
  if (!bad) {
#pragma unroll
    for (int i = 0; i < kPlanMaxPer; ++i) {
      const int b = tid * per + i;
      if (i < per && b < a.R) {
        s_first[b] = (int)before[0]; s_need[b] = (int)before[1]; s_back[b] = (int)before[2];
        s_cached[b] = c_[i];
        before[0] += add_[i]; before[1] += need_[i]; before[2] += back_[i];
      }
    }
    if (tid == 0) { s_first[a.R] = (int)total[0]; s_need[a.R] = (int)total[1]; s_back[a.R] = (int)total[2]; }
  }
  __syncthreads();   // (one CTA may write in place: all its threads have read the lengths and the stack's height)

  const int gid = blockIdx.x * threads + tid, step = gridDim.x * threads;
  if (blockIdx.x == 0) {
#pragma unroll
    for (int i = 0; i < kPlanMaxPer; ++i) {
      const int b = tid * per + i;
      if (i < per && b < a.R) {
        if (a.lengths) {
          if (!bad) a.cached_out[b] = back_[i] ? 0 : c_[i] + add_[i];
          else if (a.cached_out != a.cached) a.cached_out[b] = a.cached[b];
        }
        if (a.maps) a.first[b] = bad ? 0 : s_first[b];
      }
    }
    if (tid == 0) {
      if (a.maps) a.first[a.R] = bad ? 0 : (int)total[0];
      if (a.lengths) {
        if (!bad) *a.n_free_out = (int)(n_free + total[2] - total[1]);
        else if (a.n_free_out != a.n_free) *a.n_free_out = n_free;
      }
      if (bad && a.status) *a.status = (bad & 2) ? D3_EINVAL : D3_ECAPACITY;
    }
  }
  if (!a.maps) return;
  const int n_tok = bad ? 0 : (int)total[0], n_need = bad ? 0 : (int)total[1], n_back = bad ? 0 : (int)total[2];
  const int top = n_free + n_back;
  // entry i of (old stack ++ pages given back)
  auto stack = [&](int i) -> int {
    if (i < n_free) return a.free_pages[i];
    const int b = owner(s_back, a.R, i - n_free);
    return a.table[b * a.table_stride + (i - n_free - s_back[b])];
  };
  auto pages_of = [&](int len) { return (len + page_mask) >> a.page_shift; };   // len <= 2^31 - 1024 (checked on the host)

  // one index over the pages given back, the pages taken and the tokens by fours (one search, map entries in 16-byte
  // pieces): the three kinds run side by side
  bool strange = false;
  const long long n_all = (long long)n_back + n_need + ((long long)a.T + 3) / 4;
  for (long long at = gid; at < n_all; at += step) {
    if (at < n_back) {
      const int e = (int)at, b = owner(s_back, a.R, e);
      const int id = a.table[b * a.table_stride + (e - s_back[b])];
      if (id < 0 || id >= a.n_pages) strange = true;
      a.free_pages[n_free + e] = id;
      continue;
    }
    if (at < (long long)n_back + n_need) {
      const int e = (int)(at - n_back), b = owner(s_need, a.R, e);
      a.table[b * a.table_stride + pages_of(s_cached[b]) + (e - s_need[b])] = stack(top - 1 - e);
      continue;
    }
    const long long t0 = (at - n_back - n_need) * 4;
    long long slot[4];
    int row[4], ctx[4];
    int b = t0 < n_tok ? owner(s_first, a.R, (int)t0) : a.R;
    int last_page = -1, id = -1;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const long long t = t0 + i;
      slot[i] = -1; row[i] = -1; ctx[i] = 0;
      if (t < n_tok) {
        while (t >= s_first[b + 1]) { ++b; last_page = -1; }
        const int pos = s_cached[b] + (int)(t - s_first[b]);
        const int pg = pos >> a.page_shift, have = pages_of(s_cached[b]);
        if (pg != last_page) {
          // a page taken by this call is read from the stack: its table entry may not be written yet
          id = pg < have ? a.table[b * a.table_stride + pg] : stack(top - 1 - (s_need[b] + pg - have));
          last_page = pg;
        }
        row[i] = b;
        ctx[i] = pos + 1;
        if (id >= 0 && id < a.n_pages) slot[i] = ((long long)id << a.page_shift) | (pos & page_mask);
        else strange = true;
      }
    }
    if (t0 + 4 <= a.T) {
      reinterpret_cast<longlong2 *>(a.slots + t0)[0] = make_longlong2(slot[0], slot[1]);
      reinterpret_cast<longlong2 *>(a.slots + t0)[1] = make_longlong2(slot[2], slot[3]);
      *reinterpret_cast<int4 *>(a.row + t0) = make_int4(row[0], row[1], row[2], row[3]);
      *reinterpret_cast<int4 *>(a.context + t0) = make_int4(ctx[0], ctx[1], ctx[2], ctx[3]);
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (t0 + i < a.T) { a.slots[t0 + i] = slot[i]; a.row[t0 + i] = row[i]; a.context[t0 + i] = ctx[i]; }
    }
  }
  if (strange && a.status) *a.status = D3_EINVAL;
}

// ------------------------------------------------------------------ append
// Bandwidth: every number once in and once out.  A thread takes the pairs (8 numbers of a head's lower
// half, the 8 that they are paired with), so the rotation needs no exchange and all traffic is in
// 16-byte pieces (8 for the 8-bit cache); it does that for H neighbouring heads of one token, whose (cos, sin) it loads
// once.  q, K and V have blocks of their own, so that what a block does and where its numbers lie is uniform;
// inside, (token, group of H heads) is one index.  All loads are in flight before the slot is looked at.  The three kinds of
// blocks take turns, which keeps a token's rotary row in the caches and mixes those that compute more with those
// that compute less (all of q, then K, then V / in turn: 8191 tokens, 64 + 16 heads, 16-bit 52.1 / 51.3 us; 4097 tokens,
// 40 + 80 heads, 8-bit 39.7 / 39.0).
struct AppendPart {
  const void *src;
  void *dst;
  long long st, sh, dt, dh;     // strides of tokens (q_out alone) and heads
  const float *scale;
  int heads, groups;            // groups of H heads
  unsigned magic, shift;        // index / groups = index * magic >> shift
  int rotate;
};
struct AppendArgs {
  AppendPart part[3];           // q, K, V
  int n_tokens, rope_len;
  unsigned q_blocks, k_blocks;  // (V has as many as K)
  const long long *slots;
  const int32_t *context;
  const float *rope;
  int32_t *status;
  KvPool kv;
};

// eight numbers as they lie in memory, and widened
template <typename T> struct Raw8 { uint4 u; };
template <> struct Raw8<float> { uint4 u, w; };
template <typename T>
__device__ __forceinline__ void fetch(Raw8<T> &r, const T *p) { r.u = *reinterpret_cast<const uint4 *>(p); }
__device__ __forceinline__ void fetch(Raw8<float> &r, const float *p) {
  r.u = reinterpret_cast<const uint4 *>(p)[0];
  r.w = reinterpret_cast<const uint4 *>(p)[1];
}
__device__ __forceinline__ void widen8(const Raw8<float> &r, float *f) {
  const uint32_t w[8] = {r.u.x, r.u.y, r.u.z, r.u.w, r.w.x, r.w.y, r.w.z, r.w.w};
#pragma unroll
  for (int i = 0; i < 8; ++i) f[i] = __uint_as_float(w[i]);
}
__device__ __forceinline__ void widen8(const Raw8<bf16> &r, float *f) {
  const uint32_t w[4] = {r.u.x, r.u.y, r.u.z, r.u.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    f[2 * i] = __uint_as_float(w[i] << 16);
    f[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
  }
}
__device__ __forceinline__ void widen8(const Raw8<__half> &r, float *f) {
  const uint32_t w[4] = {r.u.x, r.u.y, r.u.z, r.u.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float2 v = __half22float2(*reinterpret_cast<const __half2 *>(&w[i]));
    f[2 * i] = v.x; f[2 * i + 1] = v.y;
  }
}
// the plain division, out of line: it is rarely taken, and 64 copies of it would crowd the instruction cache
__device__ __noinline__ float plain_division(float x, float d) { return __fdiv_rn(x, d); }
// x / d rounded once, for |x| <= 2^40 and a d in 2^-60 .. 2^60 whose correctly rounded reciprocal r is known: the remainder
// of the first quotient is exact in one FMA, and taking it times r off rounds like the division (Markstein 1990).
// In these signs a zero keeps its own.
__device__ __forceinline__ float divide(float x, float d, float r) {
  const float q = __fmul_rn(x, r);
  return __fmaf_rn(__fmaf_rn(q, d, -x), -r, q);
}
__device__ __forceinline__ void store8(float *p, const float *f) {
  reinterpret_cast<float4 *>(p)[0] = make_float4(f[0], f[1], f[2], f[3]);
  reinterpret_cast<float4 *>(p)[1] = make_float4(f[4], f[5], f[6], f[7]);
}
__device__ __forceinline__ void store8(bf16 *p, const float *f) {
  uint32_t w[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const __nv_bfloat162 v = __floats2bfloat162_rn(f[2 * i], f[2 * i + 1]);
    w[i] = *reinterpret_cast<const uint32_t *>(&v);
  }
  *reinterpret_cast<uint4 *>(p) = make_uint4(w[0], w[1], w[2], w[3]);
}
__device__ __forceinline__ void store8(__half *p, const float *f) {
  uint32_t w[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const __half2 v = __floats2half2_rn(f[2 * i], f[2 * i + 1]);
    w[i] = *reinterpret_cast<const uint32_t *>(&v);
  }
  *reinterpret_cast<uint4 *>(p) = make_uint4(w[0], w[1], w[2], w[3]);
}
__device__ __forceinline__ void store8(__nv_fp8_e4m3 *p, const float *f) {
  uint32_t w[2];
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const uint32_t lo = __nv_cvt_float2_to_fp8x2(make_float2(f[4 * i], f[4 * i + 1]), __NV_SATFINITE, __NV_E4M3);
    const uint32_t hi = __nv_cvt_float2_to_fp8x2(make_float2(f[4 * i + 2], f[4 * i + 3]), __NV_SATFINITE, __NV_E4M3);
    w[i] = lo | (hi << 16);
  }
  *reinterpret_cast<uint2 *>(p) = make_uint2(w[0], w[1]);
}

// 8-bit stores compute more per byte (a division and a conversion): four blocks an SM, 64 registers, two heads a thread
// hide that (4097 tokens, 40 + 80 heads of 128: 39.0 us; three blocks 45.5, five, which spill, 55.6).
template <typename X, typename C, int DH, int H>
__global__ void __launch_bounds__(256, sizeof(C) == 1 ? 4 : 1) k_paged_append(const __grid_constant__ AppendArgs a) {
  constexpr int HALF = DH / 2, PIECES = HALF / 8, LANES = 256 / PIECES;   // (token, group) pairs of a block
  pdl_wait();
  pdl_trigger();
  // blocks of q, K and V in turn while there are all three, then what is left (K and V have equally many)
  const unsigned m = min(a.q_blocks, a.k_blocks), id = blockIdx.x;
  int which;
  unsigned block;
  if (id < 3 * m) { which = id % 3; block = id / 3; }
  else if (a.q_blocks > m) { which = 0; block = id - 2 * m; }
  else { which = 1 + ((id - 3 * m) & 1); block = m + ((id - 3 * m) >> 1); }
  const AppendPart &p = a.part[which];
  const int j = threadIdx.x % PIECES;
  const unsigned index = block * LANES + threadIdx.x / PIECES;
  const int t = (int)(((unsigned long long)index * p.magic) >> p.shift), h0 = (int)(index - (unsigned)t * p.groups) * H;
  if (t >= a.n_tokens) return;
  const long long slot = a.slots[t];
  const int pos = a.rope ? a.context[t] - 1 : 0;

  Raw8<X> raw[H][2];
  const X *src = static_cast<const X *>(p.src) + t * p.st + h0 * p.sh + 8 * j;
#pragma unroll
  for (int i = 0; i < H; ++i)
    if (h0 + i < p.heads) {
      fetch(raw[i][0], src + i * p.sh);
      fetch(raw[i][1], src + i * p.sh + HALF);
    }
  if (slot < 0) return;
  if (slot >= ((long long)a.kv.n_pages << a.kv.page_shift) || (a.rope && (pos < 0 || pos >= a.rope_len))) {
    if (a.status) *a.status = D3_EINVAL;
    return;
  }
  float4 cs[4];   // (cos, sin) of the eight pairs
  if (p.rotate) {
    const float4 *r = reinterpret_cast<const float4 *>(a.rope + ((long long)pos * HALF + 8 * j) * 2);
#pragma unroll
    for (int i = 0; i < 4; ++i) cs[i] = __ldg(r + i);
  }
  const long long in_page = slot & ((1 << a.kv.page_shift) - 1);
  const long long entry = which == 0 ? t * p.dt : (slot >> a.kv.page_shift) * a.kv.page_stride + in_page * a.kv.token_stride;
#pragma unroll
  for (int i = 0; i < H; ++i) {
    if (h0 + i >= p.heads) break;
    float lo[8], hi[8];
    widen8(raw[i][0], lo);
    widen8(raw[i][1], hi);
    if (p.rotate) {
      // products and sums rounded one by one: no contraction, so every store rounds the same number
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float c = e & 1 ? cs[e / 2].z : cs[e / 2].x, s = e & 1 ? cs[e / 2].w : cs[e / 2].y, x = lo[e], y = hi[e];
        lo[e] = __fsub_rn(__fmul_rn(x, c), __fmul_rn(y, s));
        hi[e] = __fadd_rn(__fmul_rn(y, c), __fmul_rn(x, s));
      }
    }
    const long long at = entry + (h0 + i) * p.dh + 8 * j;
    if (std::is_same<X, C>::value || which == 0) {
      X *dst = static_cast<X *>(p.dst) + at;
      store8(dst, lo);
      store8(dst + HALF, hi);
    } else {
      if (sizeof(C) == 1 && p.scale) {
        const float d = __ldg(p.scale + h0 + i);
        float top = 0.f;   // (NaN is passed over here, and through the division)
#pragma unroll
        for (int e = 0; e < 8; ++e) top = fmaxf(top, fmaxf(fabsf(lo[e]), fabsf(hi[e])));
        if (d >= 0x1p-60f && d <= 0x1p60f && top <= 0x1p40f) {
          const float r = __frcp_rn(d);
#pragma unroll
          for (int e = 0; e < 8; ++e) { lo[e] = divide(lo[e], d, r); hi[e] = divide(hi[e], d, r); }
        } else {
#pragma unroll
          for (int e = 0; e < 8; ++e) { lo[e] = plain_division(lo[e], d); hi[e] = plain_division(hi[e], d); }
        }
      }
      C *dst = static_cast<C *>(p.dst) + at;
      store8(dst, lo);
      store8(dst + HALF, hi);
    }
  }
}

template <typename X, typename C, int DH, int H>
bool launch_append_heads(AppendArgs &a, cudaStream_t st) {
  constexpr unsigned LANES = 256 / (DH / 16);
  unsigned long long blocks = 0;
  for (int i = 0; i < 3; ++i) {
    AppendPart &p = a.part[i];
    p.groups = (p.heads + H - 1) / H;
    const unsigned long long pairs = (unsigned long long)a.n_tokens * p.groups;
    if (pairs >= (1ull << 31) - LANES) return false;
    const unsigned n = (unsigned)((pairs + LANES - 1) / LANES);
    if (i == 0) a.q_blocks = n;
    else a.k_blocks = n;
    blocks += n;
    // exact for indexes below 2^31: magic = ceil(2^(31 + s) / groups), s = ceil(log2(groups))
    unsigned s = 0;
    while ((1u << s) < (unsigned)p.groups) ++s;
    p.shift = 31 + s;
    p.magic = p.groups ? (unsigned)(((1ull << p.shift) + p.groups - 1) / p.groups) : 0;
  }
  if (blocks >= 1ull << 31) return false;
  launch_pdl(k_paged_append<X, C, DH, H>, dim3((unsigned)blocks), dim3(256), 0, st, a);
  return true;
}
template <typename X, typename C, int DH>
bool launch_append_dh(AppendArgs &a, cudaStream_t st) {
  // Several heads per thread read (cos, sin) once for all of them; with few tokens one head per thread spreads the call
  // over more SMs.
  const long long heads = a.part[0].heads + 2ll * a.kv.n_kv_heads;
  if (a.n_tokens * heads * (DH / 16) <= 4ll * 148 * 256) return launch_append_heads<X, C, DH, 1>(a, st);
  return launch_append_heads<X, C, DH, sizeof(C) == 1 ? 2 : 4>(a, st);
}
template <typename X, typename C>
bool launch_append(AppendArgs &a, int dh, cudaStream_t st) {
  return dh == 128 ? launch_append_dh<X, C, 128>(a, st) : dh == 64 ? launch_append_dh<X, C, 64>(a, st) : launch_append_dh<X, C, 32>(a, st);
}

// limit of the attention kernel's waits, and the drill of the next call
std::atomic<unsigned long long> attention_wait_ns{2000000000ull};
std::atomic<int> attention_stall_next{0};

bool int_span_ok(const void *p, unsigned align) { return p && ((uintptr_t)p & (align - 1)) == 0; }

// What a plan reads and writes: the table's rows, `width` of every `stride` entries, and vectors.
struct Span { uintptr_t at; size_t bytes; bool written; };
// Nothing that is written overlaps anything else, the table's rows included: CTAs read and write side by side.  cached_out and
// n_free_out may be what they replace, to the entry (in the vectors' order below: 0 and 1, 2 and 3).
bool plan_apart(const Span (&v)[11], uintptr_t table, int rows, size_t width_bytes, size_t stride_bytes) {
  for (int i = 0; i < 11; ++i) {
    if (!v[i].at) continue;
    for (int j = i + 1; j < 11; ++j) {
      if (!v[j].at || (!v[i].written && !v[j].written)) continue;
      if (v[i].at < v[j].at + v[j].bytes && v[j].at < v[i].at + v[i].bytes && !((i == 0 || i == 2) && j == i + 1 && v[i].at == v[j].at)) return false;
    }
    // the first row that ends behind the vector's start must start behind its end
    if (v[i].at + v[i].bytes <= table) continue;
    const size_t from = v[i].at > table ? v[i].at - table : 0;
    const size_t row = from < width_bytes ? 0 : (from - width_bytes) / stride_bytes + 1;
    if (row < (size_t)rows && table + row * stride_bytes < v[i].at + v[i].bytes) return false;
  }
  return true;
}

// ------------------------------------------------------------------ tensor maps
typedef CUresult (*EncodeTiledFn)(CUtensorMap *, CUtensorMapDataType, cuuint32_t, void *, const cuuint64_t *,
                                  const cuuint64_t *, const cuuint32_t *, const cuuint32_t *,
                                  CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion,
                                  CUtensorMapFloatOOBfill);
EncodeTiledFn pool_encoder() {
  static EncodeTiledFn fn = [] {
    void *p = nullptr;
    cudaDriverEntryPointQueryResult q;
    if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &p, cudaEnableDefault, &q) != cudaSuccess ||
        q != cudaDriverEntryPointSuccess)
      p = nullptr;
    return reinterpret_cast<EncodeTiledFn>(p);
  }();
  return fn;
}

// one float4-aligned region behind the other
struct AttnWorkspace {
  size_t part_o, part_ml, join, total;
};
AttnWorkspace attn_workspace(int dh) {
  AttnWorkspace w;
  const size_t parts = 2 * (size_t)kFusedMaxCtas * 16;   // two cut pieces per CTA, up to 16 heads each
  w.part_o = 0;
  w.part_ml = parts * dh * sizeof(float);
  w.join = w.part_ml + parts * 2 * sizeof(float);
  w.total = (w.join + kFusedMaxCtas * sizeof(int4) + 255) / 256 * 256;
  return w;
}

}  // namespace

bool encode_pool_maps(PoolMaps *out, const d3_paged_kv &kv) {
  EncodeTiledFn fn = pool_encoder();
  if (!fn) return false;
  const int es = bytes_of(kv.dtype), row = kv.head_dim * es, box_bytes = row < 128 ? row : 128;
  const int unit = unit_positions(kv.head_dim, es), rows = kv.page_size < unit ? kv.page_size : unit;
  cuuint64_t dims[4] = {(cuuint64_t)kv.head_dim, (cuuint64_t)kv.page_size, (cuuint64_t)kv.n_kv_heads, (cuuint64_t)kv.n_pages};
  cuuint64_t strides[3] = {(cuuint64_t)(kv.token_stride * es), (cuuint64_t)(kv.head_stride * es),
                           (cuuint64_t)(kv.page_stride * es)};
  cuuint32_t estr[4] = {1, 1, 1, 1};
  const CUtensorMapDataType type = kv.dtype == D3_BF16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16
                                   : kv.dtype == D3_FP16 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT16 : CU_TENSOR_MAP_DATA_TYPE_UINT8;
  const CUtensorMapSwizzle sw = box_bytes == 128 ? CU_TENSOR_MAP_SWIZZLE_128B
                                : box_bytes == 64 ? CU_TENSOR_MAP_SWIZZLE_64B : CU_TENSOR_MAP_SWIZZLE_32B;
  auto encode = [&](TMap *m, void *base, int box_rows) {
    cuuint32_t box[4] = {(cuuint32_t)(box_bytes / es), (cuuint32_t)box_rows, 1, 1};
    return fn(reinterpret_cast<CUtensorMap *>(m), type, 4, base, dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE, sw,
              CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
  };
  if (!encode(&out->k, kv.k_dev, rows) || !encode(&out->v, kv.v_dev, rows)) return false;
  if (rows == 16) { out->k16 = out->k; out->v16 = out->v; }
  else if (!encode(&out->k16, kv.k_dev, 16) || !encode(&out->v16, kv.v_dev, 16)) return false;
  out->of = kv;
  out->of.maps = nullptr;
  out->of.k_scale_dev = out->of.v_scale_dev = nullptr;
  return true;
}

}  // namespace d3

using namespace d3;

extern "C" {

int32_t d3_paged_maps(const d3_paged_kv *kv, void *maps) {
  if (!kv_ok(kv, true) || !maps || ((uintptr_t)maps & 63)) return D3_EINVAL;
  return encode_pool_maps(static_cast<PoolMaps *>(maps), *kv) ? D3_OK : D3_ECUDA;
}

int32_t d3_page_plan(const d3_page_plan_args *a, void *cuda_stream) {
  if (!a || a->struct_size != sizeof(d3_page_plan_args)) return D3_EINVAL;
  if (a->n_requests < 1 || a->n_requests > D3_MAX_REQUESTS || !page_size_ok(a->page_size)) return D3_EINVAL;
  if (a->n_pages < 1 || a->table_width < 1 || a->max_tokens < 1 || a->table_stride < a->table_width) return D3_EINVAL;
  if (a->table_stride > ((int64_t)1 << 40) ||
      (int64_t)a->table_width * a->page_size > 0x7fffffff - 1024)   // lengths and positions fit 32 bits
    return D3_EINVAL;
  if (!int_span_ok(a->cached_dev, 4) || !int_span_ok(a->new_tokens_dev, 4) || !int_span_ok(a->table_dev, 4) ||
      !int_span_ok(a->free_dev, 4) || !int_span_ok(a->n_free_dev, 4) || !int_span_ok(a->cached_out_dev, 4) ||
      !int_span_ok(a->n_free_out_dev, 4) || !int_span_ok(a->first_dev, 4) || !int_span_ok(a->slots_dev, 16) ||
      !int_span_ok(a->row_dev, 16) || !int_span_ok(a->context_dev, 16) || ((uintptr_t)a->status_dev & 3))
    return D3_EINVAL;
  const size_t R4 = (size_t)a->n_requests * 4, T4 = (size_t)a->max_tokens * 4;
  const Span spans[11] = {{(uintptr_t)a->cached_dev, R4, false}, {(uintptr_t)a->cached_out_dev, R4, true},
                          {(uintptr_t)a->n_free_dev, 4, false}, {(uintptr_t)a->n_free_out_dev, 4, true},
                          {(uintptr_t)a->new_tokens_dev, R4, false}, {(uintptr_t)a->free_dev, (size_t)a->n_pages * 4, true},
                          {(uintptr_t)a->first_dev, R4 + 4, true}, {(uintptr_t)a->slots_dev, 2 * T4, true},
                          {(uintptr_t)a->row_dev, T4, true}, {(uintptr_t)a->context_dev, T4, true}, {(uintptr_t)a->status_dev, 4, true}};
  if (!plan_apart(spans, (uintptr_t)a->table_dev, a->n_requests, (size_t)a->table_width * 4, (size_t)a->table_stride * 4)) return D3_EINVAL;
  PlanArgs p;
  p.R = a->n_requests; p.page_shift = log2_of(a->page_size); p.n_pages = a->n_pages; p.width = a->table_width;
  p.T = a->max_tokens; p.table_stride = a->table_stride;
  p.cached = a->cached_dev; p.added = a->new_tokens_dev; p.table = a->table_dev; p.free_pages = a->free_dev;
  p.n_free = a->n_free_dev; p.cached_out = a->cached_out_dev; p.n_free_out = a->n_free_out_dev; p.first = a->first_dev;
  p.slots = reinterpret_cast<long long *>(a->slots_dev); p.row = a->row_dev; p.context = a->context_dev; p.status = a->status_dev;
  const size_t smem = ((size_t)4 * a->n_requests + 3) * sizeof(int);
  // As many CTAs as there are entries for, up to one per SM (192 prompts of 129..2048 tokens, 209,000 in all: 21.3 us as
  // eight CTAs, 6.1 as 148); few tokens are one small CTA's.
  const bool in_place = a->cached_out_dev == a->cached_dev || a->n_free_out_dev == a->n_free_dev;
  const int threads = a->n_requests <= 128 && a->max_tokens <= 512 ? 128 : a->n_requests > 1024 ? 1024 : 256;
  const long long entries = ((long long)a->max_tokens + 3) / 4 + (a->max_tokens > 512 ? a->n_pages / 4 : 0);
  long long ctas = (entries + threads - 1) / threads;
  if (ctas > 148) ctas = 148;
  const bool twice = in_place && ctas > 1;
  p.maps = 1;
  p.lengths = twice ? 0 : 1;
  // sums of at most 4096 entries of at most 2^18 stay within 32 bits
  const bool narrow = a->max_tokens <= (1 << 18) && a->n_pages <= (1 << 18) && a->table_width <= (1 << 18);
  void (*kernel)(PlanArgs) = narrow ? k_page_plan<int> : k_page_plan<long long>;
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return D3_ECUDA;
  static std::atomic<bool> ready[2][64];   // the shared-memory attribute is per device; setting it twice is harmless
  if (!ready[narrow][dev].load(std::memory_order_acquire)) {
    if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (4 * D3_MAX_REQUESTS + 4) * (int)sizeof(int)) !=
        cudaSuccess)
      return D3_ECUDA;
    ready[narrow][dev].store(true, std::memory_order_release);
  }
  cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
  if (launch_pdl(kernel, dim3((unsigned)ctas), dim3((unsigned)threads), smem, st, p) != cudaSuccess) return D3_ECUDA;
  if (twice) {
    p.maps = 0;
    p.lengths = 1;
    if (launch_pdl(kernel, dim3(1), dim3((unsigned)threads), smem, st, p) != cudaSuccess) return D3_ECUDA;
  }
  return D3_OK;
}

int32_t d3_paged_append(const d3_paged_kv *kv, const d3_paged_append_args *a, void *cuda_stream) {
  if (!kv_ok(kv, true) || !a || a->struct_size != sizeof(d3_paged_append_args)) return D3_EINVAL;
  if (!types_ok(a->dtype, kv->dtype) || a->n_tokens < 0) return D3_EINVAL;
  const int xs = bytes_of(a->dtype), dh = kv->head_dim;
  if (!a->k_dev || !a->v_dev || !aligned16(a->k_dev) || !aligned16(a->v_dev) || !a->slots_dev ||
      ((uintptr_t)a->slots_dev & 7) || ((uintptr_t)a->status_dev & 3))
    return D3_EINVAL;
  if (!stride_ok(a->k_token_stride, xs, 0) || !stride_ok(a->k_head_stride, xs, 0) || !stride_ok(a->v_token_stride, xs, 0) ||
      !stride_ok(a->v_head_stride, xs, 0))
    return D3_EINVAL;
  if (!rows_apart(dh, kv->n_pages, kv->page_stride, kv->n_kv_heads, kv->head_stride, kv->page_size, kv->token_stride)) return D3_EINVAL;
  if (a->rope_dev) {
    if (!aligned16(a->rope_dev) || a->rope_len < 1 || !a->context_dev || ((uintptr_t)a->context_dev & 3)) return D3_EINVAL;
  }
  if (a->q_dev) {
    if (!a->rope_dev || a->n_q_heads < 1 || a->n_q_heads > 65535 || !a->q_out_dev || !aligned16(a->q_dev) || !aligned16(a->q_out_dev) ||
        !stride_ok(a->q_token_stride, xs, 0) || !stride_ok(a->q_head_stride, xs, 0) ||
        !stride_ok(a->q_out_token_stride, xs, dh) || !stride_ok(a->q_out_head_stride, xs, dh) ||
        !rows_apart(dh, a->n_tokens, a->q_out_token_stride, a->n_q_heads, a->q_out_head_stride))
      return D3_EINVAL;
  }
  if (a->n_tokens == 0) return D3_OK;
  const int es = bytes_of(kv->dtype);
  if (rows_meet(dh, ((intptr_t)kv->v_dev - (intptr_t)kv->k_dev) / es, kv->n_pages, kv->page_stride, kv->n_kv_heads, kv->head_stride, kv->page_size,
                kv->token_stride))
    return D3_EINVAL;
  // q_out may be q itself, or lie beside it
  if (a->q_dev && a->q_dev != a->q_out_dev && (a->n_tokens == 1 || a->q_token_stride == a->q_out_token_stride) &&
      (a->n_q_heads == 1 || a->q_head_stride == a->q_out_head_stride) &&
      rows_meet(dh, ((intptr_t)a->q_out_dev - (intptr_t)a->q_dev) / xs, a->n_tokens, a->q_out_token_stride, a->n_q_heads, a->q_out_head_stride))
    return D3_EINVAL;
  AppendArgs p;
  memset(&p, 0, sizeof(p));
  p.n_tokens = a->n_tokens; p.rope_len = a->rope_len;
  p.slots = reinterpret_cast<const long long *>(a->slots_dev); p.context = a->context_dev; p.rope = a->rope_dev; p.status = a->status_dev;
  p.kv = pool_of(*kv);
  const int rotate = a->rope_dev ? 1 : 0;
  if (a->q_dev) {
    AppendPart &q = p.part[0];
    q.src = a->q_dev; q.dst = a->q_out_dev; q.heads = a->n_q_heads; q.rotate = rotate;
    q.st = a->q_token_stride; q.sh = a->q_head_stride; q.dt = a->q_out_token_stride; q.dh = a->q_out_head_stride;
  }
  for (int i = 1; i < 3; ++i) {
    AppendPart &x = p.part[i];
    x.src = i == 1 ? a->k_dev : a->v_dev; x.dst = i == 1 ? kv->k_dev : kv->v_dev;
    x.st = i == 1 ? a->k_token_stride : a->v_token_stride; x.sh = i == 1 ? a->k_head_stride : a->v_head_stride;
    x.dh = kv->head_stride; x.scale = i == 1 ? kv->k_scale_dev : kv->v_scale_dev;
    x.heads = kv->n_kv_heads; x.rotate = i == 1 ? rotate : 0;
  }
  cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
  bool fits;
  if (kv->dtype == D3_BF16) {
    fits = a->dtype == D3_BF16 ? launch_append<bf16, bf16>(p, dh, st) : launch_append<float, bf16>(p, dh, st);
  } else if (kv->dtype == D3_FP16) {
    fits = launch_append<__half, __half>(p, dh, st);
  } else {
    fits = a->dtype == D3_BF16 ? launch_append<bf16, __nv_fp8_e4m3>(p, dh, st) : launch_append<__half, __nv_fp8_e4m3>(p, dh, st);
  }
  if (!fits) return D3_EINVAL;
  return cudaGetLastError() == cudaSuccess ? D3_OK : D3_ECUDA;
}

int32_t d3_rope_table(int32_t n_positions, int32_t head_dim, float rope_base, float *table_dev, void *cuda_stream) {
  if (n_positions < 1 || (head_dim != 32 && head_dim != 64 && head_dim != 128) || !(rope_base > 0.f) || isinf(rope_base) ||
      !table_dev || !aligned16(table_dev) || (int64_t)n_positions * (head_dim / 2) > 0x7fffff00)
    return D3_EINVAL;
  launch_rope_table(reinterpret_cast<float2 *>(table_dev), n_positions, head_dim, rope_base, static_cast<cudaStream_t>(cuda_stream));
  return cudaGetLastError() == cudaSuccess ? D3_OK : D3_ECUDA;
}

int32_t d3_paged_attention_workspace(const d3_paged_kv *kv, int32_t n_q_heads, size_t *bytes) {
  if (!kv_ok(kv, false) || !bytes || n_q_heads < 1 || n_q_heads % kv->n_kv_heads) return D3_EINVAL;
  *bytes = attn_workspace(kv->head_dim).total;
  return D3_OK;
}

int32_t d3_paged_set_wait_ns(uint64_t ns) {
  if (ns == 0) return D3_EINVAL;
  attention_wait_ns.store(ns, std::memory_order_relaxed);
  return D3_OK;
}

int32_t d3_paged_stall_next(int32_t what) {
  if (what != 0 && what != D3_STALL_COPIES && what != D3_STALL_SUMS) return D3_EINVAL;
  attention_stall_next.store(what, std::memory_order_relaxed);
  return D3_OK;
}

int32_t d3_paged_attention(const d3_paged_kv *kv, const d3_paged_attention_args *a, void *cuda_stream) {
  if (!kv_ok(kv, true) || !a || a->struct_size != sizeof(d3_paged_attention_args)) return D3_EINVAL;
  if (!types_ok(a->dtype, kv->dtype)) return D3_EINVAL;
  const int xs = bytes_of(a->dtype), dh = kv->head_dim;
  if (a->n_rows < 0 || a->n_rows > 65535 || a->n_q_heads < 1 || a->n_q_heads % kv->n_kv_heads || a->n_q_heads > 65535) return D3_EINVAL;
  if (a->table_rows < 1 || a->table_width < 1 || a->table_stride < a->table_width || a->table_stride > ((int64_t)1 << 40) ||
      (int64_t)a->table_width * kv->page_size > 0x7fffffff - 1024)
    return D3_EINVAL;
  if (!a->rows_dev && a->table_rows < a->n_rows) return D3_EINVAL;
  // a CTA counts its units in 32 bits (far beyond what any pool holds; rows may share pages)
  if ((double)a->n_rows * ((double)a->table_width * kv->page_size / 64 + 1) * a->n_q_heads > 1.0e11) return D3_EINVAL;
  if (!isfinite(a->scale)) return D3_EINVAL;
  if (!a->q_dev || !a->out_dev || !aligned16(a->q_dev) || ((uintptr_t)a->out_dev & (xs - 1)) || ((uintptr_t)a->lse_dev & 3) ||
      !a->table_dev || ((uintptr_t)a->table_dev & 3) || !a->context_dev || ((uintptr_t)a->context_dev & 3) ||
      ((uintptr_t)a->rows_dev & 3) || ((uintptr_t)a->status_dev & 3))
    return D3_EINVAL;
  if (!stride_ok(a->q_row_stride, xs, 0) || !stride_ok(a->q_head_stride, xs, 0)) return D3_EINVAL;
  if (a->out_row_stride < dh || a->out_head_stride < dh || a->out_row_stride > ((int64_t)1 << 38) || a->out_head_stride > ((int64_t)1 << 38) ||
      !rows_apart(dh, a->n_rows, a->out_row_stride, a->n_q_heads, a->out_head_stride))
    return D3_EINVAL;
  const AttnWorkspace w = attn_workspace(dh);
  if (!a->workspace_dev || ((uintptr_t)a->workspace_dev & 255) || a->workspace_bytes < w.total) return D3_EINVAL;
  const PoolMaps *maps = static_cast<const PoolMaps *>(kv->maps);
  if (maps) {   // made for this pool?
    const d3_paged_kv &o = maps->of;
    if (((uintptr_t)maps & 63) || o.struct_size != kv->struct_size || o.dtype != kv->dtype || o.n_pages != kv->n_pages ||
        o.page_size != kv->page_size || o.n_kv_heads != kv->n_kv_heads || o.head_dim != kv->head_dim ||
        o.page_stride != kv->page_stride || o.head_stride != kv->head_stride || o.token_stride != kv->token_stride ||
        o.k_dev != kv->k_dev || o.v_dev != kv->v_dev)
      return D3_EINVAL;
  }
  if (a->n_rows == 0) return D3_OK;
  PoolMaps fresh;
  if (!maps) {
    if (!encode_pool_maps(&fresh, *kv)) return D3_ECUDA;
    maps = &fresh;
  }
  PagedAttnArgs p;
  memset(&p, 0, sizeof(p));
  p.n_rows = a->n_rows; p.hq = a->n_q_heads; p.hkv = kv->n_kv_heads; p.group = a->n_q_heads / kv->n_kv_heads;
  // Query heads that share one reading of K and V: up to 8, and up to 16 where 8 rows of the score tile
  // would not do (16-bit queries; fp32 ones use those rows for their third term).
  const int most = a->dtype != D3_FP32 && p.group > 8 ? 16 : 8;
  p.tiles_per_head = (p.group + most - 1) / most;
  p.heads_per_tile = (p.group + p.tiles_per_head - 1) / p.tiles_per_head;
  p.table_rows = a->table_rows; p.table_width = a->table_width; p.page_shift = log2_of(kv->page_size); p.n_pages = kv->n_pages;
  p.table_stride = a->table_stride; p.q_row_stride = a->q_row_stride; p.q_head_stride = a->q_head_stride;
  p.out_row_stride = a->out_row_stride; p.out_head_stride = a->out_head_stride;
  p.scale = a->scale; p.q = a->q_dev; p.out = a->out_dev; p.lse = a->lse_dev;
  p.table = a->table_dev; p.context = a->context_dev; p.rows = a->rows_dev;
  p.k_scale = kv->k_scale_dev; p.v_scale = kv->v_scale_dev;
  char *ws = static_cast<char *>(a->workspace_dev);
  p.part_o = reinterpret_cast<float *>(ws + w.part_o); p.part_ml = reinterpret_cast<float *>(ws + w.part_ml);
  p.join = reinterpret_cast<int4 *>(ws + w.join);
  p.status = a->status_dev;
  p.wait_ns = attention_wait_ns.load(std::memory_order_relaxed);
  p.stall = attention_stall_next.load(std::memory_order_relaxed) ? attention_stall_next.exchange(0, std::memory_order_relaxed) : 0;
  cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
  const int rc = dh == 128 ? launch_paged_attention_128(*maps, p, a->dtype, st)
                 : dh == 64 ? launch_paged_attention_64(*maps, p, a->dtype, st)
                            : launch_paged_attention_32(*maps, p, a->dtype, st);
  const cudaError_t err = cudaGetLastError();   // (asked for whatever the launch said: no error is left for the next call)
  return rc == 0 && err == cudaSuccess ? D3_OK : D3_ECUDA;
}

}  // extern "C"
