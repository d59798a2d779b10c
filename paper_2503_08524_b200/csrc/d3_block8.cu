// 8-bit block operators: residual sum + RMSNorm + quantising, weights to 8 bits, and the C ABI of the products.
#include <math.h>

#include <atomic>

#include "d3_block8.cuh"

namespace d3 {

namespace {

// ------------------------------------------------------------------ norm
struct NormArgs {
  long long n_rows;
  int dim, x_dtype, add_dtype, gain_dtype, out_dtype;
  float eps;
  const void *x, *add, *gain;
  void *total, *out;
  float *scale;
  long long x_stride, add_stride, total_stride, out_stride, scale_stride;
};

// A thread of the kernels below has K = 8 or 16 numbers of a block of 128, in pieces of E = 4 or 8 that are 16 bytes of x, so that
// neighbouring threads' pieces lie side by side; the 128 / K threads of the block find its largest by shuffles.  Many rows are
// bound by the memory, if no more than a few instructions are spent on a number: with types told apart at run time, 8 numbers a
// thread and two divisions each, 8-bit rows of 4097 x 11008 took 44 us (now 25; 23 with quotients by a reciprocal of 2^-22,
// which gave some numbers beside a tie the other code).  Few rows are bound by the launch.
template <int kType, int K>
struct Piece {
  static constexpr int E = kType == D3_FP32 ? 4 : 8, kGroups = K / E, kLanes = 128 / K;
  // first number of group j of thread t of a row
  static __device__ __forceinline__ int at(int t, int j) { return t / kLanes * 128 + j * (kLanes * E) + t % kLanes * E; }
};
// E numbers (16-byte aligned, or 8 where four 16-bit ones are asked for)
template <int kType, int E>
__device__ __forceinline__ void read_some(const char *p, float *v) {
  if constexpr (E == 8) {
    float u[8];
    load8(p, 0, kType, u);
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = u[j];
  } else if constexpr (kType == D3_FP32) {
    const float4 u = *reinterpret_cast<const float4 *>(p);
    v[0] = u.x; v[1] = u.y; v[2] = u.z; v[3] = u.w;
  } else {
    const uint2 u = *reinterpret_cast<const uint2 *>(p);
    if (kType == D3_BF16) {
      v[0] = __uint_as_float(u.x << 16); v[1] = __uint_as_float(u.x & 0xffff0000u); v[2] = __uint_as_float(u.y << 16); v[3] = __uint_as_float(u.y & 0xffff0000u);
    } else {
      v[0] = half_lo(u.x); v[1] = half_hi(u.x); v[2] = half_lo(u.y); v[3] = half_hi(u.y);
    }
  }
}
template <int E>
__device__ __forceinline__ void write_some(char *p, int dtype, const float *v) {
#pragma unroll
  for (int j = 0; j < E; j += 4) {
    if (dtype == D3_FP32) *reinterpret_cast<float4 *>(p + 4 * j) = make_float4(v[j], v[j + 1], v[j + 2], v[j + 3]);
    else if (E == 4) *reinterpret_cast<uint2 *>(p) = make_uint2(pack2(v[0], v[1], dtype), pack2(v[2], v[3], dtype));
  }
  if (E == 8 && dtype != D3_FP32)
    *reinterpret_cast<uint4 *>(p) = make_uint4(pack2(v[0], v[1], dtype), pack2(v[2], v[3], dtype), pack2(v[4], v[5], dtype), pack2(v[6], v[7], dtype));
}
// a thread's numbers of one of its blocks, zeros behind the end of the row
template <int kType, int K, int kOf>
__device__ __forceinline__ void read_row(const char *row, int t, int dim, float (&v)[K]) {
  using P = Piece<kOf, K>;                      // (the pieces are those of x, whatever is read)
  constexpr int kSize = kType == D3_FP32 ? 4 : 2;
#pragma unroll
  for (int j = 0; j < P::kGroups; ++j) {
    const int at = P::at(t, j);
    if (at < dim) {
      read_some<kType, P::E>(row + at * kSize, v + j * P::E);
    } else {
#pragma unroll
      for (int e = 0; e < P::E; ++e) v[j * P::E + e] = 0.f;
    }
  }
}
template <int K, int kOf>
__device__ __forceinline__ void write_row(char *row, int t, int dim, int dtype, const float (&v)[K]) {
  using P = Piece<kOf, K>;
  const int size = dtype == D3_FP32 ? 4 : 2;
#pragma unroll
  for (int j = 0; j < P::kGroups; ++j) {
    const int at = P::at(t, j);
    if (at < dim) write_some<P::E>(row + at * size, dtype, v + j * P::E);
  }
}
// the same in 8 bits with the block's scale
template <int K, int kOf, bool kUp>
__device__ __forceinline__ void write_codes(char *row, int t, int dim, const float (&v)[K], const BlockScale &b) {
  using P = Piece<kOf, K>;
  constexpr float up = kUp ? kLift : 1.f;
#pragma unroll
  for (int j = 0; j < P::kGroups; ++j) {
    const int at = P::at(t, j);
    if (at < dim) {
      const float *u = v + j * P::E;
      const uint32_t lo = quantize4(u[0] * up, u[1] * up, u[2] * up, u[3] * up, b);
      if constexpr (P::E == 4) *reinterpret_cast<uint32_t *>(row + at) = lo;
      else *reinterpret_cast<uint2 *>(row + at) = make_uint2(lo, quantize4(u[4] * up, u[5] * up, u[6] * up, u[7] * up, b));
    }
  }
}
// (all threads of the warp take part.  Blocks of the smallest numbers have code of their own: with their factor in front of the one code
// fp32 rows of 4097 x 8192 took 29.4 us where this takes 26.2.)
template <int K, int kOf>
__device__ __forceinline__ void write_row_e4m3(char *row, float *scales, int t, int dim, const float (&v)[K]) {
  using P = Piece<kOf, K>;
  float top = 0.f;
#pragma unroll
  for (int j = 0; j < K; ++j) top = max_nan(top, fabsf(v[j]));
#pragma unroll
  for (int o = P::kLanes / 2; o > 0; o >>= 1) top = max_nan(top, __shfl_xor_sync(0xffffffffu, top, o));
  BlockScale b = block_scale(top);
  if (t % P::kLanes == 0 && t / P::kLanes * 128 < dim) scales[t / P::kLanes] = b.scale;
  if (__builtin_expect(lift(b), 0)) write_codes<K, kOf, true>(row, t, dim, v, b);
  else write_codes<K, kOf, false>(row, t, dim, v, b);
}

// A row is held in registers by the threads of a CTA, V times K numbers each; kWarp puts rows side by side, a warp each.
// Everything is read before anything is written, so that out and total may lie on x and add.  kAdd: the type of add, -1 for none.
template <int V, int K, bool kWarp, int kType, int kAdd>
__global__ void __launch_bounds__(1024) k_add_norm(const __grid_constant__ NormArgs a) {
  __shared__ float s_sum[32];
  constexpr int kSize = kType == D3_FP32 ? 4 : 2, kAddSize = kAdd == D3_FP32 ? 4 : 2;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int T = kWarp ? 32 : blockDim.x, t = kWarp ? lane : threadIdx.x;
  const long long row = kWarp ? (long long)blockIdx.x * (blockDim.x >> 5) + warp : blockIdx.x;
  pdl_wait();
  pdl_trigger();
  if (kWarp && row >= a.n_rows) return;
  float v[V][K];
  const char *x = static_cast<const char *>(a.x) + row * a.x_stride * kSize;
#pragma unroll
  for (int i = 0; i < V; ++i) read_row<kType, K, kType>(x, i * T + t, a.dim, v[i]);
  if constexpr (kAdd >= 0) {
    const char *add = static_cast<const char *>(a.add) + row * a.add_stride * kAddSize;
#pragma unroll
    for (int i = 0; i < V; ++i) {
      float u[K];
      read_row<kAdd, K, kType>(add, i * T + t, a.dim, u);
#pragma unroll
      for (int j = 0; j < K; ++j) v[i][j] += u[j];
    }
  }
  float r = 0.f;
  if (a.gain) {
    float sum = 0.f;
#pragma unroll
    for (int i = 0; i < V; ++i) {
      float part = 0.f;
#pragma unroll
      for (int j = 0; j < K; ++j) part = fmaf(v[i][j], v[i][j], part);
      sum += part;
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
    if (!kWarp) {
      if (lane == 0) s_sum[warp] = sum;
      __syncthreads();
      sum = lane < T / 32 ? s_sum[lane] : 0.f;
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
    }
    r = 1.f / sqrtf(sum / (float)a.dim + a.eps);
  }
  if (kAdd >= 0 && a.total) {
    char *total = static_cast<char *>(a.total) + row * a.total_stride * kAddSize;
#pragma unroll
    for (int i = 0; i < V; ++i) write_row<K, kType>(total, i * T + t, a.dim, kAdd, v[i]);
  }
  char *out = static_cast<char *>(a.out) + row * a.out_stride * (a.out_dtype == D3_E4M3 ? 1 : a.out_dtype == D3_FP32 ? 4 : 2);
  float *scales = a.scale + row * a.scale_stride;
#pragma unroll
  for (int i = 0; i < V; ++i) {
    if (a.gain) {
      float g[K];
      const char *gain = static_cast<const char *>(a.gain);
      if (a.gain_dtype == D3_BF16) read_row<D3_BF16, K, kType>(gain, i * T + t, a.dim, g);
      else if (a.gain_dtype == D3_FP16) read_row<D3_FP16, K, kType>(gain, i * T + t, a.dim, g);
      else read_row<D3_FP32, K, kType>(gain, i * T + t, a.dim, g);
#pragma unroll
      for (int j = 0; j < K; ++j) v[i][j] = v[i][j] * r * g[j];
    }
    if (a.out_dtype == D3_E4M3) write_row_e4m3<K, kType>(out, scales, i * T + t, a.dim, v[i]);
    else write_row<K, kType>(out, i * T + t, a.dim, a.out_dtype, v[i]);
  }
}

// The 8 bits alone: blocks of 128 have nothing to do with one another, so they are dealt out whatever row they are in, kQuant
// to a thread (of 8 that share a block).
constexpr int kQuant = 2, kQuantThreads = 256, kQuantBlocks = kQuantThreads / 8;
template <int kType>
__global__ void __launch_bounds__(kQuantThreads) k_quantize(const __grid_constant__ NormArgs a) {
  constexpr int kSize = kType == D3_FP32 ? 4 : 2;
  const uint32_t wide = (uint32_t)(a.dim + 127) / 128;
  pdl_wait();
  pdl_trigger();
  // (fewer than 2^31 blocks)
  const uint32_t b = blockIdx.x * (uint32_t)(kQuant * kQuantBlocks) + threadIdx.x / 8;
  uint32_t row = b / wide, c = b - row * wide;
  float v[kQuant][16];
  uint32_t rows[kQuant];
  int ts[kQuant];
#pragma unroll
  for (int i = 0; i < kQuant; ++i) {
    rows[i] = row;
    ts[i] = (int)(8 * c + threadIdx.x % 8);
    read_row<kType, 16, kType>(static_cast<const char *>(a.x) + row * a.x_stride * kSize, ts[i], row < a.n_rows ? a.dim : 0, v[i]);
    c += kQuantBlocks;
    while (c >= wide) { c -= wide; ++row; }
  }
#pragma unroll
  for (int i = 0; i < kQuant; ++i)
    write_row_e4m3<16, kType>(static_cast<char *>(a.out) + rows[i] * a.out_stride, a.scale + rows[i] * a.scale_stride, ts[i], rows[i] < a.n_rows ? a.dim : 0, v[i]);
}

// threads of a row, V times K numbers each
inline int norm_threads(int dim, int v, int k) { return ((dim + 127) / 128 * (128 / k) + 32 * v - 1) / (32 * v) * 32; }
template <int V, int K, int kType, int kAdd>
cudaError_t launch_norm(const NormArgs &a, cudaStream_t st) {
  const int threads = norm_threads(a.dim, V, K);
  if constexpr (V == 1) {
    if (threads <= 32) {
      const int rows = a.n_rows < 148 * 4 ? 1 : 8;
      return launch_pdl(k_add_norm<V, K, true, kType, kAdd>, dim3((unsigned)((a.n_rows + rows - 1) / rows)), dim3(32 * rows), 0, st, a);
    }
  }
  return launch_pdl(k_add_norm<V, K, false, kType, kAdd>, dim3((unsigned)a.n_rows), dim3(threads), 0, st, a);
}
template <int kType, int kAdd>
cudaError_t launch_norm_k(const NormArgs &a, cudaStream_t st) {
  // (us with 8 / 16 numbers a thread: 4096 x 4096 in 16 bits 23.9 / 28.8, 32 x 5120 2.4 / 2.7, 8191 x 8192 130 / 128)
  // (64 numbers a thread do not fit into its registers: 250 x 65536 takes 65 us where 500 x 32768 takes 46)
  if (a.dim <= 8192) return launch_norm<1, 8, kType, kAdd>(a, st);
  if (a.dim <= 16384) return launch_norm<1, 16, kType, kAdd>(a, st);
  if (a.dim <= 32768) return launch_norm<2, 16, kType, kAdd>(a, st);
  return launch_norm<4, 16, kType, kAdd>(a, st);
}
template <int kType>
cudaError_t launch_norm_add(const NormArgs &a, cudaStream_t st) {
  if (!a.add) return launch_norm_k<kType, -1>(a, st);
  if (a.add_dtype == D3_FP32) return launch_norm_k<kType, D3_FP32>(a, st);
  return launch_norm_k<kType, kType>(a, st);
}

// ------------------------------------------------------------------ weights to 8 bits
struct QuantWeightArgs {
  const void *w;
  int dtype, n, k;
  long long stride, q_stride;
  unsigned char *q;
  float *scale;
};
// One block of 128 x 128 per CTA: thread t has 64 numbers of row t / 2, 8 at a time (k is a multiple of 16).  A warp's load
// takes 16 bytes from each of 32 lines, and L2 moves 530 MB where 151 are read and written: 12288 x 4096 bf16 takes 53 us, 44 % of the
// copy rate.  (A weight is brought to 8 bits once.)
__global__ void __launch_bounds__(256) k_quantize_weight(const __grid_constant__ QuantWeightArgs a) {
  __shared__ float s_top[8];
  pdl_wait();
  pdl_trigger();
  const int row = blockIdx.y * 128 + (threadIdx.x >> 1), k0 = blockIdx.x * 128 + (threadIdx.x & 1) * 64;
  float v[8][8];
  float top = 0.f;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    if (row < a.n && k0 + 8 * i < a.k) {
      if (a.stride % 8 == 0 && ((uintptr_t)a.w & 15u) == 0) {
        load8(a.w, row * a.stride + k0 + 8 * i, a.dtype, v[i]);
      } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) v[i][j] = load1(a.w, row * a.stride + k0 + 8 * i + j, a.dtype);
      }
#pragma unroll
      for (int j = 0; j < 8; ++j) top = max_nan(top, fabsf(v[i][j]));
    }
  }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) top = max_nan(top, __shfl_xor_sync(0xffffffffu, top, o));
  if ((threadIdx.x & 31) == 0) s_top[threadIdx.x >> 5] = top;
  __syncthreads();
#pragma unroll
  for (int i = 0; i < 8; ++i) top = max_nan(top, s_top[i]);
  BlockScale b = block_scale(top);
  if (threadIdx.x == 0) a.scale[(size_t)blockIdx.y * gridDim.x + blockIdx.x] = b.scale;
  const float up = lift(b) ? kLift : 1.f;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    if (row < a.n && k0 + 8 * i < a.k) {
      *reinterpret_cast<uint2 *>(a.q + row * a.q_stride + k0 + 8 * i) =
          make_uint2(quantize4(v[i][0] * up, v[i][1] * up, v[i][2] * up, v[i][3] * up, b), quantize4(v[i][4] * up, v[i][5] * up, v[i][6] * up, v[i][7] * up, b));
    }
  }
}

// ------------------------------------------------------------------ tensor maps
typedef CUresult (*EncodeTiledFn)(CUtensorMap *, CUtensorMapDataType, cuuint32_t, void *, const cuuint64_t *,
                                  const cuuint64_t *, const cuuint32_t *, const cuuint32_t *,
                                  CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion,
                                  CUtensorMapFloatOOBfill);
EncodeTiledFn rows_encoder() {
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

// the largest n_rows, n and k: whole tiles of 256 end within 32 bits
constexpr int kMostOfOne = 0x7fffff00;
bool weight_ok(const d3_weight8 *w) {
  return w && w->struct_size == sizeof(d3_weight8) && w->n >= 1 && w->n <= kMostOfOne && w->k >= 16 && w->k <= kMostOfOne && w->k % 16 == 0 &&
         w->row_stride >= w->k &&
         w->row_stride % 16 == 0 && w->row_stride <= ((int64_t)1 << 38) && w->q_dev && on_bytes(w->q_dev, 16) && w->scale_dev &&
         on_bytes(w->scale_dev, 4);
}
bool made_for(const Weight8Map *m, const d3_weight8 &w) {
  return m->of.n == w.n && m->of.k == w.k && m->of.row_stride == w.row_stride && m->of.q_dev == w.q_dev;
}
int64_t scale_blocks(int64_t v) { return (v + kScaleBlock - 1) / kScaleBlock; }

std::atomic<uint32_t> wait_tries{kWaitTries};
std::atomic<int> stall_next{0};

// Two kernels: one reads the weights for up to 128 rows at a time (true; as `plan` says), one multiplies 256 rows by 256 weight rows at the
// tensor cores' rate, if there are tiles enough for every pair of SMs.
bool choose(const Mm8Args &p, int mats, FewPlan &plan) { return plan_mm8_few(p, mats, plan) <= estimate_mm8_many(p, mats); }

// the checks and the launch that both products share
int32_t product(const d3_weight8 *const (&w)[2], const d3_matmul8_args *a, cudaStream_t st) {
  const int mats = w[1] ? 2 : 1;
  for (int i = 0; i < mats; ++i)
    if (!weight_ok(w[i])) return D3_EINVAL;
  if (mats == 2 && (w[0]->n != w[1]->n || w[0]->k != w[1]->k)) return D3_EINVAL;
  if (!a || a->struct_size != sizeof(d3_matmul8_args) || a->n_rows < 0 || a->n_rows > kMostOfOne) return D3_EINVAL;
  const bool eight = a->out_dtype == D3_E4M3;
  if (!wide_type(a->out_dtype) && !(eight && mats == 2)) return D3_EINVAL;
  const int n = w[0]->n, k = w[0]->k, es = type_bytes(a->out_dtype);
  const int64_t kb = scale_blocks(k), nb = scale_blocks(n);
  if (!a->a_dev || !on_bytes(a->a_dev, 16) || !a->a_scale_dev || !on_bytes(a->a_scale_dev, 4) || !a->out_dev || !on_bytes(a->out_dev, es))
    return D3_EINVAL;
  if (a->n_rows > 1 && (a->a_stride < k || a->a_stride % 16 || a->a_stride > ((int64_t)1 << 38) || a->a_scale_stride < kb ||
                        a->a_scale_stride > ((int64_t)1 << 38) || a->out_stride < n || a->out_stride > ((int64_t)1 << 38)))
    return D3_EINVAL;
  if (eight && (!a->scale_dev || !on_bytes(a->scale_dev, 4) ||
                (a->n_rows > 1 && (a->scale_stride < nb || a->scale_stride > ((int64_t)1 << 38)))))
    return D3_EINVAL;
  if (!eight && a->scale_dev) return D3_EINVAL;
  if (!on_bytes(a->status_dev, 4)) return D3_EINVAL;
  for (int i = 0; i < mats; ++i)
    if (w[i]->map && (((uintptr_t)w[i]->map & 63) || !made_for(static_cast<const Weight8Map *>(w[i]->map), *w[i]))) return D3_EINVAL;
  if (a->n_rows == 0) return D3_OK;
  const int64_t rows = a->n_rows;
  const RowSet out = {a->out_dev, rows, a->out_stride * es, (int64_t)n * es};
  const RowSet scale = {eight ? a->scale_dev : nullptr, rows, a->scale_stride * 4, nb * 4};
  const RowSet status = {a->status_dev, 1, 4, 4};
  RowSet read[6] = {{a->a_dev, rows, a->a_stride, k}, {a->a_scale_dev, rows, a->a_scale_stride * 4, kb * 4}};
  for (int i = 0; i < mats; ++i) {
    read[2 + 2 * i] = RowSet{w[i]->q_dev, n, w[i]->row_stride, k};
    read[3 + 2 * i] = RowSet{w[i]->scale_dev, 1, 0, nb * kb * 4};
  }
  for (int i = 0; i < 2 + 2 * mats; ++i)
    if (rows_common(out, read[i]) || rows_common(scale, read[i]) || rows_common(status, read[i])) return D3_EINVAL;
  if (rows_common(out, scale) || rows_common(out, status) || rows_common(scale, status)) return D3_EINVAL;
  if (!have_encoder8()) return D3_ECUDA;

  TMap fresh[2];
  const TMap *map[2] = {nullptr, nullptr};
  for (int i = 0; i < mats; ++i) {
    if (w[i]->map) map[i] = &static_cast<const Weight8Map *>(w[i]->map)->map;
    else if (encode_rows8(&fresh[i], w[i]->q_dev, n, k, w[i]->row_stride, kScaleBlock)) map[i] = &fresh[i];
    else return D3_ECUDA;
  }
  Mm8Args p;
  memset(&p, 0, sizeof(p));
  p.n_rows = a->n_rows; p.n = n; p.k = k; p.n_kb = (int)kb;
  p.a_scale = a->a_scale_dev; p.a_scale_stride = rows > 1 ? a->a_scale_stride : kb;
  p.w_scale[0] = w[0]->scale_dev; p.w_scale[1] = mats == 2 ? w[1]->scale_dev : nullptr;
  p.out = a->out_dev; p.out_stride = rows > 1 ? a->out_stride : n; p.out_dtype = a->out_dtype;
  p.scale = a->scale_dev; p.scale_stride = rows > 1 ? a->scale_stride : nb;
  p.status = a->status_dev;
  p.wait_tries = wait_tries.load(std::memory_order_relaxed);
  p.stall = stall_next.exchange(0, std::memory_order_relaxed);
  const int64_t a_stride = rows > 1 ? a->a_stride : (int64_t)k;
  FewPlan plan;
  const bool few = choose(p, mats, plan);
  const cudaError_t e = few ? launch_mm8_few(*map[0], map[1], a->a_dev, a_stride, p, plan, st)
                            : launch_mm8_many(*map[0], map[1], a->a_dev, a_stride, p, st);
  return e == cudaSuccess ? D3_OK : D3_ECUDA;
}

}  // namespace

bool have_encoder8() { return rows_encoder() != nullptr; }

bool encode_rows8(TMap *out, const void *base, int rows, int k, int64_t stride, int box_rows) {
  EncodeTiledFn fn = rows_encoder();
  if (!fn) return false;
  cuuint64_t dims[2] = {(cuuint64_t)k, (cuuint64_t)rows}, strides[1] = {(cuuint64_t)stride};
  cuuint32_t box[2] = {(cuuint32_t)kScaleBlock, (cuuint32_t)box_rows}, estr[2] = {1, 1};
  return fn(reinterpret_cast<CUtensorMap *>(out), CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, const_cast<void *>(base), dims, strides, box, estr,
            CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
            CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

bool encode_results8(TMap *out, void *base, int rows, int n, int dtype, int64_t stride) {
  EncodeTiledFn fn = rows_encoder();
  if (!fn) return false;
  const int es = type_bytes(dtype);
  cuuint64_t dims[2] = {(cuuint64_t)n, (cuuint64_t)rows}, strides[1] = {(cuuint64_t)(stride * es)};
  cuuint32_t box[2] = {(cuuint32_t)(128 / es), 128}, estr[2] = {1, 1};
  const CUtensorMapDataType type = dtype == D3_FP32 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT32 : dtype == D3_BF16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16
                                   : dtype == D3_FP16 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT16 : CU_TENSOR_MAP_DATA_TYPE_UINT8;
  return fn(reinterpret_cast<CUtensorMap *>(out), type, 2, base, dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
            CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

}  // namespace d3

using namespace d3;

extern "C" {

int32_t d3_add_norm(const d3_add_norm_args *a, void *cuda_stream) {
  if (!a || a->struct_size != sizeof(d3_add_norm_args) || a->n_rows < 0) return D3_EINVAL;
  if (a->dim < 8 || a->dim > 65536 || a->dim % 8 || !wide_type(a->x_dtype)) return D3_EINVAL;
  const bool eight = a->out_dtype == D3_E4M3;
  if (!eight && !wide_type(a->out_dtype)) return D3_EINVAL;
  if (!(a->eps >= 0.f) || isinf(a->eps)) return D3_EINVAL;
  const int xs = type_bytes(a->x_dtype), os = type_bytes(a->out_dtype), as = type_bytes(a->add_dtype);
  const int64_t rows = a->n_rows, dim = a->dim, nb = scale_blocks(dim), most = (int64_t)1 << 38;
  auto stride_ok = [&](int64_t s, int64_t least, int bytes, int unit) {
    return rows <= 1 || (s >= least && s <= most && s * bytes % unit == 0);
  };
  if (!a->x_dev || !on_bytes(a->x_dev, 16) || !stride_ok(a->x_stride, 0, xs, 16)) return D3_EINVAL;
  if (!a->out_dev || !on_bytes(a->out_dev, eight ? 8 : 16) || !stride_ok(a->out_stride, dim, os, eight ? 8 : 16)) return D3_EINVAL;
  if (a->add_dev) {
    if (a->add_dtype != a->x_dtype && a->add_dtype != D3_FP32) return D3_EINVAL;
    if (!on_bytes(a->add_dev, 16) || !stride_ok(a->add_stride, 0, as, 16)) return D3_EINVAL;
    if (a->total_dev && (!on_bytes(a->total_dev, 16) || !stride_ok(a->total_stride, dim, as, 16))) return D3_EINVAL;
  } else if (a->total_dev) {
    return D3_EINVAL;
  }
  if (a->gain_dev && (!wide_type(a->gain_dtype) || !on_bytes(a->gain_dev, 16))) return D3_EINVAL;
  if (eight ? (!a->scale_dev || !on_bytes(a->scale_dev, 4) || !stride_ok(a->scale_stride, nb, 4, 4)) : a->scale_dev != nullptr) return D3_EINVAL;
  if (rows == 0) return D3_OK;
  const RowSet x = {a->x_dev, rows, a->x_stride * xs, dim * xs}, add = {a->add_dev, rows, a->add_stride * as, dim * as},
               total = {a->total_dev, rows, a->total_stride * as, dim * as}, out = {a->out_dev, rows, a->out_stride * os, dim * os},
               gain = {a->gain_dev, 1, 0, dim * type_bytes(a->gain_dtype)}, scale = {a->scale_dev, rows, a->scale_stride * 4, nb * 4};
  // a row is read whole before any of it is written: out on x, total on add or x, number by number
  const bool out_on_x = a->out_dtype == a->x_dtype && same_rows(out, x), total_on_add = same_rows(total, add),
             total_on_x = a->add_dtype == a->x_dtype && same_rows(total, x);
  if ((rows_common(out, x) && !(out_on_x && !(rows > 1 && !rows_distinct(x)))) || (rows_common(total, add) && !(total_on_add && rows_distinct(add))) ||
      (rows_common(total, x) && !(total_on_x && rows_distinct(x))) || rows_common(out, add) || rows_common(out, total) || rows_common(out, gain) ||
      rows_common(total, gain) || rows_common(scale, x) || rows_common(scale, add) || rows_common(scale, total) || rows_common(scale, out) ||
      rows_common(scale, gain))
    return D3_EINVAL;
  NormArgs p;
  p.n_rows = rows; p.dim = a->dim; p.x_dtype = a->x_dtype; p.add_dtype = a->add_dtype; p.gain_dtype = a->gain_dtype; p.out_dtype = a->out_dtype;
  p.eps = a->eps; p.x = a->x_dev; p.add = a->add_dev; p.gain = a->gain_dev; p.total = a->total_dev; p.out = a->out_dev; p.scale = a->scale_dev;
  p.x_stride = a->x_stride; p.add_stride = a->add_stride; p.total_stride = a->total_stride; p.out_stride = a->out_stride;
  p.scale_stride = a->scale_stride;
  cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
  cudaError_t e;
  const long long quant = (rows * nb + kQuant * kQuantBlocks - 1) / (kQuant * kQuantBlocks);
  if (eight && !a->add_dev && !a->gain_dev && quant * kQuant * kQuantBlocks <= 0x7fffffffll) {
    void (*kernel)(NormArgs) = a->x_dtype == D3_FP32 ? k_quantize<D3_FP32> : a->x_dtype == D3_BF16 ? k_quantize<D3_BF16> : k_quantize<D3_FP16>;
    e = launch_pdl(kernel, dim3((unsigned)quant), dim3(kQuantThreads), 0, st, p);
  } else {
    e = a->x_dtype == D3_FP32 ? launch_norm_add<D3_FP32>(p, st) : a->x_dtype == D3_BF16 ? launch_norm_add<D3_BF16>(p, st) : launch_norm_add<D3_FP16>(p, st);
  }
  return e == cudaSuccess ? D3_OK : D3_ECUDA;
}

int32_t d3_weight8_map(const d3_weight8 *w, void *map) {
  if (!weight_ok(w) || !map || ((uintptr_t)map & 63)) return D3_EINVAL;
  Weight8Map *m = static_cast<Weight8Map *>(map);
  if (!encode_rows8(&m->map, w->q_dev, w->n, w->k, w->row_stride, kScaleBlock)) return D3_ECUDA;
  m->of = *w;
  m->of.map = nullptr;
  m->of.scale_dev = nullptr;
  return D3_OK;
}

int32_t d3_quantize_weight(const void *w_dev, int32_t dtype, int64_t row_stride, const d3_weight8 *w8, void *cuda_stream) {
  if (!weight_ok(w8) || !wide_type(dtype) || !w_dev || !on_bytes(w_dev, type_bytes(dtype))) return D3_EINVAL;
  if (w8->n > 1 && (row_stride < w8->k || row_stride > ((int64_t)1 << 38))) return D3_EINVAL;
  const int64_t nb = scale_blocks(w8->n), kb = scale_blocks(w8->k), es = type_bytes(dtype);
  if (nb > 65535) return D3_EINVAL;
  const RowSet from = {w_dev, w8->n, row_stride * es, w8->k * es}, to = {w8->q_dev, w8->n, w8->row_stride, w8->k},
               scale = {w8->scale_dev, 1, 0, nb * kb * 4};
  if (rows_common(from, to) || rows_common(from, scale) || rows_common(to, scale)) return D3_EINVAL;
  QuantWeightArgs q;
  q.w = w_dev; q.dtype = dtype; q.n = w8->n; q.k = w8->k; q.stride = w8->n > 1 ? row_stride : 0; q.q_stride = w8->row_stride;
  q.q = static_cast<unsigned char *>(const_cast<void *>(w8->q_dev)); q.scale = const_cast<float *>(w8->scale_dev);
  return launch_pdl(k_quantize_weight, dim3((unsigned)kb, (unsigned)nb), dim3(256), 0, static_cast<cudaStream_t>(cuda_stream), q) == cudaSuccess
             ? D3_OK : D3_ECUDA;
}

int32_t d3_matmul8_set_wait_ns(uint64_t ns) {
  if (ns < 1) return D3_EINVAL;
  const uint64_t tries = ns / kTryNs + 1;
  wait_tries.store(tries < 0x7fffffffull ? (uint32_t)tries : 0x7fffffffu, std::memory_order_relaxed);
  return D3_OK;
}

int32_t d3_matmul8_stall_next(int32_t on) {
  if (on != 0 && on != 1) return D3_EINVAL;
  stall_next.store(on, std::memory_order_relaxed);
  return D3_OK;
}

int32_t d3_matmul8_plan(int32_t n_rows, int32_t n, int32_t k, int32_t gated, int32_t *plan) {
  if (n_rows < 1 || n_rows > kMostOfOne || n < 1 || n > kMostOfOne || k < 16 || k > kMostOfOne || k % 16 || gated < 0 || gated > 1 || !plan)
    return D3_EINVAL;
  Mm8Args p;
  memset(&p, 0, sizeof(p));
  p.n_rows = n_rows; p.n = n; p.k = k; p.n_kb = (int)scale_blocks(k);
  FewPlan few;
  const bool is_few = choose(p, gated ? 2 : 1, few);
  plan[0] = is_few ? few.rows : 256;
  plan[1] = is_few ? few.split : 1;
  return D3_OK;
}

int32_t d3_matmul8(const d3_weight8 *w, const d3_matmul8_args *a, void *cuda_stream) {
  return product({w, nullptr}, a, static_cast<cudaStream_t>(cuda_stream));
}

int32_t d3_gated_matmul8(const d3_weight8 *gate, const d3_weight8 *up, const d3_matmul8_args *a, void *cuda_stream) {
  if (!up) return D3_EINVAL;
  return product({gate, up}, a, static_cast<cudaStream_t>(cuda_stream));
}

}  // extern "C"
