// Constraints on logits: penalties for repeated tokens, biases, a grammar's mask, and the best token that is left.
//
// One pass over the logits, so many rows are bound by reading and writing them once and few by latency.  A row's vocabulary is cut
// between the CTAs of a cluster, and a CTA takes its part in slices that it has counters for in shared memory: it reads the
// row's history, counts the tokens that fall in the slice (whole numbers: the order of the atomics changes nothing), and
// then has everything it needs of a token at hand.  The history is read once a slice from L2, which is cheap beside the slice's logits.
// The best token is found on the way: per thread, per CTA, and between the CTAs through distributed shared memory.
#include <math.h>

#include <atomic>

#include "d3_block8.cuh"

namespace d3 {

namespace {

constexpr int kThreads = 256;
constexpr int kSlice = 8192;                 // tokens that a CTA has counters for
constexpr uint32_t kSeen = 0x80000000u;      // counter: the token is in the prompt; the bits below count it behind the prompt

struct LogitsArgs {
  int n_rows, vocab, n_history, n_bias, n_masks, dtype, split, per, wide;
  const void *logits;
  void *out;
  long long logits_stride, out_stride, history_stride, bias_stride, mask_stride;
  const int32_t *history, *lengths, *prompt;
  const float *repetition, *frequency, *presence;
  const int32_t *bias_ids;
  const float *bias;
  const int32_t *masks, *mask_of;
  int32_t *token, *status;
};

__device__ __forceinline__ void take(float &best, int &at, float v, int i) {
  if (v > best || (v == best && i < at)) { best = v; at = i; }
}
__device__ __forceinline__ float rounded(float v, int dtype) {
  if (dtype == D3_BF16) return __bfloat162float(__float2bfloat16_rn(v));
  if (dtype == D3_FP16) return __half2float(__float2half_rn(v));
  return v;
}

__global__ void __launch_bounds__(kThreads) k_constrain_logits(const __grid_constant__ LogitsArgs a) {
  extern __shared__ uint32_t s_count[];      // [slice], and behind it the biases' entries, if there are any
  __shared__ float s_best[kThreads / 32 + 1];
  __shared__ int s_at[kThreads / 32 + 1];
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int row = blockIdx.x / a.split, rank = blockIdx.x % a.split;
  const int v0 = min(a.vocab, rank * a.per), v1 = min(a.vocab, v0 + a.per);
  const int slice = min(a.per, kSlice);
  uint32_t *s_bias = s_count + slice;
  pdl_wait();
  pdl_trigger();

  bool bad = false;
  auto bounded = [&](const int32_t *p, int none) {   // an entry of lengths or prompt
    if (!p) return none;
    const int v = p[row];
    if (v < 0 || v > a.n_history) bad = true;
    return min(max(v, 0), a.n_history);
  };
  const int length = a.history ? bounded(a.lengths, a.n_history) : 0, prompt = a.history ? bounded(a.prompt, 0) : 0;
  const float rep = a.repetition ? a.repetition[row] : 1.f, freq = a.frequency ? a.frequency[row] : 0.f,
              pres = a.presence ? a.presence[row] : 0.f;
  const int32_t *mask = nullptr;
  if (a.masks) {
    const int m = a.mask_of[row];
    if (m >= a.n_masks) bad = true;
    else if (m >= 0) mask = a.masks + m * a.mask_stride;
  }
  const int32_t *history = a.history + row * a.history_stride, *ids = a.bias_ids + row * a.bias_stride;
  const float *bias = a.bias + row * a.bias_stride;
  float best = -INFINITY;
  int at = 0x7fffffff;

  for (int lo = v0; lo < v1; lo += slice) {
    const int hi = min(v1, lo + slice);
    if (a.history || a.bias_ids) {
      __syncthreads();
      for (int i = tid; i < (a.bias_ids ? 2 : 1) * slice; i += kThreads) s_count[i] = 0u;
      __syncthreads();
      for (int i = tid; i < length; i += kThreads) {
        const int id = history[i];
        if (id >= lo && id < hi) {
          if (i < prompt) atomicOr(&s_count[id - lo], kSeen);
          else atomicAdd(&s_count[id - lo], 1u);
        }
        bad |= id >= a.vocab;
      }
      for (int i = tid; i < a.n_bias; i += kThreads) {
        const int id = ids[i];
        if (id >= lo && id < hi) atomicMax(&s_bias[id - lo], (uint32_t)i + 1u);
        bad |= id >= a.vocab;
      }
      __syncthreads();
    }
    for (int i = lo + 4 * tid; i < hi; i += 4 * kThreads) {   // (lo is a multiple of 4: four tokens share a word of the mask)
      const int n = min(4, hi - i);
      float z[4];
      const long long from = row * a.logits_stride + i, to = row * a.out_stride + i;
      if (a.wide && n == 4) {
        if (a.dtype == D3_FP32) {
          const float4 v = *reinterpret_cast<const float4 *>(static_cast<const float *>(a.logits) + from);
          z[0] = v.x; z[1] = v.y; z[2] = v.z; z[3] = v.w;
        } else {
          const uint2 v = *reinterpret_cast<const uint2 *>(static_cast<const char *>(a.logits) + 2 * from);
          if (a.dtype == D3_BF16) {
            z[0] = __uint_as_float(v.x << 16); z[1] = __uint_as_float(v.x & 0xffff0000u);
            z[2] = __uint_as_float(v.y << 16); z[3] = __uint_as_float(v.y & 0xffff0000u);
          } else {
            z[0] = half_lo(v.x); z[1] = half_hi(v.x); z[2] = half_lo(v.y); z[3] = half_hi(v.y);
          }
        }
      } else {
#pragma unroll
        for (int j = 0; j < 4; ++j) z[j] = j < n ? load1(a.logits, from + j, a.dtype) : 0.f;
      }
      const uint32_t allowed = mask ? (uint32_t)mask[i >> 5] >> (i & 31) : 15u;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        if (j < n) {
          if (a.history) {
            const uint32_t c = s_count[i + j - lo];
            if (c) z[j] = z[j] > 0.f ? __fdiv_rn(z[j], rep) : __fmul_rn(z[j], rep);
            if (c & ~kSeen) z[j] = __fsub_rn(__fsub_rn(z[j], __fmul_rn(freq, (float)(c & ~kSeen))), pres);
          }
          if (a.bias_ids) {
            const uint32_t e = s_bias[i + j - lo];
            if (e) z[j] = __fadd_rn(z[j], bias[e - 1u]);
          }
          if (!((allowed >> j) & 1u)) z[j] = -INFINITY;
          z[j] = rounded(z[j], a.dtype);
          if (z[j] > best) { best = z[j]; at = i + j; }   // (a thread's tokens come in order)
        }
      }
      if (a.wide && n == 4) {
        if (a.dtype == D3_FP32) *reinterpret_cast<float4 *>(static_cast<float *>(a.out) + to) = make_float4(z[0], z[1], z[2], z[3]);
        else *reinterpret_cast<uint2 *>(static_cast<char *>(a.out) + 2 * to) = make_uint2(pack2(z[0], z[1], a.dtype), pack2(z[2], z[3], a.dtype));
      } else {
#pragma unroll
        for (int j = 0; j < 4; ++j)
          if (j < n) store1(a.out, to + j, a.dtype, z[j]);
      }
    }
  }
  if (bad && a.status) *a.status = D3_EINVAL;
  if (!a.token) return;                      // (the same for every thread of the cluster)
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) take(best, at, __shfl_xor_sync(0xffffffffu, best, o), __shfl_xor_sync(0xffffffffu, at, o));
  if (lane == 0) { s_best[warp] = best; s_at[warp] = at; }
  __syncthreads();
  if (tid == 0) {
    for (int w = 1; w < kThreads / 32; ++w) take(best, at, s_best[w], s_at[w]);
    s_best[kThreads / 32] = best;
    s_at[kThreads / 32] = at;
  }
  if (a.split > 1) {
    asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
    if (rank == 0 && warp == 0) {
      if (lane < a.split) {
        uint32_t pb, pi;
        asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(pb) : "r"(smem_at(&s_best[kThreads / 32])), "r"(lane));
        asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(pi) : "r"(smem_at(&s_at[kThreads / 32])), "r"(lane));
        asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(best) : "r"(pb) : "memory");
        asm volatile("ld.shared::cluster.s32 %0, [%1];" : "=r"(at) : "r"(pi) : "memory");
      } else {
        best = -INFINITY;
        at = 0x7fffffff;
      }
#pragma unroll
      for (int o = 4; o > 0; o >>= 1) take(best, at, __shfl_xor_sync(0xffffffffu, best, o), __shfl_xor_sync(0xffffffffu, at, o));
    }
    asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
  }
  if (rank == 0 && tid == 0) a.token[row] = at == 0x7fffffff ? -1 : at;
}

}  // namespace

}  // namespace d3

using namespace d3;

extern "C" {

int32_t d3_constrain_logits(const d3_constrain_logits_args *a, void *cuda_stream) {
  if (!a || a->struct_size != sizeof(d3_constrain_logits_args) || !wide_type(a->dtype)) return D3_EINVAL;
  if (a->n_rows < 0 || a->n_rows > 65535 || a->vocab < 1 || a->n_history < 0 || a->n_bias < 0 || a->n_masks < 0) return D3_EINVAL;
  const int es = type_bytes(a->dtype);
  const int64_t rows = a->n_rows, vocab = a->vocab, words = (vocab + 31) / 32, most = (int64_t)1 << 38;
  auto stride_ok = [&](int64_t s, int64_t least) { return rows <= 1 || (s >= least && s <= most); };
  if (vocab > (1 << 30) || !a->logits_dev || !a->out_dev || !on_bytes(a->logits_dev, es) || !on_bytes(a->out_dev, es) ||
      !stride_ok(a->logits_stride, 0) || !stride_ok(a->out_stride, vocab))
    return D3_EINVAL;
  const bool history = a->history_dev && a->n_history > 0, biased = a->bias_ids_dev && a->n_bias > 0;
  const void *words4[] = {a->history_dev, a->lengths_dev, a->prompt_dev, a->repetition_dev, a->frequency_dev, a->presence_dev, a->bias_ids_dev,
                          a->bias_dev, a->masks_dev, a->mask_of_dev, a->token_dev, a->status_dev};
  for (const void *p : words4)
    if (!on_bytes(p, 4)) return D3_EINVAL;
  if (!a->history_dev && (a->lengths_dev || a->prompt_dev || a->repetition_dev || a->frequency_dev || a->presence_dev)) return D3_EINVAL;
  if (history && !stride_ok(a->history_stride, 0)) return D3_EINVAL;
  if ((a->bias_ids_dev != nullptr) != (a->bias_dev != nullptr) || (biased && !stride_ok(a->bias_stride, 0))) return D3_EINVAL;
  if ((a->masks_dev != nullptr) != (a->mask_of_dev != nullptr) ||
      (a->masks_dev && a->n_masks > 1 && (a->mask_stride < 0 || a->mask_stride > most)))
    return D3_EINVAL;
  if (rows == 0) return D3_OK;
  const RowSet logits = {a->logits_dev, rows, a->logits_stride * es, vocab * es}, out = {a->out_dev, rows, a->out_stride * es, vocab * es},
               token = {a->token_dev, 1, 0, rows * 4}, status = {a->status_dev, 1, 0, 4};
  const RowSet read[] = {{a->history_dev, rows, a->history_stride * 4, (int64_t)a->n_history * 4}, {a->lengths_dev, 1, 0, rows * 4},
                         {a->prompt_dev, 1, 0, rows * 4}, {a->repetition_dev, 1, 0, rows * 4}, {a->frequency_dev, 1, 0, rows * 4},
                         {a->presence_dev, 1, 0, rows * 4}, {a->bias_ids_dev, rows, a->bias_stride * 4, (int64_t)a->n_bias * 4},
                         {a->bias_dev, rows, a->bias_stride * 4, (int64_t)a->n_bias * 4},
                         {a->masks_dev, a->n_masks, a->mask_stride * 4, words * 4}, {a->mask_of_dev, 1, 0, rows * 4}};
  for (const RowSet &r : read)
    if (rows_common(out, r) || rows_common(token, r) || rows_common(status, r)) return D3_EINVAL;
  if ((rows_common(out, logits) && !(same_rows(out, logits) && rows_distinct(logits))) || rows_common(token, logits) || rows_common(status, logits) ||
      rows_common(out, token) || rows_common(out, status) || rows_common(token, status))
    return D3_EINVAL;

  LogitsArgs p;
  memset(&p, 0, sizeof(p));
  p.n_rows = a->n_rows; p.vocab = a->vocab; p.n_history = a->n_history; p.n_bias = biased ? a->n_bias : 0; p.n_masks = a->n_masks; p.dtype = a->dtype;
  p.logits = a->logits_dev; p.out = a->out_dev;
  p.logits_stride = rows > 1 ? a->logits_stride : 0; p.out_stride = rows > 1 ? a->out_stride : 0;
  p.history_stride = rows > 1 ? a->history_stride : 0; p.bias_stride = rows > 1 ? a->bias_stride : 0;
  p.mask_stride = a->n_masks > 1 ? a->mask_stride : 0;
  p.history = history ? a->history_dev : nullptr; p.lengths = a->lengths_dev; p.prompt = a->prompt_dev;
  p.repetition = a->repetition_dev; p.frequency = a->frequency_dev; p.presence = a->presence_dev;
  p.bias_ids = biased ? a->bias_ids_dev : nullptr; p.bias = biased ? a->bias_dev : nullptr;
  p.masks = a->masks_dev; p.mask_of = a->mask_of_dev; p.token = a->token_dev; p.status = a->status_dev;
  p.wide = on_bytes(a->logits_dev, 4 * es) && on_bytes(a->out_dev, 4 * es) && p.logits_stride % 4 == 0 && p.out_stride % 4 == 0;
  // the parts of a row: at most eight (a portable cluster), none below 1024 tokens
  int split = 8;
  while (split > 1 && vocab < (int64_t)split * 1024) split >>= 1;
  p.split = split;
  p.per = (int)((vocab + split - 1) / split + 7) / 8 * 8;
  const int slice = p.per < kSlice ? p.per : kSlice;
  const size_t smem = (size_t)slice * 4 * ((history || biased ? 1 : 0) + (biased ? 1 : 0));
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return D3_ECUDA;
  static std::atomic<bool> ready[64];   // the shared-memory attribute is per device; setting it twice is harmless
  if (!ready[dev].load(std::memory_order_acquire)) {
    if (cudaFuncSetAttribute(k_constrain_logits, cudaFuncAttributeMaxDynamicSharedMemorySize, kSlice * 8) != cudaSuccess) return D3_ECUDA;
    ready[dev].store(true, std::memory_order_release);
  }
  cudaLaunchConfig_t cfg;
  memset(&cfg, 0, sizeof(cfg));
  cfg.gridDim = dim3((unsigned)(rows * split));
  cfg.blockDim = dim3(kThreads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = static_cast<cudaStream_t>(cuda_stream);
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = (unsigned)split;
  attr[1].val.clusterDim.y = 1;
  attr[1].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = split > 1 ? 2 : 1;
  return cudaLaunchKernelEx(&cfg, k_constrain_logits, static_cast<const LogitsArgs>(p)) == cudaSuccess ? D3_OK : D3_ECUDA;
}

}  // extern "C"
