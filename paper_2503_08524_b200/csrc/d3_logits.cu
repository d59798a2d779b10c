// Constraints on logits: penalties for repeated tokens, biases, a grammar's mask, and the best token that is left.
//
// One pass over the logits, so many rows are bound by reading and writing them once and few by latency.  A row's vocabulary is cut
// between the CTAs of a cluster, and a CTA takes its part in slices that it has a word for each token of in shared memory: it
// reads the row's history, counts the tokens that fall in the slice (whole numbers: the order of the atomics changes
// nothing), and then has everything it needs of a token at hand.  A slice's logits are all asked for before the counting, which
// they arrive behind: with one piece of 16 bytes a thread on its way at a time, 250 rows of 128001 took 244 us.  The history
// is read once a slice, from L2 or L1.  The best token is found on the way: per thread, per CTA, and between the CTAs through
// distributed shared memory.
#include <math.h>

#include <atomic>

#include "d3_block8.cuh"

namespace d3 {

namespace {

constexpr int kThreads = 512;
static_assert(D3_BF16 == 0 && D3_FP16 == 1 && D3_FP32 == 2, "types index");
constexpr int kPieces = 8;                   // pieces of four logits that a thread has of a slice
constexpr int kSlice = 4 * kThreads * kPieces;
constexpr int kBatch = 8;                    // history entries that a thread has on their way
constexpr int kMostSplit = 8;                // CTAs of a row, a portable cluster
// A token's word: the biases' entry + 1 above, below it whether the token is in the prompt and how often behind it.  Longer lists
// than these fields hold have two words a token (kTwo).
constexpr uint32_t kSeen = 0x8000u, kCount = 0x7fffu, kSeenTwo = 0x80000000u;
constexpr int kMostHistory = 0x7fff, kMostBias = 0xffff;

struct LogitsArgs {
  int n_rows, vocab, n_history, n_bias, n_masks, dtype, split, per;
  int wide;                                  // logits and out lie alike between 16-byte pieces (16-bit types: 8)
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
  if (v > best || (v == best && i < at)) { best = v; at = i; }      // (none: -inf and the largest index)
}
__device__ __forceinline__ float rounded(float v, int dtype) {
  if (dtype == D3_BF16) return __bfloat162float(__float2bfloat16_rn(v));
  if (dtype == D3_FP16) return __half2float(__float2half_rn(v));
  return v;
}

// four logits that lie in one piece of memory
template <int kType>
__device__ __forceinline__ void read4(const void *logits, long long at, float (&z)[4]) {
  if (kType == D3_FP32) {
    const float4 v = *reinterpret_cast<const float4 *>(static_cast<const float *>(logits) + at);
    z[0] = v.x; z[1] = v.y; z[2] = v.z; z[3] = v.w;
  } else {
    const uint2 v = *reinterpret_cast<const uint2 *>(static_cast<const char *>(logits) + 2 * at);
    if (kType == D3_BF16) {
      z[0] = __uint_as_float(v.x << 16); z[1] = __uint_as_float(v.x & 0xffff0000u);
      z[2] = __uint_as_float(v.y << 16); z[3] = __uint_as_float(v.y & 0xffff0000u);
    } else {
      z[0] = half_lo(v.x); z[1] = half_hi(v.x); z[2] = half_lo(v.y); z[3] = half_hi(v.y);
    }
  }
}
template <int kType>
__device__ __forceinline__ void write4(void *out, long long at, const float (&z)[4]) {
  if (kType == D3_FP32) *reinterpret_cast<float4 *>(static_cast<float *>(out) + at) = make_float4(z[0], z[1], z[2], z[3]);
  else *reinterpret_cast<uint2 *>(static_cast<char *>(out) + 2 * at) = make_uint2(pack2(z[0], z[1], kType), pack2(z[2], z[3], kType));
}
template <int kType, bool kTwo>
__global__ void __launch_bounds__(kThreads, 2) k_constrain_logits(const __grid_constant__ LogitsArgs a) {
  extern __shared__ __align__(16) uint32_t s_word[];      // [slice]; with kTwo the biases' entries behind it
  __shared__ float s_best[kThreads / 32];
  __shared__ int s_at[kThreads / 32];
  __shared__ unsigned long long s_part[kMostSplit];       // the first CTA of a row: what the others found
  __shared__ __align__(8) uint64_t s_bar;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int row = blockIdx.x / a.split, rank = blockIdx.x % a.split;
  // Places count from the last 16-byte border before the row's first logit, so that four from a multiple of four on are one piece of
  // memory: token t is at place t + shift.
  const long long from = row * a.logits_stride, to = row * a.out_stride;
  constexpr int kSize = kType == D3_FP32 ? 4 : 2;
  const int shift = a.wide ? (int)(((uintptr_t)a.logits / kSize + (uintptr_t)from) & 3u) : 0;
  const int end = a.vocab + shift;
  const int v0 = min(end, rank * a.per), v1 = min(end, v0 + a.per);
  const int slice = min(a.per, kSlice);
  const bool listed = a.history || a.bias_ids;
  const int32_t *history = a.history + row * a.history_stride, *ids = a.bias_ids + row * a.bias_stride;
  const float *bias = a.bias + row * a.bias_stride;
  auto clear = [&]() {
    if (listed)
      for (int i = 4 * tid; i < (kTwo ? 2 : 1) * slice; i += 4 * kThreads) *reinterpret_cast<uint4 *>(s_word + i) = make_uint4(0u, 0u, 0u, 0u);
  };
  if (a.split > 1) {
    if (tid == 0) {
      mbar_init(smem_at(&s_bar), 1);
      if (rank == 0) mbar_expect(smem_at(&s_bar), 8u * (uint32_t)(a.split - 1));
      asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    cluster_arrive();
  }
  clear();
  pdl_wait();
  pdl_trigger();

  bool bad = false;
  float best = -INFINITY;
  int at = 0x7fffffff;
  int length = 0, prompt = 0;
  float rep = 1.f, part = 1.f, inverse = 1.f, freq = 0.f, pres = 0.f;
  const int32_t *mask = nullptr;

  for (int lo = v0; lo < v1; lo += slice) {
    const int hi = min(v1, lo + slice);
    if (lo != v0) {
      __syncthreads();
      clear();
    }
    // A thread's pieces start at x0 + p * 4 kThreads; those from p0 up to p1 are whole.  The others (at the ends of a row, and all of
    // rows that lie differently in and out) are taken number by number in the end.
    const int x0 = lo + 4 * tid, first = lo - shift;               // (the token at the slice's first place)
    const int p0 = x0 < shift ? 1 : 0, room = min(hi, end) - 4 - x0, p1 = a.wide && room >= 0 ? min(room / (4 * kThreads) + 1, kPieces) : 0;
    const long long in0 = from + x0 - shift, out0 = to + x0 - shift;
    // everything that nothing else has to be known for is asked for first
    float z[kPieces][4];
#pragma unroll
    for (int p = 0; p < kPieces; ++p)
      if (p >= p0 && p < p1) read4<kType>(a.logits, in0 + p * (4 * kThreads), z[p]);
    int biased = -1;
    if (a.bias_ids && tid < a.n_bias) biased = ids[tid];
    if (lo == v0) {
      auto bounded = [&](const int32_t *p, int none) {   // an entry of lengths or prompt
        if (!p) return none;
        const int v = p[row];
        if (v < 0 || v > a.n_history) bad = true;
        return min(max(v, 0), a.n_history);
      };
      length = bounded(a.lengths, a.n_history);          // (a history of no entries: checked alike)
      prompt = bounded(a.prompt, 0);
      if (a.repetition) {
        rep = part = a.repetition[row];
        inverse = __frcp_rn(rep);
        if (fabsf(rep) < 0x1p-126f) {        // no number for its reciprocal: what `value` makes of the two is z * inverse * (2 - inverse * part)
          inverse = copysignf(0x1p126f, rep);
          part = (2.f - __frcp_rn(rep * inverse)) * copysignf(0x1p-126f, rep);
        }
      }
      if (a.frequency) freq = a.frequency[row];
      if (a.presence) pres = a.presence[row];
      if (a.masks) {
        const int m = a.mask_of[row];
        if (m >= a.n_masks) bad = true;
        else if (m >= 0) mask = a.masks + m * a.mask_stride;
      }
    }
    if (listed) {
      const int t0 = max(first, 0);                        // the slice's tokens are those from t0 on, `tokens` of them
      const uint32_t tokens = (uint32_t)(hi - shift - t0);
      uint32_t *words = s_word + (t0 - first);
      int most = -1;                                       // the largest id
      __syncthreads();
      if (a.bias_ids) {
        for (int i = tid; i < a.n_bias; i += kThreads) {
          const int b = i == tid ? biased : ids[i];
          if ((uint32_t)(b - t0) < tokens) atomicMax(words + (kTwo ? slice : 0) + (b - t0), kTwo ? (uint32_t)i + 1u : ((uint32_t)i + 1u) << 16);
          most = max(most, b);
        }
        if (!kTwo) __syncthreads();          // (the counts go below the entries)
      }
      for (int i0 = tid; i0 < length; i0 += kBatch * kThreads) {
        int id[kBatch];
#pragma unroll
        for (int e = 0; e < kBatch; ++e) id[e] = i0 + e * kThreads < length ? history[i0 + e * kThreads] : -1;
#pragma unroll
        for (int e = 0; e < kBatch; ++e) {
          if ((uint32_t)(id[e] - t0) < tokens) {           // (an id below 0 is far beyond)
            if (i0 + e * kThreads < prompt) atomicOr(words + (id[e] - t0), kTwo ? kSeenTwo : kSeen);
            else atomicAdd(words + (id[e] - t0), 1u);
          }
          most = max(most, id[e]);
        }
      }
      bad |= most >= a.vocab;
    }
    uint32_t allowed = 0xffffffffu;          // four bits a piece
    if (mask) {                              // (pieces are a multiple of 32 tokens apart: all start at the same bit of a word)
      const int t = x0 - shift, bit = t & 31;
      const int32_t *m = mask + (t >> 5);    // (t < 0: piece 0 is none of these)
      uint32_t w[kPieces];
      allowed = 0u;
#pragma unroll
      for (int p = 0; p < kPieces; ++p) w[p] = p >= p0 && p < p1 ? (uint32_t)m[p * (kThreads / 8)] : 0u;
#pragma unroll
      for (int p = 0; p < kPieces; ++p) allowed |= ((w[p] >> bit) & 15u) << (4 * p);
      if (bit > 28) {                        // the rest of their bits is in the words behind
#pragma unroll
        for (int p = 0; p < kPieces; ++p) w[p] = p >= p0 && p < p1 ? (uint32_t)m[p * (kThreads / 8) + 1] : 0u;
#pragma unroll
        for (int p = 0; p < kPieces; ++p) allowed |= ((w[p] << (32 - bit)) & 15u) << (4 * p);
      }
    }
    if (listed) __syncthreads();
    // What becomes of a logit.  Quotients by the penalty are made of its rounded reciprocal and the remainder, as fp32 division rounds them
    // (Markstein's division).  The division's own code here, 33 times, takes registers that are not there: 250 rows of 128001 took 113 us where
    // this takes 76; a product with the reciprocal alone, one rounding more, took 72.  An infinite quotient leaves no number, which the
    // maximum turns into one.
    auto value = [&](float v, uint32_t w, uint32_t e) {
      const uint32_t seen = kTwo ? w : w & 0xffffu, c = w & (kTwo ? ~kSeenTwo : kCount), entry = kTwo ? e : w >> 16;
      if (seen) {
        const bool above = v > 0.f;
        const float q = __fmul_rn(v, above ? inverse : rep), left = fmaxf(__fmaf_rn(-q, part, v), -3.4e38f);
        v = above ? __fmaf_rn(left, inverse, q) : q;
      }
      if (c) v = __fsub_rn(__fsub_rn(v, __fmul_rn(freq, (float)c)), pres);
      if (entry) v = __fadd_rn(v, bias[entry - 1u]);
      return v;
    };
    float top[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY}, high = -INFINITY;     // the piece with the largest number
    int high_p = 0;
#pragma unroll
    for (int p = 0; p < kPieces; ++p) {
      if (p >= p0 && p < p1) {
        if (listed) {
          const uint32_t *word = s_word + 4 * tid + p * (4 * kThreads);
          const uint4 w = *reinterpret_cast<const uint4 *>(word);
          uint4 e = make_uint4(0u, 0u, 0u, 0u);
          if (kTwo && a.bias_ids) e = *reinterpret_cast<const uint4 *>(word + slice);
          if (w.x | w.y | w.z | w.w | e.x | e.y | e.z | e.w) {
            z[p][0] = value(z[p][0], w.x, e.x); z[p][1] = value(z[p][1], w.y, e.y);
            z[p][2] = value(z[p][2], w.z, e.z); z[p][3] = value(z[p][3], w.w, e.w);
          }
        }
        if (mask) {
#pragma unroll
          for (int j = 0; j < 4; ++j)
            if (!(allowed & (1u << (4 * p + j)))) z[p][j] = -INFINITY;
        }
        if (kType != D3_FP32) {
#pragma unroll
          for (int j = 0; j < 4; ++j) z[p][j] = rounded(z[p][j], kType);
        }
        write4<kType>(a.out, out0 + p * (4 * kThreads), z[p]);
        const float m = fmaxf(fmaxf(z[p][0], z[p][1]), fmaxf(z[p][2], z[p][3]));
        if (m > high) {                      // (the first piece that has it)
          high = m; high_p = p;
#pragma unroll
          for (int j = 0; j < 4; ++j) top[j] = z[p][j];
        }
      }
    }
    if (high > best) {                       // (a thread's slices come in order)
      best = high;
      at = x0 - shift + high_p * (4 * kThreads) + (top[0] == high ? 0 : top[1] == high ? 1 : top[2] == high ? 2 : 3);
    }
    if (p0 > 0 || (p1 < kPieces && x0 + p1 * (4 * kThreads) < hi)) {
#pragma unroll 1
      for (int p = 0; p < kPieces; ++p) {
        const int x = x0 + p * (4 * kThreads);
        if ((p >= p0 && p < p1) || x >= hi) continue;
#pragma unroll 1
        for (int j = max(shift - x, 0); j < 4 && x + j < min(hi, end); ++j) {
          const int t = x + j - shift;
          float v = load1(a.logits, from + t, kType);
          if (listed) v = value(v, s_word[x + j - lo], kTwo && a.bias_ids ? s_word[slice + x + j - lo] : 0u);
          if (mask && !(((uint32_t)mask[t >> 5] >> (t & 31)) & 1u)) v = -INFINITY;
          v = rounded(v, kType);
          store1(a.out, to + t, kType, v);
          take(best, at, v, v > -INFINITY ? t : 0x7fffffff);
        }
      }
    }
  }
  if (bad && a.status) *a.status = D3_EINVAL;
  if (!a.token) {                            // (the same for every thread of the cluster)
    if (a.split > 1) cluster_wait();
    return;
  }
  // The best token: of the warps, then of the CTAs.  Each CTA but the first writes what it found to the first one's shared memory and
  // is done (CTAs that wait for the slowest of their cluster keep others from their places); the first
  // waits for them all.  Its barrier is set up before anyone can arrive: that is what the cluster's own barrier, arrived at in
  // the beginning, is for.
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) take(best, at, __shfl_xor_sync(0xffffffffu, best, o), __shfl_xor_sync(0xffffffffu, at, o));
  if (lane == 0) { s_best[warp] = best; s_at[warp] = at; }
  __syncthreads();
  if (a.split > 1) cluster_wait();
  if (warp != 0) return;
  best = lane < kThreads / 32 ? s_best[lane] : -INFINITY;
  at = lane < kThreads / 32 ? s_at[lane] : 0x7fffffff;
#pragma unroll
  for (int o = 8; o > 0; o >>= 1) take(best, at, __shfl_xor_sync(0xffffffffu, best, o), __shfl_xor_sync(0xffffffffu, at, o));
  if (rank != 0) {
    if (lane == 0) {
      uint32_t slot, bar;
      asm volatile("mapa.shared::cluster.u32 %0, %1, 0;" : "=r"(slot) : "r"(smem_at(&s_part[rank])));
      asm volatile("mapa.shared::cluster.u32 %0, %1, 0;" : "=r"(bar) : "r"(smem_at(&s_bar)));
      asm volatile("st.async.shared::cluster.mbarrier::complete_tx::bytes.b64 [%0], %1, [%2];"
                   ::"r"(slot), "l"((unsigned long long)__float_as_uint(best) | ((unsigned long long)(uint32_t)at << 32)), "r"(bar) : "memory");
    }
    return;
  }
  if (a.split > 1) {
    bool there = false;
    for (uint32_t n = 0; n < kWaitTries && !there; ++n) there = mbar_try(smem_at(&s_bar), 0u);
    if (!there && a.status) *a.status = D3_ETIMEOUT;
    if (lane > 0 && lane < a.split) {
      const unsigned long long part = s_part[lane];
      best = __uint_as_float((uint32_t)part);
      at = (int)(part >> 32);
    }
#pragma unroll
    for (int o = 8; o > 0; o >>= 1) take(best, at, __shfl_xor_sync(0xffffffffu, best, o), __shfl_xor_sync(0xffffffffu, at, o));
  }
  if (lane == 0) a.token[row] = at == 0x7fffffff ? -1 : at;
}

}  // namespace

}  // namespace d3

using namespace d3;

extern "C" {

int32_t d3_constrain_logits(const d3_constrain_logits_args *a, void *cuda_stream) {
  if (!a || a->struct_size != sizeof(d3_constrain_logits_args) || !wide_type(a->dtype)) return D3_EINVAL;
  if (a->n_rows < 0 || a->n_rows > 65535 || a->vocab < 1 || a->n_history < 0 || a->n_bias < 0 || a->n_masks < 0) return D3_EINVAL;
  if (a->n_history > (1 << 30) || a->n_bias > (1 << 30)) return D3_EINVAL;
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
  // (lists of no entries may have no address)
  if (!a->history_dev && a->n_history > 0 && (a->lengths_dev || a->prompt_dev || a->repetition_dev || a->frequency_dev || a->presence_dev))
    return D3_EINVAL;
  if (history && !stride_ok(a->history_stride, 0)) return D3_EINVAL;
  if ((a->n_bias > 0 && (a->bias_ids_dev != nullptr) != (a->bias_dev != nullptr)) || (biased && !stride_ok(a->bias_stride, 0))) return D3_EINVAL;
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
  p.n_rows = a->n_rows; p.vocab = a->vocab; p.n_history = history ? a->n_history : 0; p.n_bias = biased ? a->n_bias : 0; p.n_masks = a->n_masks; p.dtype = a->dtype;
  p.logits = a->logits_dev; p.out = a->out_dev;
  p.logits_stride = rows > 1 ? a->logits_stride : 0; p.out_stride = rows > 1 ? a->out_stride : 0;
  p.history_stride = rows > 1 ? a->history_stride : 0; p.bias_stride = rows > 1 ? a->bias_stride : 0;
  p.mask_stride = a->n_masks > 1 ? a->mask_stride : 0;
  p.history = history ? a->history_dev : nullptr; p.lengths = a->lengths_dev; p.prompt = a->prompt_dev;
  p.repetition = a->repetition_dev; p.frequency = a->frequency_dev; p.presence = a->presence_dev;
  p.bias_ids = biased ? a->bias_ids_dev : nullptr; p.bias = biased ? a->bias_dev : nullptr;
  p.masks = a->masks_dev; p.mask_of = a->mask_of_dev; p.token = a->token_dev; p.status = a->status_dev;
  p.wide = ((uintptr_t)a->logits_dev - (uintptr_t)a->out_dev) % (4 * es) == 0 && (p.logits_stride - p.out_stride) % 4 == 0;
  // The parts of a row: as many as fill two CTAs an SM, none below 1024 tokens.  More cost more than they give: clusters are started
  // one after another, some 0.2 us each (us with 1 / 2 / 4 / 8 parts: 8 rows of 32000 11.9 / 7.3 / 5.8 / 5.1, 32 rows 12.1 / 7.5 / 6.8 /
  // 6.6, 100 rows 12.6 / 10.7 / 13.1 / 21.1, 300 rows 30.6 / 30.0 / 38.6 / 60.8; 64 rows of 128001 45.7 / 26.8 / 22.0 / 25.8).
  int split = 1;
  while (split < kMostSplit && rows * split * 2 <= 2 * 148 && vocab >= (int64_t)split * 2048) split *= 2;
  p.split = split;
  p.per = (int)((vocab + 3 + split - 1) / split + 7) / 8 * 8;     // (and up to three places before the first token)
  const int slice = p.per < kSlice ? p.per : kSlice;
  const bool two = (history && a->n_history > kMostHistory) || (biased && a->n_bias > kMostBias);
  const size_t smem = history || biased ? (size_t)slice * (two ? 8 : 4) : 0;
  void (*kernel)(LogitsArgs) =
      a->dtype == D3_FP32 ? (two ? k_constrain_logits<D3_FP32, true> : k_constrain_logits<D3_FP32, false>)
      : a->dtype == D3_BF16 ? (two ? k_constrain_logits<D3_BF16, true> : k_constrain_logits<D3_BF16, false>)
                            : (two ? k_constrain_logits<D3_FP16, true> : k_constrain_logits<D3_FP16, false>);
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return D3_ECUDA;
  static std::atomic<bool> ready[2][3][64];   // the shared-memory attribute is per device; setting it twice is harmless
  std::atomic<bool> &set = ready[two][a->dtype][dev];
  if (!set.load(std::memory_order_acquire)) {
    if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kSlice * (two ? 8 : 4)) != cudaSuccess) return D3_ECUDA;
    set.store(true, std::memory_order_release);
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
  return cudaLaunchKernelEx(&cfg, kernel, static_cast<LogitsArgs>(p)) == cudaSuccess ? D3_OK : D3_ECUDA;
}

}  // extern "C"
