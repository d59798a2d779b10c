// Products of up to kFewRows rows in 8 bits with a weight matrix in 8 bits: weights stream, rows ride along.
//
//   y[row][r] = sum_b as[row][b] ws[r / 128][b] sum_{k in block b} a[row][k] w[r][k]
//
// Few rows leave 2 * rows flops for a byte of weight: the kernel is bound by reading the weights once.  The weight tile is
// the tensor core's 128-row operand (M), the rows are its narrow one (N = 16..128, rows beyond n_rows are zeros), so a
// block of 128 k is four tcgen05.mma and its sum, 128 x N in tensor memory, is small: the epilogue threads (one weight row
// each) fetch it, multiply by the two scales and add it to registers while the next block is multiplied.
//
// A CTA takes one tile of 128 weight rows (two matrices' tiles for the gated form) and a share of the k blocks; the CTAs of
// a tile are a cluster, whose sums meet in distributed shared memory in the order of their ranks.  Every CTA of the
// cluster finishes every split-th row: a warp has the 128 results of a row, four neighbouring ones a lane, which is also
// one block of scales where the result goes to 8 bits.
#include <atomic>

#include "d3_block8.cuh"

namespace d3 {

namespace {

constexpr int kTileBytes = 128 * 128;      // a stage's share of a weight matrix
constexpr int kMaxStages = 8;
constexpr int kScaleChunk = 8;             // k blocks whose scales are staged at a time
constexpr int kPairSmem = 113 * 1024 - 512;   // two CTAs of an SM side by side

__device__ __forceinline__ uint32_t cluster_rank() {
  uint32_t r;
  asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
  return r;
}
__device__ __forceinline__ void cluster_sync() {
  asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
__device__ __forceinline__ float4 cluster_load4(uint32_t at, uint32_t rank) {
  uint32_t remote;
  float4 v;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(remote) : "r"(at), "r"(rank));
  asm volatile("ld.shared::cluster.v4.f32 {%0,%1,%2,%3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(remote) : "memory");
  return v;
}

// C: rows (accumulator columns) of an epilogue thread, G: warpgroups that share the rows, W: weight matrices (2: gated)
template <int C, int G, int W>
struct Few {
  static constexpr int N = C * G;                              // padded rows
  static constexpr int kThreads = 64 + 128 * G;
  static constexpr int kBuffers = N * W <= 64 ? 4 : 2;         // of sums in tensor memory: 64 to 256 columns, 512 with N W = 256
  static constexpr int kColumns = kBuffers * N * W;
  static constexpr int kStage = W * kTileBytes + N * 128;
  static constexpr int kSums = W * N * 128 * 4;                // one CTA's sums, over the ring when it is empty
  static constexpr int kScales = 2 * kScaleChunk * (N + W) * 4;   // the rows' scales and the weights', two chunks
};

template <int C, int G, int W>
__global__ void __launch_bounds__(Few<C, G, W>::kThreads)
k_mm8_few(const __grid_constant__ CUtensorMap map_w0, const __grid_constant__ CUtensorMap map_w1, const __grid_constant__ CUtensorMap map_a,
          const __grid_constant__ Mm8Args t) {
  using F = Few<C, G, W>;
  constexpr int N = F::N;
  extern __shared__ unsigned char raw[];
  __shared__ __align__(8) uint64_t s_full[kMaxStages], s_empty[kMaxStages], s_done[F::kBuffers], s_read[F::kBuffers], s_tail;
  __shared__ uint32_t s_tmem;
  __shared__ int s_gave_up;
  const int tid = threadIdx.x, warp = __shfl_sync(0xffffffffu, tid >> 5, 0), lane = tid & 31;
  const int S = t.n_stages, split = t.split;
  const int tile = blockIdx.x / split, rank = split > 1 ? (int)cluster_rank() : 0;
  const int row0 = blockIdx.y * N;                             // first row of the call that this CTA multiplies
  const int b0 = (int)((long long)t.n_kb * rank / split), b1 = (int)((long long)t.n_kb * (rank + 1) / split);
  const uint32_t ring = (smem_at(raw) + 1023u) & ~1023u;       // the swizzle goes by the address
  float *scales = reinterpret_cast<float *>(raw + (ring - smem_at(raw)) + S * F::kStage);   // [2][kScaleChunk][N], then [2][kScaleChunk][W]
  volatile int *gave_up = &s_gave_up;

  if (tid == 0) {
    for (int s = 0; s < S; ++s) { mbar_init(smem_at(&s_full[s]), 1); mbar_init(smem_at(&s_empty[s]), 1); }
    for (int b = 0; b < F::kBuffers; ++b) { mbar_init(smem_at(&s_done[b]), 1); mbar_init(smem_at(&s_read[b]), 128 * G); }
    mbar_init(smem_at(&s_tail), 1);
    s_gave_up = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
  }
  if (warp == 1) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_at(&s_tmem)), "r"((uint32_t)F::kColumns) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = s_tmem;
  pdl_wait();
  pdl_trigger();

  float acc[W][C];
#pragma unroll
  for (int w = 0; w < W; ++w)
#pragma unroll
    for (int i = 0; i < C; ++i) acc[w][i] = 0.f;

  if (warp == 0) {
    // ------------------------------------------------------------ copies
    // (the whole warp runs the loops of this branch and the next, so that their arithmetic is the warp's and not a lane's)
    const bool one = elect_one();
    int s = 0, phase = 1, b = b0;
    for (; b < b1; ++b) {
      if (b - b0 >= S && !mbar_wait(smem_at(&s_empty[s]), (uint32_t)phase, gave_up, t.wait_tries)) break;
      const uint32_t full = smem_at(&s_full[s]), at = ring + (uint32_t)(s * F::kStage);
      if (one) {
        mbar_expect(full, F::kStage);
        tma_rows8(at, &map_w0, b * 128, tile * 128, full);
        if (W == 2) tma_rows8(at + kTileBytes, &map_w1, b * 128, tile * 128, full);
        tma_rows8(at + W * kTileBytes, &map_a, b * 128, row0, full);
      }
      if (++s == S) { s = 0; phase ^= 1; }
    }
    if (*gave_up) {   // copies in flight must land before the CTA's shared memory is given back
      for (int j = max(b0, b - S); j < b; ++j)
        mbar_wait(smem_at(&s_full[(j - b0) % S]), (uint32_t)(((j - b0) / S) & 1), gave_up, max(t.wait_tries, kDrainTries), false);
    }
    __syncwarp();
  } else if (warp == 1) {
    // ------------------------------------------------------------ products
    constexpr uint32_t idesc = idesc_e4m3(128, N);
    const bool one = elect_one();
    bool ok = true;
    int s = 0, phase = 0;
    for (int b = b0; b < b1; ++b) {
      const int it = b - b0, buf = it % F::kBuffers, use = it / F::kBuffers;
      ok = mbar_wait(smem_at(&s_full[s]), (uint32_t)phase, gave_up, t.wait_tries);
      if (ok && use) ok = mbar_wait(smem_at(&s_read[buf]), (uint32_t)((use - 1) & 1), gave_up, t.wait_tries);
      if (!ok) break;
      tc_fence_after();
      const uint32_t at = ring + (uint32_t)(s * F::kStage);
      const uint64_t bd = desc_rows8(at + W * kTileBytes);
      if (one) {
#pragma unroll
        for (int w = 0; w < W; ++w) {
          const uint64_t ad = desc_rows8(at + w * kTileBytes);
#pragma unroll
          for (int k = 0; k < 4; ++k)   // 32 numbers = 32 bytes = 2 descriptor units
            tc_mma_e4m3(tmem + (uint32_t)((buf * W + w) * N), ad + (uint64_t)(2 * k), bd + (uint64_t)(2 * k), idesc, k ? 1u : 0u);
        }
        tc_commit(smem_at(&s_done[buf]));
        tc_commit(smem_at(&s_empty[s]));
      }
      if (++s == S) { s = 0; phase ^= 1; }
    }
    if (!ok) {        // what was issued still reads shared memory and writes tensor memory
      if (one) tc_commit(smem_at(&s_tail));
      mbar_wait(smem_at(&s_tail), 0u, gave_up, max(t.wait_tries, kDrainTries), false);
    }
    __syncwarp();
  } else {
    // ------------------------------------------------------------ sums
    const int et = tid - 64, g = (warp - 2) >> 2, q = warp & 3;   // a warp reads the quarter of the lanes that its number names
    const int r = q * 32 + lane;                                  // weight row of the tile
    const uint32_t lanes = tmem + ((uint32_t)(q * 32) << 16) + (uint32_t)(g * C);
    // a chunk's scales, read one chunk ahead: entry e = row (e / kScaleChunk), block (e % kScaleChunk)
    constexpr int kMine = N * kScaleChunk / (128 * G);
    float ahead[kMine], w_ahead = 0.f;
    float *w_scales = scales + 2 * kScaleChunk * N;
    auto fetch = [&](int from) {
#pragma unroll
      for (int i = 0; i < kMine; ++i) {
        const int e = i * 128 * G + et, row = row0 + e / kScaleChunk, b = from + e % kScaleChunk;
        ahead[i] = row < t.n_rows && b < b1 ? t.a_scale[row * t.a_scale_stride + b] : 0.f;
      }
      const int b = from + et / W;
      if (et < kScaleChunk * W) w_ahead = b < b1 ? t.w_scale[et % W][(size_t)tile * t.n_kb + b] : 0.f;
    };
    auto keep = [&](int half) {
#pragma unroll
      for (int i = 0; i < kMine; ++i) {
        const int e = i * 128 * G + et;
        scales[(half * kScaleChunk + e % kScaleChunk) * N + e / kScaleChunk] = ahead[i];
      }
      if (et < kScaleChunk * W) w_scales[half * kScaleChunk * W + et] = w_ahead;
    };
    fetch(b0);
    keep(0);
    asm volatile("bar.sync 1, %0;" ::"n"(128 * G) : "memory");
    for (int c0 = b0, half = 0; c0 < b1; c0 += kScaleChunk, half ^= 1) {
      const int c1 = min(b1, c0 + kScaleChunk);
      fetch(c0 + kScaleChunk);
      for (int b = c0; b < c1; ++b) {
        const int it = b - b0, buf = it % F::kBuffers;
        float wsb[W];
#pragma unroll
        for (int w = 0; w < W; ++w) wsb[w] = w_scales[(half * kScaleChunk + b - c0) * W + w];
        mbar_wait(smem_at(&s_done[buf]), (uint32_t)((it / F::kBuffers) & 1), gave_up, t.wait_tries);   // (given up: numbers without meaning)
        __syncwarp();
        tc_fence_after();
        const float *as = scales + (half * kScaleChunk + (b - c0)) * N + g * C;
        constexpr int P = C < 32 ? C : 32;
#pragma unroll
        for (int w = 0; w < W; ++w) {
#pragma unroll
          for (int p = 0; p < C; p += P) {
            uint32_t d[P];
            tc_ld(lanes + (uint32_t)((buf * W + w) * N + p), d);
            tc_ld_wait(d);
            if (w == W - 1 && p == C - P) {
              tc_fence_before();
              mbar_arrive(smem_at(&s_read[buf]));
            }
#pragma unroll
            for (int i = 0; i < P; i += 4) {
              const float4 f = *reinterpret_cast<const float4 *>(as + p + i);
              acc[w][p + i] = fmaf(__uint_as_float(d[i]), f.x * wsb[w], acc[w][p + i]);
              acc[w][p + i + 1] = fmaf(__uint_as_float(d[i + 1]), f.y * wsb[w], acc[w][p + i + 1]);
              acc[w][p + i + 2] = fmaf(__uint_as_float(d[i + 2]), f.z * wsb[w], acc[w][p + i + 2]);
              acc[w][p + i + 3] = fmaf(__uint_as_float(d[i + 3]), f.w * wsb[w], acc[w][p + i + 3]);
            }
          }
        }
      }
      keep(half ^ 1);
      asm volatile("bar.sync 1, %0;" ::"n"(128 * G) : "memory");
    }
    // every copy has landed and every product is done: the ring holds the sums now, [matrix][row of the call][weight row]
    float *sums = reinterpret_cast<float *>(raw + (ring - smem_at(raw)));
#pragma unroll
    for (int w = 0; w < W; ++w)
#pragma unroll
      for (int i = 0; i < C; ++i) sums[(w * N + g * C + i) * 128 + r] = acc[w][i];
  }

  if (split > 1) cluster_sync();
  else __syncthreads();
  const int rows = min(N, t.n_rows - row0), n0 = tile * 128 + 4 * lane;
  for (int j = rank + split * warp; j < rows; j += split * (F::kThreads / 32)) {
    float y[W][4];
#pragma unroll
    for (int w = 0; w < W; ++w) {
      const uint32_t at = ring + (uint32_t)(((w * N + j) * 128 + 4 * lane) * 4);
      float4 part[8];
#pragma unroll
      for (int p = 0; p < 8; ++p)
        if (p < split) part[p] = cluster_load4(at, (uint32_t)p);
      float4 sum = part[0];
#pragma unroll
      for (int p = 1; p < 8; ++p)
        if (p < split) { sum.x += part[p].x; sum.y += part[p].y; sum.z += part[p].z; sum.w += part[p].w; }
      y[w][0] = sum.x; y[w][1] = sum.y; y[w][2] = sum.z; y[w][3] = sum.w;
    }
    if constexpr (W == 2) {
#pragma unroll
      for (int i = 0; i < 4; ++i) y[0][i] = gate_of(y[0][i], y[1][i]);
    }
    finish4(t, row0 + j, n0, y[0], tile, lane);
  }
  if (split > 1) cluster_sync();   // no CTA's sums go while another one reads them
  if (tid == 0 && *gave_up && t.status) *t.status = D3_ETIMEOUT;
  tc_fence_before();
  __syncthreads();
  if (warp == 1)
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"((uint32_t)F::kColumns) : "memory");
}

template <int C, int G, int W>
cudaError_t launch(const TMap &w0, const TMap &w1, const TMap &ma, Mm8Args &p, cudaStream_t st) {
  using F = Few<C, G, W>;
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  if (dev < 0 || dev >= 64) return cudaErrorInvalidDevice;
  static std::atomic<int> sms[64];   // SMs of a device whose attribute is set (setting it twice is harmless)
  int n_sm = sms[dev].load(std::memory_order_acquire);
  if (n_sm == 0) {
    if ((e = cudaDeviceGetAttribute(&n_sm, cudaDevAttrMultiProcessorCount, dev)) != cudaSuccess) return e;
    if ((e = cudaFuncSetAttribute(k_mm8_few<C, G, W>, cudaFuncAttributeMaxDynamicSharedMemorySize, 226 * 1024)) != cudaSuccess) return e;
    sms[dev].store(n_sm, std::memory_order_release);
  }
  // Two CTAs an SM where three stages of each fit side by side; one with a longer ring otherwise.
  const int fixed = F::kScales + 1024;
  int per_sm = 2, stages = (kPairSmem - fixed) / F::kStage;
  if (stages < 3 || F::kColumns > 256) { per_sm = 1; stages = (224 * 1024 - fixed) / F::kStage; }
  const int least = (F::kSums + F::kStage - 1) / F::kStage;    // the ring holds the sums in the end
  // As many CTAs as the GPU holds at once, so that they share its memory rate from the first to the last byte.
  const int tiles = (p.n + 127) / 128;
  int split = n_sm * per_sm / tiles;
  if (split > 8) split = 8;
  if (split > p.n_kb) split = p.n_kb;
  if (split < 1) split = 1;
  const int most = (p.n_kb + split - 1) / split;               // blocks of a CTA
  if (stages > most) stages = most;
  if (stages < least) stages = least;
  if (stages > kMaxStages) stages = kMaxStages;
  p.n_stages = stages;
  p.split = split;
  cudaLaunchConfig_t cfg;
  memset(&cfg, 0, sizeof(cfg));
  cfg.gridDim = dim3((unsigned)(tiles * split), (unsigned)((p.n_rows + F::N - 1) / F::N));
  cfg.blockDim = dim3(F::kThreads);
  cfg.dynamicSmemBytes = (size_t)stages * F::kStage + fixed;
  cfg.stream = st;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = (unsigned)split;
  attr[1].val.clusterDim.y = 1;
  attr[1].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = split > 1 ? 2 : 1;
  const CUtensorMap *m0 = reinterpret_cast<const CUtensorMap *>(&w0), *m1 = reinterpret_cast<const CUtensorMap *>(&w1),
                    *m = reinterpret_cast<const CUtensorMap *>(&ma);
  return cudaLaunchKernelEx(&cfg, k_mm8_few<C, G, W>, *m0, *m1, *m, static_cast<const Mm8Args>(p));
}

template <int W>
cudaError_t choose(const TMap &w0, const TMap &w1, const void *a, int64_t a_stride, Mm8Args &p, cudaStream_t st) {
  const int padded = p.n_rows <= 16 ? 16 : p.n_rows <= 32 ? 32 : p.n_rows <= 64 ? 64 : 128;
  TMap ma;
  if (!encode_rows8(&ma, a, p.n_rows, p.k, a_stride, padded)) return cudaErrorInvalidValue;
  switch (padded) {
    case 16: return launch<16, 1, W>(w0, w1, ma, p, st);
    case 32: return launch<32, 1, W>(w0, w1, ma, p, st);
    case 64: return launch<64, 1, W>(w0, w1, ma, p, st);
    default: return launch<64, 2, W>(w0, w1, ma, p, st);
  }
}

}  // namespace

cudaError_t launch_mm8_few(const TMap &w0, const TMap *w1, const void *a, int64_t a_stride, Mm8Args &p, cudaStream_t st) {
  return w1 ? choose<2>(w0, *w1, a, a_stride, p, st) : choose<1>(w0, w0, a, a_stride, p, st);
}

}  // namespace d3
