// Products of many rows in 8 bits with a weight matrix in 8 bits.
//
//   y[row][r] = sum_b as[row][b] ws[r / 128][b] sum_{k in block b} a[row][k] w[r][k]
//
// Bound by the tensor cores: 2 flops for every (row, weight row, k).  A CTA has 128 rows (the tensor core's M) times 256
// weight rows (N; the gated form: 128 of each matrix).  A block of 128 k is four tcgen05.mma whose sum, 128 x 256, goes to
// one of two buffers in tensor memory; while the next block is multiplied, eight epilogue warps fetch the sum, multiply it
// by the two scales and add it to registers (a thread has one row and 64 columns of each half), because every block has
// scales of its own.
#include <atomic>

#include "d3_block8.cuh"

namespace d3 {

namespace {

constexpr int kM = 128;                          // rows of a tile
constexpr int kBox = 128 * 128;                  // bytes of 128 rows of a stage
constexpr int kStage = 3 * kBox;                 // a's rows, and two boxes of weight rows
constexpr int kStages = 4;
constexpr int kThreads = 64 + 256;
constexpr int kColumns = 512;

template <int W>
__global__ void __launch_bounds__(kThreads, 1)
k_mm8_many(const __grid_constant__ CUtensorMap map_w0, const __grid_constant__ CUtensorMap map_w1, const __grid_constant__ CUtensorMap map_a,
           const __grid_constant__ Mm8Args t) {
  extern __shared__ unsigned char raw[];
  __shared__ __align__(8) uint64_t s_full[kStages], s_empty[kStages], s_done[2], s_read[2], s_tail;
  __shared__ float s_top[2][kM];
  __shared__ uint32_t s_tmem;
  __shared__ int s_gave_up;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const uint32_t ring = (smem_at(raw) + 1023u) & ~1023u;
  volatile int *gave_up = &s_gave_up;
  // columns of the two halves: neighbouring blocks of weight rows, or the same block of the two matrices
  const int half_n = W == 2 ? 0 : 128;
  const int n0 = blockIdx.x * (W == 2 ? 128 : 256), row0 = blockIdx.y * kM;

  if (tid == 0) {
    for (int s = 0; s < kStages; ++s) { mbar_init(smem_at(&s_full[s]), 1); mbar_init(smem_at(&s_empty[s]), 1); }
    for (int b = 0; b < 2; ++b) { mbar_init(smem_at(&s_done[b]), 1); mbar_init(smem_at(&s_read[b]), 256); }
    mbar_init(smem_at(&s_tail), 1);
    s_gave_up = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
  }
  if (warp == 1) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_at(&s_tmem)), "r"((uint32_t)kColumns) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = s_tmem;
  pdl_wait();
  pdl_trigger();

  if (warp == 0) {
    if (lane == 0) {
      int issued = 0;
      for (int b = 0; b < t.n_kb; ++b) {
        const int s = b % kStages, fill = b / kStages;
        if (fill > 0 && !mbar_wait(smem_at(&s_empty[s]), (uint32_t)((fill - 1) & 1), gave_up, t.wait_ns)) break;
        const uint32_t full = smem_at(&s_full[s]), at = ring + (uint32_t)(s * kStage);
        mbar_expect(full, kStage);
        tma_rows8(at, &map_a, b * 128, row0, full);
        tma_rows8(at + kBox, &map_w0, b * 128, n0, full);
        tma_rows8(at + 2 * kBox, W == 2 ? &map_w1 : &map_w0, b * 128, n0 + half_n, full);
        issued = b + 1;
      }
      if (*gave_up) {
        const unsigned long long bound = t.wait_ns > kDrainFloorNs ? t.wait_ns : kDrainFloorNs;
        for (int b = max(0, issued - kStages); b < issued; ++b)
          mbar_wait(smem_at(&s_full[b % kStages]), (uint32_t)((b / kStages) & 1), gave_up, bound, false);
      }
    }
    __syncwarp();
  } else if (warp == 1) {
    if (lane == 0) {
      constexpr uint32_t idesc = idesc_e4m3(kM, 256);
      bool ok = true;
      for (int b = 0; b < t.n_kb; ++b) {
        const int s = b % kStages, buf = b & 1;
        ok = b < 2 || mbar_wait(smem_at(&s_read[buf]), (uint32_t)(((b >> 1) - 1) & 1), gave_up, t.wait_ns);
        if (ok) ok = mbar_wait(smem_at(&s_full[s]), (uint32_t)((b / kStages) & 1), gave_up, t.wait_ns);
        if (!ok) break;
        tc_fence_after();
        const uint64_t ad = desc_rows8(ring + (uint32_t)(s * kStage)), bd = desc_rows8(ring + (uint32_t)(s * kStage + kBox));
#pragma unroll
        for (int k = 0; k < 4; ++k)
          tc_mma_e4m3(tmem + (uint32_t)(buf * 256), ad + (uint64_t)(2 * k), bd + (uint64_t)(2 * k), idesc, k ? 1u : 0u);
        tc_commit(smem_at(&s_empty[s]));
        tc_commit(smem_at(&s_done[buf]));
      }
      if (!ok) {
        tc_commit(smem_at(&s_tail));
        mbar_wait(smem_at(&s_tail), 0u, gave_up, t.wait_ns > kDrainFloorNs ? t.wait_ns : kDrainFloorNs, false);
      }
    }
    __syncwarp();
  } else {
    const int g = (warp - 2) >> 2, q = warp & 3;
    const int row = row0 + q * 32 + lane;
    const uint32_t lanes = tmem + ((uint32_t)(q * 32) << 16) + (uint32_t)(g * 64);
    const bool live = row < t.n_rows;
    const float *as = t.a_scale + (live ? (long long)row : 0) * t.a_scale_stride;
    const int last_block = (t.n + 127) / 128 - 1;
    const float *ws0 = t.w_scale[0] + (size_t)(n0 / 128) * t.n_kb;
    const float *ws1 = W == 2 ? t.w_scale[1] + (size_t)(n0 / 128) * t.n_kb : t.w_scale[0] + (size_t)min(n0 / 128 + 1, last_block) * t.n_kb;
    float acc[2][64];
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int i = 0; i < 64; ++i) acc[h][i] = 0.f;
    for (int b = 0; b < t.n_kb; ++b) {
      const int buf = b & 1;
      const float sa = live ? __ldg(as + b) : 0.f, f[2] = {sa * __ldg(ws0 + b), sa * __ldg(ws1 + b)};
      mbar_wait(smem_at(&s_done[buf]), (uint32_t)((b >> 1) & 1), gave_up, t.wait_ns);
      __syncwarp();
      tc_fence_after();
#pragma unroll
      for (int h = 0; h < 2; ++h) {
#pragma unroll
        for (int p = 0; p < 64; p += 32) {
          uint32_t d[32];
          tc_ld(lanes + (uint32_t)(buf * 256 + h * 128 + p), d);
          tc_ld_wait();
          if (h == 1 && p == 32) {
            tc_fence_before();
            mbar_arrive(smem_at(&s_read[buf]));
          }
#pragma unroll
          for (int i = 0; i < 32; ++i) acc[h][p + i] = fmaf(__uint_as_float(d[i]), f[h], acc[h][p + i]);
        }
      }
    }
    // ------------------------------------------------------------ results
    if constexpr (W == 2) {
#pragma unroll
      for (int i = 0; i < 64; ++i) acc[0][i] = gate_of(acc[0][i], acc[1][i]);
      if (t.out_dtype == D3_E4M3) {   // the block of scales is 128 columns: two threads have a row's
        float top = 0.f;
#pragma unroll
        for (int i = 0; i < 64; ++i)
          if (n0 + g * 64 + i < t.n) top = max_nan(top, fabsf(acc[0][i]));
        s_top[g][q * 32 + lane] = top;
        asm volatile("bar.sync 1, 256;" ::: "memory");
        top = max_nan(top, s_top[g ^ 1][q * 32 + lane]);
        float inverse;
        const float scale = block_scale(top, inverse);
        if (live) {
          if (g == 0) t.scale[row * t.scale_stride + n0 / 128] = scale;
          unsigned char *o = static_cast<unsigned char *>(t.out) + row * t.out_stride + n0 + g * 64;
#pragma unroll
          for (int i = 0; i < 64; i += 4) {
            const uint32_t v = pack_e4m3(acc[0][i] * inverse, acc[0][i + 1] * inverse, acc[0][i + 2] * inverse, acc[0][i + 3] * inverse);
            if (t.out_wide && n0 + g * 64 + i + 3 < t.n) {
              *reinterpret_cast<uint32_t *>(o + i) = v;
            } else {
#pragma unroll
              for (int j = 0; j < 4; ++j)
                if (n0 + g * 64 + i + j < t.n) o[i + j] = (unsigned char)(v >> (8 * j));
            }
          }
        }
      }
    }
    if (live && t.out_dtype != D3_E4M3) {
#pragma unroll
      for (int h = 0; h < (W == 2 ? 1 : 2); ++h) {
#pragma unroll
        for (int i = 0; i < 64; i += 4) {
          const int c = n0 + h * 128 + g * 64 + i;
          const long long at = row * t.out_stride + c;
          if (t.out_wide && c + 3 < t.n) {
            if (t.out_dtype == D3_FP32)
              *reinterpret_cast<float4 *>(static_cast<float *>(t.out) + at) = make_float4(acc[h][i], acc[h][i + 1], acc[h][i + 2], acc[h][i + 3]);
            else
              *reinterpret_cast<uint2 *>(static_cast<char *>(t.out) + 2 * at) =
                  make_uint2(pack2(acc[h][i], acc[h][i + 1], t.out_dtype), pack2(acc[h][i + 2], acc[h][i + 3], t.out_dtype));
          } else {
#pragma unroll
            for (int j = 0; j < 4; ++j)
              if (c + j < t.n) store1(t.out, at + j, t.out_dtype, acc[h][i + j]);
          }
        }
      }
    }
  }
  if (tid == 0 && *gave_up && t.status) *t.status = D3_ETIMEOUT;
  tc_fence_before();
  __syncthreads();
  if (warp == 1)
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"((uint32_t)kColumns) : "memory");
}

template <int W>
cudaError_t launch(const TMap &w0, const TMap &w1, const TMap &ma, Mm8Args &p, cudaStream_t st) {
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  if (dev < 0 || dev >= 64) return cudaErrorInvalidDevice;
  constexpr int smem = kStages * kStage + 1024;
  static std::atomic<bool> ready[64];
  if (!ready[dev].load(std::memory_order_acquire)) {
    if ((e = cudaFuncSetAttribute(k_mm8_many<W>, cudaFuncAttributeMaxDynamicSharedMemorySize, smem)) != cudaSuccess) return e;
    ready[dev].store(true, std::memory_order_release);
  }
  const int wide = W == 2 ? 128 : 256;
  const CUtensorMap *m0 = reinterpret_cast<const CUtensorMap *>(&w0), *m1 = reinterpret_cast<const CUtensorMap *>(&w1),
                    *m = reinterpret_cast<const CUtensorMap *>(&ma);
  return launch_pdl(k_mm8_many<W>, dim3((unsigned)((p.n + wide - 1) / wide), (unsigned)((p.n_rows + kM - 1) / kM)), dim3(kThreads), smem, st,
                    *m0, *m1, *m, p);
}

}  // namespace

cudaError_t launch_mm8_many(const TMap &w0, const TMap *w1, const void *a, int64_t a_stride, Mm8Args &p, cudaStream_t st) {
  TMap ma;
  if (!encode_rows8(&ma, a, p.n_rows, p.k, a_stride, kM)) return cudaErrorInvalidValue;
  return w1 ? launch<2>(w0, *w1, ma, p, st) : launch<1>(w0, w0, ma, p, st);
}

}  // namespace d3
