// Products of few rows in 8 bits with a weight matrix in 8 bits: weights stream, rows ride along.
//
//   y[row][r] = sum_b as[row][b] ws[r / 128][b] sum_{k in block b} a[row][k] w[r][k]
//
// Few rows leave 2 * rows flops for a byte of weight: the kernel is bound by reading the weights once.  A tile of 128 weight rows is
// the tensor core's M and the rows of the call are its N (16..128, rows beyond n_rows are zeros): all 128 lanes of the sums
// are in use, and an epilogue thread (one weight row) has no more columns than there are rows.  (With the rows as M, tiles can be as
// narrow as 16 weight rows and k need not be cut, but an instruction takes 40 cycles for its 128 lanes whatever its N, and
// one warp has all the sums to fetch: 32 rows, 11008 -> 4096, took 15 us.)
//
// A block of 128 k is four tcgen05.mma.  Every block has scales of its own, so its sum is fetched from tensor memory, multiplied by
// the two scales and added to registers; that is handed over a unit of U blocks at a time, while the next unit is
// multiplied into the other half of the tensor memory.
//
// A CTA has one tile (gated: of both matrices) for N rows.  Where that makes too few CTAs, k is cut between those of a cluster, whose
// sums meet in distributed shared memory in the order of their ranks; more CTAs cost more than they give (clusters are
// started one after another).  us by the number of CTAs: 1 row, 4096 -> 12288: 96 11.9, 192 12.8, 288 17.6;
// 32 rows, 11008 -> 4096: 32 24.4, 64 16.0, 128 12.5, 256 13.7; 4 rows, 8192 -> 10240: 80 19.6, 160 17.1, 320 21.8; gated,
// 8 rows, 5120 -> 13824: 108 25.9, 216 26.3.
//
// What is left over the time of the weights at the memory's rate is some 4 us a call: the last sums and results 1.2, the step from
// one call to the next 1 to 1.4, the first copies' way 1.5.  A CTA of one matrix and up to 64 rows takes at most half of an SM, so the
// next call's CTAs are set up beside it; one of two matrices (three stages in half of an SM would be too few) or of 128 rows takes
// a whole one.  Letting them ask for weights ahead of their turn gave nothing (copies
// into the ring 12.5 us where this takes 11.9) or cost (into L2 box by box 14.0, row by row 18.4).
#include <math.h>

#include <atomic>

#include "d3_block8.cuh"

namespace d3 {

namespace {

constexpr int kTileBytes = 128 * 128;            // a block's share of a weight matrix
constexpr int kMaxStages = 12;
constexpr int kChunk = 8, kChunks = 3;           // scales come in chunks of 8 blocks, through a ring of their own
constexpr int kMostSplit = 8;
constexpr int kHalfSmem = 112 * 1024, kWholeSmem = 213 * 1024;      // dynamic shared memory, of one of two CTAs on an SM or a CTA alone

__device__ __forceinline__ uint32_t cluster_rank() {
  uint32_t r;
  asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
  return r;
}
__device__ __forceinline__ float4 cluster_load4(uint32_t at, uint32_t rank) {
  uint32_t remote;
  float4 v;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(remote) : "r"(at), "r"(rank));
  asm volatile("ld.shared::cluster.v4.f32 {%0,%1,%2,%3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(remote) : "memory");
  return v;
}
__device__ __forceinline__ uint64_t mul_two(uint64_t a, uint64_t b) {
  uint64_t r;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}

// C: rows (accumulator columns) of an epilogue thread, G: warpgroups that share the rows, W: weight matrices (2: gated), U: blocks of a unit
template <int C, int G, int W, int U>
struct Few {
  static constexpr int N = C * G;                              // padded rows
  static constexpr int kThreads = 128 + 128 * G;               // copies, products, scales, an idle warp; epilogue warps
  static constexpr int kColumns = U * W * N;                   // accumulator columns of a unit, of which there are two
  static constexpr bool kHalf = 2 * kColumns <= 256;           // two CTAs' columns fit into an SM's tensor memory
  static constexpr int kStage = W * kTileBytes + N * 128;      // a block
  static constexpr int kSums = W * N * 128 * 4;                // one CTA's sums, over the ring when it is empty
  // 256 threads start with 128 registers, 384 with 168; the epilogue takes 200 (216) of them and leaves 56 (72) to the others
  // (128 * 56 + 128 * 200 = 256 * 128, 128 * 72 + 256 * 216 = 384 * 168)
  static constexpr int kRegsControl = G == 1 ? 56 : 72, kRegsSums = G == 1 ? 200 : 216;
  static_assert(kColumns <= 256, "tensor memory");
};

struct FewArgs {
  Mm8Args m;
  int stages, split;
  int wide;                // four results at a time may be written in one piece
  int late;                // the next call may begin when this one's copies are asked for, and not at once
};

// A warp has the 128 results of a row that one tile of weight rows gives, lane l those at n0 = 128 tile + 4 l: rounds and writes
// them, in 8 bits with the block's scale or in a wider type.  What is behind the last column counts and writes nothing.
__device__ __forceinline__ void finish4(const FewArgs &t, long long row, int n0, const float (&y)[4], int tile, int lane) {
  const Mm8Args &m = t.m;
  const long long at = row * m.out_stride + n0;
  if (m.out_dtype == D3_E4M3) {
    float top = 0.f;
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (n0 + i < m.n) top = max_nan(top, fabsf(y[i]));
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) top = max_nan(top, __shfl_xor_sync(0xffffffffu, top, o));
    BlockScale b = block_scale(top);
    if (lane == 0) m.scale[row * m.scale_stride + tile] = b.scale;
    const float up = lift(b) ? kLift : 1.f;
    const uint32_t q = quantize4(y[0] * up, y[1] * up, y[2] * up, y[3] * up, b);
    unsigned char *o = static_cast<unsigned char *>(m.out) + at;
    if (t.wide && n0 + 3 < m.n) {
      *reinterpret_cast<uint32_t *>(o) = q;
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (n0 + i < m.n) o[i] = (unsigned char)(q >> (8 * i));
    }
  } else if (t.wide && n0 + 3 < m.n) {
    if (m.out_dtype == D3_FP32) *reinterpret_cast<float4 *>(static_cast<float *>(m.out) + at) = make_float4(y[0], y[1], y[2], y[3]);
    else *reinterpret_cast<uint2 *>(static_cast<char *>(m.out) + 2 * at) = make_uint2(pack2(y[0], y[1], m.out_dtype), pack2(y[2], y[3], m.out_dtype));
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (n0 + i < m.n) store1(m.out, at + i, m.out_dtype, y[i]);
  }
}

template <int C, int G, int W, int U>
__global__ void __launch_bounds__(Few<C, G, W, U>::kThreads, G == 1 ? 2 : 1)
k_mm8_few(const __grid_constant__ CUtensorMap map_w0, const __grid_constant__ CUtensorMap map_w1, const __grid_constant__ CUtensorMap map_a,
          const __grid_constant__ FewArgs t) {
  using F = Few<C, G, W, U>;
  constexpr int N = F::N;
  extern __shared__ unsigned char raw[];
  __shared__ __align__(8) uint64_t s_full[kMaxStages], s_empty[kMaxStages], s_done[2], s_read[2], s_there[kChunks], s_used[kChunks], s_tail, s_never;
  __shared__ __align__(16) float s_rows[kChunks][kChunk][N], s_weights[kChunks][kChunk][2];
  __shared__ uint32_t s_tmem;
  __shared__ int s_gave_up;
  const int tid = threadIdx.x, warp = __shfl_sync(0xffffffffu, tid >> 5, 0), lane = tid & 31;
  const int S = t.stages, split = t.split;
  const int tile = blockIdx.x / split, rank = split > 1 ? (int)cluster_rank() : 0, row0 = blockIdx.y * N;
  // this CTA's blocks of k: whole chunks of scales, but for the end
  const int chunks = (t.m.n_kb + kChunk - 1) / kChunk;
  const int b0 = min(chunks * rank / split * kChunk, t.m.n_kb), b1 = min(chunks * (rank + 1) / split * kChunk, t.m.n_kb);
  const int units = (b1 - b0 + U - 1) / U;
  const uint32_t ring = (smem_at(raw) + 1023u) & ~1023u;       // the swizzle goes by the address
  volatile int *gave_up = &s_gave_up;
  if (tid == 32) {
    const uint32_t copies = t.m.stall && blockIdx.x == 0 && blockIdx.y == 0 ? 2 : 1;
    for (int s = 0; s < S; ++s) { mbar_init(smem_at(&s_full[s]), copies); mbar_init(smem_at(&s_empty[s]), 1); }
    for (int b = 0; b < 2; ++b) { mbar_init(smem_at(&s_done[b]), 1); mbar_init(smem_at(&s_read[b]), 4 * G); }
    for (int c = 0; c < kChunks; ++c) { mbar_init(smem_at(&s_there[c]), 32); mbar_init(smem_at(&s_used[c]), 4 * G); }
    mbar_init(smem_at(&s_tail), 1);
    mbar_init(smem_at(&s_never), 1);
    s_gave_up = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
  }
  if (warp == 1) {
    __syncwarp();
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_at(&s_tmem)), "r"(F::kHalf ? 256u : 512u) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = s_tmem;
  pdl_wait();
  if (!t.late) pdl_trigger();

  if (warp < 4) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(F::kRegsControl));
    // (a whole warp runs each of the loops below, so that their arithmetic is the warp's and not a lane's)
    if (warp == 0) {
      // ---------------------------------------------------------- copies
      const bool one = elect_one();
      int s = 0, phase = 1, b = b0;
      for (; b < b1; ++b) {
        if (b - b0 >= S && !mbar_wait(smem_at(&s_empty[s]), (uint32_t)phase, gave_up, t.m.wait_tries)) break;
        const uint32_t full = smem_at(&s_full[s]), at = ring + (uint32_t)(s * F::kStage);
        if (one) {
          mbar_expect(full, F::kStage);
          tma_rows8(at, &map_w0, b * 128, tile * 128, full);
          if (W == 2) tma_rows8(at + kTileBytes, &map_w1, b * 128, tile * 128, full);
          tma_rows8(at + W * kTileBytes, &map_a, b * 128, row0, full);
        }
        if (++s == S) { s = 0; phase ^= 1; }
      }
      __syncwarp();
      if (t.late) pdl_trigger();
    } else if (warp == 1) {
      // ---------------------------------------------------------- products
      constexpr uint32_t idesc = idesc_e4m3(128, N);
      const bool one = elect_one();
      bool ok = true;
      int s = 0, phase = 0;
      for (int u = 0; u < units && ok; ++u) {
        const int buf = u & 1, blocks = min(U, b1 - b0 - u * U);
        if (u >= 2) ok = mbar_wait(smem_at(&s_read[buf]), (uint32_t)(((u >> 1) - 1) & 1), gave_up, t.m.wait_tries);
#pragma unroll 1
        for (int b = 0; b < blocks && ok; ++b) {
          ok = mbar_wait(smem_at(&s_full[s]), (uint32_t)phase, gave_up, t.m.wait_tries);
          if (!ok) break;
          tc_fence_after();
          const uint32_t at = ring + (uint32_t)(s * F::kStage), to = tmem + (uint32_t)(buf * F::kColumns + b * W * N);
          const uint64_t ad = desc_rows8(at + W * kTileBytes);
          if (one) {
#pragma unroll
            for (int w = 0; w < W; ++w) {
              const uint64_t wd = desc_rows8(at + w * kTileBytes);
#pragma unroll
              for (int k = 0; k < 4; ++k)   // 32 numbers = 32 bytes = 2 descriptor units
                tc_mma_e4m3(to + (uint32_t)(w * N), wd + (uint64_t)(2 * k), ad + (uint64_t)(2 * k), idesc, k ? 1u : 0u);
            }
            if (b == blocks - 1) tc_commit(smem_at(&s_done[buf]));
            tc_commit(smem_at(&s_empty[s]));
          }
          if (++s == S) { s = 0; phase ^= 1; }
        }
      }
      if (!ok) {        // what was issued still reads shared memory and writes tensor memory
        if (one) tc_commit(smem_at(&s_tail));
        mbar_wait(smem_at(&s_tail), 0u, gave_up, max(t.m.wait_tries, kDrainTries), false);
      }
      __syncwarp();
    } else if (warp == 2) {
      // ---------------------------------------------------------- scales: of the rows, and of the tile's weight rows
      const int rows = min(N, t.m.n_rows - row0);
      const float *as = t.m.a_scale + row0 * t.m.a_scale_stride;
      for (int c = 0, b = b0; b < b1; ++c, b += kChunk) {
        const int slot = c % kChunks, fill = c / kChunks;
        if (fill > 0 && !mbar_wait(smem_at(&s_used[slot]), (uint32_t)((fill - 1) & 1), gave_up, t.m.wait_tries)) break;
        const int in = lane & 7, kb = min(b + in, b1 - 1);
        for (int r = lane >> 3; r < rows; r += 4) copy4(smem_at(&s_rows[slot][in][r]), as + r * t.m.a_scale_stride + kb);
        if (lane < 8 * W) copy4(smem_at(&s_weights[slot][in][lane >> 3]), t.m.w_scale[lane >> 3] + (size_t)tile * t.m.n_kb + kb);
        asm volatile("cp.async.mbarrier.arrive.noinc.shared::cta.b64 [%0];" ::"r"(smem_at(&s_there[slot])) : "memory");
      }
      asm volatile("cp.async.wait_all;" ::: "memory");
    }
  } else {
    // ------------------------------------------------------------ sums
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(F::kRegsSums));
    const int g = (warp - 4) >> 2, q = warp & 3;                  // a warp reads the quarter of the lanes that its number names
    const int r = q * 32 + lane;                                  // weight row of the tile
    const uint32_t lanes = tmem + ((uint32_t)(q * 32) << 16) + (uint32_t)(g * C);
    constexpr int P = C < 32 ? C : 32;                            // columns of a load
    uint64_t acc[W][C / 2];                                       // two rows each
#pragma unroll
    for (int w = 0; w < W; ++w)
#pragma unroll
      for (int i = 0; i < C / 2; ++i) acc[w][i] = 0ull;
    int slot = 0, there = 0, in = 0;
    for (int u = 0; u < units; ++u) {
      const int buf = u & 1, blocks = min(U, b1 - b0 - u * U);
      if (in == 0) mbar_wait(smem_at(&s_there[slot]), (uint32_t)there, gave_up, t.m.wait_tries);
      mbar_wait(smem_at(&s_done[buf]), (uint32_t)((u >> 1) & 1), gave_up, t.m.wait_tries);   // (given up: numbers without meaning)
      __syncwarp();
      tc_fence_after();
#pragma unroll 1
      for (int b = 0; b < blocks; ++b) {
        const uint32_t from = lanes + (uint32_t)(buf * F::kColumns + b * W * N);
        const float *as = &s_rows[slot][in + b][g * C], *ws = s_weights[slot][in + b];
#pragma unroll
        for (int w = 0; w < W; ++w) {
          const uint64_t f = two_of(__float_as_uint(ws[w]), __float_as_uint(ws[w]));
#pragma unroll
          for (int p = 0; p < C; p += P) {
            uint32_t d[P];
            tc_ld(from + (uint32_t)(w * N + p), d);
            tc_ld_wait(d);
#pragma unroll
            for (int i = 0; i < P; i += 4) {
              const uint4 a = *reinterpret_cast<const uint4 *>(as + p + i);
              fma_two(acc[w][(p + i) / 2], two_of(d[i], d[i + 1]), mul_two(two_of(a.x, a.y), f));
              fma_two(acc[w][(p + i) / 2 + 1], two_of(d[i + 2], d[i + 3]), mul_two(two_of(a.z, a.w), f));
            }
          }
        }
      }
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(smem_at(&s_read[buf]));
      in += U;
      if (in == kChunk || u == units - 1) {
        if (lane == 0) mbar_arrive(smem_at(&s_used[slot]));
        in = 0;
        if (++slot == kChunks) { slot = 0; there ^= 1; }
      }
    }
    // every copy has landed and every product is done: the ring holds the sums now, [matrix][row of the call][weight row]
    float *sums = reinterpret_cast<float *>(raw + (ring - smem_at(raw)));
    group_sync(1, 128 * G);
#pragma unroll
    for (int w = 0; w < W; ++w)
#pragma unroll
      for (int i = 0; i < C; ++i) sums[(w * N + g * C + i) * 128 + r] = i & 1 ? high_of(acc[w][i / 2]) : low_of(acc[w][i / 2]);
  }

  if (split > 1) cluster_sync();
  else __syncthreads();
  const int rows = min(N, t.m.n_rows - row0), n0 = tile * 128 + 4 * lane;
  for (int j = rank + split * warp; j < rows; j += split * (F::kThreads / 32)) {
    float y[W][4];
#pragma unroll
    for (int w = 0; w < W; ++w) {
      const uint32_t at = ring + (uint32_t)(((w * N + j) * 128 + 4 * lane) * 4);
      float4 sum;
      if (split == 1) {
        sum = *reinterpret_cast<const float4 *>(raw + (at - smem_at(raw)));
      } else {
        float4 part[kMostSplit];
#pragma unroll
        for (int p = 0; p < kMostSplit; ++p)
          if (p < split) part[p] = cluster_load4(at, (uint32_t)p);
        sum = part[0];
#pragma unroll
        for (int p = 1; p < kMostSplit; ++p)
          if (p < split) { sum.x += part[p].x; sum.y += part[p].y; sum.z += part[p].z; sum.w += part[p].w; }
      }
      y[w][0] = sum.x; y[w][1] = sum.y; y[w][2] = sum.z; y[w][3] = sum.w;
    }
    if constexpr (W == 2) {
#pragma unroll
      for (int i = 0; i < 4; ++i) y[0][i] = gate_of(y[0][i], y[1][i]);
    }
    finish4(t, row0 + j, n0, y[0], tile, lane);
  }
  if (*gave_up && warp == 0) {     // copies may be in flight, which must land before the CTA's shared memory is given back
    mbar_wait(smem_at(&s_never), 0u, gave_up, kDrainTries, false);
    if (lane == 0 && t.m.status) *t.m.status = D3_ETIMEOUT;
  }
  tc_fence_before();
  if (split > 1) cluster_sync();   // no CTA's sums go while another one reads them
  else __syncthreads();
  if (warp == 1)
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(F::kHalf ? 256u : 512u) : "memory");
}

template <int C, int G, int W, int U>
cudaError_t launch(const TMap &w0, const TMap &w1, const TMap &ma, const Mm8Args &p, int split, int dev, cudaStream_t st) {
  using F = Few<C, G, W, U>;
  static std::atomic<bool> ready[64];   // the shared-memory attribute is per device; setting it twice is harmless
  if (!ready[dev].load(std::memory_order_acquire)) {
    const cudaError_t e = cudaFuncSetAttribute(k_mm8_few<C, G, W, U>, cudaFuncAttributeMaxDynamicSharedMemorySize, kWholeSmem);
    if (e != cudaSuccess) return e;
    ready[dev].store(true, std::memory_order_release);
  }
  FewArgs t;
  t.m = p;
  const int fixed = kChunks * kChunk * (F::N + 2) * 4 + 1024 + 1024;      // static shared memory, and the alignment of the ring
  int stages = (kHalfSmem - fixed) / F::kStage;
  const bool shared = F::kHalf && G == 1 && stages >= 4;                  // two CTAs fit on an SM (one matrix, up to 64 rows)
  if (!shared) stages = (kWholeSmem - fixed) / F::kStage;
  if (stages > kMaxStages) stages = kMaxStages;
  const int least = (F::kSums + F::kStage - 1) / F::kStage;               // the ring holds the sums in the end
  if (stages < least) stages = least;
  const int tiles = (p.n + 127) / 128;
  t.stages = stages;
  t.split = split;
  // Where some SMs have two CTAs, those of a call that begins early take places that even them out (4 rows, 8192 -> 10240, call
  // after call: 20.4 us, begun late 18.2; 1 row, 4096 -> 12288, one CTA an SM: 11.8, late 12.0).  Where a CTA has an SM to itself there is
  // no place to take (gated 8 x 8192 -> 28672, call after call: 74.0, late 74.0; 32 rows of it 78.9 and 79.0).
  t.late = shared && (long long)tiles * split * ((p.n_rows + F::N - 1) / F::N) > 148;
  const int es = type_bytes(p.out_dtype);
  t.wide = on_bytes(p.out, 4 * es) && (p.n_rows == 1 || p.out_stride % 4 == 0);
  cudaLaunchConfig_t cfg;
  memset(&cfg, 0, sizeof(cfg));
  cfg.gridDim = dim3((unsigned)(tiles * split), (unsigned)((p.n_rows + F::N - 1) / F::N));
  cfg.blockDim = dim3(F::kThreads);
  cfg.dynamicSmemBytes = (size_t)stages * F::kStage + 1024;
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
  return cudaLaunchKernelEx(&cfg, k_mm8_few<C, G, W, U>, *m0, *m1, *m, static_cast<const FewArgs>(t));
}

// What a call takes with N rows a CTA and k cut in `split`, in us, as measured: a block of k takes a CTA 0.24 us (N = 16, 32), 0.315
// (64) or 0.48 (128), gated 0.335, 0.42, 0.76 and 0.95; two CTAs on an SM 1.35 times that (N = 64: 1.8); CTAs that find no
// place at first 6 us more; the memory gives 6.3 TB/s, L2 13; a call costs 3.3 us, clusters of 2, 4 and 8 CTAs 0.5, 1 and 3.5
// more.  (rows x k x n, estimate / measured, and the other kernel: 128 x 8192 x 1024: N 32 in 4 8.1 / 7.9, 32; 256 x 8192 x 1024:
// 64 in 4 9.3 / 9.9, 32; 300 x 28672 x 500: 64 in 4 21.9 / 23.7, 136; 512 x 4096 x 512: 64 in 4 6.8 / 7.0, 18.4; 2000 x 11008 x
// 300: 128 in 2 24.4 / 28.8, 80; gated 64 x 4096 x 11008: 64 27.6 / 29.0, 37.6; 128 rows of it: 128 33.7 / 35.0, 38.1.)
float few_us(const Mm8Args &p, int mats, int N, int split) {
  constexpr float kSms = 148.f;
  const float rows = (float)((p.n_rows + N - 1) / N), tiles = (float)((p.n + 127) / 128), ctas = rows * tiles * split;
  const float blocks = (float)((((p.n_kb + kChunk - 1) / kChunk + split - 1) / split) * kChunk), kb = blocks < p.n_kb ? blocks : (float)p.n_kb;
  const float each = mats == 2 ? (N == 16 ? 0.335f : N == 32 ? 0.42f : N == 64 ? 0.76f : 0.95f) : (N <= 32 ? 0.24f : N == 64 ? 0.315f : 0.48f);
  const bool shared = mats == 1 && N <= 64;                      // two CTAs fit on an SM
  const float on_sm = ceilf(ctas / kSms), waves = shared ? (on_sm > 2.f ? on_sm / 2.f : 1.f) : on_sm;
  float work = waves * kb * each * (shared && on_sm > 1.f ? (N == 64 ? 1.8f : 1.35f) : 1.f) + 6.f * (waves - 1.f);
  if (!shared && split == kMostSplit && ctas > 64.f) work *= 2.f; // (eight SMs at a time do not come out even)
  const float memory = (float)p.n * p.k * mats / 6.3e6f, l2 = ctas * kb * (mats * 16384.f + N * 128.f) / 13e6f;
  const float most = work > memory ? (work > l2 ? work : l2) : (memory > l2 ? memory : l2);
  return most + 3.3f + (split == 1 ? 0.f : split == 2 ? 0.5f : split == 4 ? 1.f : 3.5f);
}

}  // namespace

float plan_mm8_few(const Mm8Args &p, int mats, FewPlan &plan) {
  float best = INFINITY;
  for (int N = 16; N <= 128; N *= 2) {
    if (N > 16 && N / 2 >= p.n_rows) break;                      // half of it would do
    if ((p.n_rows + N - 1) / N > 65535) continue;
    for (int split = 1; split <= kMostSplit && split <= (p.n_kb + kChunk - 1) / kChunk; split *= 2) {
      const float us = few_us(p, mats, N, split);
      if (us < best) { best = us; plan.rows = N; plan.split = split; }
    }
  }
  return best;
}

cudaError_t launch_mm8_few(const TMap &w0, const TMap *w1, const void *a, int64_t a_stride, const Mm8Args &p, const FewPlan &plan, cudaStream_t st) {
  int dev = 0;
  const cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  if (dev < 0 || dev >= 64) return cudaErrorInvalidDevice;
  TMap ma;
  if (!encode_rows8(&ma, a, p.n_rows, p.k, a_stride, plan.rows)) return cudaErrorInvalidValue;
  const int s = plan.split;
  if (w1) {
    switch (plan.rows) {
      case 16: return launch<16, 1, 2, 4>(w0, *w1, ma, p, s, dev, st);
      case 32: return launch<32, 1, 2, 2>(w0, *w1, ma, p, s, dev, st);
      case 64: return launch<64, 1, 2, 1>(w0, *w1, ma, p, s, dev, st);
      default: return launch<64, 2, 2, 1>(w0, *w1, ma, p, s, dev, st);
    }
  }
  switch (plan.rows) {
    case 16: return launch<16, 1, 1, 4>(w0, w0, ma, p, s, dev, st);
    case 32: return launch<32, 1, 1, 4>(w0, w0, ma, p, s, dev, st);
    case 64: return launch<64, 1, 1, 2>(w0, w0, ma, p, s, dev, st);
    default: return launch<64, 2, 1, 1>(w0, w0, ma, p, s, dev, st);
  }
}

}  // namespace d3
