// Products of many rows in 8 bits with a weight matrix in 8 bits.
//
//   y[row][r] = sum_b as[row][b] ws[r / 128][b] sum_{k in block b} a[row][k] w[r][k]
//
// Bound by the tensor cores: 2 flops for every (row, weight row, k).  Two CTAs, a cluster, share a tile of 256 rows x 256 weight
// rows (gated: 128 of each matrix): one tcgen05.mma of cta_group::2 multiplies both CTAs' 128 rows with the 256 weight
// rows, of which each CTA has brought half, so a byte of shared memory is read for twice the work.  A block of 128 k is
// four of them, whose sum, 128 x 256 in each CTA, goes to one of two buffers in tensor memory.  Every block has scales of its own:
// while the next block is multiplied, eight epilogue warps fetch the sum, multiply it by its two scales and add it to
// registers (a thread has one row, 64 columns of each half; two numbers an instruction).  The grid is persistent, a pair
// of CTAs for each pair of SMs; results go through shared memory and leave as bulk copies while the next tile begins.
//
// Times in this file are those of short runs at full clock; in a loop of such calls the power cap (990 W, 1.48 GHz) takes a sixth more
// (8191 x 8192 x 8192: 464 us, in a loop 540 to 575).
#include <math.h>

#include <atomic>

#include "d3_block8.cuh"

namespace d3 {

namespace {

constexpr int kBox = 128 * 128;                  // bytes of 128 rows of a stage
constexpr int kStage = 2 * kBox;                 // a CTA's rows, and its half of the weight rows
constexpr int kStages = 5;
constexpr int kOutBytes = 32 * 1024;             // results on their way out
constexpr int kThreads = 384;                    // copies, products and two idle warps; eight epilogue warps
constexpr int kColumns = 512;
constexpr int kSmem = kStages * kStage + kOutBytes + 1024;
constexpr int kChunk = 4, kChunks = 8;           // scales come in chunks of 4 blocks, through a ring of their own, and are taken 4 at a time
constexpr int kGroupM = 16;                      // tiles of rows that are taken together: their a and the weights beside them stay in L2 (2: 482 us, 4: 483, 8: 474, 16: 470)
// Registers: 384 threads start with 168; the epilogue's two warpgroups take 216 and leave 72 to the third
// (128 * 72 + 256 * 216 = 384 * 168).
constexpr int kRegsControl = 72, kRegsSums = 216;

__device__ __forceinline__ uint32_t pair_rank() {
  uint32_t r;
  asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
  return r;
}
__device__ __forceinline__ uint32_t at_first(uint32_t local) {   // the same place in the first CTA of the pair
  uint32_t r;
  asm volatile("mapa.shared::cluster.u32 %0, %1, 0;" : "=r"(r) : "r"(local));
  return r;
}
__device__ __forceinline__ void pair_arrive(uint32_t bar) {
  asm volatile("mbarrier.arrive.shared::cluster.b64 _, [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ void pair_load(uint32_t dst, const void *map, int x, int y, uint32_t bar) {
  asm volatile("cp.async.bulk.tensor.2d.shared::cluster.global.tile.mbarrier::complete_tx::bytes.cta_group::2 [%0], [%1, {%2, %3}], [%4];"
               ::"r"(dst), "l"(reinterpret_cast<uint64_t>(map)), "r"(x), "r"(y), "r"(bar) : "memory");
}
__device__ __forceinline__ void pair_mma(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t add) {
  asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\ttcgen05.mma.cta_group::2.kind::f8f6f4 [%0], %1, %2, %3, p;\n\t}"
               ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(add) : "memory");
}
// an arrival at this place in both CTAs once everything given to the tensor cores so far is done
__device__ __forceinline__ void pair_commit(uint32_t bar) {
  asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;" ::"r"(bar), "h"((uint16_t)3)
               : "memory");
}
__device__ __forceinline__ void store_box(const void *map, uint32_t from, int x, int y) {
  asm volatile("cp.async.bulk.tensor.2d.global.shared::cta.tile.bulk_group [%0, {%1, %2}], [%3];"
               ::"l"(reinterpret_cast<uint64_t>(map)), "r"(x), "r"(y), "r"(from) : "memory");
}
__device__ __forceinline__ void store16(uint32_t at, uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
  asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(at), "r"(a), "r"(b), "r"(c), "r"(d) : "memory");
}

struct ManyArgs {
  Mm8Args m;
  int tiles_m, tiles_n;
  int bulk;                // results may leave as bulk copies (their rows lie on 16 bytes)
  int whole;               // the columns that do: whole pieces of 16 bytes, behind which such a copy would write the rest of the last piece
};

// A warpgroup's box is written: it leaves for the columns from c0 on.
__device__ __forceinline__ void copy_out(const ManyArgs &t, const CUtensorMap &map, uint32_t from, int c0, int row0, int g, int warp, int lane) {
  asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
  group_sync(1 + g, 128);
  if ((warp & 3) == 0 && lane == 0 && c0 < t.whole && row0 < t.m.n_rows) {
    store_box(&map, from, c0, row0);
    asm volatile("cp.async.bulk.commit_group;" ::: "memory");
  }
}

// a number of a box, at row r and `byte` of its 128
template <typename T>
__device__ __forceinline__ T box_number(uint32_t from, int r, uint32_t byte) {
  const uint32_t at = from + (uint32_t)(r * 128) + (((byte >> 4) ^ (uint32_t)(r & 7)) << 4) + (byte & 15u);
  uint32_t v;
  if (sizeof(T) == 4) asm volatile("ld.shared.u32 %0, [%1];" : "=r"(v) : "r"(at) : "memory");
  else if (sizeof(T) == 2) asm volatile("{\n\t.reg .u16 h;\n\tld.shared.u16 h, [%1];\n\tcvt.u32.u16 %0, h;\n\t}" : "=r"(v) : "r"(at) : "memory");
  else asm volatile("ld.shared.u8 %0, [%1];" : "=r"(v) : "r"(at) : "memory");
  return (T)v;
}
// The columns that no bulk copy takes, fewer than 16 bytes of a row: a thread writes those that it has put into the box itself.
template <typename T, int kColumns>
__device__ __forceinline__ void copy_rest(const ManyArgs &t, uint32_t from, int first_byte, int c0, int row, int r) {
  if (t.whole == t.m.n || row >= t.m.n_rows) return;
#pragma unroll 1
  for (int c = max(t.whole - c0, 0); c < min(t.m.n - c0, kColumns); ++c)
    static_cast<T *>(t.m.out)[row * t.m.out_stride + c0 + c] = box_number<T>(from, r, (uint32_t)(first_byte + c * (int)sizeof(T)));
}

// The same for results whose rows do not lie on 16 bytes: every warp writes the rows that its lanes have put into shared memory,
// neighbouring lanes neighbouring numbers.  (Number by number from the lanes' registers, 32 rows at a time, 2000 x 4096 ->
// 5001 took 121 us in fp32 and 159 in bf16, and gated in e4m3 176; this takes 75, 62 and 91.)
template <typename T, int kColumns>
__device__ __forceinline__ void copy_lines(const ManyArgs &t, uint32_t from, int first_byte, int c0, int row0, int q, int lane) {
  __syncwarp();
#pragma unroll 4
  for (int i = 0; i < 32; ++i) {
    const int r = q * 32 + i;
    if (row0 + r >= t.m.n_rows) break;
    T *out = static_cast<T *>(t.m.out) + (row0 + r) * t.m.out_stride + c0;
#pragma unroll
    for (int c = lane; c < kColumns; c += 32) {
      const T v = box_number<T>(from, r, (uint32_t)(first_byte + c * (int)sizeof(T)));
      if (c0 + c < t.m.n) out[c] = v;
    }
  }
  __syncwarp();
}

// tile `i` of the grid's order
__device__ __forceinline__ void tile_of(const ManyArgs &t, int i, int &tm, int &tn) {
  const int per = kGroupM * t.tiles_n, group = i / per, in = i - group * per, rows = min(kGroupM, t.tiles_m - group * kGroupM);
  tn = in / rows;
  tm = group * kGroupM + in - tn * rows;
}

template <int W>
__global__ void __launch_bounds__(kThreads, 1)
k_mm8_many(const __grid_constant__ CUtensorMap map_w0, const __grid_constant__ CUtensorMap map_w1, const __grid_constant__ CUtensorMap map_a,
           const __grid_constant__ CUtensorMap map_out, const __grid_constant__ ManyArgs t) {
  extern __shared__ unsigned char raw[];
  __shared__ __align__(8) uint64_t s_full[kStages], s_empty[kStages], s_done[2], s_read[2], s_there[kChunks], s_used[kChunks], s_tail, s_never;
  __shared__ __align__(16) float s_rows[kChunks][128][kChunk], s_weights[kChunks][2][kChunk];
  __shared__ float s_top[2][128];
  __shared__ uint32_t s_tmem;
  __shared__ int s_gave_up;
  const int tid = threadIdx.x, warp = __shfl_sync(0xffffffffu, tid >> 5, 0), lane = tid & 31, rank = (int)pair_rank();
  const uint32_t ring = (smem_at(raw) + 1023u) & ~1023u, out_at = ring + kStages * kStage;
  volatile int *gave_up = &s_gave_up;
  const int n_kb = t.m.n_kb, tiles = t.tiles_m * t.tiles_n, pairs = gridDim.x >> 1, first = blockIdx.x >> 1;
  const int wide = W == 2 ? 128 : 256;             // result columns of a tile

  if (tid == 0) {
    const uint32_t copies = t.m.stall && blockIdx.x == 0 ? 2 : 1;
    for (int s = 0; s < kStages; ++s) { mbar_init(smem_at(&s_full[s]), copies); mbar_init(smem_at(&s_empty[s]), 1); }
    for (int b = 0; b < 2; ++b) { mbar_init(smem_at(&s_done[b]), 1); mbar_init(smem_at(&s_read[b]), 16); }
    for (int c = 0; c < kChunks; ++c) { mbar_init(smem_at(&s_there[c]), 32); mbar_init(smem_at(&s_used[c]), 8); }
    mbar_init(smem_at(&s_tail), 1);
    mbar_init(smem_at(&s_never), 1);
    s_gave_up = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
  }
  if (warp == 1) {
    asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_at(&s_tmem)), "r"((uint32_t)kColumns) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
  }
  tc_fence_before();
  __syncthreads();
  cluster_sync();
  tc_fence_after();
  const uint32_t tmem = s_tmem;
  pdl_wait();
  pdl_trigger();

  if (warp < 4) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kRegsControl));
    if (warp == 0) {
      // ---------------------------------------------------------- copies: this CTA's rows, and its half of the weight rows
      // (the whole warp runs the loops of this branch and the next, so that their arithmetic is the warp's and not a lane's)
      const bool one = elect_one();
      const void *map_w = W == 2 && rank == 1 ? &map_w1 : &map_w0;
      int it = 0, s = 0, phase = 1;
      bool ok = true;
      for (int i = first; i < tiles && ok; i += pairs) {
        int tm, tn;
        tile_of(t, i, tm, tn);
        const int y_a = tm * 256 + rank * 128, y_w = W == 2 ? tn * 128 : tn * 256 + rank * 128;
        for (int b = 0; b < n_kb; ++b, ++it) {
          if (it >= kStages && !(ok = mbar_wait(smem_at(&s_empty[s]), (uint32_t)phase, gave_up, t.m.wait_tries))) break;
          const uint32_t at = ring + (uint32_t)(s * kStage), full = at_first(smem_at(&s_full[s]));
          if (one) {
            if (rank == 0) mbar_expect(smem_at(&s_full[s]), 2 * kStage);
            pair_load(at, &map_a, b * 128, y_a, full);
            pair_load(at + kBox, map_w, b * 128, y_w, full);
          }
          if (++s == kStages) { s = 0; phase ^= 1; }
        }
      }
      __syncwarp();
    } else if (warp == 1) {
      // ---------------------------------------------------------- products, by the first CTA
      if (rank == 0) {
        constexpr uint32_t idesc = idesc_e4m3(256, 256);
        const bool one = elect_one();
        bool ok = true;
        int it = 0, s = 0, phase = 0;
        for (int i = first; i < tiles && ok; i += pairs) {
          for (int b = 0; b < n_kb; ++b, ++it) {
            const int buf = it & 1;
            ok = mbar_wait(smem_at(&s_full[s]), (uint32_t)phase, gave_up, t.m.wait_tries);
            if (ok && it >= 2) ok = mbar_wait(smem_at(&s_read[buf]), (uint32_t)(((it >> 1) - 1) & 1), gave_up, t.m.wait_tries);
            if (!ok) break;
            tc_fence_after();
            const uint64_t ad = desc_rows8(ring + (uint32_t)(s * kStage)), bd = desc_rows8(ring + (uint32_t)(s * kStage + kBox));
            if (one) {
#pragma unroll
              for (int k = 0; k < 4; ++k)
                pair_mma(tmem + (uint32_t)(buf * 256), ad + (uint64_t)(2 * k), bd + (uint64_t)(2 * k), idesc, k ? 1u : 0u);
              pair_commit(smem_at(&s_done[buf]));
              pair_commit(smem_at(&s_empty[s]));
            }
            if (++s == kStages) { s = 0; phase ^= 1; }
          }
        }
        if (!ok) {   // what was issued still reads shared memory and writes tensor memory
          if (one) asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(smem_at(&s_tail)) : "memory");
          mbar_wait(smem_at(&s_tail), 0u, gave_up, max(t.m.wait_tries, kDrainTries), false);
        }
      }
      __syncwarp();
    } else if (warp == 2) {
      // ---------------------------------------------------------- scales: of this CTA's rows, and of both halves' weight rows
      const int last_block = (t.m.n + 127) / 128 - 1;
      int ch = 0;
      bool ok = true;
      for (int i = first; i < tiles && ok; i += pairs) {
        int tm, tn;
        tile_of(t, i, tm, tn);
        const int row0 = tm * 256 + rank * 128, wb = tn * wide / 128;
        const float *ws[2] = {t.m.w_scale[0] + (size_t)wb * n_kb,
                              W == 2 ? t.m.w_scale[1] + (size_t)wb * n_kb : t.m.w_scale[0] + (size_t)min(wb + 1, last_block) * n_kb};
        for (int b = 0; b < n_kb; b += kChunk, ++ch) {
          const int c = ch % kChunks, fill = ch / kChunks;
          if (fill > 0 && !(ok = mbar_wait(smem_at(&s_used[c]), (uint32_t)((fill - 1) & 1), gave_up, t.m.wait_tries))) break;
          const int kb = min(b + (lane & 3), n_kb - 1);
#pragma unroll
          for (int e = 0; e < 16; ++e) {       // 4 blocks of 8 rows at a time
            const int r = e * 8 + (lane >> 2);
            if (row0 + r < t.m.n_rows) copy4(smem_at(&s_rows[c][r][lane & 3]), t.m.a_scale + (long long)(row0 + r) * t.m.a_scale_stride + kb);
          }
          if (lane < 2 * kChunk) copy4(smem_at(&s_weights[c][lane >> 2][lane & 3]), ws[lane >> 2] + kb);
          asm volatile("cp.async.mbarrier.arrive.noinc.shared::cta.b64 [%0];" ::"r"(smem_at(&s_there[c])) : "memory");
        }
      }
      asm volatile("cp.async.wait_all;" ::: "memory");
    }
  } else {
    // ------------------------------------------------------------ sums
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kRegsSums));
    const int g = (warp - 4) >> 2, q = warp & 3, r = q * 32 + lane;
    const uint32_t lanes = tmem + ((uint32_t)(q * 32) << 16) + (uint32_t)(g * 64);
    const uint32_t read_bar[2] = {at_first(smem_at(&s_read[0])), at_first(smem_at(&s_read[1]))};
    const int dtype = t.m.out_dtype, es = dtype == D3_FP32 ? 4 : dtype == D3_E4M3 ? 1 : 2;
    int it = 0, chunk = 0, there = 0;
    for (int i = first; i < tiles; i += pairs) {
      int tm, tn;
      tile_of(t, i, tm, tn);
      const int row0 = tm * 256 + rank * 128, row = row0 + r, n0 = tn * wide;
      const bool live = row < t.m.n_rows;
      uint64_t acc[2][32];
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int j = 0; j < 32; ++j) acc[h][j] = 0ull;
      // Scales of four blocks at a time, this row's times those of the two halves' weights (fetched block by block they took a third of
      // the epilogue's time).
      float f0[kChunk], f1[kChunk];
      // (64 columns a load: with 32, two on their way, the longer code took 495 us where this takes 470)
      uint32_t d[64];
      auto begin = [&]() {
        mbar_wait(smem_at(&s_done[it & 1]), (uint32_t)((it >> 1) & 1), gave_up, t.m.wait_tries);   // (given up: numbers without meaning)
        __syncwarp();
        tc_fence_after();
        tc_ld(lanes + (uint32_t)((it & 1) * 256), d);
      };
      begin();
      for (int b0 = 0; b0 < n_kb; b0 += kChunk) {
        mbar_wait(smem_at(&s_there[chunk]), (uint32_t)there, gave_up, t.m.wait_tries);
        const float4 sa = *reinterpret_cast<const float4 *>(s_rows[chunk][r]), w0 = *reinterpret_cast<const float4 *>(s_weights[chunk][0]),
                     w1 = *reinterpret_cast<const float4 *>(s_weights[chunk][1]);
        f0[0] = sa.x * w0.x; f0[1] = sa.y * w0.y; f0[2] = sa.z * w0.z; f0[3] = sa.w * w0.w;
        f1[0] = sa.x * w1.x; f1[1] = sa.y * w1.y; f1[2] = sa.z * w1.z; f1[3] = sa.w * w1.w;
        __syncwarp();
        if (lane == 0) mbar_arrive(smem_at(&s_used[chunk]));
        __syncwarp();
        if (++chunk == kChunks) { chunk = 0; there ^= 1; }
#pragma unroll 1                               // (the loop's code has to stay within reach: four blocks unrolled took 563 us where this takes 502)
        for (int j = 0; j < kChunk; ++j) {
          if (b0 + j >= n_kb) break;
          const uint32_t at = lanes + (uint32_t)((it & 1) * 256), read = read_bar[it & 1];
          const uint64_t f[2] = {two_of(__float_as_uint(f0[0]), __float_as_uint(f0[0])), two_of(__float_as_uint(f1[0]), __float_as_uint(f1[0]))};
#pragma unroll
          for (int e = 0; e + 1 < kChunk; ++e) { f0[e] = f0[e + 1]; f1[e] = f1[e + 1]; }
          ++it;
          tc_ld_wait(d);
#pragma unroll
          for (int e = 0; e < 32; ++e) fma_two(acc[0][e], two_of(d[2 * e], d[2 * e + 1]), f[0]);
          tc_ld(at + 128u, d);                 // the second half
          tc_ld_wait(d);
          tc_fence_before();
          __syncwarp();
          if (lane == 0) pair_arrive(read);
#pragma unroll
          for (int e = 0; e < 32; ++e) fma_two(acc[1][e], two_of(d[2 * e], d[2 * e + 1]), f[1]);
          if (b0 + j + 1 < n_kb) begin();
        }
      }
      // ---------------------------------------------------------- results
      if constexpr (W == 2) {
#pragma unroll
        for (int j = 0; j < 32; ++j)
          acc[0][j] = two_of(__float_as_uint(gate_of(low_of(acc[0][j]), low_of(acc[1][j]))),
                              __float_as_uint(gate_of(high_of(acc[0][j]), high_of(acc[1][j]))));
      }
      // what the last tile left must be out of the staging area
      if (t.bulk) {
        if ((warp & 3) == 0 && lane == 0) asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory");
        if (W == 2 && dtype == D3_E4M3) group_sync(3, 256);
        else group_sync(1 + g, 128);
      }
      if (W == 2 && dtype == D3_E4M3) {   // the block of scales is 128 columns: two threads have a row's
        const int c0 = n0 + g * 64;
        float top = 0.f;
#pragma unroll
        for (int j = 0; j < 32; ++j) {
          top = max_nan(top, fabsf(low_of(acc[0][j])));     // (columns behind the last one are of zero weights)
          top = max_nan(top, fabsf(high_of(acc[0][j])));
        }
        s_top[g][r] = top;
        group_sync(3, 256);
        top = max_nan(top, s_top[g ^ 1][r]);
        BlockScale b = block_scale(top);
        if (live && g == 0) t.m.scale[row * t.m.scale_stride + n0 / 128] = b.scale;
        if (lift(b)) {
#pragma unroll
          for (int j = 0; j < 32; ++j)
            acc[0][j] = two_of(__float_as_uint(low_of(acc[0][j]) * kLift), __float_as_uint(high_of(acc[0][j]) * kLift));
        }
        uint32_t v[16];
#pragma unroll
        for (int j = 0; j < 16; ++j) v[j] = quantize4(low_of(acc[0][2 * j]), high_of(acc[0][2 * j]), low_of(acc[0][2 * j + 1]), high_of(acc[0][2 * j + 1]), b);
        // one box: rows of 128 bytes in the 128-byte swizzle
#pragma unroll
        for (int j = 0; j < 4; ++j)
          store16(out_at + (uint32_t)(r * 128 + (((g * 4 + j) ^ (r & 7)) << 4)), v[4 * j], v[4 * j + 1], v[4 * j + 2], v[4 * j + 3]);
        if (t.bulk) {
          copy_rest<unsigned char, 64>(t, out_at, g * 64, c0, row, r);
          asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
          group_sync(3, 256);
          if (warp == 4 && lane == 0 && n0 < t.whole && row0 < t.m.n_rows) {
            store_box(&map_out, out_at, n0, row0);
            asm volatile("cp.async.bulk.commit_group;" ::: "memory");
          }
        } else {
          copy_lines<unsigned char, 64>(t, out_at, g * 64, c0, row0, q, lane);
          group_sync(3, 256);   // s_top is written again
        }
      } else {
        const uint32_t mine = out_at + (uint32_t)(g * (kOutBytes / 2));
#pragma unroll
        for (int h = 0; h < (W == 2 ? 1 : 2); ++h) {
          const int c0 = n0 + h * 128 + g * 64;
          if (t.bulk && h == 1) {         // the second half takes the first one's place
            if ((warp & 3) == 0 && lane == 0) asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory");
            group_sync(1 + g, 128);
          }
          if (es == 2) {                  // a box of 64 columns: rows of 128 bytes
#pragma unroll
            for (int j = 0; j < 8; ++j) {
              uint32_t v[4];
#pragma unroll
              for (int e = 0; e < 4; ++e) v[e] = pack2(low_of(acc[h][4 * j + e]), high_of(acc[h][4 * j + e]), dtype);
              store16(mine + (uint32_t)(r * 128 + ((j ^ (r & 7)) << 4)), v[0], v[1], v[2], v[3]);
            }
            if (t.bulk) copy_rest<unsigned short, 64>(t, mine, 0, c0, row, r);
            if (t.bulk) copy_out(t, map_out, mine, c0, row0, g, warp, lane);
            else copy_lines<unsigned short, 64>(t, mine, 0, c0, row0, q, lane);
          } else {                        // boxes of 32 columns, one behind the other
#pragma unroll
            for (int part = 0; part < 2; ++part) {
              if (t.bulk && part == 1) {
                if ((warp & 3) == 0 && lane == 0) asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory");
                group_sync(1 + g, 128);
              }
#pragma unroll
              for (int j = 0; j < 8; ++j)
                store16(mine + (uint32_t)(r * 128 + ((j ^ (r & 7)) << 4)), (uint32_t)acc[h][16 * part + 2 * j], (uint32_t)(acc[h][16 * part + 2 * j] >> 32),
                        (uint32_t)acc[h][16 * part + 2 * j + 1], (uint32_t)(acc[h][16 * part + 2 * j + 1] >> 32));
              if (t.bulk) copy_rest<unsigned int, 32>(t, mine, 0, c0 + 32 * part, row, r);
              if (t.bulk) copy_out(t, map_out, mine, c0 + 32 * part, row0, g, warp, lane);
              else copy_lines<unsigned int, 32>(t, mine, 0, c0 + 32 * part, row0, q, lane);
            }
          }
        }
      }
    }
    if ((warp & 3) == 0 && lane == 0) asm volatile("cp.async.bulk.wait_group 0;" ::: "memory");
  }
  __syncthreads();
  if (*gave_up && warp == 0) {     // copies may be in flight, which must land before the CTA's shared memory is given back
    mbar_wait(smem_at(&s_never), 0u, gave_up, kDrainTries, false);
    if (lane == 0 && t.m.status) *t.m.status = D3_ETIMEOUT;
  }
  tc_fence_before();
  cluster_sync();   // neither CTA goes while the other one's products read its shared memory or arrive at its barriers
  if (warp == 1)
    asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"((uint32_t)kColumns) : "memory");
}

template <int W>
cudaError_t launch(const TMap &w0, const TMap &w1, const TMap &ma, const Mm8Args &p, cudaStream_t st) {
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  if (dev < 0 || dev >= 64) return cudaErrorInvalidDevice;
  static std::atomic<int> sms[64];   // SMs of a device whose attribute is set (setting it twice is harmless)
  int n_sm = sms[dev].load(std::memory_order_acquire);
  if (n_sm == 0) {
    if ((e = cudaDeviceGetAttribute(&n_sm, cudaDevAttrMultiProcessorCount, dev)) != cudaSuccess) return e;
    if ((e = cudaFuncSetAttribute(k_mm8_many<W>, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmem)) != cudaSuccess) return e;
    sms[dev].store(n_sm, std::memory_order_release);
  }
  ManyArgs t;
  t.m = p;
  const int wide = W == 2 ? 128 : 256;
  t.tiles_m = (p.n_rows + 255) / 256;
  t.tiles_n = (p.n + wide - 1) / wide;
  const long long tiles = (long long)t.tiles_m * t.tiles_n;
  if (tiles > 0x3fffffff) return cudaErrorInvalidValue;
  // results as bulk copies: boxes of 128 bytes x 128 rows
  TMap mo = ma;
  const int es = type_bytes(p.out_dtype);
  t.whole = p.n - p.n % (16 / es);
  t.bulk = t.whole > 0 && on_bytes(p.out, 16) && (p.out_stride * es) % 16 == 0 &&
           encode_results8(&mo, p.out, p.n_rows, t.whole, p.out_dtype, p.out_stride);
  const long long pairs = tiles < n_sm / 2 ? tiles : n_sm / 2;
  cudaLaunchConfig_t cfg;
  memset(&cfg, 0, sizeof(cfg));
  cfg.gridDim = dim3((unsigned)(2 * pairs));
  cfg.blockDim = dim3(kThreads);
  cfg.dynamicSmemBytes = kSmem;
  cfg.stream = st;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = 2;
  attr[1].val.clusterDim.y = 1;
  attr[1].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 2;
  const CUtensorMap *m0 = reinterpret_cast<const CUtensorMap *>(&w0), *m1 = reinterpret_cast<const CUtensorMap *>(&w1),
                    *m = reinterpret_cast<const CUtensorMap *>(&ma), *out = reinterpret_cast<const CUtensorMap *>(&mo);
  return cudaLaunchKernelEx(&cfg, k_mm8_many<W>, *m0, *m1, *m, *out, static_cast<const ManyArgs>(t));
}

}  // namespace

// What a call takes, in us, as measured: a block of k 0.46, the results of a tile 1, and 4 for the call (1000 x 4096 x 11008: 51 / 52;
// 200 x 11008 x 4096: 45 / 44).
float estimate_mm8_many(const Mm8Args &p, int mats) {
  const float wide = mats == 2 ? 128.f : 256.f, tiles = ceilf(p.n_rows / 256.f) * ceilf(p.n / wide);
  return ceilf(tiles / 74.f) * (0.46f * p.n_kb + 1.f) + 4.f;
}

cudaError_t launch_mm8_many(const TMap &w0, const TMap *w1, const void *a, int64_t a_stride, const Mm8Args &p, cudaStream_t st) {
  TMap ma;
  if (!encode_rows8(&ma, a, p.n_rows, p.k, a_stride, 128)) return cudaErrorInvalidValue;
  return w1 ? launch<2>(w0, *w1, ma, p, st) : launch<1>(w0, w0, ma, p, st);
}

}  // namespace d3
