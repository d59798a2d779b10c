// Shared by the paged key-value operators: host-side checks and device helpers.
#pragma once

#include "d3_internal.cuh"

namespace d3 {

// What the kernels know of a pool (strides in elements).
struct KvPool {
  int n_pages, page_shift, n_kv_heads;
  long long page_stride, head_stride, token_stride;
  void *k, *v;
  const float *k_scale, *v_scale;
};

inline int log2_of(int v) {
  int s = 0;
  while ((1 << s) < v) ++s;
  return s;
}
inline bool page_size_ok(int p) { return p >= 16 && p <= 1024 && (p & (p - 1)) == 0; }
inline int bytes_of(int dtype) { return dtype == D3_FP32 ? 4 : dtype == D3_E4M3 ? 1 : 2; }
inline bool aligned16(const void *p) { return ((uintptr_t)p & 15u) == 0; }
// a stride of whole 16-byte pieces whose byte value leaves room for 64-bit offsets
inline bool stride_ok(int64_t s, int elem_bytes, int64_t at_least) {
  return s >= at_least && s <= ((int64_t)1 << 38) && (s * elem_bytes) % 16 == 0;
}
// Rows of `dh` numbers at all combinations of three indexes (count, stride) do not overlap: every stride reaches over what
// the smaller ones span.  (Written memory: two rows at one address would be a race.)
inline bool rows_apart(int dh, int64_t n0, int64_t s0, int64_t n1, int64_t s1, int64_t n2 = 1, int64_t s2 = 0) {
  int64_t n[3] = {n0, n1, n2}, s[3] = {s0, s1, s2};
  double span = dh;   // (exact as far as any memory reaches)
  for (int done = 0; done < 3; ++done) {
    int at = -1;
    for (int i = 0; i < 3; ++i)
      if (n[i] > 1 && (at < 0 || s[i] < s[at])) at = i;
    if (at < 0) return true;
    if ((double)s[at] < span) return false;
    span += (double)(n[at] - 1) * (double)s[at];
    n[at] = 1;
  }
  return true;
}
// Two such sets of rows, with the same counts and strides (which keep the rows of either apart) and `delta` numbers between their
// bases, have a number in common: delta is a sum of multiples of the strides, within the counts, and less than a row.  Each
// stride reaches over what the smaller ones span, so only the two multiples next to what is left can be meant.
inline bool rows_meet(int dh, int64_t delta, int64_t n0, int64_t s0, int64_t n1, int64_t s1, int64_t n2 = 1, int64_t s2 = 0) {
  int64_t n[3] = {n0, n1, n2}, s[3] = {s0, s1, s2};
  int at = -1;
  for (int i = 0; i < 3; ++i)
    if (n[i] > 1 && (at < 0 || s[i] > s[at])) at = i;
  if (at < 0) return delta > -dh && delta < dh;
  const int64_t count = n[at], stride = s[at];
  n[at] = 1;
  int64_t q = delta / stride;
  if (q * stride > delta) --q;
  for (int i = 0; i < 2; ++i, ++q)
    if (q > -count && q < count && rows_meet(dh, delta - q * stride, n[0], s[0], n[1], s[1], n[2], s[2])) return true;
  return false;
}
// (type of q, k, v as given, type of the cache) pairs that the operators serve
inline bool types_ok(int x, int cache) {
  return (cache == D3_BF16 && (x == D3_BF16 || x == D3_FP32)) || (cache == D3_FP16 && x == D3_FP16) ||
         (cache == D3_E4M3 && (x == D3_BF16 || x == D3_FP16));
}
// sizes, types and strides of a pool (pointers only when `data`)
inline bool kv_ok(const d3_paged_kv *kv, bool data) {
  if (!kv || kv->struct_size != sizeof(d3_paged_kv)) return false;
  if (kv->dtype != D3_BF16 && kv->dtype != D3_FP16 && kv->dtype != D3_E4M3) return false;
  if (kv->n_pages < 1 || kv->n_kv_heads < 1 || kv->n_kv_heads > 65535 || !page_size_ok(kv->page_size)) return false;
  if (kv->head_dim != 32 && kv->head_dim != 64 && kv->head_dim != 128) return false;
  if (!data) return true;
  const int es = bytes_of(kv->dtype);
  if (!stride_ok(kv->token_stride, es, kv->head_dim) || !stride_ok(kv->head_stride, es, kv->head_dim) ||
      !stride_ok(kv->page_stride, es, kv->head_dim))
    return false;
  if (!kv->k_dev || !kv->v_dev || !aligned16(kv->k_dev) || !aligned16(kv->v_dev)) return false;
  return kv->dtype == D3_E4M3 || (!kv->k_scale_dev && !kv->v_scale_dev);
}
inline KvPool pool_of(const d3_paged_kv &kv) {
  KvPool p;
  p.n_pages = kv.n_pages; p.page_shift = log2_of(kv.page_size); p.n_kv_heads = kv.n_kv_heads;
  p.page_stride = kv.page_stride; p.head_stride = kv.head_stride; p.token_stride = kv.token_stride;
  p.k = kv.k_dev; p.v = kv.v_dev; p.k_scale = kv.k_scale_dev; p.v_scale = kv.v_scale_dev;
  return p;
}

// Positions of a unit, the attention kernel's stage: up to 32 KB of K and V.
__host__ __device__ constexpr int unit_positions(int head_dim, int elem_bytes) {
  return head_dim * elem_bytes > 128 ? 64 : head_dim * elem_bytes > 64 ? 128 : 256;
}
// Tensor maps of a pool: (dim, position, kv head, page), boxes of min(128 bytes, a row) x up to a page's or a unit's
// positions (k, v) and x 16 positions (k16, v16); `of` is the pool they were made for.
struct PoolMaps {
  TMap k, v, k16, v16;
  d3_paged_kv of;
};
static_assert(sizeof(PoolMaps) <= D3_PAGED_MAPS_BYTES, "room for the maps");
bool encode_pool_maps(PoolMaps *out, const d3_paged_kv &kv);   // false when the driver refuses or has no encoder

// What the attention launch gets (device pointers; strides in elements).
struct PagedAttnArgs {
  int n_rows, hq, hkv, group;          // group = query heads of a kv head
  int tiles_per_head, heads_per_tile;  // a tile: up to 8 (16) query heads of one kv head
  int table_rows, table_width, page_shift, n_pages;
  long long table_stride, q_row_stride, q_head_stride, out_row_stride, out_head_stride;
  float scale;
  int out_wide;                        // results may be written DH / 32 numbers at a time
  const void *q;
  void *out;
  float *lse;
  const int32_t *table, *context, *rows;
  const float *k_scale, *v_scale;
  float *part_o, *part_ml;             // partial results of rows that are cut between CTAs
  int4 *join;                          // per CTA: what the joining kernel has to do
  int32_t *status;
  int n_stages;
  int cluster;                         // CTAs that share an item, as a cluster (0: none)
  int whole;                           // no row is cut between CTAs: no join
  int few;                             // the rows are summed up by the producer warps alone, in 32 bits
  unsigned long long wait_ns;
  int stall;                           // drill: D3_STALL_*, 0 otherwise
};
// one translation unit per head dimension (each compiles every type pair)
int launch_paged_attention_32(const PoolMaps &m, const PagedAttnArgs &a, int x, cudaStream_t st);
int launch_paged_attention_64(const PoolMaps &m, const PagedAttnArgs &a, int x, cudaStream_t st);
int launch_paged_attention_128(const PoolMaps &m, const PagedAttnArgs &a, int x, cudaStream_t st);

}  // namespace d3
