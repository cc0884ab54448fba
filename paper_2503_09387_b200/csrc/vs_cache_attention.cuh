// What the kernels of the attention over a paged cache share: the cut of the work and the parts that a later kernel joins.
#pragma once
#include "vs_operators.cuh"

namespace vs {

constexpr int kFewCols = 16;      // sequences of at most as many packed rows: vs_cache_attention.cu; more: vs_cache_attention_tc.cu
constexpr int kFewCtas = 3 * 148, kManyCtas = 148, kManyWide = 256;

struct CacheAttnArgs {
  vs_cache c;
  vs_cache_seqs r;
  const bf16* q;
  void* out;
  float* lse;                     // [n_rows][Hq], or null
  float* parts;                   // workspace: unnormalised rows of items that several CTAs share
  int4* joins;                    // ... and, per CTA, which item it was the last to work on
  int* status;                    // VS_ERR_DEVICE_TIMEOUT if a wait ran out
  long long q_row, q_head, out_row, out_head;
  float scale_log2e;
  int Hq, G, causal, window, out_fp32;
  int min_pages;                  // pages that are worth a CTA of their own
  int take_few;                   // whether the launch takes the sequences of few rows or the others
};

#ifdef __CUDACC__
// A sequence's packed rows -- row t, head g of the group: t * G + g -- are cut into tiles of W; an item is a tile of one KV head, its work
// the pages of 64 keys that any of the tile's rows sees (one page at least: an item without keys still has its rows to store).
struct SeqShape { int first, n, len, tiles; };
template <int W>
__device__ __forceinline__ SeqShape shape_of(const CacheAttnArgs& a, int i) {
  const SeqRows s = rows_of(a.r, i);
  SeqShape q = {s.first, s.n, max(a.r.tokens[i], 0), 0};
  const long long cols = (long long)s.n * a.G;
  if ((cols <= kFewCols) == (a.take_few != 0)) q.tiles = (int)((cols + W - 1) / W);
  return q;
}
// keys [lo, hi) that row t of a sequence sees
struct KeyRange { int lo, hi; };
__device__ __forceinline__ KeyRange keys_of(const CacheAttnArgs& a, const SeqShape& s, int t) {
  const long long pos = (long long)s.len - s.n + t;
  const long long held = min((long long)s.len, (long long)a.r.table_width * kPage);
  const long long hi = a.causal ? max(min(held, pos + 1), 0ll) : held, lo = a.window > 0 ? max(pos - a.window + 1, 0ll) : 0ll;
  return {(int)min(lo, hi), (int)hi};
}
// pages [first, first + n) that tile `tile` sees: those of its first row to those of its last
struct PageRange { int first, n; };
template <int W>
__device__ __forceinline__ PageRange pages_of(const CacheAttnArgs& a, const SeqShape& s, int tile) {
  const int t0 = (int)((long long)tile * W / a.G), t1 = (int)min(((long long)tile * W + W - 1) / a.G, (long long)s.n - 1);
  const int lo = keys_of(a, s, t0).lo, hi = keys_of(a, s, t1).hi;
  const int first = lo / kPage;
  return {first, max((hi + kPage - 1) / kPage - first, 1)};
}
template <int W>
__device__ __forceinline__ long long units_of(const CacheAttnArgs& a, const SeqShape& s) {
  long long u = 0;
  for (int tile = 0; tile < s.tiles; ++tile) u += pages_of<W>(a, s, tile).n;
  return u * a.c.n_kv_heads;
}

// The units (item, page) of all sequences lie end to end and are cut into equal runs, one a CTA.  `before` (shared memory, n_seqs + 1):
// units of the sequences ahead of each.  Called by the whole block; ends with a barrier.
template <int W>
__device__ __forceinline__ long long count_units(const CacheAttnArgs& a, long long* before) {
  if (threadIdx.x < 32) {
    const int lane = threadIdx.x;
    long long sum0 = 0;
    for (int base = 0; base < a.r.n_seqs; base += 32) {
      const int i = base + lane;
      long long u = 0;
      if (i < a.r.n_seqs) u = units_of<W>(a, shape_of<W>(a, i));
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) { const long long t = __shfl_up_sync(0xffffffffu, u, o); if (lane >= o) u += t; }
      if (i < a.r.n_seqs) before[i + 1] = sum0 + u;
      sum0 += __shfl_sync(0xffffffffu, u, 31);
    }
    if (lane == 0) before[0] = 0;
  }
  __syncthreads();
  return before[a.r.n_seqs];
}
__device__ __forceinline__ int ctas_at_work(const CacheAttnArgs& a, long long units, int grid) {
  return (int)max(min((long long)grid, (units + a.min_pages - 1) / a.min_pages), 1ll);
}

// An item's pages that this CTA works on: [page, page + n) of the pages [first, first + of).
struct AttnItem { int seq, tile, head, page, n, first, of; };
template <int W>
__device__ __forceinline__ AttnItem item_at(const CacheAttnArgs& a, const long long* before, long long unit, long long end) {
  int lo = 0, hi = a.r.n_seqs - 1;
  while (lo < hi) { const int mid = (lo + hi + 1) >> 1; if (before[mid] <= unit) lo = mid; else hi = mid - 1; }
  const SeqShape s = shape_of<W>(a, lo);
  long long u = unit - before[lo];
  AttnItem it = {lo, 0, 0, 0, 0, 0, 0};
  for (int tile = 0; tile < s.tiles; ++tile) {
    const PageRange p = pages_of<W>(a, s, tile);
    const long long here = (long long)p.n * a.c.n_kv_heads;
    if (u < here) {
      it.tile = tile;
      it.head = (int)(u / p.n);
      const int at = (int)(u - (long long)it.head * p.n);
      it.page = p.first + at;
      it.n = (int)min((long long)(p.n - at), end - unit);
      it.first = p.first;
      it.of = p.n;
      break;
    }
    u -= here;
  }
  return it;
}

// Parts.  A CTA has two places for rows that it does not finish alone: place 0 for an item that began before its run, place 1 for one that goes on
// behind it.  Each holds W rows of D numbers relative to the row's m, then W pairs (m, l).  The CTA whose run holds an item's last
// page notes the item in joins[CTA]: (1 + first CTA, item's first row in the call, tile's first packed row, head | columns << 16).
template <int W, int D>
__device__ __forceinline__ float* part_rows(float* parts, int cta, int place) { return parts + (size_t)(2 * cta + place) * W * (D + 2); }
template <int W, int D>
__device__ __forceinline__ float2* part_stats(float* parts, int cta, int place) { return reinterpret_cast<float2*>(part_rows<W, D>(parts, cta, place) + (size_t)W * D); }

__device__ __forceinline__ long long run_begin(long long units, int ctas, int cta) { return units * cta / ctas; }
// the CTA whose run holds `unit`
__device__ __forceinline__ int cta_of(long long units, int ctas, long long unit) {
  int c = (int)(unit * ctas / units);
  while (c + 1 < ctas && run_begin(units, ctas, c + 1) <= unit) ++c;
  while (c > 0 && run_begin(units, ctas, c) > unit) --c;
  return c;
}

// A row's sum l goes by the scores alone and its reference m by score and page exponent: with pages whose exponents lie 230 apart 2^d, d <= 0, may
// be nothing where l 2^d is not.  In two halves.
__device__ __forceinline__ float times_power(float l, float d) {
  const float h = exp2f(0.5f * d);
  return l * h * h;
}
constexpr float kFar = 40.f;      // a page whose largest x lies as far below m adds nothing to a row's O; to its l perhaps

// where packed row r (of a sequence whose rows begin at `first`) of KV head h is stored
__device__ __forceinline__ void store_row_piece(const CacheAttnArgs& a, int first, int r, int head, int d, float4 v) {
  const int t = r / a.G, g = r - t * a.G;
  const long long at = (long long)(first + t) * a.out_row + (long long)(head * a.G + g) * a.out_head + d;
  if (a.out_fp32) *reinterpret_cast<float4*>(static_cast<float*>(a.out) + at) = v;
  else {
    const __nv_bfloat162 x = __floats2bfloat162_rn(v.x, v.y), y = __floats2bfloat162_rn(v.z, v.w);
    *reinterpret_cast<uint2*>(static_cast<bf16*>(a.out) + at) = make_uint2(*reinterpret_cast<const uint32_t*>(&x), *reinterpret_cast<const uint32_t*>(&y));
  }
}
__device__ __forceinline__ void store_lse(const CacheAttnArgs& a, int first, int r, int head, float m, float l) {
  if (a.lse == nullptr) return;
  const int t = r / a.G, g = r - t * a.G;
  a.lse[(long long)(first + t) * a.Hq + head * a.G + g] = l == 0.f ? -INFINITY : (m + log2f(l)) * 0.6931471805599453f;
}
#endif

int launch_cache_attention_few(const CacheAttnArgs& a, int cols, int ctas, cudaStream_t st);
int launch_cache_attention_many(const CacheAttnArgs& a, int ctas, cudaStream_t st);
int launch_cache_attention_join(const CacheAttnArgs& a, int width, int ctas, cudaStream_t st);

}  // namespace vs
