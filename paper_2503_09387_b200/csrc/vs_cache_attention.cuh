// What the kernels of the attention over a paged cache share: the cut of the work and the parts that a later kernel joins.
// (A block runs all of this once, from a cold instruction cache, at some 100 clocks for every eight instructions: hence 32-bit numbers, products
// in the place of divisions, and as little of it as will do.)
#pragma once
#include "vs_operators.cuh"

namespace vs {

constexpr int kFewWide = 16, kFewCtas = 3 * 148, kManyWide = 256, kManyCtas = 148;      // packed rows of a tile (at most) and CTAs of either kernel

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
  uint32_t rcp_g;                 // 2^32 / G, rounded up (0: G = 1)
  int rows_each;                  // of every sequence; -1: by row_offsets
  int max_held;                   // tokens that a sequence's row of the table has pages for
  int page_shift;                 // log2 of the pages that are worth a CTA of their own
  int side_shift;                 // log2 of the lanes that count a sequence's units: 32 / n_seqs, rounded down to a power of two
  int few_cols, take_few;         // packed rows of a sequence of few rows, at most; whether the launch takes these or the others
};

#ifdef __CUDACC__
// x / G, x < 2^30
__device__ __forceinline__ int by_group(const CacheAttnArgs& a, int x) { return a.rcp_g == 0u ? x : (int)__umulhi((uint32_t)x, a.rcp_g); }

// A sequence's packed rows -- row t, head g of the group: t * G + g -- are cut into tiles of W; an item is a tile of one KV head, its work
// the pages of 64 keys that any of the tile's rows sees (one page at least: an item without keys still has its rows to store).
struct SeqShape { int first, n, len, tiles; };
template <int W>
__device__ __forceinline__ SeqShape shape_of(const CacheAttnArgs& a, int i) {
  SeqShape q;
  q.first = a.rows_each * i;
  q.n = a.rows_each;
  if (a.rows_each < 0) { const SeqRows s = rows_of(a.r, i); q.first = s.first; q.n = s.n; }
  q.len = max(a.r.tokens[i], 0);
  const int cols = q.n * a.G;                       // (the host has seen to it that this is below 2^30)
  q.tiles = (cols <= a.few_cols) == (a.take_few != 0) ? (cols + W - 1) / W : 0;
  return q;
}
// keys [lo, hi) that row t of a sequence sees
struct KeyRange { int lo, hi; };
__device__ __forceinline__ KeyRange keys_of(const CacheAttnArgs& a, const SeqShape& s, int t) {
  const int pos = s.len - s.n + t, held = min(s.len, a.max_held);
  const int hi = a.causal ? max(min(held, pos + 1), 0) : held;
  const int lo = a.window > 0 && pos >= a.window ? pos - a.window + 1 : 0;
  return {min(lo, hi), hi};
}
// pages [first, first + n) that tile `tile` sees: those of its first row to those of its last
struct PageRange { int first, n; };
template <int W>
__device__ __forceinline__ PageRange pages_of(const CacheAttnArgs& a, const SeqShape& s, int tile) {
  const int first = keys_of(a, s, by_group(a, tile * W)).lo / kPage;
  return {first, max((keys_of(a, s, min(by_group(a, tile * W + W - 1), s.n - 1)).hi + kPage - 1) / kPage - first, 1)};
}

__device__ __forceinline__ long long divide(long long x, long long y) { return ((x | y) >> 31) == 0 ? (long long)((uint32_t)x / (uint32_t)y) : x / y; }
// x / y, rounded up, 0 <= x <= 2^20: the quotient's relative error of 2^-22 is below 1 / x, so that its whole part is off, if at all, by 1 downwards where y
// divides x.  (A division of integers is some forty instructions.)
__device__ __forceinline__ int divide_up(int x, int y) { const int q = (int)__fdividef((float)x, (float)y); return q * y < x ? q + 1 : q; }
constexpr uint32_t kMostWhole = 1u << 20;
__device__ __forceinline__ int rounded_up(int x, int to) { return to <= 1 ? x : divide_up(x, to) * to; }

// The units (item, page) of all sequences lie end to end and are cut into equal runs, one a CTA: n_ctas of `each` units, the first `longer` of them
// of one more.  A run that crosses from one item to the next pays for a beginning and an end twice, and an item in parts for the parts and the join: either
// takes about as long as kJoinPages pages.  So where it costs no more than that a CTA, each item is counted as a whole number of runs and none
// crosses (one row over 211 pages, four heads: 13.1 us from first to last, of which two CTAs that crossed took 3.5), or as one (four
// sequences of 332 tokens, 32 rows of each: 29.5 us in parts of four pages, 21.5); with more items than CTAs a run may be several whole ones.
constexpr int kJoinPages = 5;
struct AttnRuns {
  long long units, each;
  int n_ctas, longer, whole;           // whole: units that an item is rounded up to (0: they are as they are)
  __device__ __forceinline__ long long begin(int cta) const { return each * cta + min(cta, longer); }
  // the CTA whose run holds `unit`
  __device__ __forceinline__ int cta_of(long long unit) const {
    const long long head = (each + 1) * longer;
    return unit < head ? (int)divide(unit, each + 1) : longer + (int)divide(unit - head, each);
  }
};
// `before` (shared memory, n_seqs + 1 numbers and kCutWords): units of the sequences ahead of each; how the units are cut.  Called by the
// whole block; ends with a barrier.
constexpr int kCutWords = 3;
template <int W>
__device__ __forceinline__ AttnRuns cut_units(const CacheAttnArgs& a, long long* before, int grid) {
  if (threadIdx.x < 32) {
    const int lane = threadIdx.x, least = 1 << a.page_shift;
    const int shift = a.side_shift, sub = lane & ((1 << shift) - 1), abreast = 32 >> shift;       // a sequence's tiles are dealt to 2^shift lanes
    auto units_of = [&](int i, int whole, int& items, int& most) {
      const SeqShape s = shape_of<W>(a, i);
      long long u = 0;
#pragma unroll 1
      for (int tile = sub; tile < s.tiles; tile += 1 << shift) {
        const int n = pages_of<W>(a, s, tile).n;
        most = max(most, n);
        u += rounded_up(n, whole);
      }
      if (sub == 0) items = min(items + min(s.tiles, (int)kMostWhole) * a.c.n_kv_heads, (int)kMostWhole);      // (of 256 heads at most)
      return u * a.c.n_kv_heads;
    };
    // all units and items and the longest item, as far as the rule asks for them.  (An item has a unit at least: where the units are fewer than
    // kMostWhole the items are all counted, and with them the runs below are at most `grid`: no run may be left without a CTA.)
    uint32_t units = 0u;
    int items = 0, most = 0, whole = 0;
#pragma unroll 1
    for (int i = lane >> shift; i < a.r.n_seqs; i += abreast) units = min(units + (uint32_t)min(units_of(i, 0, items, most), (long long)kMostWhole), kMostWhole);
    units = __reduce_add_sync(0xffffffffu, units);
    items = max(__reduce_add_sync(0xffffffffu, items), 1);
    most = max(__reduce_max_sync(0xffffffffu, most), 1);
    int per_cta = 1;                                        // (of runs of `whole` units)
    if (units < kMostWhole) {
      const int equal = divide_up((int)units, grid);
      if (items <= grid) {
        int runs = (int)__fdividef((float)grid, (float)items);                    // of an item, as many as all of them can have
        if (runs * items > grid) --runs;
        int rounded = divide_up(most, max(runs, 1));
        if (items < grid) rounded = min(rounded, divide_up((int)units, grid - items));
        rounded = max(rounded, least);
        if (rounded + kJoinPages >= most) rounded = most;
        if (rounded - max(equal, least) <= kJoinPages) whole = rounded;
      } else {
        per_cta = divide_up(items, grid);
        if (per_cta * most <= equal + 2 * kJoinPages) whole = most;
      }
    }
    long long ahead = 0;
#pragma unroll 1
    for (int base = 0; base < a.r.n_seqs; base += abreast) {
      const int i = base + (lane >> shift);
      int again = 0;
      long long u = i < a.r.n_seqs ? units_of(i, whole, again, most) : 0;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) { const long long t = __shfl_up_sync(0xffffffffu, u, o); if (lane >= o) u += t; }
      if (i < a.r.n_seqs && sub + 1 == 1 << shift) before[i + 1] = ahead + u;
      ahead += __shfl_sync(0xffffffffu, u, 31);
    }
    if (lane == 0) {
      // (more items than CTAs: no item is cut for want of others, so a run may be short)
      const int run = whole * per_cta;
      const int n = whole > 0 ? max(divide_up((int)ahead, run), 1) : max((int)min((long long)grid, items > grid ? ahead : (ahead + least - 1) >> a.page_shift), 1);
      const long long each = whole > 0 ? run : divide(ahead, n);
      before[0] = 0;
      before[a.r.n_seqs + 1] = each;
      before[a.r.n_seqs + 2] = n | (whole > 0 ? 0 : (ahead - each * n) << 32);
      before[a.r.n_seqs + 3] = whole;
    }
  }
  __syncthreads();
  AttnRuns c;
  c.units = before[a.r.n_seqs];
  c.each = before[a.r.n_seqs + 1];
  c.n_ctas = (int)before[a.r.n_seqs + 2];
  c.longer = (int)(before[a.r.n_seqs + 2] >> 32);
  c.whole = (int)before[a.r.n_seqs + 3];
  return c;
}

// An item's pages that this CTA works on: [page, page + n) of the pages [first, first + of); `span` units of its run.
struct AttnItem { SeqShape s; int seq, r0, n_cols, head, page, n, first, of; long long span; };
// Where a warp's last item lies: the next one is looked for from there.  (Looked for from the sequence's first tile, the items of a sequence of t tiles cost
// t^2 steps: 100000 rows of 28 heads over 64 keys took 32.7 ms so.)  In shared memory, the warp's own; seq = -1 ahead of the first.
struct ItemPlace { long long at; int seq, tile; };       // units of the sequence ahead of the tile
template <int W>
__device__ __forceinline__ AttnItem item_at(const CacheAttnArgs& a, const long long* before, const AttnRuns& runs, long long unit, long long end,
                                            ItemPlace* place = nullptr) {
  int lo = 0;
  if (a.r.n_seqs > 1) {
    int hi = a.r.n_seqs - 1;
    while (lo < hi) { const int mid = (lo + hi + 1) >> 1; if (before[mid] <= unit) lo = mid; else hi = mid - 1; }
  }
  AttnItem it;
  it.seq = lo;
  it.s = shape_of<W>(a, lo);
  it.n = 0;                           // (stays 0 only if the sequences changed under the kernel)
  long long u = unit - before[lo];
  int tile = 0;
  if (place != nullptr && place->seq == lo) { tile = place->tile; u -= place->at; }      // (units ascend)
#pragma unroll 1
  for (; tile < it.s.tiles; ++tile) {
    const PageRange p = pages_of<W>(a, it.s, tile);
    const int of = rounded_up(p.n, runs.whole);
    const long long here = (long long)of * a.c.n_kv_heads;
    if (u < here) {
      if (place != nullptr) {
        __syncwarp();                 // (every lane has read the last one)
        if ((threadIdx.x & 31) == 0) *place = {unit - before[lo] - u, lo, tile};
        __syncwarp();
      }
      it.r0 = tile * W;
      it.n_cols = min(W, it.s.n * a.G - it.r0);
      int head = 0;
      while (u >= of) { u -= of; ++head; }
      it.head = head;
      it.page = p.first + (int)u;
      it.span = min((long long)of - u, end - unit);
      it.n = (int)min((long long)p.n - u, it.span);
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

// A row's sum l goes by the scores alone and its reference m by score and page exponent: l = sum of 2^{x - m + lift - ev}, where a page's exponent ev is
// anything from -110 (values of nothing but zeros) to 120.  The low end fits fp32: all of l is 2^-113 at the least, and what counts beside that 2^-137.  The high end
// does not, 2^125 a key.  So a sum is held times 2^-64 from the first page on whose largest score lies 70 above m, and has its sign set to say so; as it is
// again once it would be small that way.  Either way 2^31 keys are far from an overflow and nothing that counts is lost, and pages of usual exponents pay
// a comparison.  (Held in fp64: frames 182 -> 192 us.)
constexpr float kSumTop = 70.f, kSumShift = 64.f, kSumDown = 0x1p-64f, kSumUp = 0x1p64f;
__device__ __forceinline__ bool shifted(float l) { return __float_as_int(l) < 0; }
__device__ __forceinline__ int value_exponent(float scale) { return max(exponent_of(scale), kScaleMinExp); }      // (a scale of 0 belongs to zeros)
__device__ __forceinline__ float times_power(float l, float d) {          // in two halves: 2^d, d <= 0, may be nothing where l 2^d is not
  const float h = exp2f(0.5f * d);
  return l * h * h;
}
__device__ __forceinline__ float sum_factor(float l, float down) { return shifted(l) ? -kSumDown * down : down; }      // of a page's weights, to be added to l
__device__ __forceinline__ float shift_sum(float l) { return shifted(l) ? l : -kSumDown * l; }
__device__ __forceinline__ float moved_sum(float l, float d) {            // for a reference that moved by -d
  if (shifted(l) && l * exp2f(d) > -1e-6f) { l = -l; d += kSumShift; }
  return times_power(l, d);
}
// A sum of sums, where any of them is held times 2^-64: added up as they are and all times 2^-64, and chosen.
__device__ __forceinline__ float as_is(float l, float d) { return shifted(l) ? times_power(-l, d + kSumShift) : times_power(l, d); }
__device__ __forceinline__ float as_shifted(float l, float d) { return shifted(l) ? times_power(-l, d) : times_power(l, d - kSumShift); }
__device__ __forceinline__ float chosen(float l, float by_2_64) { return l < 0x1p60f ? l : -by_2_64; }
// 1 / l as two factors; 0 of 0 (a row that sees nothing)
__device__ __forceinline__ float2 reciprocal(float l) { return make_float2(l == 0.f ? 0.f : 1.f / fabsf(l), shifted(l) ? kSumDown : 1.f); }
__device__ __forceinline__ float4 times(float4 v, float2 by) { return make_float4(v.x * by.x * by.y, v.y * by.x * by.y, v.z * by.x * by.y, v.w * by.x * by.y); }
constexpr float kFar = 40.f;      // a page whose largest x lies as far below m adds nothing to a row's O; to its l perhaps

// place in [n_rows][Hq] of packed row r (of a sequence whose rows begin at `first`) of KV head h: row and head
struct RowHead { int row, head; };
__device__ __forceinline__ RowHead row_head(const CacheAttnArgs& a, int first, int r, int h) {
  const int t = by_group(a, r);
  return {first + t, h * a.G + (r - t * a.G)};
}
__device__ __forceinline__ void store_row_piece(const CacheAttnArgs& a, RowHead p, int d, float4 v) {
  const long long at = (long long)p.row * a.out_row + (long long)p.head * a.out_head + d;
  if (a.out_fp32) *reinterpret_cast<float4*>(static_cast<float*>(a.out) + at) = v;
  else {
    const __nv_bfloat162 x = __floats2bfloat162_rn(v.x, v.y), y = __floats2bfloat162_rn(v.z, v.w);
    *reinterpret_cast<uint2*>(static_cast<bf16*>(a.out) + at) = make_uint2(*reinterpret_cast<const uint32_t*>(&x), *reinterpret_cast<const uint32_t*>(&y));
  }
}
__device__ __forceinline__ void store_lse(const CacheAttnArgs& a, RowHead p, float m, float l) {
  if (a.lse == nullptr) return;
  float log2_l = m + log2f(l);
  if (shifted(l)) {                    // (the whole powers of two to m first, which undo one another: some 2^70, -125)
    const float x = -l, e = (float)exponent_of(x);
    log2_l = (m + (e + kSumShift)) + log2f(x * exp2f(-e));
  }
  a.lse[(long long)p.row * a.Hq + p.head] = l == 0.f ? -INFINITY : log2_l * 0.6931471805599453f;
}
#endif

int launch_cache_attention_few(const CacheAttnArgs& a, int cols, cudaStream_t st);
int launch_cache_attention_many(const CacheAttnArgs& a, bool behind_few, cudaStream_t st);

}  // namespace vs
