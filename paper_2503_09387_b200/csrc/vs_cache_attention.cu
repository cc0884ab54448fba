// vs_cache_attention: softmax attention over a paged cache of 8-bit keys and values.  Here: the call, the kernel for sequences of few
// rows (an answer's token), and the kernel that joins what several CTAs worked out of the same rows.
//
//   o = sum_j w_j v_j / sum_j w_j,   w_j = e^{scale q k_j},   k_j = 2^{ek} * code, v_j = 2^{ev} * code  (a page's and head's own exponents)
//
// Codes go to the tensor cores as fp16, which holds every e4m3 value exactly; a page's exponents are applied to scores and weights, never
// to the codes.  Scores are s = f (q' code) with q' the query row times a power of two that brings its largest magnitude to 2^14 .. 2^15
// (bf16 values are then exact in fp16 down to 2^-39 of that) and f the rest of the scale.  With x = s + ev, in the log2 domain, and m the running maximum of x:
//   O += 2^{x - m + 15} code_v,   l += 2^{x - m + 15} 2^{-ev},   o = O / l:
// the reference goes by what a key adds to the output, so pages of different exponents need no rescaling between them.  Weights are
// rounded to fp16 (a half step, 2^-12 relative; the smallest, 2^-40 of the largest, is far below any sum's last bit); maxima, sums and rows are fp32.
//
// What bounds the few-row kernel: the codes' bytes, once from HBM.  All heads of a KV group, and a few tokens, are the 8 (or 16)
// columns of mma.sync: S^T = K q^T and O^T += V^T P^T, so a page is read once for the whole group; a tcgen05 tile of 128
// rows would hold 7.  A CTA is four warps, each with half a page in a ring of its own, filled by 16-byte asynchronous copies
// ahead of their turn and placed so that both operands' fragments are read without bank conflicts: no barrier in the loop.
// The work of all sequences is cut into equal runs of pages (cut_units): long and short sequences side by side leave no CTA idle.
// Measured: sixteen sequences of 2000 to 65000 tokens, seven heads a group, 522 MB of codes: 90 us, 5.8 TB/s (89 % of what a copy reaches); one sequence of 13504:
// 11.3 us from first to last -- 1.5 until the units are counted, 1 to the pages' numbers and first loads, 0.9 to their arrival, 1.7 for two steps, 1.2 for the
// warps' rows, then 3.3 for the join behind the launch's end.
#include "vs_cache_attention.cuh"
#include "vs_ptx.cuh"

namespace vs {

namespace {

constexpr int kWarps = 4, kThreads = 32 * kWarps, kWarpKeys = 32, kStepPages = kWarps * kWarpKeys / kPage;
constexpr float kLift = 15.f;

__device__ __forceinline__ void mma_f16(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
               : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t half2_of(float lo, float hi) {
  const __half2 h = __floats2half2_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&h);
}
__device__ __forceinline__ uint4 lds128(uint32_t addr) {
  uint4 v;
  asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(addr) : "memory");
  return v;
}
__device__ __forceinline__ uint2 lds64(uint32_t addr) {
  uint2 v;
  asm volatile("ld.shared.v2.u32 {%0, %1}, [%2];" : "=r"(v.x), "=r"(v.y) : "r"(addr) : "memory");
  return v;
}

template <int D, int NT>
struct Few {
  static constexpr int W = 8 * NT, kStages = D == 128 ? 2 : 4;
  static constexpr int kTile = kWarpKeys * D;                      // a warp's keys (or values) of a page, bytes
  static constexpr int kStage = 2 * kTile;
  static constexpr int kRing = kWarps * kStages * kStage;
  static constexpr int kRowF = D + 4;                              // (a warp's rows, at the end of an item, lie in the ring)
  static_assert(kWarps * W * (kRowF + 2) * 4 <= kRing, "rows of the four warps");
  static constexpr int kMeta = kRing;                              // [warp][stage] (scale of K, scale of V)
  static constexpr int kBefore = kMeta + kWarps * kStages * 8;     // units ahead of each sequence
  static int bytes(int n_seqs) { return kBefore + 8 * (n_seqs + 1 + kCutWords); }
};

// Places of a 16-byte piece c of row r: keys are read by quads of lanes, eight rows side by side; values by eight lanes of one
// piece each, rows 2 q apart.  The exclusive or spreads either over all banks.
__device__ __forceinline__ uint32_t k_place(int r, int c, int D) { return (uint32_t)(r * D + ((D == 128 ? c ^ ((r & 1) << 2) : c) << 4)); }
__device__ __forceinline__ uint32_t v_place(int r, int c, int D) { return (uint32_t)(r * D + ((D == 128 ? c ^ (r & 6) : c) << 4)); }

template <int D, int NT>
__global__ void __launch_bounds__(kThreads) cache_attention_few_kernel(const __grid_constant__ CacheAttnArgs a) {
  using F = Few<D, NT>;
  constexpr int W = F::W, KS = D / 16, CPR = D / 16;               // k-steps of a score; 16-byte pieces of a row
  extern __shared__ __align__(128) uint8_t smem[];
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, g = lane >> 2, q4 = lane & 3;
  long long* before = reinterpret_cast<long long*>(smem + F::kBefore);
  const AttnRuns runs = cut_units<W>(a, before, (int)gridDim.x);
  const int cta = (int)blockIdx.x;
  if (tid == 0) a.joins[cta] = make_int4(0, 0, 0, 0);
  if (cta >= runs.n_ctas || runs.units == 0) return;
  const long long u_begin = runs.begin(cta), u_end = runs.begin(cta + 1);
  const uint32_t ring = smem_u32(smem) + (uint32_t)(warp * F::kStages * F::kStage);
  float2* meta = reinterpret_cast<float2*>(smem + F::kMeta) + warp * F::kStages;

  for (long long u = u_begin; u < u_end;) {
    const AttnItem it = item_at<W>(a, before, runs, u, u_end);
    if (it.n < 1) break;
    const SeqShape& s = it.s;
    const int r0 = it.r0, n_cols = it.n_cols;
    u += it.span;

    // ---- pages on their way: step i of the item, the warp's half of one of its two pages ----------------------------
    int id = -1;                     // page (of the 32 that the step being loaded is among) lane `lane`, and its scales
    float2 sc_mine = make_float2(-1.f, 1.f);
    auto load_step = [&](int i) {
      if (kStepPages * i < it.n) {
        const int p = kStepPages * i + warp / 2;
        if (((kStepPages * i) & 31) == 0) {
          id = kStepPages * i + lane < it.n ? page_of(a.r, a.c.n_pages, it.seq, it.page + kStepPages * i + lane) : -1;
          const size_t at = (size_t)max(id, 0) * a.c.n_kv_heads + it.head;
          sc_mine = id >= 0 ? make_float2(a.c.k_scale[at], a.c.v_scale[at]) : make_float2(-1.f, 1.f);       // (no page has a negative scale)
        }
        const int page = __shfl_sync(0xffffffffu, id, p & 31);
        const size_t from = ((size_t)max(page, 0) * a.c.n_kv_heads + it.head) * (size_t)(kPage * D) + (size_t)((warp & 1) * F::kTile + lane * 16);
        const uint8_t *k = static_cast<const uint8_t*>(a.c.k) + from, *v = static_cast<const uint8_t*>(a.c.v) + from;
        const uint32_t at = ring + (uint32_t)((i % F::kStages) * F::kStage);
#pragma unroll
        for (int j = 0; j < F::kTile / 512; ++j) {
          const int r = (j * 32 + lane) / CPR, c = lane % CPR;
          cp_async16(at + k_place(r, c, D), k + j * 512, page >= 0);
          cp_async16(at + (uint32_t)F::kTile + v_place(r, c, D), v + j * 512, page >= 0);
        }
        if (lane == (p & 31)) meta[i % F::kStages] = sc_mine;
      }
      cp_async_commit();
    };
    __syncthreads();                 // the rows of the item before, in the ring, have been read
#pragma unroll
    for (int i = 0; i < F::kStages - 1; ++i) load_step(i);

    // ---- the query: column n of a B operand, 16 (q4 + 4 i) + 4 w + e of the row in k-step 4 i + w --------------------
    uint32_t qf[NT][KS][2];
    float factor[NT][2];             // of the columns 2 q4, 2 q4 + 1 that the lane has scores of
    int hi_of[NT][2], lo_of[NT][2];  // keys that they see
#pragma unroll
    for (int n = 0; n < NT; ++n) {
      const int col = 8 * n + g, r = r0 + min(col, n_cols - 1), t = by_group(a, r);
      const bf16* row = a.q + (long long)(s.first + t) * a.q_row + (long long)(it.head * a.G + (r - t * a.G)) * a.q_head;
      uint4 raw[KS / 4][2];
      float amax = 0.f;
#pragma unroll
      for (int i = 0; i < KS / 4; ++i) {
        raw[i][0] = *reinterpret_cast<const uint4*>(row + 16 * (q4 + 4 * i));
        raw[i][1] = *reinterpret_cast<const uint4*>(row + 16 * (q4 + 4 * i) + 8);
#pragma unroll
        for (int w = 0; w < 8; ++w) {
          const uint32_t two = word(raw[i][w >> 2], w & 3);
          const float x = fabsf(__uint_as_float(two << 16)), y = fabsf(__uint_as_float(two & 0xffff0000u));
          amax = fmaxf(amax, fmaxf(x <= 3.402823466e38f ? x : 0.f, y <= 3.402823466e38f ? y : 0.f));
        }
      }
      amax = fmaxf(amax, __shfl_xor_sync(0xffffffffu, amax, 1));
      amax = fmaxf(amax, __shfl_xor_sync(0xffffffffu, amax, 2));
      const int e = max(exponent_of(amax), -100) - 14;
      const float up = power_of_two(-e), back = power_of_two(e) * a.scale_log2e;
#pragma unroll
      for (int i = 0; i < KS / 4; ++i)
#pragma unroll
        for (int w = 0; w < 8; ++w) {
          const uint32_t two = word(raw[i][w >> 2], w & 3);
          qf[n][4 * i + (w >> 1)][w & 1] = half2_of(__uint_as_float(two << 16) * up, __uint_as_float(two & 0xffff0000u) * up);
        }
      const KeyRange seen = keys_of(a, s, t);
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        const int from = (2 * q4 + j) * 4;                       // a lane of that column
        factor[n][j] = __shfl_sync(0xffffffffu, back, from);
        hi_of[n][j] = __shfl_sync(0xffffffffu, seen.hi, from);
        lo_of[n][j] = __shfl_sync(0xffffffffu, seen.lo, from);
      }
    }
    // keys that every column sees, and that any does
    int all_lo = 0, all_hi = 0x7fffffff, any_hi = 0, any_lo = 0x7fffffff;
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        all_lo = max(all_lo, lo_of[n][j]); all_hi = min(all_hi, hi_of[n][j]);
        any_lo = min(any_lo, lo_of[n][j]); any_hi = max(any_hi, hi_of[n][j]);
      }
    all_lo = __reduce_max_sync(0xffffffffu, all_lo); all_hi = __reduce_min_sync(0xffffffffu, all_hi);
    any_lo = __reduce_min_sync(0xffffffffu, any_lo); any_hi = __reduce_max_sync(0xffffffffu, any_hi);

    const bool uneven = any_lo < all_lo || all_hi < any_hi;

    float o[NT][KS][4];              // O^T: tile m of 16 dims; rows g -> (D / 8) g + 2 m, g + 8 -> that + 1; columns 2 q4, 2 q4 + 1
    float m_run[NT][2], l_run[NT][2];
#pragma unroll
    for (int n = 0; n < NT; ++n) {
#pragma unroll
      for (int i = 0; i < KS; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) o[n][i][j] = 0.f;
      m_run[n][0] = m_run[n][1] = -INFINITY;
      l_run[n][0] = l_run[n][1] = 0.f;
    }

    for (int i = 0; kStepPages * i < it.n; ++i) {
      __syncwarp();                  // every lane is done with the step before: its place in the ring is free
      load_step(i + F::kStages - 1);
      cp_async_wait<F::kStages - 1>();
      __syncwarp();                  // this step's codes are here
      const uint32_t at = ring + (uint32_t)((i % F::kStages) * F::kStage);
      const bool mine = kStepPages * i + warp / 2 < it.n;
      const float2 scales = mine ? meta[i % F::kStages] : make_float2(-1.f, 1.f);
      const int key0 = (it.page + kStepPages * i + warp / 2) * kPage + (warp & 1) * kWarpKeys;
      if (scales.x < 0.f || key0 >= any_hi || key0 + kWarpKeys <= any_lo) continue;      // (the same for the whole warp)
      // S^T = K q^T, two tiles of 16 keys
      float sc[NT][2][4];
#pragma unroll
      for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int b = 0; b < 2; ++b) sc[n][b][0] = sc[n][b][1] = sc[n][b][2] = sc[n][b][3] = 0.f;
#pragma unroll
      for (int b = 0; b < 2; ++b)
#pragma unroll
        for (int h = 0; h < KS / 4; ++h) {
          const uint4 ka = lds128(at + k_place(16 * b + g, q4 + 4 * h, D)), kb = lds128(at + k_place(16 * b + g + 8, q4 + 4 * h, D));
#pragma unroll
          for (int w = 0; w < 4; ++w) {
            uint32_t a0, a1, a2, a3;
            codes_to_half2(word(ka, w), a0, a2);
            codes_to_half2(word(kb, w), a1, a3);
#pragma unroll
            for (int n = 0; n < NT; ++n) mma_f16(sc[n][b], a0, a1, a2, a3, qf[n][4 * h + w][0], qf[n][4 * h + w][1]);
          }
        }
      const int ev = value_exponent(scales.y);
      const float evf = (float)ev, down = power_of_two(-ev);
      const bool edge = key0 < all_lo || key0 + kWarpKeys > all_hi;
      uint32_t pf[NT][2][2];
#pragma unroll
      for (int n = 0; n < NT; ++n) {
        // x of keys g + 8 k of columns 2 q4, 2 q4 + 1: x[2 k], x[2 k + 1]
        float x[8], mx[2], m_new[2];
        bool moved = false, far[2];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          x[j] = fmaf(sc[n][j >> 2][j & 3], factor[n][j & 1] * scales.x, evf);
          const int key = key0 + g + 8 * (j >> 1);
          if (edge && (key >= hi_of[n][j & 1] || key < lo_of[n][j & 1])) x[j] = -INFINITY;
        }
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          mx[j] = fmaxf(fmaxf(x[j], x[j + 2]), fmaxf(x[j + 4], x[j + 6]));
          mx[j] = fmaxf(mx[j], __shfl_xor_sync(0xffffffffu, mx[j], 4));
          mx[j] = fmaxf(mx[j], __shfl_xor_sync(0xffffffffu, mx[j], 8));
          mx[j] = fmaxf(mx[j], __shfl_xor_sync(0xffffffffu, mx[j], 16));
          m_new[j] = fmaxf(m_run[n][j], mx[j]);
          moved = moved || m_new[j] > m_run[n][j];
          far[j] = mx[j] < m_new[j] - kFar && mx[j] > -INFINITY;
        }
        if (__any_sync(0xffffffffu, moved)) {
          float r[2];
#pragma unroll
          for (int j = 0; j < 2; ++j) {
            const float d = m_run[n][j] - m_new[j];
            r[j] = m_run[n][j] == -INFINITY ? 1.f : ex2_approx(d);
            l_run[n][j] = m_run[n][j] == -INFINITY ? l_run[n][j] : moved_sum(l_run[n][j], d);
            m_run[n][j] = m_new[j];
          }
#pragma unroll
          for (int i2 = 0; i2 < KS; ++i2)
#pragma unroll
            for (int j = 0; j < 4; ++j) o[n][i2][j] *= r[j & 1];
        }
        if ((float)ev < -kSumTop)
#pragma unroll
          for (int j = 0; j < 2; ++j) if (mx[j] - evf - m_run[n][j] > kSumTop) l_run[n][j] = shift_sum(l_run[n][j]);
        const float ref[2] = {m_run[n][0] == -INFINITY ? 0.f : m_run[n][0] - kLift, m_run[n][1] == -INFINITY ? 0.f : m_run[n][1] - kLift};
        float p[8];
        if (!__any_sync(0xffffffffu, far[0] || far[1])) {
#pragma unroll
          for (int j = 0; j < 8; ++j) p[j] = ex2_approx(x[j] - ref[j & 1]);
#pragma unroll
          for (int j = 0; j < 2; ++j) l_run[n][j] = fmaf((p[j] + p[j + 2]) + (p[j + 4] + p[j + 6]), sum_factor(l_run[n][j], down), l_run[n][j]);
        } else {
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            const int c = j & 1;
            p[j] = ex2_approx(x[j] - (far[c] ? mx[c] : ref[c]));
            l_run[n][c] = fmaf(p[j], sum_factor(l_run[n][c], far[c] ? exp2f(mx[c] - ref[c] - evf) : down), l_run[n][c]);
            if (far[c]) p[j] = 0.f;
          }
        }
#pragma unroll
        for (int b = 0; b < 2; ++b) {
          pf[n][b][0] = transpose_8x8(half2_of(p[4 * b], p[4 * b + 1]));
          pf[n][b][1] = transpose_8x8(half2_of(p[4 * b + 2], p[4 * b + 3]));
        }
      }
      // O^T += V^T P^T: the lane's piece of dims, keys 2 q4, 2 q4 + 1, 2 q4 + 8, 2 q4 + 9 of either tile
#pragma unroll
      for (int b = 0; b < 2; ++b) {
        uint32_t vw[4][D / 32];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const int r = 16 * b + 2 * q4 + (j & 1) + 8 * (j >> 1);
          if constexpr (D == 128) {
            const uint4 v = lds128(at + (uint32_t)F::kTile + v_place(r, g, D));
            vw[j][0] = v.x; vw[j][1] = v.y; vw[j][2] = v.z; vw[j][3] = v.w;
          } else {
            const uint2 v = lds64(at + (uint32_t)F::kTile + v_place(r, g >> 1, D) + 8u * (uint32_t)(g & 1));
            vw[j][0] = v.x; vw[j][1] = v.y;
          }
          // what no row sees may be anything, NaN among it, which a weight of 0 does not stop
          if (edge && (key0 + r >= any_hi || key0 + r < any_lo))
#pragma unroll
            for (int w = 0; w < D / 32; ++w) vw[j][w] = 0u;
        }
        // what some columns see and others do not: its NaN goes to those that do
        if (edge && uneven) {
          uint32_t nan = 0u;
#pragma unroll
          for (int j = 0; j < 4; ++j)
#pragma unroll
            for (int w = 0; w < D / 32; ++w) nan |= nan_codes(vw[j][w]);
          if (__any_sync(0xffffffffu, nan != 0u)) {
            // ... by a product of its own, of ones: NaN's codes times the keys that a column sees
            uint32_t sf[NT][2];
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
              for (int k = 0; k < 2; ++k) {
                const int key = key0 + 16 * b + g + 8 * k;
                sf[n][k] = transpose_8x8(half2_of(key >= lo_of[n][0] && key < hi_of[n][0] ? 1.f : 0.f, key >= lo_of[n][1] && key < hi_of[n][1] ? 1.f : 0.f));
              }
#pragma unroll
            for (int w = 0; w < D / 32; ++w) {
              uint32_t one[4];
#pragma unroll
              for (int j = 0; j < 4; ++j) {
                const uint32_t at_nan = nan_codes(vw[j][w]);
                one[j] = at_nan * 0x38u;                     // (the code of 1)
                vw[j][w] &= ~(at_nan * 0xffu);
              }
#pragma unroll
              for (int hh = 0; hh < 2; ++hh) {
                uint32_t a0, a1, a2, a3;
                codes_to_half2(__byte_perm(one[0], one[1], hh ? 0x7362 : 0x5140), a0, a1);
                codes_to_half2(__byte_perm(one[2], one[3], hh ? 0x7362 : 0x5140), a2, a3);
#pragma unroll
                for (int n = 0; n < NT; ++n) {
                  float c[4] = {0.f, 0.f, 0.f, 0.f};
                  mma_f16(c, a0, a1, a2, a3, sf[n][0], sf[n][1]);
#pragma unroll
                  for (int k = 0; k < 4; ++k) if (c[k] > 0.f) o[n][2 * w + hh][k] = __int_as_float(0x7fc00000);
                }
              }
            }
          }
        }
#pragma unroll
        for (int w = 0; w < D / 32; ++w)
#pragma unroll
          for (int hh = 0; hh < 2; ++hh) {
            // bytes 2 hh and 2 hh + 1 of the four keys' words
            uint32_t a0, a1, a2, a3;
            codes_to_half2(__byte_perm(vw[0][w], vw[1][w], hh ? 0x7362 : 0x5140), a0, a1);
            codes_to_half2(__byte_perm(vw[2][w], vw[3][w], hh ? 0x7362 : 0x5140), a2, a3);
#pragma unroll
            for (int n = 0; n < NT; ++n) mma_f16(o[n][2 * w + hh], a0, a1, a2, a3, pf[n][b][0], pf[n][b][1]);
          }
      }
    }
    cp_async_wait<0>();
    __syncthreads();                 // nobody reads the ring any more

    // ---- the four warps' rows, joined --------------------------------------------------------------------------
    float* rows = reinterpret_cast<float*>(smem);                  // [warp][column][kRowF], then [warp][column] (m, l)
    float2* stats = reinterpret_cast<float2*>(rows + kWarps * W * F::kRowF);
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        auto of_column = [&](float l) {
          l += __shfl_xor_sync(0xffffffffu, l, 4);
          l += __shfl_xor_sync(0xffffffffu, l, 8);
          return l + __shfl_xor_sync(0xffffffffu, l, 16);
        };
        const bool wide = shifted(l_run[n][j]);
        float l = of_column(l_run[n][j]);
        if (__any_sync(0xffffffffu, wide))
          l = chosen(of_column(wide ? -kSumUp * l_run[n][j] : l_run[n][j]), of_column(wide ? -l_run[n][j] : kSumDown * l_run[n][j]));
        const int col = 8 * n + 2 * q4 + j;
        if (g == 0) stats[warp * W + col] = make_float2(l == l ? m_run[n][j] : INFINITY, l);      // (NaN goes on as infinity - infinity)
        float* row = rows + (warp * W + col) * F::kRowF + (D / 8) * g;
#pragma unroll
        for (int i = 0; i < KS; ++i) { row[2 * i] = o[n][i][j]; row[2 * i + 1] = o[n][i][j + 2]; }
      }
    __syncthreads();
    const bool begun = it.page > it.first, goes_on = it.page + it.n < it.first + it.of;
    float* part = nullptr;
    if (begun || goes_on) part = part_rows<W, D>(a.parts, cta, begun ? 0 : 1);
    for (int i = tid; i < n_cols * (D / 4); i += kThreads) {
      const int col = i / (D / 4), d = (i - col * (D / 4)) * 4;
      float m = -INFINITY;
#pragma unroll
      for (int w = 0; w < kWarps; ++w) m = fmaxf(m, stats[w * W + col].x);
      float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
      float l = 0.f;
      bool wide = false;
#pragma unroll
      for (int w = 0; w < kWarps; ++w) {
        const float2 st = stats[w * W + col];
        const float f = st.x == -INFINITY ? 0.f : exp2f(st.x - m);
        const float4 x = *reinterpret_cast<const float4*>(rows + (w * W + col) * F::kRowF + d);
        v.x = fmaf(f, x.x, v.x); v.y = fmaf(f, x.y, v.y); v.z = fmaf(f, x.z, v.z); v.w = fmaf(f, x.w, v.w);
        l += st.x == -INFINITY ? 0.f : times_power(st.y, st.x - m);
        wide = wide || shifted(st.y);
      }
      if (wide) {
        float by_2_64 = l = 0.f;
#pragma unroll 1
        for (int w = 0; w < kWarps; ++w) {
          const float2 st = stats[w * W + col];
          if (st.x == -INFINITY) continue;
          l += as_is(st.y, st.x - m);
          by_2_64 += as_shifted(st.y, st.x - m);
        }
        l = chosen(l, by_2_64);
      }
      if (part != nullptr) {
        *reinterpret_cast<float4*>(part + (size_t)col * D + d) = v;
        if (d == 0) part_stats<W, D>(a.parts, cta, begun ? 0 : 1)[col] = make_float2(m - kLift, l);
      } else {
        const RowHead to = row_head(a, s.first, r0 + col, it.head);
        store_row_piece(a, to, d, times(v, reciprocal(l)));
        if (d == 0) store_lse(a, to, m - kLift, l);
      }
    }
    if (begun && !goes_on && tid == 0) {
      a.joins[cta] = make_int4(1 + runs.cta_of(u - it.span - (it.page - it.first)), s.first, r0, it.head | (n_cols << 16));
    }
  }
}

// ---- rows that several CTAs worked on ------------------------------------------------------------------------------
constexpr int kJoinWarps = 8, kJoinThreads = 32 * kJoinWarps, kJoinBlocks = 4 * 148;
struct JoinShared {
  int4 list[kFewCtas];                  // what the last CTA of an item noted
  int last[kFewCtas], count[(kFewCtas + 31) / 32];
  float2 st[kJoinWarps];
  float4 o[kJoinWarps][32];
};
// Parts of a row, up to 32 side by side: a lane knows one's reference and sum (on: there is one), and has four dims of each, which `get` gives
// for any of them.  m, l: of all of them, in every lane; o: the lane's dims relative to m.
template <typename Get>
__device__ __forceinline__ void join_parts(int n, bool on, float2 st, float& m, float& l, float4& o, Get get) {
  constexpr int U = 8;                                     // on their way at a time
  float4 v[U];
#pragma unroll
  for (int i = 0; i < U; ++i) v[i] = i < n ? get(i) : make_float4(0.f, 0.f, 0.f, 0.f);
  on = on && st.x != -INFINITY;
  float top = on ? st.x : -INFINITY;
#pragma unroll
  for (int k = 16; k > 0; k >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, k));
  top = fmaxf(top, m);
  const float f = on ? exp2f(st.x - top) : -1.f;           // (-1: nothing there)
  float sum = on ? times_power(st.y, st.x - top) : 0.f;
#pragma unroll
  for (int k = 16; k > 0; k >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, k);
  if (m != -INFINITY) {
    const float r = exp2f(m - top);
    o.x *= r; o.y *= r; o.z *= r; o.w *= r;
    sum += times_power(l, m - top);
  }
  l = sum;
  m = top;
#pragma unroll 1
  for (int c = 0; c < n; c += U) {
#pragma unroll
    for (int i = 0; i < U; ++i) {
      const float fi = __shfl_sync(0xffffffffu, f, c + i);
      if (c + i < n && fi != -1.f) { o.x = fmaf(fi, v[i].x, o.x); o.y = fmaf(fi, v[i].y, o.y); o.z = fmaf(fi, v[i].z, o.z); o.w = fmaf(fi, v[i].w, o.w); }
    }
#pragma unroll
    for (int i = 0; i < U; ++i) v[i] = c + U + i < n ? get(c + U + i) : make_float4(0.f, 0.f, 0.f, 0.f);
  }
}
// one more part of a row: a lane four dims of it
struct Sum { float m, l; float4 o; };
__device__ __forceinline__ void add_part(Sum& s, float2 st, float4 v) {
  if (st.x == -INFINITY) return;
  const float m = fmaxf(s.m, st.x), fa = s.m == -INFINITY ? 0.f : exp2f(s.m - m), fb = exp2f(st.x - m);
  s.o.x = s.o.x * fa + v.x * fb; s.o.y = s.o.y * fa + v.y * fb; s.o.z = s.o.z * fa + v.z * fb; s.o.w = s.o.w * fa + v.w * fb;
  s.l = (s.m == -INFINITY ? 0.f : times_power(s.l, s.m - m)) + times_power(st.y, st.x - m);
  s.m = m;
}
// l of a row of which a part's sum is held times 2^-64, by a warp: m is the largest reference of CTAs first ... last.  (Apart from the rest, which
// knows of none: 0.5 us of a question's join otherwise.)
template <int W, int D>
__device__ __noinline__ float sum_of_parts(float* parts, int first, int last, int col, float m) {
  float l = 0.f, by_2_64 = 0.f;
  for (int c = first + (int)(threadIdx.x & 31); c <= last; c += 32) {
    const float2 st = part_stats<W, D>(parts, c, c == first ? 1 : 0)[col];
    if (st.x == -INFINITY) continue;
    l += as_is(st.y, st.x - m);
    by_2_64 += as_shifted(st.y, st.x - m);
  }
#pragma unroll
  for (int k = 16; k > 0; k >>= 1) { l += __shfl_xor_sync(0xffffffffu, l, k); by_2_64 += __shfl_xor_sync(0xffffffffu, by_2_64, k); }
  return chosen(l, by_2_64);
}
// The items that a kernel's CTAs left in parts, by all blocks: a block lists the CTAs that were the last on an item others had begun.  Where
// these are many, and so of few parts each, it takes eight columns of an item at a time, a warp to each; else one, its parts shared by the warps.
// (Sixteen items of two parts, 224 columns: 7 us more column by column.  Four of 36 parts: 8 us, 16.5 MB of parts.)
template <int W, int D>
__device__ __forceinline__ void join_items(const CacheAttnArgs& a, const int4* joins, float* parts, int ctas, JoinShared& sm) {
  constexpr int CHUNKS = (kFewCtas + 31) / 32, PER = (CHUNKS + kJoinWarps - 1) / kJoinWarps;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  // (in the order of the CTAs: the same list in every block)
  unsigned set[PER];
  int4 note[PER];
#pragma unroll
  for (int k = 0; k < PER; ++k) {
    const int chunk = warp + kJoinWarps * k, c = 32 * chunk + lane;
    note[k] = joins[min(c, ctas - 1)];
    set[k] = __ballot_sync(0xffffffffu, c < ctas && note[k].x != 0);
    if (lane == 0 && chunk < CHUNKS) sm.count[chunk] = __popc(set[k]);
  }
  __syncthreads();
  int listed = 0;
  for (int i = 0; i < CHUNKS; ++i) listed += sm.count[i];
#pragma unroll
  for (int k = 0; k < PER; ++k) {
    const int chunk = warp + kJoinWarps * k;
    int at = __popc(set[k] & ((1u << lane) - 1u));
    for (int i = 0; i < min(chunk, CHUNKS); ++i) at += sm.count[i];
    if ((set[k] >> lane) & 1u) { sm.list[at] = note[k]; sm.last[at] = 32 * chunk + lane; }
  }
  __syncthreads();
  auto finish = [&](const int4& j, int col, float m, float l, const float4& o) {
    const RowHead to = row_head(a, j.y, j.z + col, j.w & 0xffff);
    if (lane < D / 4) store_row_piece(a, to, 4 * lane, times(o, reciprocal(l)));
    if (lane == 0) store_lse(a, to, m, l);
  };
  if constexpr (W >= 8 * kJoinWarps) {
    constexpr int U = 4, groups = W / kJoinWarps;                       // parts on their way at a time
    if (2 * listed * groups >= (int)gridDim.x) {
      for (int at = (int)blockIdx.x; at < listed * groups; at += (int)gridDim.x) {
        const int item = at / groups, col = (at % groups) * kJoinWarps + warp;
        const int4 j = sm.list[item];
        const int first = j.x - 1, last = sm.last[item];
        if (col >= (j.w >> 16)) continue;                   // (the whole warp)
        Sum s = {-INFINITY, 0.f, make_float4(0.f, 0.f, 0.f, 0.f)};
        bool wide = false;
#pragma unroll 1
        for (int c0 = first; c0 <= last; c0 += U) {
          float2 st[U];
          float4 v[U];
#pragma unroll
          for (int i = 0; i < U; ++i) {
            const int c = min(c0 + i, last), place = c == first ? 1 : 0;
            st[i] = c0 + i <= last ? part_stats<W, D>(parts, c, place)[col] : make_float2(-INFINITY, 0.f);
            v[i] = c0 + i <= last && lane < D / 4 ? *reinterpret_cast<const float4*>(part_rows<W, D>(parts, c, place) + (size_t)col * D + 4 * lane)
                                                  : make_float4(0.f, 0.f, 0.f, 0.f);
          }
#pragma unroll
          for (int i = 0; i < U; ++i) { add_part(s, st[i], v[i]); wide = wide || shifted(st[i].y); }
        }
        if (wide) s.l = sum_of_parts<W, D>(parts, first, last, col, s.m);
        finish(j, col, s.m, s.l, s.o);
      }
      return;
    }
  }
  for (int at = (int)blockIdx.x; at < listed * W; at += (int)gridDim.x) {
    const int item = at / W, col = at % W;
    const int4 j = sm.list[item];
    const int first = j.x - 1, last = sm.last[item];
    if (col >= (j.w >> 16)) continue;                      // (the whole block)
    float m = -INFINITY, l = 0.f;
    float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
    bool wide = false;
#pragma unroll 1
    for (int c0 = first + warp; c0 <= last; c0 += 32 * kJoinWarps) {
      const int n = min(32, (last - c0) / kJoinWarps + 1);
      auto place = [&](int c) { return c == first ? 1 : 0; };
      const int mine = c0 + min(lane, n - 1) * kJoinWarps;
      const float2 st = part_stats<W, D>(parts, mine, place(mine))[col];
      wide = wide || shifted(st.y);
      join_parts(n, lane < n, st, m, l, o, [&](int i) {
        const int c = c0 + i * kJoinWarps;
        return lane < D / 4 ? *reinterpret_cast<const float4*>(part_rows<W, D>(parts, c, place(c)) + (size_t)col * D + 4 * lane) : make_float4(0.f, 0.f, 0.f, 0.f);
      });
    }
    __syncthreads();                                        // (the round before has been read)
    if (__any_sync(0xffffffffu, wide)) l = -1.f;            // (to be summed up apart)
    if (lane == 0) sm.st[warp] = make_float2(m, l);
    sm.o[warp][lane] = o;
    __syncthreads();
    if (warp != 0) continue;
    m = -INFINITY;
    o = make_float4(0.f, 0.f, 0.f, 0.f);
    const float2 of_warp = sm.st[lane & (kJoinWarps - 1)];
    join_parts(kJoinWarps, lane < kJoinWarps, of_warp, m, l, o, [&](int i) { return sm.o[i][lane]; });
    if (__any_sync(0xffffffffu, shifted(of_warp.y))) l = sum_of_parts<W, D>(parts, first, last, col, m);
    finish(j, col, m, l, o);
  }
}
struct Parts { int4* joins; float* parts; int ctas; };
template <int D, int WF, bool kMany>
__global__ void __launch_bounds__(kJoinThreads, kJoinBlocks / 148) cache_attention_join_kernel(const __grid_constant__ CacheAttnArgs a, Parts few, Parts many) {
  __shared__ JoinShared sm;
  pdl_wait();
  if constexpr (WF > 0) join_items<WF, D>(a, few.joins, few.parts, few.ctas, sm);
  if constexpr (WF > 0 && kMany) __syncthreads();
  if constexpr (kMany) join_items<kManyWide, D>(a, many.joins, many.parts, many.ctas, sm);
}

// as many as are resident: three an SM of 168 registers a thread, two of 255 (sixteen sequences of 13440 tokens, two rows of seven heads: 58.7 us; in one and a half
// rounds 78.2)
int few_ctas(int cols) { return cols <= 8 ? kFewCtas : 2 * 148; }
template <int D, int NT>
int launch_few(const CacheAttnArgs& a, cudaStream_t st) {
  using F = Few<D, NT>;
  // (the limit is the function's, not the call's: that of the most sequences, so that calls of other threads set the same)
  if (cudaFuncSetAttribute(cache_attention_few_kernel<D, NT>, cudaFuncAttributeMaxDynamicSharedMemorySize, F::bytes(VS_CACHE_MAX_SEQS)) != cudaSuccess) return VS_ERR_CUDA;
  cache_attention_few_kernel<D, NT><<<few_ctas(8 * NT), kThreads, F::bytes(a.r.n_seqs), st>>>(a);
  return launched();
}

template <int D, int WF, bool kMany>
int launch_join(const CacheAttnArgs& a, Parts few, Parts many, cudaStream_t st) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(kJoinBlocks);
  cfg.blockDim = dim3(kJoinThreads);
  cfg.stream = st;
  // (Its blocks come when those ahead have ended; let in from the start, they take 1.5 us from a call of 13.8 that they wait through.)
  cudaLaunchAttribute at = {};
  at.id = cudaLaunchAttributeProgrammaticStreamSerialization;
  at.val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = &at;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, cache_attention_join_kernel<D, WF, kMany>, a, few, many) == cudaSuccess ? launched() : VS_ERR_CUDA;
}
template <int D>
int join(const CacheAttnArgs& a, Parts few, Parts many, int cols, bool with_many, cudaStream_t st) {
  if (cols == 0) return launch_join<D, 0, true>(a, few, many, st);
  if (with_many) return launch_join<D, 16, true>(a, few, many, st);
  return cols <= 8 ? launch_join<D, 8, false>(a, few, many, st) : launch_join<D, 16, false>(a, few, many, st);
}

}  // namespace

int launch_cache_attention_few(const CacheAttnArgs& a, int cols, cudaStream_t st) {
  if (cols <= 8) return a.c.head_dim == 128 ? launch_few<128, 1>(a, st) : launch_few<64, 1>(a, st);
  return a.c.head_dim == 128 ? launch_few<128, 2>(a, st) : launch_few<64, 2>(a, st);
}

}  // namespace vs

namespace {
constexpr int kFewPageShift = 2, kManyPageShift = 2;            // four pages at least
// the workspace: status word, the CTAs' notes and parts of either kernel
constexpr size_t kFewJoinsAt = 256, kManyJoinsAt = kFewJoinsAt + vs::kFewCtas * 16, kPartsAt = 16384;
static_assert(kManyJoinsAt + vs::kManyCtas * 16 <= kPartsAt && vs::kManyCtas <= vs::kFewCtas, "notes of the CTAs");
size_t few_bytes(int head_dim) { return (size_t)vs::kFewCtas * 2 * vs::kFewWide * (head_dim + 2) * 4; }
size_t many_bytes(int head_dim) { return (size_t)vs::kManyCtas * 2 * vs::kManyWide * (head_dim + 2) * 4; }
}

extern "C" int vs_cache_attention_bytes(int32_t head_dim, size_t* out_bytes) {
  if (out_bytes == nullptr) return VS_ERR_INVALID_ARG;
  if (head_dim != 64 && head_dim != 128) return VS_ERR_UNSUPPORTED;
  *out_bytes = kPartsAt + few_bytes(head_dim) + many_bytes(head_dim);
  return VS_OK;
}

extern "C" int vs_cache_attention(const vs_cache* cache, const vs_cache_queries* x, void* cuda_stream) {
  using namespace vs;
  if (x == nullptr) return VS_ERR_INVALID_ARG;
  const vs_cache_seqs* rows = &x->seqs;
  const int rc = check_cache(cache, rows);
  if (rc != VS_OK) return rc;
  if (x->n_q_heads < 1 || x->window < 0 || x->out_dtype < 0 || x->out_dtype > 1 || !(x->scale > 0.f) || !std::isfinite(x->scale)) return VS_ERR_INVALID_ARG;
  if (x->n_q_heads % cache->n_kv_heads != 0 || x->n_q_heads / cache->n_kv_heads > 8) return VS_ERR_UNSUPPORTED;
  const int G = x->n_q_heads / cache->n_kv_heads;
  if (rows->n_rows > (1 << 27)) return VS_ERR_UNSUPPORTED;
  size_t need = 0;
  vs_cache_attention_bytes(cache->head_dim, &need);
  if (rows->n_rows == 0) return VS_OK;
  if (x->q == nullptr || x->out == nullptr || x->workspace == nullptr) return VS_ERR_INVALID_ARG;
  if (x->workspace_bytes < need) return VS_ERR_CAPACITY;
  if (!aligned(x->q, 16) || !aligned(x->out, x->out_dtype == 1 ? 16 : 8) || !aligned(x->workspace, 256) || !aligned(x->lse, 4)) return VS_ERR_INVALID_ARG;
  if (x->q_row_stride % 8 != 0 || x->q_head_stride % 8 != 0 || x->out_row_stride % 4 != 0 || x->out_head_stride % 4 != 0) return VS_ERR_INVALID_ARG;
  // (in place: an item's rows of q are read before they are written, by the CTA that writes them or two launches ahead)
  if (x->q == x->out && (x->out_dtype != 0 || x->q_row_stride != x->out_row_stride || x->q_head_stride != x->out_head_stride)) return VS_ERR_INVALID_ARG;
  OnDevice on(cache->device);
  if (!on.ok) return VS_ERR_CUDA;
  CacheAttnArgs a = {};
  a.c = *cache; a.r = *rows;
  a.q = static_cast<const bf16*>(x->q); a.out = x->out; a.lse = x->lse;
  uint8_t* ws = static_cast<uint8_t*>(x->workspace);
  a.status = reinterpret_cast<int*>(ws);
  a.q_row = x->q_row_stride; a.q_head = x->q_head_stride; a.out_row = x->out_row_stride; a.out_head = x->out_head_stride;
  a.scale_log2e = x->scale * 1.4426950408889634f;
  a.Hq = x->n_q_heads; a.G = G; a.causal = x->causal != 0; a.window = x->window; a.out_fp32 = x->out_dtype;
  a.rcp_g = G == 1 ? 0u : (uint32_t)(((1ull << 32) + G - 1) / G);
  const bool uniform = rows->row_offsets == nullptr;
  while (a.side_shift < 5 && rows->n_seqs << (a.side_shift + 1) <= 32) ++a.side_shift;
  a.rows_each = uniform ? rows->n_rows / rows->n_seqs : -1;
  a.max_held = rows->table_width >= (1 << 25) ? 0x7fffffff - (kPage - 1) : rows->table_width * kPage;      // (whole pages)
  // Which sequences have few rows the device knows; the host, from the number of rows, that all of them have (or none, where they have the
  // same number each).  Either kind has its kernel; what their CTAs left in parts one launch joins.
  const long long most = (long long)(uniform ? a.rows_each : rows->n_rows) * G;
  // The kernel of few rows takes a sequence of up to 32 packed rows, two of its tiles (seven heads a group, four KV heads, four rows: 16.0 us against the
  // other's 19.2 over 13440 tokens, 97 against 107 for sixteen sequences; six rows, three tiles: 20.7 and 20.6, 136 and 108), and any while there are few
  // tiles and pages: the other one's items begin and end slowly (32 rows over 300 tokens 14.1 and 21.0, over 1500 19.5 and 23.3, over 6000 31.4 and 24.7; four
  // sequences of 32 rows over 300 tokens, 1568 tiles times pages of a table, 16.5 and 21.5; of 12 over 1500, 2496, 22.4 and 18.5).
  const long long tiles = uniform ? (long long)rows->n_seqs * ((a.rows_each * G + kFewWide - 1) / kFewWide) : (long long)rows->n_rows * G / kFewWide + rows->n_seqs;
  const long long items = tiles * cache->n_kv_heads;
  a.few_cols = items <= few_ctas(kFewWide) && items * rows->table_width <= 1600 ? 0x7fffffff : 32;
  const bool any_few = most <= a.few_cols || !uniform, any_many = most > a.few_cols;
  const int cols = any_few ? (most <= 8 ? 8 : kFewWide) : 0;
  const Parts few = {reinterpret_cast<int4*>(ws + kFewJoinsAt), reinterpret_cast<float*>(ws + kPartsAt), few_ctas(cols)};
  const Parts many = {reinterpret_cast<int4*>(ws + kManyJoinsAt), reinterpret_cast<float*>(ws + kPartsAt + few_bytes(cache->head_dim)), kManyCtas};
  cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
  if (any_few) {
    a.take_few = 1; a.page_shift = kFewPageShift; a.joins = few.joins; a.parts = few.parts;
    const int r = launch_cache_attention_few(a, cols, st);
    if (r != VS_OK) return r;
  }
  if (any_many) {
    a.take_few = 0; a.page_shift = kManyPageShift; a.joins = many.joins; a.parts = many.parts;
    const int r = launch_cache_attention_many(a, any_few, st);
    if (r != VS_OK) return r;
  }
  return cache->head_dim == 128 ? join<128>(a, few, many, cols, any_many, st) : join<64>(a, few, many, cols, any_many, st);
}
