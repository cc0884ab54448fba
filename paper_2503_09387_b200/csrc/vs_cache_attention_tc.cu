// Attention over the paged 8-bit cache for sequences of many rows (a question, a frame, several frames), on the 5th-generation
// tensor cores.  Mathematics and the cut of the work as in vs_cache_attention.cu: O += 2^{x - m + lift} code_v, l += that * 2^{-ev}, o = O / l.
//
// A CTA (one an SM) takes runs of (item, page) units one after the other; an item is 256 packed rows (row t, head g of the group: t G + g) of one KV
// head: two tiles of 128, the MMA's M.  Steps of two pages = 128 keys:
//   loader     pages' codes by bulk copies (8 KB each at 128 dims: a page and head lies side by side) into a ring of raw tiles
//   converters (4 warps) codes -> fp16, exactly, into the operands' 128-byte-swizzled layout, a ring of three 128-key tiles K, V, K, ...
//   issuer     S_i = Q_i K^T (M 128, N 128), O_i += P_i V (A = P_i from tensor memory), tile 0 and tile 1 by turns: one's softmax runs under the
//              other's products
//   softmax    (4 warps a tile, a thread a row) S from tensor memory, P (fp16) back over it; a row of O is rescaled there only when its
//              maximum has grown by more than 2^8
// Tensor memory: S_0, S_1 (P over their first half), O_0, O_1, 128 columns each: all 512.
//
// The codes go to fp16 once a step and CTA and serve 256 rows: fewer rows would convert more than they multiply, and fp8 operands would need the weights in
// 8 bits, whose range of 2^18 loses a long row's many small ones beside one large one.  The query is held as fp16, exactly (see there).
// All waits are bounded.
#include "vs_cache_attention.cuh"
#include "vs_ptx.cuh"

namespace vs {

namespace {

constexpr int kRows = 128, kTiles = 2, kWide = kRows * kTiles, kStepKeys = 2 * kPage;
constexpr int kSoftWarps = 4 * kTiles, kConvWarps = 4, kLoaderWarp = kSoftWarps + kConvWarps, kIssuerWarp = kLoaderWarp + 1;
constexpr int kThreads = 32 * 16;                       // (warpgroups: softmax of either tile, converters, loader + issuer)
constexpr int kSoftRegs = 184, kConvRegs = 72, kRestRegs = 72;
static_assert(2 * kSoftRegs + kConvRegs + kRestRegs <= 512, "the registers the block is launched with: 128 a thread");
constexpr float kLift = 7.f, kLazy = 8.f;              // weights reach 2^(lift + lazy) <= 2^15
constexpr int kRaw = 7, kSlots = 3;

template <int D>
struct Tc {
  static constexpr int kQTile = kRows * D * 2, kSlot = kStepKeys * D * 2, kRawTile = kPage * D;
  static constexpr int kQ = 0, kF16 = kTiles * kQTile, kRawAt = kF16 + kSlots * kSlot, kCtl = kRawAt + kRaw * kRawTile;
  static constexpr int kBars = 2 * kRaw + 2 * kSlots + 6 * kTiles;
  static constexpr int kFlags = kCtl + 8 * kBars;       // [raw tile] first and end of the rows that count (end 0: the page is not there)
  static constexpr int kSlotWord = kFlags + 8 * kRaw;
  static constexpr int kBefore = (kSlotWord + 8 + 7) / 8 * 8;
  static int bytes(int n_seqs) { return kBefore + 8 * (n_seqs + 1); }
};

// kind::f16 instruction descriptor: D fp32, A = B = fp16, M 128, N = n; b_mn = 1: B is MN-major
__device__ __forceinline__ uint32_t idesc_f16(int n, int b_mn) { return (1u << 4) | ((uint32_t)b_mn << 16) | ((uint32_t)(n >> 3) << 17) | ((uint32_t)(kRows >> 4) << 24); }

// a thread's TMEM lane, 32 columns
__device__ __forceinline__ void tmem_ld_row32(uint32_t taddr, uint32_t* r) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x32.b32 "
      "{%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]),
        "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]), "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]),
        "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
      : "r"(taddr) : "memory");
}
__device__ __forceinline__ void tmem_st_row32(uint32_t taddr, const uint32_t* r) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x32.b32 [%0], "
      "{%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31,%32};"
      ::"r"(taddr), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]), "r"(r[10]),
        "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]), "r"(r[16]), "r"(r[17]), "r"(r[18]), "r"(r[19]), "r"(r[20]), "r"(r[21]),
        "r"(r[22]), "r"(r[23]), "r"(r[24]), "r"(r[25]), "r"(r[26]), "r"(r[27]), "r"(r[28]), "r"(r[29]), "r"(r[30]), "r"(r[31]) : "memory");
}
// the loads before it have arrived in r (the registers as operands: no use of them moves ahead)
__device__ __forceinline__ void tmem_arrived32(uint32_t* r) {
  asm volatile("tcgen05.wait::ld.sync.aligned;"
               : "+r"(r[0]), "+r"(r[1]), "+r"(r[2]), "+r"(r[3]), "+r"(r[4]), "+r"(r[5]), "+r"(r[6]), "+r"(r[7]), "+r"(r[8]), "+r"(r[9]), "+r"(r[10]),
                 "+r"(r[11]), "+r"(r[12]), "+r"(r[13]), "+r"(r[14]), "+r"(r[15]), "+r"(r[16]), "+r"(r[17]), "+r"(r[18]), "+r"(r[19]), "+r"(r[20]),
                 "+r"(r[21]), "+r"(r[22]), "+r"(r[23]), "+r"(r[24]), "+r"(r[25]), "+r"(r[26]), "+r"(r[27]), "+r"(r[28]), "+r"(r[29]), "+r"(r[30]), "+r"(r[31])
               :: "memory");
}
__device__ __forceinline__ void tmem_ld_row16(uint32_t taddr, uint32_t* r) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];\n\t"
      "tcgen05.wait::ld.sync.aligned;"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]),
        "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
      : "r"(taddr) : "memory");
}
__device__ __forceinline__ void tmem_st_row16(uint32_t taddr, const uint32_t* r) {
  asm volatile("tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16};"
               ::"r"(taddr), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]), "r"(r[10]),
                 "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]) : "memory");
}
__device__ __forceinline__ float max3_nan(float a, float b, float c) {
  float r;
  asm("max.NaN.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
  return r;
}
// 2^y of a pair, y <= 16: by the special-function unit (four lanes a clock and scheduler, what bounds the softmax), and by arithmetic for a share of the
// weights: y = n + f, n the nearest integer, 2^f by the polynomial of degree 4 with the least relative error on [-1/2, 1/2] (Remez exchange;
// 2.6e-6, against half a step of 2^-12 that rounding to fp16 adds), n added to the exponent.  Below 2^-126: 2^-126.
constexpr int kByUnit = 8;             // of eight pairs
__device__ __forceinline__ float2 power_by_unit(uint64_t y) {
  const float2 v = f32x2_parts(y);
  return make_float2(ex2_approx(v.x), ex2_approx(v.y));
}
__device__ __forceinline__ float2 power_by_polynomial(uint64_t y) {
  const float2 v = f32x2_parts(y);
  const uint64_t t = f32x2(fmaxf(v.x, -126.f), fmaxf(v.y, -126.f));
  const uint64_t n = add_f32x2(t, f32x2(12582912.f, 12582912.f));         // 1.5 * 2^23: the integer in the low bits
  const uint64_t f = fma_f32x2(add_f32x2(n, f32x2(-12582912.f, -12582912.f)), f32x2(-1.f, -1.f), t);
  uint64_t q = fma_f32x2(f, f32x2(0.009570102207f, 0.009570102207f), f32x2(0.055917859077f, 0.055917859077f));
  q = fma_f32x2(q, f, f32x2(0.240247443318f, 0.240247443318f));
  q = fma_f32x2(q, f, f32x2(0.693121790886f, 0.693121790886f));
  q = fma_f32x2(q, f, f32x2(0.999999284744f, 0.999999284744f));
  const float2 p = f32x2_parts(q), e = f32x2_parts(n);
  return make_float2(__int_as_float(__float_as_int(p.x) + (__float_as_int(e.x) << 23)), __int_as_float(__float_as_int(p.y) + (__float_as_int(e.y) << 23)));
}
__device__ __forceinline__ uint32_t half2_of(float lo, float hi) {
  const __half2 h = __floats2half2_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&h);
}
__device__ __forceinline__ void sts128(uint32_t addr, uint32_t x, uint32_t y, uint32_t z, uint32_t w) {
  asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(addr), "r"(x), "r"(y), "r"(z), "r"(w) : "memory");
}
__device__ __forceinline__ uint4 lds128(uint32_t addr) {
  uint4 v;
  asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(addr) : "memory");
  return v;
}

template <int D>
__global__ void __launch_bounds__(kThreads, 1) cache_attention_tc_kernel(const __grid_constant__ CacheAttnArgs a) {
  using L = Tc<D>;
  extern __shared__ __align__(1024) uint8_t smem[];
  const uint32_t base = smem_u32(smem), ctl = base + L::kCtl;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, group = warp >> 2;
  auto bar_raw_full = [&](uint32_t i) { return ctl + 8u * i; };                                    // a raw tile's bytes are here
  auto bar_raw_free = [&](uint32_t i) { return ctl + 8u * (kRaw + i); };                           // ... converted (an arrival a converter warp)
  auto bar_full = [&](uint32_t i) { return ctl + 8u * (2 * kRaw + i); };                            // an fp16 tile is there (an arrival a converter warp)
  auto bar_free = [&](uint32_t i) { return ctl + 8u * (2 * kRaw + kSlots + i); };                   // ... and multiplied (tcgen05.commit)
  constexpr int kTileBars = 2 * kRaw + 2 * kSlots;
  auto bar_q = [&](int i) { return ctl + 8u * (uint32_t)(kTileBars + i); };                         // the tile's query is in place (an arrival a warp)
  auto bar_p = [&](int i, int h) { return ctl + 8u * (uint32_t)(kTileBars + kTiles * (1 + h) + i); };   // P_i of page h of the step is there, O_i rescaled (an arrival a warp)
  auto bar_s = [&](int i) { return ctl + 8u * (uint32_t)(kTileBars + 3 * kTiles + i); };            // S_i is there (tcgen05.commit)
  auto bar_h = [&](int i) { return ctl + 8u * (uint32_t)(kTileBars + 4 * kTiles + i); };            // page 0 of the step has been added to O_i (tcgen05.commit)
  auto bar_o = [&](int i) { return ctl + 8u * (uint32_t)(kTileBars + 5 * kTiles + i); };            // all of the item's products in O_i (tcgen05.commit)
  volatile int2* flags = reinterpret_cast<volatile int2*>(smem + L::kFlags);
  volatile uint32_t* tmem_slot = reinterpret_cast<volatile uint32_t*>(smem + L::kSlotWord);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(smem + L::kSlotWord + 4);
  long long* before = reinterpret_cast<long long*>(smem + L::kBefore);

  pdl_launch_dependents();
  if (warp == kIssuerWarp) {
    if (lane < L::kBars) {
      const uint32_t i = (uint32_t)lane;
      const bool by_warps = (i >= kRaw && i < 2 * kRaw + kSlots) || (i >= kTileBars && i < kTileBars + 3 * kTiles);
      mbar_init(ctl + 8u * i, by_warps ? 4u : 1u);
    }
    if (lane == 0) *abort_flag = (base & 1023u) != 0;     // (the swizzled layouts need the alignment that the declaration asks for)
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    fence_async_proxy();
  } else if (warp == kLoaderWarp) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32((const void*)tmem_slot)), "r"(512u) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  static_assert(L::kBars <= 32, "a lane a barrier");
  tc_fence_before();
  const long long units = count_units<kWide>(a, before);           // (ends with a barrier of the block)
  tc_fence_after();
  const uint32_t tmem = *tmem_slot, tmem_o = tmem + kTiles * 128u;
  const AttnRuns runs(a, units, (int)gridDim.x);
  const int cta = (int)blockIdx.x;
  if (tid == 0) a.joins[cta] = make_int4(0, 0, 0, 0);
  const bool works = cta < runs.n_ctas && units > 0;
  const long long u_begin = works ? runs.begin(cta) : 0, u_end = works ? runs.begin(cta + 1) : 0;
  auto steps_of = [](const AttnItem& it) { return (it.n + 1) / 2; };

  if (group == 3) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kRestRegs));
    if (warp == kLoaderWarp) {
      // ---- pages' codes: K, K, V, V of a step ------------------------------------------------------------------
      uint32_t loaded = 0;
      bool ok = true;
      for (long long u = u_begin; u < u_end && ok;) {
        const AttnItem it = item_at<kWide>(a, before, u, u_end);
        if (it.n < 1) break;
        u += it.n;
        // keys that any row of the item sees
        const int lo = keys_of(a, it.s, by_group(a, it.r0)).lo, hi = keys_of(a, it.s, by_group(a, it.r0 + it.n_cols - 1)).hi;
        int mine = -1;
        for (int p0 = 0; p0 < it.n && ok; p0 += 2) {
          if ((p0 & 31) == 0) mine = p0 + lane < it.n ? page_of(a.r, a.c.n_pages, it.seq, it.page + p0 + lane) : -1;
          const int two[2] = {__shfl_sync(0xffffffffu, mine, p0 & 31), __shfl_sync(0xffffffffu, mine, (p0 & 31) + 1)};
#pragma unroll 1
          for (int e = 0; e < 4; ++e) {
            const int page = (e & 1) ? two[1] : two[0], stage = (int)(loaded % kRaw);     // (lane 0's count)
            if (lane == 0 && ok) {
              ok = loaded < kRaw || mbar_wait(bar_raw_free(stage), (loaded / kRaw - 1) & 1u, abort_flag);
              if (ok) {
                const int key0 = (it.page + p0 + (e & 1)) * kPage;
                const_cast<int2*>(flags)[stage] = page >= 0 ? make_int2(max(min(lo - key0, kPage), 0), max(min(hi - key0, kPage), 0)) : make_int2(0, 0);
                if (page >= 0) {
                  const uint8_t* from = static_cast<const uint8_t*>(e < 2 ? a.c.k : a.c.v) + ((size_t)page * a.c.n_kv_heads + it.head) * (size_t)L::kRawTile;
                  mbar_arrive_expect_tx(bar_raw_full(stage), (uint32_t)L::kRawTile);
                  bulk_load(base + L::kRawAt + (uint32_t)(stage * L::kRawTile), from, (uint32_t)L::kRawTile, bar_raw_full(stage));
                } else {
                  mbar_arrive(bar_raw_full(stage));
                }
                ++loaded;
              }
            }
          }
          ok = __shfl_sync(0xffffffffu, ok, 0);
        }
      }
      __syncwarp();
      if (lane == 0 && *abort_flag) {
        // let the copies in flight land before the shared memory is given up
        for (uint32_t e = loaded > kRaw ? loaded - kRaw : 0; e < loaded; ++e) {
          const unsigned long long t = global_ns();
          while (!mbar_try_wait(bar_raw_full(e % kRaw), (e / kRaw) & 1u)) { if (global_ns() - t > kWaitLimitNs) break; }
        }
      }
    } else if (warp == kIssuerWarp) {
      // ---- MMAs run in the order they are issued: S_i of the next step may go where P_i is read from by the product ahead of it
      const uint32_t elected = elect_lane();
      const uint32_t idesc_qk = idesc_f16(kStepKeys, 0), idesc_pv = idesc_f16(D, 1);
      auto wait_all = [&](uint32_t bar, uint32_t parity) { return (bool)__all_sync(0xffffffffu, mbar_wait(bar, parity, abort_flag)); };
      uint32_t slot = 0, n_steps[kTiles] = {0, 0}, n_items[kTiles] = {0, 0};     // fp16 tiles; steps and items of either tile so far
      bool ok = true;
      for (long long u = u_begin; u < u_end && ok;) {
        const AttnItem it = item_at<kWide>(a, before, u, u_end);
        if (it.n < 1) break;
        u += it.n;
        const int tiles = it.n_cols > kRows ? 2 : 1, steps = steps_of(it);
        auto issue_qk = [&](int i, uint32_t sl) {
          const uint64_t dq = make_desc(base + L::kQ + (uint32_t)(i * L::kQTile), 16, 1024), dk = make_desc(base + L::kF16 + sl * L::kSlot, 16, 1024);
#pragma unroll
          for (int ks = 0; ks < D / 16; ++ks) {
            const uint32_t off = (uint32_t)((ks >> 2) * (kRows * 128) + (ks & 3) * 32) >> 4;       // (query and keys: 128 rows of 128 bytes a 64-dim block)
            umma_ss(tmem + (uint32_t)i * 128u, dq + off, dk + off, idesc_qk, (uint32_t)(ks != 0), elected);
          }
          umma_commit(bar_s(i), elected);
        };
        // first scores
        ok = wait_all(bar_full(slot % kSlots), (slot / kSlots) & 1u);
        for (int i = 0; i < tiles && ok; ++i) {
          ok = wait_all(bar_q(i), n_items[i] & 1u);
          if (!ok) break;
          ++n_items[i];
          tc_fence_after();
          issue_qk(i, slot % kSlots);
        }
        if (!ok) break;
        umma_commit(bar_free(slot % kSlots), elected);
        ++slot;
        for (int j = 0; j < steps && ok; ++j) {
          const uint32_t sv = slot, sk = slot + 1;
          const uint64_t dv = make_desc(base + L::kF16 + (sv % kSlots) * L::kSlot, kStepKeys * 128, 1024);
          ok = wait_all(bar_full(sv % kSlots), (sv / kSlots) & 1u);
          const bool more = j + 1 < steps;
#pragma unroll
          for (int h = 0; h < 2; ++h)
            for (int i = 0; i < tiles && ok; ++i) {
              ok = wait_all(bar_p(i, h), n_steps[i] & 1u);
              if (!ok) break;
              tc_fence_after();
#pragma unroll
              for (int kk = 0; kk < kPage / 16; ++kk)
                umma_ts(tmem_o + (uint32_t)i * 128u, tmem + (uint32_t)(i * 128 + h * kPage + kk * 8), dv + (uint64_t)((h * kPage * 128 + kk * 2048) >> 4), idesc_pv,
                        (uint32_t)((j | h | kk) != 0), elected);
              if (h == 0) { umma_commit(bar_h(i), elected); continue; }
              if (!more) { umma_commit(bar_o(i), elected); continue; }
              if (i == 0) {
                ok = wait_all(bar_full(sk % kSlots), (sk / kSlots) & 1u);
                if (!ok) break;
                tc_fence_after();
              }
              issue_qk(i, sk % kSlots);
            }
          if (!ok) break;
          for (int i = 0; i < tiles; ++i) ++n_steps[i];
          umma_commit(bar_free(sv % kSlots), elected);
          if (more) umma_commit(bar_free(sk % kSlots), elected);
          slot += more ? 2u : 1u;
        }
      }
      if (!ok) *abort_flag = 1;
    }
  } else if (group == 2) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kConvRegs));
    // ---- codes -> fp16.  A lane takes 16-byte pieces (r + k) mod 8 of row r: eight lanes side by side read eight rows' pieces from
    // different banks, and write them to different ones.
    const int w = warp - kSoftWarps;
    uint32_t raw = 0, slot = 0;
    bool ok = true;
    for (long long u = u_begin; u < u_end && ok;) {
      const AttnItem it = item_at<kWide>(a, before, u, u_end);
      if (it.n < 1) break;
      u += it.n;
      const int steps = steps_of(it);
#pragma unroll 1
      for (int e = 0; e < 2 * steps && ok; ++e) {                          // K, V of a step
        const uint32_t sl = slot % kSlots;
        if (slot >= kSlots) ok = mbar_wait(bar_free(sl), (slot / kSlots - 1) & 1u, abort_flag);
        const uint32_t to = base + L::kF16 + sl * (uint32_t)L::kSlot;
#pragma unroll 1
        for (int h = 0; h < 2 && ok; ++h) {                                // the step's two pages
          const uint32_t st = raw % kRaw;
          ok = mbar_wait(bar_raw_full(st), (raw / kRaw) & 1u, abort_flag);
          if (!ok) break;
          const int2 rows = const_cast<const int2*>(flags)[st];
          const uint32_t from = base + L::kRawAt + st * (uint32_t)L::kRawTile;
          constexpr int CPR = D / 16, PER = kPage * CPR / 128;             // pieces of a row, of a lane
          uint4 v[PER];
          int row[PER], piece[PER];
#pragma unroll
          for (int i = 0; i < PER; ++i) {
            // rows 16 w ... + 15, pieces by (lane / 16, i); 64 dims: four pieces a row, 0, 2, 3, 1 of its pair's number
            const int r = 16 * w + (lane & 15), k = (lane >> 4) + 2 * i;
            row[i] = r;
            piece[i] = D == 128 ? (r + k) & 7 : ((0x78 >> (r & 6)) ^ k) & 3;
            v[i] = lds128(from + (uint32_t)(r * D + piece[i] * 16));
            // what no row of the item sees may be anything, NaN among it, which a weight of 0 does not stop
            if (r < rows.x || r >= rows.y) v[i] = make_uint4(0u, 0u, 0u, 0u);
          }
          __syncwarp();
          if (lane == 0) mbar_arrive(bar_raw_free(st));
#pragma unroll
          for (int i = 0; i < PER; ++i) {
            const int r = h * kPage + row[i], c = 2 * (piece[i] & 3);
            const uint32_t at = to + (uint32_t)((piece[i] >> 2) * (kStepKeys * 128) + r * 128);
            uint32_t x[8];
            codes_to_half2(v[i].x, x[0], x[1]);
            codes_to_half2(v[i].y, x[2], x[3]);
            codes_to_half2(v[i].z, x[4], x[5]);
            codes_to_half2(v[i].w, x[6], x[7]);
            sts128(at + (uint32_t)((c ^ (r & 7)) << 4), x[0], x[1], x[2], x[3]);
            sts128(at + (uint32_t)(((c + 1) ^ (r & 7)) << 4), x[4], x[5], x[6], x[7]);
          }
          ++raw;
        }
        if (!ok) break;
        fence_async_proxy();
        __syncwarp();
        if (lane == 0) mbar_arrive(bar_full(sl));
        ++slot;
      }
    }
  } else {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kSoftRegs));
    // ---- softmax: tile `group`, a thread a row --------------------------------------------------------------------
    const int i = group, row = tid & 127;
    const uint32_t lane_base = (uint32_t)(32 * (warp & 3)) << 16;
    const uint32_t ts = tmem + (uint32_t)i * 128u + lane_base, to = tmem_o + (uint32_t)i * 128u + lane_base;
    const uint32_t q_at = base + L::kQ + (uint32_t)(i * L::kQTile);
    auto q_place = [&](int r, int c) { return q_at + (uint32_t)((c >> 3) * (kRows * 128) + r * 128 + (((c & 7) ^ (r & 7)) << 4)); };
    uint32_t n_s = 0, n_o = 0;
    bool ok = true;
    for (long long u = u_begin; u < u_end && ok;) {
      const AttnItem it = item_at<kWide>(a, before, u, u_end);
      if (it.n < 1) break;
      u += it.n;
      const int col = i * kRows + row;                                     // packed row of the item
      const bool on = col < it.n_cols;
      if (i * kRows >= it.n_cols) continue;                                // (no second tile)
      const int t = by_group(a, it.r0 + (on ? col : 0));
      const RowHead rh = row_head(a, it.s.first, it.r0 + (on ? col : 0), it.head);
      // the query, first as it is: the lanes of a warp side by side along its rows
      {
        constexpr int LPR = D / 8, RPI = 32 / LPR;
        const long long from = (long long)rh.row * a.q_row + (long long)rh.head * a.q_head;
        const unsigned valid = __ballot_sync(0xffffffffu, on);
        const int c = lane % LPR;
#pragma unroll 1
        for (int r = lane / LPR; r < 32; r += RPI) {
          const long long at = __shfl_sync(0xffffffffu, from, r);
          cp_async16(q_place(32 * (warp & 3) + r, c), a.q + at + 8 * c, (valid >> r) & 1u);
        }
        cp_async_commit();
        cp_async_wait<0>();
        __syncwarp();
      }
      // ... then as fp16, a thread a row: times the power of two that brings its largest magnitude to 2^14 .. 2^15
      float factor;
      {
        __nv_bfloat162 most2 = __float2bfloat162_rn(0.f);
#pragma unroll 4
        for (int c = 0; c < D / 8; ++c) {
          const uint4 v = lds128(q_place(row, c));
          __nv_bfloat162 x[4];
#pragma unroll
          for (int w = 0; w < 4; ++w) { const uint32_t two = word(v, w); x[w] = __habs2(*reinterpret_cast<const __nv_bfloat162*>(&two)); }
          most2 = __hmax2(most2, __hmax2(__hmax2(x[0], x[1]), __hmax2(x[2], x[3])));            // (NaN is passed over)
        }
        const float2 m2 = __bfloat1622float2(most2);
        const int e = min(max(exponent_of(fmaxf(m2.x, m2.y)), -100), 127) - 14;
        const float up = power_of_two(-e);
        factor = power_of_two(e) * a.scale_log2e;
#pragma unroll 2
        for (int c = 0; c < D / 8; ++c) {
          const uint4 v = lds128(q_place(row, c));
          uint32_t h[4];
#pragma unroll
          for (int w = 0; w < 4; ++w) {
            const uint32_t two = word(v, w);
            h[w] = half2_of(__uint_as_float(two << 16) * up, __uint_as_float(two & 0xffff0000u) * up);
          }
          sts128(q_place(row, c), h[0], h[1], h[2], h[3]);
        }
      }
      fence_async_proxy();
      __syncwarp();
      if (lane == 0) mbar_arrive(bar_q(i));
      const KeyRange seen = on ? keys_of(a, it.s, t) : KeyRange{0, 0x7fffffff};
      // m_run: the reference of the row's P, O and l, in the log2 domain; ref = lift - m_run (0: no key so far)
      float m_run = -INFINITY, l_run = 0.f, ref = 0.f;
      float ks_mine = 0.f, vs_mine = 1.f;
      int there_mine = 0;
      const int steps = steps_of(it);
#pragma unroll 1
      for (int j = 0; j < steps; ++j) {
        // scales of the next 32 pages, a page a lane; of the step's two
        if ((j & 15) == 0) {
          const int p = 2 * j + lane, page = p < it.n ? page_of(a.r, a.c.n_pages, it.seq, it.page + p) : -1;
          there_mine = page >= 0;
          const size_t at = (size_t)max(page, 0) * a.c.n_kv_heads + it.head;
          ks_mine = a.c.k_scale[at];
          vs_mine = a.c.v_scale[at];
        }
        float f_of[2];
        int ev_of[2], lo_of[2], hi_of[2];
        unsigned edges = 0u;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const int src = (2 * j + h) & 31, key0 = (it.page + 2 * j + h) * kPage;
          f_of[h] = fmaxf(factor * __shfl_sync(0xffffffffu, ks_mine, src), 1.2e-38f);              // (0 would make NaN of a hidden key's -inf)
          ev_of[h] = exponent_of(__shfl_sync(0xffffffffu, vs_mine, src));
          const bool there = __shfl_sync(0xffffffffu, there_mine, src) != 0;
          lo_of[h] = there ? seen.lo - key0 : kPage;
          hi_of[h] = there ? seen.hi - key0 : 0;
          edges |= __any_sync(0xffffffffu, lo_of[h] > 0 || hi_of[h] < kPage) ? 1u << h : 0u;
        }
        ok = mbar_wait(bar_s(i), n_s & 1u, abort_flag) && ok;
        __syncwarp();
        tc_fence_after();
#pragma unroll 1
        for (int h = 0; h < 2; ++h) {
          const uint32_t ts_p = ts + (uint32_t)(h * kPage);
          uint32_t sc[kPage];
          tmem_ld_row32(ts_p, sc);
          tmem_ld_row32(ts_p + 32u, sc + 32);
          const float f = h ? f_of[1] : f_of[0];
          const int ev = h ? ev_of[1] : ev_of[0];
          const float evf = (float)ev;
          float down = power_of_two(-ev);
          tmem_arrived32(sc);
          tmem_arrived32(sc + 32);
          if ((edges >> h) & 1u) {
            const int lo = h ? lo_of[1] : lo_of[0], hi = h ? hi_of[1] : hi_of[0];
#pragma unroll
            for (int c = 0; c < kPage; ++c) if (c < lo || c >= hi) sc[c] = 0xff800000u;
          }
          float mx[4];
#pragma unroll
          for (int c = 0; c < 4; ++c) mx[c] = __uint_as_float(sc[c]);
#pragma unroll
          for (int c = 4; c < kPage - 4; c += 8)
#pragma unroll
            for (int d = 0; d < 4; ++d) mx[d] = max3_nan(mx[d], __uint_as_float(sc[c + d]), __uint_as_float(sc[c + 4 + d]));
          const float top = max3_nan(max3_nan(mx[0], mx[1], mx[2]), max3_nan(mx[3], __uint_as_float(sc[kPage - 4]), __uint_as_float(sc[kPage - 3])),
                                     max3_nan(__uint_as_float(sc[kPage - 2]), __uint_as_float(sc[kPage - 1]), mx[3]));
          const float most = fmaf(top, f, evf);                              // (f > 0: the largest score has the largest x)
          const bool some = most > -INFINITY, moves = some && most > m_run + kLazy, far = some && most < m_run - kFar;
          if (!(most == most)) l_run = most;                                 // a NaN among the scores: the row is NaN
          float shift = evf + ref;
          if (__any_sync(0xffffffffu, moves || far)) {
            float alpha = 1.f;
            if (moves) {
              if (m_run > -INFINITY) { alpha = exp2f(m_run - most); l_run = times_power(l_run, m_run - most); }
              m_run = most;
              ref = kLift - most;
            }
            shift = evf + (far ? -most : ref);
            if (far) down = exp2f(most + ref - evf);
            // rows whose reference moved.  (S of this step told that the step before has been added to O; of its own first page a barrier tells.)
            if ((j | h) != 0 && __any_sync(0xffffffffu, moves)) {
              if (h != 0) {
                ok = mbar_wait(bar_h(i), n_s & 1u, abort_flag) && ok;
                __syncwarp();
                tc_fence_after();
              }
#pragma unroll 1
              for (int c = 0; c < D; c += 16) {
                uint32_t o[16];
                tmem_ld_row16(to + (uint32_t)c, o);
#pragma unroll
                for (int k = 0; k < 16; ++k) o[k] = __float_as_uint(__uint_as_float(o[k]) * alpha);
                tmem_st_row16(to + (uint32_t)c, o);
              }
            }
          }
          const uint64_t f2 = f32x2(f, f), c2 = f32x2(shift, shift);
          uint64_t sum[2] = {0ull, 0ull};
          uint32_t pw[kPage / 2];
#pragma unroll
          for (int c = 0; c < kPage / 2; ++c) {
            const uint64_t y = fma_f32x2(f32x2(__uint_as_float(sc[2 * c]), __uint_as_float(sc[2 * c + 1])), f2, c2);
            const float2 p = (c & 7) >= kByUnit ? power_by_polynomial(y) : power_by_unit(y);
            sum[c & 1] = add_f32x2(sum[c & 1], f32x2(p.x, p.y));
            pw[c] = half2_of(p.x, p.y);
          }
          if (__any_sync(0xffffffffu, far)) {
#pragma unroll
            for (int c = 0; c < kPage / 2; ++c) pw[c] = far ? 0u : pw[c];
          }
          tmem_st_row32(ts_p, pw);
          const float2 s2 = f32x2_parts(add_f32x2(sum[0], sum[1]));
          if (some) l_run = fmaf(s2.x + s2.y, down, l_run);
          tmem_st_wait();
          tc_fence_before();
          __syncwarp();
          if (lane == 0) mbar_arrive(bar_p(i, h));
        }
        ++n_s;
      }
      // ---- rows out -----------------------------------------------------------------------------------------------
      ok = mbar_wait(bar_o(i), n_o & 1u, abort_flag) && ok;
      ++n_o;
      __syncwarp();
      tc_fence_after();
      if (!ok) { *abort_flag = 1; break; }
      const bool begun = it.page > it.first, goes_on = it.page + it.n < it.first + it.of, whole = !begun && !goes_on;
      if (l_run != l_run) m_run = INFINITY;                                // (goes on in other parts as infinity - infinity)
      if (on) {
        if (whole) store_lse(a, rh, m_run - kLift, l_run);
        else part_stats<kWide, D>(a.parts, cta, begun ? 0 : 1)[col] = make_float2(m_run - kLift, l_run);
      }
      // a quad of lanes to two rows: where they go, as fp32 (parts always) or bf16
      const float mul = whole ? (l_run == 0.f ? 0.f : 1.f / l_run) : 1.f;
      const bool fp32 = !whole || a.out_fp32;
      char* const to_base = whole ? static_cast<char*>(a.out) : reinterpret_cast<char*>(part_rows<kWide, D>(a.parts, cta, begun ? 0 : 1));
      const long long to_row = (whole ? (long long)rh.row * a.out_row + (long long)rh.head * a.out_head : (long long)col * D) * (fp32 ? 4 : 2);
#pragma unroll 1
      for (int b = 0; b < 4; ++b) {                                        // rows 16 (b / 2) + 8 half, 64 dims
        const int c = (b & 1) * 64, r0 = 16 * (b >> 1) + (lane >> 2);
        if (c >= D) continue;
        float v[32];
        __syncwarp();
        tmem_ld_16x64(to + ((uint32_t)(16 * (b >> 1)) << 16) + (uint32_t)c, v);
        tmem_ld_wait();
#pragma unroll
        for (int half = 0; half < 2; ++half) {
          const float f = __shfl_sync(0xffffffffu, mul, r0 + 8 * half);
          char* dst = to_base + __shfl_sync(0xffffffffu, to_row, r0 + 8 * half) + (c + 2 * (lane & 3)) * (fp32 ? 4 : 2);
          if (i * kRows + 32 * (warp & 3) + r0 + 8 * half >= it.n_cols) continue;
          if (fp32) {
#pragma unroll
            for (int k = 0; k < 8; ++k) *reinterpret_cast<float2*>(dst + 32 * k) = make_float2(v[4 * k + 2 * half] * f, v[4 * k + 2 * half + 1] * f);
          } else {
#pragma unroll
            for (int k = 0; k < 8; ++k) *reinterpret_cast<uint32_t*>(dst + 16 * k) = pack2(v[4 * k + 2 * half] * f, v[4 * k + 2 * half + 1] * f);
          }
        }
      }
      tc_fence_before();
      if (begun && !goes_on && tid == 0) a.joins[cta] = make_int4(1 + runs.cta_of(u - it.of), it.s.first, it.r0, it.head | (it.n_cols << 16));
    }
    if (!ok) *abort_flag = 1;
  }
  pdl_wait();                          // (so that this launch has completed only once the one ahead of it has)
  __syncthreads();
  if (warp == kLoaderWarp) {
    tc_fence_after();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512u) : "memory");
  }
  if (tid == 0 && *abort_flag) atomicExch(a.status, VS_ERR_DEVICE_TIMEOUT);
}

template <int D>
int launch_tc(const CacheAttnArgs& a, bool behind_few, cudaStream_t st) {
  const int bytes = Tc<D>::bytes(a.r.n_seqs);
  static_assert(Tc<D>::kBefore + 8 * (VS_CACHE_MAX_SEQS + 1) <= 227 * 1024, "shared memory of an SM");
  if (cudaFuncSetAttribute(cache_attention_tc_kernel<D>, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes) != cudaSuccess) return VS_ERR_CUDA;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(kManyCtas);
  cfg.blockDim = dim3(kThreads);
  cfg.dynamicSmemBytes = (size_t)bytes;
  cfg.stream = st;
  cudaLaunchAttribute at = {};
  at.id = cudaLaunchAttributeProgrammaticStreamSerialization;      // (other rows, other parts of the workspace: nothing to wait for but its end)
  at.val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = &at;
  cfg.numAttrs = behind_few ? 1 : 0;
  return cudaLaunchKernelEx(&cfg, cache_attention_tc_kernel<D>, a) == cudaSuccess ? launched() : VS_ERR_CUDA;
}

}  // namespace

int launch_cache_attention_many(const CacheAttnArgs& a, bool behind_few, cudaStream_t st) {
  return a.c.head_dim == 128 ? launch_tc<128>(a, behind_few, st) : launch_tc<64>(a, behind_few, st);
}

}  // namespace vs
