// Attention over the paged 8-bit cache for sequences of many rows (a question, a frame, several frames), on the 5th-generation
// tensor cores.  Mathematics and the cut of the work as in vs_cache_attention.cu: O += 2^{x - m + lift} code_v, l += that * 2^{-ev}, o = O / l.
//
// A CTA (one an SM) takes runs of (item, page) units one after the other; an item is 256 packed rows (row t, head g of the group: t G + g) of one KV
// head: two tiles of 128, the MMA's M.  Page by page, 64 keys:
//   loader     codes by bulk copies (8 KB at 128 dims: a page and head lies side by side) into a ring of raw tiles, in the order of their use
//   converters (8 warps) codes -> fp16, exactly, into the operands' 128-byte-swizzled layout, a ring of page tiles of keys and values
//   issuers    (a warp a row tile) S_i = Q_i K^T (M 128, N 64) two pages ahead, O_i += P_i V (A = P_i from tensor memory)
//   softmax    (4 warps a row tile, a thread a row) S from tensor memory, P (fp16) back over it; a row of O is rescaled there only when its
//              maximum has grown by more than 2^8
// Tensor memory: two buffers of S (P over the first half of each) and O of either row tile: all 512 columns.  With two buffers a row tile's
// softmax runs while its next scores are worked out.  (One buffer of 128 keys, N 128: a quarter less of the tensor pipe, but softmax, P V and the next
// Q K^T of a row tile one after the other.)
//
// The codes go to fp16 once a page and CTA and serve 256 rows: fewer rows would convert more than they multiply, and fp8 operands would need the weights in
// 8 bits, whose range of 2^18 loses a long row's many small ones beside one large one.  The query is held as fp16, exactly (see there).
// Measured: 16600 pages and heads of four sequences' frames, 256 rows each: 183 us, 710 TFLOP/s; 13440 causal rows of one sequence 2.32 ms, 559; a page takes some 2000 clocks of a
// CTA, of which the tensor pipe is busy 40 %, the exponentials' unit 41 %, the schedulers 49 %: a row's page is a chain -- scores out of tensor memory 250, maximum and votes 170, exponentials 1000,
// back 40, barriers 450 -- of which a scheduler has two at a time, all that tensor memory has room for.  (Two threads a row 205 us, too many registers;
// a part of the exponentials by a polynomial 183 against 182; a scheduler's two warps taking turns at the exponentials 194 against 185.)
// All waits are bounded.
#include "vs_cache_attention.cuh"
#include "vs_ptx.cuh"

namespace vs {

namespace {

constexpr int kRows = 128, kTiles = 2, kWide = kRows * kTiles;
constexpr int kTileWarps = 4, kSoftWarps = kTileWarps * kTiles, kConvWarps = 4, kLoaderWarp = kSoftWarps + 2 * kConvWarps, kIssuerWarp = kLoaderWarp + 1;
constexpr int kThreads = 32 * 20;                       // (warpgroups: softmax of either tile, converters of every second page tile, loader + issuer)
constexpr int kSoftRegs = 144, kConvRegs = 64, kRestRegs = 64;
static_assert(2 * kSoftRegs + 2 * kConvRegs + kRestRegs <= 5 * 96, "the registers the block is launched with: 96 a thread");
constexpr float kLift = 7.f, kLazy = 8.f;              // weights reach 2^(lift + lazy) <= 2^15
// Places of either ring, raw codes and fp16.  (Even: every second tile has converters of its own, who may be some tiles ahead of the others; in a place
// that both used in turn they would take a phase that the others have yet to see for one that is past.)
constexpr int kRing = 6;
static_assert(kRing % 2 == 0, "a place in a ring belongs to one half of the converters");

template <int D>
struct Tc {
  static constexpr int kQTile = kRows * D * 2, kTile = kPage * D * 2, kRawTile = kPage * D;
  static constexpr int kQ = 0, kF16 = kTiles * kQTile, kRawAt = kF16 + kRing * kTile, kCtl = kRawAt + kRing * kRawTile;
  static constexpr int kBars = 4 * kRing + 7 * kTiles;
  static constexpr int kFlags = kCtl + 8 * kBars;       // [place] first and end of the rows of the raw tile that count (end 0: the page is not there); 256 in the first: values that not all rows of the item see alike
  static constexpr int kSlotWord = kFlags + 8 * kRing;
  static constexpr int kNanWord = kSlotWord + 8;        // whether a value that only some rows of an item see was NaN
  static constexpr int kPlaces = (kNanWord + 4 + 15) / 16 * 16;               // [warp] where its last item lies
  static constexpr int kBefore = kPlaces + 16 * (kThreads / 32);
  static constexpr int bytes(int n_seqs) { return kBefore + 8 * (n_seqs + 1 + kCutWords); }
};

// The page tiles of an item of n pages in the order of their use: K(0), K(1), V(0), K(2), V(1), ... K(n - 1), V(n - 2), V(n - 1)
__device__ __forceinline__ int tile_of_k(int p) { return p == 0 ? 0 : 2 * p - 1; }
__device__ __forceinline__ int tile_of_v(int p, int n) { return p == n - 1 ? 2 * n - 1 : 2 * p + 2; }
__device__ __forceinline__ bool tile_is_v(int e, int n) { return e == 2 * n - 1 || (e > 0 && (e & 1) == 0); }
__device__ __forceinline__ int page_of_tile(int e, int n) { return tile_is_v(e, n) ? (e == 2 * n - 1 ? n - 1 : e / 2 - 1) : (e + 1) / 2; }

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

// Keys [lo, hi) that any row of an item sees; of the pages that begin ahead of `ahead` or behind `behind` some rows see other keys than others.  (Both ends go
// up with the row.)
constexpr int kUneven = 256;
struct ItemKeys {
  int lo, hi, ahead, behind;
  __device__ __forceinline__ bool uneven(int key0) const { return key0 < ahead || key0 > behind; }
};
__device__ __forceinline__ ItemKeys keys_of_item(const CacheAttnArgs& a, const AttnItem& it) {
  const KeyRange first = keys_of(a, it.s, by_group(a, it.r0)), last = keys_of(a, it.s, by_group(a, it.r0 + it.n_cols - 1));
  return {first.lo, last.hi, first.lo < last.lo ? last.lo : 0, first.hi < last.hi ? first.hi - kPage : 0x7fffffff};
}

// The NaN of values that some rows of an item see and others do not.  The converters put zeros in their place; here, once the last product is
// complete, every thread sets to NaN the dims of its row of O whose NaN the row sees.  It reads the pages in question once more.
template <int D>
__device__ __forceinline__ void set_seen_nan(const CacheAttnArgs& a, const AttnItem& it, int col, uint32_t to) {
  const ItemKeys keys = keys_of_item(a, it);
  const KeyRange seen = col < it.n_cols ? keys_of(a, it.s, by_group(a, it.r0 + col)) : KeyRange{0, 0};
  uint32_t dims[D / 32];
#pragma unroll
  for (int w = 0; w < D / 32; ++w) dims[w] = 0u;
  for (int p = it.page; p < it.page + it.n; ++p) {
    const int key0 = p * kPage;
    if (!keys.uneven(key0)) continue;
    const int page = page_of(a.r, a.c.n_pages, it.seq, p);
    if (page < 0) continue;
    const uint8_t* const from = static_cast<const uint8_t*>(a.c.v) + ((size_t)page * a.c.n_kv_heads + it.head) * (size_t)(kPage * D);
    for (int k = max(seen.lo - key0, 0); k < min(seen.hi - key0, kPage); ++k)
#pragma unroll
      for (int w = 0; w < D / 32; ++w)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const uint4 v = *reinterpret_cast<const uint4*>(from + k * D + 32 * w + 16 * h);
#pragma unroll
          for (int c = 0; c < 4; ++c) {
            const uint32_t n = nan_codes(word(v, c));
            dims[w] |= ((n | n >> 7 | n >> 14 | n >> 21) & 15u) << (16 * h + 4 * c);
          }
        }
  }
#pragma unroll 1
  for (int c = 0; c < D; c += 16) {
    uint32_t o[16], set = 0u;
#pragma unroll
    for (int w = 0; w < D / 32; ++w) if (c / 32 == w) set = dims[w] >> (c & 31);
    __syncwarp();
    tmem_ld_row16(to + (uint32_t)c, o);
#pragma unroll
    for (int k = 0; k < 16; ++k) if (set >> k & 1u) o[k] = 0x7fc00000u;
    tmem_st_row16(to + (uint32_t)c, o);
  }
  tmem_st_wait();
}

template <int D>
__global__ void __launch_bounds__(kThreads, 1) cache_attention_tc_kernel(const __grid_constant__ CacheAttnArgs a) {
  using L = Tc<D>;
  extern __shared__ __align__(1024) uint8_t smem[];
  const uint32_t base = smem_u32(smem), ctl = base + L::kCtl;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  auto bar_raw_full = [&](uint32_t x) { return ctl + 8u * x; };                                    // a raw tile's bytes are here
  auto bar_raw_free = [&](uint32_t x) { return ctl + 8u * (kRing + x); };                          // ... converted (an arrival a converter warp)
  auto bar_full = [&](uint32_t x) { return ctl + 8u * (2 * kRing + x); };                          // an fp16 tile is there (an arrival a converter warp)
  auto bar_free = [&](uint32_t x) { return ctl + 8u * (3 * kRing + x); };                          // ... and multiplied (tcgen05.commit, by either issuer)
  constexpr uint32_t kTileBars = 4 * kRing;
  auto bar_q = [&](int i) { return ctl + 8u * (kTileBars + (uint32_t)i); };                         // the tile's query is in place (an arrival a warp)
  auto bar_p = [&](int i, uint32_t b) { return ctl + 8u * (kTileBars + kTiles + 2u * (uint32_t)i + b); };          // P_i of buffer b is there, O_i rescaled (an arrival a warp)
  auto bar_s = [&](int i, uint32_t b) { return ctl + 8u * (kTileBars + 3 * kTiles + 2u * (uint32_t)i + b); };      // S_i of buffer b is there (tcgen05.commit)
  // The page of buffer b has been added to O_i (tcgen05.commit).  (One for either buffer: a wait tells a phase only from the one before it, and what is
  // known when a page's scores are there is that the page two before it has been added.)
  auto bar_o = [&](int i, uint32_t b) { return ctl + 8u * (kTileBars + 5 * kTiles + 2u * (uint32_t)i + b); };
  volatile int2* flags = reinterpret_cast<volatile int2*>(smem + L::kFlags);
  volatile uint32_t* tmem_slot = reinterpret_cast<volatile uint32_t*>(smem + L::kSlotWord);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(smem + L::kSlotWord + 4);
  volatile int* nan_flag = reinterpret_cast<volatile int*>(smem + L::kNanWord);
  long long* before = reinterpret_cast<long long*>(smem + L::kBefore);
  ItemPlace* const place_of = reinterpret_cast<ItemPlace*>(smem + L::kPlaces) + warp;

  if (lane == 0) *place_of = {0, -1, 0};
  if (warp == kIssuerWarp) {
    for (uint32_t x = (uint32_t)lane; x < (uint32_t)L::kBars; x += 32u)
      mbar_init(ctl + 8u * x, (x >= kRing && x < 3 * kRing) || (x >= kTileBars && x < kTileBars + 3 * kTiles) ? 4u : (x >= 3 * kRing && x < 4 * kRing ? 2u : 1u));       // (converters, softmax: four warps; issuers: two)
    if (lane == 0) *nan_flag = 0;
    if (lane == 0) *abort_flag = (base & 1023u) != 0;     // (the swizzled layouts need the alignment that the declaration asks for)
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    fence_async_proxy();
  } else if (warp == kLoaderWarp) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32((const void*)tmem_slot)), "r"(512u) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  tc_fence_before();
  const AttnRuns runs = cut_units<kWide>(a, before, (int)gridDim.x);         // (ends with a barrier of the block)
  tc_fence_after();
  const uint32_t tmem = *tmem_slot, tmem_o = tmem + kTiles * 128u;
  const int cta = (int)blockIdx.x;
  if (tid == 0) a.joins[cta] = make_int4(0, 0, 0, 0);
  const bool works = cta < runs.n_ctas && runs.units > 0;
  const long long u_begin = works ? runs.begin(cta) : 0, u_end = works ? runs.begin(cta + 1) : 0;

  if (warp >= kLoaderWarp) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kRestRegs));
    if (warp == kLoaderWarp) {
      // ---- pages' codes, four tiles at a time, a lane each (what a lane does one after the other takes 500 clocks a tile) ------------------
      uint32_t done = 0;                                                   // tiles of the items so far
      bool ok = true;
      for (long long u = u_begin; u < u_end && ok;) {
        const AttnItem it = item_at<kWide>(a, before, runs, u, u_end, place_of);
        if (it.n < 1) break;
        u += it.span;
        const ItemKeys seen = keys_of_item(a, it);
        uint32_t place = (done + (uint32_t)lane) % kRing, phase = ((done + (uint32_t)lane) / kRing + 1u) & 1u;      // (phase: of bar_raw_free, before this use)
        int p = page_of_tile(lane, it.n), page = lane < 4 && lane < 2 * it.n ? page_of(a.r, a.c.n_pages, it.seq, it.page + p) : -1;
        for (int e0 = 0; e0 < 2 * it.n && ok; e0 += 4) {
          const int e = e0 + lane;
          if (lane < 4 && e < 2 * it.n) {
            const bool is_v = tile_is_v(e, it.n);
            const int key0 = (it.page + p) * kPage;
            const uint8_t* const from = static_cast<const uint8_t*>(is_v ? a.c.v : a.c.k) + ((size_t)max(page, 0) * a.c.n_kv_heads + it.head) * (size_t)L::kRawTile;
            ok = mbar_wait(bar_raw_free(place), phase, abort_flag);
            if (ok) {
              const_cast<int2*>(flags)[place] = page >= 0 ? make_int2(max(min(seen.lo - key0, kPage), 0) + (is_v && seen.uneven(key0) ? kUneven : 0), max(min(seen.hi - key0, kPage), 0)) : make_int2(0, 0);
              if (page >= 0) {
                mbar_arrive_expect_tx(bar_raw_full(place), (uint32_t)L::kRawTile);
                bulk_load(base + L::kRawAt + place * (uint32_t)L::kRawTile, from, (uint32_t)L::kRawTile, bar_raw_full(place));
              } else {
                mbar_arrive(bar_raw_full(place));
              }
            }
            p = page_of_tile(e + 4, it.n);
            page = e + 4 < 2 * it.n ? page_of(a.r, a.c.n_pages, it.seq, it.page + p) : -1;
          }
          ok = __all_sync(0xffffffffu, ok);
          place += 4u;
          if (place >= kRing) { place -= kRing; phase ^= 1u; }
        }
        done += 2u * (uint32_t)it.n;
      }
      __syncwarp();
      if (*abort_flag) {
        // Let the copies in flight land before the shared memory is given up: a place's last phase, complete or not.  (One that nothing was asked for
        // any more is seen as complete or waited for until the limit.)
        if (lane < kRing) {
          const unsigned long long t = global_ns();
          for (uint32_t parity = 0; parity < 2; ++parity)
            while (!mbar_try_wait(bar_raw_full((uint32_t)lane), parity)) { if (global_ns() - t > kWaitLimitNs) break; }
        }
        __syncwarp();
      }
    } else if (warp < kIssuerWarp + kTiles) {
      // ---- products of row tile i
      const int i = warp - kIssuerWarp;
      const uint32_t elected = elect_lane();
      const uint32_t idesc_qk = idesc_f16(kPage, 0), idesc_pv = idesc_f16(D, 1);
      auto wait_all = [&](uint32_t bar, uint32_t parity) { return (bool)__all_sync(0xffffffffu, mbar_wait(bar, parity, abort_flag)); };
      uint32_t done = 0, g = 0, n_items = 0;                               // page tiles of the items so far; pages and items of the row tile
      bool ok = true;
      for (long long u = u_begin; u < u_end && ok;) {
        const AttnItem it = item_at<kWide>(a, before, runs, u, u_end, place_of);
        if (it.n < 1) break;
        u += it.span;
        const bool mine = it.n_cols > i * kRows;                           // (else the page tiles are only let go)
        auto wait_tile = [&](int e) { const uint32_t x = done + (uint32_t)e; return wait_all(bar_full(x % kRing), (x / kRing) & 1u); };
        auto tile_at = [&](int e) { return base + L::kF16 + ((done + (uint32_t)e) % kRing) * (uint32_t)L::kTile; };
        auto let_go = [&](int e) { umma_commit(bar_free((done + (uint32_t)e) % kRing), elected); };
        auto issue_qk = [&](int p) {                                       // S of page p, in the buffer of its number
          const uint32_t b = (g + (uint32_t)p) & 1u;
          const uint64_t dq = make_desc(base + L::kQ + (uint32_t)(i * L::kQTile), 16, 1024), dk = make_desc(tile_at(tile_of_k(p)), 16, 1024);
          tc_fence_after();
#pragma unroll
          for (int ks = 0; ks < D / 16; ++ks)
            umma_ss(tmem + (uint32_t)i * 128u + b * 64u, dq + ((uint32_t)((ks >> 2) * (kRows * 128) + (ks & 3) * 32) >> 4),
                    dk + ((uint32_t)((ks >> 2) * (kPage * 128) + (ks & 3) * 32) >> 4), idesc_qk, (uint32_t)(ks != 0), elected);
          umma_commit(bar_s(i, b), elected);
        };
        // the first two pages' scores
        if (mine) ok = wait_all(bar_q(i), n_items & 1u);
#pragma unroll 1
        for (int p = 0; p < min(2, it.n) && ok; ++p) {
          ok = wait_tile(tile_of_k(p));
          if (!ok) break;
          if (mine) issue_qk(p);
          let_go(tile_of_k(p));
        }
#pragma unroll 1
        for (int p = 0; p < it.n && ok; ++p) {
          const int ev = tile_of_v(p, it.n), ek = tile_of_k(p + 2);
          const uint32_t x = g + (uint32_t)p, b = x & 1u;
          ok = wait_tile(ev);
          if (ok && mine) ok = wait_all(bar_p(i, b), (x >> 1) & 1u);
          if (!ok) break;
          if (mine) {
            const uint64_t dv = make_desc(tile_at(ev), kPage * 128, 1024);
            tc_fence_after();
#pragma unroll
            for (int kk = 0; kk < kPage / 16; ++kk)                          // (P of a page lies over the first half of its scores)
              umma_ts(tmem_o + (uint32_t)i * 128u, tmem + (uint32_t)(i * 128) + b * 64u + (uint32_t)(kk * 8), dv + (uint64_t)((kk * 2048) >> 4), idesc_pv,
                      (uint32_t)((p | kk) != 0), elected);
            umma_commit(bar_o(i, b), elected);
          }
          let_go(ev);
          if (p + 2 >= it.n) continue;
          // the scores of the page after next go where P of this one was read from: once that product is complete (products into different places of
          // tensor memory are not ordered by their issue alone)
          ok = wait_tile(ek);
          if (ok && mine) ok = wait_all(bar_o(i, b), (x >> 1) & 1u);
          if (!ok) break;
          if (mine) issue_qk(p + 2);
          let_go(ek);
        }
        if (mine) { g += (uint32_t)it.n; ++n_items; }
        done += 2u * (uint32_t)it.n;
      }
      if (!ok) *abort_flag = 1;
    }
  } else if (warp >= kSoftWarps) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kConvRegs));
    // ---- codes -> fp16, every second page tile by one half of the warps, the others by the other.  A lane takes 16-byte pieces (r + k) mod 8 of
    // row r: eight lanes side by side read eight rows' pieces from different banks, and write them to different ones.
    const uint32_t half = warp >= kSoftWarps + kConvWarps ? 1u : 0u;
    const int w = (warp - kSoftWarps) % kConvWarps;
    constexpr int CPR = D / 16, PER = kPage * CPR / 128;                   // pieces of a row, of a lane
    const int r = 16 * w + (lane & 15);                                    // its row of the page; pieces by (lane / 16, p)
    // (64 dims: four pieces a row, 0, 2, 3, 1 of its pair's number)
    auto piece_of = [&](int p) { const int k = (lane >> 4) + 2 * p; return D == 128 ? (r + k) & 7 : ((0x78 >> (r & 6)) ^ k) & 3; };
    uint32_t end = 0, x = half;                                            // page tiles to the end of the item; the tile at hand
    bool ok = true;
    for (long long u = u_begin; u < u_end && ok;) {
      const AttnItem it = item_at<kWide>(a, before, runs, u, u_end, place_of);
      if (it.n < 1) break;
      u += it.span;
      end += 2u * (uint32_t)it.n;
#pragma unroll 1
      for (; x < end; x += 2u) {
        const uint32_t place = x % kRing, phase = (x / kRing) & 1u, from = base + L::kRawAt + place * (uint32_t)L::kRawTile + (uint32_t)(r * D);
        ok = ok && mbar_wait(bar_raw_full(place), phase, abort_flag);
        int2 rows = const_cast<const int2*>(flags)[place];
        const bool uneven = rows.x >= kUneven;
        rows.x &= kUneven - 1;
        uint4 v[PER];
#pragma unroll
        for (int p = 0; p < PER; ++p) v[p] = lds128(from + (uint32_t)(piece_of(p) * 16));
        // what no row of the item sees may be anything, NaN among it, which a weight of 0 does not stop
        if (r < rows.x || r >= rows.y)
#pragma unroll
          for (int p = 0; p < PER; ++p) v[p] = make_uint4(0u, 0u, 0u, 0u);
        if (uneven) {                                                       // (the rows that see a NaN have it from set_seen_nan)
          uint32_t nan = 0u;
#pragma unroll
          for (int p = 0; p < PER; ++p) {
            uint32_t* const x = &v[p].x;
#pragma unroll
            for (int c = 0; c < 4; ++c) { const uint32_t n = nan_codes(x[c]); nan |= n; x[c] &= ~(n * 0xffu); }
          }
          if (nan != 0u) *nan_flag = 1;
        }
        __syncwarp();
        if (lane == 0) mbar_arrive(bar_raw_free(place));
        ok = ok && mbar_wait(bar_free(place), phase ^ 1u, abort_flag);
        ok = __all_sync(0xffffffffu, ok);
        if (!ok) break;
        const uint32_t to = base + L::kF16 + place * (uint32_t)L::kTile + (uint32_t)(r * 128);
#pragma unroll
        for (int p = 0; p < PER; ++p) {
          const int piece = piece_of(p), c = 2 * (piece & 3);
          const uint32_t at = to + (uint32_t)((piece >> 2) * (kPage * 128));
          uint32_t y[8];
          codes_to_half2(v[p].x, y[0], y[1]);
          codes_to_half2(v[p].y, y[2], y[3]);
          codes_to_half2(v[p].z, y[4], y[5]);
          codes_to_half2(v[p].w, y[6], y[7]);
          sts128(at + (uint32_t)((c ^ (r & 7)) << 4), y[0], y[1], y[2], y[3]);
          sts128(at + (uint32_t)(((c + 1) ^ (r & 7)) << 4), y[4], y[5], y[6], y[7]);
        }
        fence_async_proxy();
        __syncwarp();
        if (lane == 0) mbar_arrive(bar_full(place));
      }
    }
  } else {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kSoftRegs));
    // ---- softmax: tile i, a thread a row ----------------------------------------------------------------------------
    const int i = warp / kTileWarps, quarter = warp & 3, row = 32 * quarter + lane;
    const uint32_t lane_base = (uint32_t)(32 * quarter) << 16;
    const uint32_t ts = tmem + (uint32_t)(i * 128) + lane_base, to = tmem_o + (uint32_t)i * 128u + lane_base;
    const uint32_t q_at = base + L::kQ + (uint32_t)(i * L::kQTile);
    auto q_place = [&](int r, int c) { return q_at + (uint32_t)((c >> 3) * (kRows * 128) + r * 128 + (((c & 7) ^ (r & 7)) << 4)); };
    uint32_t g = 0;                                                        // pages so far
    bool ok = true;
    for (long long u = u_begin; u < u_end && ok;) {
      const AttnItem it = item_at<kWide>(a, before, runs, u, u_end, place_of);
      if (it.n < 1) break;
      u += it.span;
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
          cp_async16(q_place(32 * quarter + r, c), a.q + at + 8 * c, (valid >> r) & 1u);
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
          uint32_t x[4];
#pragma unroll
          for (int w = 0; w < 4; ++w) {
            const uint32_t two = word(v, w);
            x[w] = half2_of(__uint_as_float(two << 16) * up, __uint_as_float(two & 0xffff0000u) * up);
          }
          sts128(q_place(row, c), x[0], x[1], x[2], x[3]);
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
#pragma unroll 1
      for (int p = 0; p < it.n; ++p, ++g) {
        // scales of the next 32 pages, a page a lane
        if ((p & 31) == 0) {
          const int page = p + lane < it.n ? page_of(a.r, a.c.n_pages, it.seq, it.page + p + lane) : -1;
          there_mine = page >= 0;
          const size_t at = (size_t)max(page, 0) * a.c.n_kv_heads + it.head;
          ks_mine = a.c.k_scale[at];
          vs_mine = a.c.v_scale[at];
        }
        const int key0 = (it.page + p) * kPage;
        const float f = fmaxf(factor * __shfl_sync(0xffffffffu, ks_mine, p & 31), 1.2e-38f);      // (0 would make NaN of a hidden key's -inf)
        const int ev = value_exponent(__shfl_sync(0xffffffffu, vs_mine, p & 31));
        const bool there = __shfl_sync(0xffffffffu, there_mine, p & 31) != 0;
        const bool edge = __any_sync(0xffffffffu, !there || seen.lo > key0 || seen.hi < key0 + kPage);
        const float evf = (float)ev;
        const uint32_t tp = ts + (g & 1u) * 64u;
        ok = ok && mbar_wait(bar_s(i, g & 1u), (g >> 1) & 1u, abort_flag);
        __syncwarp();
        tc_fence_after();
        if (edge) {                                                         // what a row does not see: -inf, back in tensor memory
          const int lo = there ? seen.lo - key0 : kPage, hi = there ? seen.hi - key0 : 0;
#pragma unroll 1
          for (int c0 = 0; c0 < kPage; c0 += 16) {
            uint32_t x[16];
            tmem_ld_row16(tp + (uint32_t)c0, x);
#pragma unroll
            for (int c = 0; c < 16; ++c) if (c0 + c < lo || c0 + c >= hi) x[c] = 0xff800000u;
            tmem_st_row16(tp + (uint32_t)c0, x);
          }
          tmem_st_wait();
        }
        uint32_t x[kPage];
        tmem_ld_row32(tp, x);
        tmem_ld_row32(tp + 32u, x + 32);
        tmem_arrived32(x);
        tmem_arrived32(x + 32);
        float mx[4];
#pragma unroll
        for (int c = 0; c < 4; ++c) mx[c] = __uint_as_float(x[c]);
#pragma unroll
        for (int c = 4; c < kPage - 4; c += 8)
#pragma unroll
          for (int d = 0; d < 4; ++d) mx[d] = max3_nan(mx[d], __uint_as_float(x[c + d]), __uint_as_float(x[c + 4 + d]));
        const float top = max3_nan(max3_nan(mx[0], mx[1], mx[2]), max3_nan(mx[3], __uint_as_float(x[kPage - 4]), __uint_as_float(x[kPage - 3])),
                                   max3_nan(__uint_as_float(x[kPage - 2]), __uint_as_float(x[kPage - 1]), mx[3]));
        const float most = fmaf(top, f, evf);                               // (f > 0: the largest score has the largest x)
        const bool some = most > -INFINITY, moves = most > m_run + kLazy, far = some && most < m_run - kFar;
        if (!(most == most)) l_run = most;                                   // a NaN among the scores: the row is NaN
        float down = power_of_two(-ev), shift = evf + ref;
        const bool rare = __any_sync(0xffffffffu, moves || far);
        if (rare) {
          float alpha = 1.f;
          if (moves) {
            if (m_run > -INFINITY) { alpha = exp2f(m_run - most); l_run = moved_sum(l_run, m_run - most); }
            m_run = most;
            ref = kLift - most;
          }
          shift = evf + (far ? -most : ref);
          if (far) down = exp2f(most + ref - evf);
          // rows whose reference moved, once the page before has been added to O
          if (p != 0 && __any_sync(0xffffffffu, moves)) {
            ok = ok && mbar_wait(bar_o(i, (g - 1u) & 1u), ((g - 1u) >> 1) & 1u, abort_flag);
            __syncwarp();
            tc_fence_after();
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
        if (evf < -kSumTop && some && most - evf - m_run > kSumTop) l_run = shift_sum(l_run);
        const uint64_t f2 = f32x2(f, f), c2 = f32x2(shift, shift);
        uint64_t sum[2] = {0ull, 0ull};
#pragma unroll
        for (int q = 0; q < 2; ++q) {
          uint32_t pw[kPage / 4];
#pragma unroll
          for (int c = 0; c < kPage / 4; ++c) {
            const int k = 2 * (q * (kPage / 4) + c);
            const float2 y = f32x2_parts(fma_f32x2(f32x2(__uint_as_float(x[k]), __uint_as_float(x[k + 1])), f2, c2));
            const float w0 = ex2_approx(y.x), w1 = ex2_approx(y.y);
            sum[c & 1] = add_f32x2(sum[c & 1], f32x2(w0, w1));
            pw[c] = half2_of(w0, w1);
          }
          if (rare) {
#pragma unroll
            for (int c = 0; c < kPage / 4; ++c) pw[c] = far ? 0u : pw[c];
          }
          tmem_st_row16(tp + 16u * (uint32_t)q, pw);
        }
        const float2 s2 = f32x2_parts(add_f32x2(sum[0], sum[1]));
        if (some) l_run = fmaf(s2.x + s2.y, sum_factor(l_run, down), l_run);
        tmem_st_wait();
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(bar_p(i, g & 1u));
      }
      // ---- rows out -----------------------------------------------------------------------------------------------
      ok = ok && mbar_wait(bar_o(i, (g - 1u) & 1u), ((g - 1u) >> 1) & 1u, abort_flag);         // (the last product: those before it are complete as well)
      ok = __all_sync(0xffffffffu, ok);
      tc_fence_after();
      if (!ok) { *abort_flag = 1; break; }
      // (the item looked for once more: what it takes need not stay in registers for the rest of the time)
      if (__any_sync(0xffffffffu, *nan_flag != 0)) set_seen_nan<D>(a, item_at<kWide>(a, before, runs, u - it.span, u_end, place_of), col, to);
      const bool begun = it.page > it.first, goes_on = it.page + it.n < it.first + it.of, whole = !begun && !goes_on;
      if (l_run != l_run) m_run = INFINITY;                                // (goes on in other parts as infinity - infinity)
      if (on) {
        if (whole) store_lse(a, rh, m_run - kLift, l_run);
        else part_stats<kWide, D>(a.parts, cta, begun ? 0 : 1)[col] = make_float2(m_run - kLift, l_run);
      }
      // a quad of lanes to two rows: where they go, as fp32 (parts always) or bf16
      const float2 mul = whole ? reciprocal(l_run) : make_float2(1.f, 1.f);
      const bool fp32 = !whole || a.out_fp32;
      char* const to_base = whole ? static_cast<char*>(a.out) : reinterpret_cast<char*>(part_rows<kWide, D>(a.parts, cta, begun ? 0 : 1));
      const long long to_row = (whole ? (long long)rh.row * a.out_row + (long long)rh.head * a.out_head : (long long)col * D) * (fp32 ? 4 : 2);
#pragma unroll 1
      for (int b = 0; b < 2 * (D / 64); ++b) {                             // rows 16 (b / (D / 64)) + 8 half, 64 dims
        const int c = (b % (D / 64)) * 64, r16 = 16 * (b / (D / 64)), r0 = r16 + (lane >> 2);
        float v[32];
        __syncwarp();
        tmem_ld_16x64(to + ((uint32_t)r16 << 16) + (uint32_t)c, v);
        tmem_ld_wait();
#pragma unroll
        for (int half = 0; half < 2; ++half) {
          const float m = __shfl_sync(0xffffffffu, mul.x, r0 + 8 * half), m2 = __shfl_sync(0xffffffffu, mul.y, r0 + 8 * half);
          char* dst = to_base + __shfl_sync(0xffffffffu, to_row, r0 + 8 * half) + (c + 2 * (lane & 3)) * (fp32 ? 4 : 2);
          if (i * kRows + 32 * quarter + r0 + 8 * half >= it.n_cols) continue;
          if (fp32) {
#pragma unroll
            for (int k = 0; k < 8; ++k) *reinterpret_cast<float2*>(dst + 32 * k) = make_float2(v[4 * k + 2 * half] * m * m2, v[4 * k + 2 * half + 1] * m * m2);
          } else {
#pragma unroll
            for (int k = 0; k < 8; ++k) *reinterpret_cast<uint32_t*>(dst + 16 * k) = pack2(v[4 * k + 2 * half] * m * m2, v[4 * k + 2 * half + 1] * m * m2);
          }
        }
      }
      tc_fence_before();
      if (begun && !goes_on && tid == 0) a.joins[cta] = make_int4(1 + runs.cta_of(u - it.span - (it.page - it.first)), it.s.first, it.r0, it.head | (it.n_cols << 16));
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
  static_assert(Tc<D>::bytes(VS_CACHE_MAX_SEQS) <= 227 * 1024, "shared memory of an SM");
  // (the limit is the function's, not the call's: that of the most sequences, so that calls of other threads set the same)
  if (cudaFuncSetAttribute(cache_attention_tc_kernel<D>, cudaFuncAttributeMaxDynamicSharedMemorySize, Tc<D>::bytes(VS_CACHE_MAX_SEQS)) != cudaSuccess) return VS_ERR_CUDA;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(kManyCtas);
  cfg.blockDim = dim3(kThreads);
  cfg.dynamicSmemBytes = (size_t)Tc<D>::bytes(a.r.n_seqs);
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
