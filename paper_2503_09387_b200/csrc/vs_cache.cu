// vs_cache_write, vs_cache_read: rows of keys and values into and out of a paged cache of 8-bit codes.
//
// A page holds 64 tokens; its codes of one head (e4m3) share a scale 2^e, the smallest with every finite magnitude of the page at
// most 448 * 2^e.  A power of two costs a floating format nothing -- dividing by it only moves exponents -- and makes the codes a
// matter of one rounding with no border to fall on either side of.  A page grows as its sequence does: rows that need a larger
// scale than the page has raise it, and the codes that are there are rounded once more at the new one (exactly, but for those
// that become subnormal).  The first token of a page starts it afresh.
//
// What bounds them: the rows' bytes and the codes', for long reads the conversions as well (issue slots 69 %: four of codes, eight widenings, eight
// products and four packings for eight elements).  A block takes the rows of one page and head, keys or values: it holds them in
// registers from the load to the codes, the maximum in between, so that they are read once.  Blocks find their page by
// the sequences' rows on the device; the host knows how many there can be.
// Measured: 13440 tokens of four heads of 128 read as bf16 (13.8 MB in, 27.5 MB out) 9.6 us, 4.3 TB/s; 2950 written from bf16 8 us, one of each of sixteen
// sequences 3: beyond the launch, two dependent loads (the sequence's length, its page) and the rows.
#include "vs_operators.cuh"

namespace vs {

namespace {

constexpr int kThreads = 256;

struct CacheArgs {
  vs_cache c;
  vs_cache_seqs r;
  void *k, *v;                        // rows
  long long k_row, k_head, v_row, v_head;
};

// The `unit`-th page that the call's rows lie in, counted through the sequences: rows [row, row + n) are tokens at ... at + n - 1
// of the page.
struct PageRows { int seq, page, at, row, n; };
__device__ __forceinline__ PageRows find_page(const vs_cache_seqs& r, int n_pages, int unit) {
  const int lane = threadIdx.x & 31;
  PageRows found = {-1, -1, 0, 0, 0};
  long long before = 0;
  for (int base = 0; base < r.n_seqs; base += 32) {
    const int i = base + lane;
    SeqRows s = {0, 0};
    int held = 0;
    if (i < r.n_seqs) { s = rows_of(r, i); held = max(r.tokens[i], 0); }
    const int at = held % kPage, pages = s.n > 0 ? (int)(((long long)at + s.n + kPage - 1) / kPage) : 0;
    int sum = pages;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) { const int t = __shfl_up_sync(0xffffffffu, sum, o); if (lane >= o) sum += t; }
    const bool mine = before + sum > unit;
    const unsigned who = __ballot_sync(0xffffffffu, mine);
    if (who != 0u) {
      const int w = __ffs(who) - 1;
      const int seq = base + w, first = __shfl_sync(0xffffffffu, s.first, w), n = __shfl_sync(0xffffffffu, s.n, w);
      const int local = (int)(unit - before) - __shfl_sync(0xffffffffu, sum - pages, w);        // page of the sequence's, from the first touched on
      const int at0 = __shfl_sync(0xffffffffu, at, w), held0 = __shfl_sync(0xffffffffu, held, w);
      const int skip = local == 0 ? 0 : local * kPage - at0;                                 // rows in the pages before
      found.seq = seq;
      found.at = local == 0 ? at0 : 0;
      found.row = first + skip;
      found.n = min(kPage - found.at, n - skip);
      const long long p = (long long)held0 / kPage + local;
      found.page = p < r.table_width ? page_of(r, n_pages, seq, (int)p) : -1;
      return found;
    }
    before += __shfl_sync(0xffffffffu, sum, 31);
  }
  return found;
}

template <typename T, int D>
__global__ void __launch_bounds__(kThreads) cache_write_kernel(const __grid_constant__ CacheArgs a) {
  constexpr int CPR = D / 8, PER = kPage * CPR / kThreads;             // pieces of eight elements: of a row, of a thread
  const PageRows p = find_page(a.r, a.c.n_pages, (int)blockIdx.x);
  if (p.page < 0) return;                                               // no rows left, or none that the table has a page for
  const int head = (int)blockIdx.y >> 1, is_v = (int)blockIdx.y & 1;
  const T* rows = static_cast<const T*>(is_v ? a.v : a.k) + (long long)p.row * (is_v ? a.v_row : a.k_row) + (long long)head * (is_v ? a.v_head : a.k_head);
  const long long step = is_v ? a.v_row : a.k_row;
  const size_t tile = (size_t)p.page * a.c.n_kv_heads + head;
  uint8_t* codes = static_cast<uint8_t*>(is_v ? a.c.v : a.c.k) + tile * (kPage * D);
  float* scale = (is_v ? a.c.v_scale : a.c.k_scale) + tile;
  const int e_old = p.at > 0 ? min(max(exponent_of(*scale), kScaleMinExp), kScaleMaxExp) : kScaleMinExp;
  float x[PER][8], amax = 0.f;
#pragma unroll
  for (int u = 0; u < PER; ++u) {
    const int i = (int)threadIdx.x + u * kThreads, t = i / CPR, c = i - t * CPR;
    if (t < p.n) load8(rows + t * step + c * 8, x[u]);
    else
#pragma unroll
      for (int e = 0; e < 8; ++e) x[u][e] = 0.f;
  }
#pragma unroll
  for (int u = 0; u < PER; ++u)
#pragma unroll
    for (int e = 0; e < 8; ++e) { const float m = fabsf(x[u][e]); amax = m <= 3.402823466e38f ? fmaxf(amax, m) : amax; }      // (neither infinity nor NaN)
  amax = __uint_as_float(__reduce_max_sync(0xffffffffu, __float_as_uint(amax)));
  __shared__ float warp_max[kThreads / 32];
  if ((threadIdx.x & 31) == 0) warp_max[threadIdx.x >> 5] = amax;
  __syncthreads();                                                      // (every thread has read the old scale by now)
#pragma unroll
  for (int i = 0; i < kThreads / 32; ++i) amax = fmaxf(amax, warp_max[i]);
  // amax = f 2^(x), 1 <= f < 2, and 448 = 1.75 * 2^8: the exponent is x - 8, one more where f > 1.75.  (0 and subnormal values: the least)
  const uint32_t bits = __float_as_uint(amax);
  const int e_rows = (int)(bits >> 23) - 127 - 8 + ((bits & 0x7fffffu) > 0x600000u ? 1 : 0);
  const int e = max(min(max(e_rows, kScaleMinExp), kScaleMaxExp), e_old);
  if (e > e_old && p.at > 0) {
    const float down = power_of_two(e_old - e);
    for (int i = threadIdx.x; i < p.at * CPR; i += kThreads) {
      uint2* at = reinterpret_cast<uint2*>(codes + (size_t)i * 8);
      const uint2 w = *at;
      uint32_t q[2] = {0u, 0u};
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        float f[4];
        codes_to_floats(h ? w.y : w.x, f);
        q[h] = float2_to_codes(f[0] * down, f[1] * down) | float2_to_codes(f[2] * down, f[3] * down) << 16;
      }
      *at = make_uint2(q[0], q[1]);
    }
  }
  const float inv = power_of_two(-e);
#pragma unroll
  for (int u = 0; u < PER; ++u) {
    const int i = (int)threadIdx.x + u * kThreads, t = i / CPR, c = i - t * CPR;
    if (t >= p.n) continue;
    uint32_t q[2] = {0u, 0u};
#pragma unroll
    for (int h = 0; h < 4; ++h) q[h >> 1] |= float2_to_codes(x[u][2 * h] * inv, x[u][2 * h + 1] * inv) << (16 * (h & 1));
    *reinterpret_cast<uint2*>(codes + (size_t)(p.at + t) * D + c * 8) = make_uint2(q[0], q[1]);
  }
  if (threadIdx.x == 0) *scale = power_of_two(e);
}

template <typename T, int D>
__global__ void __launch_bounds__(kThreads) cache_read_kernel(const __grid_constant__ CacheArgs a) {
  constexpr int CPR = D / 8, PER = kPage * CPR / kThreads;
  const PageRows p = find_page(a.r, a.c.n_pages, (int)blockIdx.x);
  if (p.n == 0) return;
  const int head = (int)blockIdx.y >> 1, is_v = (int)blockIdx.y & 1;
  T* rows = static_cast<T*>(is_v ? a.v : a.k) + (long long)p.row * (is_v ? a.v_row : a.k_row) + (long long)head * (is_v ? a.v_head : a.k_head);
  const long long step = is_v ? a.v_row : a.k_row;
  const size_t tile = (size_t)max(p.page, 0) * a.c.n_kv_heads + head;
  const uint8_t* codes = static_cast<const uint8_t*>(is_v ? a.c.v : a.c.k) + tile * (kPage * D);
  const float scale = p.page >= 0 ? (is_v ? a.c.v_scale : a.c.k_scale)[tile] : 0.f;
  uint2 w[PER];
#pragma unroll
  for (int u = 0; u < PER; ++u) {
    const int i = (int)threadIdx.x + u * kThreads, t = i / CPR, c = i - t * CPR;
    w[u] = (t < p.n && p.page >= 0) ? *reinterpret_cast<const uint2*>(codes + (size_t)(p.at + t) * D + c * 8) : make_uint2(0u, 0u);
  }
#pragma unroll
  for (int u = 0; u < PER; ++u) {
    const int i = (int)threadIdx.x + u * kThreads, t = i / CPR, c = i - t * CPR;
    if (t >= p.n) continue;
    float x[8];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      float f[4];
      codes_to_floats(h ? w[u].y : w[u].x, f);
#pragma unroll
      for (int e = 0; e < 4; ++e) x[4 * h + e] = f[e] * scale;
    }
    store8(rows + t * step + c * 8, x);
  }
}

int run(const vs_cache* c, const vs_cache_rows* rows, void* cuda_stream, bool write) {
  if (rows == nullptr) return VS_ERR_INVALID_ARG;
  const vs_cache_seqs* r = &rows->seqs;
  const int rc = check_cache(c, r);
  if (rc != VS_OK) return rc;
  const int32_t dtype = rows->dtype;
  if (dtype < 0 || dtype > 1) return VS_ERR_INVALID_ARG;
  if (r->n_rows == 0) return VS_OK;
  if (rows->k == nullptr || rows->v == nullptr || !aligned(rows->k, 16) || !aligned(rows->v, 16)) return VS_ERR_INVALID_ARG;
  const int64_t piece = dtype == 1 ? 4 : 8, strides[4] = {rows->k_row_stride, rows->k_head_stride, rows->v_row_stride, rows->v_head_stride};
  for (int64_t s : strides) if (s % piece != 0) return VS_ERR_INVALID_ARG;
  OnDevice on(c->device);
  if (!on.ok) return VS_ERR_CUDA;
  CacheArgs a = {*c, *r, rows->k, rows->v, strides[0], strides[1], strides[2], strides[3]};
  // most pages that the rows can lie in: a sequence's first and last one are perhaps not full
  const long long pages = (long long)r->n_rows / kPage + 2ll * r->n_seqs;
  const dim3 grid((unsigned)(pages < r->n_rows ? pages : r->n_rows), (unsigned)(2 * c->n_kv_heads));
  cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
  const int form = (write ? 4 : 0) + (dtype == 1 ? 2 : 0) + (c->head_dim == 128 ? 1 : 0);
  switch (form) {
    case 0: cache_read_kernel<bf16, 64><<<grid, kThreads, 0, st>>>(a); break;
    case 1: cache_read_kernel<bf16, 128><<<grid, kThreads, 0, st>>>(a); break;
    case 2: cache_read_kernel<float, 64><<<grid, kThreads, 0, st>>>(a); break;
    case 3: cache_read_kernel<float, 128><<<grid, kThreads, 0, st>>>(a); break;
    case 4: cache_write_kernel<bf16, 64><<<grid, kThreads, 0, st>>>(a); break;
    case 5: cache_write_kernel<bf16, 128><<<grid, kThreads, 0, st>>>(a); break;
    case 6: cache_write_kernel<float, 64><<<grid, kThreads, 0, st>>>(a); break;
    default: cache_write_kernel<float, 128><<<grid, kThreads, 0, st>>>(a); break;
  }
  return launched();
}

}  // namespace

}  // namespace vs

extern "C" int vs_cache_write(const vs_cache* cache, const vs_cache_rows* rows, void* cuda_stream) { return vs::run(cache, rows, cuda_stream, true); }
extern "C" int vs_cache_read(const vs_cache* cache, const vs_cache_rows* rows, void* cuda_stream) { return vs::run(cache, rows, cuda_stream, false); }
