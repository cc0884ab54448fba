// What the stand-alone operators share: the device a call is for, the rows of a call's sequences, 8-bit codes.
#pragma once
#include <cuda_fp8.h>
#include <cuda_fp16.h>
#include <cmath>

#include "vs_common.cuh"

namespace vs {

// The device of a call made current for as long as the call runs.
struct OnDevice {
  int before = -1;
  bool ok = false;
  explicit OnDevice(int device) {
    if (device < 0 || cudaGetDevice(&before) != cudaSuccess) return;
    ok = before == device || cudaSetDevice(device) == cudaSuccess;
    if (!ok) cudaGetLastError();                       // (the caller is told; the next launch must not find it)
    if (before == device || !ok) before = -1;          // nothing to put back
  }
  ~OnDevice() { if (before >= 0) cudaSetDevice(before); }
  OnDevice(const OnDevice&) = delete;
  OnDevice& operator=(const OnDevice&) = delete;
};

inline int launched() { return cudaGetLastError() == cudaSuccess ? VS_OK : VS_ERR_CUDA; }
inline bool aligned(const void* p, size_t to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) == 0; }

constexpr int kPage = VS_CACHE_PAGE;
constexpr int kScaleMinExp = -110, kScaleMaxExp = 120;

// The checks that the calls on a cache share.
inline int check_cache(const vs_cache* c, const vs_cache_seqs* r) {
  if (c == nullptr || r == nullptr || c->k == nullptr || c->v == nullptr || c->k_scale == nullptr || c->v_scale == nullptr) return VS_ERR_INVALID_ARG;
  if (r->page_table == nullptr || r->tokens == nullptr) return VS_ERR_INVALID_ARG;
  if (c->n_pages < 1 || c->n_kv_heads < 1 || r->table_width < 1 || r->n_rows < 0 || r->n_seqs < 1) return VS_ERR_INVALID_ARG;
  if (c->head_dim != 64 && c->head_dim != 128) return VS_ERR_UNSUPPORTED;
  if (c->n_kv_heads > VS_CACHE_MAX_HEADS) return VS_ERR_UNSUPPORTED;
  if (r->n_seqs > VS_CACHE_MAX_SEQS) return VS_ERR_CAPACITY;
  if (r->row_offsets == nullptr && r->n_rows % r->n_seqs != 0) return VS_ERR_INVALID_ARG;
  if (!aligned(c->k, 16) || !aligned(c->v, 16) || !aligned(c->k_scale, 4) || !aligned(c->v_scale, 4)) return VS_ERR_INVALID_ARG;
  if (!aligned(r->page_table, 4) || !aligned(r->tokens, 4) || !aligned(r->row_offsets, 4)) return VS_ERR_INVALID_ARG;
  return VS_OK;
}

#ifdef __CUDACC__
// Rows [first, first + n) of the call are sequence i's.  Whatever the offsets hold, the rows named lie in [0, n_rows).
struct SeqRows { int first, n; };
__device__ __forceinline__ SeqRows rows_of(const vs_cache_seqs& r, int i) {
  if (r.row_offsets == nullptr) { const int n = r.n_rows / r.n_seqs; return {i * n, n}; }
  const int a = min(max(r.row_offsets[i], 0), r.n_rows), b = min(max(r.row_offsets[i + 1], a), r.n_rows);
  return {a, b - a};
}
// Page of tokens 64 p ... 64 p + 63 of sequence i; -1 where the table has none that the pool holds.
__device__ __forceinline__ int page_of(const vs_cache_seqs& r, int n_pages, int i, int p) {
  if (p < 0 || p >= r.table_width) return -1;
  const int page = r.page_table[(size_t)i * r.table_width + p];
  return page >= 0 && page < n_pages ? page : -1;
}

__device__ __forceinline__ int exponent_of(float scale) { return (int)((__float_as_uint(scale) >> 23) & 255u) - 127; }
__device__ __forceinline__ float power_of_two(int e) { return __uint_as_float((uint32_t)min(max(e + 127, 0), 254) << 23); }   // (0 below 2^-126)

// e4m3 codes (low byte first) -> values
__device__ __forceinline__ void codes_to_half2(uint32_t four, uint32_t& low, uint32_t& high) {
  asm("{\n\t.reg .b16 l, h;\n\tmov.b32 {l, h}, %2;\n\tcvt.rn.f16x2.e4m3x2 %0, l;\n\tcvt.rn.f16x2.e4m3x2 %1, h;\n\t}" : "=r"(low), "=r"(high) : "r"(four));
}
__device__ __forceinline__ void codes_to_floats(uint32_t four, float (&x)[4]) {
  uint32_t l, h;
  codes_to_half2(four, l, h);
  const float2 a = __half22float2(*reinterpret_cast<const __half2*>(&l)), b = __half22float2(*reinterpret_cast<const __half2*>(&h));
  x[0] = a.x; x[1] = a.y; x[2] = b.x; x[3] = b.y;
}
// 1 in every byte that is NaN's code
__device__ __forceinline__ uint32_t nan_codes(uint32_t four) { return ((four & 0x7f7f7f7fu) + 0x01010101u) >> 7 & 0x01010101u; }
// nearest code, ties to the even one, magnitudes above 448 to 448, NaN to NaN
__device__ __forceinline__ uint32_t float2_to_codes(float lo, float hi) {
  return (uint32_t)__nv_cvt_float2_to_fp8x2(make_float2(lo, hi), __NV_SATFINITE, __NV_E4M3);
}

// eight elements of a bf16 or fp32 row (16-byte aligned) <-> fp32
__device__ __forceinline__ void load8(const bf16* p, float (&x)[8]) {
  const uint4 u = *reinterpret_cast<const uint4*>(p);
  const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) { x[2 * i] = __uint_as_float(w[i] << 16); x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u); }
}
__device__ __forceinline__ void load8(const float* p, float (&x)[8]) {
  const float4 a = *reinterpret_cast<const float4*>(p), b = *reinterpret_cast<const float4*>(p + 4);
  x[0] = a.x; x[1] = a.y; x[2] = a.z; x[3] = a.w; x[4] = b.x; x[5] = b.y; x[6] = b.z; x[7] = b.w;
}
__device__ __forceinline__ void store8(bf16* p, const float (&x)[8]) {
  uint32_t w[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const __nv_bfloat162 t = __floats2bfloat162_rn(x[2 * i], x[2 * i + 1]);
    w[i] = *reinterpret_cast<const uint32_t*>(&t);
  }
  *reinterpret_cast<uint4*>(p) = make_uint4(w[0], w[1], w[2], w[3]);
}
__device__ __forceinline__ void store8(float* p, const float (&x)[8]) {
  *reinterpret_cast<float4*>(p) = make_float4(x[0], x[1], x[2], x[3]);
  *reinterpret_cast<float4*>(p + 4) = make_float4(x[4], x[5], x[6], x[7]);
}
#endif  // __CUDACC__

}  // namespace vs
