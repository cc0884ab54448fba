// vs_rope_axes: rotary positions with several axes (a video token's time, height and width).
//
// Pair k of a head, (x_k, x_{k + D/2}), turns by the angle  pos[axis(k)] theta^(-2k / D): the frequency goes by the pair, the
// position by the axis that the pair belongs to.  The inverse turns back, which is also the gradient with respect to x.
//
// What bounds it: the rows' bytes once in and once out; a call of one row is a launch and two dependent loads.  A warp takes some heads of a
// row and asks for its pieces of them first (16 bytes of either half), works out the angles while those are on their way -- a lane some pairs'
// each, once for all of the warp's heads -- and hands them round through shared memory: a lane turns the same eight pairs of every head
// that it meets, so it keeps them in registers.  No warp waits for another.  A far position loses nothing: the angle is
// formed in turns in fp64, and only the fraction of a turn goes on in fp32.
// Measured: 3376 rows of 32 bf16 heads of 128, 11.3 us (4.9 TB/s; a floor of 8.5), where a block a row with its angles behind a barrier takes 15.0 (two rows
// a block the same, four 15.7); one row 2 us beyond an empty launch.
#include "vs_operators.cuh"

namespace vs {

namespace {

constexpr int kWarps = 4, kMaxHalf = 128, kLoads = 4;

struct RopeAxesArgs {
  const void* x;
  void* out;
  const int64_t* positions;
  long long x_row, x_head, out_row, out_head, pos_stride;
  int rows, heads, half, inverse, per_row, beside;     // warps of a row; heads that a warp takes side by side
  uint32_t axis[kMaxHalf / 16];        // of a pair, two bits each
  double turns[32], step;              // theta^(-2k / D) / 2 pi of the first 32 pairs, and theta^(-64 / D)
};

// eight elements as they are stored
template <typename T> struct Raw;
template <> struct Raw<bf16> { uint4 a; __device__ __forceinline__ void load(const bf16* p) { a = *reinterpret_cast<const uint4*>(p); } };
template <> struct Raw<float> {
  uint4 a, b;
  __device__ __forceinline__ void load(const float* p) { a = *reinterpret_cast<const uint4*>(p); b = *reinterpret_cast<const uint4*>(p + 4); }
};
__device__ __forceinline__ void values(const Raw<bf16>& r, float (&x)[8]) { load8(reinterpret_cast<const bf16*>(&r), x); }
__device__ __forceinline__ void values(const Raw<float>& r, float (&x)[8]) { load8(reinterpret_cast<const float*>(&r), x); }

template <typename T>
__global__ void __launch_bounds__(32 * kWarps) rope_axes_kernel(const __grid_constant__ RopeAxesArgs a) {
  // (eight pairs and 16 bytes of nothing: what eight lanes read side by side lies in different banks)
  __shared__ __align__(16) float2 turn[kWarps][kMaxHalf / 8 * 10];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const long long w = (long long)blockIdx.x * kWarps + warp;
  const int row = (int)(w / a.per_row), part = (int)(w - (long long)row * a.per_row);
  if (row >= a.rows) return;
  const int per_head = a.half / 8, mine = lane / per_head, k0 = (lane - mine * per_head) * 8;      // the lane's head of those side by side
  const int head0 = part * kLoads * a.beside + mine;
  const bool idle = mine >= a.beside;
  const T* x = static_cast<const T*>(a.x) + (long long)row * a.x_row + k0;
  T* out = static_cast<T*>(a.out) + (long long)row * a.out_row + k0;
  Raw<T> lo[kLoads], hi[kLoads];
#pragma unroll
  for (int u = 0; u < kLoads; ++u) {
    const int head = head0 + u * a.beside;
    if (idle || head >= a.heads) continue;
    lo[u].load(x + (long long)head * a.x_head);
    hi[u].load(x + (long long)head * a.x_head + a.half);
  }
  double turns = a.turns[lane];
  for (int k = lane; k < a.half; k += 32, turns *= a.step) {
    const int axis = (int)(a.axis[k >> 4] >> (2 * (k & 15))) & 3;
    const double t = (double)a.positions[(long long)axis * a.pos_stride + row] * turns;
    float s, c;
    sincospif(2.f * (float)(t - rint(t)), &s, &c);
    turn[warp][k + (k >> 3) * 2] = make_float2(c, a.inverse ? -s : s);
  }
  __syncwarp();
  if (idle) return;
  float4 cs[4];
#pragma unroll
  for (int e = 0; e < 4; ++e) cs[e] = reinterpret_cast<const float4*>(&turn[warp][k0 + (k0 >> 3) * 2])[e];
#pragma unroll
  for (int u = 0; u < kLoads; ++u) {
    const int head = head0 + u * a.beside;
    if (head >= a.heads) break;
    float l[8], h[8], y[8], z[8];
    values(lo[u], l);
    values(hi[u], h);
#pragma unroll
    for (int e = 0; e < 8; e += 2) {
      const float4 t = cs[e / 2];
      y[e] = l[e] * t.x - h[e] * t.y;
      z[e] = h[e] * t.x + l[e] * t.y;
      y[e + 1] = l[e + 1] * t.z - h[e + 1] * t.w;
      z[e + 1] = h[e + 1] * t.z + l[e + 1] * t.w;
    }
    T* at = out + (long long)head * a.out_head;
    store8(at, y);
    store8(at + a.half, z);
  }
}

// The axis whose position turns pair k: the sections one behind the other, or the pairs dealt to the axes in turn, one that has its share
// left out.
void deal_axes(const int32_t* sections, int n_axes, int half, bool interleaved, uint32_t* axis) {
  int left[VS_MAX_AXES];
  for (int i = 0; i < n_axes; ++i) left[i] = sections[i];
  for (int k = 0, i = 0; k < half; i = interleaved ? i + 1 : i) {
    if (i == n_axes) i = 0;
    if (left[i] == 0) { if (!interleaved) ++i; continue; }
    --left[i];
    axis[k >> 4] |= (uint32_t)i << (2 * (k & 15));
    ++k;
  }
}

// theta^(-2k / D) / 2 pi of the first pairs: kept by the calling thread for its next call of the same base and size (32 powers take longer
// than the launch)
struct Turns { double theta = 0.0; int half = 0; double of[32]; };
const double* turns_of(double theta, int half) {
  static thread_local Turns kept;
  if (kept.theta != theta || kept.half != half) {
    for (int k = 0; k < 32; ++k) kept.of[k] = std::pow(theta, -(double)k / half) * 0.15915494309189533577;
    kept.theta = theta;
    kept.half = half;
  }
  return kept.of;
}

}  // namespace

}  // namespace vs

extern "C" int vs_rope_axes(const vs_rope* r, void* cuda_stream) {
  using namespace vs;
  if (r == nullptr || r->rows < 0 || r->heads < 1 || r->dtype < 0 || r->dtype > 1) return VS_ERR_INVALID_ARG;
  if (r->n_axes < 1 || r->n_axes > VS_MAX_AXES || !(r->theta > 0.0) || !std::isfinite(r->theta)) return VS_ERR_INVALID_ARG;
  if (r->head_dim < 16 || r->head_dim > 2 * kMaxHalf || r->head_dim % 16 != 0) return VS_ERR_UNSUPPORTED;
  if (r->heads > 65536) return VS_ERR_UNSUPPORTED;
  const int half = r->head_dim / 2;
  long long sum = 0;
  for (int i = 0; i < r->n_axes; ++i) {
    if (r->sections[i] < 0) return VS_ERR_INVALID_ARG;
    sum += r->sections[i];
  }
  if (sum != half) return VS_ERR_INVALID_ARG;
  if (r->rows == 0) return VS_OK;
  if (r->x == nullptr || r->out == nullptr || r->positions == nullptr || !aligned(r->positions, 8)) return VS_ERR_INVALID_ARG;
  const int64_t piece = r->dtype == 1 ? 4 : 8;                           // elements of 16 bytes
  const int64_t strides[4] = {r->x_row_stride, r->x_head_stride, r->out_row_stride, r->out_head_stride};
  for (int64_t s : strides) if (s % piece != 0) return VS_ERR_INVALID_ARG;
  if (!aligned(r->x, 16) || !aligned(r->out, 16)) return VS_ERR_INVALID_ARG;
  if (r->x == r->out && (strides[0] != strides[2] || strides[1] != strides[3])) return VS_ERR_INVALID_ARG;      // (in place: row by row)
  OnDevice on(r->device);
  if (!on.ok) return VS_ERR_CUDA;
  RopeAxesArgs a = {};
  a.x = r->x; a.out = r->out; a.positions = r->positions;
  a.x_row = strides[0]; a.x_head = strides[1]; a.out_row = strides[2]; a.out_head = strides[3]; a.pos_stride = r->pos_stride;
  a.rows = r->rows; a.heads = r->heads; a.half = half; a.inverse = r->inverse != 0;
  a.beside = 32 / (half / 8);
  a.per_row = (r->heads + kLoads * a.beside - 1) / (kLoads * a.beside);
  deal_axes(r->sections, r->n_axes, half, r->interleaved != 0, a.axis);
  const double* turns = turns_of(r->theta, half);
  for (int k = 0; k < 32; ++k) a.turns[k] = turns[k];
  a.step = std::pow(r->theta, -32.0 / half);
  const long long blocks = ((long long)r->rows * a.per_row + kWarps - 1) / kWarps;
  if (blocks > 0x7fffffffll) return VS_ERR_UNSUPPORTED;
  cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
  if (r->dtype == 1) rope_axes_kernel<float><<<(unsigned)blocks, 32 * kWarps, 0, st>>>(a);
  else rope_axes_kernel<bf16><<<(unsigned)blocks, 32 * kWarps, 0, st>>>(a);
  return launched();
}
