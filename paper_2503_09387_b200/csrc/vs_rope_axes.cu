// vs_rope_axes: rotary positions with several axes (a video token's time, height and width).
//
// Pair k of a head, (x_k, x_{k + D/2}), turns by the angle  pos[axis(k)] theta^(-2k / D): the frequency goes by the pair, the
// position by the axis that the pair belongs to.  The inverse turns back, which is also the gradient with respect to x.
//
// What bounds it: the rows' bytes once in and once out; a call of one row is a launch and two dependent loads.  A block takes
// kRows rows: its threads ask for their pieces of the rows first, then work out one angle each (row, pair) while those are on
// their way, and turn every head of the rows by the angles in shared memory.  (cos, sin) of a far position loses nothing: the
// angle is formed in turns in fp64, and only the fraction of a turn goes on in fp32.
#include "vs_operators.cuh"

namespace vs {

namespace {

constexpr int kThreads = 256, kMaxHalf = 128, kAhead = 4;

struct RopeAxesArgs {
  const void* x;
  void* out;
  const int64_t* positions;
  long long x_row, x_head, out_row, out_head, pos_stride;
  double log2_theta;
  int rows, heads, half, axes, interleaved, inverse;
  int section[VS_MAX_AXES];
};

// the axis whose position turns pair k
__device__ __forceinline__ int axis_of(const RopeAxesArgs& a, int k) {
  if (!a.interleaved) {
    int axis = 0;
#pragma unroll
    for (int i = 0; i < VS_MAX_AXES - 1; ++i) { if (i < a.axes - 1 && axis == i && k >= a.section[i]) { k -= a.section[i]; axis = i + 1; } }
    return axis;
  }
  // the pairs are dealt to the axes in turn, one that has its share left out: round r has a pair for every axis with more than r
  int dealt = 0;
  for (int r = 0;; ++r) {
    int in_round = 0;
#pragma unroll
    for (int i = 0; i < VS_MAX_AXES; ++i) in_round += i < a.axes && a.section[i] > r;
    if (in_round == 0) return 0;                                         // (k is below the sections' sum)
    if (k < dealt + in_round) {
      int left = k - dealt;
#pragma unroll
      for (int i = 0; i < VS_MAX_AXES; ++i)
        if (i < a.axes && a.section[i] > r && left-- == 0) return i;
    }
    dealt += in_round;
  }
}

template <typename T, int kRows>
__global__ void __launch_bounds__(kThreads) rope_axes_kernel(const __grid_constant__ RopeAxesArgs a) {
  __shared__ float2 turn[kRows][kMaxHalf];
  const int row0 = (int)blockIdx.x * kRows, n_rows = min(kRows, a.rows - row0);
  const int per_head = a.half / 8, per_row = a.heads * per_head, n = n_rows * per_row;      // pieces of eight pairs
  const T* x = static_cast<const T*>(a.x);
  T* out = static_cast<T*>(a.out);
  struct Piece { int row, head, k; };
  auto piece = [&](int i) {
    Piece p;
    p.row = i / per_row;
    const int j = i - p.row * per_row;
    p.head = j / per_head;
    p.k = (j - p.head * per_head) * 8;
    return p;
  };
  float lo[kAhead][8], hi[kAhead][8];
  auto load = [&](int i, float (&l)[8], float (&h)[8]) {
    if (i >= n) return;
    const Piece p = piece(i);
    const T* at = x + (long long)(row0 + p.row) * a.x_row + (long long)p.head * a.x_head + p.k;
    load8(at, l);
    load8(at + a.half, h);
  };
#pragma unroll
  for (int u = 0; u < kAhead; ++u) load((int)threadIdx.x + u * kThreads, lo[u], hi[u]);
  for (int i = threadIdx.x; i < n_rows * a.half; i += kThreads) {
    const int row = i / a.half, k = i - row * a.half;
    const double pos = (double)a.positions[(long long)axis_of(a, k) * a.pos_stride + row0 + row];
    constexpr double kInv2Pi = 0.15915494309189533577;
    const double t = pos * (exp2(-a.log2_theta * (double)k / (double)a.half) * kInv2Pi);
    float s, c;
    sincospif(2.f * (float)(t - rint(t)), &s, &c);
    turn[row][k] = make_float2(c, a.inverse ? -s : s);
  }
  __syncthreads();
  for (int i0 = 0; i0 < n; i0 += kAhead * kThreads) {
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
      const int i = i0 + (int)threadIdx.x + u * kThreads;
      if (i >= n) continue;
      if (i0 > 0) load(i, lo[u], hi[u]);
      const Piece p = piece(i);
      float y[8], z[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float2 cs = turn[p.row][p.k + e];
        y[e] = lo[u][e] * cs.x - hi[u][e] * cs.y;
        z[e] = hi[u][e] * cs.x + lo[u][e] * cs.y;
      }
      T* at = out + (long long)(row0 + p.row) * a.out_row + (long long)p.head * a.out_head + p.k;
      store8(at, y);
      store8(at + a.half, z);
    }
  }
}

}  // namespace

}  // namespace vs

extern "C" int vs_rope_axes(const void* x, int64_t x_row_stride, int64_t x_head_stride, void* out, int64_t out_row_stride,
                            int64_t out_head_stride, int32_t dtype, int32_t rows, int32_t heads, int32_t head_dim,
                            const int64_t* positions, int64_t pos_stride, int32_t n_axes, const int32_t* sections,
                            int32_t interleaved, int32_t inverse, double theta, int32_t device, void* cuda_stream) {
  using namespace vs;
  if (rows < 0 || heads < 1 || dtype < 0 || dtype > 1) return VS_ERR_INVALID_ARG;
  if (sections == nullptr || n_axes < 1 || n_axes > VS_MAX_AXES || !(theta > 0.0) || !std::isfinite(theta)) return VS_ERR_INVALID_ARG;
  if (head_dim < 16 || head_dim > 2 * kMaxHalf || head_dim % 16 != 0) return VS_ERR_UNSUPPORTED;
  if (heads > 65536) return VS_ERR_UNSUPPORTED;
  RopeAxesArgs a = {};
  long long sum = 0;
  for (int i = 0; i < n_axes; ++i) {
    if (sections[i] < 0) return VS_ERR_INVALID_ARG;
    a.section[i] = sections[i];
    sum += sections[i];
  }
  if (sum != head_dim / 2) return VS_ERR_INVALID_ARG;
  if (rows == 0) return VS_OK;
  if (x == nullptr || out == nullptr || positions == nullptr || !aligned(positions, 8)) return VS_ERR_INVALID_ARG;
  const int64_t piece = dtype == 1 ? 4 : 8;                              // elements of 16 bytes
  const int64_t strides[4] = {x_row_stride, x_head_stride, out_row_stride, out_head_stride};
  for (int64_t s : strides) if (s % piece != 0) return VS_ERR_INVALID_ARG;
  if (!aligned(x, 16) || !aligned(out, 16)) return VS_ERR_INVALID_ARG;
  OnDevice on(device);
  if (!on.ok) return VS_ERR_CUDA;
  a.x = x; a.out = out; a.positions = positions;
  a.x_row = x_row_stride; a.x_head = x_head_stride; a.out_row = out_row_stride; a.out_head = out_head_stride; a.pos_stride = pos_stride;
  a.log2_theta = std::log2(theta);
  a.rows = rows; a.heads = heads; a.half = head_dim / 2; a.axes = n_axes; a.interleaved = interleaved != 0; a.inverse = inverse != 0;
  cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
  if (dtype == 1) rope_axes_kernel<float, 1><<<rows, kThreads, 0, st>>>(a);
  else rope_axes_kernel<bf16, 1><<<rows, kThreads, 0, st>>>(a);
  return launched();
}
