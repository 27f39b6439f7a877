// The norms after and before a block, with the block's gate and the scale of
// the residual stream, in one pass over a row:
//
//   y' = y * post / rms(y)                      (y' = y without post)
//   h' = residual_scale * h + gate * y'         (gate of every channel, or of every token and channel)
//   x  = h' * pre / rms(h')                     rms(v) = sqrt(mean(v^2) + eps)
//
// A row is read once into registers and both sums of squares are taken from
// there in fp32, so a pass moves h, y, h' and x once: HBM bounds it for many
// rows, the launch and two reductions for few (4096 columns, bf16: 4093 rows
// with a gate each, 268 MB, 52 us, 5.1 TB/s; one row 4.2 us on the GPU).
#include "common.hpp"

namespace moe {
namespace {

// Sum over the WAVES waves of a workgroup, on every lane.  `slot`: a region of
// its own for each sum, so that one barrier is enough.
template <int WAVES>
__device__ __forceinline__ float group_sum(float v, float *slot) {
  v = wave_sum(v);
  if constexpr (WAVES > 1) {
    if (threadIdx.x % kWave == 0) slot[threadIdx.x / kWave] = v;
    __syncthreads();
    v = 0.0f;
#pragma unroll
    for (int w = 0; w < WAVES; ++w) v += slot[w];
  }
  return v;
}

// A row by WAVES waves, a lane holding NV chunks of 8 columns; rows of narrow
// models go to single waves, four rows a workgroup and no barrier.
template <int WAVES, int NV, typename T>
__global__ __launch_bounds__(256) void norm_residual_kernel(NormArgs a) {
  constexpr int kLanes = WAVES * kWave, kRows = 256 / kLanes;
  __shared__ float sums[2][WAVES];
  const int row = blockIdx.x * kRows + (WAVES == 1 ? (int)threadIdx.x / kWave : 0);
  if (row >= a.rows) return;
  const int lane = threadIdx.x % kLanes;
  float h[NV][8], y[NV][8];
  float ss = 0.0f;
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const int c = (i * kLanes + lane) * 8;
#pragma unroll
    for (int e = 0; e < 8; ++e) h[i][e] = y[i][e] = 0.0f;
    if (c < a.d) {
      load8(a.h + row * a.h_stride + c, h[i]);
      if (a.y) load8(static_cast<const T *>(a.y) + row * a.y_stride + c, y[i]);
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) ss = fmaf(y[i][e], y[i][e], ss);
  }
  float inv = 1.0f;
  if (a.post) inv = 1.0f / sqrtf(group_sum<WAVES>(ss, sums[0]) / (float)a.d + a.eps);
  ss = 0.0f;
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const int c = (i * kLanes + lane) * 8;
    if (c < a.d) {
      float post[8], gate[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) post[e] = gate[e] = 1.0f;
      if (a.post) load8(a.post + c, post);
      if (a.gate) load8(a.gate + row * a.gate_stride + c, gate);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        h[i][e] = fmaf(gate[e], y[i][e] * inv * post[e], a.residual_scale * h[i][e]);
        ss = fmaf(h[i][e], h[i][e], ss);
      }
      if (a.h_out) store8(a.h_out + row * a.h_out_stride + c, h[i]);
    }
  }
  if (!a.x_out) return;
  inv = 1.0f / sqrtf(group_sum<WAVES>(ss, sums[1]) / (float)a.d + a.eps);
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const int c = (i * kLanes + lane) * 8;
    if (c < a.d) {
      float pre[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) pre[e] = 1.0f;
      if (a.pre) load8(a.pre + c, pre);
#pragma unroll
      for (int e = 0; e < 8; ++e) h[i][e] *= inv * pre[e];
      store8(static_cast<T *>(a.x_out) + row * a.x_stride + c, h[i]);
    }
  }
}

template <int WAVES, int NV>
void launch(const NormArgs &a, bool f32, hipStream_t s) {
  const unsigned grid = (unsigned)norm_groups(a.rows, a.d);
  if (f32) hipLaunchKernelGGL((norm_residual_kernel<WAVES, NV, float>), dim3(grid), dim3(256), 0, s, a);
  else hipLaunchKernelGGL((norm_residual_kernel<WAVES, NV, uint16_t>), dim3(grid), dim3(256), 0, s, a);
}

}  // namespace

hipError_t launch_norm_residual(const NormArgs &a, bool f32, hipStream_t s) {
  if (a.d <= 512) launch<1, 1>(a, f32, s);
  else if (a.d <= kNormNarrow) launch<1, 2>(a, f32, s);
  else if (a.d <= 2048) launch<4, 1>(a, f32, s);
  else if (a.d <= 4096) launch<4, 2>(a, f32, s);
  else if (a.d <= 8192) launch<4, 4>(a, f32, s);
  else launch<4, 8>(a, f32, s);
  return hipGetLastError();
}

}  // namespace moe
