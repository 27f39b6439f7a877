// Products with 4-bit weights: y[t][n] = sum_c x[t][c] W[n][c].
//
// W [n x k] (k a multiple of 64) is three planes back to back: codes [n][k/2]
// bytes (column c in nibble c % 2 of byte c / 2), fp16 scales [n][k/64] and
// uint8 zero codes [n][k/64]; weight = (q - zero / 16) * scale.
#include "common.hpp"

namespace moe {
namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float floatx4 __attribute__((ext_vector_type(4)));

// Few rows of x.  A workgroup owns 16 weight rows and 16 * MT rows of x; its
// eight waves share out the groups of 64 columns and add their results through
// LDS.  A lane holds a quarter of a weight row's group, 16 codes, the operand
// of two matrix instructions whose sum over k spans one group; so the scale and
// the zero are applied to sums in fp32 and the codes enter exactly: bits
// 0x4180 | q << 3 are the bf16 number 16 + q, and
//   sum (q - z) x = sum (16 + q) x - (16 + z) sum x,
// the sum of x coming from one more matrix instruction against ones.  x in fp32
// is three bf16 numbers that add up to it, a matrix instruction each.
constexpr int kSmallWaves = 8;

// Elements 0 4 1 5 2 6 3 7 of eight codes, the order in which two at a time
// fall out of a word, as 16 + q.
__device__ __forceinline__ bf16x8 codes_plus_16(uint32_t w) {
  uint4 v;
  v.x = (w << 3 & 0x00780078u) | 0x41804180u;
  v.y = (w >> 1 & 0x00780078u) | 0x41804180u;
  v.z = (w >> 5 & 0x00780078u) | 0x41804180u;
  v.w = (w >> 9 & 0x00780078u) | 0x41804180u;
  return __builtin_bit_cast(bf16x8, v);
}

// Eight elements of x in that order as PARTS bf16 numbers each.
template <int PARTS>
__device__ __forceinline__ void split8(const float *f, bf16x8 *out) {
  float r[8] = {f[0], f[4], f[1], f[5], f[2], f[6], f[3], f[7]};
#pragma unroll
  for (int p = 0; p < PARTS; ++p)
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      out[p][e] = (__bf16)r[e];
      if (p + 1 < PARTS) r[e] -= (float)out[p][e];
    }
}

template <int MT, typename T>
__global__ __launch_bounds__(kSmallWaves * kWave) void q4_small_kernel(Q4Args a) {
  constexpr int PARTS = sizeof(T) == 4 ? 3 : 1;
  __shared__ float sums[kSmallWaves][MT][16][17];
  const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
  const int c = lane & 15, j = lane >> 4;
  const int n0 = blockIdx.x * 16, t0 = blockIdx.y * (16 * MT);
  const int row = min(n0 + c, a.n - 1), groups = a.k / 64;
  const uint8_t *codes = a.codes + (size_t)row * (a.k / 2) + 8 * j;
  const _Float16 *scales = reinterpret_cast<const _Float16 *>(a.scales) + (size_t)row * groups;
  const uint8_t *zeros = a.zeros + (size_t)row * groups;
  const T *x[MT];
#pragma unroll
  for (int m = 0; m < MT; ++m) x[m] = static_cast<const T *>(a.x) + min(t0 + 16 * m + c, a.rows - 1) * a.x_stride + 16 * j;
  bf16x8 ones;
#pragma unroll
  for (int e = 0; e < 8; ++e) ones[e] = (__bf16)1.0f;
  floatx4 y[MT] = {};
  for (int g = wave; g < groups; g += kSmallWaves) {
    const uint2 w = *reinterpret_cast<const uint2 *>(codes + (size_t)g * 32);
    const float scale = (float)scales[g], zero = 16.0f + (float)zeros[g] * (1.0f / 16.0f);
    const bf16x8 q0 = codes_plus_16(w.x), q1 = codes_plus_16(w.y);
#pragma unroll
    for (int m = 0; m < MT; ++m) {
      float f[16];
      load8(x[m] + (size_t)g * 64, f);
      load8(x[m] + (size_t)g * 64 + 8, f + 8);
      bf16x8 x0[PARTS], x1[PARTS];
      split8<PARTS>(f, x0);
      split8<PARTS>(f + 8, x1);
      floatx4 dot = {}, sum = {};
#pragma unroll
      for (int p = PARTS - 1; p >= 0; --p) {
        dot = __builtin_amdgcn_mfma_f32_16x16x32_bf16(x0[p], q0, dot, 0, 0, 0);
        sum = __builtin_amdgcn_mfma_f32_16x16x32_bf16(x0[p], ones, sum, 0, 0, 0);
        dot = __builtin_amdgcn_mfma_f32_16x16x32_bf16(x1[p], q1, dot, 0, 0, 0);
        sum = __builtin_amdgcn_mfma_f32_16x16x32_bf16(x1[p], ones, sum, 0, 0, 0);
      }
#pragma unroll
      for (int i = 0; i < 4; ++i) y[m][i] = fmaf(scale, fmaf(-zero, sum[i], dot[i]), y[m][i]);
    }
  }
#pragma unroll
  for (int m = 0; m < MT; ++m)
#pragma unroll
    for (int i = 0; i < 4; ++i) sums[wave][m][4 * j + i][c] = y[m][i];
  __syncthreads();
  for (int o = threadIdx.x; o < MT * 256; o += kSmallWaves * kWave) {
    const int m = o / 256, r = o / 16 % 16, n = n0 + o % 16, t = t0 + 16 * m + r;
    float v = 0.0f;
#pragma unroll
    for (int w = 0; w < kSmallWaves; ++w) v += sums[w][m][r][o % 16];
    if (n < a.n && t < a.rows) {
      T *out = static_cast<T *>(a.y) + t * a.y_stride + n;
      if constexpr (sizeof(T) == 4) *out = v;
      else *out = (uint16_t)bf16_pair(v, 0.0f);
    }
  }
}

template <int MT>
void launch_small(const Q4Args &a, bool f32, hipStream_t s) {
  const dim3 grid((a.n + 15) / 16, (a.rows + 16 * MT - 1) / (16 * MT));
  if (f32) hipLaunchKernelGGL((q4_small_kernel<MT, float>), grid, dim3(kSmallWaves * kWave), 0, s, a);
  else hipLaunchKernelGGL((q4_small_kernel<MT, uint16_t>), grid, dim3(kSmallWaves * kWave), 0, s, a);
}

}  // namespace

hipError_t launch_q4_matmul(const Q4Args &a, bool f32, hipStream_t s) {
  if (a.rows <= 16) launch_small<1>(a, f32, s);
  else launch_small<2>(a, f32, s);
  return hipGetLastError();
}

}  // namespace moe
