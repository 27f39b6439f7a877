// Products with 4-bit weights: y[t][n] = sum_c x[t][c] W[n][c].
//
// W [n x k] (k a multiple of 64) is three planes back to back: codes [n][k/2]
// bytes (column c in nibble c % 2 of byte c / 2), fp16 scales [n][k/64] and
// uint8 zero codes [n][k/64]; weight = (q - zero / 16) * scale.
#include "common.hpp"

#include <type_traits>

namespace moe {
namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float floatx4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef float floatx16 __attribute__((ext_vector_type(16)));

// Stores a result; one that is not finite, from an infinity in x or past
// fp32's range, is NaN whichever kernel computed it.
template <typename T>
__device__ __forceinline__ void store_result(T *out, float v) {
  v = fmaf(v, 0.0f, v);
  if constexpr (sizeof(T) == 4) *out = v;
  else *out = (uint16_t)bf16_pair(v, 0.0f);
}

// Few rows of x.  A workgroup owns 16 weight rows and 16 * MT rows of x; its
// eight waves share out the groups of 64 columns and add their results through
// LDS.  A lane holds a quarter of a weight row's group, 16 codes, the operand
// of two matrix instructions whose sum over k spans one group; so the scale and
// the zero are applied to sums in fp32 and the codes enter exactly: bits
// 0x4180 | q << 3 are the bf16 number 16 + q, and
//   sum (q - z) x = sum (16 + q) x - (16 + z) sum x,
// the sum of x coming from one more matrix instruction against ones.  The two
// sums are several times their difference, and so is their rounding: single fp32
// tokens come out 2 to 4e-7 off fp64 (relative, all elements), 2e-7 with weights
// multiplied out in fp32.  x in fp32 is three bf16 numbers that add up to it, a
// matrix instruction each.
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

// Sixteen elements of x in that order, eight by eight, as PARTS bf16 numbers each.
__device__ __forceinline__ void load_x(const uint16_t *p, u32x4 (&raw)[2]) {
  raw[0] = reinterpret_cast<const u32x4 *>(p)[0], raw[1] = reinterpret_cast<const u32x4 *>(p)[1];
}
__device__ __forceinline__ void load_x(const float *p, u32x4 (&raw)[4]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) raw[i] = reinterpret_cast<const u32x4 *>(p)[i];
}
__device__ __forceinline__ void split_x(const u32x4 (&raw)[2], bf16x8 (&out)[2][1]) {
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const u32x4 v = raw[h];
    const u32x4 o = {__builtin_amdgcn_perm(v[2], v[0], 0x05040100u), __builtin_amdgcn_perm(v[2], v[0], 0x07060302u),
                     __builtin_amdgcn_perm(v[3], v[1], 0x05040100u), __builtin_amdgcn_perm(v[3], v[1], 0x07060302u)};
    out[h][0] = __builtin_bit_cast(bf16x8, o);
  }
}
__device__ __forceinline__ void split_x(const u32x4 (&raw)[4], bf16x8 (&out)[2][3]) {
#pragma unroll
  for (int h = 0; h < 2; ++h)
#pragma unroll
    for (int e = 0; e < 8; e += 2) {
      float a = __uint_as_float(raw[2 * h][e / 2]), b = __uint_as_float(raw[2 * h + 1][e / 2]);  // elements e / 2 and 4 + e / 2
#pragma unroll
      for (int p = 0; p < 3; ++p) {
        out[h][p][e] = (__bf16)a, out[h][p][e + 1] = (__bf16)b;
        a -= (float)out[h][p][e], b -= (float)out[h][p][e + 1];
      }
    }
}

// Unsigned integers of CH fp16 scales and of CH zeros.
template <int CH> struct MetaWords;
template <> struct MetaWords<1> { typedef uint16_t S; typedef uint8_t Z; };
template <> struct MetaWords<2> { typedef uint32_t S; typedef uint16_t Z; };
template <> struct MetaWords<4> { typedef uint64_t S; typedef uint32_t Z; };

// A wave takes runs of CH groups: four (rows of a multiple of 256 columns) fill
// a line of a row's codes, whose four loads follow one another.  With single
// groups the waves ask for parts of the same lines at different times, 16 rows
// apart by a power of two where k is one: one token by 6144 x 4096 takes 14.5 us
// so, 9.4 with runs (by 6144 x 4160 9.6).  The next run's codes and the next
// group's x are on their way while a group is multiplied.  Two workgroups fit a
// compute unit for 16 rows (runs of two groups in fp32).
template <int MT, int CH, typename T>
__global__ __launch_bounds__(kSmallWaves * kWave, MT == 1 ? 4 : 2) void q4_small_kernel(Q4Args a) {
  constexpr int PARTS = sizeof(T) == 4 ? 3 : 1, kStep = kSmallWaves * CH;
  __shared__ float sums[kSmallWaves][MT][16][17];
  const int lane = threadIdx.x % kWave, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const int c = lane & 15, j = lane >> 4;
  const int n0 = blockIdx.x * 16, t0 = blockIdx.y * (16 * MT);
  const int row = min(n0 + c, a.n - 1), groups = a.k / 64;
  const uint8_t *codes = a.codes + (size_t)row * (a.k / 2) + 8 * j;
  const uint16_t *scales = reinterpret_cast<const uint16_t *>(a.scales) + (size_t)row * groups;
  const uint8_t *zeros = a.zeros + (size_t)row * groups;
  const T *x[MT];
#pragma unroll
  for (int m = 0; m < MT; ++m) x[m] = static_cast<const T *>(a.x) + min(t0 + 16 * m + c, a.rows - 1) * a.x_stride + 16 * j;
  bf16x8 ones;
#pragma unroll
  for (int e = 0; e < 8; ++e) ones[e] = (__bf16)1.0f;

  struct Run {
    uint2 w[CH];
    typename MetaWords<CH>::S s;
    typename MetaWords<CH>::Z z;
  };
  struct Rows {
    u32x4 x[MT][sizeof(T)];
  };
  auto fetch_run = [&](Run &r, int g) {
#pragma unroll
    for (int i = 0; i < CH; ++i) r.w[i] = *reinterpret_cast<const uint2 *>(codes + (size_t)(g + i) * 32);
    r.s = *reinterpret_cast<const decltype(r.s) *>(scales + g);
    r.z = *reinterpret_cast<const decltype(r.z) *>(zeros + g);
  };
  auto fetch_rows = [&](Rows &r, int g) {
#pragma unroll
    for (int m = 0; m < MT; ++m) load_x(x[m] + (size_t)g * 64, r.x[m]);
  };
  floatx4 y[MT] = {};
  auto multiply = [&](const Run &run, int i, const Rows &r) {
    const float scale = (float)__builtin_bit_cast(_Float16, (uint16_t)(run.s >> (16 * i)));
    const float zero = 16.0f + (float)(uint8_t)(run.z >> (8 * i)) * (1.0f / 16.0f);
    const bf16x8 q[2] = {codes_plus_16(run.w[i].x), codes_plus_16(run.w[i].y)};
#pragma unroll
    for (int m = 0; m < MT; ++m) {
      bf16x8 xs[2][PARTS];
      split_x(r.x[m], xs);
      floatx4 dot = {}, sum = {};
#pragma unroll
      for (int p = PARTS - 1; p >= 0; --p)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          dot = __builtin_amdgcn_mfma_f32_16x16x32_bf16(xs[h][p], q[h], dot, 0, 0, 0);
          sum = __builtin_amdgcn_mfma_f32_16x16x32_bf16(xs[h][p], ones, sum, 0, 0, 0);
        }
#pragma unroll
      for (int e = 0; e < 4; ++e) y[m][e] = fmaf(scale, fmaf(-zero, sum[e], dot[e]), y[m][e]);
    }
  };
  // One run, `next` its successor's first group; with MORE that one is fetched.
  // Group i's x is in rows[(FIRST + i) % 2].
  Run run[2];
  Rows rows[2];
  auto step = [&](const Run &now, Run &after, int g, auto more, auto first) {
#pragma unroll
    for (int i = 0; i < CH; ++i) {
      constexpr int kFirst = decltype(first)::value;
      if (i + 1 < CH) fetch_rows(rows[(kFirst + i + 1) % 2], g + i + 1);
      else if (decltype(more)::value) fetch_rows(rows[(kFirst + CH) % 2], g + kStep);
      if (i == 0 && decltype(more)::value) fetch_run(after, g + kStep);
      multiply(now, i, rows[(kFirst + i) % 2]);
    }
  };
  typedef std::integral_constant<bool, true> Yes;
  typedef std::integral_constant<bool, false> No;
  typedef std::integral_constant<int, 0> Even;
  typedef std::integral_constant<int, CH % 2> Other;
  int g = wave * CH;
  if (g < groups) {
    fetch_run(run[0], g);
    fetch_rows(rows[0], g);
    for (;; g += 2 * kStep) {
      if (g + kStep >= groups) {
        step(run[0], run[1], g, No(), Even());
        break;
      }
      step(run[0], run[1], g, Yes(), Even());
      if (g + 2 * kStep >= groups) {
        step(run[1], run[0], g + kStep, No(), Other());
        break;
      }
      step(run[1], run[0], g + kStep, Yes(), Other());
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
    for (int i = 0; i < kSmallWaves; ++i) v += sums[i][m][r][o % 16];
    if (n < a.n && t < a.rows) {
      store_result(static_cast<T *>(a.y) + t * a.y_stride + n, v);
    }
  }
}

// Many rows of x: tiles of BM rows by 128 weight rows, a group of 64 columns a
// step.  Four waves, two by two, own BM / 2 rows by 64 each.  The step's
// weights are expanded once a workgroup, to the integers 16 q - zero (at most
// 8 bits and a sign: exact in bf16), and wait with the rows of x in LDS, 128
// bytes a row, 16-byte chunk c of row r at c ^ (r / 2 % 8) so that a fragment
// read touches every bank once.  The products of one group are summed by
// themselves and added to the result with the group's scale / 16, one fp32
// fused multiply-add an element and group.  The next step's bytes are on their
// way to registers while a step is multiplied; two LDS buffers, one barrier a
// step.  What bounds it is that expansion, LDS and products of a wave run mostly
// one after another: 2037 rows by 6144 x 4096 in bf16 take 143 us, 720 TFLOP/s,
// where a bf16 product of 8192 cubed reaches 1165.
constexpr int kTileN = 128;

// Sixteen codes as bf16 16 q - zero, in column order.
__device__ __forceinline__ void expand16(uint2 w, float zero, uint4 *out) {
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const uint32_t v = h ? w.y : w.x, even = v << 4 & 0xF0F0F0F0u, odd = v & 0xF0F0F0F0u;
    // two exact differences make a pair of bf16 from their upper halves
    auto pair = [&](float a, float c) {
      return __builtin_amdgcn_perm(__float_as_uint(c - zero), __float_as_uint(a - zero), 0x07060302u);
    };
    out[h] = make_uint4(pair(byte_to_f32<0>(even), byte_to_f32<0>(odd)), pair(byte_to_f32<1>(even), byte_to_f32<1>(odd)),
                        pair(byte_to_f32<2>(even), byte_to_f32<2>(odd)), pair(byte_to_f32<3>(even), byte_to_f32<3>(odd)));
  }
}

template <int BM, typename T>
__global__ __launch_bounds__(256, BM <= 128 && sizeof(T) == 2 ? 2 : 1) void q4_tile_kernel(Q4Args a, int m_blocks, int n_blocks) {
  constexpr int PARTS = sizeof(T) == 4 ? 3 : 1;
  constexpr int XB = BM * 128, BUF = PARTS * XB + kTileN * 128;  // bytes of a part of x, of a step
  constexpr int MI = BM / 64;          // 32-row blocks of a wave
  constexpr int NX = BM * 8 / 256;     // 16-byte chunks of bf16 that a thread stages
  constexpr int SROW = 18, ZROW = 20;  // a weight row's 16 scales (of 18 halves) and zeros (of 20 bytes): rows on different banks
  __shared__ __align__(16) uint8_t lds[2 * BUF];
  __shared__ __align__(16) _Float16 lds_s[2][kTileN * SROW];
  __shared__ __align__(16) uint8_t lds_z[2][kTileN * ZROW];
  const int tid = threadIdx.x, lane = tid % kWave, wave = __builtin_amdgcn_readfirstlane(tid / kWave);
  // Runs of tiles to each XCD (workgroup i is on XCD i % 8), row blocks
  // fastest, so that an XCD's L2 sees few weights.
  const int tiles = m_blocks * n_blocks, per = tiles / 8, extra = tiles % 8;
  const int xcd = blockIdx.x % 8, tile = xcd * per + min(xcd, extra) + blockIdx.x / 8;
  const int t0 = tile % m_blocks * BM, n0 = tile / m_blocks * kTileN;
  const int groups = a.k / 64;

  // what this thread stages: chunk tid % 8 of rows tid / 8 + 32 i of x, half a group of weight row tid / 2
  const T *xp[NX];
#pragma unroll
  for (int i = 0; i < NX; ++i) xp[i] = static_cast<const T *>(a.x) + min(t0 + tid / 8 + 32 * i, a.rows - 1) * a.x_stride + tid % 8 * 8;
  const int wrow = min(n0 + tid / 2, a.n - 1);
  const uint8_t *wp = a.codes + (size_t)wrow * (a.k / 2) + tid % 2 * 16;
  const uint8_t *zp = a.zeros + (size_t)wrow * groups;
  const uint16_t *sp = reinterpret_cast<const uint16_t *>(a.scales) + (size_t)wrow * groups;
  const uint32_t x_at = tid / 8 * 128 + ((tid % 8 ^ (tid / 16 & 7)) << 4);  // rows 32 i further: + 4096 i
  const int wm = wave / 2, wn = wave % 2, r32 = lane & 31, hi = lane >> 5;

  u32x4 xr[NX][sizeof(T) / 2], wc[4], wn4[4], sr;
  u32x2 zr;
  auto fetch_x = [&](int g) {
#pragma unroll
    for (int i = 0; i < NX; ++i)
#pragma unroll
      for (int h = 0; h < (int)sizeof(T) / 2; ++h) xr[i][h] = reinterpret_cast<const u32x4 *>(xp[i] + g * 64)[h];
  };
  // Codes of four groups at a time: they share a line.
  auto fetch_w = [&](u32x4 *w, int g) {
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = *reinterpret_cast<const u32x4 *>(wp + (size_t)min(g + i, groups - 1) * 32);
  };
  // Scales and zeros of sixteen groups, eight a thread; one by one where rows are not multiples of eight groups.
  auto fetch_meta = [&](int g) {
    g += tid % 2 * 8;
    if (groups % 8 == 0) {
      g = min(g, groups - 8);
      sr = *reinterpret_cast<const u32x4 *>(sp + g);
      zr = *reinterpret_cast<const u32x2 *>(zp + g);
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) sr[i] = (uint32_t)sp[min(g + 2 * i, groups - 1)] | (uint32_t)sp[min(g + 2 * i + 1, groups - 1)] << 16;
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        zr[i] = 0;
#pragma unroll
        for (int b = 0; b < 4; ++b) zr[i] |= (uint32_t)zp[min(g + 4 * i + b, groups - 1)] << (8 * b);
      }
    }
  };
  auto stage_meta = [&](int chunk) {
    uint32_t *s = reinterpret_cast<uint32_t *>(&lds_s[chunk & 1][tid / 2 * SROW + tid % 2 * 8]);
    uint32_t *z = reinterpret_cast<uint32_t *>(&lds_z[chunk & 1][tid / 2 * ZROW + tid % 2 * 8]);
#pragma unroll
    for (int i = 0; i < 4; ++i) s[i] = sr[i];
    z[0] = zr[0], z[1] = zr[1];
  };
  auto stage = [&](int g, u32x4 codes) {
    uint8_t *to = lds + (g & 1) * BUF;
#pragma unroll
    for (int i = 0; i < NX; ++i) {
      if constexpr (PARTS == 1) {
        *reinterpret_cast<u32x4 *>(to + x_at + i * 4096) = xr[i][0];
      } else {
        float f[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) f[e] = __uint_as_float(xr[i][e / 4][e % 4]);
#pragma unroll
        for (int p = 0; p < PARTS; ++p) {
          uint4 v;
          v.x = bf16_pair(f[0], f[1]), v.y = bf16_pair(f[2], f[3]), v.z = bf16_pair(f[4], f[5]), v.w = bf16_pair(f[6], f[7]);
          *reinterpret_cast<uint4 *>(to + p * XB + x_at + i * 4096) = v;
          if (p + 1 < PARTS) {
            float b[8];
            bf16x8_to_f32(v, b);
#pragma unroll
            for (int e = 0; e < 8; ++e) f[e] -= b[e];
          }
        }
      }
    }
    const float zero = (float)lds_z[g / 16 & 1][tid / 2 * ZROW + g % 16];
    uint4 v[4];
    expand16(make_uint2(codes[0], codes[1]), zero, v);
    expand16(make_uint2(codes[2], codes[3]), zero, v + 2);
#pragma unroll
    for (int c = 0; c < 4; ++c)
      *reinterpret_cast<uint4 *>(to + PARTS * XB + tid / 2 * 128 + (((tid % 2 * 4 + c) ^ (tid / 4 & 7)) << 4)) = v[c];
  };

  floatx16 y[MI][2];
#pragma unroll
  for (int m = 0; m < MI; ++m)
#pragma unroll
    for (int j = 0; j < 2; ++j)
#pragma unroll
      for (int i = 0; i < 16; ++i) y[m][j][i] = 0.0f;

  fetch_meta(0);
  fetch_x(0);
  fetch_w(wc, 0);
  stage_meta(0);
  __syncthreads();
  stage(0, wc[0]);
  fetch_x(min(1, groups - 1));
  __syncthreads();
  const uint32_t sw = (r32 >> 1) & 7;
  for (int g0 = 0; g0 < groups; g0 += 4) {
    if (g0 % 16 == 0) fetch_meta(g0 + 16);
    if (g0 % 16 == 8) stage_meta(g0 / 16 + 1);
    fetch_w(wn4, g0 + 4);
#pragma unroll
    for (int step = 0; step < 4; ++step) {
      const int g = g0 + step;
      if (g >= groups) break;
      const uint8_t *from = lds + (g & 1) * BUF;
      float scale[2];
#pragma unroll
      for (int j = 0; j < 2; ++j) scale[j] = (float)lds_s[g / 16 & 1][(wn * 64 + j * 32 + r32) * SROW + g % 16] * 0.0625f;
      bf16x8 w[2][4];
#pragma unroll
      for (int j = 0; j < 2; ++j)
#pragma unroll
        for (int c = 0; c < 4; ++c)
          w[j][c] = *reinterpret_cast<const bf16x8 *>(from + PARTS * XB + (wn * 64 + j * 32 + r32) * 128 + (((2 * c + hi) ^ sw) << 4));
      stage(g + 1, step < 3 ? wc[(step + 1) % 4] : wn4[0]);
      fetch_x(min(g + 2, groups - 1));
#pragma unroll
      for (int m = 0; m < MI; ++m) {
        floatx16 d[2];
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
          for (int i = 0; i < 16; ++i) d[j][i] = 0.0f;
#pragma unroll
        for (int p = PARTS - 1; p >= 0; --p)
#pragma unroll
          for (int c = 0; c < 4; ++c) {
            const bf16x8 x = *reinterpret_cast<const bf16x8 *>(from + p * XB + (wm * (BM / 2) + m * 32 + r32) * 128 + (((2 * c + hi) ^ sw) << 4));
#pragma unroll
            for (int j = 0; j < 2; ++j) d[j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(x, w[j][c], d[j], 0, 0, 0);
          }
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
          for (int i = 0; i < 16; ++i) y[m][j][i] = fmaf(scale[j], d[j][i], y[m][j][i]);
      }
      __syncthreads();
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) wc[i] = wn4[i];
  }
#pragma unroll
  for (int m = 0; m < MI; ++m)
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const int n = n0 + wn * 64 + j * 32 + r32;
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const int t = t0 + wm * (BM / 2) + m * 32 + 8 * (i / 4) + 4 * hi + i % 4;
        if (n < a.n && t < a.rows) store_result(static_cast<T *>(a.y) + t * a.y_stride + n, y[m][j][i]);
      }
    }
}

template <int BM, typename T>
void launch_tile(const Q4Args &a, hipStream_t s) {
  const int mb = (a.rows + BM - 1) / BM, nb = (a.n + kTileN - 1) / kTileN;
  hipLaunchKernelGGL((q4_tile_kernel<BM, T>), dim3((unsigned)mb * nb), dim3(256), 0, s, a, mb, nb);
}

template <int MT, typename T>
void launch_small(const Q4Args &a, hipStream_t s) {
  const dim3 grid((a.n + 15) / 16, (a.rows + 16 * MT - 1) / (16 * MT)), block(kSmallWaves * kWave);
  // runs where rows of W are a multiple of them and give every wave one
  constexpr int CH = MT == 1 && sizeof(T) == 4 ? 2 : 4;
  if (a.k % (64 * CH) == 0 && a.k >= 64 * CH * kSmallWaves) hipLaunchKernelGGL((q4_small_kernel<MT, CH, T>), grid, block, 0, s, a);
  else hipLaunchKernelGGL((q4_small_kernel<MT, 1, T>), grid, block, 0, s, a);
}

// Estimated times (us) on the 256 compute units, each with `load` workgroups of
// a launch one after another (two at a time for tiles of bf16).  Measured, us
// small 16 / 32 / 64 rows a workgroup, tiles of 64 / 128 rows, and the choice:
//   bf16, 6144 x 4096,   17 rows:  18.0  17.0  21.0  48.4  60.0   16
//                        64:       39.4  32.4  36.5  49.5  60.7   32
//                       128:       75.9  63.1  54.0  49.7  60.7   64-row tiles
//                       384:      221   186   159    63.7  61.0   128-row tiles
//   bf16, 4096 x 14336,  64:       85.3  68.6  59.3  170   200    64
//                       200:      266   223   202   170   200     64-row tiles
//   bf16, 513 x 8192,   128:       27.1  21.2  35.3  94.3  115    32
//   bf16, 512 x 512,    512:        6.5   4.8   4.7   9.3  11.7   64
//   f32,  2048 x 2048,   48:       13.2  11.0    -   42.1  71.4   32
//                       512:       88.4  75.3    -   44.7  72.2   64-row tiles
//   f32,  9225 x 704,    32:       11.1  13.2    -   18.4  29.3   32
// Over 60 drawn shapes, 64 to 16384 by 128 to 14000 of 16 to 2048 rows, the choice
// took at most 10% more than the best of the five, the last line's 20% apart.
constexpr float kNever = 1e30f;
struct Cost {
  float first, pair;  // us a column (small) or a step of 64 columns (tiles): one workgroup, two at a time
};
float small_cost(const Q4Args &a, int mt, float column) {
  const int64_t wgs = (int64_t)((a.n + 15) / 16) * ((a.rows + 16 * mt - 1) / (16 * mt));
  return 2.0f + column * (float)a.k * (float)((wgs + 255) / 256);
}
float tile_cost(const Q4Args &a, int bm, Cost c) {
  const int64_t load = ((int64_t)((a.n + kTileN - 1) / kTileN) * ((a.rows + bm - 1) / bm) + 255) / 256;
  return 3.0f + (float)(a.k / 64) * ((float)(load / 2) * c.pair + (float)(load % 2) * c.first);
}

}  // namespace

hipError_t launch_q4_matmul(const Q4Args &a, bool f32, hipStream_t s) {
  const float cost[5] = {small_cost(a, 1, f32 ? 2.8e-3f : 1.6e-3f), small_cost(a, 2, f32 ? 4.4e-3f : 2.5e-3f),
                         f32 ? kNever : small_cost(a, 4, 4.25e-3f), tile_cost(a, 64, f32 ? Cost{1.27f, 2.54f} : Cost{0.77f, 1.0f}),
                         tile_cost(a, 128, f32 ? Cost{2.17f, 4.34f} : Cost{0.93f, 1.31f})};
  int best = 0;
  for (int i = 1; i < 5; ++i)
    if (cost[i] < cost[best]) best = i;
  switch (best) {
    case 0: f32 ? launch_small<1, float>(a, s) : launch_small<1, uint16_t>(a, s); break;
    case 1: f32 ? launch_small<2, float>(a, s) : launch_small<2, uint16_t>(a, s); break;
    case 2: launch_small<4, uint16_t>(a, s); break;
    case 3: f32 ? launch_tile<64, float>(a, s) : launch_tile<64, uint16_t>(a, s); break;
    default: f32 ? launch_tile<128, float>(a, s) : launch_tile<128, uint16_t>(a, s);
  }
  return hipGetLastError();
}

}  // namespace moe
