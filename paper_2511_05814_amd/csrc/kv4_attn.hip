// Attention over the 4-bit paged cache (kv4.hip has its layout):
//   o[t][h] = sum_j softmax_j(scale q[t][h] . k_j) v_j,
// j over the positions 0 .. p of t's sequence, p the position of t; a row
// without any gets zeros.
#include "common.hpp"

namespace moe {
namespace {

typedef _Float16 half8 __attribute__((ext_vector_type(8)));
typedef _Float16 half2v __attribute__((ext_vector_type(2)));
typedef float floatx4 __attribute__((ext_vector_type(4)));

constexpr int kThreads = 256;
constexpr int kWaves = kThreads / kWave;
constexpr int kTile = 32;           // tokens of a wave's step
constexpr float kLog2e = 1.44269504088896340736f;
constexpr float kPShift = 14.0f;    // probabilities are held times 2^14: fp16 keeps 2^-38 of the largest

// 2^(s - top) in that scale.  s - top is exact near the top, so that 2^14 is
// not passed even where a score's last place is worth more than 1.
__device__ __forceinline__ float power(float s, float top) {
#pragma clang fp contract(off)
  return __builtin_amdgcn_exp2f((s - top) + kPShift);
}
__device__ __forceinline__ float scaled(float dot, float down) {
#pragma clang fp contract(off)
  return dot * down;
}

// Codes of a word that lie 16 bits apart, as pairs of fp16 1024 + q (low
// nibbles) or 1024 + 16 q (high ones): 0x6400 is 1024, whose last place is 1.
__device__ __forceinline__ half2v low_nibbles(uint32_t w) { return __builtin_bit_cast(half2v, (w & 0x000F000Fu) | 0x64006400u); }
__device__ __forceinline__ half2v high_nibbles(uint32_t w) { return __builtin_bit_cast(half2v, (w & 0x00F000F0u) | 0x64006400u); }
__device__ __forceinline__ half2v both(float v) { return half2v{(_Float16)v, (_Float16)v}; }

// scale(k), which fp16 holds exactly; NaN for the mark of a group that could not be stored
__device__ __forceinline__ float meta_scale(uint32_t meta) {
  const uint32_t k = meta >> 8;
  return k == 255 ? __builtin_nanf("") : __uint_as_float((k + 848) << 20);
}

// Eight key codes as fp16 values, dimensions in the order 0 4 1 5 2 6 3 7.
// Every step is exact.
__device__ __forceinline__ half8 key_values(uint32_t w, half2v minus_low, half2v minus_high, half2v scale) {
  const half2v sixteenth = both(0.0625f);
  half2v v[4];
  v[0] = (low_nibbles(w) + minus_low) * scale;
  v[1] = __builtin_elementwise_fma(high_nibbles(w), sixteenth, minus_high) * scale;
  v[2] = (low_nibbles(w >> 8) + minus_low) * scale;
  v[3] = __builtin_elementwise_fma(high_nibbles(w >> 8), sixteenth, minus_high) * scale;
  return half8{v[0][0], v[0][1], v[1][0], v[1][1], v[2][0], v[2][1], v[3][0], v[3][1]};
}

__device__ __forceinline__ float max_over_j(float v) {
  v = fmaxf(v, __shfl_xor(v, 16, kWave));
  return fmaxf(v, __shfl_xor(v, 32, kWave));
}
__device__ __forceinline__ float sum_over_j(float v) {
  v += __shfl_xor(v, 16, kWave);
  return v + __shfl_xor(v, 32, kWave);
}

// What a workgroup needs to know of its sequence.
struct Seq {
  int start, rows;   // first new token; rows = new tokens * heads a kv head
  int first, held;   // position of the first new token; tokens that the table can name
};
__device__ __forceinline__ Seq sequence(const KvAttnArgs &a, int b, int group) {
  Seq s;
  s.start = min(max(a.kv.q_start[b], 0), a.kv.tokens);
  const int end = min(max(a.kv.q_start[b + 1], s.start), a.kv.tokens);
  const int len = max(a.kv.kv_len[b], 0);
  s.rows = (end - s.start) * group;
  s.first = len - (end - s.start);
  s.held = (int)min((int64_t)len, (int64_t)a.kv.table_cols << a.kv.page_log2);
  return s;
}

// One tile of 16 rows (a row is a new token and one of its heads that share a
// kv head) against every (4 * splits)-th block of 32 tokens, by one wave.
//
// Scores are computed transposed, S^T = K Q^T, so that a lane holds one row's
// scores of tokens 4 j .. 4 j + 3 of both halves of the block (row = lane % 16,
// j = lane / 16).  That is the operand layout of O^T = V^T P^T when its sum
// runs over the tokens in the same order: probabilities never leave their
// lanes, and the rows' maxima and sums rescale lane-locally.  Keys and values
// are exact in fp16; q (and p, in fp32 calls) is one fp16 number or, for fp32
// calls, the sum of two.
template <int D, typename T>
__global__ __launch_bounds__(kThreads) void kv4_attention_kernel(KvAttnArgs a) {
  constexpr int PARTS = sizeof(T) == 4 ? 2 : 1;
  constexpr int KW = D / 32;   // words of codes of a lane's part of a key, steps of the dot product
  constexpr int NU = D / 16;   // output blocks of 16 dimensions
  __shared__ float s_o[kWaves][16][D + 4];
  __shared__ float s_ml[kWaves][16][2];
  const int lane = threadIdx.x % kWave;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const int r = lane & 15, j = lane >> 4;
  const int b = blockIdx.x / a.kv.kv_heads, g = blockIdx.x % a.kv.kv_heads;
  const int group = a.heads / a.kv.kv_heads;
  const Seq seq = sequence(a, b, group);
  const size_t page_bytes = (size_t)(D * 9 / 8) << a.kv.page_log2;
  const int32_t *table = a.kv.page_table + b * a.kv.table_stride;
  const int page_mask = (1 << a.kv.page_log2) - 1;

  for (int row0 = blockIdx.y * 16; row0 < seq.rows; row0 += gridDim.y * 16) {
    const int row = min(row0 + r, seq.rows - 1);
    const int token = seq.start + row / group, head = g * group + row % group;
    const int last = min(seq.first + row / group, seq.held - 1);  // this row's last position
    const int end = min(seq.first + (min(row0 + 15, seq.rows - 1)) / group, seq.held - 1) + 1;

    // the row of q, scaled by a power of two to a largest value of 2^9 .. 2^10
    half8 q[PARTS][KW];
    float amax = 0.0f;
    const T *qp = static_cast<const T *>(a.q) + token * a.q_stride + head * D + (D / 4) * j;
    float f[KW][8];
#pragma unroll
    for (int t = 0; t < KW; ++t) {
      load8(qp + 8 * t, f[t]);
#pragma unroll
      for (int e = 0; e < 8; ++e) amax = fmaxf(amax, fabsf(f[t][e]));
    }
    amax = max_over_j(amax);
    const int exponent = min(max((int)(__float_as_uint(amax) >> 23) - 127, -110), 127);
    const float up = ldexpf(1.0f, 9 - exponent), down = a.scale * kLog2e * ldexpf(1.0f, exponent - 9);
#pragma unroll
    for (int t = 0; t < KW; ++t)
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const int from = e / 2 + 4 * (e & 1);
        float v = f[t][from] * up;
        q[0][t][e] = (_Float16)v;
        if constexpr (PARTS == 2) q[1][t][e] = (_Float16)(v - (float)q[0][t][e]);
      }

    float m = -__builtin_inff(), l = 0.0f;
    floatx4 o[NU] = {};
    for (int t0 = ((int)blockIdx.z * kWaves + wave) * kTile; t0 < end; t0 += a.splits * kWaves * kTile) {
      float s[2][4];
      uint32_t vw[2][4], vm[2][4];   // value words and metas of the lane's eight tokens
      const int c = r, oct = D == 64 ? c & 7 : c;
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int at = t0 + 16 * h, in_page = at & page_mask;
        int page = (at >> a.kv.page_log2) < a.kv.table_cols ? table[at >> a.kv.page_log2] : -1;
        page = __builtin_amdgcn_readfirstlane(page);
        const bool held = page >= 0 && page < a.kv.pages;
        const uint8_t *rec = a.kv.pool + ((size_t)(held ? page : 0) * a.kv.kv_heads + g) * page_bytes;
        const uint8_t *metas = rec + ((size_t)D << a.kv.page_log2);
        // keys: lane (r, j) has dimensions (D / 4) j .. of token at + r
        uint32_t kw[KW];
        const uint8_t *kp = rec + (size_t)(in_page + r) * (D / 2) + (D / 8) * j;
        if constexpr (KW == 4) *reinterpret_cast<uint4 *>(kw) = *reinterpret_cast<const uint4 *>(kp);
        else *reinterpret_cast<uint2 *>(kw) = *reinterpret_cast<const uint2 *>(kp);
        const uint32_t km = *reinterpret_cast<const uint16_t *>(metas + (in_page + r) * (D / 16) + (D == 128 ? j : j / 2) * 2);
        // values: lane (c, j) has dimensions 8 oct .. of tokens at + 4 j ..
        const int quad = (in_page >> 2) + j;
        *reinterpret_cast<uint4 *>(vw[h]) = *reinterpret_cast<const uint4 *>(
            rec + ((size_t)(D / 2) << a.kv.page_log2) + (size_t)quad * (2 * D) + oct * 16);
        const uint2 mm = *reinterpret_cast<const uint2 *>(metas + ((size_t)(D / 16) << a.kv.page_log2) + quad * (D / 4) + (oct / 4) * 8);
        vm[h][0] = mm.x & 0xFFFF, vm[h][1] = mm.x >> 16, vm[h][2] = mm.y & 0xFFFF, vm[h][3] = mm.y >> 16;

        const float z = (float)(km & 255);
        const half2v scale = both(meta_scale(km)), low = both(-1024.0f - z), high = both(-64.0f - z);
        floatx4 acc = {};
#pragma unroll
        for (int t = 0; t < KW; ++t) {
          const half8 k = key_values(kw[t], low, high, scale);
#pragma unroll
          for (int p = PARTS - 1; p >= 0; --p) acc = __builtin_amdgcn_mfma_f32_16x16x32_f16(k, q[p][t], acc, 0, 0, 0);
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) s[h][i] = held && at + 4 * j + i <= last ? scaled(acc[i], down) : -__builtin_inff();
        // tokens that no row of the tile sees must not reach the products, whatever their bytes are
#pragma unroll
        for (int i = 0; i < 4; ++i)
          if (!held || at + 4 * j + i >= end) vm[h][i] = 0;
      }
      // softmax of the block
      float top = s[0][0];
#pragma unroll
      for (int i = 1; i < 8; ++i) top = fmaxf(top, s[i / 4][i % 4]);
      top = fmaxf(m, max_over_j(top));
      const float ref = top == -__builtin_inff() ? 0.0f : top;
      const float keep = __builtin_amdgcn_exp2f(m - ref);
      m = top;
      half8 p[PARTS];
      float add = 0.0f;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float v = power(s[i / 4][i % 4], ref);
        p[0][i] = (_Float16)v;
        float used = (float)p[0][i];
        if constexpr (PARTS == 2) {
          p[1][i] = (_Float16)(v - used);
          used += (float)p[1][i];
        }
        add += used;
      }
      l = l * keep + add;
#pragma unroll
      for (int u = 0; u < NU; ++u) o[u] *= keep;
      // values: word of token e, dimension u in nibble u
      half2v scale[4], low[4], high[4];
      bool marked = false;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const uint32_t m0 = vm[e / 2][e % 2 * 2], m1 = vm[e / 2][e % 2 * 2 + 1];
        marked |= (m0 >> 8) == 255 || (m1 >> 8) == 255;
        scale[e] = half2v{(_Float16)__uint_as_float(((m0 >> 8) + 848) << 20), (_Float16)__uint_as_float(((m1 >> 8) + 848) << 20)};
        const half2v z = half2v{(_Float16)(float)(m0 & 255), (_Float16)(float)(m1 & 255)};
        low[e] = both(-1024.0f) - z;
        high[e] = both(-64.0f) - z;
      }
      const half2v sixteenth = both(0.0625f);
#pragma unroll
      for (int bt = 0; bt < NU / 2; ++bt) {
        half8 v0, v1;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          uint32_t w0 = vw[e / 2][e % 2 * 2], w1 = vw[e / 2][e % 2 * 2 + 1];
          if constexpr (D == 64) {  // lanes 8 .. 15 of a row take dimensions 4 .. 7
            w0 >>= (c >> 3) * 16;
            w1 >>= (c >> 3) * 16;
          }
          const uint32_t x = __builtin_amdgcn_perm(w1, w0, 0x0C000C00u | bt | (uint32_t)(4 + bt) << 16);
          const half2v a0 = (low_nibbles(x) + low[e]) * scale[e];
          const half2v a1 = __builtin_elementwise_fma(high_nibbles(x), sixteenth, high[e]) * scale[e];
          v0[2 * e] = a0[0], v0[2 * e + 1] = a0[1];
          v1[2 * e] = a1[0], v1[2 * e + 1] = a1[1];
        }
#pragma unroll
        for (int part = PARTS - 1; part >= 0; --part) {
          o[2 * bt] = __builtin_amdgcn_mfma_f32_16x16x32_f16(v0, p[part], o[2 * bt], 0, 0, 0);
          o[2 * bt + 1] = __builtin_amdgcn_mfma_f32_16x16x32_f16(v1, p[part], o[2 * bt + 1], 0, 0, 0);
        }
      }
      // A group marked as not stored counts as NaN for the rows that see it and
      // must not touch the others, which multiply it with a zero.  It took part
      // above with a finite scale; here the marked tokens that a row sees are
      // counted, for the dimensions of the group.
      if (__builtin_amdgcn_ballot_w64(marked)) {
        half8 mark, seen;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          mark[e] = (_Float16)((vm[e / 4][e % 4] >> 8) == 255 ? 1.0f : 0.0f);
          seen[e] = (_Float16)(t0 + 16 * (e / 4) + 4 * j + e % 4 <= last ? 1.0f : 0.0f);
        }
        floatx4 count = {};
        count = __builtin_amdgcn_mfma_f32_16x16x32_f16(mark, seen, count, 0, 0, 0);
#pragma unroll
        for (int u = 0; u < NU; ++u)
#pragma unroll
          for (int i = 0; i < 4; ++i) o[u][i] = count[i] > 0.0f ? __builtin_nanf("") : o[u][i];
      }
    }
    l = sum_over_j(l);

    // join the four waves: lane (r, j) has dimensions dim(i, u) of row r
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int cc = 4 * j + i, dim = D == 128 ? 8 * cc : 8 * (cc & 7) + 4 * (cc >> 3);
#pragma unroll
      for (int u = 0; u < NU; u += 4)
        *reinterpret_cast<float4 *>(&s_o[wave][r][dim + u]) = make_float4(o[u][i], o[u + 1][i], o[u + 2][i], o[u + 3][i]);
    }
    if (j == 0) {
      s_ml[wave][r][0] = m;
      s_ml[wave][r][1] = l;
    }
    __syncthreads();
    constexpr int kPer = 16 * D / kThreads;   // 8 or 4 dimensions a thread
    const int orow = threadIdx.x / (D / kPer), dim = threadIdx.x % (D / kPer) * kPer;
    float top = -__builtin_inff(), total = 0.0f, acc[kPer] = {};
#pragma unroll
    for (int w = 0; w < kWaves; ++w) top = fmaxf(top, s_ml[w][orow][0]);
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
      const float f = s_ml[w][orow][0] == -__builtin_inff() ? (s_ml[w][orow][1] == 0.0f ? 0.0f : 1.0f)
                                                             : __builtin_amdgcn_exp2f(s_ml[w][orow][0] - top);
      if (f == 0.0f) continue;
      total += s_ml[w][orow][1] * f;
#pragma unroll
      for (int e = 0; e < kPer; ++e) acc[e] += s_o[w][orow][dim + e] * f;
    }
    if (row0 + orow < seq.rows) {
      const int64_t out_row = (int64_t)(seq.start + (row0 + orow) / group) * a.heads + g * group + (row0 + orow) % group;
      if (a.splits == 1) {
        const float inv = total == 0.0f ? 0.0f : 1.0f / total;
        T *out = static_cast<T *>(a.o) + (int64_t)(seq.start + (row0 + orow) / group) * a.o_stride +
                 (g * group + (row0 + orow) % group) * D + dim;
#pragma unroll
        for (int e = 0; e < kPer; ++e) {
          if constexpr (sizeof(T) == 4) out[e] = acc[e] * inv;
          else out[e] = (uint16_t)bf16_pair(acc[e] * inv, 0.0f);
        }
      } else {
        const int64_t at = (int64_t)blockIdx.z * a.kv.tokens * a.heads + out_row;
#pragma unroll
        for (int e = 0; e < kPer; ++e) a.part[at * D + dim + e] = acc[e];
        if (dim == 0) {
          a.ml[2 * at] = top;
          a.ml[2 * at + 1] = total;
        }
      }
    }
    __syncthreads();
  }
}

// Joins the splits of a row; D / 4 lanes a row.
template <int D, typename T>
__global__ __launch_bounds__(kThreads) void kv4_join_kernel(KvAttnArgs a) {
  constexpr int kLanes = D / 4;
  const int64_t rows = (int64_t)a.kv.tokens * a.heads;
  const int64_t row = ((int64_t)blockIdx.x * kThreads + threadIdx.x) / kLanes;
  if (row >= rows) return;
  const int dim = threadIdx.x % kLanes * 4;
  float top = -__builtin_inff(), total = 0.0f;
  float4 acc = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
  for (int s = 0; s < a.splits; ++s) top = fmaxf(top, a.ml[2 * (s * rows + row)]);
  for (int s = 0; s < a.splits; ++s) {
    const float m = a.ml[2 * (s * rows + row)], l = a.ml[2 * (s * rows + row) + 1];
    if (m == -__builtin_inff() && l == 0.0f) continue;
    const float f = m == -__builtin_inff() ? 1.0f : __builtin_amdgcn_exp2f(m - top);
    const float4 o = *reinterpret_cast<const float4 *>(a.part + (s * rows + row) * D + dim);
    total += l * f;
    acc.x += o.x * f, acc.y += o.y * f, acc.z += o.z * f, acc.w += o.w * f;
  }
  const float inv = total == 0.0f ? 0.0f : 1.0f / total;
  T *out = static_cast<T *>(a.o) + row / a.heads * a.o_stride + row % a.heads * D + dim;
  if constexpr (sizeof(T) == 4) *reinterpret_cast<float4 *>(out) = make_float4(acc.x * inv, acc.y * inv, acc.z * inv, acc.w * inv);
  else *reinterpret_cast<uint2 *>(out) = make_uint2(bf16_pair(acc.x * inv, acc.y * inv), bf16_pair(acc.z * inv, acc.w * inv));
}

template <int D, typename T>
void launch(const KvAttnArgs &a, hipStream_t s) {
  const dim3 grid(a.kv.seqs * a.kv.kv_heads, a.row_blocks, a.splits);
  hipLaunchKernelGGL((kv4_attention_kernel<D, T>), grid, dim3(kThreads), 0, s, a);
  if (a.splits > 1) {
    const int64_t lanes = (int64_t)a.kv.tokens * a.heads * (D / 4);
    hipLaunchKernelGGL((kv4_join_kernel<D, T>), dim3((unsigned)((lanes + kThreads - 1) / kThreads)), dim3(kThreads), 0, s, a);
  }
}

}  // namespace

// Enough workgroups for four on each of the 256 compute units, none with less
// than one block of 32 tokens a wave.
void kv4_attention_shape(int seqs, int kv_heads, int heads, int max_new, int max_len, int *splits, int *row_blocks) {
  const int64_t rows = (int64_t)max_new * (heads / kv_heads);
  *row_blocks = (int)((rows + 15) / 16 < 1 ? 1 : (rows + 15) / 16 > 65535 ? 65535 : (rows + 15) / 16);
  const int64_t units = (int64_t)seqs * kv_heads * *row_blocks, most = ((int64_t)max_len + kWaves * kTile - 1) / (kWaves * kTile);
  int64_t n = 1024 / units;
  n = n > most ? most : n;
  *splits = (int)(n < 1 ? 1 : n);
}

hipError_t launch_kv4_attention(const KvAttnArgs &a, int head_dim, bool f32, hipStream_t s) {
  if (head_dim == 64) {
    if (f32) launch<64, float>(a, s);
    else launch<64, uint16_t>(a, s);
  } else {
    if (f32) launch<128, float>(a, s);
    else launch<128, uint16_t>(a, s);
  }
  return hipGetLastError();
}

}  // namespace moe
