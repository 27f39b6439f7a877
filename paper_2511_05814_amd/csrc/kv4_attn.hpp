// What the attention kernels over the 4-bit paged cache share: expansion of
// cache entries, scales of rows, softmax pieces, and the places of workgroups.
#pragma once
#include "common.hpp"

namespace moe {
namespace {

typedef _Float16 half8 __attribute__((ext_vector_type(8)));
typedef _Float16 half2v __attribute__((ext_vector_type(2)));
typedef float floatx4 __attribute__((ext_vector_type(4)));
typedef float floatx16 __attribute__((ext_vector_type(16)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

constexpr int kThreads = 256;
constexpr int kWaves = kThreads / kWave;
constexpr int kTile = 32;           // tokens of a wave's step
constexpr float kLog2e = 1.44269504088896340736f;

// Probabilities are held times 2^shift, relative to a row's reference score: its
// largest up to now, or one at most `slack` powers of two below it, so that sums
// are rescaled only now and then.  fp16 then keeps at least 2^-(24 + shift) of
// the largest and 2^(shift + slack) does not pass its range.  (fp32 calls, which
// hold a probability as two numbers, need the finer end.)
template <int PARTS> struct Hold { static constexpr float shift = 8.0f, slack = 7.0f; };
template <> struct Hold<2> { static constexpr float shift = 14.0f, slack = 1.0f; };

// 2^((dot - ref) down) in that scale.  The difference of dot products is exact
// near the reference, so that the range is kept even where the last place of a
// score is worth more than 1.
template <int PARTS>
__device__ __forceinline__ float power(float dot, float ref, float down) {
  return __builtin_amdgcn_exp2f(fmaf(dot - ref, down, Hold<PARTS>::shift));
}

// Codes of a word that lie 16 bits apart, as pairs of fp16 1024 + q (low
// nibbles) or 1024 + 16 q (high ones): 0x6400 is 1024, whose last place is 1.
// The constants live in registers, the masks in scalar ones, which one
// v_and_or_b32 can name together; as literals they take two instructions.
struct Masks {
  uint32_t low, high, magic;
};
__device__ __forceinline__ Masks masks() {
  Masks m = {0x000F000Fu, 0x00F000F0u, 0x64006400u};
  asm volatile("" : "+s"(m.low), "+s"(m.high), "+v"(m.magic));
  return m;
}
__device__ __forceinline__ half2v low_nibbles(uint32_t w, const Masks &m) { return __builtin_bit_cast(half2v, (w & m.low) | m.magic); }
__device__ __forceinline__ half2v high_nibbles(uint32_t w, const Masks &m) { return __builtin_bit_cast(half2v, (w & m.high) | m.magic); }
__device__ __forceinline__ half2v both(float v) { return half2v{(_Float16)v, (_Float16)v}; }

// Elements i and i + 1 of the operand p from two probabilities, as one fp16
// number each (rounded toward zero, in one instruction) or two that add up to
// it; adds what the operand holds to `sum`, so that the weights of a row add up
// to one and the rounding's bias cancels.
template <int PARTS>
__device__ __forceinline__ void add_pair(float v0, float v1, int i, half8 (&p)[PARTS], float &sum) {
  const half2v one = both(1.0f), h = __builtin_bit_cast(half2v, __builtin_amdgcn_cvt_pkrtz(v0, v1));
  p[0][i] = h[0], p[0][i + 1] = h[1];
  sum = __builtin_amdgcn_fdot2(h, one, sum, false);
  if constexpr (PARTS == 2) {
    const half2v rest = __builtin_bit_cast(half2v, __builtin_amdgcn_cvt_pkrtz(v0 - (float)h[0], v1 - (float)h[1]));
    p[1][i] = rest[0], p[1][i + 1] = rest[1];
    sum = __builtin_amdgcn_fdot2(rest, one, sum, false);
  }
}

// A row of q goes to fp16 times a power of two that brings its largest element
// to 2^9 .. 2^10 (and the sign of the scale).  Its dot products times unit(),
// exactly, are those of q and k (unless `down` stops at an end), and times `down`
// the exponents of 2.
struct RowScale {
  float up, down;
};
// |scale| log2(e), kept off zero so that a masked score is minus infinity in any scale
__device__ __forceinline__ float exponent_factor(float scale) { return fminf(fmaxf(fabsf(scale) * kLog2e, 0x1p-126f), 0x1p127f); }
// Scales below fp32's normal range count as zero: every score is 0.  Scores are
// below 2^32 (values below 2^15, up to 128 of them), so that `down` may stop at
// 2^-100: less makes every difference of exponents nothing all the same.
__device__ __forceinline__ RowScale row_scale(float amax, float scale) {
  const int exponent = min(max((int)(__float_as_uint(amax) >> 23) - 127, -116), 127);
  RowScale r;
  r.up = fabsf(scale) < 0x1p-126f ? 0.0f : copysignf(ldexpf(1.0f, 9 - exponent), scale);
  // A scale that is not finite makes every score that a row sees a NaN, and so
  // does an infinity in q: its scores are infinities or NaN, and where all of
  // them are minus infinity the row would pass for one that sees nothing.
  if (!(fabsf(scale) < __builtin_inff()) || amax == __builtin_inff()) r.up = __builtin_nanf("");
  r.down = fminf(fmaxf(exponent_factor(scale) * ldexpf(1.0f, exponent - 9), 0x1p-100f), 0x1p126f);
  return r;
}
// The power of two in `down`, from the exponents alone (a register less in loops).
__device__ __forceinline__ float unit(float down, float factor) {
  return __uint_as_float((__float_as_uint(down) & 0x7F800000u) - (__float_as_uint(factor) & 0x7F800000u) + 0x3F800000u);
}

// A row's largest dot product as the joins compare it.  Past fp32's range there is
// no telling parts of a row apart: the sum becomes a NaN.
__device__ __forceinline__ float joined_max(float m, float unit, float &l) {
  const float v = m * unit;
  if (fabsf(v) == __builtin_inff() && fabsf(m) < __builtin_inff()) l = __builtin_nanf("");
  return v;
}

// scale(k), which fp16 holds exactly; NaN for the mark of a group that could not be stored
__device__ __forceinline__ float meta_scale(uint32_t meta) {
  const uint32_t k = meta >> 8;
  return k == 255 ? __builtin_nanf("") : __uint_as_float((k + 848) << 20);
}

// What two metas (uint16 k << 8 | z each) turn codes into values with.
struct Pair {
  half2v scale, low, high;   // of 1024 + q: + low, times scale; of 1024 + 16 q: / 16 + high, times scale
};
typedef unsigned short ushort2v __attribute__((ext_vector_type(2)));
// For 8 <= k < 248, k << 7 are the bits of scale(k) * 2^6 in fp16.  `far` grows to
// 0x7800 or more in the half of a k outside that range (a step below 2^-20 or
// from 2^10 on, or a mark), for which far_pair has the scale.
__device__ __forceinline__ Pair pair_of(uint32_t two, ushort2v &far) {
  const uint32_t k = two >> 1 & 0x7F807F80u;
  far = __builtin_elementwise_max(far, (ushort2v)(__builtin_bit_cast(ushort2v, k) - (unsigned short)0x0400));
  Pair p;
  p.scale = __builtin_bit_cast(half2v, k) * both(0.015625f);
  p.low = __builtin_bit_cast(half2v, (two & 0x00FF00FFu) | 0xE400E400u);        // -(1024 + z)
  p.high = __builtin_bit_cast(half2v, (two << 4 & 0x0FF00FF0u) | 0xD400D400u);  // -(64 + z)
  return p;
}
__device__ __forceinline__ bool is_far(ushort2v far) { return far[0] >= 0x7800 || far[1] >= 0x7800; }
constexpr uint32_t kPlainMeta = 8u << 8;   // k = 8, z = 0

// Eight key codes as fp16 values, dimensions in the order 0 4 1 5 2 6 3 7.
// Every step is exact.
__device__ __forceinline__ half8 key_values(uint32_t w, const Pair &m, const Masks &k) {
  const half2v sixteenth = both(0.0625f);
  half2v v[4];
  v[0] = (low_nibbles(w, k) + m.low) * m.scale;
  v[1] = __builtin_elementwise_fma(high_nibbles(w, k), sixteenth, m.high) * m.scale;
  v[2] = (low_nibbles(w >> 8, k) + m.low) * m.scale;
  v[3] = __builtin_elementwise_fma(high_nibbles(w >> 8, k), sixteenth, m.high) * m.scale;
  return half8{v[0][0], v[0][1], v[1][0], v[1][1], v[2][0], v[2][1], v[3][0], v[3][1]};
}

// The meta of a key's group, for both halves of a pair; NaN where it is marked.
__device__ __forceinline__ Pair key_pair(uint32_t meta) {
  ushort2v far = {0, 0};
  Pair p = pair_of(meta | meta << 16, far);
  if (__builtin_amdgcn_ballot_w64(is_far(far)) != 0) p.scale = both(meta_scale(meta));
  return p;
}

// What four pairs of metas of a lane's eight value tokens say.  Returns whether
// one is marked as not stored; its values are finite all the same.
__device__ __forceinline__ bool value_pairs(const uint32_t (&two)[4], Pair (&p)[4]) {
  ushort2v far = {0, 0};
#pragma unroll
  for (int e = 0; e < 4; ++e) p[e] = pair_of(two[e], far);
  bool marked = false;
  if (__builtin_amdgcn_ballot_w64(is_far(far)) != 0) {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const uint32_t k0 = two[e] >> 8 & 255, k1 = two[e] >> 24;
      marked |= k0 == 255 || k1 == 255;
      p[e].scale = half2v{(_Float16)__uint_as_float((k0 + 848) << 20), (_Float16)__uint_as_float((k1 + 848) << 20)};
    }
  }
  return marked;
}

// Two dimensions (the nibbles of a byte) of eight tokens as fp16 values;
// `pick`: that byte of two tokens' words, each in a half.
__device__ __forceinline__ void value_byte(const u32x4 (&w)[2], uint32_t pick, const Pair (&p)[4], const Masks &k, half8 &v0, half8 &v1) {
  const half2v sixteenth = both(0.0625f);
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const uint32_t x = __builtin_amdgcn_perm(w[e / 2][e % 2 * 2 + 1], w[e / 2][e % 2 * 2], pick);
    const half2v a0 = (low_nibbles(x, k) + p[e].low) * p[e].scale;
    const half2v a1 = __builtin_elementwise_fma(high_nibbles(x, k), sixteenth, p[e].high) * p[e].scale;
    v0[2 * e] = a0[0], v0[2 * e + 1] = a0[1];
    v1[2 * e] = a1[0], v1[2 * e + 1] = a1[1];
  }
}
__device__ __forceinline__ uint32_t pick_byte(uint32_t b) { return 0x0C000C00u | b | (b + 4) << 16; }

// Metas of tokens at .. at + 1 that may lie at or past `end`, or on no page.
__device__ __forceinline__ uint32_t inside(uint32_t two, int at, int end) {
  if (at >= end) return kPlainMeta | kPlainMeta << 16;
  return at + 1 >= end ? (two & 0xFFFF) | kPlainMeta << 16 : two;
}

// The other operand of a reduction over lanes i and i ^ 32 (i ^ 16), without the
// LDS: the halves (the rows of 16 lanes) of a copy swapped.
__device__ __forceinline__ void swap32(float v, float &a, float &b) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  a = __uint_as_float(r[0]);
  b = __uint_as_float(r[1]);
}
__device__ __forceinline__ void swap16(float v, float &a, float &b) {
  const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  a = __uint_as_float(r[0]);
  b = __uint_as_float(r[1]);
}
// Over the two lanes of a row of 32, and the four of a row of 16.
__device__ __forceinline__ float max_of_halves(float v) {
  float a, b;
  swap32(v, a, b);
  return fmaxf(a, b);
}
__device__ __forceinline__ float sum_of_halves(float v) {
  float a, b;
  swap32(v, a, b);
  return a + b;
}
__device__ __forceinline__ float max_over_j(float v) {
  float a, b;
  swap16(v, a, b);
  return max_of_halves(fmaxf(a, b));
}
__device__ __forceinline__ float sum_over_j(float v) {
  float a, b;
  swap16(v, a, b);
  return sum_of_halves(a + b);
}

// A workgroup's split, kv head, sequence and block of rows, from a launch's one
// dimension.  Workgroups start in its order and go to the XCDs, and there to the
// four shader engines, in turn.  Short calls: splits first, so that every
// sequence is spread over all of them.  Prompts: blocks last and the later rows,
// which see most, first, so that the longest work starts first; the sequences of
// a block rotate with it, or one in four, long, would put all of its work on one
// engine of each XCD (2048 new tokens of one sequence over 2048 and single tokens
// of three others: 682 us so, 188 with the blocks of a sequence one after
// another, 183 as it is, all three before the products were reordered, since when
// it takes 166).
struct Place {
  int split, block, seq, kv_head;
};
__device__ __forceinline__ Place place(const KvAttnArgs &a) {
  Place p;
  uint32_t id = blockIdx.x;
  p.split = id % (uint32_t)a.splits;
  id /= (uint32_t)a.splits;
  if (a.prompt) {
    p.kv_head = id % (uint32_t)a.kv.kv_heads;
    id /= (uint32_t)a.kv.kv_heads;
    const uint32_t turn = id / (uint32_t)a.kv.seqs;
    p.seq = (id + turn) % (uint32_t)a.kv.seqs;
    p.block = a.row_blocks - 1 - (int)turn;
  } else {
    p.block = id % (uint32_t)a.row_blocks;
    id /= (uint32_t)a.row_blocks;
    p.kv_head = id % (uint32_t)a.kv.kv_heads;
    p.seq = id / (uint32_t)a.kv.kv_heads;
  }
  return p;
}

// Arrays that a launch only reads, at addresses that a wave agrees on: scalar
// loads, which wait for nothing but themselves.
typedef const int32_t __attribute__((address_space(4))) *ScalarInts;
__device__ __forceinline__ ScalarInts scalar_ints(const int32_t *p) { return (ScalarInts)(uintptr_t)p; }

// A row's view of the 32 tokens from `rel` places past the first new one on, as
// bits: tokens that were cached are seen by all, new ones where the row of
// `words` words says so.
__device__ __forceinline__ uint32_t tree_bits(const uint32_t *row, int words, int rel) {
  const int w = rel >> 5;
  const uint32_t lo = w < 0 ? ~0u : w < words ? row[w] : 0u, hi = w + 1 < 0 ? ~0u : w + 1 < words ? row[w + 1] : 0u;
  return __builtin_amdgcn_alignbit(hi, lo, rel & 31);
}

// What a workgroup needs to know of its sequence.
struct Seq {
  int start, rows;   // first new token; rows = new tokens * heads a kv head
  int first, held;   // position of the first new token; tokens that the table can name
};
__device__ __forceinline__ Seq sequence(const KvAttnArgs &a, int b, int group) {
  Seq s;
  const ScalarInts start = scalar_ints(a.kv.q_start) + b;
  s.start = min(max(start[0], 0), a.kv.tokens);
  const int end = min(max(start[1], s.start), a.kv.tokens);
  const int len = max(scalar_ints(a.kv.kv_len)[b], 0);
  s.rows = (end - s.start) * group;
  s.first = len - (end - s.start);
  s.held = (int)min((int64_t)len, (int64_t)a.kv.table_cols << a.kv.page_log2);
  return s;
}

}  // namespace
}  // namespace moe
