// Attention over the 4-bit paged cache (kv4.hip has its layout):
//   o[t][h] = sum_j softmax_j(scale q[t][h] . k_j) v_j,
// j over the positions 0 .. p of t's sequence, p the position of t, or, of a tree
// of tokens, over the cached tokens and the new ones that t's bits name; a row
// without any gets zeros.
#include "kv4_attn.hpp"

namespace moe {
namespace {

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
// It reads the cache once.  Below HBM's rate it is held by the vector instructions
// that expand the cache (about 360 a wave and block) and by the latency of its
// loads, of which one block a wave is in flight: 32 sequences of up to 4096
// tokens, 91 MB, in 29 us (3.1 TB/s), vector lanes busy 61% of the kernel's time,
// and the splits, as many for every sequence, leave the shorter ones' waves idle;
// one of 131072, 151 MB, in 41 us with the join (3.7 TB/s), vector lanes busy 79%.
//
// A probability is rounded to fp16 in bf16 calls, up to 2^-10 of itself toward zero,
// where fp32 would need a second product: the row's sum counts the rounded ones,
// so only their differences reach the result, which then takes 2^-8 in bf16.  fp32
// calls hold q and the probabilities in 22 bits, two numbers each; a third would
// be half as many products again for bits that sums of fp32 lose.
//
// TREE: rows see the cached tokens and what their words of `seen` name.
template <int D, typename T, bool TREE>
__global__ __launch_bounds__(kThreads, sizeof(T) == 4 && D == 128 ? 3 : 4) void kv4_attention_kernel(KvAttnArgs a) {
  constexpr int PARTS = sizeof(T) == 4 ? 2 : 1;
  constexpr int KW = D / 32;   // words of codes of a lane's part of a key, steps of the dot product
  constexpr int NU = D / 16;   // output blocks of 16 dimensions
  __shared__ float s_o[kWaves][16][D + 4];
  __shared__ float s_ml[kWaves][16][2];
  const int lane = threadIdx.x % kWave;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const int r = lane & 15, j = lane >> 4;
  const Masks masks_ = masks();
  const Place where = place(a);
  const int b = where.seq, g = where.kv_head, split = where.split;
  const int group = a.heads / a.kv.kv_heads;
  const Seq seq = sequence(a, b, group);
  const size_t page_bytes = (size_t)(D * 9 / 8) << a.kv.page_log2;
  const uint32_t values = (uint32_t)(D / 2) << a.kv.page_log2, kmetas = 2 * values, vmetas = kmetas + ((uint32_t)(D / 16) << a.kv.page_log2);
  const ScalarInts table = scalar_ints(a.kv.page_table + b * a.kv.table_stride);
  const int page_mask = (1 << a.kv.page_log2) - 1;
  const float factor = exponent_factor(a.scale);

  for (int row0 = where.block * 16; row0 < seq.rows; row0 += a.row_blocks * 16) {
    const int row = min(row0 + r, seq.rows - 1);
    const int token = seq.start + row / group, head = g * group + row % group;
    const int last = min(seq.first + row / group, seq.held - 1);  // this row's last position
    const int least = TREE ? min(seq.first, seq.held) - 1 : min(seq.first + row0 / group, seq.held - 1);  // the last that all rows see
    const int end = TREE ? min(seq.first + seq.rows / group, seq.held)
                         : min(seq.first + (min(row0 + 15, seq.rows - 1)) / group, seq.held - 1) + 1;
    const uint32_t *mine = TREE ? a.seen + (int64_t)token * a.words : nullptr;

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
    const RowScale rs = row_scale(amax, a.scale);
    const float down = rs.down;
#pragma unroll
    for (int t = 0; t < KW; ++t)
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const int from = e / 2 + 4 * (e & 1);
        float v = f[t][from] * rs.up;
        q[0][t][e] = (_Float16)v;
        if constexpr (PARTS == 2) q[1][t][e] = (_Float16)(v - (float)q[0][t][e]);
      }

    float m = -__builtin_inff(), l = 0.0f;
    floatx4 o[NU] = {};
    // The bytes of a block, by halves of 16 tokens (whose page is the wave's):
    // of key `at + r` dimensions (D / 4) j .., of values `at + 4 j ..` the octet
    // of dimensions that the lane's output rows lie in.
    const int c = r;
    const uint32_t oct = D == 64 ? c & 7 : c;
    uint32_t kw[2][KW], km[2];
    u32x4 vw[2];
    u32x2 vm[2];
    bool held[2], next_held[2];
    int page[2];
    const uint32_t k_lane = r * (D / 2) + (D / 8) * j, km_lane = kmetas + r * (D / 16) + (D == 128 ? j : j / 2) * 2;
    const uint32_t v_lane = values + j * (2 * D) + oct * 16, vm_lane = vmetas + j * (D / 4) + oct / 4 * 8;
    auto find = [&](int t0) {
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int col = (t0 + 16 * h) >> a.kv.page_log2;
        page[h] = col < a.kv.table_cols ? table[col] : -1;
      }
    };
    auto record = [&](int h) {
      next_held[h] = page[h] >= 0 && page[h] < a.kv.pages;
      return a.kv.pool + ((size_t)(next_held[h] ? page[h] : 0) * a.kv.kv_heads + g) * page_bytes;
    };
    // Offsets stay 32 bits wide, added to scalar bases; widened ahead of the loop
    // they would take two registers each.
    auto here = [](uint32_t offset) {
      asm volatile("" : "+v"(offset));
      return offset;
    };
    auto fetch_keys = [&](int t0) {
      const uint32_t ko = here(k_lane), mo = here(km_lane);
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const uint8_t *rec = record(h);
        const uint32_t in = (t0 + 16 * h) & page_mask;
        const uint8_t *kp = rec + in * (D / 2) + ko;
        if constexpr (KW == 4) *reinterpret_cast<u32x4 *>(kw[h]) = *reinterpret_cast<const u32x4 *>(kp);
        else *reinterpret_cast<u32x2 *>(kw[h]) = *reinterpret_cast<const u32x2 *>(kp);
        km[h] = *reinterpret_cast<const uint16_t *>(rec + in * (D / 16) + mo);
      }
    };
    auto fetch_values = [&](int t0) {
      const uint32_t vo = here(v_lane), mo = here(vm_lane);
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const uint8_t *rec = record(h);
        const uint32_t in = (t0 + 16 * h) & page_mask;
        vw[h] = *reinterpret_cast<const u32x4 *>(rec + in * (D / 2) + vo);
        vm[h] = *reinterpret_cast<const u32x2 *>(rec + in * (D / 16) + mo);
      }
    };
    // D 64: lanes 8 .. 15 of a row take dimensions 4 .. 7 of their octet
    const uint32_t first_byte = pick_byte(D == 64 ? (c >> 3) * 2 : 0);
    const int step = a.splits * kWaves * kTile;
    int t0 = (split * kWaves + wave) * kTile;
    if (t0 < end) {
      find(t0);
      fetch_keys(t0);
      fetch_values(t0);
      find(t0 + step);
    }
    // Fetches past the end read some page again (no branch: behind one the wait
    // for the values would be for the next keys too).
    for (; t0 < end; t0 += step) {
      float s[2][4];
      held[0] = next_held[0], held[1] = next_held[1];
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const Pair pair = key_pair(km[h]);
        floatx4 acc = {};
#pragma unroll
        for (int t = 0; t < KW; ++t) {
          const half8 k = key_values(kw[h][t], pair, masks_);
#pragma unroll
          for (int p = PARTS - 1; p >= 0; --p) acc = __builtin_amdgcn_mfma_f32_16x16x32_f16(k, q[p][t], acc, 0, 0, 0);
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) s[h][i] = acc[i];
      }
      const bool whole = held[0] && held[1] && t0 + kTile - 1 <= least;
      uint32_t bits = ~0u;   // TREE: of this lane's tokens 4 j .. and 16 + 4 j .. of the block
      if (!whole) {
        if constexpr (TREE) bits = tree_bits(mine, a.words, t0 - seq.first) >> (4 * j);
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const int at = t0 + 16 * h + 4 * j + i;
            if (!held[h] || (TREE ? at >= end || !(bits >> (16 * h + i) & 1) : at > last)) s[h][i] = -__builtin_inff();
          }
      }
      fetch_keys(t0 + step);
      // softmax of the block
      float top = s[0][0];
#pragma unroll
      for (int i = 1; i < 8; ++i) top = fmaxf(top, s[i / 4][i % 4]);
      top = max_over_j(top);
      if (__builtin_amdgcn_ballot_w64((top - m) * down > Hold<PARTS>::slack)) {
        top = fmaxf(m, top);
        const float keep = m == -__builtin_inff() ? 0.0f : __builtin_amdgcn_exp2f((m - top) * down);
        m = top;
        l *= keep;
#pragma unroll
        for (int u = 0; u < NU; ++u) o[u] *= keep;
      }
      const float ref = m == -__builtin_inff() ? 0.0f : m;
      half8 p[PARTS];
#pragma unroll
      for (int i = 0; i < 8; i += 2) {
        const float v0 = power<PARTS>(s[i / 4][i % 4], ref, down), v1 = power<PARTS>(s[i / 4][i % 4 + 1], ref, down);
        add_pair<PARTS>(v0, v1, i, p, l);
      }
      // values: word of token e, dimension u in nibble u; tokens that no row of
      // the tile sees must not reach the products, whatever their bytes are
      uint32_t metas[4] = {vm[0][0], vm[0][1], vm[1][0], vm[1][1]};   // of two tokens each
      if (!whole) {
#pragma unroll
        for (int e = 0; e < 4; ++e) metas[e] = inside(metas[e], t0 + 16 * (e / 2) + 4 * j + 2 * (e % 2), held[e / 2] ? end : 0);
      }
      Pair pairs[4];
      const bool marked = value_pairs(metas, pairs);
#pragma unroll
      for (int bt = 0; bt < NU / 2; ++bt) {
        half8 v0, v1;
        value_byte(vw, first_byte + bt * 0x00010001u, pairs, masks_, v0, v1);
#pragma unroll
        for (int part = PARTS - 1; part >= 0; --part) {
          o[2 * bt] = __builtin_amdgcn_mfma_f32_16x16x32_f16(v0, p[part], o[2 * bt], 0, 0, 0);
          o[2 * bt + 1] = __builtin_amdgcn_mfma_f32_16x16x32_f16(v1, p[part], o[2 * bt + 1], 0, 0, 0);
        }
      }
      fetch_values(t0 + step);
      find(t0 + 2 * step);
      // A group marked as not stored counts as NaN for the rows that see it and
      // must not touch the others, which multiply it with a zero.  It took part
      // above with a finite scale; here the marked tokens that a row sees are
      // counted, for the dimensions of the group.
      if (__builtin_amdgcn_ballot_w64(marked)) {
        half8 mark, seen;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          mark[e] = (_Float16)((metas[e / 2] >> (16 * (e % 2) + 8) & 255) == 255 ? 1.0f : 0.0f);
          seen[e] = (_Float16)((TREE ? bits >> (16 * (e / 4) + e % 4) & 1 : t0 + 16 * (e / 4) + 4 * j + e % 4 <= last) ? 1.0f : 0.0f);
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
      s_ml[wave][r][0] = joined_max(m, unit(down, factor), l);
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
      // no sum: no tokens; one of NaN scores alone has no maximum.  A wave far
      // below the others counts all the same: its NaN times 0 is NaN.
      if (s_ml[w][orow][1] == 0.0f) continue;
      const float f = s_ml[w][orow][0] == -__builtin_inff() ? 1.0f : __builtin_amdgcn_exp2f((s_ml[w][orow][0] - top) * factor);
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
        const int64_t at = (int64_t)split * a.kv.tokens * a.heads + out_row;
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

// Rows of prompts: 128 rows a workgroup, 32 a wave, over tiles of 64 tokens.
//
// The workgroup expands a tile's keys and values once, into LDS and in the
// order of the operands, 16 bytes a lane, so that reads and writes go through
// the banks in lane order.  Scores are again transposed: a lane has a row's
// (lane % 32) scores of tokens 8 b + 4 (lane / 32) + 0 .. 3 of each block of 32,
// which is the operand of O^T = V^T P^T when its sum takes the tokens in that
// order.  Two tiles of LDS, one barrier a tile; the bytes of the tile after
// next are on their way to registers.
// Vector instructions (an exponential a score, the expansion) and matrix
// instructions run mostly one after another, busy 48% and 26% of the time: 2048
// new tokens of one sequence over 2048, and single ones of three others, 32 heads
// to 8, 103 GFLOP, in 166 us, 620 TFLOP/s.
constexpr int kPromptTile = 64, kPromptRows = 128;
template <int D, typename T, bool TREE>
__global__ __launch_bounds__(kThreads, sizeof(T) == 4 ? 1 : 2) void kv4_prompt_kernel(KvAttnArgs a) {
  constexpr int PARTS = sizeof(T) == 4 ? 2 : 1;
  constexpr int KS = D / 16;           // steps of a score's dot product
  constexpr int NB = D / 32;           // output blocks of 32 dimensions
  constexpr int KW = D / 32;           // words of a key that a thread expands
  constexpr int KB = 32 * D * 2;       // LDS bytes of 32 keys, or of 32 values
  __shared__ __align__(16) uint8_t s_kv[2][4 * KB];          // keys of both blocks, values of both
  __shared__ __align__(16) uint8_t s_mark[2][D / 32][kPromptTile];  // marks of value groups, where s_any says there are
  __shared__ __align__(16) uint32_t s_any[2][kWaves];        // bit 0: marks in the wave's share, bit 1: a page is missing
  const int lane = threadIdx.x % kWave;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const int r = lane & 31, hi = lane >> 5;
  const Masks masks_ = masks();
  const Place where = place(a);
  const int b = where.seq, g = where.kv_head, split = where.split;
  const int group = a.heads / a.kv.kv_heads;
  const Seq seq = sequence(a, b, group);
  const size_t page_bytes = (size_t)(D * 9 / 8) << a.kv.page_log2;
  const uint32_t values = (uint32_t)(D / 2) << a.kv.page_log2, kmetas = 2 * values, vmetas = kmetas + ((uint32_t)(D / 16) << a.kv.page_log2);
  const ScalarInts table = scalar_ints(a.kv.page_table + b * a.kv.table_stride);
  const int page_mask = (1 << a.kv.page_log2) - 1;
  const int stride = a.splits * kPromptTile;

  // the page of token `at`, and whether there is one
  auto page_of = [&](int at, bool &held) {
    const int col = at >> a.kv.page_log2;
    const int page = col < a.kv.table_cols ? table[col] : -1;
    held = page >= 0 && page < a.kv.pages;
    return a.kv.pool + ((size_t)(held ? page : 0) * a.kv.kv_heads + g) * page_bytes;
  };

  for (int block = where.block; block * kPromptRows < seq.rows; block += a.row_blocks) {
    const int wrow = block * kPromptRows + wave * 32;   // the wave's first row
    const int row = min(wrow + r, seq.rows - 1);
    const int token = seq.start + row / group, head = g * group + row % group;
    const int last = min(seq.first + row / group, seq.held - 1);
    const int wfirst = TREE ? min(seq.first, seq.held) - 1 : min(seq.first + min(wrow, seq.rows - 1) / group, seq.held - 1);
    const int all = min(seq.first + seq.rows / group, seq.held);   // TREE: where the sequence ends
    const int wend = wrow >= seq.rows ? 0 : TREE ? all : min(seq.first + min(wrow + 31, seq.rows - 1) / group, seq.held - 1) + 1;
    const int end = TREE ? all : min(seq.first + min(block * kPromptRows + kPromptRows - 1, seq.rows - 1) / group, seq.held - 1) + 1;
    const uint32_t *mine = TREE ? a.seen + (int64_t)token * a.words : nullptr;

    half8 q[PARTS][KS];
    const T *qp = static_cast<const T *>(a.q) + token * a.q_stride + head * D + 8 * hi;
    float amax = 0.0f;
#pragma unroll
    for (int t = 0; t < KS; ++t) {
      float f[8];
      load8(qp + 16 * t, f);
#pragma unroll
      for (int e = 0; e < 8; ++e) amax = fmaxf(amax, fabsf(f[e]));
    }
    const RowScale rs = row_scale(max_of_halves(amax), a.scale);
#pragma unroll
    for (int t = 0; t < KS; ++t) {
      float f[8];
      load8(qp + 16 * t, f);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float v = f[e / 2 + 4 * (e & 1)] * rs.up;
        q[0][t][e] = (_Float16)v;
        if constexpr (PARTS == 2) q[1][t][e] = (_Float16)(v - (float)q[0][t][e]);
      }
    }

    float m = -__builtin_inff(), l = 0.0f;
    floatx16 o[NB];
#pragma unroll
    for (int u = 0; u < NB; ++u)
#pragma unroll
      for (int i = 0; i < 16; ++i) o[u][i] = 0.0f;

    // A thread's share of a tile: words KW * (2 (wave / 2) + hi) .. of key
    // 32 (wave % 2) + r, and, of the 8 dimensions of octet r / (8 / NB), NB of
    // values 32 (wave % 2) + 16 (wave / 2) + 4 hi + 0 .. 3 and + 8.
    uint32_t kw[KW], km;
    u32x4 vw[2];
    u32x2 vm[2];
    bool v_held, both_held;
    auto fetch = [&](int t0) {
      const int sub = t0 + 32 * (wave & 1);
      bool h0, h1;
      const uint8_t *p0 = page_of(sub, h0), *p1 = page_of(sub + 16, h1);
      const uint8_t *rec = r < 16 ? p0 : p1;
      const uint32_t in = (sub + r) & page_mask, part = 2 * (wave >> 1) + hi;
      const uint8_t *kp = rec + in * (D / 2) + KW * 4 * part;
      if constexpr (KW == 4) *reinterpret_cast<u32x4 *>(kw) = *reinterpret_cast<const u32x4 *>(kp);
      else *reinterpret_cast<u32x2 *>(kw) = *reinterpret_cast<const u32x2 *>(kp);
      km = *reinterpret_cast<const uint16_t *>(rec + kmetas + in * (D / 16) + (D == 128 ? part : part / 2) * 2);
      const uint8_t *vrec = wave >> 1 ? p1 : p0;
      v_held = wave >> 1 ? h1 : h0;
      both_held = h0 && h1;
      const uint32_t quad = (((sub + 16 * (wave >> 1)) & page_mask) >> 2) + hi, oct = (uint32_t)r / (8 / NB);
#pragma unroll
      for (int x = 0; x < 2; ++x) {
        vw[x] = *reinterpret_cast<const u32x4 *>(vrec + values + (quad + 2 * x) * (2 * D) + oct * 16);
        vm[x] = *reinterpret_cast<const u32x2 *>(vrec + vmetas + (quad + 2 * x) * (D / 4) + oct / 4 * 8);
      }
    };
    auto stage = [&](int t0, int buf) {
      uint8_t *to = s_kv[buf];
      {
        const Pair pair = key_pair(km);
        const int w0 = KW * (2 * (wave >> 1) + hi);
#pragma unroll
        for (int x = 0; x < KW; ++x)
          *reinterpret_cast<half8 *>(to + (wave & 1) * KB + (w0 + x) * 512 + r * 16) = key_values(kw[x], pair, masks_);
      }
      // tokens that no row sees must not reach the products, whatever their bytes are
      uint32_t metas[4] = {vm[0][0], vm[0][1], vm[1][0], vm[1][1]};
      if (!v_held || t0 + kPromptTile > end) {
        const int tok = t0 + 32 * (wave & 1) + 16 * (wave >> 1) + 4 * hi;
#pragma unroll
        for (int e = 0; e < 4; ++e) metas[e] = inside(metas[e], tok + 8 * (e / 2) + 2 * (e % 2), v_held ? end : 0);
      }
      Pair pairs[4];
      const bool marked = value_pairs(metas, pairs);
      const uint32_t first_byte = pick_byte(r % (8 / NB) * (NB / 2));
#pragma unroll
      for (int bt = 0; bt < NB / 2; ++bt) {
        half8 v0, v1;
        value_byte(vw, first_byte + bt * 0x00010001u, pairs, masks_, v0, v1);
        uint8_t *at = to + 2 * KB + (wave & 1) * KB + (wave >> 1) * 1024 + lane * 16;
        *reinterpret_cast<half8 *>(at + (2 * bt) * 2048) = v0;
        *reinterpret_cast<half8 *>(at + (2 * bt + 1) * 2048) = v1;
      }
      const bool any = __builtin_amdgcn_ballot_w64(marked) != 0;
      if (lane == 0) s_any[buf][wave] = (any ? 1u : 0u) | (both_held ? 0u : 2u);
      if (any && r % 8 == 0) {   // a lane of each group of 32 dimensions (D 64: of each half)
        uint8_t *mp = &s_mark[buf][r / (8 / NB) / 4][32 * (wave & 1) + 16 * (wave >> 1) + 4 * hi];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const uint32_t two = metas[e];
          *reinterpret_cast<uint16_t *>(mp + 8 * (e / 2) + 2 * (e % 2)) = (uint16_t)((two >> 8 & 255) == 255 ? 1 : 0) | (uint16_t)(two >> 24 == 255 ? 256 : 0);
        }
      }
    };

    // the first pass only stages; t0 is then negative
    int t0 = (split - a.splits) * kPromptTile, buf = 1;
    if (t0 + stride < end) fetch(t0 + stride);
    for (; t0 < end; t0 += stride, buf ^= 1, __syncthreads()) {
      const uint8_t *from = s_kv[buf];
      if (t0 + stride < end) {
        stage(t0 + stride, buf ^ 1);
        if (t0 + 2 * stride < end) fetch(t0 + 2 * stride);
      }
      if (t0 < 0 || t0 >= wend) continue;
      __builtin_amdgcn_sched_barrier(0);   // staging's registers are free again before the scores take theirs
      // two chains of products, the operands of the next two steps on their way
      floatx16 s[2];
#pragma unroll
      for (int x = 0; x < 2; ++x)
#pragma unroll
        for (int i = 0; i < 16; ++i) s[x][i] = 0.0f;
      half8 k[3][2];
      auto keys = [&](int x, int t) { return *reinterpret_cast<const half8 *>(from + x * KB + t * 1024 + lane * 16); };
#pragma unroll
      for (int t = 0; t < 2; ++t) k[t][0] = keys(0, t), k[t][1] = keys(1, t);
#pragma unroll
      for (int t = 0; t < KS; ++t) {
        if (t + 2 < KS) k[(t + 2) % 3][0] = keys(0, t + 2), k[(t + 2) % 3][1] = keys(1, t + 2);
#pragma unroll
        for (int p = PARTS - 1; p >= 0; --p)
#pragma unroll
          for (int x = 0; x < 2; ++x) s[x] = __builtin_amdgcn_mfma_f32_32x32x16_f16(k[t % 3][x], q[p][t], s[x], 0, 0, 0);
      }
      // in this order: left to itself the compiler reads an operand, waits and multiplies
      __builtin_amdgcn_sched_group_barrier(0x100, 4, 0);   // reads of LDS
#pragma unroll
      for (int t = 0; t < KS; ++t) {
        __builtin_amdgcn_sched_group_barrier(0x008, 2 * PARTS, 0);   // matrix instructions
        if (t + 2 < KS) __builtin_amdgcn_sched_group_barrier(0x100, 2, 0);
      }
      __builtin_amdgcn_sched_barrier(0);
      const u32x4 any4 = *reinterpret_cast<const u32x4 *>(s_any[buf]);
      const uint32_t any = __builtin_amdgcn_readfirstlane(any4[0] | any4[1] | any4[2] | any4[3]);
      uint32_t bits[2] = {~0u, ~0u};   // TREE: of this lane's tokens of both blocks, shifted by 4 hi
      if (t0 + kPromptTile - 1 > wfirst || (any & 2)) {
        if constexpr (TREE) {
#pragma unroll
          for (int x = 0; x < 2; ++x) bits[x] = tree_bits(mine, a.words, t0 + 32 * x - seq.first) >> (4 * hi);
        }
#pragma unroll
        for (int x = 0; x < 4; ++x) {
          bool held;
          page_of(t0 + 16 * x, held);
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            const int at = t0 + 16 * x + 8 * (i / 4) + 4 * hi + i % 4;
            if ((TREE ? at >= end || !(bits[x / 2] >> (16 * (x % 2) + 8 * (i / 4) + i % 4) & 1) : at > last) || !held)
              s[x / 2][8 * (x % 2) + i] = -__builtin_inff();
          }
        }
      }
      float top = s[0][0];
#pragma unroll
      for (int i = 1; i < 32; ++i) top = fmaxf(top, s[i / 16][i % 16]);
      top = max_of_halves(top);
      if (__builtin_amdgcn_ballot_w64((top - m) * rs.down > Hold<PARTS>::slack)) {
        top = fmaxf(m, top);
        const float keep = m == -__builtin_inff() ? 0.0f : __builtin_amdgcn_exp2f((m - top) * rs.down);
        m = top;
        l *= keep;
#pragma unroll
        for (int u = 0; u < NB; ++u) o[u] *= keep;
      }
      const float ref = m == -__builtin_inff() ? 0.0f : m;
      // probabilities of the next 16 tokens ahead of the products of these
      half8 p[4][PARTS];
      auto weigh = [&](int part) {
#pragma unroll
        for (int e = 0; e < 8; e += 2)
          add_pair<PARTS>(power<PARTS>(s[part / 2][8 * (part % 2) + e], ref, rs.down), power<PARTS>(s[part / 2][8 * (part % 2) + e + 1], ref, rs.down), e,
                          p[part], l);
      };
      weigh(0);
#pragma unroll
      for (int part = 0; part < 4; ++part) {
        half8 v[NB];
#pragma unroll
        for (int u = 0; u < NB; ++u) v[u] = *reinterpret_cast<const half8 *>(from + 2 * KB + part / 2 * KB + u * 2048 + part % 2 * 1024 + lane * 16);
        if (part < 3) weigh(part + 1);
#pragma unroll
        for (int n = PARTS - 1; n >= 0; --n)
#pragma unroll
          for (int u = 0; u < NB; ++u) o[u] = __builtin_amdgcn_mfma_f32_32x32x16_f16(v[u], p[part][n], o[u], 0, 0, 0);
      }
      // Groups marked as not stored: counted for the rows that see them, as in
      // the kernel above.
      if (any & 1) {
        floatx16 count;
#pragma unroll
        for (int i = 0; i < 16; ++i) count[i] = 0.0f;
        const uint8_t *marks = s_mark[buf][r / (8 / NB) / 4];
#pragma unroll
        for (int x = 0; x < 4; ++x) {
          half8 mark, seen;
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            const int at = 16 * x + 8 * (e / 4) + 4 * hi + e % 4;
            mark[e] = (_Float16)(any4[x / 2 + 2 * (x % 2)] & 1 ? (float)marks[at] : 0.0f);
            seen[e] = (_Float16)((TREE ? bits[x / 2] >> (16 * (x % 2) + 8 * (e / 4) + e % 4) & 1 : t0 + at <= last) ? 1.0f : 0.0f);
          }
          count = __builtin_amdgcn_mfma_f32_32x32x16_f16(mark, seen, count, 0, 0, 0);
        }
#pragma unroll
        for (int u = 0; u < NB; ++u)
#pragma unroll
          for (int i = 0; i < 16; ++i) o[u][i] = count[i] > 0.0f ? __builtin_nanf("") : o[u][i];
      }
    }
    l = sum_of_halves(l);
    if (wrow + r >= seq.rows) continue;
    const int64_t at = (int64_t)split * a.kv.tokens * a.heads + (int64_t)token * a.heads + head;
    const float inv = a.splits > 1 ? 1.0f : l == 0.0f ? 0.0f : 1.0f / l;
#pragma unroll
    for (int x = 0; x < 4; ++x) {
      // block x of output rows: NB * 4 consecutive dimensions
      float f[4 * NB];
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int u = 0; u < NB; ++u) f[NB * i + u] = o[u][4 * x + i] * inv;
      const int dim = (8 * NB) * x + 4 * NB * hi;
#pragma unroll
      for (int e = 0; e < 4 * NB; e += 8) {
        if (a.splits > 1) store8(a.part + at * D + dim + e, f + e);
        else store8(static_cast<T *>(a.o) + token * a.o_stride + head * D + dim + e, f + e);
      }
    }
    if (a.splits > 1 && hi == 0) {
      a.ml[2 * at] = joined_max(m, unit(rs.down, exponent_factor(a.scale)), l);
      a.ml[2 * at + 1] = l;
    }
  }
}

// Joins the splits of a row.  With WIDE a workgroup has 32 dimensions of one row
// and its groups of 8 lanes share out the splits (few rows, many splits: one
// sequence of 131072 tokens, 128 splits, 5.5 us instead of 83); otherwise D / 4
// lanes take a row (100 tokens of a prompt, 16 splits, 8 us instead of 34).
template <int D, typename T, bool WIDE>
__global__ __launch_bounds__(kThreads) void kv4_join_kernel(KvAttnArgs a) {
  constexpr int kLanes = WIDE ? 8 : D / 4, kGroups = kThreads / kLanes;
  const int64_t rows = (int64_t)a.kv.tokens * a.heads;
  const int grp = threadIdx.x / kLanes, dim = threadIdx.x % kLanes * 4 + (WIDE ? blockIdx.x % (D / 32) * 32 : 0);
  const int64_t row = WIDE ? blockIdx.x / (D / 32) : (int64_t)blockIdx.x * kGroups + grp;
  if (row >= rows) return;
  const float factor = exponent_factor(a.scale);
  const float2 *ml = reinterpret_cast<const float2 *>(a.ml) + row;
  // four splits at a time, so that their loads go out together
  float top = -__builtin_inff(), total = 0.0f;
  float4 acc = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
  constexpr int kStep = WIDE ? kGroups : 1;
  for (int s0 = WIDE ? grp : 0; s0 < a.splits; s0 += 4 * kStep) {
    float2 v[4];
    float4 o[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int s = min(s0 + i * kStep, a.splits - 1);
      v[i] = ml[s * rows];
      o[i] = *reinterpret_cast<const float4 *>(a.part + (s * rows + row) * D + dim);
    }
    float most = top;
#pragma unroll
    for (int i = 0; i < 4; ++i) most = fmaxf(most, v[i].x);
    const float keep = top == most ? 1.0f : __builtin_amdgcn_exp2f((top - most) * factor);
    top = most;
    total *= keep;
    acc.x *= keep, acc.y *= keep, acc.z *= keep, acc.w *= keep;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      // a split without tokens has no sum (and left its outputs unwritten); one
      // of NaN scores alone has no maximum
      if (s0 + i * kStep >= a.splits || v[i].y == 0.0f) continue;
      const float f = v[i].x == top ? 1.0f : v[i].x == -__builtin_inff() ? 1.0f : __builtin_amdgcn_exp2f((v[i].x - top) * factor);
      total += v[i].y * f;
      acc.x += o[i].x * f, acc.y += o[i].y * f, acc.z += o[i].z * f, acc.w += o[i].w * f;
    }
  }
  if constexpr (WIDE) {
    __shared__ float4 s_acc[kGroups][kLanes];
    __shared__ float2 s_ml[kGroups];
    s_acc[grp][dim / 4 % kLanes] = acc;
    if (threadIdx.x % kLanes == 0) s_ml[grp] = make_float2(top, total);
    __syncthreads();
    if (grp) return;
#pragma unroll
    for (int i = 0; i < kGroups; ++i) top = fmaxf(top, s_ml[i].x);
    total = 0.0f;
    acc = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll 8
    for (int i = 0; i < kGroups; ++i) {
      const float2 v = s_ml[i];
      const float4 o = s_acc[i][dim / 4 % kLanes];
      if (v.y == 0.0f) continue;
      const float f = v.x == -__builtin_inff() ? 1.0f : __builtin_amdgcn_exp2f((v.x - top) * factor);
      total += v.y * f;
      acc.x += o.x * f, acc.y += o.y * f, acc.z += o.z * f, acc.w += o.w * f;
    }
  }
  const float inv = total == 0.0f ? 0.0f : 1.0f / total;
  T *out = static_cast<T *>(a.o) + row / a.heads * a.o_stride + row % a.heads * D + dim;
  if constexpr (sizeof(T) == 4) *reinterpret_cast<float4 *>(out) = make_float4(acc.x * inv, acc.y * inv, acc.z * inv, acc.w * inv);
  else *reinterpret_cast<uint2 *>(out) = make_uint2(bf16_pair(acc.x * inv, acc.y * inv), bf16_pair(acc.z * inv, acc.w * inv));
}

template <int D, typename T>
void join(const KvAttnArgs &a, hipStream_t s) {
  const int64_t rows = (int64_t)a.kv.tokens * a.heads;
  constexpr int kGroups = kThreads / (D / 4);
  if (a.splits >= 8 && rows * (D / 32) <= 1024) hipLaunchKernelGGL((kv4_join_kernel<D, T, true>), dim3((unsigned)(rows * (D / 32))), dim3(kThreads), 0, s, a);
  else hipLaunchKernelGGL((kv4_join_kernel<D, T, false>), dim3((unsigned)((rows + kGroups - 1) / kGroups)), dim3(kThreads), 0, s, a);
}

template <int D, typename T>
void launch(const KvAttnArgs &a, hipStream_t s) {
  const dim3 grid((unsigned)a.kv.seqs * a.kv.kv_heads * a.row_blocks * a.splits);
  if (a.prompt && a.seen) hipLaunchKernelGGL((kv4_prompt_kernel<D, T, true>), grid, dim3(kThreads), 0, s, a);
  else if (a.prompt) hipLaunchKernelGGL((kv4_prompt_kernel<D, T, false>), grid, dim3(kThreads), 0, s, a);
  else if (a.seen) hipLaunchKernelGGL((kv4_attention_kernel<D, T, true>), grid, dim3(kThreads), 0, s, a);
  else hipLaunchKernelGGL((kv4_attention_kernel<D, T, false>), grid, dim3(kThreads), 0, s, a);
  if (a.splits > 1) join<D, T>(a, s);
}

}  // namespace

// Rows in blocks of 16, or of 128 from 64 rows a sequence and kv head on.  Enough
// workgroups for four on each of the 256 compute units, two with large blocks,
// or again four from eight sequences on, whose lengths differ, as long as a split
// keeps 768 tokens.  us with two / with four, over 4096 tokens, 32 heads to 8:
//   new tokens of some sequences, single ones of the rest
//     256 of every second of 8, 24, 64    130 / 109   243 / 237   536 / 537
//     256 of every eighth of 8, 16, 24     48 / 50     87 / 78    135 / 103
//     32 of every eighth of 8, 16, 24      27 / 27     42 / 49     64 / 52
//   24 of every one of 8, 16, 24, 32, 64   44 / 44    61 / 76     96 / 93   101 / 112   176 / 196
//   a third of 11 with 32 over up to 23050, 32 heads to 4    154 / 115
// so that equal sequences can lose (640 workgroups take two rounds of 512) what
// unequal ones gain; without the 768 all of 8 with 24 take 56.  Below eight, 3 with
// up to 100 over 6000: 55 / 60.  What counts are
// blocks that can have rows: 215 tokens of one sequence of 28854 and single ones
// of seven others, 20 heads to 4, take 1145 us cut as 288 blocks and 171 as 68.
// No split has less than one block of 32 tokens a wave, or four tiles (512 tokens
// over 2048, 4 heads, fp32: 42 us with one, 30 with four, 36 with eight).  Short
// calls of up to 512 tokens are not split: what the second launch costs is more
// than it saves (32 heads, 300 tokens 9.0 us split, 7.4 not; 1023 tokens 12.1 and
// 12.8).
KvAttnShape kv4_attention_shape(int seqs, int kv_heads, int heads, int tokens, int max_new, int max_len) {
  KvAttnShape s;
  const int64_t rows = (int64_t)max_new * (heads / kv_heads);
  s.prompt = rows >= 64;
  const int per = s.prompt ? kPromptRows : 16, tile = s.prompt ? 4 * kPromptTile : kWaves * kTile;
  const int64_t full = (int64_t)tokens * (heads / kv_heads);   // rows, were they all of one sequence
  const int64_t blocks = ((rows < full ? rows : full) + per - 1) / per;
  const int64_t pairs = (int64_t)seqs * kv_heads, room = kMaxGroups / pairs;  // of a launch's workgroups
  s.row_blocks = (int)(blocks < 1 || room < 1 ? 1 : blocks > room ? room : blocks);
  // blocks with rows: no more than the batch's tokens fill, and one more a sequence
  const int64_t filled = full / per + seqs, all = (int64_t)seqs * s.row_blocks;
  const int64_t units = kv_heads * (filled < all ? filled : all), most = ((int64_t)max_len + tile - 1) / tile;
  int64_t n = (s.prompt ? 512 : 1024) / units;
  if (s.prompt && seqs >= 8) {  // finer, down to 768 tokens a split
    const int64_t fine = 1024 / units, longest = max_len / 768;
    const int64_t m = fine < longest ? fine : longest;
    n = m > n ? m : n;
  }
  n = n > most ? most : n;
  if (!s.prompt && max_len <= 512) n = 1;
  if ((int64_t)tokens * heads > 8 * kMaxGroups) n = 1;   // rows past a launch of the join (of hints far too small)
  s.splits = (int)(n < 1 ? 1 : n);
  return s;
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
