// Attention of trees of drafted tokens over the 4-bit paged cache: some tens of
// rows (new tokens times the heads that share a kv head) against long caches whose
// lengths differ.  Expanding a cache entry takes most of the vector instructions, so
// one expansion serves as many rows as there are; and workgroups take equal
// shares of all sequences' work, where a cut of every sequence into the same number of
// parts leaves most of the chip waiting for the longest (32 trees of 8 tokens
// over up to 4095: 48 us so, 37 here).
#include "kv4_attn.hpp"

namespace moe {
namespace {

// tree_bits of the block of 32 tokens at t0, without what lies at or past `end`
// or, by halves of 16 tokens, on no page.
__device__ __forceinline__ uint32_t block_bits(const uint32_t *row, int words, int t0, int first, int end, bool held0, bool held1) {
  uint32_t b = tree_bits(row, words, t0 - first);
  if (end - t0 < 32) b &= end > t0 ? (1u << (end - t0)) - 1 : 0u;
  if (!held0) b &= 0xFFFF0000u;
  if (!held1) b &= 0x0000FFFFu;
  return b;
}
__device__ __forceinline__ floatx4 all_four(float v) { return floatx4{v, v, v, v}; }
// 2^(score - reference), in the scale of Hold; `above` is the difference of the
// dot products, which the matrix cores have from their start at minus the
// reference.
template <int PARTS>
__device__ __forceinline__ float weight(float above, float down) {
  return __builtin_amdgcn_exp2f(fmaf(above, down, Hold<PARTS>::shift));
}
constexpr float kRange = 32768.0f;   // 2^(shift + slack): weights below it fit fp16
// Whether one of a lane's eight weights passes the range or is a NaN, or any is
// relative to no reference.  bf16 calls hold a weight at the reference as 2^8: eight of
// them stay far below the range, so their sum tells.  fp32 calls hold it as
// 2^14, of which two make the range already: the largest tells, and the sum a NaN.
template <int PARTS>
__device__ __forceinline__ bool out_of_range(float sum, float most) {
  if constexpr (PARTS == 1) return !(sum < kRange);
  return !(sum < 8 * kRange) || most >= kRange;
}

// Sums over a wave's lanes up to each.
template <int CTRL, int ROWS>
__device__ __forceinline__ int dpp_plus(int v) { return v + __builtin_amdgcn_update_dpp(0, v, CTRL, ROWS, 0xF, false); }
__device__ __forceinline__ int wave_scan(int v) {
  v = dpp_plus<0x111, 0xF>(v);  // row_shr:1
  v = dpp_plus<0x112, 0xF>(v);  // row_shr:2
  v = dpp_plus<0x114, 0xF>(v);  // row_shr:4
  v = dpp_plus<0x118, 0xF>(v);  // row_shr:8
  v = dpp_plus<0x142, 0xA>(v);  // row_bcast:15
  v = dpp_plus<0x143, 0xC>(v);  // row_bcast:31
  return v;
}

// A launch's work: units, each ROWS rows of a sequence and kv head, of as many
// steps as the sequence has STEP tokens, and AHEAD more for what it takes to begin
// and end one, all one behind the other.  Each of W workgroups takes as much of all
// T as the others (W is at most T), whatever the lengths are.  A unit that lies in
// several workgroups is joined afterwards: a workgroup has at most one whose first
// steps others have and one whose last ones others have, and a place for the rows
// of each.
constexpr int kMaxSeqs = 256;   // of a call; workgroups have no fewer threads
template <int ROWS, int STEP, int AHEAD>
struct Plan {
  int before[kMaxSeqs + 1];   // T of the sequences before each
  int start[kMaxSeqs], rows[kMaxSeqs], first[kMaxSeqs], held[kMaxSeqs];
  int sums[kMaxSeqs / kWave];

  static __device__ __forceinline__ int blocks_of(int rows) { return (rows + ROWS - 1) / ROWS; }
  // rows that see nothing have a step as well: it writes their zeros
  static __device__ __forceinline__ int steps_of(int rows, int first, int held, int group) {
    return max(1, (min(first + rows / group, held) + STEP - 1) / STEP);
  }
  // by the whole workgroup
  __device__ __forceinline__ void make(const KvAttnArgs &a, int group) {
    const int b = threadIdx.x, lane = b % kWave, wave = b / kWave;
    int mine = 0;
    if (b < a.kv.seqs) {
      const Seq s = sequence(a, b, group);
      start[b] = s.start, rows[b] = s.rows, first[b] = s.first, held[b] = s.held;
      mine = blocks_of(s.rows) * a.kv.kv_heads * (steps_of(s.rows, s.first, s.held, group) + AHEAD);
    }
    int upto = wave_scan(mine);
    constexpr int kScan = kMaxSeqs / kWave;   // waves that have sequences
    if (lane == kWave - 1 && wave < kScan) sums[wave] = upto;
    __syncthreads();
    if (wave < kScan) {
      for (int w = 0; w < wave; ++w) upto += sums[w];
      before[b + 1] = upto;
      if (b == 0) before[0] = 0;
    }
    __syncthreads();
  }
};

// Steps first .. last - 1 of a unit, of `steps`.
struct Work {
  Seq seq;
  int b, g, row0, first, last, steps, span;   // span: of T
};
template <int ROWS, int STEP, int AHEAD>
__device__ __forceinline__ Work work_at(const KvAttnArgs &a, const Plan<ROWS, STEP, AHEAD> &p, int at, int stop, int group) {
  const int lane = threadIdx.x % kWave;
  Work w;
  w.b = 0;
  for (int b0 = 0; b0 < a.kv.seqs; b0 += kWave) {
    const uint64_t hit = __builtin_amdgcn_ballot_w64(b0 + lane < a.kv.seqs && p.before[b0 + lane] <= at && at < p.before[b0 + lane + 1]);
    if (hit) {
      w.b = b0 + __builtin_ctzll(hit);
      break;
    }
  }
  w.b = __builtin_amdgcn_readfirstlane(w.b);
  w.seq.start = __builtin_amdgcn_readfirstlane(p.start[w.b]);
  w.seq.rows = __builtin_amdgcn_readfirstlane(p.rows[w.b]);
  w.seq.first = __builtin_amdgcn_readfirstlane(p.first[w.b]);
  w.seq.held = __builtin_amdgcn_readfirstlane(p.held[w.b]);
  w.steps = p.steps_of(w.seq.rows, w.seq.first, w.seq.held, group);
  const int length = w.steps + AHEAD, in = at - __builtin_amdgcn_readfirstlane(p.before[w.b]);
  const int index = in / length, from = in - index * length, blocks = p.blocks_of(w.seq.rows);
  w.g = index / blocks;
  w.row0 = (index - w.g * blocks) * ROWS;
  w.span = min(length - from, stop - at);
  w.first = max(0, from - AHEAD);
  w.last = max(0, from + w.span - AHEAD);
  return w;
}
// T among W workgroups: the first T % W have one more than the others.
struct Shares {
  int each, more;
};
__device__ __forceinline__ Shares shares(int total, int groups) {
  Shares s;
  s.each = total / groups;
  s.more = total - s.each * groups;
  return s;
}
__device__ __forceinline__ int begin_of(const Shares &s, int w) { return w * s.each + min(w, s.more); }
// The workgroup that has `at` of T.
__device__ __forceinline__ int owner_of(const Shares &s, int at) {
  const int larger = s.more * (s.each + 1);
  return at < larger ? at / (s.each + 1) : s.more + (at - larger) / s.each;
}
// What a kernel leaves for the join, and its own range.
struct Range {
  int me, at, stop;
};
template <int ROWS, int STEP, int AHEAD>
__device__ __forceinline__ Range range_of(const KvAttnArgs &a, const Plan<ROWS, STEP, AHEAD> &p) {
  const int all = p.before[a.kv.seqs], groups = min((int)gridDim.x, all);
  Range r;
  r.me = blockIdx.x;
  if (r.me == 0)
    for (int b = threadIdx.x; b <= a.kv.seqs; b += blockDim.x) a.plan[b] = p.before[b];
  r.at = r.stop = 0;
  if (r.me < groups) {
    const Shares s = shares(all, groups);
    r.at = begin_of(s, r.me);
    r.stop = begin_of(s, r.me + 1);
  }
  return r;
}

constexpr int kStepTokens = kWaves * kTile, kAhead = 4;
template <int R> using TilePlan = Plan<16 * R, kStepTokens, kAhead>;

// R tiles of 16 rows against blocks of 32 tokens, by one wave, four of them on
// neighbouring blocks: the layout of kv4_attention_kernel, but a block's keys and
// values are expanded once for all tiles.  The queries lie in LDS, in operand
// order.  The products of a score start from minus the row's reference, which the
// matrix cores add for nothing; whether a weight passes fp16's range shows in
// a lane's own sum (fp32 calls: largest, see out_of_range), so that blocks need no
// maximum over lanes until a row's scores rise past its reference: some 30
// instructions a tile and block (four more in fp32), beside 330 of the expansion.
// Two tiles, 32 trees of 8 tokens over up to 4095: 31 to 33 us, of which vector
// instructions take half, matrix instructions 14%; the rest is what a workgroup needs to begin and end
// (prefix sums, table, queries, first block, join of its waves: some 12000 clocks beside
// 3200 a step) and waiting for loads, of which a block a wave is in flight.
template <int D, typename T, int R>
__global__ __launch_bounds__(kThreads, R == 1 && sizeof(T) == 2 ? 3 : 2) void kv4_tree_kernel(KvAttnArgs a) {
  constexpr int PARTS = sizeof(T) == 4 ? 2 : 1;
  constexpr int KW = D / 32;   // words of codes of a lane's part of a key, steps of the dot product
  constexpr int NU = D / 16;   // output blocks of 16 dimensions
  constexpr int kQueries = R * PARTS * KW * kWave * 16, kJoin = R * kWaves * 16 * (D + 4) * 4;
  __shared__ __align__(16) uint8_t s_mem[kQueries > kJoin ? kQueries : kJoin];
  __shared__ float s_down[R * 16];
  __shared__ float s_ml[R][kWaves][16][2];
  __shared__ TilePlan<R> s_plan;
  half8 *const s_q = reinterpret_cast<half8 *>(s_mem);                               // [tile][part][step][lane]
  float (*const s_o)[kWaves][16][D + 4] = reinterpret_cast<float (*)[kWaves][16][D + 4]>(s_mem);   // [tile][wave], after the loop
  const int lane = threadIdx.x % kWave;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const int r = lane & 15, j = lane >> 4;
  const Masks masks_ = masks();
  const int group = a.heads / a.kv.kv_heads;
  s_plan.make(a, group);
  const Range range = range_of(a, s_plan);
  const size_t page_bytes = (size_t)(D * 9 / 8) << a.kv.page_log2;
  const uint32_t values = (uint32_t)(D / 2) << a.kv.page_log2, kmetas = 2 * values, vmetas = kmetas + ((uint32_t)(D / 16) << a.kv.page_log2);
  const int page_mask = (1 << a.kv.page_log2) - 1;
  const float factor = exponent_factor(a.scale);

  for (int at = range.at, span; at < range.stop; at += span) {
    const Work work = work_at(a, s_plan, at, range.stop, group);
    span = work.span;
    if (work.last == work.first) continue;
    const Seq seq = work.seq;
    const int b = work.b, g = work.g, row0 = work.row0;
    const ScalarInts table = scalar_ints(a.kv.page_table + b * a.kv.table_stride);
    const int least = min(seq.first, seq.held);                        // tokens that all rows see
    const int held_end = min(seq.first + seq.rows / group, seq.held);  // tokens that there are
    const int end = min(held_end, work.last * kStepTokens);
    const bool divided = work.last - work.first < work.steps;
    const int tiles = min(R, (seq.rows - row0 + 15) / 16);

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
    const uint32_t first_byte = pick_byte(D == 64 ? (c >> 3) * 2 : 0);
    constexpr int step = kStepTokens;
    int t0 = (work.first * kWaves + wave) * kTile;
    if (t0 < end) {
      find(t0);
      fetch_keys(t0);
      fetch_values(t0);
      find(t0 + step);
    }
    // queries, scaled by a power of two to a largest value of 2^9 .. 2^10
    for (int x = wave; x < R; x += kWaves) {
      const int row = min(row0 + 16 * x + r, seq.rows - 1);
      const T *qp = static_cast<const T *>(a.q) + (seq.start + row / group) * a.q_stride + (g * group + row % group) * D + (D / 4) * j;
      float f[KW][8], amax = 0.0f;
#pragma unroll
      for (int t = 0; t < KW; ++t) {
        load8(qp + 8 * t, f[t]);
#pragma unroll
        for (int e = 0; e < 8; ++e) amax = fmaxf(amax, fabsf(f[t][e]));
      }
      const RowScale rs = row_scale(max_over_j(amax), a.scale);
#pragma unroll
      for (int t = 0; t < KW; ++t) {
        half8 q[PARTS];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const float v = f[t][e / 2 + 4 * (e & 1)] * rs.up;
          q[0][e] = (_Float16)v;
          if constexpr (PARTS == 2) q[1][e] = (_Float16)(v - (float)q[0][e]);
        }
#pragma unroll
        for (int p = 0; p < PARTS; ++p) s_q[((x * PARTS + p) * KW + t) * kWave + lane] = q[p];
      }
      if (j == 0) s_down[16 * x + r] = rs.down;
    }
    __syncthreads();
    float down[R], l[R];
    int mine[R];       // the row's words of `seen`
    floatx4 under[R];  // minus the row's reference score, four times: what the products start from
    floatx4 o[R][NU];
#pragma unroll
    for (int x = 0; x < R; ++x) {
      const int row = min(row0 + 16 * x + r, seq.rows - 1);
      down[x] = s_down[16 * x + r];
      mine[x] = (seq.start + row / group) * a.words;
      l[x] = 0.0f;
      under[x] = all_four(__builtin_inff());
#pragma unroll
      for (int u = 0; u < NU; ++u) o[x][u] = floatx4{0.0f, 0.0f, 0.0f, 0.0f};
    }

    for (; t0 < end; t0 += step) {
      held[0] = next_held[0], held[1] = next_held[1];
      half8 k[2][KW];
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const Pair pair = key_pair(km[h]);
#pragma unroll
        for (int t = 0; t < KW; ++t) k[h][t] = key_values(kw[h][t], pair, masks_);
      }
      fetch_keys(t0 + step);
      const bool whole = held[0] && held[1] && t0 + kTile <= least;
      // scores of tile x above `from`
      auto scores = [&](int x, floatx4 from, floatx4 (&s)[2]) {
        s[0] = s[1] = from;
#pragma unroll
        for (int t = 0; t < KW; ++t)
#pragma unroll
          for (int n = PARTS - 1; n >= 0; --n) {
            const half8 q = s_q[((x * PARTS + n) * KW + t) * kWave + lane];
            s[0] = __builtin_amdgcn_mfma_f32_16x16x32_f16(k[0][t], q, s[0], 0, 0, 0);
            s[1] = __builtin_amdgcn_mfma_f32_16x16x32_f16(k[1][t], q, s[1], 0, 0, 0);
          }
      };
      half8 p[R][PARTS];
      float sum[R], most[R];   // of a lane's weights; most: fp32 calls alone
      auto weigh = [&](int x, const floatx4 (&s)[2]) {
        sum[x] = most[x] = 0.0f;
#pragma unroll
        for (int i = 0; i < 8; i += 2) {
          const float w0 = weight<PARTS>(s[i / 4][i % 4], down[x]), w1 = weight<PARTS>(s[i / 4][i % 4 + 1], down[x]);
          if constexpr (PARTS == 2) most[x] = fmaxf(most[x], fmaxf(w0, w1));
          add_pair<PARTS>(w0, w1, i, p[x], sum[x]);
        }
      };
      // Blocks that all rows see: weights relative to the reference as it is, unless
      // a sum says that one passes the range (or that there is no reference, or
      // that a score is a NaN).
      bool passed = !whole;
      if (whole) {
        floatx4 s[2][2];
        scores(0, under[0], s[0]);
#pragma unroll
        for (int x = 0; x < R; ++x) {
          if (x + 1 < R) scores(x + 1, under[x + 1], s[(x + 1) % 2]);   // on the matrix cores while these are weighed
          weigh(x, s[x % 2]);
          passed |= out_of_range<PARTS>(sum[x], most[x]);
        }
      }
      // Others, and those: with the reference no less than the block's largest.
      if (__builtin_amdgcn_ballot_w64(passed)) {
#pragma unroll
        for (int x = 0; x < R; ++x) {
          const uint32_t bits = whole ? ~0u : block_bits(a.seen + mine[x], a.words, t0, seq.first, end, held[0], held[1]) >> (4 * j);
          floatx4 s[2];
          auto masked = [&](floatx4 from) {
            scores(x, from, s);
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
              for (int i = 0; i < 4; ++i)
                if (!(bits >> (16 * h + i) & 1)) s[h][i] = -__builtin_inff();
          };
          masked(all_four(0.0f));
          float top = s[0][0];
#pragma unroll
          for (int i = 1; i < 8; ++i) top = fmaxf(top, s[i / 4][i % 4]);
          const float m = -under[x][0], high = fmaxf(m, max_over_j(top));
          const float keep = m == -__builtin_inff() ? 0.0f : __builtin_amdgcn_exp2f((m - high) * down[x]);
          under[x] = all_four(-high);
          l[x] *= keep;
#pragma unroll
          for (int u = 0; u < NU; ++u) o[x][u] *= keep;
          masked(under[x]);
          weigh(x, s);
        }
      }
#pragma unroll
      for (int x = 0; x < R; ++x) l[x] += sum[x];
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
        for (int x = 0; x < R; ++x) {
#pragma unroll
          for (int n = PARTS - 1; n >= 0; --n) {
            o[x][2 * bt] = __builtin_amdgcn_mfma_f32_16x16x32_f16(v0, p[x][n], o[x][2 * bt], 0, 0, 0);
            o[x][2 * bt + 1] = __builtin_amdgcn_mfma_f32_16x16x32_f16(v1, p[x][n], o[x][2 * bt + 1], 0, 0, 0);
          }
        }
      }
      fetch_values(t0 + step);
      find(t0 + 2 * step);
      // groups marked as not stored, as in kv4_attention_kernel
      if (__builtin_amdgcn_ballot_w64(marked)) {
        half8 mark;
#pragma unroll
        for (int e = 0; e < 8; ++e) mark[e] = (_Float16)((metas[e / 2] >> (16 * (e % 2) + 8) & 255) == 255 ? 1.0f : 0.0f);
#pragma unroll
        for (int x = 0; x < R; ++x) {
          const uint32_t bits = tree_bits(a.seen + mine[x], a.words, t0 - seq.first) >> (4 * j);
          half8 seen;
#pragma unroll
          for (int e = 0; e < 8; ++e) seen[e] = (_Float16)(bits >> (16 * (e / 4) + e % 4) & 1 ? 1.0f : 0.0f);
          floatx4 count = {};
          count = __builtin_amdgcn_mfma_f32_16x16x32_f16(mark, seen, count, 0, 0, 0);
#pragma unroll
          for (int u = 0; u < NU; ++u)
#pragma unroll
            for (int i = 0; i < 4; ++i) o[x][u][i] = count[i] > 0.0f ? __builtin_nanf("") : o[x][u][i];
        }
      }
    }

    // join the four waves: lane (r, j) has dimensions dim(i, u) of row r of each tile
    constexpr int kPer = 16 * D / kThreads;   // 8 or 4 dimensions a thread
    const int orow = threadIdx.x / (D / kPer), dim = threadIdx.x % (D / kPer) * kPer;
    __syncthreads();   // the queries are done with
#pragma unroll
    for (int x = 0; x < R; ++x) {
      float sum = sum_over_j(l[x]);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int cc = 4 * j + i, at = D == 128 ? 8 * cc : 8 * (cc & 7) + 4 * (cc >> 3);
#pragma unroll
        for (int u = 0; u < NU; u += 4)
          *reinterpret_cast<float4 *>(&s_o[x][wave][r][at + u]) = make_float4(o[x][u][i], o[x][u + 1][i], o[x][u + 2][i], o[x][u + 3][i]);
      }
      if (j == 0) {
        s_ml[x][wave][r][0] = joined_max(-under[x][0], unit(down[x], factor), sum);
        s_ml[x][wave][r][1] = sum;
      }
    }
    __syncthreads();
#pragma unroll
    for (int x = 0; x < R; ++x) {
      if (x >= tiles) break;
      float top = -__builtin_inff(), total = 0.0f, acc[kPer] = {};
#pragma unroll
      for (int w = 0; w < kWaves; ++w) top = fmaxf(top, s_ml[x][w][orow][0]);
#pragma unroll
      for (int w = 0; w < kWaves; ++w) {
        if (s_ml[x][w][orow][1] == 0.0f) continue;
        const float f = s_ml[x][w][orow][0] == -__builtin_inff() ? 1.0f : __builtin_amdgcn_exp2f((s_ml[x][w][orow][0] - top) * factor);
        total += s_ml[x][w][orow][1] * f;
#pragma unroll
        for (int e = 0; e < kPer; ++e) acc[e] += s_o[x][w][orow][dim + e] * f;
      }
      const int row = row0 + 16 * x + orow;
      if (row < seq.rows) {
        if (!divided) {
          const float inv = total == 0.0f ? 0.0f : 1.0f / total;
          T *out = static_cast<T *>(a.o) + (int64_t)(seq.start + row / group) * a.o_stride + (g * group + row % group) * D + dim;
#pragma unroll
          for (int e = 0; e < kPer; ++e) {
            if constexpr (sizeof(T) == 4) out[e] = acc[e] * inv;
            else out[e] = (uint16_t)bf16_pair(acc[e] * inv, 0.0f);
          }
        } else {
          const int64_t to = ((int64_t)range.me * 2 + (work.first ? 0 : 1)) * (16 * R) + 16 * x + orow;
#pragma unroll
          for (int e = 0; e < kPer; ++e) a.part[to * D + dim + e] = acc[e];
          if (dim == 0) {
            a.ml[2 * to] = top;
            a.ml[2 * to + 1] = total;
          }
        }
      }
    }
    __syncthreads();
  }
}

// bf16: rows in blocks of 32 a wave, the layout of kv4_prompt_kernel, whose tiles of
// LDS four waves fill or, where there are rows for them, eight: with those the
// expansion of a tile serves 256 rows.  A wave fetches from one page, so that its
// addresses are a scalar and constants of the lane (24 tokens over 131071: 104 -> 99
// us), and scores start from minus the row's reference, as above (97 -> 95).
// 8 trees of up to 64 tokens over up to 16383, 71 GFLOP: 98 us with 9 for the join, 720
// TFLOP/s; 1 of 24 over 131071, 52 GFLOP: 96 and 9.  A tile takes some 5000 clocks, of
// which the matrix cores work 2000; what a workgroup needs to begin and to write its parts
// is 11 us.  Waves in two groups half a tile apart, products of one beside weights of
// the other, come to the same: vector instructions of one wave alone take 5 to 6
// clocks each, and both groups' follow each other.
constexpr int kWideTile = 64;
template <int D, int WAVES>
__global__ __launch_bounds__(kWave * WAVES, 2) void kv4_tree_wide_kernel(KvAttnArgs a) {
  typedef uint16_t T;
  constexpr int KS = D / 16;           // steps of a score's dot product
  constexpr int NB = D / 32;           // output blocks of 32 dimensions
  constexpr int KW = D / 32;           // words of a key that a thread expands
  constexpr int KB = 32 * D * 2;       // LDS bytes of 32 keys, or of 32 values
  __shared__ __align__(16) uint8_t s_kv[2][4 * KB];          // keys of both blocks, values of both
  __shared__ __align__(16) uint8_t s_mark[2][D / 32][kWideTile];  // marks of value groups, where s_any says there are
  __shared__ __align__(16) uint32_t s_any[2][4];        // bit 0: marks in the wave's share, bit 1: a page is missing
  const int lane = threadIdx.x % kWave;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const int r = lane & 31, hi = lane >> 5;
  const Masks masks_ = masks();
  __shared__ Plan<32 * WAVES, kWideTile, kAhead> s_plan;
  const int group = a.heads / a.kv.kv_heads;
  s_plan.make(a, group);
  const Range range = range_of(a, s_plan);
  const size_t page_bytes = (size_t)(D * 9 / 8) << a.kv.page_log2;
  const uint32_t values = (uint32_t)(D / 2) << a.kv.page_log2, kmetas = 2 * values, vmetas = kmetas + ((uint32_t)(D / 16) << a.kv.page_log2);
  const int page_mask = (1 << a.kv.page_log2) - 1;

  for (int at_ = range.at, span; at_ < range.stop; at_ += span) {
    const Work work = work_at(a, s_plan, at_, range.stop, group);
    span = work.span;
    if (work.last == work.first) continue;
    const Seq seq = work.seq;
    const int g = work.g;
    const ScalarInts table = scalar_ints(a.kv.page_table + work.b * a.kv.table_stride);
    // the page of token `at`, and whether there is one
    auto page_of = [&](int at, bool &held) {
      const int col = at >> a.kv.page_log2;
      const int page = col < a.kv.table_cols ? table[col] : -1;
      held = page >= 0 && page < a.kv.pages;
      return a.kv.pool + ((size_t)(held ? page : 0) * a.kv.kv_heads + g) * page_bytes;
    };
    const int wrow = work.row0 + wave * 32;   // the wave's first row
    const int row = min(wrow + r, seq.rows - 1);
    const int token = seq.start + row / group, head = g * group + row % group;
    const int least = min(seq.first, seq.held);                        // tokens that all rows see
    const int held_end = min(seq.first + seq.rows / group, seq.held);  // tokens that there are
    const int end = min(held_end, work.last * kWideTile);
    const bool divided = work.last - work.first < work.steps;
    const int mine = (seq.start + row / group) * a.words;   // the row's words of `seen`

    half8 q[KS];
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
        q[t][e] = (_Float16)v;
      }
    }

    float m = -__builtin_inff(), l = 0.0f;
    floatx16 o[NB], under;   // under: minus the row's reference score, or 0
#pragma unroll
    for (int i = 0; i < 16; ++i) under[i] = 0.0f;
#pragma unroll
    for (int u = 0; u < NB; ++u)
#pragma unroll
      for (int i = 0; i < 16; ++i) o[u][i] = 0.0f;

    // A wave expands 16 tokens of a tile; with eight waves four their keys and four
    // their values, so that none expands both metas for half of the codes.  A
    // thread's are the KW words of key lane % 16 from word w0 on, and, of the 8 dimensions
    // of octet r / (8 / NB), NB of values 4 hi + 0 .. 3 and + 8.
    const bool does_keys = wave < 4, does_values = WAVES == 4 || wave >= 4;
    const int block = wave & 1, half16 = wave >> 1 & 1;
    const int w0 = KW * (lane >> 4);
    const uint32_t k_lane = (lane & 15) * (D / 2) + w0 * 4, km_lane = kmetas + (lane & 15) * (D / 16) + w0 / 4 * 2;
    const uint32_t oct = (uint32_t)r / (8 / NB), v_lane = values + hi * (2 * D) + oct * 16, vm_lane = vmetas + hi * (D / 4) + oct / 4 * 8;
    u32x4 kw, vw[2];
    uint32_t km;
    u32x2 vm[2];
    bool v_held;
    const int base = work.first * kWideTile, count = max(0, (end - base + kWideTile - 1) / kWideTile);
    int page;   // of the tile that is fetched next
    auto find = [&](int n) {
      const int col = (base + n * kWideTile + 32 * block + 16 * half16) >> a.kv.page_log2;
      page = col < a.kv.table_cols ? table[col] : -1;
    };
    auto fetch = [&](int n) {
      if (n >= count) return;
      v_held = page >= 0 && page < a.kv.pages;
      const uint8_t *rec = a.kv.pool + ((size_t)(v_held ? page : 0) * a.kv.kv_heads + g) * page_bytes;
      const uint32_t in = (base + n * kWideTile + 32 * block + 16 * half16) & page_mask;
      if (does_keys) {
        const uint8_t *kp = rec + in * (D / 2) + k_lane;
        if constexpr (KW == 4) {
          kw = *reinterpret_cast<const u32x4 *>(kp);
        } else {
          const u32x2 two = *reinterpret_cast<const u32x2 *>(kp);
          kw[0] = two[0], kw[1] = two[1];
        }
        km = *reinterpret_cast<const uint16_t *>(rec + in * (D / 16) + km_lane);
      }
      if (does_values) {
#pragma unroll
        for (int x = 0; x < 2; ++x) {
          vw[x] = *reinterpret_cast<const u32x4 *>(rec + in * (D / 2) + 2 * x * (2 * D) + v_lane);
          vm[x] = *reinterpret_cast<const u32x2 *>(rec + in * (D / 16) + 2 * x * (D / 4) + vm_lane);
        }
      }
      find(n + 1);
    };
    auto stage = [&](int n) {
      const int t0 = base + n * kWideTile, buf = n & 1;
      if (does_keys) {
        const Pair pair = key_pair(km);
#pragma unroll
        for (int x = 0; x < KW; ++x)
          *reinterpret_cast<half8 *>(s_kv[buf] + block * KB + (w0 + x) * 512 + (16 * half16 + (lane & 15)) * 16) = key_values(kw[x], pair, masks_);
      }
      if (!does_values) return;
      // tokens that no row sees must not reach the products, whatever their bytes are
      uint32_t metas[4] = {vm[0][0], vm[0][1], vm[1][0], vm[1][1]};
      if (!v_held || t0 + kWideTile > end) {
        const int tok = t0 + 32 * block + 16 * half16 + 4 * hi;
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
        uint8_t *at = s_kv[buf] + 2 * KB + block * KB + half16 * 1024 + lane * 16;
        *reinterpret_cast<half8 *>(at + (2 * bt) * 2048) = v0;
        *reinterpret_cast<half8 *>(at + (2 * bt + 1) * 2048) = v1;
      }
      const bool any = __builtin_amdgcn_ballot_w64(marked) != 0;
      if (lane == 0) s_any[buf][wave & 3] = (any ? 1u : 0u) | (v_held ? 0u : 2u);
      if (any && r % 8 == 0) {   // a lane of each group of 32 dimensions (D 64: of each half)
        uint8_t *mp = &s_mark[buf][r / (8 / NB) / 4][32 * block + 16 * half16 + 4 * hi];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const uint32_t two = metas[e];
          *reinterpret_cast<uint16_t *>(mp + 8 * (e / 2) + 2 * (e % 2)) = (uint16_t)((two >> 8 & 255) == 255 ? 1 : 0) | (uint16_t)(two >> 24 == 255 ? 256 : 0);
        }
      }
    };
    __syncthreads();   // the unit before is done with
    if (count) {
      find(0);
      fetch(0);
      stage(0);
      fetch(1);
      __syncthreads();
    }
    for (int n = 0; n < count; ++n, __syncthreads()) {
      const int t0 = base + n * kWideTile, buf = n & 1;
      const uint8_t *from = s_kv[buf];
      if (n + 1 < count) stage(n + 1);
      fetch(n + 2);
      if (wrow >= seq.rows) continue;
      __builtin_amdgcn_sched_barrier(0);   // staging's registers are free again before the scores take theirs
      const u32x4 any4 = *reinterpret_cast<const u32x4 *>(s_any[buf]);
      const uint32_t any = __builtin_amdgcn_readfirstlane(any4[0] | any4[1] | any4[2] | any4[3]);
      // two chains of products, the operands of the next two steps on their way
      floatx16 s[2] = {under, under};
      half8 k[3][2];
      auto keys = [&](int x, int t) { return *reinterpret_cast<const half8 *>(from + x * KB + t * 1024 + lane * 16); };
#pragma unroll
      for (int t = 0; t < 2; ++t) k[t][0] = keys(0, t), k[t][1] = keys(1, t);
#pragma unroll
      for (int t = 0; t < KS; ++t) {
        if (t + 2 < KS) k[(t + 2) % 3][0] = keys(0, t + 2), k[(t + 2) % 3][1] = keys(1, t + 2);
#pragma unroll
        for (int x = 0; x < 2; ++x) s[x] = __builtin_amdgcn_mfma_f32_32x32x16_f16(k[t % 3][x], q[t], s[x], 0, 0, 0);
      }
      // in this order: left to itself the compiler reads an operand, waits and multiplies
      __builtin_amdgcn_sched_group_barrier(0x100, 4, 0);   // reads of LDS
#pragma unroll
      for (int t = 0; t < KS; ++t) {
        __builtin_amdgcn_sched_group_barrier(0x008, 2, 0);   // matrix instructions
        if (t + 2 < KS) __builtin_amdgcn_sched_group_barrier(0x100, 2, 0);
      }
      __builtin_amdgcn_sched_barrier(0);
      uint32_t bits[2] = {~0u, ~0u};   // of this lane's tokens of both blocks, shifted by 4 hi
      if (t0 + kWideTile > least || (any & 2)) {
        bool held[4];
#pragma unroll
        for (int x = 0; x < 4; ++x) page_of(t0 + 16 * x, held[x]);
#pragma unroll
        for (int x = 0; x < 2; ++x) {
          bits[x] = block_bits(a.seen + mine, a.words, t0 + 32 * x, seq.first, end, held[2 * x], held[2 * x + 1]) >> (4 * hi);
#pragma unroll
          for (int i = 0; i < 16; ++i)
            if (!(bits[x] >> (16 * (i / 8) + 8 * (i % 8 / 4) + i % 4) & 1)) s[x][i] = -__builtin_inff();
        }
      }
      float top = s[0][0];
#pragma unroll
      for (int i = 1; i < 32; ++i) top = fmaxf(top, s[i / 16][i % 16]);
      top = max_of_halves(top);
      if (__builtin_amdgcn_ballot_w64(m == -__builtin_inff() || top * rs.down > Hold<1>::slack)) {
        // without a reference, what is largest up to now, else no less than that
        const float by = m == -__builtin_inff() ? (top == -__builtin_inff() ? 0.0f : top) : fmaxf(top, 0.0f);
        const float high = m == -__builtin_inff() ? top : m + by, keep = m == -__builtin_inff() ? 0.0f : __builtin_amdgcn_exp2f(-by * rs.down);
        m = high;
        l *= keep;
#pragma unroll
        for (int u = 0; u < NB; ++u) o[u] *= keep;
#pragma unroll
        for (int i = 0; i < 16; ++i) under[i] -= by, s[0][i] -= by, s[1][i] -= by;
      }
      // probabilities of the next 16 tokens ahead of the products of these
      half8 p[4][1];
      auto weigh = [&](int part) {
#pragma unroll
        for (int e = 0; e < 8; e += 2)
          add_pair<1>(weight<1>(s[part / 2][8 * (part % 2) + e], rs.down), weight<1>(s[part / 2][8 * (part % 2) + e + 1], rs.down), e, p[part], l);
      };
      weigh(0);
#pragma unroll
      for (int part = 0; part < 4; ++part) {
        half8 v[NB];
#pragma unroll
        for (int u = 0; u < NB; ++u) v[u] = *reinterpret_cast<const half8 *>(from + 2 * KB + part / 2 * KB + u * 2048 + part % 2 * 1024 + lane * 16);
        if (part < 3) weigh(part + 1);
#pragma unroll
        for (int u = 0; u < NB; ++u) o[u] = __builtin_amdgcn_mfma_f32_32x32x16_f16(v[u], p[part][0], o[u], 0, 0, 0);
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
            const int in = 8 * (e / 4) + e % 4, at = 16 * x + 4 * hi + in;
            mark[e] = (_Float16)(any4[x / 2 + 2 * (x % 2)] & 1 ? (float)marks[at] : 0.0f);
            seen[e] = (_Float16)(bits[x / 2] >> (16 * (x % 2) + in) & 1 ? 1.0f : 0.0f);
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
    const int64_t to = ((int64_t)range.me * 2 + (work.first ? 0 : 1)) * (32 * WAVES) + wave * 32 + r;
    const float inv = divided ? 1.0f : l == 0.0f ? 0.0f : 1.0f / l;
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
        if (divided) store8(a.part + to * D + dim + e, f + e);
        else store8(static_cast<T *>(a.o) + token * a.o_stride + head * D + dim + e, f + e);
      }
    }
    if (divided && hi == 0) {
      a.ml[2 * to] = joined_max(m, unit(rs.down, exponent_factor(a.scale)), l);
      a.ml[2 * to + 1] = l;
    }
  }
}

// Joins the parts of a divided unit.  D / 4 lanes take a row; with SHARE the
// groups of lanes of a workgroup share out the parts of one row, otherwise each has
// a row of its own.
template <int D, typename T, int ROWS, int STEP, int AHEAD, bool SHARE>
__global__ __launch_bounds__(kThreads) void kv4_tree_join_kernel(KvAttnArgs a) {
  typedef Plan<ROWS, STEP, AHEAD> P;
  constexpr int kLanes = D / 4, kGroups = kThreads / kLanes, kJoinRows = SHARE ? 1 : kGroups, kSlices = ROWS / kJoinRows;
  __shared__ float4 s_o[kGroups][kLanes];
  __shared__ float2 s_ml[kGroups];
  const int group = a.heads / a.kv.kv_heads;
  int id = blockIdx.x;
  const int slice = id % kSlices;
  id /= kSlices;
  const int g = id % a.kv.kv_heads;
  id /= a.kv.kv_heads;
  const int first_block = id % a.row_blocks, b = id / a.row_blocks;
  const Seq seq = sequence(a, b, group);
  const int steps = P::steps_of(seq.rows, seq.first, seq.held, group), blocks = P::blocks_of(seq.rows);
  const int all = a.plan[a.kv.seqs], before = a.plan[b];
  if (all == 0) return;
  const Shares of = shares(all, min(a.splits, all));
  const int lanes = threadIdx.x / kLanes, in = slice * kJoinRows + (SHARE ? 0 : lanes), dim = threadIdx.x % kLanes * 4;
  const float factor = exponent_factor(a.scale);
  for (int block = first_block; block < blocks; block += a.row_blocks) {
    const int from = before + (g * blocks + block) * (steps + AHEAD) + AHEAD;
    const int w0 = owner_of(of, from), w1 = owner_of(of, from + steps - 1);
    const int row = block * ROWS + in;
    if (w0 == w1 || row >= seq.rows) continue;   // SHARE: the whole workgroup's
    float top = -__builtin_inff(), total = 0.0f;
    float4 acc = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
    // some parts at a time, so that their loads go out together
    constexpr int kAtOnce = 4, kStride = SHARE ? kGroups : 1;
    for (int w = w0 + (SHARE ? lanes : 0); w <= w1; w += kAtOnce * kStride) {
      float2 v[kAtOnce];
      float4 o[kAtOnce];
#pragma unroll
      for (int i = 0; i < kAtOnce; ++i) {
        const int part = min(w + i * kStride, w1);
        const int64_t at = ((int64_t)part * 2 + (part == w0 ? 1 : 0)) * ROWS + in;
        v[i] = reinterpret_cast<const float2 *>(a.ml)[at];
        o[i] = *reinterpret_cast<const float4 *>(a.part + at * D + dim);
      }
      float most = top;
#pragma unroll
      for (int i = 0; i < kAtOnce; ++i) most = fmaxf(most, v[i].x);
      const float keep = top == most ? 1.0f : __builtin_amdgcn_exp2f((top - most) * factor);
      top = most;
      total *= keep;
      acc.x *= keep, acc.y *= keep, acc.z *= keep, acc.w *= keep;
#pragma unroll
      for (int i = 0; i < kAtOnce; ++i) {
        // a part without tokens has no sum; one of NaN scores alone has no maximum
        if (w + i * kStride > w1 || v[i].y == 0.0f) continue;
        const float f = v[i].x == top || v[i].x == -__builtin_inff() ? 1.0f : __builtin_amdgcn_exp2f((v[i].x - top) * factor);
        total += v[i].y * f;
        acc.x += o[i].x * f, acc.y += o[i].y * f, acc.z += o[i].z * f, acc.w += o[i].w * f;
      }
    }
    if constexpr (SHARE) {
      __syncthreads();   // the block's before
      s_o[lanes][dim / 4] = acc;
      if (dim == 0) s_ml[lanes] = make_float2(top, total);
      __syncthreads();
      if (lanes) continue;
#pragma unroll
      for (int i = 0; i < kGroups; ++i) top = fmaxf(top, s_ml[i].x);
      total = 0.0f;
      acc = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll
      for (int i = 0; i < kGroups; ++i) {
        const float2 v = s_ml[i];
        const float4 o = s_o[i][dim / 4];
        if (v.y == 0.0f) continue;
        const float f = v.x == top || v.x == -__builtin_inff() ? 1.0f : __builtin_amdgcn_exp2f((v.x - top) * factor);
        total += v.y * f;
        acc.x += o.x * f, acc.y += o.y * f, acc.z += o.z * f, acc.w += o.w * f;
      }
    }
    const float inv = total == 0.0f ? 0.0f : 1.0f / total;
    T *out = static_cast<T *>(a.o) + (int64_t)(seq.start + row / group) * a.o_stride + (g * group + row % group) * D + dim;
    if constexpr (sizeof(T) == 4) *reinterpret_cast<float4 *>(out) = make_float4(acc.x * inv, acc.y * inv, acc.z * inv, acc.w * inv);
    else *reinterpret_cast<uint2 *>(out) = make_uint2(bf16_pair(acc.x * inv, acc.y * inv), bf16_pair(acc.z * inv, acc.w * inv));
  }
}

template <int D, typename T, int ROWS, int STEP, int AHEAD>
void launch_join(const KvAttnArgs &a, unsigned units, hipStream_t s) {
  // units of many parts, some ten and more
  if ((unsigned)a.splits >= 12 * units) hipLaunchKernelGGL((kv4_tree_join_kernel<D, T, ROWS, STEP, AHEAD, true>), dim3(units * ROWS), dim3(kThreads), 0, s, a);
  else hipLaunchKernelGGL((kv4_tree_join_kernel<D, T, ROWS, STEP, AHEAD, false>), dim3(units * (ROWS * D / 4 / kThreads)), dim3(kThreads), 0, s, a);
}

template <int D, typename T, int R>
void launch_tiles(const KvAttnArgs &a, hipStream_t s) {
  const unsigned units = (unsigned)a.kv.seqs * a.kv.kv_heads * a.row_blocks;
  hipLaunchKernelGGL((kv4_tree_kernel<D, T, R>), dim3((unsigned)a.splits), dim3(kThreads), 0, s, a);
  launch_join<D, T, 16 * R, kStepTokens, kAhead>(a, units, s);
}

template <int D, int WAVES>
void launch_wide(const KvAttnArgs &a, hipStream_t s) {
  const unsigned units = (unsigned)a.kv.seqs * a.kv.kv_heads * a.row_blocks;
  hipLaunchKernelGGL((kv4_tree_wide_kernel<D, WAVES>), dim3((unsigned)a.splits), dim3(kWave * WAVES), 0, s, a);
  launch_join<D, uint16_t, 32 * WAVES, kWideTile, kAhead>(a, units, s);
}

template <int D, typename T>
void launch(const KvAttnArgs &a, int tiles, hipStream_t s) {
  if (tiles == 1) return launch_tiles<D, T, 1>(a, s);
  if constexpr (sizeof(T) == 2)
    if (tiles == 8) return launch_wide<D, 4>(a, s);
  if constexpr (sizeof(T) == 2 && D == 128)
    if (tiles == 16) return launch_wide<D, 8>(a, s);
  launch_tiles<D, T, 2>(a, s);
}

}  // namespace

// Which kernels: by `units`, blocks of 16 rows of all sequences and kv heads, `steps`
// of 128 tokens of the longest sequence, and their product `work`.  us of a pass, 32
// heads to 8 of 128, bf16 unless said otherwise; "split" are the kernels of
// kv4_attn.hip, which cut every sequence alike (from 64 rows on, those of prompts):
//                                             units steps  split 1 tile 2 tiles 128 rows  256
//   up to 16 rows: 64 of 4 tokens over 2047     512    17     33     34      43       62   96
//     1 of 4 over 8000                            8    63     16     17      18       18
//   up to 63: 64 of 8 over 700                 1024     6     25     32      30       42   61
//     64 of 8 over 1200                        1024    10     35     36      34       48
//     64 of 8 over 1800                        1024    15     50     50      44       63
//     16 of 8 over 1200                         256    10     18     20      20       22
//     1 of 8 over 2000                           16    17     13     13      13       15
//     1 of 8 over 4096                           16    33     19     17      17       19   18
//     32 of 8 over up to 4095, ragged           512    33     48     43      37       50   67
//     1 of 8 over 131071                         16  1025     68     71      56       75
//   from 64: 1 of 16 over 1500                   32    12     18     14      14       16   18
//     4 of 16 over 8191                         128    65     36     27      27       32   31
//     100 of 16 over 1024                      3200     9     74     85      67       75   98
//     64 of 32 over 100                        4096     2     20     52      46       35   47
//     16 of 24 over 8191                        768    65     91    109      77       71   77
//     32 of 32 over 1000                       2048     9     44     56      45       37   43
//     4 of 64 over 1500                         512    13     31     27      26       30   32
//     2 of 1000 over 1000                      4000    16    121    159     112       79   74
//     1 of 24 over 131071                        48  1025    112    180     118       97  103
//     8 of up to 64 over up to 16383           1024   129    145    247     157      111   99
//   fp32, scores of a row with a standard deviation of 2.4 / of 0.24, which needs the
//   reference moved less often:
//     16 of 12 over 8191                        384    65    70/67  65/52   75/53
//     10 of 49 over 1393                       1040    12    50/47  47/40   51/38
//     4 of 48 over 16000                        384   126   178/167 134/116 124/86
//     16 heads to 16, 32 of 32 over 2047       1024    17    56/53  63/52   68/49
//     the same over 6000                       1024    48   130/127 123/101 124/89
//   heads of 64: 64 of 8 over 700              1024     6     20     24      23       31
//     64 of 8 over 1800                        1024    15     37     38      34       46
//     32 of 8 over up to 4095                   512    33     36     31      28       37
//     1 of 8 over 4096                           16    33     15     13      14       16
//     4 of 16 over 8191                         128    65     30     22      23       28
//     16 of 24 over 8191                        768    65     68     79      56       51
//     1 of 24 over 131071                        48  1025     88    131      84       70
//     8 of up to 64 over up to 16383           1024   129    112    179     113       77
// The plan and the join cost more than they save where units have few steps, and where there
// is little to share out.
KvAttnShape kv4_tree_shape(int seqs, int kv_heads, int heads, int tokens, int max_new, int max_len, int64_t table_tokens, int head_dim, bool f32) {
  KvAttnShape s = kv4_attention_shape(seqs, kv_heads, heads, tokens, max_new, max_len);
  const int64_t full = (int64_t)tokens * (heads / kv_heads);   // rows, were they all of one sequence
  const int64_t hinted = (int64_t)max_new * (heads / kv_heads), rows = hinted < full ? hinted : full;
  const int64_t pairs = (int64_t)seqs * kv_heads, units = pairs * ((rows + 15) / 16), steps = ((int64_t)max_len + kStepTokens - 1) / kStepTokens;
  const int64_t work = units * steps;
  if (seqs > kMaxSeqs) return s;
  if (rows < 64 && (steps <= 12 || work < 512 || (units >= 512 && steps <= 20 && (f32 || rows <= 16)))) return s;
  if (work < 64 || (units >= 512 && steps <= 2)) return s;
  int tiles;
  if (f32) tiles = rows >= 64 && work >= 24576 ? 2 : 1;
  else if (rows > 64 && work >= 8192) tiles = head_dim == 128 && rows > 224 ? 16 : 8;
  else tiles = rows > 16 && work >= (rows < 64 ? 12288 : 4096) ? 2 : 1;
  const int per = 16 * tiles;
  // T has to fit an int, for the longest sequences that the table has room for and
  // whatever q_start holds
  if ((full / per + 1) * pairs >= ((int64_t)1 << 31) / (table_tokens / kWideTile + kAhead + 2)) return s;
  s.tiles = tiles;
  const int64_t blocks = (rows + per - 1) / per, room = kMaxGroups / (pairs * per);
  s.row_blocks = (int)(blocks < 1 || room < 1 ? 1 : blocks > room ? room : blocks);
  s.splits = tiles == 16 ? 256 : 512;   // workgroups, of 512 threads one a compute unit, others two
  return s;
}

hipError_t launch_kv4_tree(const KvAttnArgs &a, int tiles, int head_dim, bool f32, hipStream_t s) {
  if (head_dim == 64) {
    if (f32) launch<64, float>(a, tiles, s);
    else launch<64, uint16_t>(a, tiles, s);
  } else {
    if (f32) launch<128, float>(a, tiles, s);
    else launch<128, uint16_t>(a, tiles, s);
  }
  return hipGetLastError();
}

}  // namespace moe
