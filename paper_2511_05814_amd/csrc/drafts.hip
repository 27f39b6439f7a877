// Trees of drafted tokens: their plan, and their verification against the
// target's probabilities.
#include <type_traits>

#include "common.hpp"

namespace moe {
namespace {

// The new tokens of a sequence.
struct Tree {
  int start, n;
};
__device__ __forceinline__ Tree tree_of(const int32_t *q_start, int seq, int tokens) {
  Tree t;
  t.start = min(max(q_start[seq], 0), tokens);
  t.n = min(max(q_start[seq + 1], t.start), tokens) - t.start;
  return t;
}

// pos[t] = place of the sequence's first new token + depth(t); bit j of seen[t]:
// new token j is t or one of its ancestors.  A parent that is not before its
// token is none.
//
// Tokens lie in blocks of 32, a half wave each.  Within a block five rounds, in
// which every token takes over what the ancestor that it has come to has, give its
// ancestors there and the first one in front of the block; from there on a token goes
// up a block at a time.  A walk up the parents one by one takes as long as the tree
// is deep: 747 tokens, some 500 deep, 60 us so.  What is left is the launch and the
// few loads that depend on each other; many long rows, their stores.
__global__ __launch_bounds__(kMaxTree) void draft_tree_kernel(DraftTreeArgs a) {
  __shared__ uint32_t s_mask[kMaxTree];
  __shared__ int16_t s_exit[kMaxTree];
  const int seq = blockIdx.x, lane = threadIdx.x % kWave, half = lane & 32;
  const Tree tree = tree_of(a.q_start, seq, a.tokens);
  const int n = min(tree.n, 32 * a.words), first = a.kv_len[seq] - tree.n;
  for (int i0 = 0; i0 < n; i0 += blockDim.x) {
    const int i = i0 + threadIdx.x, p = i < n ? a.parent[tree.start + i] : -1;
    uint32_t mask = 1u << (i & 31);
    int exit = p >= 0 && p < i ? p : -1, up = exit >= 0 && exit >> 5 == i >> 5 ? exit & 31 : -1;
#pragma unroll
    for (int round = 0; round < 5; ++round) {
      const int from = half + max(up, 0);
      const uint32_t theirs = __shfl(mask, from, kWave);
      const int their_exit = __shfl(exit, from, kWave), their_up = __shfl(up, from, kWave);
      if (up >= 0) mask |= theirs, exit = their_exit, up = their_up;
    }
    if (i < n) s_mask[i] = mask, s_exit[i] = (int16_t)exit;
  }
  __syncthreads();
  for (int i = threadIdx.x; i < tree.n; i += blockDim.x) {
    uint32_t *row = a.seen + (int64_t)(tree.start + i) * a.words;
    int depth = -1, x = i < n ? i : -1;
    auto word = [&](int w) {
      if (x < 32 * w) return 0u;
      const uint32_t bits = s_mask[x];
      x = s_exit[x];
      depth += __builtin_popcount(bits);
      return bits;
    };
    // lanes write to rows of their own: four words at a time where rows allow it (15
    // chains of 1024: 20 us word by word)
    if (a.words % 4 == 0 && reinterpret_cast<uintptr_t>(a.seen) % 16 == 0) {
      for (int w = a.words - 4; w >= 0; w -= 4) {
        uint4 four;
        four.w = word(w + 3), four.z = word(w + 2), four.y = word(w + 1), four.x = word(w);
        *reinterpret_cast<uint4 *>(row + w) = four;
      }
    } else {
      for (int w = a.words - 1; w >= 0; --w) row[w] = word(w);
    }
    a.pos[tree.start + i] = i < n ? first + depth : -1;
  }
}

// Verification.  `clusters` workgroups share a sequence's row: each sums its own
// stretch of it, tells the others through the workspace and does the same walk as
// they do, from the same numbers.  What is left of a row after refusals is max(p -
// share q, 0) with one number, share, as max(max(p - s q, 0) - t q, 0) = max(p - (s +
// t) q, 0) for q >= 0, so nothing but sums is kept between passes.
//
// Latency bounds it: the launch, three loads of which each needs the last one's
// result, a pass for every refused child but the first of a token, and the draw;
// within a pass the widening to fp64, 16 clocks an entry and wave where other
// instructions take 4.
//
// What a pass over the rows gives, left = sum max(p - share q, 0), is a sum of the
// stretches' sums in their order, whoever has summed them: a workgroup that does
// not hear of a stretch in time sums it itself.  So no workgroup has to run beside
// another, and every one of them ends.
constexpr int kVerifyThreads = 1024, kVerifyWaves = kVerifyThreads / kWave;
constexpr uint64_t kUnset = ~(uint64_t)0;     // a NaN that no sum is written as
constexpr int kPolls = 256;                   // some tens of us, after which a workgroup helps itself

__device__ __forceinline__ float widened(float x) { return x; }
__device__ __forceinline__ float widened(uint16_t x) { return __uint_as_float((uint32_t)x << 16); }
// Sums over the lanes up to each: wave_sum_d_to_lane63's steps leave them.
__device__ __forceinline__ double wave_scan_d(double v) { return wave_sum_d_to_lane63(v); }
// NaN kept
__device__ __forceinline__ double positive(double v) { return v <= 0.0 ? 0.0 : v; }

// 16 bytes of a row, which need not be aligned to more than an entry.
typedef uint32_t WordsBy2 __attribute__((ext_vector_type(4), aligned(2)));
typedef uint32_t WordsBy4 __attribute__((ext_vector_type(4), aligned(4)));
template <typename T>
struct Entries {
  typedef std::conditional_t<sizeof(T) == 2, WordsBy2, WordsBy4> Words;
  static constexpr int kCount = 16 / sizeof(T);
  Words w;
  __device__ __forceinline__ void load(const T *row) { w = *reinterpret_cast<const Words *>(row); }
  // of a row of n < kCount
  __device__ __forceinline__ void load_end(const T *row, int n) {
#pragma unroll
    for (int k = 0; k < kCount; ++k) {
      const uint32_t bits = k < n ? __builtin_bit_cast(std::conditional_t<sizeof(T) == 2, uint16_t, uint32_t>, row[k]) : 0u;
      if constexpr (sizeof(T) == 4) w[k] = bits;
      else w[k / 2] = k % 2 ? w[k / 2] | bits << 16 : bits;
    }
  }
  __device__ __forceinline__ void clear(int k) {
    if constexpr (sizeof(T) == 4) w[k] = 0;
    else w[k / 2] &= k % 2 ? 0x0000FFFFu : 0xFFFF0000u;
  }
  __device__ __forceinline__ float at(int k) const {
    if constexpr (sizeof(T) == 4) return __uint_as_float(w[k]);
    else return __uint_as_float(k % 2 ? w[k / 2] & 0xFFFF0000u : w[k / 2] << 16);
  }
};
__device__ __forceinline__ double sum_of(const double (&w)[4]) { return (w[0] + w[1]) + (w[2] + w[3]); }
__device__ __forceinline__ double sum_of(const double (&w)[8]) { return ((w[0] + w[1]) + (w[2] + w[3])) + ((w[4] + w[5]) + (w[6] + w[7])); }

__global__ __launch_bounds__(256) void verify_clear_kernel(uint64_t *slots, int n) {
  const int i = blockIdx.x * 256 + threadIdx.x;
  if (i < n) slots[i] = kUnset;
}

template <typename T, bool DRAWN>
__global__ __launch_bounds__(kVerifyThreads) void verify_drafts_kernel(VerifyArgs a) {
  constexpr int kRow = Entries<T>::kCount;   // entries of a lane's step
  constexpr int kStep = kWave * kRow;        // of a wave's
  constexpr int kAhead = 32 / kRow;          // steps whose loads go out together
  __shared__ int16_t s_parent[kMaxTree], s_path[kMaxTree];
  __shared__ int32_t s_id[kMaxTree];
  __shared__ float s_p[kMaxTree], s_q[kMaxTree], s_u[kMaxTree];
  __shared__ double s_wave[kVerifyWaves], s_own[kVerifyWaves], s_chunk[kMaxClusters];
  __shared__ uint32_t s_tried[128];   // without q: which groups of ids that a lane reads at once, by their last 12 bits, hold one that was tried
  const int lane = threadIdx.x % kWave, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const int seq = blockIdx.x / a.clusters, chunk = blockIdx.x % a.clusters;
  const Tree tree = tree_of(a.q_start, seq, a.tokens);
  if (tree.n == 0) {
    if (chunk == 0 && threadIdx.x == 0) a.count[seq] = 0, a.next[seq] = -1;
    return;
  }
  const int n = min(tree.n, kMaxTree);
  const T *const p0 = static_cast<const T *>(a.p) + (int64_t)tree.start * a.p_stride;
  const T *const q0 = DRAWN ? static_cast<const T *>(a.q) + (int64_t)tree.start * a.q_stride : nullptr;

  // every token with the entries of p and q that decide about it
  for (int i = threadIdx.x; i < n; i += kVerifyThreads) {
    const int up = i ? a.parent[tree.start + i] : -1, id = a.ids[tree.start + i];
    const bool known = up >= 0 && up < i && id >= 0 && id < a.vocab;
    s_parent[i] = (int16_t)(up >= 0 && up < i ? up : -1);
    s_id[i] = id;
    s_u[i] = fmaxf(a.u[tree.start + i], 0.0f);
    s_p[i] = known ? widened(p0[up * a.p_stride + id]) : 0.0f;
    if constexpr (DRAWN) s_q[i] = known ? widened(q0[up * a.q_stride + id]) : 0.0f;
    s_path[i] = i ? -1 : 0;
  }
  __syncthreads();

  // A wave's part of stretch c: steps first .. first + steps - 1.
  const int all_steps = (a.vocab + kStep - 1) / kStep;
  auto part_of = [&](int c, int w, int &first, int &steps) {
    const int unit = c * kVerifyWaves + w, units = a.clusters * kVerifyWaves;
    first = (int)((int64_t)all_steps * unit / units);
    steps = (int)((int64_t)all_steps * (unit + 1) / units) - first;
  };
  int cur = 0, depth = 0, pass = 0;
  bool masked = false;   // without q: cur's children were tried and have no weight
  bool bare = false;     // p as it is
  double share = 0.0, left = 1.0;

  // Up to AHEAD steps of 64 lanes with 16 bytes each, loaded at once: f(first
  // entry of the lane, its weights) for each step from t on below `upto`.  Lanes past the
  // row's end read its last entries again and have no weights; of 16 bytes that
  // the end cuts the last ones are read, those that are not the lane's left out.
  auto steps_of = [&](auto ahead, int t, int upto, auto f) {
    constexpr int AHEAD = decltype(ahead)::value;
    // p itself, where no child was refused or nothing is left, is p less 0 times p: no
    // choice to make for every entry, and a row of q that drew nothing may hold anything
    const T *const p = p0 + cur * a.p_stride, *const q = DRAWN && share != 0.0 ? q0 + cur * a.q_stride : p;
    Entries<T> fs[AHEAD], gs[AHEAD];
#pragma unroll
    for (int x = 0; x < AHEAD; ++x) {
      if (t + x >= upto) break;
      const int i = min((t + x) * kStep + lane * kRow, a.vocab - kRow);
      if (a.vocab >= kRow) {
        fs[x].load(p + i);
        if constexpr (DRAWN) gs[x].load(q + i);
      } else {
        fs[x].load_end(p, a.vocab);
        if constexpr (DRAWN) gs[x].load_end(q, a.vocab);
      }
    }
#pragma unroll
    for (int x = 0; x < AHEAD; ++x) {
      if (t + x >= upto) break;
      const int i = (t + x) * kStep + lane * kRow, skip = a.vocab >= kRow ? i - min(i, a.vocab - kRow) : i;
      if ((t + x + 1) * kStep > a.vocab) {
#pragma unroll
        for (int k = 0; k < kRow; ++k) {
          if (k >= skip) continue;
          fs[x].clear(k);
          if constexpr (DRAWN) gs[x].clear(k);
        }
      }
      double w[kRow];
#pragma unroll
      for (int k = 0; k < kRow; ++k) {
        const float e = fs[x].at(k);
        w[k] = positive(DRAWN ? fma(-share, (double)gs[x].at(k), (double)e) : (double)e);
      }
      const int first = i - skip;
      if (!DRAWN && masked) {
        // ids that were tried
        const uint32_t lo = (uint32_t)first / kRow & 4095, hi = (uint32_t)(first + kRow - 1) / kRow & 4095;
        if ((s_tried[lo / 32] >> (lo % 32) | s_tried[hi / 32] >> (hi % 32)) & 1) {
          for (int c = cur + 1; c < n; ++c) {
            if (s_parent[c] != cur) continue;
#pragma unroll
            for (int k = 0; k < kRow; ++k) w[k] = s_id[c] == first + k ? 0.0 : w[k];
          }
        }
      }
      f(first, w);
    }
  };
  // this workgroup's sum over stretch c; its waves' in s_wave
  auto stretch = [&](int c) {
    int first, steps;
    part_of(c, wave, first, steps);
    double sum = 0.0;
    for (int t = 0; t < steps; t += kAhead)
      steps_of(std::integral_constant<int, kAhead>(), first + t, first + steps, [&](int, const double (&w)[kRow]) { sum += sum_of(w); });
    sum = wave_scan_d(sum);
    __syncthreads();   // s_wave is free
    if (lane == kWave - 1) s_wave[wave] = sum;
    __syncthreads();
    double all = 0.0;
#pragma unroll
    for (int w = 0; w < kVerifyWaves; ++w) all += s_wave[w];
    return all != all ? __builtin_nan("") : all;
  };
  // the sum over the row, the stretches' in s_chunk, this one's waves' in s_own
  auto whole_row = [&] {
    const bool shared = pass < kVerifyPasses;
    uint64_t *slots = a.slots + ((int64_t)seq * kVerifyPasses + (shared ? pass : 0)) * a.clusters;
    ++pass;
    for (int x = -1; x < a.clusters; ++x) {
      if (x >= 0 && __builtin_bit_cast(uint64_t, s_chunk[x]) != kUnset) continue;
      const double v = stretch(x < 0 ? chunk : x);
      if (x >= 0) {
        if (threadIdx.x == 0) s_chunk[x] = v;
        continue;
      }
      if (threadIdx.x < kVerifyWaves) s_own[threadIdx.x] = s_wave[threadIdx.x];
      if (a.clusters == 1) return v;
      if (wave == 0) {
        uint64_t got = kUnset;
        if (shared) {
          if (lane == 0) __hip_atomic_store(slots + chunk, __builtin_bit_cast(uint64_t, v), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
          for (int i = 0; i < kPolls; ++i) {
            if (lane < a.clusters && got == kUnset) got = __hip_atomic_load(slots + lane, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
            if (__builtin_amdgcn_ballot_w64(lane < a.clusters && got == kUnset) == 0) break;
          }
        }
        if (lane == chunk) got = __builtin_bit_cast(uint64_t, v);
        if (lane < a.clusters) s_chunk[lane] = __builtin_bit_cast(double, got);
      }
      __syncthreads();
    }
    __syncthreads();
    double all = 0.0;
    for (int c = 0; c < a.clusters; ++c) all += s_chunk[c];
    __syncthreads();   // the next pass writes s_chunk
    return all;
  };

  // The walk goes on until it wants a sum: `left` for the next child, or, with no
  // child left, the weights' sum for the draw.
  double total = 0.0;
  bool ended = false, stale = false;
  for (int from = 0;;) {   // children up to here were tried
    while (!ended) {
      uint64_t children = 0;
      int c0 = (from + 1) / kWave * kWave;
      for (; c0 < n; c0 += kWave) {
        const int c = c0 + lane;
        children = __builtin_amdgcn_ballot_w64(c > from && c < n && s_parent[min(c, n - 1)] == cur);
        if (children) break;
      }
      if (!children) {
        ended = true;
        break;
      }
      if (stale) break;
      const int c = c0 + __builtin_ctzll(children);
      bool accepted;
      if constexpr (DRAWN) {
        const double guess = (double)s_q[c], w = positive(fma(-share, guess, (double)s_p[c]));
        accepted = (double)s_u[c] * left * guess < w;
        if (!accepted) share += left, stale = true;
      } else {
        bool before = false;   // an id that was tried has no weight left
        for (int e0 = (cur + 1) / kWave * kWave; e0 < c; e0 += kWave) {
          const int e = min(e0 + lane, n - 1);
          before |= __builtin_amdgcn_ballot_w64(e0 + lane < c && s_parent[e] == cur && s_id[e] == s_id[c]) != 0;
        }
        const double w = before ? 0.0 : positive((double)s_p[c]);
        accepted = (double)s_u[c] * left < w;
        if (!accepted) left = positive(left - w), masked = true;
      }
      from = c;
      if (accepted) {
        cur = c;
        ++depth;
        if (threadIdx.x == 0) s_path[depth] = (int16_t)cur;
        share = 0.0, left = 1.0;
        masked = false;
      }
    }
    if (!DRAWN && masked) {
      __syncthreads();
      for (int i = threadIdx.x; i < 128; i += kVerifyThreads) s_tried[i] = 0;
      __syncthreads();
      for (int i = cur + 1 + threadIdx.x; i < n; i += kVerifyThreads) {
        const uint32_t octet = (uint32_t)s_id[i] / kRow & 4095;
        if (s_parent[i] == cur) atomicOr(&s_tried[octet / 32], 1u << (octet % 32));
      }
      __syncthreads();
    }
    total = whole_row();
    if (!ended) left = total, stale = false;
    else if (total == 0.0 && !bare) bare = true, masked = false, share = 0.0;   // nothing is left: p itself
    else break;
  }
  if (chunk == 0) {
    __syncthreads();
    for (int i = threadIdx.x; i < tree.n; i += kVerifyThreads) a.path[tree.start + i] = i < n ? s_path[i] : -1;
    if (threadIdx.x == 0) a.count[seq] = depth + 1;
  }
  if (!(total > 0.0 && total < __builtin_inf())) {
    if (chunk == 0 && threadIdx.x == 0) a.next[seq] = -1;
    return;
  }
  // The stretch, then the wave's part of it, then the step, lane and entry at
  // which the sum of weights passes the goal; where rounding keeps it below, the
  // last with weight.  pass_at: of the lanes' sums, which come behind `before`, the
  // one that passes, and what comes before that.
  const double goal = (double)s_u[0] * total;
  double before = 0.0;
  bool passed, some;
  auto pass_at = [&](double v) {
    const double upto = wave_scan_d(v);
    const uint64_t with = __builtin_amdgcn_ballot_w64(v > 0.0), hit = __builtin_amdgcn_ballot_w64(v > 0.0 && before + upto > goal);
    passed = hit != 0, some = with != 0;
    const int who = hit ? __builtin_ctzll(hit) : some ? 63 - __builtin_clzll(with) : 0;
    before += lane_value_d(upto - v, who);
    return who;
  };
  if (a.clusters > 1 && pass_at(lane < a.clusters ? s_chunk[lane] : 0.0) != chunk) return;
  const int part = pass_at(lane < kVerifyWaves ? s_own[lane] : 0.0);
  int first, steps;
  part_of(chunk, part, first, steps);
  // a step a wave, in rounds; the last round with weight again if none passes
  int last_t = -1;
  double last_before = before;
  bool forced = false;
  for (int t = 0;;) {
    double w[kRow] = {}, mine = 0.0;
    int i = 0;
    if (t + wave < steps) {
      steps_of(std::integral_constant<int, 1>(), first + t + wave, first + t + wave + 1, [&](int from, const double (&v)[kRow]) {
        i = from;
#pragma unroll
        for (int k = 0; k < kRow; ++k) w[k] = v[k];
        mine = sum_of(v);
      });
    }
    const double upto = wave_scan_d(mine);
    __syncthreads();   // s_wave is free
    if (lane == kWave - 1) s_wave[wave] = upto;
    __syncthreads();
    const double sum = lane < kVerifyWaves ? s_wave[lane] : 0.0, start = before;
    const int who = pass_at(sum);
    if (some) last_t = t, last_before = start;
    if (passed || forced) {
      if (who != wave) return;
      const int at = pass_at(mine);
      double run = before;   // of lane `at`; others' are not looked at
      int found = -1, last = -1;
#pragma unroll
      for (int k = 0; k < kRow; ++k) {
        run += w[k];
        if (w[k] > 0.0) {
          last = i + k;
          if (found < 0 && run > goal) found = i + k;
        }
      }
      const int next = lane_value(found >= 0 ? found : last, at);
      if (lane == 0) a.next[seq] = next;
      return;
    }
    before = start + lane_value_d(wave_scan_d(sum), kWave - 1);
    t += kVerifyWaves;
    if (t < steps) continue;
    if (last_t < 0) return;   // not with weights whose sum is positive
    t = last_t, before = last_before, forced = true;
  }
}

}  // namespace

hipError_t launch_draft_tree(const DraftTreeArgs &a, hipStream_t s) {
  const int threads = a.words <= 2 ? 64 : 32 * a.words;   // a token each, in whole blocks
  hipLaunchKernelGGL(draft_tree_kernel, dim3((unsigned)a.seqs), dim3((unsigned)threads), 0, s, a);
  return hipGetLastError();
}

// Workgroups that share a sequence's rows, one a compute unit at most.  A pass of
// one workgroup costs some 2 us and 0.09 for each 1024 entries (fp32, 131072: 13
// us); shared by eight 5.3 us, half of it for hearing of the others, and the call a
// launch that clears what they tell each other through.  A walk's passes past the
// first kVerifyPasses are no longer shared: every workgroup works out all of such a
// row, 20 us a pass.  (With 16 shared ones a root that refuses 60 children took 959
// us, with 128 320; the clearing launch takes the same.)
int verify_clusters(int seqs, int vocab) {
  if (vocab < 65536) return 1;
  const int fill = 256 / seqs, most = vocab / 16384;
  const int n = fill < most ? fill : most;
  return n < 1 ? 1 : n > kMaxClusters ? kMaxClusters : n;
}

hipError_t launch_verify_drafts(const VerifyArgs &a, bool f32, hipStream_t s) {
  if (a.clusters > 1) {
    const int n = a.seqs * kVerifyPasses * a.clusters;
    hipLaunchKernelGGL(verify_clear_kernel, dim3((unsigned)((n + 255) / 256)), dim3(256), 0, s, a.slots, n);
  }
  const dim3 grid((unsigned)a.seqs * a.clusters), block(kVerifyThreads);
  if (a.q) {
    if (f32) hipLaunchKernelGGL((verify_drafts_kernel<float, true>), grid, block, 0, s, a);
    else hipLaunchKernelGGL((verify_drafts_kernel<uint16_t, true>), grid, block, 0, s, a);
  } else {
    if (f32) hipLaunchKernelGGL((verify_drafts_kernel<float, false>), grid, block, 0, s, a);
    else hipLaunchKernelGGL((verify_drafts_kernel<uint16_t, false>), grid, block, 0, s, a);
  }
  return hipGetLastError();
}

}  // namespace moe
