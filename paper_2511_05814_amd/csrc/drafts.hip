// Trees of drafted tokens: their plan, and their verification against the
// target's probabilities.
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
constexpr int kPlanThreads = 256;
__global__ __launch_bounds__(kPlanThreads) void draft_tree_kernel(DraftTreeArgs a) {
  __shared__ int16_t s_parent[kMaxTree];
  const int seq = blockIdx.x;
  const Tree tree = tree_of(a.q_start, seq, a.tokens);
  const int n = min(tree.n, 32 * a.words), first = a.kv_len[seq] - tree.n;
  for (int i = threadIdx.x; i < n; i += kPlanThreads) {
    const int p = a.parent[tree.start + i];
    s_parent[i] = (int16_t)(p >= 0 && p < i ? p : -1);
  }
  __syncthreads();
  for (int i = threadIdx.x; i < tree.n; i += kPlanThreads) {
    uint32_t *row = a.seen + (int64_t)(tree.start + i) * a.words;
    int depth = -1, x = i < n ? i : -1;
    for (int w = a.words - 1; w >= 0; --w) {
      uint32_t bits = 0;
      while (x >= 32 * w) {
        bits |= 1u << (x & 31);
        x = s_parent[x];
        ++depth;
      }
      row[w] = bits;
    }
    a.pos[tree.start + i] = i < n ? first + depth : -1;
  }
}

// Elements as fp32, the weight that is left of an entry once a share of the
// draft's is taken, NaN kept.
__device__ __forceinline__ float entry(const float *row, int64_t i) { return row[i]; }
__device__ __forceinline__ float entry(const uint16_t *row, int64_t i) { return __uint_as_float((uint32_t)row[i] << 16); }
__device__ __forceinline__ double positive(double v) { return v <= 0.0 ? 0.0 : v; }

// A walk down the tree of a sequence: cur's children in their order, each
// accepted with the probability that makes the accepted token, or the one drawn
// from what is left, one of the target's.
constexpr int kVerifyThreads = 1024;
template <typename T, bool DRAWN>
__global__ __launch_bounds__(kVerifyThreads) void verify_drafts_kernel(VerifyArgs a) {
  __shared__ int16_t s_parent[kMaxTree];
  __shared__ int32_t s_id[kMaxTree];
  __shared__ double s_part[kVerifyThreads / kWave];
  __shared__ int s_found;
  const int seq = blockIdx.x, lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
  const Tree tree = tree_of(a.q_start, seq, a.tokens);
  if (tree.n == 0) {
    if (threadIdx.x == 0) a.count[seq] = 0, a.next[seq] = -1;
    return;
  }
  const int n = min(tree.n, kMaxTree);
  for (int i = threadIdx.x; i < n; i += kVerifyThreads) {
    s_parent[i] = (int16_t)(i ? min(max(a.parent[tree.start + i], -1), kMaxTree) : -1);
    s_id[i] = a.ids[tree.start + i];
  }
  for (int i = threadIdx.x; i < tree.n; i += kVerifyThreads) a.path[tree.start + i] = i ? -1 : 0;
  __syncthreads();
  const T *p = nullptr, *q = nullptr;
  int cur = 0, depth = 0;

  auto total_of = [&](double v) {
    v = lane_value_d(wave_sum_d_to_lane63(v), 63);
    __syncthreads();
    if (lane == 0) s_part[wave] = v;
    __syncthreads();
    double sum = 0.0;
    for (int w = 0; w < kVerifyThreads / kWave; ++w) sum += s_part[w];
    return sum;
  };
  // whether id is a child of cur that was refused
  auto tried = [&](int id) {
    for (int c = cur + 1; c < n; ++c)
      if (s_parent[c] == cur && s_id[c] == id) return true;
    return false;
  };
  auto weight = [&](int id, double share) {
    if constexpr (DRAWN) return positive((double)entry(p, id) - share * (double)entry(q, id));
    else return positive(tried(id) ? 0.0 : (double)entry(p, id));
  };
  double share, left;
  for (;;) {
    p = static_cast<const T *>(a.p) + (int64_t)(tree.start + cur) * a.p_stride;
    if constexpr (DRAWN) q = static_cast<const T *>(a.q) + (int64_t)(tree.start + cur) * a.q_stride;
    share = 0.0, left = 1.0;
    int accepted = -1;
    bool stale = false;   // `left` is to be summed
    for (int c = cur + 1; c < n && accepted < 0; ++c) {
      if (s_parent[c] != cur) continue;
      if (stale) {
        double v = 0.0;
        for (int i = threadIdx.x; i < a.vocab; i += kVerifyThreads) v += weight(i, share);
        left = total_of(v);
        stale = false;
      }
      const int id = s_id[c];
      const bool inside = id >= 0 && id < a.vocab;
      const double u = fmax((double)a.u[tree.start + c], 0.0);
      if constexpr (DRAWN) {
        const double w = inside ? weight(id, share) : 0.0, guess = inside ? (double)entry(q, id) : 0.0;
        if (u * left * guess < w) accepted = c;
        else share += left, stale = true;
      } else {
        bool before = false;
        for (int e = cur + 1; e < c; ++e) before |= s_parent[e] == cur && s_id[e] == id;
        const double w = inside && !before ? positive((double)entry(p, id)) : 0.0;
        if (u * left < w) accepted = c;
        else left = positive(left - w);
      }
    }
    if (accepted < 0) break;
    cur = accepted;
    ++depth;
    if (threadIdx.x == 0) a.path[tree.start + depth] = cur;
  }
  // the next token from what is left, or, where that is nothing, from p itself
  bool whole = false;
  auto rest = [&](int id) { return whole ? positive((double)entry(p, id)) : weight(id, share); };
  double v = 0.0;
  for (int i = threadIdx.x; i < a.vocab; i += kVerifyThreads) v += rest(i);
  double total = total_of(v);
  if (total == 0.0) {
    whole = true;
    v = 0.0;
    for (int i = threadIdx.x; i < a.vocab; i += kVerifyThreads) v += rest(i);
    total = total_of(v);
  }
  int next = -1;
  if (total > 0.0 && total < __builtin_inf()) {
    const double goal = fmax((double)a.u[tree.start], 0.0) * total;
    double before = 0.0;
    int last = -1;
    for (int i0 = 0; i0 < a.vocab && next < 0; i0 += kVerifyThreads) {
      const int i = i0 + threadIdx.x;
      const double w = i < a.vocab ? rest(i) : 0.0;
      // running sum over the workgroup
      double run = w;
      for (int d = 1; d < kWave; d <<= 1) {
        const double other = __shfl_up(run, d, kWave);
        if (lane >= d) run += other;
      }
      __syncthreads();
      if (lane == kWave - 1) s_part[wave] = run;
      if (threadIdx.x == 0) s_found = a.vocab;
      __syncthreads();
      double ahead = before;
      for (int x = 0; x < kVerifyThreads / kWave; ++x) {
        if (x < wave) ahead += s_part[x];
        before += s_part[x];
      }
      if (w > 0.0 && ahead + run > goal) atomicMin(&s_found, i);
      __syncthreads();
      if (s_found < a.vocab) next = s_found;
      else if (w > 0.0) last = i;
    }
    if (next < 0) {   // rounding kept every sum below the goal: the last that has weight
      if (threadIdx.x == 0) s_found = -1;
      __syncthreads();
      atomicMax(&s_found, last);
      __syncthreads();
      next = s_found;
    }
  }
  if (threadIdx.x == 0) a.count[seq] = depth + 1, a.next[seq] = next;
}

}  // namespace

hipError_t launch_draft_tree(const DraftTreeArgs &a, hipStream_t s) {
  hipLaunchKernelGGL(draft_tree_kernel, dim3((unsigned)a.seqs), dim3(kPlanThreads), 0, s, a);
  return hipGetLastError();
}

hipError_t launch_verify_drafts(const VerifyArgs &a, bool f32, hipStream_t s) {
  const dim3 grid((unsigned)a.seqs), block(kVerifyThreads);
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
