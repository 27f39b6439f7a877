// Writing to and reading from a paged cache of keys and values in 4 bits.
//
// A group is 32 consecutive dimensions of one token's key or value.  With
// lo = min(0, min x) and hi = max(0, max x) its scale is the smallest
//   scale(k) = (8 + k % 8) * 2^(k / 8 - 24),  0 <= k <= 254,
// that spans hi - lo in 15 steps (the largest one where none does), its zero
// z = round(-lo / scale) and its codes q = round(x / scale) + z, both clipped
// to 0 .. 15 (round half to even); it stands for (q - z) * scale.  A scale has
// 4 significant bits and q - z has 4, so every value has at most 8 and is a
// multiple of 2^-24: exact in bf16 and in fp16 alike, which is what lets the
// attention kernels multiply cache entries on the matrix cores without another
// rounding.  The scale grid costs at most an eighth of a step's width against
// the finest scale.  A group that holds an infinity or a NaN cannot be stored;
// k = 255 marks it and it reads as NaN.
//
// The record of one kv head's P tokens (P * D * 9 / 8 bytes):
//   key codes    [P][D / 2]           dimension c in nibble c % 2 of byte c / 2
//   value codes  [P / 4][D / 8][4]    uint32: eight dimensions of each of four tokens
//   key metas    [P][D / 32]          uint16 k << 8 | z
//   value metas  [P / 4][D / 32][4]   uint16
// Keys lie token by token because scores sum over dimensions; values in blocks
// of four tokens because outputs sum over tokens, so a lane of the attention
// kernels finds the tokens it multiplies side by side.  Each token's bytes are
// its own: appending writes without reading.
#include "common.hpp"

namespace moe {
namespace {

constexpr int kThreads = 256;

__device__ __forceinline__ float group_scale(int k) { return __uint_as_float((uint32_t)(k + 848) << 20); }

// The sequence that new token t belongs to: the last b with q_start[b] <= t.
__device__ __forceinline__ int sequence_of(const Kv4 &kv, int t) {
  int lo = 0, hi = kv.seqs - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (kv.q_start[mid] <= t) lo = mid;
    else hi = mid - 1;
  }
  return lo;
}

__device__ __forceinline__ int position_of(const Kv4 &kv, int seq, int t) {
  return kv.kv_len[seq] - kv.q_start[seq + 1] + t;
}

// The record that holds position pos of a sequence for one head; nullptr where
// the table names no page of the pool.
template <int D>
__device__ __forceinline__ uint8_t *record_of(const Kv4 &kv, int seq, int pos, int head) {
  if (pos < 0) return nullptr;
  const int col = pos >> kv.page_log2;
  if (col >= kv.table_cols) return nullptr;
  const int page = kv.page_table[seq * kv.table_stride + col];
  if (page < 0 || page >= kv.pages) return nullptr;
  return kv.pool + ((size_t)page * kv.kv_heads + head) * ((size_t)(D * 9 / 8) << kv.page_log2);
}

// Byte offsets of the codes of dimensions 8 o .. 8 o + 7 and of the meta of
// group g of the page's token t.
template <int D>
__device__ __forceinline__ size_t code_at(const Kv4 &kv, bool value, int t, int o) {
  return value ? ((size_t)(D / 2) << kv.page_log2) + (size_t)(t >> 2) * (2 * D) + o * 16 + (t & 3) * 4
               : (size_t)t * (D / 2) + o * 4;
}
template <int D>
__device__ __forceinline__ size_t meta_at(const Kv4 &kv, bool value, int t, int g) {
  const size_t metas = (size_t)D << kv.page_log2;
  return value ? metas + ((size_t)(D / 16) << kv.page_log2) + (size_t)(t >> 2) * (D / 4) + g * 8 + (t & 3) * 2
               : metas + (size_t)t * (D / 16) + g * 2;
}

// D / 8 lanes take one head's vector of one token, a lane eight dimensions.
// Items are (token, head), the query, key and value heads of a token in a row.
// Rotation and quantisation round after each operation (no contraction), so
// that codes do not depend on how an expression was compiled.  A token's bytes
// pass once, so HBM bounds it: 4098 tokens of 16 heads of 128 in fp32 take 31
// us, and reading them back in fp32 18.  A few tokens take the launch.
// AT: rotated for positions of the caller's.
template <int D, typename T, bool AT>
__global__ __launch_bounds__(kThreads) void kv4_append_kernel(KvAppendArgs a) {
#pragma clang fp contract(off)
  constexpr int kLanes = D / 8;
  const int slots = a.heads + 2 * a.kv.kv_heads;
  const int64_t item = ((int64_t)blockIdx.x * kThreads + threadIdx.x) / kLanes;
  const int o = threadIdx.x % kLanes;
  if (item >= (int64_t)a.kv.tokens * slots) return;
  const int t = (int)(item / slots), slot = (int)(item % slots);
  const int seq = sequence_of(a.kv, t), pos = position_of(a.kv, seq, t);
  const bool query = slot < a.heads, value = slot >= a.heads + a.kv.kv_heads;
  const int head = query ? slot : slot - a.heads - (value ? a.kv.kv_heads : 0);
  const T *src = query   ? static_cast<const T *>(a.q) + t * a.q_stride
                 : value ? static_cast<const T *>(a.v) + t * a.v_stride
                         : static_cast<const T *>(a.k) + t * a.k_stride;
  src += head * D;
  float x[8];
  load8(src + 8 * o, x);
  const int turn = AT ? a.pos[t] : pos;   // the position that it is rotated for
  const bool placed = pos >= 0 && turn >= 0 && turn < a.max_pos;
  if (!value && 8 * o < a.rot && placed) {
    const int half = a.rot / 2, i = 8 * o < half ? 8 * o : 8 * o - half;
    float other[8], c[8], s[8];
    load8(src + (8 * o < half ? 8 * o + half : 8 * o - half), other);
    load8(a.cos + (size_t)turn * half + i, c);
    load8(a.sin + (size_t)turn * half + i, s);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const float p = x[e] * c[e], r = other[e] * s[e];
      x[e] = 8 * o < half ? p - r : p + r;
    }
  }
  if (query) {
    if (!placed) {
#pragma unroll
      for (int e = 0; e < 8; ++e) x[e] = 0.0f;
    }
    store8(static_cast<T *>(a.q_out) + t * a.q_out_stride + head * D + 8 * o, x);
    return;
  }
  // the group's range, over the four lanes that share it
  bool fine = true;
  float lo = 0.0f, hi = 0.0f;
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    fine &= fabsf(x[e]) < __builtin_inff();
    lo = fminf(lo, x[e]);
    hi = fmaxf(hi, x[e]);
  }
  int bad = !fine;
#pragma unroll
  for (int m = 1; m <= 2; m <<= 1) {
    lo = fminf(lo, __shfl_xor(lo, m, kWave));
    hi = fmaxf(hi, __shfl_xor(hi, m, kWave));
    bad |= __shfl_xor(bad, m, kWave);
  }
  uint8_t *rec = placed ? record_of<D>(a.kv, seq, pos, head) : nullptr;
  if (!rec) return;
  int k = 255, z = 0;
  uint32_t w = 0;
  if (!bad) {
    // a fifteenth of the range, rounded, lies less than a step of the scale
    // grid off: its code rounded down, or the next one
    const float range = hi - lo;
    k = min(max((int)(__float_as_uint(range * (1.0f / 15.0f)) >> 20) - 848, 0), 254);
    if (15.0f * group_scale(k) < range) k = min(k + 1, 254);
    const float scale = group_scale(k);
    const float zf = fminf(fmaxf(rintf(-lo / scale), 0.0f), 15.0f);
    z = (int)zf;
#pragma unroll
    for (int e = 0; e < 8; ++e) w |= (uint32_t)(int)fminf(fmaxf(rintf(x[e] / scale) + zf, 0.0f), 15.0f) << (4 * e);
  }
  const int in_page = pos & ((1 << a.kv.page_log2) - 1);
  *reinterpret_cast<uint32_t *>(rec + code_at<D>(a.kv, value, in_page, o)) = w;
  if (o % 4 == 0) *reinterpret_cast<uint16_t *>(rec + meta_at<D>(a.kv, value, in_page, o / 4)) = (uint16_t)(k << 8 | z);
}

// The stored values of the same tokens; zeros where nothing is stored.
template <int D, typename T>
__global__ __launch_bounds__(kThreads) void kv4_read_kernel(KvReadArgs a) {
  constexpr int kLanes = D / 8;
  const int slots = 2 * a.kv.kv_heads;
  const int64_t item = ((int64_t)blockIdx.x * kThreads + threadIdx.x) / kLanes;
  const int o = threadIdx.x % kLanes;
  if (item >= (int64_t)a.kv.tokens * slots) return;
  const int t = (int)(item / slots), slot = (int)(item % slots);
  const int seq = sequence_of(a.kv, t), pos = position_of(a.kv, seq, t);
  const bool value = slot >= a.kv.kv_heads;
  const int head = slot - (value ? a.kv.kv_heads : 0);
  const uint8_t *rec = record_of<D>(a.kv, seq, pos, head);
  float x[8] = {};
  if (rec) {
    const int in_page = pos & ((1 << a.kv.page_log2) - 1);
    const uint32_t w = *reinterpret_cast<const uint32_t *>(rec + code_at<D>(a.kv, value, in_page, o));
    const uint32_t meta = *reinterpret_cast<const uint16_t *>(rec + meta_at<D>(a.kv, value, in_page, o / 4));
    const float scale = (meta >> 8) == 255 ? __builtin_nanf("") : group_scale((int)(meta >> 8));
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = (float)((int)(w >> (4 * e) & 15) - (int)(meta & 255)) * scale;
  }
  T *out = static_cast<T *>(value ? a.v : a.k);
  store8(out + ((int64_t)t * a.kv.kv_heads + head) * D + 8 * o, x);
}

// Entry base + path[k] of a sequence to base + k, k below count, base its first
// new place; one workgroup a cache and sequence, D / 8 lanes an entry, and as many
// heads at once as the kept entries leave lanes.  Every group of entries is read
// whole before it is written.  Paths that do not go back (path[k] > k; other entries
// stay) let groups go in order: what a group reads lies past its own first
// place, and earlier groups wrote in front of that.  The loads bound it, three that
// each need the one before: path, page, entry.  32 layers of 32 sequences: 5.4 to 7 us a call, one
// head after another 9.
template <int D>
__global__ __launch_bounds__(kThreads) void kv4_keep_kernel(KvKeepArgs a) {
  constexpr int kLanes = D / 8, kItems = kThreads / kLanes, kAhead = 4;
  const int seq = blockIdx.x, o = threadIdx.x % kLanes, item = threadIdx.x / kLanes;
  Kv4 kv = a.kv;
  kv.pool = a.pools[blockIdx.y];
  const int start = min(max(kv.q_start[seq], 0), kv.tokens), end = min(max(kv.q_start[seq + 1], start), kv.tokens);
  const int n = end - start, kept = min(a.count[seq], n), base = kv.kv_len[seq] - n, mask = (1 << kv.page_log2) - 1;
  if (kept <= 1) return;   // the first stays in any case
  // entries of a group, a power of two; heads of a step, kAhead steps at a time
  const int group = kept >= kItems ? kItems : 1 << (32 - __builtin_clz(kept - 1)), heads = kItems / group;
  for (int k0 = 0; k0 < kept; k0 += group) {
    const int k = k0 + item % group, source = k < kept ? a.path[start + k] : 0;
    const bool moves = k < kept && source > k && source < n;
    const int in = (base + source) & mask, in_to = (base + k) & mask;
    for (int h0 = item / group; h0 - item / group < kv.kv_heads; h0 += heads * kAhead) {
      uint8_t *to[kAhead];
      uint32_t codes[kAhead][2];
      uint16_t metas[kAhead][2];
#pragma unroll
      for (int x = 0; x < kAhead; ++x) {
        const int head = h0 + x * heads;
        uint8_t *from = nullptr;
        to[x] = nullptr;
        if (moves && head < kv.kv_heads) {
          from = record_of<D>(kv, seq, base + source, head);
          to[x] = from ? record_of<D>(kv, seq, base + k, head) : nullptr;
        }
        if (!to[x]) continue;
#pragma unroll
        for (int v = 0; v < 2; ++v) {
          codes[x][v] = *reinterpret_cast<const uint32_t *>(from + code_at<D>(kv, v, in, o));
          metas[x][v] = *reinterpret_cast<const uint16_t *>(from + meta_at<D>(kv, v, in, o / 4));
        }
      }
      __syncthreads();
#pragma unroll
      for (int x = 0; x < kAhead; ++x) {
        if (!to[x]) continue;
#pragma unroll
        for (int v = 0; v < 2; ++v) {
          *reinterpret_cast<uint32_t *>(to[x] + code_at<D>(kv, v, in_to, o)) = codes[x][v];
          if (o % 4 == 0) *reinterpret_cast<uint16_t *>(to[x] + meta_at<D>(kv, v, in_to, o / 4)) = metas[x][v];
        }
      }
    }
    __syncthreads();   // written before the next group reads
  }
}

template <int D>
unsigned blocks(int64_t items) {
  return (unsigned)((items * (D / 8) + kThreads - 1) / kThreads);
}

template <int D, typename T>
void append(const KvAppendArgs &a, hipStream_t s) {
  const dim3 grid(blocks<D>((int64_t)a.kv.tokens * (a.heads + 2 * a.kv.kv_heads)));
  if (a.pos) hipLaunchKernelGGL((kv4_append_kernel<D, T, true>), grid, dim3(kThreads), 0, s, a);
  else hipLaunchKernelGGL((kv4_append_kernel<D, T, false>), grid, dim3(kThreads), 0, s, a);
}

}  // namespace

hipError_t launch_kv4_append(const KvAppendArgs &a, int head_dim, bool f32, hipStream_t s) {
  if (head_dim == 64) {
    if (f32) append<64, float>(a, s);
    else append<64, uint16_t>(a, s);
  } else {
    if (f32) append<128, float>(a, s);
    else append<128, uint16_t>(a, s);
  }
  return hipGetLastError();
}

hipError_t launch_kv4_keep(const KvKeepArgs &a, int pools, int head_dim, hipStream_t s) {
  const dim3 grid((unsigned)a.kv.seqs, (unsigned)pools);
  if (head_dim == 64) hipLaunchKernelGGL((kv4_keep_kernel<64>), grid, dim3(kThreads), 0, s, a);
  else hipLaunchKernelGGL((kv4_keep_kernel<128>), grid, dim3(kThreads), 0, s, a);
  return hipGetLastError();
}

hipError_t launch_kv4_read(const KvReadArgs &a, int head_dim, bool f32, hipStream_t s) {
  const int64_t items = (int64_t)a.kv.tokens * 2 * a.kv.kv_heads;
  if (head_dim == 64) {
    if (f32) hipLaunchKernelGGL((kv4_read_kernel<64, float>), dim3(blocks<64>(items)), dim3(kThreads), 0, s, a);
    else hipLaunchKernelGGL((kv4_read_kernel<64, uint16_t>), dim3(blocks<64>(items)), dim3(kThreads), 0, s, a);
  } else {
    if (f32) hipLaunchKernelGGL((kv4_read_kernel<128, float>), dim3(blocks<128>(items)), dim3(kThreads), 0, s, a);
    else hipLaunchKernelGGL((kv4_read_kernel<128, uint16_t>), dim3(blocks<128>(items)), dim3(kThreads), 0, s, a);
  }
  return hipGetLastError();
}

}  // namespace moe
