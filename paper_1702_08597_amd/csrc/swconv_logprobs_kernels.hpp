// HIP kernels of the log probabilities at a network's end.  For a row of scores x_j:
//   m = max x_j,  s = sum exp(x_j - m),  ls = log s,  log p_j = (x_j - m) - ls,  H = -sum p_j log p_j
// and H = ls - (sum (x_j - m) exp(x_j - m)) / s, whose two terms are both positive.  One pass over the scores: every lane
// keeps the largest score it has seen and both sums relative to it, scaled when that one changes; lanes, waves and
// parts of a row are joined in the same way.  All of it in fp32 whatever the scores' type.
//   d x_j = g ([j = label] - p_j) - h p_j (log p_j + H)
// A class of score -inf is masked: exp gives 0, and it never is among the best.  NaN and +inf make the row's largest
// score NaN or +inf (the maximum used propagates NaN), from which the row's results are made NaN.
// The best t classes, t <= 64: lane i of a wave holds its i-th best as a 64-bit key (score, then the lower class), a
// score that beats the t-th goes to a list in LDS, and lists of 64 are sorted and merged.
#pragma once
#include "swconv_elements.hpp"

namespace swconv {

constexpr int kLogpThreads = 256;
constexpr int kLogpUnroll = 2;        // 16-byte loads per lane in flight and tile
constexpr int kTopMax = 64;           // one lane each
constexpr float kFarBelow = -256.0f;  // exp(-256) is 0 in fp32; keeps 0 * inf out of the sums
constexpr float kLog2e = 1.44269504088896340736f, kLn2 = 0.693147180559945309417f;

template <Elem E>
constexpr int kLogpVec = 16 / sizeof(elem_t<E>);

struct RowSums {
  float m, s, t;  // largest score, sum of exp(x - m), sum of (x - m) exp(x - m)
};
constexpr float kLowest = -3.402823466e38f;

__device__ __forceinline__ float exp_fast(float x) { return __builtin_amdgcn_exp2f(x * kLog2e); }

__device__ __forceinline__ void rescale(RowSums& a, float m) {
  const float d = fmaxf(a.m - m, kFarBelow), f = exp_fast(d);
  a.t = f * (a.t + d * a.s);
  a.s *= f;
  a.m = m;
}
__device__ __forceinline__ RowSums join(RowSums a, RowSums b) {
  const float m = __builtin_elementwise_maximum(a.m, b.m);
  rescale(a, m);
  rescale(b, m);
  return {m, a.s + b.s, a.t + b.t};
}
__device__ __forceinline__ RowSums join_lanes(RowSums a) {
#pragma unroll
  for (int off = 32; off; off /= 2) a = join(a, {__shfl_xor(a.m, off), __shfl_xor(a.s, off), __shfl_xor(a.t, off)});
  return a;
}

// ---- the best classes -------------------------------------------------------------------------------------------
using TopKey = uint64_t;  // 0: none

__device__ __forceinline__ TopKey top_key(float x, int32_t index) {
  const uint32_t b = __float_as_uint(x + 0.0f);  // -0 counts as 0
  return (uint64_t)(b & 0x80000000u ? ~b : b | 0x80000000u) << 32 | (uint32_t)~index;
}
__device__ __forceinline__ float top_score(TopKey k) {
  const uint32_t o = (uint32_t)(k >> 32);
  return k ? __uint_as_float(o & 0x80000000u ? o & 0x7fffffffu : ~o) : -INFINITY;
}
__device__ __forceinline__ int32_t top_index(TopKey k) { return k ? (int32_t)~(uint32_t)k : -1; }

template <typename K>
__device__ __forceinline__ K exchange(K key, int off, bool keep_larger) {
  const K other = __shfl_xor(key, off);
  return keep_larger ? (other > key ? other : key) : (other < key ? other : key);
}
// 64 keys, one per lane, into descending order
template <typename K>
__device__ __forceinline__ K sort_lanes(K key, int lane) {
#pragma unroll
  for (int size = 2; size <= 64; size *= 2)
#pragma unroll
    for (int off = size / 2; off; off /= 2) key = exchange(key, off, ((lane & off) == 0) == ((lane & size) == 0));
  return key;
}
// the 64 largest of two descending lists, descending
__device__ __forceinline__ TopKey merge_lanes(TopKey a, TopKey b, int lane) {
  const TopKey mirrored = __shfl_xor(b, 63);
  TopKey key = a > mirrored ? a : mirrored;
#pragma unroll
  for (int off = 32; off; off /= 2) key = exchange(key, off, (lane & off) == 0);
  return key;
}

struct TopList {
  TopKey best;        // lane i: the i-th best so far
  TopKey* waiting;    // LDS, 128
  int count;          // of them
  float score;        // what a score has to beat: the t-th best's,
  int32_t index;      // or equal it at a lower class

  __device__ __forceinline__ void start(TopKey* lds) {
    best = 0;
    waiting = lds;
    count = 0;
    score = -INFINITY;
    index = -1;
  }
  __device__ __forceinline__ void take(int lane, int top) {
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    const int n = min(count, 64);
    best = merge_lanes(best, sort_lanes(lane < n ? waiting[lane] : (TopKey)0, lane), lane);
    const TopKey rest = lane < count - 64 ? waiting[64 + lane] : (TopKey)0;
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    if (lane < count - 64) waiting[lane] = rest;
    count -= n;
    const TopKey bar = __shfl(best, top - 1);
    if (bar) {
      score = top_score(bar);
      index = top_index(bar);
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  }
  // one score from each lane
  __device__ __forceinline__ void offer(float x, int32_t j, int lane, int top) {
    const bool hit = x > score || (x == score && j < index);
    const uint64_t hits = __ballot(hit);
    if (hits == 0) return;
    if (hit) waiting[count + __builtin_amdgcn_mbcnt_hi((uint32_t)(hits >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)hits, 0))] = top_key(x, j);
    count += __popcll(hits);
    if (count >= 64) take(lane, top);
  }
};

// ---- forward ----------------------------------------------------------------------------------------------------
struct LogprobsOut {
  float *logprob, *entropy, *stats;
  int32_t* top_class;
  float* top_logprob;
};

// A row's results from its sums and its best classes; called by one wave.
template <Elem E>
__device__ __forceinline__ void finish_row(const LogprobsOut& out, const elem_t<E>* scores, int64_t row_stride, int64_t classes,
                                           const int32_t* labels, int64_t row, RowSums a, TopKey best, int top, int lane) {
  const bool poisoned = !(a.m <= -kLowest);  // NaN or +inf among the scores
  const bool empty = a.s == 0.0f && !poisoned;
  const float ls = empty ? 0.0f : poisoned ? NAN : logf(a.s);
  const float m = empty ? -INFINITY : poisoned ? NAN : a.m;
  if (lane == 0) {
    if (out.logprob) {
      const int32_t label = labels[row];
      float lp = NAN;
      if (label < 0)
        lp = 0.0f;
      else if (label < classes)
        lp = empty ? -INFINITY : ((float)scores[row * row_stride + label] - m) - ls;
      out.logprob[row] = lp;
    }
    if (out.entropy) out.entropy[row] = empty ? 0.0f : poisoned ? NAN : ls - a.t / a.s;
    if (out.stats) {
      out.stats[2 * row] = m;
      out.stats[2 * row + 1] = ls;
    }
  }
  if (lane < top) {
    out.top_class[row * top + lane] = poisoned ? -1 : top_index(best);
    out.top_logprob[row * top + lane] = poisoned ? NAN : best ? (top_score(best) - m) - ls : -INFINITY;
  }
}

// Parts of rows whose results wait for their join, in the workspace.
struct PartSums {
  float m, s, t, unused;
};

// WAVES waves of a workgroup share a part of a row, tile by tile (a tile: kLogpUnroll 16-byte loads from each lane).
template <Elem E, int WAVES, bool TOP, bool ENTROPY>
__global__ __launch_bounds__(kLogpThreads) void logprobs_kernel(int64_t rows, int64_t classes, const elem_t<E>* __restrict__ scores,
                                                                int64_t row_stride, const int32_t* __restrict__ labels, int top,
                                                                int parts, int64_t part_classes, LogprobsOut out,
                                                                PartSums* __restrict__ part_sums, TopKey* __restrict__ part_keys) {
  constexpr int V = kLogpVec<E>, U = kLogpUnroll, kWaves = kLogpThreads / 64, kTile = 64 * V * U;
  __shared__ TopKey lists[TOP ? kWaves : 1][128];
  __shared__ RowSums wave_sums[kWaves];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, part_wave = wave % WAVES;
  constexpr int kPartsPerGroup = kWaves / WAVES;
  const int64_t n_parts = rows * parts;
  for (int64_t group = blockIdx.x; group * kPartsPerGroup < n_parts; group += gridDim.x) {
    const int64_t id = group * kPartsPerGroup + wave / WAVES;
    RowSums a{kLowest, 0.0f, 0.0f};
    TopList list;
    if constexpr (TOP) list.start(lists[wave]);
    const int64_t row = parts == 1 ? id : id / parts;
    if (id < n_parts) {
      const int64_t begin = parts == 1 ? 0 : (id - row * parts) * part_classes;
      const int64_t end = min(classes, begin + part_classes);
      const elem_t<E>* x_row = scores + row * row_stride;
      for (int64_t tile = begin + (int64_t)part_wave * kTile; tile < end; tile += (int64_t)WAVES * kTile) {
        Pack<E, V> raw[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
          const int64_t j = tile + (u * 64 + lane) * V;
          if (j + V <= end)
            raw[u] = load_pack<E, V>(x_row + j);
          else
            raw[u] = load_part<E, V>(x_row + j, (int)max((int64_t)0, end - j), -INFINITY);
        }
        float group_max[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
          group_max[u] = (float)raw[u].v[0];
#pragma unroll
          for (int i = 1; i < V; ++i) group_max[u] = __builtin_elementwise_maximum(group_max[u], (float)raw[u].v[i]);
        }
        float m = a.m;
#pragma unroll
        for (int u = 0; u < U; ++u) m = __builtin_elementwise_maximum(m, group_max[u]);
        rescale(a, m);
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
          for (int i = 0; i < V; ++i) {
            const float d = fmaxf((float)raw[u].v[i] - m, kFarBelow), e = exp_fast(d);
            a.s += e;
            if constexpr (ENTROPY) a.t += d * e;
          }
        if constexpr (TOP) {
#pragma unroll
          for (int u = 0; u < U; ++u)
            if (__ballot(group_max[u] >= list.score))
#pragma unroll
              for (int i = 0; i < V; ++i) list.offer((float)raw[u].v[i], (int32_t)(tile + (u * 64 + lane) * V + i), lane, top);
        }
      }
    }
    a = join_lanes(a);
    if constexpr (TOP) list.take(lane, top);
    if constexpr (WAVES > 1) {
      static_assert(WAVES == kWaves, "one part per workgroup");
      if (lane == 0) wave_sums[wave] = a;
      if constexpr (TOP) lists[wave][lane] = list.best;
      __syncthreads();
      if (wave == 0) {
        for (int w = 1; w < WAVES; ++w) {
          a = join(a, wave_sums[w]);
          if constexpr (TOP) list.best = merge_lanes(list.best, lists[w][lane], lane);
        }
      }
      __syncthreads();
    }
    if (part_wave == 0 && id < n_parts) {
      if (parts == 1) {
        finish_row<E>(out, scores, row_stride, classes, labels, row, a, TOP ? list.best : 0, top, lane);
      } else {
        if (lane == 0) part_sums[id] = {a.m, a.s, a.t, 0.0f};
        if constexpr (TOP)
          if (lane < top) part_keys[id * top + lane] = list.best;
      }
    }
  }
}

// Joins the parts of a row: a wave per row.
template <Elem E>
__global__ __launch_bounds__(64) void logprobs_join_kernel(int64_t rows, int64_t classes, const elem_t<E>* __restrict__ scores,
                                                           int64_t row_stride, const int32_t* __restrict__ labels, int top, int parts,
                                                           LogprobsOut out, const PartSums* __restrict__ part_sums,
                                                           const TopKey* __restrict__ part_keys) {
  const int lane = threadIdx.x;
  for (int64_t row = blockIdx.x; row < rows; row += gridDim.x) {
    RowSums a{kLowest, 0.0f, 0.0f};
    for (int p = lane; p < parts; p += 64) {
      const PartSums b = part_sums[row * parts + p];
      a = join(a, {b.m, b.s, b.t});
    }
    a = join_lanes(a);
    TopKey best = 0;
    if (top)
      for (int p = 0; p < parts; ++p)
        best = merge_lanes(best, lane < top ? part_keys[(row * parts + p) * top + lane] : (TopKey)0, lane);
    finish_row<E>(out, scores, row_stride, classes, labels, row, a, best, top, lane);
  }
}

// ---- backward ---------------------------------------------------------------------------------------------------
// `across` threads (a power of two) share a row or, of a long row, a chunk; a thread takes one 16-byte group.
template <Elem E>
__global__ __launch_bounds__(kLogpThreads) void logprobs_grad_kernel(int64_t rows, int64_t classes, const elem_t<E>* scores,
                                                                     int64_t row_stride, const int32_t* __restrict__ labels,
                                                                     const float* __restrict__ stats, const float* __restrict__ entropy,
                                                                     const float* __restrict__ dlogprob,
                                                                     const float* __restrict__ dentropy, int across_shift,
                                                                     int64_t chunks, elem_t<E>* out, int64_t out_stride) {
  constexpr int V = kLogpVec<E>;
  const int across = 1 << across_shift, down = kLogpThreads >> across_shift;
  const int64_t turns = (rows + down - 1) / down * chunks;
  for (int64_t turn = blockIdx.x; turn < turns; turn += gridDim.x) {
    const int64_t row0 = chunks == 1 ? turn : turn / chunks;
    const int64_t row = row0 * down + (threadIdx.x >> across_shift);
    const int64_t j = ((turn - row0 * chunks) * across + (threadIdx.x & (across - 1))) * V;
    if (row >= rows || j >= classes) continue;
    const float m = stats[2 * row], ls = stats[2 * row + 1];
    const int32_t label = labels ? labels[row] : -1;
    float g = 0.0f;
    if (dlogprob && label >= 0) g = label < classes ? dlogprob[row] : NAN;
    const float h = dentropy ? dentropy[row] : 0.0f, H = dentropy ? entropy[row] : 0.0f;
    const bool empty = m == -INFINITY;
    const elem_t<E>* x_row = scores + row * row_stride + j;
    const int n = (int)min((int64_t)V, classes - j);
    const Pack<E, V> x = n == V ? load_pack<E, V>(x_row) : load_part<E, V>(x_row, n, -INFINITY);
    Pack<E, V> dx;
#pragma unroll
    for (int i = 0; i < V; ++i) {
      const float xi = (float)x.v[i];
      const float lp = fmaxf(xi - m, kFarBelow) - ls;  // far below p is 0
      const float p = exp_fast(lp);
      float d = -p * (g + h * (lp + H));
      if (j + i == label) d += g;
      if (m != m) d = NAN;
      dx.v[i] = (elem_t<E>)(empty || xi == -INFINITY ? 0.0f : d);
    }
    if (n == V)
      store_pack<E, V>(out + row * out_stride + j, dx);
    else
      store_part<E, V>(out + row * out_stride + j, n, dx);
  }
}

}  // namespace swconv
