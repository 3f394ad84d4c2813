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
#include <type_traits>
#include "swconv_elements.hpp"

namespace swconv {

constexpr int kLogpUnroll = 4;        // 16-byte loads per lane and tile
constexpr int kTopMax = 64;           // one lane each
constexpr float kFarBelow = -256.0f;  // exp(-256) is 0 in fp32; keeps 0 * inf out of the sums
constexpr float kLog2e = 1.44269504088896340736f, kLn2 = 0.693147180559945309417f;
constexpr float kLowest = -3.402823466e38f;

template <Elem E>
constexpr int kLogpVec = 16 / sizeof(elem_t<E>);

__device__ __forceinline__ float exp_fast(float x) { return __builtin_amdgcn_exp2f(x * kLog2e); }

// ---- lanes ------------------------------------------------------------------------------------------------------
// The value of lane ^ OFF by moves within the vector unit: a trip through LDS takes ten times as long.
template <int OFF>
__device__ __forceinline__ uint32_t lane_xor(uint32_t v, int lane) {
  auto dpp = [](uint32_t a, auto control) { return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)a, decltype(control)::value, 0xf, 0xf, true); };
  using std::integral_constant;
  if constexpr (OFF == 1) return dpp(v, integral_constant<int, 0xB1>{});         // quad_perm 1 0 3 2
  else if constexpr (OFF == 2) return dpp(v, integral_constant<int, 0x4E>{});    // quad_perm 2 3 0 1
  else if constexpr (OFF == 4) return dpp(dpp(v, integral_constant<int, 0x141>{}), integral_constant<int, 0x1B>{});  // 7, then 3
  else if constexpr (OFF == 7) return dpp(v, integral_constant<int, 0x141>{});   // row_half_mirror
  else if constexpr (OFF == 8) return dpp(v, integral_constant<int, 0x128>{});   // row_ror 8
  else if constexpr (OFF == 15) return dpp(v, integral_constant<int, 0x140>{});  // row_mirror
  else if constexpr (OFF == 16) {
    const auto s = __builtin_amdgcn_permlane16_swap(v, v, false, false);
    return lane & 16 ? s[0] : s[1];
  } else if constexpr (OFF == 32) {
    const auto s = __builtin_amdgcn_permlane32_swap(v, v, false, false);
    return lane & 32 ? s[0] : s[1];
  } else {
    static_assert(OFF == 63, "no such exchange");
    return lane_xor<32>(lane_xor<16>(lane_xor<15>(v, lane), lane), lane);
  }
}
template <int OFF>
__device__ __forceinline__ float lane_xor(float v, int lane) { return __uint_as_float(lane_xor<OFF>(__float_as_uint(v), lane)); }
template <int OFF>
__device__ __forceinline__ uint64_t lane_xor(uint64_t v, int lane) {
  return (uint64_t)lane_xor<OFF>((uint32_t)(v >> 32), lane) << 32 | lane_xor<OFF>((uint32_t)v, lane);
}
template <typename F>
__device__ __forceinline__ float reduce_lanes(float v, int lane, F&& f) {
  v = f(v, lane_xor<1>(v, lane));
  v = f(v, lane_xor<2>(v, lane));
  v = f(v, lane_xor<7>(v, lane));
  v = f(v, lane_xor<15>(v, lane));
  v = f(v, lane_xor<16>(v, lane));
  return f(v, lane_xor<32>(v, lane));
}

template <int OFF, typename K>
__device__ __forceinline__ K exchange(K key, int lane, bool keep_larger) {
  const K other = lane_xor<OFF>(key, lane);
  return (other > key) == keep_larger ? other : key;
}
template <int OFF, typename K>
__device__ __forceinline__ K halve(K key, int lane, bool down) {
  key = exchange<OFF>(key, lane, ((lane & OFF) == 0) == down);
  if constexpr (OFF > 1) key = halve<OFF / 2>(key, lane, down);
  return key;
}
// 64 keys, one per lane, into descending order
template <typename K>
__device__ __forceinline__ K sort_lanes(K key, int lane) {
  key = halve<1>(key, lane, (lane & 2) == 0);
  key = halve<2>(key, lane, (lane & 4) == 0);
  key = halve<4>(key, lane, (lane & 8) == 0);
  key = halve<8>(key, lane, (lane & 16) == 0);
  key = halve<16>(key, lane, (lane & 32) == 0);
  return halve<32>(key, lane, true);
}
// the 64 largest of two descending lists, descending
template <typename K>
__device__ __forceinline__ K merge_lanes(K a, K b, int lane) {
  const K mirrored = lane_xor<63>(b, lane);
  return halve<32>(a > mirrored ? a : mirrored, lane, true);
}

// ---- the sums of a row ------------------------------------------------------------------------------------------
// The scores that equal the largest one are counted, not added: a sum that starts at 1 would lose the digits of the
// others, which are all that is left of ls and H in a row with one likely class.
struct RowSums {
  float m;  // the largest score
  float n;  // how often
  float s;  // sum of exp(x - m) over the others
  float t;  // sum of (x - m) exp(x - m)
};

// Relative to a larger score m.
__device__ __forceinline__ RowSums raised(const RowSums& a, float m) {
  const float d = fmaxf(a.m - m, kFarBelow), f = exp_fast(d);
  return {m, 0.0f, f * (a.s + a.n), f * (a.t + d * (a.s + a.n))};
}
__device__ __forceinline__ RowSums join(const RowSums& a, const RowSums& b) {
  const float m = __builtin_elementwise_maximum(a.m, b.m);
  const RowSums x = a.m == m ? a : raised(a, m), y = b.m == m ? b : raised(b, m);
  return {m, x.n + y.n, x.s + y.s, x.t + y.t};
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
  // The t-th largest of 64 lanes' largest scores is no larger than the t-th best: nearly all scores fall below it.
  __device__ __forceinline__ void guess(float lane_max, int lane, int top) {
    const float bar = __shfl(sort_lanes(lane_max, lane), top - 1);
    if (bar > -INFINITY) {
      score = bar;
      index = INT32_MAX;
    }
  }
  __device__ __forceinline__ void take(int lane, int top) {
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    const int n = min(count, 64);
    const TopKey sorted = sort_lanes(lane < n ? waiting[lane] : (TopKey)0, lane);
    best = merge_lanes(best, sorted, lane);
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
    if (__ballot(x >= score) == 0) return;
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
                                           const int32_t* labels, int64_t row, const RowSums& a, TopKey best, int top, int lane) {
  const bool poisoned = !(a.m <= -kLowest);  // NaN or +inf among the scores
  const bool empty = a.n == 0.0f && !poisoned;
  const float ls = empty ? 0.0f : poisoned ? NAN : a.n == 1.0f ? log1pf(a.s) : logf(a.n + a.s);
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
    if (out.entropy) out.entropy[row] = empty ? 0.0f : poisoned ? NAN : ls - a.t / (a.n + a.s);
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

// The waves of a workgroup join theirs in a tree; wave 0 has the result.  Ends with LDS free for the next turn.
template <int WAVES, bool TOP>
__device__ __forceinline__ void join_waves(RowSums& a, TopKey& best, RowSums* lds_sums, TopKey (*lds_keys)[128], int wave, int lane) {
#pragma unroll
  for (int half = WAVES / 2; half; half /= 2) {
    if (wave >= half && wave < 2 * half) {
      if (lane == 0) lds_sums[wave] = a;
      if constexpr (TOP) lds_keys[wave][lane] = best;
    }
    __syncthreads();
    if (wave < half) {
      a = join(a, lds_sums[wave + half]);
      if constexpr (TOP) best = merge_lanes(best, lds_keys[wave + half][lane], lane);
    }
  }
}

// WAVES waves share a part of a row, tile by tile (a tile: kLogpUnroll 16-byte loads from each lane).  All lanes of a
// wave keep their sums relative to one score, the largest that the wave has seen: it changes in every i-th tile or so,
// and the other tiles take no scaling.
template <Elem E, int WAVES, bool TOP, bool ENTROPY>
__global__ __launch_bounds__(WAVES > 4 ? WAVES * 64 : 256) void logprobs_kernel(int64_t rows, int64_t classes, const elem_t<E>* __restrict__ scores,
                                                                int64_t row_stride, const int32_t* __restrict__ labels, int top,
                                                                int parts, int64_t part_classes, LogprobsOut out,
                                                                RowSums* __restrict__ part_sums, TopKey* __restrict__ part_keys) {
  constexpr int V = kLogpVec<E>, U = kLogpUnroll, kWaves = WAVES > 4 ? WAVES : 4, kTile = 64 * V * U;
  __shared__ TopKey lists[TOP ? kWaves : 1][128];
  __shared__ RowSums wave_sums[kWaves];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, part_wave = wave % WAVES;
  constexpr int kPartsPerGroup = kWaves / WAVES;
  const int64_t n_parts = rows * parts;
  for (int64_t group = blockIdx.x; group * kPartsPerGroup < n_parts; group += gridDim.x) {
    const int64_t id = group * kPartsPerGroup + wave / WAVES;
    RowSums a{kLowest, 0.0f, 0.0f, 0.0f};
    TopList list;
    if constexpr (TOP) list.start(lists[wave]);
    const int64_t row = parts == 1 ? id : id / parts;
    if (id < n_parts) {
      const int64_t begin = parts == 1 ? 0 : (id - row * parts) * part_classes;
      const int64_t end = min(classes, begin + part_classes);
      const elem_t<E>* x_row = scores + row * row_stride;
      bool first = true;
      for (int64_t tile = begin + (int64_t)part_wave * kTile; tile < end; tile += (int64_t)WAVES * kTile) {
        Pack<E, V> raw[U];
        if (tile + kTile <= end) {
#pragma unroll
          for (int u = 0; u < U; ++u) raw[u] = stream_pack<E, V>(x_row + tile + (u * 64 + lane) * V);
        } else {
#pragma unroll
          for (int u = 0; u < U; ++u) {
            const int64_t j = tile + (u * 64 + lane) * V;
            if (j + V <= end)
              raw[u] = load_pack<E, V>(x_row + j);
            else
              raw[u] = load_part<E, V>(x_row + j, (int)max((int64_t)0, end - j), -INFINITY);
          }
        }
        float group_max[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
          group_max[u] = (float)raw[u].v[0];
#pragma unroll
          for (int i = 1; i < V; ++i) group_max[u] = __builtin_elementwise_maximum(group_max[u], (float)raw[u].v[i]);
        }
        float lane_max = group_max[0];
#pragma unroll
        for (int u = 1; u < U; ++u) lane_max = __builtin_elementwise_maximum(lane_max, group_max[u]);
        if (__ballot(!(lane_max < a.m)) == 0) {
#pragma unroll
          for (int u = 0; u < U; ++u)
#pragma unroll
            for (int i = 0; i < V; ++i) {
              const float d = fmaxf((float)raw[u].v[i] - a.m, kFarBelow), e = exp_fast(d);
              a.s += e;
              if constexpr (ENTROPY) a.t += d * e;
            }
        } else {
          const float m = reduce_lanes(__builtin_elementwise_maximum(lane_max, a.m), lane, [](float x, float y) { return __builtin_elementwise_maximum(x, y); });
          if (!(m == a.m)) a = raised(a, m);
#pragma unroll
          for (int u = 0; u < U; ++u)
#pragma unroll
            for (int i = 0; i < V; ++i) {
              const float x = (float)raw[u].v[i], d = fmaxf(x - m, kFarBelow), e = exp_fast(d);
              a.n += x == m ? 1.0f : 0.0f;
              a.s += x == m ? 0.0f : e;
              if constexpr (ENTROPY) a.t += d * e;
            }
        }
        if constexpr (TOP) {
          if (first) list.guess(lane_max, lane, top);
          first = false;
          if (__ballot(lane_max >= list.score)) {
#pragma unroll
            for (int u = 0; u < U; ++u)
              if (__ballot(group_max[u] >= list.score))
#pragma unroll
                for (int i = 0; i < V; ++i) list.offer((float)raw[u].v[i], (int32_t)(tile + (u * 64 + lane) * V + i), lane, top);
          }
        }
      }
    }
    auto add = [](float x, float y) { return x + y; };
    a.n = reduce_lanes(a.n, lane, add);
    a.s = reduce_lanes(a.s, lane, add);
    if constexpr (ENTROPY) a.t = reduce_lanes(a.t, lane, add);
    if constexpr (TOP) list.take(lane, top);
    if constexpr (WAVES > 1) {
      static_assert(WAVES == kWaves, "one part per workgroup");
      join_waves<WAVES, TOP>(a, list.best, wave_sums, lists, wave, lane);
    }
    if (part_wave == 0 && id < n_parts) {
      if (parts == 1) {
        finish_row<E>(out, scores, row_stride, classes, labels, row, a, TOP ? list.best : 0, top, lane);
      } else {
        if (lane == 0) part_sums[id] = a;
        if constexpr (TOP)
          if (lane < top) part_keys[id * top + lane] = list.best;
      }
    }
    if constexpr (WAVES > 1) __syncthreads();  // wave 0 has read the last list
  }
}

// Joins the parts of a row: a workgroup per row, its waves take every fourth part.
template <Elem E>
__global__ __launch_bounds__(256) void logprobs_join_kernel(int64_t rows, int64_t classes, const elem_t<E>* __restrict__ scores,
                                                           int64_t row_stride, const int32_t* __restrict__ labels, int top, int parts,
                                                           LogprobsOut out, const RowSums* __restrict__ part_sums,
                                                           const TopKey* __restrict__ part_keys) {
  __shared__ TopKey lists[4][128];
  __shared__ RowSums wave_sums[4];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  for (int64_t row = blockIdx.x; row < rows; row += gridDim.x) {
    RowSums a{kLowest, 0.0f, 0.0f, 0.0f};
    TopKey best = 0;
    for (int p = wave; p < parts; p += 4) {
      a = join(a, part_sums[row * parts + p]);
      if (top) best = merge_lanes(best, lane < top ? part_keys[(row * parts + p) * top + lane] : (TopKey)0, lane);
    }
    join_waves<4, true>(a, best, wave_sums, lists, wave, lane);
    if (wave == 0) finish_row<E>(out, scores, row_stride, classes, labels, row, a, best, top, lane);
    __syncthreads();
  }
}

// ---- backward ---------------------------------------------------------------------------------------------------
// `across` threads (a power of two) share a row or, of a long row, a chunk; a thread takes one 16-byte group.
constexpr int kGradThreads = 256;
template <Elem E>
__global__ __launch_bounds__(kGradThreads) void logprobs_grad_kernel(int64_t rows, int64_t classes, const elem_t<E>* scores,
                                                                     int64_t row_stride, const int32_t* __restrict__ labels,
                                                                     const float* __restrict__ stats, const float* __restrict__ entropy,
                                                                     const float* __restrict__ dlogprob,
                                                                     const float* __restrict__ dentropy, int across_shift,
                                                                     int64_t chunks, elem_t<E>* out, int64_t out_stride) {
  constexpr int V = kLogpVec<E>;
  const int across = 1 << across_shift, down = kGradThreads >> across_shift;
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
