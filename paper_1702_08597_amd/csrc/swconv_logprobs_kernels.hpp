// HIP kernels of the log probabilities at a network's end.  For a row of scores x_j:
//   m = max x_j,  s = sum exp(x_j - m),  ls = log s,  log p_j = (x_j - m) - ls,  H = -sum p_j log p_j
// and H = ls - (sum (x_j - m) exp(x_j - m)) / s, whose two terms are both positive.  One pass over the scores: every wave
// keeps the largest score it has seen, its lanes both sums relative to it, scaled when that one changes; waves and parts of a
// row are joined in the same way.  All of it in fp32 whatever the scores' type.
//   d x_j = g ([j = label] - p_j) - h p_j (log p_j + H)
// A class of score -inf is masked: exp gives 0, and it never is among the best.  NaN and +inf make the row's largest
// score NaN or +inf (the maximum used propagates NaN), from which the row's results are made NaN.
// The best t classes, t <= 64: the pass over the scores only notes the largest one of each lane and segment (16 to a wave's
// share of a row).  The t-th largest of the lanes' largest scores is a bar that t scores reach and few others: the lanes and
// segments that reach it are read again, a lane to a score, and what reaches it is sorted, as 64-bit keys (score, then
// the lower class), one to a lane.  (Keeping the best up to date within the pass, 4096 x 131072 bf16 took 239 us for the best
// one and 413 for 64; so it takes 191 and 241, without any 186.)
// What bounds the forward pass: the vector units for many long rows - 4096 x 131072 bf16 with entropies and the best class at 5.6
// TB/s, 10 vector instructions to a score, which keep them 95 % busy; the way through one wave's tile, sorts and joins for few
// rows (1 x 32768 10 us, 256 x 1000 with the best 5 7 us, 4 without any).
#pragma once
#include "swconv_elements.hpp"
#include "swconv_lanes.hpp"

namespace swconv {

constexpr int kLogpUnroll = 4;        // 16-byte loads per lane and tile
constexpr int kTopMax = 64;           // one lane each
constexpr float kFarBelow = -256.0f;  // exp(-256) is 0 in fp32; keeps 0 * inf out of the sums
constexpr float kLog2e = 1.44269504088896340736f, kLn2 = 0.693147180559945309417f;
constexpr float kLowest = -3.402823466e38f;

// ---- lanes ------------------------------------------------------------------------------------------------------
// The calling lane's number among those of a mask.
__device__ __forceinline__ int lanes_below(uint64_t mask) {
  return __builtin_amdgcn_mbcnt_hi((uint32_t)(mask >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)mask, 0));
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
// 64 keys, one per lane, into descending order; `n`: keys behind lane n - 1 are all 0 (only the first 16 lanes, half of
// the steps, where that says so)
template <typename K>
__device__ __forceinline__ K sort_lanes(K key, int lane, int n) {
  key = halve<1>(key, lane, (lane & 2) == 0);
  key = halve<2>(key, lane, (lane & 4) == 0);
  key = halve<4>(key, lane, (lane & 8) == 0);
  key = halve<8>(key, lane, (lane & 16) == 0);
  if (n <= 16) return key;
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
  float t;  // sum of log2(exp(x - m)) exp(x - m)
};

// exp(x - m) for x < m as 2^(x log2 e - c) with c = m log2 e rounded: one fused multiply-add whose only error is its own
// rounding; what c is off by (at most 64) is put right once per row (finish_row).  From 2^30 on the next lower score is at least
// 64 further down, where exp is nothing next to 1: c = inf makes it 0.
__device__ __forceinline__ float reference(float m) { return fabsf(m) >= 1073741824.0f ? INFINITY : m * kLog2e; }

// The sums relative to a larger score m, which makes the scores that were largest ordinary ones.
__device__ __forceinline__ RowSums raised(const RowSums& a, float m) {
  const float c = reference(m);
  const float d = fmaxf(fminf(reference(a.m) - c, 0.0f), kFarBelow), f = __builtin_amdgcn_exp2f(d);
  const float d_n = fmaxf(__builtin_fmaf(a.m, kLog2e, -c), kFarBelow), n = a.n * __builtin_amdgcn_exp2f(d_n);
  return {m, 0.0f, f * a.s + n, f * (a.t + d * a.s) + d_n * n};
}
__device__ __forceinline__ RowSums join(const RowSums& a, const RowSums& b) {
  const float m = __builtin_elementwise_maximum(a.m, b.m);
  const RowSums x = a.m == m ? a : raised(a, m), y = b.m == m ? b : raised(b, m);
  return {m, x.n + y.n, x.s + y.s, x.t + y.t};
}

// A lane's sum over a tile: its groups of 16 bytes each for itself, then together (with four strands side by side, or with all
// groups kept to the end, f16 took 5 % longer; one term behind the other loses as much as the rest of the way).
template <int V>
struct GroupedSum {
  float total, group;
  __device__ __forceinline__ void add(int k, float x, float y) {  // x * y, the k-th term
    group = k % V ? __builtin_fmaf(x, y, group) : x * y;
    if (k % V == V - 1) total = k < V ? group : total + group;
  }
};
// sum += x with what the addition before rounded off (Kahan, "Further remarks on reducing truncation errors", 1965): for
// terms of one sign the sum is off by two roundings however many there are.  (Equal terms one by one are all rounded the same way:
// with 262143 equal f16 scores below one, ls was off by up to 4.5e-5 and the entropy by 4.4e-4, so by 3e-7 and 1e-6.)
__device__ __forceinline__ void add_exactly(float& sum, float& low, float x) {
  const float y = x - low, next = sum + y;
  low = (next - sum) - y;
  sum = next;
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

constexpr int kSegments = 16;
constexpr int kWaiting = 128;  // a list in LDS: fewer than 64 and 64 more

struct TopList {
  TopKey best;        // lane i: the i-th best so far, if any
  TopKey* waiting;    // LDS, kWaiting
  int count;          // of them, fewer than 64 between calls
  bool any;           // best holds some
  float score;        // what a score has to beat,
  int32_t index;      // or equal at a lower class

  __device__ __forceinline__ void start(TopKey* lds, float bar) {
    best = 0;
    waiting = lds;
    count = 0;
    any = false;
    score = bar;
    index = INT32_MAX;
  }
  // Sorts what waits into the best.
  __device__ __forceinline__ void take(int lane, int top) {
    if (count == 0) return;
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    const int n = min(count, 64);
    count -= n;
    const TopKey sorted = sort_lanes(lane < n ? waiting[count + lane] : (TopKey)0, lane, n);
    best = any ? merge_lanes(best, sorted, lane) : sorted;
    any = true;
    const TopKey bar = __shfl(best, top - 1);
    if (bar) {
      score = top_score(bar);
      index = top_index(bar);
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  }
  // One score from each lane.
  __device__ __forceinline__ void offer(float x, int32_t j, int lane, int top) {
    const bool hit = x > score || (x == score && j < index);
    const uint64_t hits = __ballot(hit);
    if (hit) waiting[count + lanes_below(hits)] = top_key(x, j);
    count += __popcll(hits);
    if (count >= 64) take(lane, top);
  }
};

// Calls see(score or -inf, class) for one score to a lane, for all that a wave's lanes hold in segments whose largest score
// reaches bar(): a lane's scores of a tile are U runs of V.  `owners`: LDS, room for 128 (segment, lane) pairs; all of
// them are read in one go, 64 scores at a time and four such reads in flight.
template <Elem E, typename Bar, typename See>
__device__ __forceinline__ void look_again(const elem_t<E>* x_row, const float (*segment_max)[64], uint16_t* owners,
                                           int segments, int segment_tiles, int64_t first, int64_t step, int64_t end,
                                           int lane, Bar&& bar, See&& see) {
  constexpr int V = kWordsElems<E>, U = kLogpUnroll, kFlight = 4;
  int n = 0;
  for (int s = 0; s < segments; ++s) {
    const bool reaches = segment_max[s][lane] >= bar();
    const uint64_t reaching = __ballot(reaches);
    if (reaches) owners[n + lanes_below(reaching)] = (uint16_t)(s << 6 | lane);
    n += __popcll(reaching);
    if (n == 0 || (n < 64 && s + 1 < segments)) continue;
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    for (int i = 0; i < segment_tiles; ++i)
      for (int q0 = 0; q0 < n * (U * V); q0 += 64 * kFlight) {
        float x[kFlight];
        int64_t j[kFlight];
#pragma unroll
        for (int f = 0; f < kFlight; ++f) {
          const int q = q0 + 64 * f + lane, in_tile = q % (U * V);
          const int owner = q < n * (U * V) ? owners[q / (U * V)] : 0;
          j[f] = first + ((int64_t)(owner >> 6) * segment_tiles + i) * step + (in_tile / V * 64 + (owner & 63)) * V + in_tile % V;
          x[f] = q < n * (U * V) && j[f] < end ? (float)x_row[j[f]] : -INFINITY;
        }
#pragma unroll
        for (int f = 0; f < kFlight; ++f)
          if (q0 + 64 * f < n * (U * V)) see(x[f], (int32_t)j[f]);
      }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    n = 0;
  }
}

// ---- forward ----------------------------------------------------------------------------------------------------
struct LogprobsOut {
  float *logprob, *entropy, *stats;
  int32_t* top_class;
  float* top_logprob;
};

// The class asked for (below 0: none) and its score, NaN where there is no such class.
struct Label {
  int32_t at;
  float score;
};
template <Elem E>
__device__ __forceinline__ Label label_at(int32_t at, const elem_t<E>* x_row, int64_t classes) {
  return {at, at < 0 ? 0.0f : at < classes ? (float)x_row[at] : NAN};
}

// A row's results from its sums and its best classes; called by one wave.
template <Elem E>
__device__ __forceinline__ void finish_row(const LogprobsOut& out, int64_t row, Label label, const RowSums& a,
                                           TopKey best, int top, int lane) {
  const bool poisoned = !(a.m <= -kLowest);  // NaN or +inf among the scores
  const bool empty = a.n == 0.0f && !poisoned;
  // m log2 e = c + off: every exponential, 2^(x log2 e - c), is 2^off too large, its logarithm off too high
  const float c = reference(a.m), off = isinf(c) ? 0.0f : __builtin_fmaf(a.m, kLog2e, -c), back = __builtin_amdgcn_exp2f(-off);
  const float s = a.s * back, t = kLn2 * (a.t - off * a.s) * back;
  const float ls = empty ? 0.0f : poisoned ? NAN : a.n == 1.0f ? log1pf(s) : logf(a.n + s);
  const float m = empty ? -INFINITY : poisoned ? NAN : a.m;
  if (lane == 0) {
    if (out.logprob) {
      float lp = label.score;
      if (label.at >= 0) lp = empty && lp == lp ? -INFINITY : (lp - m) - ls;
      out.logprob[row] = lp;
    }
    if (out.entropy) out.entropy[row] = empty ? 0.0f : poisoned ? NAN : ls - t / (a.n + s);
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

// The sums of up to 16 waves, one from each of the first lanes.
template <int WAVES>
__device__ __forceinline__ RowSums join_sums(const RowSums* lds_sums, int lane) {
  RowSums a = lane < WAVES ? lds_sums[lane] : RowSums{kLowest, 0.0f, 0.0f, 0.0f};
  auto step = [&](auto off) {
    constexpr int OFF = decltype(off)::value;
    a = join(a, {lane_xor<OFF>(a.m, lane), lane_xor<OFF>(a.n, lane), lane_xor<OFF>(a.s, lane), lane_xor<OFF>(a.t, lane)});
  };
  using std::integral_constant;
  if constexpr (WAVES > 1) step(integral_constant<int, 1>{});
  if constexpr (WAVES > 2) step(integral_constant<int, 2>{});
  if constexpr (WAVES > 4) step(integral_constant<int, 7>{});
  if constexpr (WAVES > 8) step(integral_constant<int, 15>{});
  auto first = [](float v) { return __int_as_float(__builtin_amdgcn_readfirstlane(__float_as_int(v))); };
  return {first(a.m), first(a.n), first(a.s), first(a.t)};
}
// The best of all waves' descending lists by merges in a tree; wave 0 has the result.
template <int WAVES, typename K, int N>
__device__ __forceinline__ K join_best(K best, K (*lds_keys)[N], int wave, int lane) {
#pragma unroll
  for (int half = WAVES / 2; half; half /= 2) {
    if (wave >= half && wave < 2 * half) lds_keys[wave][lane] = best;
    __syncthreads();
    if (wave < half) best = merge_lanes(best, lds_keys[wave + half][lane], lane);
  }
  return best;
}

// A tile's 16-byte groups of one lane.  Groups that reach past the end of a row (or part) lie on its last V elements
// instead - so that every tile is read in one way, without the waits of several - and what other groups hold of these then
// counts as -inf (cut_tile).  The row has V elements at least.
template <Elem E, bool ONCE>
__device__ __forceinline__ void load_tile(Words (&raw)[kLogpUnroll], const elem_t<E>* x_row, int64_t tile, int64_t end,
                                          int lane) {
  constexpr int V = kWordsElems<E>;
  const int64_t last = end - V;
#pragma unroll
  for (int u = 0; u < kLogpUnroll; ++u)
    raw[u] = load_words<E>(x_row + min(tile + (u * 64 + lane) * V, last), ONCE);
}
template <Elem E>
__device__ __forceinline__ void cut_tile(Words (&raw)[kLogpUnroll], int64_t tile, int64_t end, int lane) {
  constexpr int V = kWordsElems<E>;
#pragma unroll
  for (int u = 0; u < kLogpUnroll; ++u) {
    const int64_t past = tile + (u * 64 + lane) * V - (end - V);
    raw[u] = without_first<E>(raw[u], (int)max(min(past, (int64_t)V), (int64_t)0));
  }
}

// WAVES waves share a part of a row, tile by tile (a tile: kLogpUnroll 16-byte loads from each lane).  All lanes of a
// wave keep their sums relative to one score, the largest that the wave has seen: it changes in every i-th tile or so,
// and the other tiles take no scaling.
template <Elem E, int WAVES, bool TOP, bool ENTROPY>
__global__ __launch_bounds__(WAVES == 1 ? 256 : WAVES * 64) void logprobs_kernel(
    int64_t rows, int64_t classes, const elem_t<E>* __restrict__ scores, int64_t row_stride,
    const int32_t* __restrict__ labels, int top, int parts, int64_t part_classes, bool once, LogprobsOut out,
    RowSums* __restrict__ part_sums, TopKey* __restrict__ part_keys) {
  constexpr int V = kWordsElems<E>, U = kLogpUnroll, kWaves = WAVES == 1 ? 4 : WAVES, kTile = 64 * V * U;
  __shared__ TopKey lists[TOP ? kWaves : 1][kWaiting];
  __shared__ float segment_max[TOP ? kWaves : 1][kSegments][64];
  __shared__ RowSums wave_sums[kWaves];
  __shared__ float lane_lists[TOP && WAVES > 1 ? kWaves : 1][64];
  __shared__ uint16_t owners[TOP ? kWaves : 1][kWaiting];
  __shared__ float bars[kWaves];
  __shared__ int waiting;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), part_wave = wave % WAVES;
  constexpr int kPartsPerGroup = kWaves / WAVES;
  // Four waves to a row ask for the next tile before they work on one: 4096 x 131072 without the best classes 191 -> 183 us,
  // 64 x 150001 16.8 -> 16.0.  One wave to a row gains nothing (16384 x 8192 71 -> 78), sixteen lack the registers.
  constexpr bool PREFETCH = WAVES == 4;
  const int64_t n_parts = rows * parts;
  for (int64_t group = blockIdx.x; group * kPartsPerGroup < n_parts; group += gridDim.x) {
    const int64_t id = group * kPartsPerGroup + wave / WAVES;
    if (WAVES == 1 && id >= n_parts) break;
    const int64_t row = parts == 1 ? id : id / parts;
    const int64_t begin = parts == 1 ? 0 : (id - row * parts) * part_classes;
    const int64_t end = min(classes, begin + part_classes);
    const elem_t<E>* x_row = scores + row * row_stride;
    RowSums a{kLowest, 0.0f, 0.0f, 0.0f};
    int32_t wanted = -1;  // asked for here, waited for behind the row's own loads
    if (parts == 1 && part_wave == 0 && out.logprob) wanted = labels[row];
    constexpr int64_t kStep = (int64_t)WAVES * kTile;
    const int64_t first = begin + (int64_t)part_wave * kTile;
    const int segment_tiles = (int)((end - begin + kStep * kSegments - 1) / (kStep * kSegments));
    float c = reference(a.m), seen_max = -INFINITY, lane_best = -INFINITY;
    int segment = 0, in_segment = 0;
    float n = 0.0f;  // scores equal to a.m in the whole wave
    float n_low = 0.0f, s_low = 0.0f, t_low = 0.0f;
    auto see_tile = [&](const Words (&raw)[U], bool last) {
      float lane_max = word_elem<E>(raw[0], 0);
#pragma unroll
      for (int k = 1; k < U * V; ++k) lane_max = __builtin_elementwise_maximum(lane_max, word_elem<E>(raw[k / V], k % V));
      GroupedSum<V> s, t;
      if (__ballot(!(lane_max < a.m)) == 0) {
#pragma unroll
        for (int k = 0; k < U * V; ++k) {
          const float x = word_elem<E>(raw[k / V], k % V);
          const float d = fmaxf(__builtin_fmaf(x, kLog2e, -c), kFarBelow), e = __builtin_amdgcn_exp2f(d);
          s.add(k, 1.0f, e);
          if constexpr (ENTROPY) t.add(k, d, e);
        }
      } else {
        auto larger = [](float x, float y) { return __builtin_elementwise_maximum(x, y); };
        const float m = reduce_lanes(larger(lane_max, a.m), lane, larger);
        if (!(m == a.m)) {
          a.n = lane == 0 ? n : 0.0f;
          a = raised(a, m);
          c = reference(m);
          n = 0.0f;
          n_low = s_low = t_low = 0.0f;
        }
        int equal = 0;
#pragma unroll
        for (int k = 0; k < U * V; ++k) {
          float x = word_elem<E>(raw[k / V], k % V);
          equal += __popcll(__ballot(x == m));
          x = x == m ? -INFINITY : x;
          const float d = fmaxf(__builtin_fmaf(x, kLog2e, -c), kFarBelow), e = __builtin_amdgcn_exp2f(d);
          s.add(k, 1.0f, e);
          if constexpr (ENTROPY) t.add(k, d, e);
        }
        add_exactly(n, n_low, (float)equal);
      }
      add_exactly(a.s, s_low, s.total);
      if constexpr (ENTROPY) add_exactly(a.t, t_low, t.total);
      if constexpr (TOP) {
        lane_best = fmaxf(lane_best, lane_max);
        seen_max = fmaxf(seen_max, lane_max);
        if (++in_segment == segment_tiles || last) {
          segment_max[wave][segment++][lane] = seen_max;
          seen_max = -INFINITY;
          in_segment = 0;
        }
      }
    };
    auto look_through = [&](auto once_or_not) {
      constexpr bool ONCE = decltype(once_or_not)::value;
      Words next[U];
      if constexpr (PREFETCH) load_tile<E, ONCE>(next, x_row, first, end, lane);
      for (int64_t tile = first; tile < end; tile += kStep) {
        Words raw[U];
        if constexpr (PREFETCH) {
#pragma unroll
          for (int u = 0; u < U; ++u) raw[u] = next[u];
          load_tile<E, ONCE>(next, x_row, tile + kStep, end, lane);
        } else {
          load_tile<E, ONCE>(raw, x_row, tile, end, lane);
        }
        if (tile + kTile > end) cut_tile<E>(raw, tile, end, lane);
        see_tile(raw, tile + kStep >= end);
      }
    };
    if (end < V) {  // one wave's, one lane's
      Words raw[U];
#pragma unroll
      for (int u = 0; u < U; ++u) raw[u] = load_words_part<E>(x_row, u == 0 && lane == 0 && first < end ? (int)end : 0);
      see_tile(raw, true);
    } else if (first < end) {
      if (once)
        look_through(std::true_type{});
      else
        look_through(std::false_type{});
    }
    const Label label = label_at<E>(wanted, x_row, classes);
    auto add = [](float x, float y) { return x + y; };
    a.n = n;
    a.s = reduce_lanes(a.s, lane, add);
    if constexpr (ENTROPY) a.t = reduce_lanes(a.t, lane, add);
    if constexpr (WAVES > 1) {
      if (lane == 0) wave_sums[wave] = a;
      if (wave == 0 && lane == 0) waiting = 0;
      if constexpr (!TOP) __syncthreads();
    }
    TopList list;
    if constexpr (TOP) {
      float bar = sort_lanes(lane_best, lane, 64);
      if (WAVES > 1 && top > 8) bar = join_best<WAVES>(bar, lane_lists, wave, lane);
      bar = fmaxf(__shfl(bar, top - 1), kLowest);  // never -inf: a masked class, or what lies behind the row
      if constexpr (WAVES > 1) {
        // the bar of all lanes, or for few classes the highest of the waves': with less waiting, if a little lower
        if (lane == 0) bars[wave] = bar;
        __syncthreads();
        bar = bars[0];
        if (top <= 8)
          for (int w = 1; w < WAVES; ++w) bar = fmaxf(bar, bars[w]);
      }
      auto look = [&](auto&& least, auto&& see) {
        look_again<E>(x_row, segment_max[wave], owners[wave], segment, segment_tiles, first, kStep, end, lane, least, see);
      };
      auto alone = [&] {  // every wave keeps its own best, whatever comes
        list.start(lists[wave], bar);
        look([&] { return list.score; }, [&](float x, int32_t j) { list.offer(x, j, lane, top); });
        list.take(lane, top);
      };
      if constexpr (WAVES == 1) {
        alone();
      } else {
        // all waves into one list, which nearly always takes it
        TopKey* all = lists[0];
        look([&] { return bar; }, [&](float x, int32_t j) {
          const uint64_t hits = __ballot(x >= bar);
          if (hits == 0) return;
          int at = 0;
          if (lane == 0) at = __hip_atomic_fetch_add(&waiting, __popcll(hits), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP);
          at = __builtin_amdgcn_readfirstlane(at) + lanes_below(hits);
          if (x >= bar && at < kWaiting) all[at] = top_key(x, j);
        });
        __syncthreads();
        const int n = waiting;
        if (n <= kWaiting) {
          if (wave == 0) {
            list.best = sort_lanes(lane < n ? all[lane] : (TopKey)0, lane, n);
            if (n > 64) {
              const TopKey rest = sort_lanes(lane < n - 64 ? all[64 + lane] : (TopKey)0, lane, n - 64);
              list.best = merge_lanes(list.best, rest, lane);
            }
          }
        } else {
          __syncthreads();  // all have read `waiting`
          alone();
          list.best = join_best<WAVES>(list.best, lists, wave, lane);
        }
      }
    }
    if constexpr (WAVES > 1)
      if (wave == 0) a = join_sums<WAVES>(wave_sums, lane);
    if (part_wave == 0) {
      if (parts == 1) {
        finish_row<E>(out, row, label, a, TOP ? list.best : 0, top, lane);
      } else {
        if (lane == 0) part_sums[id] = a;
        if constexpr (TOP)
          if (lane < top) part_keys[id * top + lane] = list.best;
      }
    }
    if constexpr (WAVES > 1) __syncthreads();  // LDS is free for the next part
  }
}

// Joins the parts of a row: a workgroup per row, its waves take every fourth part.
template <Elem E>
__global__ __launch_bounds__(256) void logprobs_join_kernel(int64_t rows, int64_t classes, const elem_t<E>* __restrict__ scores,
                                                           int64_t row_stride, const int32_t* __restrict__ labels, int top, int parts,
                                                           LogprobsOut out, const RowSums* __restrict__ part_sums,
                                                           const TopKey* __restrict__ part_keys) {
  __shared__ TopKey lists[4][kWaiting];
  __shared__ RowSums wave_sums[4];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  for (int64_t row = blockIdx.x; row < rows; row += gridDim.x) {
    RowSums a{kLowest, 0.0f, 0.0f, 0.0f};
    TopKey best = 0;
    const int32_t wanted = out.logprob ? labels[row] : -1;
    for (int p = wave; p < parts; p += 4) {
      a = join(a, part_sums[row * parts + p]);
      if (top) best = merge_lanes(best, lane < top ? part_keys[(row * parts + p) * top + lane] : (TopKey)0, lane);
    }
    const Label label = label_at<E>(wanted, scores + row * row_stride, classes);
    if (lane == 0) wave_sums[wave] = a;
    best = join_best<4>(best, lists, wave, lane);  // its barriers are the sums' too
    a = join_sums<4>(wave_sums, lane);
    if (wave == 0) finish_row<E>(out, row, label, a, best, top, lane);
    __syncthreads();
  }
}

// ---- backward ---------------------------------------------------------------------------------------------------
// With e = exp(x - m) and p = e exp(-ls):  d x = -p (g + h (x - m - ls + H)) = e (b + a log2 e), a and b by row.  The
// exponent holds x - m alone: ls in it would cost the digits of its size.  Bound by memory: 4096 x 131072 bf16 at 6.0 TB/s
// read and written.
struct GradRow {
  float m, a, b, g;
  int32_t label;
  bool plain;  // all of them are finite, and b + a log2 e for every exponential
};
struct GradIn {
  const int32_t* labels;
  const float *stats, *entropy, *dlogprob, *dentropy;
};
__device__ __forceinline__ GradRow grad_row(const GradIn& in, int64_t row, int64_t classes) {
  GradRow r;
  r.m = in.stats[2 * row];
  const float ls = in.stats[2 * row + 1];
  r.label = in.labels ? in.labels[row] : -1;
  const float g = in.dlogprob ? in.dlogprob[row] : 0.0f;
  r.g = !in.dlogprob || r.label < 0 ? 0.0f : r.label < classes ? g : NAN;
  const float h = in.dentropy ? in.dentropy[row] : 0.0f, H = in.dentropy ? in.entropy[row] : 0.0f;
  const float u = ls * kLog2e, low = __builtin_fmaf(ls, kLog2e, -u);  // exp(-ls) to the digits of ls, not of u
  const float scale = -__builtin_amdgcn_exp2f(-u) * __builtin_fmaf(-low, kLn2, 1.0f);
  r.a = scale * h * kLn2;
  r.b = scale * (r.g + h * (H - ls));
  r.plain = fabsf(r.m) < INFINITY && fabsf(r.a) < 1e35f && fabsf(r.b) < 1e38f;
  return r;
}
// 16 bytes of scores that begin with class j into 16 bytes of gradients.
template <Elem E, bool ENTROPY>
__device__ __forceinline__ Words grad_words(const GradRow& r, const Words& x, int64_t j) {
  constexpr int V = kWordsElems<E>;
  Pack<E, V> out;
  const int64_t hot = r.label - j;
  if (r.plain) {
#pragma unroll
    for (int i = 0; i < V; ++i) {
      float d = (word_elem<E>(x, i) - r.m) * kLog2e;
      if constexpr (ENTROPY) d = fmaxf(d, kFarBelow);
      const float e = __builtin_amdgcn_exp2f(d);
      out.v[i] = (elem_t<E>)(e * (ENTROPY ? __builtin_fmaf(r.a, d, r.b) : r.b));
    }
    if (hot >= 0 && hot < V)
#pragma unroll
      for (int i = 0; i < V; ++i)
        if (hot == i) {
          const float xi = word_elem<E>(x, i), d = fmaxf((xi - r.m) * kLog2e, kFarBelow);
          out.v[i] = (elem_t<E>)(xi > -INFINITY ? r.g + __builtin_amdgcn_exp2f(d) * __builtin_fmaf(r.a, d, r.b) : 0.0f);
        }
  } else {
    // no class left (all 0), a row of NaN, or a gradient that is not finite or near the end of fp32, where an exponential of 0
    // comes before any product; masked classes get 0 here too
#pragma unroll
    for (int i = 0; i < V; ++i) {
      const float xi = word_elem<E>(x, i), d = fmaxf((xi - r.m) * kLog2e, kFarBelow);
      const float e = __builtin_amdgcn_exp2f(d);
      float v = r.m != r.m ? NAN : e * r.a * d + e * r.b;
      if (hot == i) v += r.g;
      out.v[i] = (elem_t<E>)(xi == -INFINITY ? 0.0f : v);
    }
  }
  return __builtin_bit_cast(Words, out);
}
template <Elem E, bool ENTROPY>
__device__ __forceinline__ void grad_group(const GradRow& r, const elem_t<E>* x_row, elem_t<E>* out_row, int64_t j, int64_t classes) {
  constexpr int V = kWordsElems<E>;
  if (j + V <= classes) {
    store_words<E>(out_row + j, grad_words<E, ENTROPY>(r, load_words<E>(x_row + j, false), j), false);
  } else if (j < classes) {
    const int n = (int)(classes - j);
    const Pack<E, V> dx = __builtin_bit_cast(Pack<E, V>, grad_words<E, ENTROPY>(r, load_words_part<E>(x_row + j, n), j));
    store_part<E, V>(out_row + j, n, dx);
  }
}

// Rows of at least 128 groups of 16 bytes: workgroups along a row, in the order of memory; the row's numbers are scalars
// and arrive with the scores.  Groups to a thread: 4096 x 131072 bf16 with one 446 us, two 354, four 368; 4096 x 65536 f32
// 337, 362, 361.
constexpr int kGradThreads = 256;
template <Elem E>
constexpr int kGradUnroll = E == Elem::f32 ? 1 : 2;
template <Elem E, bool ENTROPY>
__global__ __launch_bounds__(kGradThreads) void logprobs_grad_kernel(int64_t rows, int64_t classes,
                                                                     const elem_t<E>* scores, int64_t row_stride,
                                                                     GradIn in, bool once, elem_t<E>* out,
                                                                     int64_t out_stride) {
  constexpr int V = kWordsElems<E>, U = kGradUnroll<E>;
  const int64_t j = ((int64_t)blockIdx.x * (kGradThreads * U) + threadIdx.x) * V;
  for (int64_t row = blockIdx.y; row < rows; row += gridDim.y) {
    const elem_t<E>* x_row = scores + row * row_stride;
    elem_t<E>* out_row = out + row * out_stride;
    if (((int64_t)blockIdx.x + 1) * (kGradThreads * U) * V <= classes) {
      Words x[U];
      if (once) {
#pragma unroll
        for (int u = 0; u < U; ++u) x[u] = load_words<E>(x_row + j + u * (kGradThreads * V), true);
      } else {
#pragma unroll
        for (int u = 0; u < U; ++u) x[u] = load_words<E>(x_row + j + u * (kGradThreads * V), false);
      }
      const GradRow r = grad_row(in, row, classes);
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int64_t at = j + u * (kGradThreads * V);
        store_words<E>(out_row + at, grad_words<E, ENTROPY>(r, x[u], at), once);
      }
    } else {
      const GradRow r = grad_row(in, row, classes);
#pragma unroll
      for (int u = 0; u < U; ++u) grad_group<E, ENTROPY>(r, x_row, out_row, j + u * (kGradThreads * V), classes);
    }
  }
}
// Shorter rows: `across` threads (a power of two) to a row.
template <Elem E, bool ENTROPY>
__global__ __launch_bounds__(kGradThreads) void logprobs_grad_short_kernel(int64_t rows, int64_t classes, const elem_t<E>* scores,
                                                                           int64_t row_stride, GradIn in, int across_shift,
                                                                           elem_t<E>* out, int64_t out_stride) {
  const int across = 1 << across_shift, down = kGradThreads >> across_shift;
  const int64_t j = (threadIdx.x & (across - 1)) * kWordsElems<E>;
  for (int64_t row = (int64_t)blockIdx.x * down + (threadIdx.x >> across_shift); row < rows; row += (int64_t)gridDim.x * down)
    grad_group<E, ENTROPY>(grad_row(in, row, classes), scores + row * row_stride, out + row * out_stride, j, classes);
}

}  // namespace swconv
