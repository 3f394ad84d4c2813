// HIP kernels of bias, ReLU and dropout between two layers, and of their backward pass:
//   z = x + bias[k],  a = relu ? max(z, 0) : z,  y = keep ? a * scale : 0
//   dz = keep and (z > 0 or no relu) ? dy * scale : 0,  dx = dz,  dbias[k] = sum over n, s of dz
// The mask is never stored: keep(row, col) = 16-bit field col % 8 of philox4x32-10 (Salmon, Moraes, Dror, Shaw,
// "Parallel random numbers: as easy as 1, 2, 3", 2011) at counter {col / 8, row, step}, so that any thread makes any
// element's decision alone and the backward pass makes the forward pass's.  A group of 8 columns costs one call, 20
// products of 32 x 32 bits.  16 bits an element round the rate to a multiple of 2^-16; the scale is that rate's, so the
// mean is kept exactly.  Arithmetic in fp32, one rounding to the element type at the end.
#pragma once
#include "swconv_elements.hpp"

namespace swconv {

constexpr int kDropThreads = 256;
constexpr int kDropItems = 2;      // groups of 8 columns per thread and turn
constexpr int kDropUnit = 512;     // groups that a wave of the gradient of maps sums up at a time

struct DropoutRule {
  const uint64_t* rng;  // seed, step; not read when threshold is 0
  uint64_t offset;
  uint32_t threshold;   // drop a field below it, 0 .. 65536
  float scale;
  int relu;
};

// Rows of the generator: planes (n, k) of S columns, or with S = 1 images of K columns.
struct DropoutShape {
  Divisor groups;       // of 8 columns in a row
  Divisor32 groups32, channels;
  uint64_t items;       // rows * groups
  uint32_t cols;
  int features;         // S = 1: columns are channels
};

__device__ __forceinline__ void philox_round(uint32_t (&c)[4], uint32_t k0, uint32_t k1) {
  const uint64_t a = (uint64_t)0xD2511F53u * c[0], b = (uint64_t)0xCD9E8D57u * c[2];
  c[0] = (uint32_t)(b >> 32) ^ c[1] ^ k0;
  c[1] = (uint32_t)b;
  c[2] = (uint32_t)(a >> 32) ^ c[3] ^ k1;
  c[3] = (uint32_t)a;
}

// The decisions for 8 columns, bit i: column 8 * group + i is kept.
__device__ __forceinline__ uint32_t keep_bits(const DropoutRule& rule, uint64_t seed, uint64_t step, uint32_t row, uint32_t group) {
  if (rule.threshold == 0) return 0xffu;
  uint32_t c[4] = {group, row, (uint32_t)step, (uint32_t)(step >> 32)};
  uint32_t k0 = (uint32_t)seed, k1 = (uint32_t)(seed >> 32);
#pragma unroll
  for (int r = 0; r < 10; ++r) {
    philox_round(c, k0, k1);
    k0 += 0x9E3779B9u;
    k1 += 0xBB67AE85u;
  }
  uint32_t keep = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) keep |= (uint32_t)(((c[i / 2] >> (i % 2 * 16)) & 0xffffu) >= rule.threshold) << i;
  return keep;
}

// Where a row of the generator lies in a tensor of the given image stride, and its channel.
__device__ __forceinline__ int64_t row_offset(const DropoutShape& sh, uint32_t row, int64_t stride, uint32_t* k) {
  if (sh.features) {
    *k = 0;
    return (int64_t)row * stride;
  }
  const uint32_t n = sh.channels.quotient(row);
  *k = row - n * sh.channels.d;
  return (int64_t)n * stride + (int64_t)*k * sh.cols;
}

__device__ __forceinline__ void load_bias(const DropoutShape& sh, const float* bias, uint32_t k, uint32_t col, int n, float (&b)[8]) {
  if (!bias) {
#pragma unroll
    for (int i = 0; i < 8; ++i) b[i] = 0.0f;
  } else if (!sh.features) {
    const float v = bias[k];
#pragma unroll
    for (int i = 0; i < 8; ++i) b[i] = v;
  } else {
    const Pack<Elem::f32, 8> v = n == 8 ? load_pack<Elem::f32, 8>(bias + col) : load_part<Elem::f32, 8>(bias + col, n, 0.0f);
#pragma unroll
    for (int i = 0; i < 8; ++i) b[i] = v.v[i];
  }
}

template <Elem E>
__device__ __forceinline__ Pack<E, 8> load_group(const elem_t<E>* p, int n) {
  return n == 8 ? load_pack<E, 8>(p) : load_part<E, 8>(p, n, 0.0f);
}
template <Elem E>
__device__ __forceinline__ void store_group(elem_t<E>* p, int n, const Pack<E, 8>& a) {
  if (n == 8)
    store_pack<E, 8>(p, a);
  else
    store_part<E, 8>(p, n, a);
}

// A dropped element is 0 whatever it was; a NaN that is kept stays one.
template <Elem E>
__device__ __forceinline__ Pack<E, 8> forward_group(const DropoutRule& rule, const Pack<E, 8>& x, const float (&b)[8], uint32_t keep) {
  Pack<E, 8> y;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    float z = (float)x.v[i] + b[i];
    if (rule.relu && z < 0.0f) z = 0.0f;
    y.v[i] = (elem_t<E>)(keep >> i & 1 ? z * rule.scale : 0.0f);
  }
  return y;
}
// dz of a group; the sum of its 8 in a fixed order.
template <Elem E>
__device__ __forceinline__ void backward_group(const DropoutRule& rule, const Pack<E, 8>& dy, const Pack<E, 8>& x, const float (&b)[8],
                                               uint32_t keep, float (&dz)[8]) {
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    bool pass = keep >> i & 1;
    if (rule.relu) pass = pass && !((float)x.v[i] + b[i] <= 0.0f);
    dz[i] = pass ? (float)dy.v[i] * rule.scale : 0.0f;
  }
}
template <Elem E>
__device__ __forceinline__ Pack<E, 8> rounded(const float (&v)[8]) {
  Pack<E, 8> a;
#pragma unroll
  for (int i = 0; i < 8; ++i) a.v[i] = (elem_t<E>)v[i];
  return a;
}

// Forward, and backward without a bias gradient: threads over all groups of all rows.  Bound by memory: a group in
// and a group out.
template <Elem E, bool BACKWARD>
__global__ __launch_bounds__(kDropThreads) void dropout_kernel(DropoutShape sh, DropoutRule rule, const elem_t<E>* x,
                                                               int64_t x_stride, const float* __restrict__ bias, const elem_t<E>* dy,
                                                               int64_t dy_stride, elem_t<E>* out, int64_t out_stride) {
  constexpr uint64_t kTurn = kDropThreads * kDropItems;
  uint64_t seed = 0, step = 0;
  if (rule.threshold) {
    seed = rule.rng[0];
    step = rule.rng[1] + rule.offset;
  }
  for (uint64_t first = blockIdx.x * kTurn; first < sh.items; first += gridDim.x * kTurn) {
    const uint64_t row0 = sh.groups.quotient(first);
    const uint32_t group0 = (uint32_t)(first - row0 * sh.groups.d);
#pragma unroll
    for (int u = 0; u < kDropItems; ++u) {
      const uint32_t t = u * kDropThreads + threadIdx.x;
      if (first + t >= sh.items) break;
      const uint32_t over = sh.groups32.quotient(group0 + t);
      const uint32_t row = (uint32_t)row0 + over, group = group0 + t - over * sh.groups32.d;
      const uint32_t col = group * 8;
      const int n = min(8u, sh.cols - col);
      uint32_t k;
      const int64_t o = row_offset(sh, row, out_stride, &k) + col;
      const uint32_t keep = keep_bits(rule, seed, step, row, group);
      float b[8];
      load_bias(sh, bias, k, col, n, b);
      if constexpr (!BACKWARD) {
        const Pack<E, 8> a = load_group<E>(x + row_offset(sh, row, x_stride, &k) + col, n);
        store_group<E>(out + o, n, forward_group<E>(rule, a, b, keep));
      } else {
        const Pack<E, 8> g = load_group<E>(dy + row_offset(sh, row, dy_stride, &k) + col, n);
        Pack<E, 8> a = g;
        if (rule.relu) a = load_group<E>(x + row_offset(sh, row, x_stride, &k) + col, n);
        float dz[8];
        backward_group<E>(rule, g, a, b, keep, dz);
        store_group<E>(out + o, n, rounded<E>(dz));
      }
    }
  }
}

// Backward of maps with the bias gradient: a wave takes `planes` whole planes of together at most 512 groups, or 512
// groups of one larger plane (`segments` of them), lanes over the groups whatever the planes' size; the groups' sums
// meet in LDS, and 64 / planes lanes add up each plane's.  partial[segment * N + n][k].
struct MapUnits {
  uint64_t units;
  Divisor32 segments;
  uint32_t rows;          // planes in all
  uint32_t images;
  int planes, lane_shift; // planes per unit; lanes per plane in the final sum, as a shift
};
template <Elem E>
__global__ __launch_bounds__(kDropThreads) void dropout_maps_grad_kernel(DropoutShape sh, MapUnits mu, DropoutRule rule,
                                                                         const elem_t<E>* x, int64_t x_stride,
                                                                         const float* __restrict__ bias, const elem_t<E>* dy,
                                                                         int64_t dy_stride, elem_t<E>* dx, int64_t dx_stride,
                                                                         float* __restrict__ partial) {
  __shared__ float sums[kDropThreads / 64][kDropUnit];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  uint64_t seed = 0, step = 0;
  if (rule.threshold) {
    seed = rule.rng[0];
    step = rule.rng[1] + rule.offset;
  }
  for (uint64_t unit = blockIdx.x * (uint64_t)(kDropThreads / 64) + wave; unit < mu.units; unit += gridDim.x * (uint64_t)(kDropThreads / 64)) {
    const uint32_t bundle = mu.segments.d == 1 ? (uint32_t)unit : (uint32_t)(unit / mu.segments.d);
    const uint32_t segment = (uint32_t)(unit - (uint64_t)bundle * mu.segments.d);
    const uint32_t row0 = bundle * mu.planes, group0 = segment * kDropUnit;
    const uint32_t planes = min((uint32_t)mu.planes, mu.rows - row0);
    const uint32_t width = min((uint32_t)kDropUnit, sh.groups32.d - group0);
    for (uint32_t it = lane; it < planes * width; it += 64) {
      const uint32_t p = mu.segments.d == 1 ? sh.groups32.quotient(it) : 0;
      const uint32_t row = row0 + p, group = group0 + it - p * width;
      const uint32_t col = group * 8;
      const int n = min(8u, sh.cols - col);
      uint32_t k;
      const Pack<E, 8> g = load_group<E>(dy + row_offset(sh, row, dy_stride, &k) + col, n);
      Pack<E, 8> a = g;
      if (rule.relu) a = load_group<E>(x + row_offset(sh, row, x_stride, &k) + col, n);
      float b[8], dz[8];
      load_bias(sh, bias, k, col, n, b);
      backward_group<E>(rule, g, a, b, keep_bits(rule, seed, step, row, group), dz);
      if (dx) store_group<E>(dx + row_offset(sh, row, dx_stride, &k) + col, n, rounded<E>(dz));
      float sum = 0.0f;  // columns behind the row hold 0
#pragma unroll
      for (int i = 0; i < 8; ++i) sum += i < n ? dz[i] : 0.0f;
      sums[wave][it] = sum;
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    const uint32_t p = lane >> mu.lane_shift, lanes = 1u << mu.lane_shift;
    float sum = 0.0f;
    if (p < planes)
      for (uint32_t i = lane & (lanes - 1); i < width; i += lanes) sum += sums[wave][p * width + i];
    for (uint32_t off = lanes / 2; off; off /= 2) sum += __shfl_xor(sum, off);
    if (p < planes && (lane & (lanes - 1)) == 0) {
      const uint32_t n = sh.channels.quotient(row0 + p);
      partial[((uint64_t)segment * mu.images + n) * sh.channels.d + (row0 + p - n * sh.channels.d)] = sum;
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  }
}

// Backward of feature rows with the bias gradient: a thread keeps 8 columns and walks down rows; the threads of a
// workgroup that share columns meet in LDS.  partial[chunk][column].
template <Elem E>
__global__ __launch_bounds__(kDropThreads) void dropout_features_grad_kernel(
    DropoutShape sh, uint32_t rows, int across_shift, uint32_t rows_per_chunk, DropoutRule rule, const elem_t<E>* x, int64_t x_stride,
    const float* __restrict__ bias, const elem_t<E>* dy, int64_t dy_stride, elem_t<E>* dx, int64_t dx_stride, float* __restrict__ partial) {
  __shared__ float sums[kDropThreads][8];
  const uint32_t across = 1u << across_shift, down = kDropThreads >> across_shift;
  const uint32_t group = blockIdx.x * across + (threadIdx.x & (across - 1));
  const uint32_t col = group * 8;
  const bool inside = group < sh.groups32.d;
  const int n = inside ? min(8u, sh.cols - col) : 0;
  uint64_t seed = 0, step = 0;
  if (rule.threshold) {
    seed = rule.rng[0];
    step = rule.rng[1] + rule.offset;
  }
  float total[8] = {0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f};
  if (inside) {
    float b[8];
    load_bias(sh, bias, 0, col, n, b);
    const uint32_t begin = blockIdx.y * rows_per_chunk, end = min(rows, begin + rows_per_chunk);
#pragma unroll 2
    for (uint32_t row = begin + (threadIdx.x >> across_shift); row < end; row += down) {
      const Pack<E, 8> g = load_group<E>(dy + (int64_t)row * dy_stride + col, n);
      Pack<E, 8> a = g;
      if (rule.relu) a = load_group<E>(x + (int64_t)row * x_stride + col, n);
      float dz[8];
      backward_group<E>(rule, g, a, b, keep_bits(rule, seed, step, row, group), dz);
      if (dx) store_group<E>(dx + (int64_t)row * dx_stride + col, n, rounded<E>(dz));
#pragma unroll
      for (int i = 0; i < 8; ++i) total[i] += dz[i];
    }
  }
#pragma unroll
  for (int i = 0; i < 8; ++i) sums[threadIdx.x][i] = total[i];
  __syncthreads();
  // thread t takes column t of the workgroup's, if there is one
  for (uint32_t c = threadIdx.x; c < across * 8; c += kDropThreads) {
    float sum = 0.0f;
    for (uint32_t d = 0; d < down; ++d) sum += sums[d * across + c / 8][c % 8];
    const uint64_t at = (uint64_t)blockIdx.x * across * 8 + c;
    if (at < sh.cols) partial[(uint64_t)blockIdx.y * sh.cols + at] = sum;
  }
}

// dbias[k] = sum of `parts` rows of partial sums, always in the same order: 64 threads take every 64th row, their sums
// are added in a tree.  Two groups of 8 columns a workgroup.
constexpr int kBiasCols = 16, kBiasDown = 64;
__global__ __launch_bounds__(kBiasCols * kBiasDown) void bias_grad_kernel(const float* __restrict__ partial, uint32_t parts, uint32_t K,
                                                                          float* __restrict__ dbias) {
  __shared__ float sums[kBiasDown][kBiasCols];
  const uint32_t c = threadIdx.x % kBiasCols, d = threadIdx.x / kBiasCols;
  const uint64_t k = (uint64_t)blockIdx.x * kBiasCols + c;
  float sum = 0.0f;
  if (k < K)
    for (uint64_t i = d; i < parts; i += kBiasDown) sum += partial[i * K + k];
  sums[d][c] = sum;
  for (uint32_t half = kBiasDown / 2; half; half /= 2) {
    __syncthreads();
    if (d < half) sums[d][c] += sums[d + half][c];
  }
  if (d == 0 && k < K) dbias[k] = sums[0][c];
}

}  // namespace swconv
