// Host side of what stands around a layer in training and at a network's end: bias, ReLU and dropout, and log
// probabilities, each with its gradient.  Independent of any plan; the calls keep nothing, allocate nothing and only
// enqueue kernels.
#include "../../include/swconv.h"

#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <type_traits>

#include "swconv_dropout_kernels.hpp"
#include "swconv_logprobs_kernels.hpp"

using namespace swconv;

namespace {

constexpr int64_t kMost = (int64_t)1 << 40;  // elements between a tensor's first and last one
// What a pass may read and leave in the 256 MB cache for the next one (a gradient reads its scores again).
constexpr int64_t kCacheBytes = (int64_t)192 << 20;
constexpr int64_t kMaxGroups = (int64_t)1 << 20;  // workgroups of a launch; more work is done in turns

// The stream's device while a call launches, if that is not the current one.
class StreamDevice {
 public:
  explicit StreamDevice(hipStream_t st) {
    static const int count = [] {
      int n = 0;
      if (hipGetDeviceCount(&n) != hipSuccess) (void)hipGetLastError();
      return n;
    }();
    if (count < 2 || !st || st == hipStreamLegacy || st == hipStreamPerThread) return;
    hipDevice_t dev = 0;
    int now = 0;
    if (hipStreamGetDevice(st, &dev) != hipSuccess || hipGetDevice(&now) != hipSuccess) {
      (void)hipGetLastError();
      return;
    }
    if ((int)dev != now && hipSetDevice((int)dev) == hipSuccess) back_ = now;
  }
  ~StreamDevice() {
    if (back_ >= 0 && hipSetDevice(back_) != hipSuccess) (void)hipGetLastError();
  }
  StreamDevice(const StreamDevice&) = delete;

 private:
  int back_ = -1;
};

template <typename... Params, typename... Args>
int launch(void (*kern)(Params...), dim3 grid, int block, hipStream_t st, Args... args) {
  hipLaunchKernelGGL(kern, grid, dim3(block), 0, st, Params(args)...);
  return hipGetLastError() == hipSuccess ? SWCONV_OK : SWCONV_EHIP;
}

bool known_type(int dtype) { return dtype == SWCONV_F32 || dtype == SWCONV_F16 || dtype == SWCONV_BF16; }
int64_t size_of(int dtype) { return dtype == SWCONV_F32 ? 4 : 2; }

template <typename F>
int dispatch_type(int dtype, F&& f) {
  using std::integral_constant;
  if (dtype == SWCONV_F32) return f(integral_constant<Elem, Elem::f32>{});
  if (dtype == SWCONV_F16) return f(integral_constant<Elem, Elem::f16>{});
  return f(integral_constant<Elem, Elem::bf16>{});
}

template <typename F>
int dispatch_bias(int64_t S, int64_t K, const float* bias, F&& f) {
  using std::integral_constant;
  if (S > 1) return f(integral_constant<Bias, Bias::planes>{});
  if (!bias || K % 8 == 0) return f(integral_constant<Bias, Bias::columns>{});  // none: 8 zeros for all
  return K > 8 ? f(integral_constant<Bias, Bias::ragged>{}) : f(integral_constant<Bias, Bias::elements>{});
}

// Rows of `span` elements, `stride` apart.
struct Rows {
  const void* p;
  int64_t rows, span, stride;
};
template <Elem E>
Images<E> images(const Rows& a) {
  return {(elem_t<E>*)a.p, a.stride - a.span, (a.rows - 1) * a.stride + a.span};
}
bool placed(const Rows& a, int64_t size) { return a.p && (uintptr_t)a.p % size == 0; }
// An output may be the input itself, or share no element with it (one row may lie between two of the other's).
bool may_write(const Rows& out, const Rows& in, int64_t size) {
  if (!in.p || !out.p || (out.p == in.p && out.stride == in.stride)) return true;
  const int64_t out_len = ((out.rows - 1) * out.stride + out.span) * size, in_len = ((in.rows - 1) * in.stride + in.span) * size;
  const uintptr_t o = (uintptr_t)out.p, i = (uintptr_t)in.p;
  if (o + (uintptr_t)out_len <= i || i + (uintptr_t)in_len <= o) return true;
  if (out.stride != in.stride) return false;
  const int64_t step = out.stride * size, off = (int64_t)(o - i) % step, at = off < 0 ? off + step : off;
  return at >= in.span * size && at + out.span * size <= step;
}

int ceil_log2(int64_t n) {
  int s = 0;
  while (((int64_t)1 << s) < n) ++s;
  return s;
}

// ---- dropout ------------------------------------------------------------------------------------------------------

// Sizes: the generator counts rows in 32 bits, a tensor spans at most 2^40 elements.
int check_sizes(int64_t N, int64_t K, int64_t S) {
  if (N < 0 || K < 1 || S < 1) return SWCONV_EINVAL;
  if (N >= (int64_t)1 << 31 || K >= (int64_t)1 << 31 || S >= (int64_t)1 << 31) return SWCONV_EUNSUPPORTED;
  if (S > 1 && N * K >= (int64_t)1 << 32) return SWCONV_EUNSUPPORTED;
  if (K * S > kMost) return SWCONV_EUNSUPPORTED;
  return SWCONV_OK;
}
int image_stride(int64_t N, int64_t K, int64_t S, int64_t given, int64_t* stride) {
  *stride = given ? given : K * S;
  if (*stride < K * S) return SWCONV_EINVAL;
  return *stride > kMost || (N > 1 && (N - 1) > kMost / *stride) ? SWCONV_EUNSUPPORTED : SWCONV_OK;
}

DropoutShape shape_of(int dtype, int64_t N, int64_t K, int64_t S) {
  const int64_t rows = S == 1 ? N : N * K, cols = S == 1 ? K : S, groups = (cols + 7) / 8, channels = S == 1 ? 1 : K;
  const uint32_t items = dtype == SWCONV_F32 ? 32 : 64;
  return {Divisor((uint64_t)groups),       Divisor32((uint32_t)groups),   Divisor32((uint32_t)channels),
          (uint64_t)(rows * groups),       (uint32_t)cols,                (uint32_t)(8 * groups - cols),
          (uint32_t)(items % groups),      (uint32_t)(items / groups)};
}

template <Elem E>
dim3 item_grid(const DropoutShape& sh) {
  const int64_t turn = kDropThreads * kDropSteps<E>;
  return dim3((unsigned)std::min<int64_t>(((int64_t)sh.items + turn - 1) / turn, kMaxGroups));
}

int rule_of(int64_t N, int relu, float p, const uint64_t* rng, uint64_t offset, DropoutRule* rule) {
  if (!(p >= 0.0f && p <= 1.0f)) return SWCONV_EINVAL;
  const uint32_t threshold = (uint32_t)std::lrint((double)p * 65536.0);
  if (N && threshold && (!rng || (uintptr_t)rng % sizeof(uint64_t))) return SWCONV_EINVAL;
  *rule = {rng, offset, threshold, threshold < 65536 ? 65536.0f / (float)(65536 - threshold) : 0.0f, relu != 0};
  return SWCONV_OK;
}

// How the bias gradient is summed: partial sums in `parts` rows of K (whatever the type).
struct BiasParts {
  int64_t parts;
  MapUnits units{0, Divisor32(1), 0, 0, 1, 6};
};
BiasParts bias_parts(int64_t N, int64_t K, int64_t S) {
  BiasParts b;
  const int64_t cols = S == 1 ? K : S, groups = (cols + 7) / 8;
  if (S > 1) {
    const int64_t segments = (groups + kDropUnit - 1) / kDropUnit;
    // planes to a wave: what fills its steps of 64 items best, in 4096 waves at least if there is as much work (64 x 384
    // planes of 13 x 13 fp32: 23 planes to a wave 15.6 us, 5 planes 11.7; 4 x 384 planes 11.9 and 4.8).
    const int64_t most = std::clamp<int64_t>(N * K * groups / 4096, groups, std::max<int64_t>(groups, kDropUnit));
    int planes = 1;
    double best = 0;
    for (int p = 1; p <= 64 && p * groups <= most; ++p) {
      const double filled = (double)(p * groups) / (double)((p * groups + 63) / 64 * 64);
      if (filled >= best) planes = p, best = filled;
    }
    b.units = {(uint64_t)((N * K + planes - 1) / planes * segments), Divisor32((uint32_t)segments), (uint32_t)(N * K),
               (uint32_t)N, planes, 6 - ceil_log2(planes)};
    b.parts = N * segments;
  } else {
    // 1024 workgroups of the 16-bit types, each with its rows in flight at least
    const int64_t across = std::min<int64_t>(kDropThreads, (int64_t)1 << ceil_log2(groups));
    const int64_t col_blocks = (groups + across - 1) / across, down = kBiasRows * (kDropThreads / across);
    b.parts = std::clamp<int64_t>((N + down - 1) / down, 1, std::max<int64_t>(1, 1024 / col_blocks));
  }
  return b;
}

// ---- log probabilities --------------------------------------------------------------------------------------------

int check_scores(int dtype, int64_t rows, int64_t classes, int64_t given, int64_t* stride) {
  if (!known_type(dtype) || rows < 0 || classes < 1) return SWCONV_EINVAL;
  if (classes >= ((int64_t)1 << 31) - 4096) return SWCONV_EUNSUPPORTED;  // class numbers of 32 bits, a tile further
  *stride = given ? given : classes;
  if (*stride < classes) return SWCONV_EINVAL;
  return rows > kMost || *stride > kMost || (rows > 1 && rows - 1 > kMost / *stride) ? SWCONV_EUNSUPPORTED : SWCONV_OK;
}

// How many waves share a row, and into how many parts it is cut.  A tile is what a wave reads at a time, 4 KB; aligned: every
// row begins on 4 bytes.  Times of bf16 rows with entropies and the best class in us, inputs from memory:
//   a wave per row where rows alone fill the chip, 7 to a CU (32768 classes of 1536 rows 35, four waves 31; of 1792 36 and 37,
//   of 4096 64 and 74), for short rows, of which four waves get few tiles each, from 160 rows to a tile on (256 without best
//   classes, whose second look costs four waves more), 4 to a CU at least (5): 16384 classes of 1024 rows 20 and 19, of 1280 22
//   and 21, of 1536 22 and 23.  Up to 24 tiles: 49152 classes of 4096 rows 86 and 95, 131072 of them 228 and 221, fp32 24576
//   classes 82 and 85, 65536 classes 222 and 208; up to 10 without best classes: 20480 classes of 4096 rows 37 and 41, 32768 60
//   and 54.  Rows that are not aligned, which four waves read more slowly (131035 classes of 4096 rows 231 and 263), at any
//   length, with more than 8 best classes up to 32 tiles (2048 rows with the best 20: 65499 classes 80 and 81, 131035 classes
//   158 and 144).  Rows of one or two tiles in any case;
//   four waves of a workgroup, sixteen for rows of 12 tiles at least while a CU has only one of them: 131072 classes of 256
//   rows 22 (four waves 25), 257 rows 35 (28); 24576 classes 10 (11) and 17 (12);
//   parts of at least 6 tiles and a second launch for few rows, up to two workgroups a CU, here with the best 5: 1 x 131072 13
//   (one workgroup 18), 64 x 131072 18 (20); from 64 rows on parts of 16 tiles, past 128 rows none: 256 x 131072 in two parts
//   27 (23).
struct Parts {
  int waves, parts;
  int64_t part_classes;
};
Parts parts_of(int dtype, int64_t rows, int64_t classes, int top, bool aligned) {
  const int64_t tile = 64 * (16 / size_of(dtype)) * kLogpUnroll, tiles = (classes + tile - 1) / tile;
  const int64_t filled = top ? std::clamp<int64_t>(160 * tiles, 1024, 1792) : std::clamp<int64_t>(256 * tiles, 1280, 1792);
  const int64_t longest = aligned ? (top ? 24 : 10) : top > 8 ? 32 : tiles;
  if (tiles <= 2 || (rows >= filled && tiles <= longest)) return {1, 1, classes};
  if (rows > 256 || tiles < 12) return {4, 1, classes};
  int64_t parts = 1;
  if (rows > 0 && rows <= 128)
    parts = std::min({(int64_t)512 / rows, tiles / (rows >= 64 ? 16 : 6), 16 + tiles / 64, (int64_t)64});
  if (parts < 3) return {16, 1, classes};
  const int64_t each = ((tiles + parts - 1) / parts + 3) / 4 * 4 * tile;  // as many tiles to each of its four waves
  return {4, (int)((classes + each - 1) / each), each};
}
int64_t parts_bytes(const Parts& p, int64_t rows, int top) {
  return p.parts == 1 ? 0 : rows * p.parts * ((int64_t)sizeof(RowSums) + top * (int64_t)sizeof(TopKey));
}

}  // namespace

extern "C" {

int swconv_dropout_forward(int dtype, int64_t N, int64_t K, int64_t S, const void* x_dev, int64_t x_stride,
                           const float* bias_dev, int relu, float p, const uint64_t* rng_dev, uint64_t offset,
                           void* hip_stream, void* y_dev, int64_t y_stride) {
  int rc;
  DropoutRule rule;
  if (!known_type(dtype)) return SWCONV_EINVAL;
  if ((rc = check_sizes(N, K, S)) || (rc = image_stride(N, K, S, x_stride, &x_stride)) ||
      (rc = image_stride(N, K, S, y_stride, &y_stride)) || (rc = rule_of(N, relu, p, rng_dev, offset, &rule)))
    return rc;
  if (N == 0) return SWCONV_OK;
  const int64_t size = size_of(dtype);
  const Rows x{x_dev, N, K * S, x_stride}, y{y_dev, N, K * S, y_stride};
  if (!placed(x, size) || !placed(y, size) || !may_write(y, x, size) || (uintptr_t)bias_dev % 4) return SWCONV_EINVAL;
  const hipStream_t st = (hipStream_t)hip_stream;
  const StreamDevice device(st);
  const DropoutShape sh = shape_of(dtype, N, K, S);
  const bool once = 2 * N * K * S * size > kCacheBytes;
  const bool dense = sh.pad == 0 && x_stride == K * S && y_stride == K * S;
  return dispatch_type(dtype, [&](auto e) {
    constexpr Elem E = decltype(e)::value;
    const dim3 grid = item_grid<E>(sh);
    return dispatch_bias(S, K, bias_dev, [&](auto by) {
      return launch(dropout_kernel<E, Pass::forward, decltype(by)::value>, grid, kDropThreads, st, sh, rule,
                    images<E>(x), bias_dev, Images<E>{}, images<E>(y), dense, once);
    });
  });
}

int swconv_dropout_workspace_bytes(int64_t N, int64_t K, int64_t S, int64_t* bytes) {
  if (!bytes) return SWCONV_EINVAL;
  if (int rc = check_sizes(N, K, S)) return rc;
  const int64_t parts = bias_parts(N, K, S).parts;
  *bytes = parts > 1 ? parts * K * (int64_t)sizeof(float) : 0;
  return SWCONV_OK;
}

int swconv_dropout_backward(int dtype, int64_t N, int64_t K, int64_t S, const void* dy_dev, int64_t dy_stride, const void* x_dev,
                            int64_t x_stride, const float* bias_dev, int relu, float p, const uint64_t* rng_dev, uint64_t offset,
                            void* workspace_dev, int64_t workspace_bytes, void* hip_stream, void* dx_dev, int64_t dx_stride,
                            float* dbias_dev) {
  int rc;
  DropoutRule rule;
  if (!known_type(dtype)) return SWCONV_EINVAL;
  if ((rc = check_sizes(N, K, S)) || (rc = image_stride(N, K, S, dy_stride, &dy_stride)) ||
      (rc = image_stride(N, K, S, x_stride, &x_stride)) || (rc = image_stride(N, K, S, dx_stride, &dx_stride)) ||
      (rc = rule_of(N, relu, p, rng_dev, offset, &rule)))
    return rc;
  if ((uintptr_t)bias_dev % 4 || (uintptr_t)dbias_dev % 4 || (uintptr_t)workspace_dev % 4) return SWCONV_EINVAL;
  const hipStream_t st = (hipStream_t)hip_stream;
  const BiasParts bp = bias_parts(N, K, S);
  const dim3 sum_grid((unsigned)std::min<int64_t>((K + kBiasCols - 1) / kBiasCols, kMaxGroups));
  if (N == 0) {
    if (!dbias_dev) return SWCONV_OK;
    const StreamDevice device(st);
    return launch(bias_grad_kernel, sum_grid, kBiasCols * kBiasDown, st, (const float*)nullptr, 0u, (uint32_t)K, dbias_dev);
  }
  const int64_t size = size_of(dtype);
  const Rows dy{dy_dev, N, K * S, dy_stride}, x{relu ? x_dev : nullptr, N, K * S, x_stride}, dx{dx_dev, N, K * S, dx_stride};
  if (!placed(dy, size) || (relu && !placed(x, size)) || (!dx_dev && !dbias_dev)) return SWCONV_EINVAL;
  if (dx_dev && (!placed(dx, size) || !may_write(dx, dy, size) || !may_write(dx, x, size))) return SWCONV_EINVAL;
  const DropoutShape sh = shape_of(dtype, N, K, S);
  if (dbias_dev && bp.parts > 1 &&
      (!workspace_dev || workspace_bytes < bp.parts * K * (int64_t)sizeof(float)))
    return SWCONV_EINVAL;
  float* partial = bp.parts > 1 ? (float*)workspace_dev : dbias_dev;
  const bool once = (relu ? 3 : 2) * N * K * S * size > kCacheBytes;
  const bool dense = sh.pad == 0 && dy_stride == K * S && dx_stride == K * S && (!relu || x_stride == K * S);
  const StreamDevice device(st);
  rc = dispatch_type(dtype, [&](auto e) {
    constexpr Elem E = decltype(e)::value;
    const Images<E> g = images<E>(dy), a = images<E>(x), d = images<E>(dx);
    if (!dbias_dev) {
      const dim3 grid = item_grid<E>(sh);
      if (!relu)
        return launch(dropout_kernel<E, Pass::backward, Bias::planes>, grid, kDropThreads, st, sh, rule, a, bias_dev, g,
                      d, dense, once);
      return dispatch_bias(S, K, bias_dev, [&](auto by) {
        return launch(dropout_kernel<E, Pass::backward_relu, decltype(by)::value>, grid, kDropThreads, st, sh, rule, a,
                      bias_dev, g, d, dense, once);
      });
    }
    if (S > 1) {
      const int64_t waves = kDropThreads / 64;
      const dim3 grid((unsigned)std::min<int64_t>(((int64_t)bp.units.units + waves - 1) / waves, kMaxGroups));
      auto kernel = relu ? dropout_maps_grad_kernel<E, true> : dropout_maps_grad_kernel<E, false>;
      return launch(kernel, grid, kDropThreads, st, sh, bp.units, rule, a, bias_dev, g, d, partial, once);
    }
    const int64_t chunks = (K + 7) / 8 * kHalves<E>;  // of 16 bytes
    const int across_shift = std::min(8, ceil_log2(chunks));
    const dim3 grid((unsigned)((chunks + (1 << across_shift) - 1) >> across_shift), (unsigned)bp.parts);
    auto kernel = !relu                     ? dropout_features_grad_kernel<E, false, Bias::columns>
                  : !bias_dev || K % 8 == 0 ? dropout_features_grad_kernel<E, true, Bias::columns>
                                            : dropout_features_grad_kernel<E, true, Bias::elements>;
    return launch(kernel, grid, kDropThreads, st, sh, (uint32_t)N, across_shift, rule, a, bias_dev, g, d,
                  partial, once);
  });
  if (rc || !dbias_dev || bp.parts == 1) return rc;
  return launch(bias_grad_kernel, sum_grid, kBiasCols * kBiasDown, st, (const float*)partial, (uint32_t)bp.parts,
                (uint32_t)K, dbias_dev);
}

int swconv_logprobs_workspace_bytes(int dtype, int64_t rows, int64_t classes, int top, int64_t* bytes) {
  int64_t stride;
  if (!bytes) return SWCONV_EINVAL;
  if (int rc = check_scores(dtype, rows, classes, 0, &stride)) return rc;
  if (top < 0) return SWCONV_EINVAL;
  if (top > kTopMax) return SWCONV_EUNSUPPORTED;
  *bytes = parts_bytes(parts_of(dtype, rows, classes, top, true), rows, top);  // parts are of few rows, aligned or not
  return SWCONV_OK;
}

int swconv_logprobs_forward(int dtype, int64_t rows, int64_t classes, const void* scores_dev, int64_t row_stride,
                            const int32_t* labels_dev, int top, void* workspace_dev, int64_t workspace_bytes,
                            void* hip_stream, float* logprob_dev, float* entropy_dev, float* stats_dev,
                            int32_t* top_class_dev, float* top_logprob_dev) {
  if (int rc = check_scores(dtype, rows, classes, row_stride, &row_stride)) return rc;
  if (top < 0) return SWCONV_EINVAL;
  if (top > kTopMax) return SWCONV_EUNSUPPORTED;
  if (rows == 0) return SWCONV_OK;
  const int64_t size = size_of(dtype);
  const Rows x{scores_dev, rows, classes, row_stride};
  if (!placed(x, size) || (logprob_dev && !labels_dev) || (top > 0) != (top_class_dev && top_logprob_dev) ||
      (!logprob_dev && !entropy_dev && !stats_dev && !top))
    return SWCONV_EINVAL;
  for (const void* p : {(const void*)labels_dev, (const void*)logprob_dev, (const void*)entropy_dev, (const void*)stats_dev,
                        (const void*)top_class_dev, (const void*)top_logprob_dev})
    if ((uintptr_t)p % 4) return SWCONV_EINVAL;
  const bool aligned = (uintptr_t)scores_dev % 4 == 0 && row_stride * size % 4 == 0;
  const Parts pt = parts_of(dtype, rows, classes, top, aligned);
  if (pt.parts > 1 &&
      (!workspace_dev || (uintptr_t)workspace_dev % 16 || workspace_bytes < parts_bytes(pt, rows, top)))
    return SWCONV_EINVAL;
  auto* part_sums = (RowSums*)workspace_dev;
  auto* part_keys = (TopKey*)(part_sums + rows * pt.parts);
  const LogprobsOut out{logprob_dev, entropy_dev, stats_dev, top_class_dev, top_logprob_dev};
  const hipStream_t st = (hipStream_t)hip_stream;
  const StreamDevice device(st);
  const bool once = rows * classes * size > kCacheBytes;
  return dispatch_type(dtype, [&](auto e) {
    constexpr Elem E = decltype(e)::value;
    const auto* s = (const elem_t<E>*)scores_dev;
    auto part = [&](auto waves, auto with_top, auto with_entropy) {
      constexpr int W = decltype(waves)::value;
      constexpr int kRows = W == 1 ? 4 : 1;  // parts of a workgroup
      const dim3 grid((unsigned)std::min((rows * pt.parts + kRows - 1) / kRows, kMaxGroups));
      return launch(logprobs_kernel<E, W, decltype(with_top)::value, decltype(with_entropy)::value>, grid,
                    W == 1 ? 256 : W * 64, st, rows, classes, s, row_stride, labels_dev, top, pt.parts, pt.part_classes,
                    once, out, part_sums, part_keys);
    };
    auto entropy = [&](auto waves, auto with_top) {
      return entropy_dev ? part(waves, with_top, std::true_type{}) : part(waves, with_top, std::false_type{});
    };
    auto best = [&](auto waves) { return top ? entropy(waves, std::true_type{}) : entropy(waves, std::false_type{}); };
    using std::integral_constant;
    const int rc = pt.waves == 1   ? best(integral_constant<int, 1>{})
                   : pt.waves == 4 ? best(integral_constant<int, 4>{})
                                   : best(integral_constant<int, 16>{});
    if (rc || pt.parts == 1) return rc;
    return launch(logprobs_join_kernel<E>, dim3((unsigned)std::min(rows, kMaxGroups)), 256, st, rows, classes, s,
                  row_stride, labels_dev, top, pt.parts, out, (const RowSums*)part_sums, (const TopKey*)part_keys);
  });
}

int swconv_logprobs_backward(int dtype, int64_t rows, int64_t classes, const void* scores_dev, int64_t row_stride,
                             const int32_t* labels_dev, const float* stats_dev, const float* entropy_dev,
                             const float* dlogprob_dev, const float* dentropy_dev, void* hip_stream, void* dscores_dev,
                             int64_t dscores_stride) {
  if (int rc = check_scores(dtype, rows, classes, row_stride, &row_stride)) return rc;
  if (int rc = check_scores(dtype, rows, classes, dscores_stride, &dscores_stride)) return rc;
  if (rows == 0) return SWCONV_OK;
  const int64_t size = size_of(dtype);
  const Rows x{scores_dev, rows, classes, row_stride}, dx{dscores_dev, rows, classes, dscores_stride};
  if (!placed(x, size) || !placed(dx, size) || !may_write(dx, x, size) || !stats_dev || (dlogprob_dev && !labels_dev) ||
      (dentropy_dev && !entropy_dev) || (!dlogprob_dev && !dentropy_dev))
    return SWCONV_EINVAL;
  for (const void* p : {(const void*)labels_dev, (const void*)stats_dev, (const void*)entropy_dev, (const void*)dlogprob_dev,
                        (const void*)dentropy_dev})
    if ((uintptr_t)p % 4) return SWCONV_EINVAL;
  const hipStream_t st = (hipStream_t)hip_stream;
  const StreamDevice device(st);
  const GradIn in{labels_dev, stats_dev, entropy_dev, dlogprob_dev, dentropy_dev};
  const bool once = 2 * rows * classes * size > kCacheBytes;
  return dispatch_type(dtype, [&](auto e) {
    constexpr Elem E = decltype(e)::value;
    const auto* s = (const elem_t<E>*)scores_dev;
    auto* d = (elem_t<E>*)dscores_dev;
    const int64_t groups = (classes + kWordsElems<E> - 1) / kWordsElems<E>;
    auto grad = [&](auto with_entropy) {
      constexpr bool H = decltype(with_entropy)::value;
      if (groups >= 128) {
        constexpr int64_t kGroups = kGradThreads * kGradUnroll<E>;
        const dim3 grid((unsigned)((groups + kGroups - 1) / kGroups), (unsigned)std::min<int64_t>(rows, 65535));
        return launch(logprobs_grad_kernel<E, H>, grid, kGradThreads, st, rows, classes, s, row_stride, in, once, d,
                      dscores_stride);
      }
      const int shift = ceil_log2(groups);
      const int64_t down = kGradThreads >> shift;
      const dim3 grid((unsigned)std::min((rows + down - 1) / down, kMaxGroups));
      return launch(logprobs_grad_short_kernel<E, H>, grid, kGradThreads, st, rows, classes, s, row_stride, in, shift, d,
                    dscores_stride);
    };
    return dentropy_dev ? grad(std::true_type{}) : grad(std::false_type{});
  });
}

}  // extern "C"
