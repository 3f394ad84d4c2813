// HIP kernels of bias, ReLU and dropout between two layers, and of their backward pass:
//   z = x + bias[k],  a = relu ? max(z, 0) : z,  y = keep ? a * scale : 0
//   dz = keep and (z > 0 or no relu) ? dy * scale : 0,  dx = dz,  dbias[k] = sum over n, s of dz
// The mask is never stored: keep(row, col) = 16-bit field col % 8 of philox4x32-10 (Salmon, Moraes, Dror, Shaw,
// "Parallel random numbers: as easy as 1, 2, 3", 2011) at counter {col / 8, row, step}, so that any thread makes any
// element's decision alone and the backward pass makes the forward pass's.  An item of 8 columns costs one call, 20
// products of 32 x 32 bits.  16 bits an element round the rate to a multiple of 2^-16; the scale is that rate's, so the
// mean is kept exactly.  Arithmetic in fp32, one rounding to the element type at the end.
// Bound by memory: 32 x 256 x 56 x 56 fp32 5.0 TB/s read and written (41 us), 16384 x 4096 fp32 5.6, bf16 5.0 (53 us), where the
// generator's products and the unpacking keep the vector units 69 % busy.
#pragma once
#include "swconv_elements.hpp"
#include "swconv_lanes.hpp"

namespace swconv {

constexpr int kDropThreads = 256;
template <Elem E>
constexpr int kDropSteps = E == Elem::f32 ? 1 : 2;  // of 64 items, to a wave and turn: 32 bytes of loads to a lane
constexpr int kDropUnit = 512;                      // items that a wave of the gradient of maps sums up at a time

struct DropoutRule {
  const uint64_t* rng;  // seed, step; not read when threshold is 0
  uint64_t offset;
  uint32_t threshold;   // drop a field below it, 0 .. 65536
  float scale;
  int relu;
};
struct Generator {
  uint64_t seed, step;
  __device__ __forceinline__ explicit Generator(const DropoutRule& rule)
      : seed(rule.threshold ? rule.rng[0] : 0), step(rule.threshold ? rule.rng[1] + rule.offset : 0) {}
};

// Rows of the generator: planes (n, k) of S columns, or with S = 1 images (n, 0) of K columns.  An item is a group of 8
// columns of a row.
struct DropoutShape {
  Divisor groups;       // in a row
  Divisor32 groups32, channels;
  uint64_t items;       // rows * groups
  uint32_t cols;
  uint32_t pad;         // columns that the last item of a row lacks
  uint32_t stride_group, stride_row;  // 64 / kHalves items, taken apart
};

// An item; `ahead` counts it from the first one of its wave's turn.
struct Place {
  uint32_t row, group, ahead;
};
// The item `ahead` (below 2^31) behind a first one.
__device__ __forceinline__ Place place_at(const DropoutShape& sh, uint64_t first, uint32_t ahead) {
  const uint32_t row0 = (uint32_t)sh.groups.quotient(first);
  const uint32_t at = (uint32_t)(first - (uint64_t)row0 * sh.groups.d) + ahead, over = sh.groups32.quotient(at);
  return {row0 + over, at - over * sh.groups32.d, ahead};
}
template <int STRIDE>
__device__ __forceinline__ Place next_place(const DropoutShape& sh, Place p) {
  p.group += sh.stride_group;
  const uint32_t wrap = p.group >= sh.groups32.d;
  p.group -= wrap ? sh.groups32.d : 0;
  p.row += sh.stride_row + wrap;
  p.ahead += STRIDE;
  return p;
}

struct KeepWords {
  uint32_t w[4];  // 8 fields of 16 bits
};
__device__ __forceinline__ KeepWords keep_words(const Generator& g, uint32_t row, uint32_t group) {
  uint32_t c[4] = {group, row, (uint32_t)g.step, (uint32_t)(g.step >> 32)};
  uint32_t k0 = (uint32_t)g.seed, k1 = (uint32_t)(g.seed >> 32);
#pragma unroll
  for (int r = 0; r < 10; ++r) {
    const uint64_t a = (uint64_t)0xD2511F53u * c[0], b = (uint64_t)0xCD9E8D57u * c[2];
    c[0] = __builtin_amdgcn_bitop3_b32((uint32_t)(b >> 32), c[1], k0, 0x96);  // the exclusive or of all three
    c[1] = (uint32_t)b;
    c[2] = __builtin_amdgcn_bitop3_b32((uint32_t)(a >> 32), c[3], k1, 0x96);
    c[3] = (uint32_t)a;
    k0 += 0x9E3779B9u;
    k1 += 0xBB67AE85u;
  }
  return {{c[0], c[1], c[2], c[3]}};
}

// A lane works on chunks of 16 bytes, so that a wave's accesses are runs of 1 KB.  A chunk of the 16-bit types is an item.
// Of fp32 an item is two chunks: a pair of lanes holds two items, each lane one half of both (half 0 of the even lane
// first), makes the words of one and gets those of its half of the other from its neighbour.
template <Elem E>
constexpr int kChunk = kWordsElems<E>;
template <Elem E>
constexpr int kHalves = 8 / kChunk<E>;

template <Elem E>
__device__ __forceinline__ uint32_t lane_item(int lane) {
  return kHalves<E> == 1 ? lane : lane / 2;
}
template <Elem E>
__device__ __forceinline__ uint32_t first_column(const Place& p, int lane) {
  return p.group * 8 + (kHalves<E> == 1 ? 0 : (lane & 1) * 4);
}
// The keep words of a lane's chunks: kChunk / 2 for each.
template <Elem E>
__device__ __forceinline__ void chunk_words(const Generator& g, const Place& first, const Place& second, int lane,
                                            uint32_t (&w)[kHalves<E>][kChunk<E> / 2]) {
  if constexpr (kHalves<E> == 1) {
    const KeepWords k = keep_words(g, first.row, first.group);
#pragma unroll
    for (int i = 0; i < 4; ++i) w[0][i] = k.w[i];
  } else {
    const bool odd = lane & 1;
    const uint32_t row0 = first.row, row1 = second.row, group0 = first.group, group1 = second.group;
    const KeepWords k = keep_words(g, odd ? row1 : row0, odd ? group1 : group0);
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const uint32_t got = lane_xor<1>(odd ? k.w[i] : k.w[2 + i], lane);
      w[0][i] = odd ? got : k.w[i];
      w[1][i] = odd ? k.w[2 + i] : got;
    }
  }
}
template <int N>
__device__ __forceinline__ bool kept(const uint32_t (&w)[N], int i, uint32_t threshold) {
  return (i % 2 ? w[i / 2] >> 16 : w[i / 2] & 0xffffu) >= threshold;
}

// A tensor of images; `gap`: elements between one and the next, `span`: from the first to behind the last.
template <Elem E>
struct Images {
  elem_t<E>* p;
  int64_t gap, span;
};
// Where a lane's chunks begin: items of 8 columns, less what the rows before lack, and the gaps between images.
template <Elem E, int COUNT>
__device__ __forceinline__ void chunk_offsets(const DropoutShape& sh, uint64_t first, const Place (&at)[COUNT],
                                              int64_t gap, int lane, int64_t (&offset)[COUNT]) {
  const int half = kHalves<E> == 1 ? 0 : (lane & 1) * 4;
#pragma unroll
  for (int c = 0; c < COUNT; ++c) {
    offset[c] = (int64_t)(first * 8) + (at[c].ahead * 8 + half) - (int64_t)((uint64_t)at[c].row * sh.pad);
    if (gap) offset[c] += (int64_t)sh.channels.quotient(at[c].row) * gap;
  }
}
// Whether 16 bytes can be read at all of a wave's chunks.  A chunk that its row does not fill is read to its end all the same
// (what is behind a row is not used); only behind the tensor's last elements nothing is.
template <Elem E, int COUNT>
__device__ __forceinline__ bool readable(const DropoutShape& sh, const Images<E>& x, uint64_t first, const Place (&at)[COUNT],
                                         const int (&n)[COUNT], int lane) {
  int64_t offset[COUNT];
  chunk_offsets<E>(sh, first, at, x.gap, lane, offset);
  bool end = x.span < kChunk<E>;
#pragma unroll
  for (int c = 0; c < COUNT; ++c) end |= n[c] > 0 && offset[c] + kChunk<E> > x.span;
  return __ballot(end) == 0;
}
// Where readable() said no, chunks are read by the element.  The way is fixed at compile time for a whole turn: where ways
// meet behind loads, the compiler waits for them, and they would not go out together.
enum class Read { whole, once, elements };
template <Elem E, Read HOW, int COUNT>
__device__ __forceinline__ void load_chunks(const Images<E>& x, const int64_t (&offset)[COUNT], const int (&n)[COUNT],
                                            Words (&w)[COUNT]) {
#pragma unroll
  for (int c = 0; c < COUNT; ++c) {
    if constexpr (HOW != Read::elements)
      w[c] = load_words<E>(x.p + (n[c] > 0 ? offset[c] : 0), HOW == Read::once);
    else if (n[c] > 0)
      w[c] = n[c] == kChunk<E> ? load_words<E>(x.p + offset[c], false) : load_words_part<E>(x.p + offset[c], n[c]);
  }
}
template <typename F>
__device__ __forceinline__ void choose_read(bool whole, bool once, F&& f) {
  using std::integral_constant;
  if (!whole)
    f(integral_constant<Read, Read::elements>{});
  else if (once)
    f(integral_constant<Read, Read::once>{});
  else
    f(integral_constant<Read, Read::whole>{});
}
template <Elem E>
__device__ __forceinline__ void store_chunk(elem_t<E>* p, int n, const float (&v)[kChunk<E>], bool once) {
  Pack<E, kChunk<E>> a;
#pragma unroll
  for (int i = 0; i < kChunk<E>; ++i) a.v[i] = (elem_t<E>)v[i];
  if (n >= kChunk<E>)
    store_words<E>(p, __builtin_bit_cast(Words, a), once);
  else
    store_part<E, kChunk<E>>(p, n, a);
}
// Columns of a chunk that its row has (0 or less: none).
template <Elem E>
__device__ __forceinline__ int chunk_size(const DropoutShape& sh, uint32_t col) {
  return (int)min((int64_t)sh.cols - col, (int64_t)kChunk<E>);
}
// The bias by channels of maps, by columns of features, by columns that fill no item at the end of a row: there the bias's
// last V are read for its last chunk, and shift_biases moves them; rows of less than a chunk and kernels that read their bias
// once take it by the element (7416 x 8603 fp16 by the element 142 us, so 60.6).  None: zeros.
enum class Bias { planes, columns, ragged, elements };
__device__ const float kNoBias[8] = {};
struct BiasAt {
  const float* p;
  uint32_t step;  // 0: none
  __device__ __forceinline__ explicit BiasAt(const float* bias) : p(bias ? bias : kNoBias), step(bias ? 1 : 0) {}
};
template <Elem E, Bias B>
__device__ __forceinline__ void load_bias(const DropoutShape& sh, const BiasAt& bias, uint32_t row, uint32_t col, int n,
                                          float (&b)[kChunk<E>]) {
  constexpr int V = kChunk<E>;
  if constexpr (B == Bias::planes) {
    const uint32_t k = row - sh.channels.quotient(row) * sh.channels.d;
    const float one = bias.p[(n > 0 ? k : 0) * bias.step];
#pragma unroll
    for (int i = 0; i < V; ++i) b[i] = one;
  } else if constexpr (B == Bias::columns) {
    const Pack<Elem::f32, V> v = load_pack<Elem::f32, V>(bias.p + (n > 0 ? col : 0) * bias.step);
#pragma unroll
    for (int i = 0; i < V; ++i) b[i] = v.v[i];
  } else if constexpr (B == Bias::ragged) {
    const Pack<Elem::f32, V> v = load_pack<Elem::f32, V>(bias.p + (n > 0 ? min(col, sh.cols - V) : 0) * bias.step);
#pragma unroll
    for (int i = 0; i < V; ++i) b[i] = v.v[i];
  } else {
#pragma unroll
    for (int i = 0; i < V; ++i) b[i] = bias.p[min(col + i, sh.cols - 1) * bias.step];
  }
}

// The biases of chunks of n columns each from those of a row's last V, n of which are their own; few waves have such chunks.
// fp32 looks at each chunk for itself (3708 x 8603 47 us, at all of a turn at once 53), the 16-bit types at all at once (7416 x
// 8603 fp16 60.6 us in 40 registers; chunk by chunk 67).
template <Elem E, int COUNT>
__device__ __forceinline__ void shift_biases(const int* n, float (*b)[kChunk<E>]) {
  constexpr int V = kChunk<E>;
  bool any = false;
#pragma unroll
  for (int c = 0; c < COUNT; ++c) any |= n[c] > 0 && n[c] < V;
  if (__ballot(any) == 0) return;
#pragma unroll
  for (int c = 0; c < COUNT; ++c) {
    const int by = n[c] > 0 ? V - n[c] : 0;
#pragma unroll
    for (int step = V / 2; step; step /= 2)
#pragma unroll
      for (int i = 0; i + step < V; ++i) b[c][i] = by & step ? b[c][i + step] : b[c][i];
  }
}

// A dropped element is 0 whatever it was; a NaN that is kept stays one.
template <Elem E>
__device__ __forceinline__ void forward_chunk(const DropoutRule& rule, const Words& x, const float (&b)[kChunk<E>],
                                              const uint32_t (&w)[kChunk<E> / 2], float (&y)[kChunk<E>]) {
#pragma unroll
  for (int i = 0; i < kChunk<E>; ++i) {
    float z = word_elem<E>(x, i) + b[i];
    if (rule.relu) z = __builtin_elementwise_maximum(z, 0.0f);
    y[i] = kept(w, i, rule.threshold) ? z * rule.scale : 0.0f;
  }
}
template <Elem E, bool RELU>
__device__ __forceinline__ void backward_chunk(const DropoutRule& rule, const Words& dy, const Words& x, const float (&b)[kChunk<E>],
                                               const uint32_t (&w)[kChunk<E> / 2], float (&dz)[kChunk<E>]) {
#pragma unroll
  for (int i = 0; i < kChunk<E>; ++i) {
    bool pass = kept(w, i, rule.threshold);
    if constexpr (RELU) pass = pass && !(word_elem<E>(x, i) + b[i] <= 0.0f);
    dz[i] = pass ? word_elem<E>(dy, i) * rule.scale : 0.0f;
  }
}

// Forward, and backward without a bias gradient: waves over all items in the order of memory.  Bound by memory: a chunk in
// (two with ReLU backward) and a chunk out.
enum class Pass { forward, backward, backward_relu };
template <Elem E>
constexpr int kTurnChunks = kDropSteps<E> * kHalves<E>;

// The chunks of a wave's turn: their items, and how many columns of each there are.
template <Elem E>
__device__ __forceinline__ void turn_places(const DropoutShape& sh, uint64_t first, int lane, Place (&at)[kTurnChunks<E>]) {
  at[0] = place_at(sh, first, lane_item<E>(lane));
#pragma unroll
  for (int c = 1; c < kTurnChunks<E>; ++c) at[c] = next_place<64 / kHalves<E>>(sh, at[c - 1]);
}

// DENSE: rows of whole items and no gaps anywhere.  Then a chunk lies where its number says, and the loads go out before the
// places are worked out (which takes as long, with eight waves to a SIMD, as the loads).
template <Elem E, Pass PASS, Bias B, Read HOW, bool DENSE>
__device__ __forceinline__ void dropout_turn(const DropoutShape& sh, const DropoutRule& rule, const Images<E>& x, const float* bias,
                                             const Images<E>& dy, const Images<E>& out, uint64_t first, uint32_t left,
                                             Place (&at)[kTurnChunks<E>], int lane) {
  constexpr int H = kHalves<E>, V = kChunk<E>, COUNT = kTurnChunks<E>;
  Words in[COUNT], gate[COUNT];
  int64_t offset[COUNT];
  int n[COUNT];
  float b[COUNT][V];
  const Images<E>& from = PASS == Pass::forward ? x : dy;
  if constexpr (DENSE) {
#pragma unroll
    for (int c = 0; c < COUNT; ++c) {
      const uint32_t ahead = lane_item<E>(lane) + c * (64 / H);
      offset[c] = (int64_t)(first * 8) + (ahead * 8 + (H == 1 ? 0 : (lane & 1) * 4));
      n[c] = ahead < left ? V : 0;
    }
  } else {
#pragma unroll
    for (int c = 0; c < COUNT; ++c) n[c] = at[c].ahead < left ? chunk_size<E>(sh, first_column<E>(at[c], lane)) : 0;
    chunk_offsets<E>(sh, first, at, from.gap, lane, offset);
  }
  load_chunks<E, HOW>(from, offset, n, in);
  if constexpr (PASS == Pass::backward_relu) {
    if (!DENSE && x.gap != dy.gap) chunk_offsets<E>(sh, first, at, x.gap, lane, offset);
    load_chunks<E, HOW>(x, offset, n, gate);
  }
  if constexpr (DENSE) turn_places<E>(sh, first, lane, at);
  if constexpr (PASS != Pass::backward) {
    const BiasAt by(bias);
#pragma unroll
    for (int c = 0; c < COUNT; ++c) load_bias<E, B>(sh, by, at[c].row, first_column<E>(at[c], lane), n[c], b[c]);
  }
  const Generator g(rule);
  if (!DENSE && out.gap != (PASS == Pass::backward_relu ? x.gap : from.gap))
    chunk_offsets<E>(sh, first, at, out.gap, lane, offset);
  uint32_t w[kDropSteps<E>][H][V / 2] = {};
  if (rule.threshold)
#pragma unroll
    for (int s = 0; s < kDropSteps<E>; ++s) chunk_words<E>(g, at[s * H], at[s * H + H - 1], lane, w[s]);
  constexpr bool kShift = B == Bias::ragged && PASS != Pass::backward;
  if constexpr (kShift && H == 1) shift_biases<E, COUNT>(n, b);
#pragma unroll
  for (int s = 0; s < kDropSteps<E>; ++s) {
#pragma unroll
    for (int h = 0; h < H; ++h) {
      const int c = s * H + h;
      float v[V];
      if constexpr (kShift && H == 2) shift_biases<E, 1>(n + c, b + c);
      if constexpr (PASS == Pass::forward)
        forward_chunk<E>(rule, in[c], b[c], w[s][h], v);
      else
        backward_chunk<E, PASS == Pass::backward_relu>(rule, in[c], gate[c], b[c], w[s][h], v);
      if (n[c] > 0) store_chunk<E>(out.p + offset[c], n[c], v, HOW == Read::once);
    }
  }
}
template <Elem E, Pass PASS, Bias B>
__global__ __launch_bounds__(kDropThreads) void dropout_kernel(DropoutShape sh, DropoutRule rule, Images<E> x,
                                                               const float* __restrict__ bias, Images<E> dy,
                                                               Images<E> out, bool dense, bool once) {
  constexpr int COUNT = kTurnChunks<E>;
  constexpr uint64_t kTurn = 64 * kDropSteps<E>, kWaves = kDropThreads / 64;  // items to a wave's turn
  const int lane = threadIdx.x & 63;
  const uint64_t wave = (uint64_t)blockIdx.x * kWaves + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  for (uint64_t first = wave * kTurn; first < sh.items; first += gridDim.x * (kTurn * kWaves)) {
    const uint32_t left = (uint32_t)min(sh.items - first, kTurn);
    Place at[COUNT];
    if constexpr (B == Bias::planes || B == Bias::columns) {  // the other two are for rows that end inside an item
      if (dense) {
        if (once)
          dropout_turn<E, PASS, B, Read::once, true>(sh, rule, x, bias, dy, out, first, left, at, lane);
        else
          dropout_turn<E, PASS, B, Read::whole, true>(sh, rule, x, bias, dy, out, first, left, at, lane);
        continue;
      }
    }
    turn_places<E>(sh, first, lane, at);
    bool whole = sh.items - first - left >= 8;  // 8 elements at least lie behind
    if (!whole) {
      int n[COUNT];
#pragma unroll
      for (int c = 0; c < COUNT; ++c) n[c] = at[c].ahead < left ? 1 : 0;
      whole = PASS == Pass::backward || readable(sh, x, first, at, n, lane);
      whole = whole && (PASS == Pass::forward || readable(sh, dy, first, at, n, lane));
    }
    choose_read(whole, once, [&](auto how) {
      dropout_turn<E, PASS, B, decltype(how)::value, false>(sh, rule, x, bias, dy, out, first, left, at, lane);
    });
  }
}

// Backward of maps with the bias gradient: a wave takes `planes` whole planes of together at most 512 items, or 512
// items of one larger plane (`segments` of them), lanes over the items whatever the planes' size; the items' sums
// meet in LDS, and 64 / planes lanes add up each plane's.  partial[segment * N + n][k].
struct MapUnits {
  uint64_t units;
  Divisor32 segments;
  uint32_t rows;          // planes in all
  uint32_t images;
  int planes, lane_shift; // planes per unit; lanes per plane in the final sum, as a shift
};
template <Elem E, bool RELU>
__global__ __launch_bounds__(kDropThreads) void dropout_maps_grad_kernel(
    DropoutShape sh, MapUnits mu, DropoutRule rule, Images<E> x, const float* __restrict__ bias, Images<E> dy,
    Images<E> dx, float* __restrict__ partial, bool once) {
  constexpr int H = kHalves<E>, V = kChunk<E>;
  constexpr uint64_t kWaves = kDropThreads / 64;
  __shared__ float sums[kDropThreads / 64][kDropUnit];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  for (uint64_t unit = blockIdx.x * kWaves + wave; unit < mu.units; unit += gridDim.x * kWaves) {
    const uint32_t bundle = mu.segments.d == 1 ? (uint32_t)unit : (uint32_t)(unit / mu.segments.d);
    const uint32_t segment = (uint32_t)(unit - (uint64_t)bundle * mu.segments.d);
    const uint32_t row0 = bundle * mu.planes, group0 = segment * kDropUnit;
    const uint32_t planes = min((uint32_t)mu.planes, mu.rows - row0);
    const uint32_t width = min((uint32_t)kDropUnit, sh.groups32.d - group0), items = planes * width;
    const uint64_t first = (uint64_t)row0 * sh.groups32.d + group0;
    Place p = place_at(sh, first, lane_item<E>(lane));
    for (uint32_t step = 0; step < items; step += 64) {
      Place at[H];
      int n[H];
      float sum[H];
#pragma unroll
      for (int h = 0; h < H; ++h) {
        at[h] = p;
        p = next_place<64 / H>(sh, p);
        n[h] = at[h].ahead < items ? chunk_size<E>(sh, first_column<E>(at[h], lane)) : 0;
      }
      auto turn = [&](auto how) {
        constexpr Read HOW = decltype(how)::value;
        Words in[H], gate[H];
        float b[H][V];
        int64_t offset[H];
        chunk_offsets<E>(sh, first, at, dy.gap, lane, offset);
        load_chunks<E, HOW>(dy, offset, n, in);
        if constexpr (RELU) {
          if (x.gap != dy.gap) chunk_offsets<E>(sh, first, at, x.gap, lane, offset);
          load_chunks<E, HOW>(x, offset, n, gate);
          const BiasAt by(bias);
#pragma unroll
          for (int h = 0; h < H; ++h) load_bias<E, Bias::planes>(sh, by, at[h].row, 0, n[h], b[h]);
        }
        const Generator g(rule);
        uint32_t w[H][V / 2] = {};
        if (rule.threshold) chunk_words<E>(g, at[0], at[H - 1], lane, w);
        if (dx.gap != (RELU ? x.gap : dy.gap)) chunk_offsets<E>(sh, first, at, dx.gap, lane, offset);
#pragma unroll
        for (int h = 0; h < H; ++h) {
          float dz[V];
          backward_chunk<E, RELU>(rule, in[h], gate[h], b[h], w[h], dz);
          if (dx.p && n[h] > 0) store_chunk<E>(dx.p + offset[h], n[h], dz, HOW == Read::once);
          sum[h] = 0.0f;
#pragma unroll
          for (int i = 0; i < V; ++i) sum[h] += i < n[h] ? dz[i] : 0.0f;
        }
      };
      bool whole = sh.items - first - items >= 8;  // 8 elements at least lie behind
      if (!whole) whole = readable(sh, dy, first, at, n, lane) && (!RELU || readable(sh, x, first, at, n, lane));
      choose_read(whole, once, turn);
      if constexpr (H == 1) {
        if (step + lane < items) sums[wave][step + lane] = sum[0];
      } else {  // the even lane ends with the first item's sum, the odd one with the second's
        const bool odd = lane & 1;
        const float total = (odd ? sum[1] : sum[0]) + lane_xor<1>(odd ? sum[0] : sum[1], lane);
        const uint32_t it = step + (odd ? 32 : 0) + lane / 2;
        if (it < items) sums[wave][it] = total;
      }
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    const uint32_t plane = lane >> mu.lane_shift, lanes = 1u << mu.lane_shift;
    float sum = 0.0f;
    if (plane < planes)
      for (uint32_t i = lane & (lanes - 1); i < width; i += lanes) sum += sums[wave][plane * width + i];
    for (uint32_t off = lanes / 2; off; off /= 2) sum += __shfl_xor(sum, off);
    if (plane < planes && (lane & (lanes - 1)) == 0) {
      const uint32_t n = sh.channels.quotient(row0 + plane);
      partial[((uint64_t)segment * mu.images + n) * sh.channels.d + (row0 + plane - n * sh.channels.d)] = sum;
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  }
}

// Backward of feature rows with the bias gradient: a lane keeps a chunk of columns and walks down rows, four at a time
// (fp32: the pair of lanes makes the words of one of two rows each); the threads of a workgroup that share columns meet
// in LDS. partial[blockIdx.y][column]. The workgroups' rows alternate, so that those in flight read one stretch of memory:
// 16384 rows of 4096 bf16 (402 MB) 79 us, 84 with a run of rows to each; 32768 of fp32 (1.6 GB) 294 us, 314 with runs,
// two rows at a time.
constexpr int kBiasRows = 4;
template <Elem E, bool RELU, Bias B>
__global__ __launch_bounds__(kDropThreads) void dropout_features_grad_kernel(
    DropoutShape sh, uint32_t rows, int across_shift, DropoutRule rule, Images<E> x, const float* __restrict__ bias,
    Images<E> dy, Images<E> dx, float* __restrict__ partial, bool once) {
  constexpr int H = kHalves<E>, V = kChunk<E>, kRows = kBiasRows;  // rows in flight
  __shared__ float sums[kDropThreads][V];
  const uint32_t across = 1u << across_shift, down = kDropThreads >> across_shift, lane = threadIdx.x & 63;
  const uint32_t col = (blockIdx.x * across + (threadIdx.x & (across - 1))) * V;
  const int size = chunk_size<E>(sh, col);
  float total[V] = {}, b[V];
  if constexpr (RELU) load_bias<E, B>(sh, BiasAt(bias), 0, col, size, b);
  for (uint32_t row0 = blockIdx.y * kRows * down; row0 < rows; row0 += gridDim.y * kRows * down) {
    Place at[kRows];
    int n[kRows];
    int64_t from[kRows], of[kRows];
    bool behind = false;  // a chunk that reaches past a tensor's last element
#pragma unroll
    for (int r = 0; r < kRows; ++r) {
      at[r] = {row0 + r * down + (threadIdx.x >> across_shift), col / 8, 0};
      n[r] = at[r].row < rows ? size : 0;
      from[r] = (int64_t)at[r].row * (sh.cols + x.gap) + col;
      of[r] = (int64_t)at[r].row * (sh.cols + dy.gap) + col;
      behind |= n[r] > 0 && (of[r] + V > dy.span || (RELU && from[r] + V > x.span));
    }
    const bool whole = dy.span >= V && (!RELU || x.span >= V) && __ballot(behind) == 0;
    auto turn = [&](auto how) {
      constexpr Read HOW = decltype(how)::value;
      Words in[kRows], gate[kRows];
      load_chunks<E, HOW>(dy, of, n, in);
      if constexpr (RELU) load_chunks<E, HOW>(x, from, n, gate);
      const Generator g(rule);
      uint32_t w[kRows][V / 2] = {};
      if (rule.threshold) {
#pragma unroll
        for (int r = 0; r < kRows; r += H) {
          uint32_t words[H][V / 2];
          chunk_words<E>(g, at[r], at[r + H - 1], lane, words);
#pragma unroll
          for (int i = 0; i < H * V / 2; ++i) w[r + i / (V / 2)][i % (V / 2)] = words[i / (V / 2)][i % (V / 2)];
        }
      }
#pragma unroll
      for (int r = 0; r < kRows; ++r) {
        float dz[V];
        backward_chunk<E, RELU>(rule, in[r], gate[r], b, w[r], dz);
        if (dx.p && n[r] > 0) store_chunk<E>(dx.p + (int64_t)at[r].row * (sh.cols + dx.gap) + col, n[r], dz, HOW == Read::once);
#pragma unroll
        for (int i = 0; i < V; ++i) total[i] += n[r] > 0 ? dz[i] : 0.0f;
      }
    };
    choose_read(whole, once, turn);
  }
#pragma unroll
  for (int i = 0; i < V; ++i) sums[threadIdx.x][i] = total[i];
  __syncthreads();
  for (uint32_t c = threadIdx.x; c < across * V; c += kDropThreads) {
    float sum = 0.0f;
    for (uint32_t d = 0; d < down; ++d) sum += sums[d * across + c / V][c % V];
    const uint64_t at = (uint64_t)blockIdx.x * across * V + c;
    if (at < sh.cols) partial[(uint64_t)blockIdx.y * sh.cols + at] = sum;
  }
}

// dbias[k] = sum of `parts` rows of partial sums, always in the same order: 64 threads take every 64th row, their sums
// are added in a tree.
constexpr int kBiasCols = 16, kBiasDown = 64;
__global__ __launch_bounds__(kBiasCols * kBiasDown) void bias_grad_kernel(const float* __restrict__ partial, uint32_t parts, uint32_t K,
                                                                          float* __restrict__ dbias) {
  __shared__ float sums[kBiasDown][kBiasCols];
  const uint32_t c = threadIdx.x % kBiasCols, d = threadIdx.x / kBiasCols;
  for (uint64_t first = (uint64_t)blockIdx.x * kBiasCols; first < K; first += (uint64_t)gridDim.x * kBiasCols) {
    const uint64_t k = first + c;
    float sum = 0.0f;
    if (k < K)
      for (uint64_t i = d; i < parts; i += kBiasDown) sum += partial[i * K + k];
    sums[d][c] = sum;
    for (uint32_t half = kBiasDown / 2; half; half /= 2) {
      __syncthreads();
      if (d < half) sums[d][c] += sums[d + half][c];
    }
    if (d == 0 && k < K) dbias[k] = sums[0][c];
    __syncthreads();
  }
}

}  // namespace swconv
