// Rows of elements in fp32, fp16 or bf16: 16 bytes to a lane, from and to addresses that are aligned to the element only
// (rows of odd length, channel groups).  The compiler makes 16-byte accesses of them: global memory takes any alignment.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace swconv {

enum class Elem { f32, f16, bf16 };

template <Elem E>
struct ElemTraits;
template <>
struct ElemTraits<Elem::f32> {
  using type = float;
};
template <>
struct ElemTraits<Elem::f16> {
  using type = _Float16;
};
template <>
struct ElemTraits<Elem::bf16> {
  using type = __bf16;
};
template <Elem E>
using elem_t = typename ElemTraits<E>::type;

// V elements of a row as they lie in memory
template <Elem E, int V>
struct Pack {
  elem_t<E> v[V];
};

template <Elem E, int V>
__device__ __forceinline__ Pack<E, V> load_pack(const elem_t<E>* p) {
  Pack<E, V> a;
  __builtin_memcpy(&a, p, sizeof(a));
  return a;
}

// 16 bytes of a row as words, so that an element is one operation away from its float.
typedef uint32_t Words __attribute__((ext_vector_type(4)));
typedef uint32_t LooseWords __attribute__((ext_vector_type(4), aligned(2)));
template <Elem E>
constexpr int kWordsElems = 16 / sizeof(elem_t<E>);

template <Elem E>
__device__ __forceinline__ float word_elem(const Words& w, int i) {
  if constexpr (E == Elem::f32) return __uint_as_float(w[i]);
  if constexpr (E == Elem::bf16) return __uint_as_float(i % 2 ? w[i / 2] & 0xffff0000u : w[i / 2] << 16);
  if constexpr (E == Elem::f16) return (float)__builtin_bit_cast(_Float16, (uint16_t)(w[i / 2] >> (i % 2 * 16)));
}
// `once`: nothing reads these bytes again soon (more of them than the 256 MB cache keeps).  With the hint a read of 1 GB runs
// at 6.9 TB/s, without at 6.3, a copy at 6.4 and 6.1; but a gradient that reads its scores again takes 48 us after a forward pass
// with the hint and 36 after one without (78 MB).
template <Elem E>
__device__ __forceinline__ Words load_words(const elem_t<E>* p, bool once) {
  const auto* q = reinterpret_cast<const LooseWords*>(p);
  return once ? (Words)__builtin_nontemporal_load(q) : (Words)*q;
}
template <Elem E>
__device__ __forceinline__ void store_words(elem_t<E>* p, const Words& w, bool once) {
  auto* q = reinterpret_cast<LooseWords*>(p);
  if (once)
    __builtin_nontemporal_store((LooseWords)w, q);
  else
    *q = w;
}
template <Elem E>
constexpr uint32_t kMinusInf = E == Elem::f32 ? 0xff800000u : E == Elem::bf16 ? 0xff80u : 0xfc00u;
// The first n elements of a row that is shorter than 16 bytes, -inf behind them.
template <Elem E>
__device__ __forceinline__ Words load_words_part(const elem_t<E>* p, int n) {
  Words w;
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    if constexpr (E == Elem::f32) {
      w[k] = k < n ? __float_as_uint(p[k]) : kMinusInf<E>;
    } else {
      const uint32_t lo = 2 * k < n ? __builtin_bit_cast(uint16_t, p[2 * k]) : kMinusInf<E>;
      const uint32_t hi = 2 * k + 1 < n ? __builtin_bit_cast(uint16_t, p[2 * k + 1]) : kMinusInf<E>;
      w[k] = hi << 16 | lo;
    }
  }
  return w;
}
// -inf in place of the first n elements.
template <Elem E>
__device__ __forceinline__ Words without_first(Words w, int n) {
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    if constexpr (E == Elem::f32) {
      w[k] = k < n ? kMinusInf<E> : w[k];
    } else {
      const uint32_t lo = 2 * k < n ? kMinusInf<E> : w[k] & 0xffffu;
      w[k] = 2 * k + 1 < n ? kMinusInf<E> << 16 | lo : (w[k] & 0xffff0000u) | lo;
    }
  }
  return w;
}

template <Elem E, int V>
__device__ __forceinline__ void store_part(elem_t<E>* p, int n, const Pack<E, V>& a) {
#pragma unroll
  for (int i = 0; i < V; ++i)
    if (i < n) p[i] = a.v[i];
}

// n / d for an n of 32 or 64 bits and a d that stays: the rounded-down reciprocal gives the quotient or one less.
struct Divisor {
  uint64_t d, reciprocal;
  explicit Divisor(uint64_t divisor)
      : d(divisor), reciprocal(divisor == 1 ? ~0ull : (uint64_t)(((unsigned __int128)1 << 64) / divisor)) {}
  __device__ __forceinline__ uint64_t quotient(uint64_t n) const {
    const uint64_t q = __umul64hi(n, reciprocal);
    return q + (n - q * d >= d);
  }
};
struct Divisor32 {
  uint32_t d, reciprocal;
  explicit Divisor32(uint32_t divisor)
      : d(divisor), reciprocal(divisor == 1 ? ~0u : (uint32_t)((1ull << 32) / divisor)) {}
  __device__ __forceinline__ uint32_t quotient(uint32_t n) const {
    const uint32_t q = __umulhi(n, reciprocal);
    return q + (n - q * d >= d);
  }
};

}  // namespace swconv
