// Rows of elements in fp32, fp16 or bf16: several per lane as floats, from and to addresses that are aligned to
// the element only (rows of odd length, channel groups).  The compiler makes 16-byte accesses of them: global memory
// takes any alignment.
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

// 16 bytes of a stream that is read once: without the hint a read of 1 GB runs at 6.3 TB/s, with it at 7.0, a copy at 6.2
// and, hinted on both sides, 6.5.
typedef uint32_t Stream16 __attribute__((ext_vector_type(4), aligned(2)));
template <Elem E, int V>
__device__ __forceinline__ Pack<E, V> stream_pack(const elem_t<E>* p) {
  static_assert(sizeof(Pack<E, V>) == 16, "one access");
  return __builtin_bit_cast(Pack<E, V>, (Stream16)__builtin_nontemporal_load(reinterpret_cast<const Stream16*>(p)));
}

// The first n of V elements (n < V), `fill` behind them.
template <Elem E, int V>
__device__ __forceinline__ Pack<E, V> load_part(const elem_t<E>* p, int n, float fill) {
  Pack<E, V> a;
#pragma unroll
  for (int i = 0; i < V; ++i) a.v[i] = i < n ? p[i] : (elem_t<E>)fill;
  return a;
}

template <Elem E, int V>
__device__ __forceinline__ void store_pack(elem_t<E>* p, const Pack<E, V>& a) {
  __builtin_memcpy(p, &a, sizeof(a));
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
  explicit Divisor(uint64_t divisor) : d(divisor), reciprocal(divisor == 1 ? ~0ull : (uint64_t)(((unsigned __int128)1 << 64) / divisor)) {}
  __device__ __forceinline__ uint64_t quotient(uint64_t n) const {
    const uint64_t q = __umul64hi(n, reciprocal);
    return q + (n - q * d >= d);
  }
};
struct Divisor32 {
  uint32_t d, reciprocal;
  explicit Divisor32(uint32_t divisor) : d(divisor), reciprocal(divisor == 1 ? ~0u : (uint32_t)((1ull << 32) / divisor)) {}
  __device__ __forceinline__ uint32_t quotient(uint32_t n) const {
    const uint32_t q = __umulhi(n, reciprocal);
    return q + (n - q * d >= d);
  }
};

}  // namespace swconv
