// Exchanges between the lanes of a wave.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>
#include <type_traits>

namespace swconv {

// The value of lane ^ OFF by moves within the vector unit: a trip through LDS takes ten times as long.
template <int OFF>
__device__ __forceinline__ uint32_t lane_xor(uint32_t v, int lane) {
  auto dpp = [](uint32_t a, auto control) {
    return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)a, decltype(control)::value, 0xf, 0xf, true);
  };
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

}  // namespace swconv
