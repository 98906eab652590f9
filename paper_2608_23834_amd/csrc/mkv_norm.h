// Sums over the lanes that share a row of a head, for the norms of query and key heads.
#pragma once

#include <type_traits>

#include "mkv_attn.h"
#include "mkv_rope.h"

namespace mkv {

// sum over the LT lanes of a row, in each of them
template <int LT>
__device__ __forceinline__ double row_sum(double x, int lane) {
  auto add = [&](auto mc) {
    constexpr int M = decltype(mc)::value;
    const uint64_t b = __builtin_bit_cast(uint64_t, x);
    const uint32_t lo = __float_as_uint(lane_xor<M>(__uint_as_float((uint32_t)b), lane));
    const uint32_t hi = __float_as_uint(lane_xor<M>(__uint_as_float((uint32_t)(b >> 32)), lane));
    x += __builtin_bit_cast(double, (uint64_t)hi << 32 | lo);
  };
  add(std::integral_constant<int, 1>{});
  add(std::integral_constant<int, 2>{});
  add(std::integral_constant<int, 4>{});
  add(std::integral_constant<int, 8>{});
  if constexpr (LT > 16) add(std::integral_constant<int, 16>{});
  if constexpr (LT > 32) add(std::integral_constant<int, 32>{});
  return x;
}

}  // namespace mkv
