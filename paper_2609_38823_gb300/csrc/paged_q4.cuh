// The layout of a key-value pool in 4 bits (the contract is in decomoe.h).
#pragma once

#include <cfloat>
#include <type_traits>

#include "decomoe_internal.cuh"

namespace decomoe {

// Eight rows of a KV head: codes of their keys, (step, low) pairs of their keys, and the
// same of their values. G groups a row. A row's codes are ordered so that a lane's operands
// of the attention's products lie together: eight features 32 i + 8 c .. + 7 of keys in
// the 32-bit word c (D / 32) + i, four features 32 i + 4 r .. + 3 of values in the 16-bit
// word r (D / 32) + i.
template <int D, int G>
struct Q4Tile {
  static constexpr int ROWS = 8;
  static constexpr int CODES = D / 2;                   // bytes of a row's codes
  static constexpr int PARAMS = 4 * G;                  // and of its parameters
  static constexpr int K = 0, KP = ROWS * CODES;        // places in a tile
  static constexpr int V = KP + ROWS * PARAMS, VP = V + ROWS * CODES;
  static constexpr int BYTES = VP + ROWS * PARAMS;
  static_assert(BYTES % 16 == 0 && KP % 16 == 0 && V % 16 == 0 && VP % 16 == 0, "bulk copies");
};

inline int64_t q4_tile_bytes(int D, int group) { return 16 * (D / 2 + 4 * static_cast<int64_t>(D / group)); }
inline bool q4_shape_ok(int D, int group) {
  return (D == 64 && (group == 32 || group == 64)) || (D == 128 && (group == 32 || group == 64 || group == 128));
}

// f(D, G) for a shape that q4_shape_ok.
template <class F>
inline int q4_dispatch(int D, int group, F f) {
  if (D == 128) {
    if (group == 32) return f(std::integral_constant<int, 128>(), std::integral_constant<int, 4>());
    if (group == 64) return f(std::integral_constant<int, 128>(), std::integral_constant<int, 2>());
    return f(std::integral_constant<int, 128>(), std::integral_constant<int, 1>());
  }
  if (group == 32) return f(std::integral_constant<int, 64>(), std::integral_constant<int, 2>());
  return f(std::integral_constant<int, 64>(), std::integral_constant<int, 1>());
}

}  // namespace decomoe
