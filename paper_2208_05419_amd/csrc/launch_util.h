// launch_util.h -- what launchers share: a kernel's template arguments from run-time values.
#pragma once
#include <stdint.h>

#include <type_traits>

#include "kernels_norm.h"

namespace afno {

template <typename F>
auto by_type(int dtype, F f) {
  return dtype == 0 ? f(float()) : f(bf16());
}
template <typename F>
auto by_flag(bool v, F f) {
  return v ? f(std::true_type()) : f(std::false_type());
}
inline bool at16(const void* p) { return ((uintptr_t)p & 15) == 0; }  // null counts as aligned

// the kernels that hold a row in registers, by the channels that they have room for and the waves that
// share a row: all of a row's loads are under way at once, and fewer registers leave more rows to a CU.  From
// 1,025 to 2,048 channels one wave holds a row (295 to 368 registers backward), which serves many rows: of 64,800,
// backward 170 us against 259 with four waves (1,152 bf16), 256 and 267 (2,048 bf16), 407 and 425 (fp32), forward
// 106 and 113, 191 and 175, 386 and 365.  Few rows leave CUs to it half empty: 5,187 x 2,048 backward 50 against 34
// (fp32 53 and 35), 500 x 2,048 18.3 and 17.2, forward about even.
template <typename F>
void by_capacity(int64_t C, F f) {
  const auto one = std::integral_constant<int, 1>();
  const auto four = std::integral_constant<int, 4>();
  if (C <= 512) f(std::integral_constant<int, 512>(), one);
  else if (C <= 1024) f(std::integral_constant<int, 1024>(), one);
  else if (C <= 2048) f(std::integral_constant<int, 2048>(), one);
  else if (C <= 4096) f(std::integral_constant<int, 4096>(), four);
  else f(std::integral_constant<int, kNormRowMax>(), four);
}
inline int64_t norm_row_waves(int64_t C) { return C <= 2048 ? 1 : 4; }

}  // namespace afno
