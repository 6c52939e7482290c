// Attention of beams over pages of 4 bits.
#include "attend.hpp"

namespace restkv {

int run_attend_beams_q4(const AttendArgs& a, int R, hipStream_t st) {
  auto go = [&](auto d, auto np, auto t) {
    constexpr int D = decltype(d)::value, NP = decltype(np)::value;
    using T = decltype(t);
    if constexpr (planes_of<T> == 1 || D == 64)
      if (R == 2) return run_attend_beams<FMT_Q4, T, D, NP, 2>(a, st);
    return run_attend_beams<FMT_Q4, T, D, NP, 1>(a, st);
  };
  auto by_d = [&](auto np, auto t) {
    return a.pg.d == 128 ? go(std::integral_constant<int, 128>{}, np, t) : go(std::integral_constant<int, 64>{}, np, t);
  };
  if (a.pg.dtype == RESTKV_F32) return by_d(std::integral_constant<int, 3>{}, 0.f);
  return a.pg.out_dtype == RESTKV_F32 ? by_d(std::integral_constant<int, 3>{}, bf16_t{}) : by_d(std::integral_constant<int, 2>{}, bf16_t{});
}

}  // namespace restkv
