// Attention of beams over pages of 4 bits.
#include "attend.hpp"

namespace restkv {

int run_attend_beams_q4(const AttendArgs& a, hipStream_t st) {
  auto by_d = [&](auto np, auto t) {
    constexpr int NP = decltype(np)::value;
    return a.pg.d == 128 ? run_attend_beams<FMT_Q4, decltype(t), 128, NP, 1>(a, st) : run_attend_beams<FMT_Q4, decltype(t), 64, NP, 1>(a, st);
  };
  if (a.pg.dtype == RESTKV_F32) return by_d(std::integral_constant<int, 3>{}, 0.f);
  return a.pg.out_dtype == RESTKV_F32 ? by_d(std::integral_constant<int, 3>{}, bf16_t{}) : by_d(std::integral_constant<int, 2>{}, bf16_t{});
}

}  // namespace restkv
