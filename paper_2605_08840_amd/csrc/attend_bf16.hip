// Attention over bfloat16 pages, up to 16 rows.
#include "attend.hpp"

namespace restkv {

int run_attend_bf16(const AttendArgs& a, hipStream_t st) {
  auto go = [&](auto d, auto np) {
    constexpr int D = decltype(d)::value, NP = decltype(np)::value;
    return run_attend<FMT_BF16, bf16_t, D, NP, 1>(a, st);
  };
  auto by_d = [&](auto np) {
    return a.pg.d == 128 ? go(std::integral_constant<int, 128>{}, np) : go(std::integral_constant<int, 64>{}, np);
  };
  return a.pg.out_dtype == RESTKV_F32 ? by_d(std::integral_constant<int, 3>{}) : by_d(std::integral_constant<int, 2>{});
}

}  // namespace restkv
