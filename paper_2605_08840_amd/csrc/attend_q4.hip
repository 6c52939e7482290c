// Attention over pages of 4 bits.
#include "attend.hpp"

namespace restkv {

int run_attend_q4(const AttendArgs& a, int R, hipStream_t st) {
  auto go = [&](auto d, auto np, auto t) {
    constexpr int D = decltype(d)::value, NP = decltype(np)::value;
    using T = decltype(t);
    if constexpr (planes_of<T> == 1) {      // (parts of float32 queries, a copy each, are more than the registers hold)
      // copies of few rows: 1 / 2 / 4 of them, us, 16 sequences of 2k keys of 8 KV heads of 128: 1 row 21.7 / 20.1 / 19.9,
      // 4 rows 21.9 / 20.9 / 20.8, 8 rows 22.4 / 21.6
      const int64_t rows = (int64_t)a.pg.G * a.pg.max_new;
      if (rows <= 4) return run_attend<FMT_Q4, T, D, NP, 1, 4>(a, st);
      if (rows <= 8) return run_attend<FMT_Q4, T, D, NP, 1, 2>(a, st);
    }
    if constexpr (planes_of<T> == 1 || D == 64)
      if (R == 2) return run_attend<FMT_Q4, T, D, NP, 2>(a, st);
    return run_attend<FMT_Q4, T, D, NP, 1>(a, st);
  };
  auto by_d = [&](auto np, auto t) {
    return a.pg.d == 128 ? go(std::integral_constant<int, 128>{}, np, t) : go(std::integral_constant<int, 64>{}, np, t);
  };
  if (a.pg.dtype == RESTKV_F32) return by_d(std::integral_constant<int, 3>{}, 0.f);
  return a.pg.out_dtype == RESTKV_F32 ? by_d(std::integral_constant<int, 3>{}, bf16_t{}) : by_d(std::integral_constant<int, 2>{}, bf16_t{});
}

}  // namespace restkv
