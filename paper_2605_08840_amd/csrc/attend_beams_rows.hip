// Attention of beams over bfloat16 pages, where a group has many rows: the shared positions by tiles in LDS for 64 or 128 rows a workgroup,
// what each beam has behind them as for few rows.
#include "attend_rows.hpp"

namespace restkv {

int run_attend_beams_rows(const AttendArgs& a, hipStream_t st) {
  auto go = [&](auto d, auto np) {
    constexpr int D = decltype(d)::value, NP = decltype(np)::value;
    constexpr size_t tiles = 2 * 2 * 64 * (size_t)D * 2, join = (8 * 16 + (size_t)4 * 16 * (D + 4)) * 4;
    const size_t lds = tiles > join ? tiles : join;
    auto launch = [&](auto kern) { hipLaunchKernelGGL(kern, unit_grid(a), dim3(256), lds, st, a); };
    if (a.spread) launch(k_attend_rows<D, NP, 1, 4, BEAMS_PARTS>);       // (64 rows)
    else if (a.front_rows == 128) launch(k_attend_rows<D, NP, 2, 4, BEAMS_LIST>);
    else launch(k_attend_rows<D, NP, 1, 4, BEAMS_LIST>);
    return hip_status();
  };
  auto by_d = [&](auto np) {
    return a.pg.d == 128 ? go(std::integral_constant<int, 128>{}, np) : go(std::integral_constant<int, 64>{}, np);
  };
  return a.pg.out_dtype == RESTKV_F32 ? by_d(std::integral_constant<int, 3>{}) : by_d(std::integral_constant<int, 2>{});
}

}  // namespace restkv
