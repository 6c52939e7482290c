// Attention over bfloat16 pages for many rows.
#include "attend_rows.hpp"

namespace restkv {

namespace {

template <int D, int NP, int R, int NW>
int run_rows(const AttendArgs& a, hipStream_t st) {
  constexpr size_t lds = 2 * 2 * 64 * (size_t)D * 2;
  hipLaunchKernelGGL((k_attend_rows<D, NP, R, NW, NO_BEAMS>), unit_grid(a), dim3(64 * NW), lds, st, a);
  return hip_status();
}

}  // namespace

int run_attend_rows(const AttendArgs& a, int R, int waves, hipStream_t st) {
  auto go = [&](auto d, auto np) {
    constexpr int D = decltype(d)::value, NP = decltype(np)::value;
    return R == 1 ? run_rows<D, NP, 1, 4>(a, st) : waves == 4 ? run_rows<D, NP, 2, 4>(a, st) : run_rows<D, NP, 2, 8>(a, st);
  };
  auto by_d = [&](auto np) {
    return a.pg.d == 128 ? go(std::integral_constant<int, 128>{}, np) : go(std::integral_constant<int, 64>{}, np);
  };
  return a.pg.out_dtype == RESTKV_F32 ? by_d(std::integral_constant<int, 3>{}) : by_d(std::integral_constant<int, 2>{});
}

}  // namespace restkv
