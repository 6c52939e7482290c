// Attention over float32 pages: products on the float32 matrix instruction.
#include "attend.hpp"

namespace restkv {

int run_attend_f32(const AttendArgs& a, int R, hipStream_t st) {
  auto go = [&](auto d) {
    constexpr int D = decltype(d)::value;
    return R == 1 ? run_attend<FMT_F32, float, D, 1, 1>(a, st) : run_attend<FMT_F32, float, D, 1, 2>(a, st);
  };
  return a.pg.d == 128 ? go(std::integral_constant<int, 128>{}) : go(std::integral_constant<int, 64>{});
}

}  // namespace restkv
