// Attention of beams over float32 pages.
#include "attend.hpp"

namespace restkv {

int run_attend_beams_f32(const AttendArgs& a, int R, hipStream_t st) {
  auto go = [&](auto d) {
    constexpr int D = decltype(d)::value;
    return R == 1 ? run_attend_beams<FMT_F32, float, D, 1, 1>(a, st) : run_attend_beams<FMT_F32, float, D, 1, 2>(a, st);
  };
  return a.pg.d == 128 ? go(std::integral_constant<int, 128>{}) : go(std::integral_constant<int, 64>{});
}

}  // namespace restkv
