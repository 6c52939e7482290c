// Attention of beams over float32 pages.
#include "attend.hpp"

namespace restkv {

int run_attend_beams_f32(const AttendArgs& a, hipStream_t st) {
  return a.pg.d == 128 ? run_attend_beams<FMT_F32, float, 128, 1, 1>(a, st) : run_attend_beams<FMT_F32, float, 64, 1, 1>(a, st);
}

}  // namespace restkv
