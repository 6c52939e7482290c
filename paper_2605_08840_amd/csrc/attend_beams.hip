// Attention over pages that the beams of a group have in common in front.
#include "beams.hpp"

namespace restkv {

size_t attend_beams_ws_bytes(const Pages& pg, int) { return attend_ws_bytes(pg); }

int launch_attend_beams(const Pages& pg, int, const int32_t*, const void* q, const void* k_pages, const void* v_pages,
                        const void* k_scale, const void* v_scale, void* out, float* lse, char* ws, hipStream_t st) {
  return launch_attend(pg, q, k_pages, v_pages, k_scale, v_scale, out, lse, ws, st);
}

}  // namespace restkv
