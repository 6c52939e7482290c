// Attention over bfloat16 pages for many rows.
#include "attend_rows.hpp"

namespace restkv {

namespace {

template <int D, int NP, int R, int NW>
__global__ __attribute__((amdgpu_flat_work_group_size(64 * NW, 64 * NW), amdgpu_waves_per_eu(2)))
void k_attend_rows(AttendArgs a) {
  extern __shared__ __align__(16) char lds[];        // [2][keys | values][TILE]
  const int unit = unit_of_block();
  if (unit >= a.units) return;
  Chunk ch;
  if (!find_chunk<NW>(a, unit / a.Hy, (int*)lds, ch)) return;
  rows_chunk<D, NP, R, NW, false>(a, ch, unit % a.Hy, blockIdx.x >> 3, 0, lds);
}

template <int D, int NP, int R, int NW>
int run_rows(const AttendArgs& a, hipStream_t st) {
  constexpr size_t lds = 2 * 2 * 64 * (size_t)D * 2;
  hipLaunchKernelGGL((k_attend_rows<D, NP, R, NW>), unit_grid(a), dim3(64 * NW), lds, st, a);
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
