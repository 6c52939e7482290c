// Attention of beams over bfloat16 pages, where a group has many rows: the shared positions by tiles in LDS for 64 or 128 rows a
// workgroup, what each beam has behind them as for few rows.
#include "attend_rows.hpp"

namespace restkv {

namespace {

template <int D, int NP, int R>
__global__ __attribute__((amdgpu_flat_work_group_size(256, 256), amdgpu_waves_per_eu(2)))
void k_beams_rows(AttendArgs a) {
  extern __shared__ __align__(16) char lds[];
  const int unit = unit_of_block(), hy = unit % a.Hy;
  if (unit >= a.units) return;
  BeamsWork w;
  if (!beams_work<4>(a, unit, blockIdx.x >> 3, (int*)lds, w)) return;
  while (w.todo) {
    bool front;
    int slot;
    next_part(a, w, front, slot);
    if (front) rows_chunk<D, NP, R, 4, true>(a, w.ch, hy, w.rb, slot, lds);
    else attend_chunk<FMT_BF16, bf16_t, D, NP, 1, 1, true>(a, w.ch, hy, w.rb, false, slot, (float*)lds);
    if (w.todo) __syncthreads();
  }
}

template <int D, int NP, int R>
int run_rows(const AttendArgs& a, hipStream_t st) {
  constexpr size_t tiles = 2 * 2 * 64 * (size_t)D * 2, join = (8 * 16 + (size_t)4 * 16 * (D + 4)) * 4;
  hipLaunchKernelGGL((k_beams_rows<D, NP, R>), unit_grid(a), dim3(256), tiles > join ? tiles : join, st, a);
  return hip_status();
}

}  // namespace

int run_attend_beams_rows(const AttendArgs& a, int R, hipStream_t st) {
  auto go = [&](auto d, auto np) {
    constexpr int D = decltype(d)::value, NP = decltype(np)::value;
    return R == 1 ? run_rows<D, NP, 1>(a, st) : run_rows<D, NP, 2>(a, st);
  };
  auto by_d = [&](auto np) {
    return a.pg.d == 128 ? go(std::integral_constant<int, 128>{}, np) : go(std::integral_constant<int, 64>{}, np);
  };
  return a.pg.out_dtype == RESTKV_F32 ? by_d(std::integral_constant<int, 3>{}) : by_d(std::integral_constant<int, 2>{});
}

}  // namespace restkv
