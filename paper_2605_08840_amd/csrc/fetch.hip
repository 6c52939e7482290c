// Rows of a paged cache as dense keys and values (4-bit rows as the values they stand for).
#include "pages.hpp"

namespace restkv {

namespace {

// Sixteen lanes a row, a lane the d/16 channels of a unit; a workgroup 16 U rows of a head, of keys or of values, a lane with U
// of them in flight.  U = 4: with two, 24 caches of 2k 4-bit positions take 22.4 us in place of 20.3, with eight the same.  Bound by
// memory (270 MB in and out 6.05 TB/s), where it is short by the chain length, page, row, store.
template <typename T, int D, bool Q4, int U, bool PAST>
__global__ __launch_bounds__(256) void k_fetch(Pages pg, const char* k_pages, const char* v_pages, const uint32_t* k_scale,
                                               const uint32_t* v_scale, const int32_t* __restrict__ idx, int first, int n_rows,
                                               T* k_out, T* v_out) {
  constexpr int UN = D / 16, NG = D / 32;
  constexpr int B = Q4 ? UN / 2 : UN * (int)sizeof(T);            // bytes of a unit in its page: 2, 4, 8, 16 or 32
  constexpr int N = B < 4 ? 1 : B / 4;
  const int u = threadIdx.x & 15;
  const int64_t b = wide_block();
  const int blocks = (n_rows + 16 * U - 1) / (16 * U);
  const bool is_v = b & 1;
  const int64_t e = (b >> 1) / blocks;
  const int j0 = (int)((b >> 1) % blocks) * (16 * U) + (threadIdx.x >> 4);
  if (e >= (int64_t)pg.n_seqs * pg.Hkv) return;
  const int s = (int)(e / pg.Hkv), h = (int)(e % pg.Hkv), len = cache_len(pg, s, h);
  const char* src = is_v ? v_pages : k_pages;
  const uint32_t* scales = is_v ? v_scale : k_scale;
  T* dst = (is_v ? v_out : k_out) + e * n_rows * D + u * UN;
  int64_t slot[U];
#pragma unroll
  for (int c = 0; c < U; ++c) {
    const int j = min(j0 + 16 * c, n_rows - 1), t = idx ? idx[e * n_rows + j] : first + j;
    int page = -1;
    if (t >= 0 && t < len) page = page_of(pg, s, h, t);
    slot[c] = page >= 0 ? (int64_t)row_of(pg, page, h, t) : -1;
  }
  uint32_t w[U][N], sc[U][Q4 ? NG : 1];
#pragma unroll
  for (int c = 0; c < U; ++c) {
    const char* p = src + max(slot[c], (int64_t)0) * (B * 16) + u * B;
    if constexpr (B == 2) w[c][0] = *(const uint16_t*)p;
    else if constexpr (B == 4) w[c][0] = *(const uint32_t*)p;
    else if constexpr (B == 8) *(Words<2>*)w[c] = get<PAST, Words<2>>(p);
    else
#pragma unroll
      for (int i = 0; i < N; i += 4) *(Words<4>*)&w[c][i] = get<PAST && B == 16, Words<4>>(p + 4 * i);
    if constexpr (Q4) {
      const uint32_t* q = scales + max(slot[c], (int64_t)0) * NG;
      if constexpr (NG == 4) *(uint4*)sc[c] = *(const uint4*)q;
      else *(uint2*)sc[c] = *(const uint2*)q;
    }
  }
#pragma unroll
  for (int c = 0; c < U; ++c) {
    const int j = j0 + 16 * c;
    if (j >= n_rows) break;
    constexpr int M = UN * (int)sizeof(T) / 4;
    uint32_t y[M];
    if constexpr (Q4) {
      float x[UN];
#pragma unroll
      for (int i = 0; i < UN; ++i)
        x[i] = __uint_as_float(sc[c][i / 2] & 0xFFFF0000u) + __uint_as_float(sc[c][i / 2] << 16) * (float)(w[c][0] >> (4 * i) & 15u);
#pragma unroll
      for (int i = 0; i < M; ++i) {
        if constexpr (sizeof(T) == 4) y[i] = __float_as_uint(x[i]);
        else y[i] = __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{x[2 * i], x[2 * i + 1]}, bf16x2));
      }
    } else {
#pragma unroll
      for (int i = 0; i < M; ++i) y[i] = w[c][i];
    }
#pragma unroll
    for (int i = 0; i < M; ++i) y[i] = slot[c] < 0 ? 0u : y[i];
    T* o = dst + (int64_t)j * D;
    if constexpr (M == 2) put<true>(o, Words<2>{y[0], y[1]});
    else
#pragma unroll
      for (int i = 0; i < M; i += 4) put<M == 4>((uint32_t*)o + i, Words<4>{y[i], y[i + 1], y[i + 2], y[i + 3]});
  }
}

}  // namespace

int launch_fetch(const Pages& pg, const void* k_pages, const void* v_pages, const void* k_scale, const void* v_scale,
                 const int32_t* idx, int first, int n_rows, void* k_out, void* v_out, hipStream_t st) {
  constexpr int U = 4;
  auto go = [&](auto kern, auto* out) {
    hipLaunchKernelGGL(kern, wide_grid((int64_t)((n_rows + 16 * U - 1) / (16 * U)) * pg.n_seqs * pg.Hkv * 2), dim3(256), 0, st, pg, (const char*)k_pages,
                       (const char*)v_pages, (const uint32_t*)k_scale, (const uint32_t*)v_scale, idx, first, n_rows,
                       (decltype(out))k_out, (decltype(out))v_out);
    return hip_status();
  };
  const bool q4 = pg.fmt == RESTKV_Q4;
  // what is read goes past the caches too (whole lines: rows that are not 4 bits, nor float32 of 128 channels) if it is more than the last-level one holds:
  // 270 MB 98 -> 91 us, but 67 MB that the last call has read too 41.2 -> 46.5.  (4 bits, a line in parts: 9.7 -> 12.5.)
  const bool past = (int64_t)pg.n_seqs * pg.Hkv * n_rows * pg.d * (pg.dtype == RESTKV_F32 ? 8 : 4) > (int64_t)256 << 20;
  auto by = [&](auto* t, auto d) {
    using T = std::remove_pointer_t<decltype(t)>;
    constexpr int D = decltype(d)::value;
    if (q4) return go(k_fetch<T, D, true, U, false>, t);
    return past ? go(k_fetch<T, D, false, U, true>, t) : go(k_fetch<T, D, false, U, false>, t);
  };
  auto by_d = [&](auto* t) { return pg.d == 128 ? by(t, std::integral_constant<int, 128>{}) : by(t, std::integral_constant<int, 64>{}); };
  return pg.dtype == RESTKV_F32 ? by_d((float*)nullptr) : by_d((bf16_t*)nullptr);
}

}  // namespace restkv
