// Rows of a paged cache as dense keys and values (4-bit rows as the values they stand for).
#include "pages.hpp"

namespace restkv {

namespace {

// Sixteen lanes a row, a lane the d/16 channels of a unit; sixteen rows of a head, of keys or of values, a workgroup.
template <typename T, int D, bool Q4>
__global__ __launch_bounds__(256) void k_fetch(Pages pg, const char* k_pages, const char* v_pages, const uint32_t* k_scale,
                                               const uint32_t* v_scale, const int32_t* __restrict__ idx, int first, int n_rows,
                                               T* k_out, T* v_out) {
  constexpr int UN = D / 16, NG = D / 32;
  const int u = threadIdx.x & 15;
  const int64_t b = wide_block();
  const int blocks = (n_rows + 15) / 16;
  const bool is_v = b & 1;
  const int64_t e = (b >> 1) / blocks;
  const int j = (int)((b >> 1) % blocks) * 16 + (threadIdx.x >> 4);
  if (e >= (int64_t)pg.n_seqs * pg.Hkv || j >= n_rows) return;
  const int s = (int)(e / pg.Hkv), h = (int)(e % pg.Hkv);
  const int64_t o = e * n_rows + j;
  const int t = idx ? idx[o] : first + j;
  int page = -1;
  if (t >= 0 && t < cache_len(pg, s, h)) page = page_of(pg, s, h, t);
  const int64_t slot = page >= 0 ? row_of(pg, page, h, t) : 0;
  const char* src = is_v ? v_pages : k_pages;
  T* dst = (is_v ? v_out : k_out) + o * D + u * UN;
  if constexpr (!Q4) {
    constexpr int B = UN * sizeof(T);            // bytes of a unit: 8, 16 or 32
    const char* p = src + slot * (D * (int64_t)sizeof(T)) + u * B;
    if constexpr (B == 8) {
      *(uint2*)dst = page >= 0 ? *(const uint2*)p : make_uint2(0, 0);
    } else {
#pragma unroll
      for (int i = 0; i < B / 16; ++i) ((uint4*)dst)[i] = page >= 0 ? ((const uint4*)p)[i] : make_uint4(0, 0, 0, 0);
    }
  } else {
    float x[UN];
    if (page >= 0) {
      const uint32_t* sc = (is_v ? v_scale : k_scale) + slot * NG;
      const uint32_t code = UN == 8 ? *(const uint32_t*)(src + slot * (D / 2) + u * 4)
                                    : *(const uint16_t*)(src + slot * (D / 2) + u * 2);
#pragma unroll
      for (int i = 0; i < UN; ++i) {
        const uint32_t w = sc[i / 2];
        x[i] = __uint_as_float(w & 0xFFFF0000u) + __uint_as_float(w << 16) * (float)(code >> (4 * i) & 15u);
      }
    } else {
#pragma unroll
      for (int i = 0; i < UN; ++i) x[i] = 0.f;
    }
    if constexpr (sizeof(T) == 4) {
#pragma unroll
      for (int i = 0; i < UN; i += 4) *(float4*)((float*)dst + i) = make_float4(x[i], x[i + 1], x[i + 2], x[i + 3]);
    } else {
      uint32_t w[UN / 2];
#pragma unroll
      for (int i = 0; i < UN / 2; ++i)
        w[i] = __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{x[2 * i], x[2 * i + 1]}, bf16x2));
      if constexpr (UN == 8) *(uint4*)dst = make_uint4(w[0], w[1], w[2], w[3]);
      else *(uint2*)dst = make_uint2(w[0], w[1]);
    }
  }
}

}  // namespace

int launch_fetch(const Pages& pg, const void* k_pages, const void* v_pages, const void* k_scale, const void* v_scale,
                 const int32_t* idx, int first, int n_rows, void* k_out, void* v_out, hipStream_t st) {
  auto go = [&](auto kern, auto* out) {
    hipLaunchKernelGGL(kern, wide_grid((int64_t)((n_rows + 15) / 16) * pg.n_seqs * pg.Hkv * 2), dim3(256), 0, st, pg, (const char*)k_pages,
                       (const char*)v_pages, (const uint32_t*)k_scale, (const uint32_t*)v_scale, idx, first, n_rows,
                       (decltype(out))k_out, (decltype(out))v_out);
    return hip_status();
  };
  const bool q4 = pg.fmt == RESTKV_Q4;
  if (pg.dtype == RESTKV_F32) {
    float* t = nullptr;
    if (pg.d == 128) return q4 ? go(k_fetch<float, 128, true>, t) : go(k_fetch<float, 128, false>, t);
    return q4 ? go(k_fetch<float, 64, true>, t) : go(k_fetch<float, 64, false>, t);
  }
  bf16_t* t = nullptr;
  if (pg.d == 128) return q4 ? go(k_fetch<bf16_t, 128, true>, t) : go(k_fetch<bf16_t, 128, false>, t);
  return q4 ? go(k_fetch<bf16_t, 64, true>, t) : go(k_fetch<bf16_t, 64, false>, t);
}

}  // namespace restkv
