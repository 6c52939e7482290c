// New keys (rotated by their position) and values into the pages of a cache, and new queries rotated beside them.
#include "pages.hpp"

namespace restkv {

namespace {

template <typename T, int UN, bool VEC>
__device__ __forceinline__ void load_unit(const T* p, float (&x)[UN]) {
  if constexpr (!VEC) {
#pragma unroll
    for (int i = 0; i < UN; ++i) x[i] = to_float(p[i]);
  } else if constexpr (sizeof(T) == 4) {
#pragma unroll
    for (int i = 0; i < UN; i += 4) {
      const float4 v = *(const float4*)(p + i);
      x[i] = v.x; x[i + 1] = v.y; x[i + 2] = v.z; x[i + 3] = v.w;
    }
  } else {
    uint32_t w[UN / 2];
    if constexpr (UN == 8) {
      const uint4 v = *(const uint4*)p;
      w[0] = v.x; w[1] = v.y; w[2] = v.z; w[3] = v.w;
    } else {
      const uint2 v = *(const uint2*)p;
      w[0] = v.x; w[1] = v.y;
    }
#pragma unroll
    for (int i = 0; i < UN / 2; ++i) {
      x[2 * i] = __uint_as_float(w[i] << 16);
      x[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
    }
  }
}

template <typename T, int UN, bool VEC>
__device__ __forceinline__ void store_unit(T* p, const float (&x)[UN]) {
  if constexpr (sizeof(T) == 4) {
    if constexpr (VEC) {
#pragma unroll
      for (int i = 0; i < UN; i += 4) *(float4*)((float*)p + i) = make_float4(x[i], x[i + 1], x[i + 2], x[i + 3]);
    } else {
#pragma unroll
      for (int i = 0; i < UN; ++i) ((float*)p)[i] = x[i];
    }
  } else {
    uint32_t w[UN / 2];
#pragma unroll
    for (int i = 0; i < UN / 2; ++i)
      w[i] = __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{x[2 * i], x[2 * i + 1]}, bf16x2));
    if constexpr (!VEC) {
#pragma unroll
      for (int i = 0; i < UN; ++i) p[i].x = (uint16_t)(w[i / 2] >> (16 * (i & 1)));
    } else if constexpr (UN == 8) {
      *(uint4*)p = make_uint4(w[0], w[1], w[2], w[3]);
    } else {
      *(uint2*)p = make_uint2(w[0], w[1]);
    }
  }
}

// Rotation of the unit at channel c0: each product and each sum rounded to 32 bits (no contraction), so that the codes of
// a 4-bit cache follow from the definition bit by bit.
template <typename T, int UN, bool VEC>
__device__ __forceinline__ void rotate_unit(const Pages& pg, const T* row, int c0, const float* cos, const float* sin, int pos,
                                            float (&x)[UN]) {
#pragma clang fp contract(off)
  if (c0 >= pg.rot) return;
  const int half = pg.rot >> 1;
  if (pg.rot_pairs) {
    const int64_t at = (int64_t)pos * half + c0 / 2;
#pragma unroll
    for (int i = 0; i < UN / 2; ++i) {
      const float c = cos[at + i], s = sin[at + i], a = x[2 * i], b = x[2 * i + 1];
      x[2 * i] = a * c - b * s;
      x[2 * i + 1] = b * c + a * s;
    }
  } else {
    const bool second = c0 >= half;
    const int f0 = second ? c0 - half : c0;
    float other[UN];
    load_unit<T, UN, VEC>(row + (second ? f0 : c0 + half), other);
    const float* cp = cos + (int64_t)pos * half + f0;
    const float* sp = sin + (int64_t)pos * half + f0;
#pragma unroll
    for (int i = 0; i < UN; ++i) {
      const float p = x[i] * cp[i], r = other[i] * sp[i];
      x[i] = second ? p + r : p - r;
    }
  }
}

// One wavefront per four rows of a token (rows: KV heads' keys, their values, query heads), sixteen lanes a row, a lane the
// d/16 channels of a unit: accesses run along rows, and a group's extremes are a reduction over sixteen lanes.
template <typename T, int D, bool Q4, bool VEC>
__global__ __launch_bounds__(256) void k_append(Pages pg, const T* k, const T* v, char* k_pages, char* v_pages,
                                                uint32_t* k_scale, uint32_t* v_scale, const int32_t* __restrict__ positions,
                                                const float* __restrict__ cos, const float* __restrict__ sin, const T* q, T* q_out,
                                                int chunks, int n_rows) {
  constexpr int UN = D / 16, NG = D / 32;
  const int lane = threadIdx.x & 63;
  const int64_t w = wide_block() * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int t = (int)(w / chunks), r = (int)(w % chunks) * 4 + (lane >> 4);
  if (w >= (int64_t)pg.n_tokens * chunks) return;
  // the sequence of token t: the last one that starts at or before it
  int s;
  if (pg.new_start) {
    int lo = 0;
    for (int base = 0; base < pg.n_seqs; base += 64) {
      const int e = base + lane;
      const unsigned long long before = __ballot(e < pg.n_seqs && pg.new_start[e] <= t);
      if (before) lo = base + 63 - __builtin_clzll(before);
      if (before != ~0ull) break;
    }
    s = lo;
  } else {
    s = t / pg.max_new;
  }
  if (s >= pg.n_seqs) return;
  const NewRows nr = new_rows(pg, s);
  const int i = t - nr.first;
  if (i < 0 || i >= nr.n || r >= n_rows) return;
  const bool is_q = r >= 2 * pg.Hkv, is_v = !is_q && r >= pg.Hkv;
  const int h = is_q ? r - 2 * pg.Hkv : is_v ? r - pg.Hkv : r;
  const int u = lane & 15, c0 = u * UN;
  const T* row = is_q ? q + t * pg.q_st + h * pg.q_sh : (is_v ? v : k) + t * pg.kv_st + h * pg.kv_sh;
  float x[UN];
  load_unit<T, UN, VEC>(row + c0, x);
  const int at = told_len(pg, s, is_q ? 0 : h) - nr.n + i;
  if (pg.rot) {
    const int pos = positions ? positions[t] : at;
    if (pos < 0 || pos >= pg.n_pos) return;        // (all rows of the token alike)
    if (!is_v) rotate_unit<T, UN, VEC>(pg, row, c0, cos, sin, pos, x);
  }
  if (is_q) {
    store_unit<T, UN, VEC>(q_out + t * pg.q_st + h * pg.q_sh + c0, x);
    return;
  }
  if (at < 0 || at >= pg.max_len) return;
  const int page = page_of(pg, s, h, at);
  if (page < 0) return;
  const int64_t slot = row_of(pg, page, h, at);
  char* dst = is_v ? v_pages : k_pages;
  if constexpr (!Q4) {
    store_unit<T, UN, true>((T*)dst + slot * D + c0, x);
  } else {
    uint32_t code = 0u, scale[NG];
#pragma unroll
    for (int f = 0; f < NG; ++f) {
#pragma clang fp contract(off)
      const float a = x[2 * f], b = x[2 * f + 1];
      // (a NaN or an infinity leaves a difference that is not zero)
      const float off = row16_max(a - a == 0.f && b - b == 0.f ? 0.f : 1.f);
      float step, zero, inverse;
      group_scale(row16_min(fminf(a, b)), row16_max(fmaxf(a, b)), off == 0.f, step, zero, inverse);
      const float ca = __builtin_rintf((a - zero) * inverse), cb = __builtin_rintf((b - zero) * inverse);
      const uint32_t ia = step > 0.f ? (uint32_t)fminf(fmaxf(ca, 0.f), 15.f) : 0u;
      const uint32_t ib = step > 0.f ? (uint32_t)fminf(fmaxf(cb, 0.f), 15.f) : 0u;
      code |= (ia | ib << 4) << (8 * f);
      scale[f] = __float_as_uint(step) >> 16 | (__float_as_uint(zero) & 0xFFFF0000u);
    }
    uint32_t* sc = (is_v ? v_scale : k_scale) + slot * NG;
    if constexpr (UN == 8) {
      *(uint32_t*)(dst + slot * (D / 2) + u * 4) = code;
      if (u == 0) *(uint4*)sc = make_uint4(scale[0], scale[1], scale[2], scale[3]);
    } else {
      *(uint16_t*)(dst + slot * (D / 2) + u * 2) = (uint16_t)code;
      if (u == 0) *(uint2*)sc = make_uint2(scale[0], scale[1]);
    }
  }
}

template <typename T, int D, bool Q4>
int run_append(const Pages& pg, const void* k, const void* v, void* k_pages, void* v_pages, void* k_scale, void* v_scale,
               const int32_t* positions, const float* cos, const float* sin, const void* q, void* q_out, hipStream_t st) {
  const int n_rows = 2 * pg.Hkv + (q ? pg.Hq : 0), chunks = (n_rows + 3) / 4;
  const int64_t blocks = ((int64_t)pg.n_tokens * chunks + 3) / 4;
  const int unit = D / 16 * (int)sizeof(T), mask = (unit < 16 ? unit : 16) - 1, el = (mask + 1) / (int)sizeof(T) - 1;
  const bool vec = !(((uintptr_t)k | (uintptr_t)v | (uintptr_t)q | (uintptr_t)q_out) & mask) &&
                   !((pg.kv_st | pg.kv_sh | (q ? pg.q_st | pg.q_sh : 0)) & el);
  auto go = [&](auto kern) {
    hipLaunchKernelGGL(kern, wide_grid(blocks), dim3(256), 0, st, pg, (const T*)k, (const T*)v, (char*)k_pages, (char*)v_pages,
                       (uint32_t*)k_scale, (uint32_t*)v_scale, positions, cos, sin, (const T*)q, (T*)q_out, chunks, n_rows);
  };
  if (vec) go(k_append<T, D, Q4, true>);
  else go(k_append<T, D, Q4, false>);
  return hip_status();
}

}  // namespace

int launch_append(const Pages& pg, const void* k, const void* v, void* k_pages, void* v_pages, void* k_scale, void* v_scale,
                  const int32_t* positions, const float* cos, const float* sin, const void* q, void* q_out, hipStream_t st) {
  auto go = [&](auto f) { return f(pg, k, v, k_pages, v_pages, k_scale, v_scale, positions, cos, sin, q, q_out, st); };
  const bool q4 = pg.fmt == RESTKV_Q4;
  if (pg.dtype == RESTKV_F32) {
    if (pg.d == 128) return q4 ? go(run_append<float, 128, true>) : go(run_append<float, 128, false>);
    return q4 ? go(run_append<float, 64, true>) : go(run_append<float, 64, false>);
  }
  if (pg.d == 128) return q4 ? go(run_append<bf16_t, 128, true>) : go(run_append<bf16_t, 128, false>);
  return q4 ? go(run_append<bf16_t, 64, true>) : go(run_append<bf16_t, 64, false>);
}

}  // namespace restkv
