// New keys (rotated by their position) and values into the pages of a cache, and new queries rotated beside them.
#include "pages.hpp"

namespace restkv {

namespace {

template <typename T, int UN, bool VEC, bool PAST>
__device__ __forceinline__ void load_unit(const T* p, float (&x)[UN]) {
  if constexpr (!VEC) {
#pragma unroll
    for (int i = 0; i < UN; ++i) x[i] = to_float(p[i]);
  } else if constexpr (sizeof(T) == 4) {
#pragma unroll
    for (int i = 0; i < UN; i += 4) {
      const f32x4 v = get<PAST && UN == 4, f32x4>(p + i);
      x[i] = v[0]; x[i + 1] = v[1]; x[i + 2] = v[2]; x[i + 3] = v[3];
    }
  } else {
    uint32_t w[UN / 2];
    if constexpr (UN == 8) {
      const Words<4> v = get<PAST, Words<4>>(p);
      w[0] = v[0]; w[1] = v[1]; w[2] = v[2]; w[3] = v[3];
    } else {
      const Words<2> v = get<PAST, Words<2>>(p);
      w[0] = v[0]; w[1] = v[1];
    }
#pragma unroll
    for (int i = 0; i < UN / 2; ++i) {
      x[2 * i] = __uint_as_float(w[i] << 16);
      x[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
    }
  }
}

template <typename T, int UN, bool VEC, bool PAST>
__device__ __forceinline__ void store_unit(T* p, const float (&x)[UN]) {
  if constexpr (sizeof(T) == 4) {
    if constexpr (VEC) {
#pragma unroll
      for (int i = 0; i < UN; i += 4) put<PAST>((float*)p + i, f32x4{x[i], x[i + 1], x[i + 2], x[i + 3]});
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
      put<PAST>(p, Words<4>{w[0], w[1], w[2], w[3]});
    } else {
      put<PAST>(p, Words<2>{w[0], w[1]});
    }
  }
}

__device__ __forceinline__ float other_half(float x) {       // the value eight lanes on, of sixteen
  return __uint_as_float(__builtin_amdgcn_mov_dpp(__float_as_uint(x), 0x128, 0xF, 0xF, true));
}

// Angles of the unit at channel c0: UN cosines and sines (UN / 2 where neighbours turn together).
template <int UN>
struct Turn { float c[UN], s[UN]; };
template <int UN>
__device__ __forceinline__ Turn<UN> angles(const Pages& pg, int c0, const float* cos, const float* sin, int pos) {
  Turn<UN> t;
  const int half = pg.rot >> 1;
  if (pg.rot_pairs) {
    const int64_t at = (int64_t)pos * half + c0 / 2;
#pragma unroll
    for (int i = 0; i < UN / 2; ++i) { t.c[i] = cos[at + i]; t.s[i] = sin[at + i]; }
  } else {
    const int64_t at = (int64_t)pos * half + (c0 >= half ? c0 - half : c0);
#pragma unroll
    for (int i = 0; i < UN; ++i) { t.c[i] = cos[at + i]; t.s[i] = sin[at + i]; }
  }
  return t;
}

// Rotation of the unit at channel c0: each product and each sum rounded to 32 bits (no contraction), so that the codes of
// a 4-bit cache follow from the definition bit by bit.  other: the channels it turns with (where not its own).
template <int UN>
__device__ __forceinline__ void rotate_unit(const Pages& pg, int c0, const Turn<UN>& t, const float (&other)[UN], float (&x)[UN]) {
#pragma clang fp contract(off)
  if (pg.rot_pairs) {
#pragma unroll
    for (int i = 0; i < UN / 2; ++i) {
      const float a = x[2 * i], b = x[2 * i + 1];
      x[2 * i] = a * t.c[i] - b * t.s[i];
      x[2 * i + 1] = b * t.c[i] + a * t.s[i];
    }
  } else {
    const bool second = c0 >= pg.rot >> 1;
#pragma unroll
    for (int i = 0; i < UN; ++i) {
      const float p = x[i] * t.c[i], r = other[i] * t.s[i];
      x[i] = p + (second ? r : -r);
    }
  }
}

// Codes of the unit, a group's extremes over the sixteen lanes of the row, and the row's {step, zero} of every group.
// Lane u works out the scale of group u mod NG for all.
template <int UN>
__device__ __forceinline__ uint32_t unit_codes(const float (&x)[UN], int u, uint32_t (&scale)[UN / 2]) {
#pragma clang fp contract(off)
  constexpr int NG = UN / 2;
  int low = 0, high = 0;
#pragma unroll
  for (int f = 0; f < NG; ++f) {
    const int a = order_of(x[2 * f]), b = order_of(x[2 * f + 1]);
    const int lo = row16_min(min(a, b)), hi = row16_max(max(a, b));
    if (f == (u & (NG - 1))) { low = lo; high = hi; }
  }
  float step, zero, inverse;
  group_scale(of_order(low), of_order(high), step, zero, inverse);
  const uint32_t packed = __float_as_uint(step) >> 16 | (__float_as_uint(zero) & 0xFFFF0000u);
  auto codes = [&](auto rare) {
    uint32_t code = 0u;
#pragma unroll
    for (int f = NG - 1; f >= 0; --f) {
      // lane f of every NG: quad_perm
      auto of = [&](uint32_t v) -> uint32_t {
        if constexpr (NG == 4) return f == 0 ? __builtin_amdgcn_mov_dpp(v, 0x00, 0xF, 0xF, true) : f == 1 ? __builtin_amdgcn_mov_dpp(v, 0x55, 0xF, 0xF, true)
                                    : f == 2 ? __builtin_amdgcn_mov_dpp(v, 0xAA, 0xF, 0xF, true) : __builtin_amdgcn_mov_dpp(v, 0xFF, 0xF, 0xF, true);
        else return f == 0 ? __builtin_amdgcn_mov_dpp(v, 0xA0, 0xF, 0xF, true) : __builtin_amdgcn_mov_dpp(v, 0xF5, 0xF, 0xF, true);
      };
      scale[f] = of(packed);
      const float z = __uint_as_float(scale[f] & 0xFFFF0000u), inv = __uint_as_float(of(__float_as_uint(inverse)));
#pragma unroll
      for (int i = 1; i >= 0; --i) {
        // 0 <= (x - zero) / step <= 15 (1 + 2^-21), since zero and step are rounded outwards: adding 2^23 rounds it to the
        // nearest whole number, even at a tie, which then is in the low bits
        float t = (x[2 * f + i] - z) * inv;
        if (rare && !(z == z)) t = 0.f;
        code = (code << 4) + __float_as_uint(t + 8388608.f);
      }
    }
    return code - 0xFB000000u;       // 0x4B000000 (1 + 16 + 256 + ...), mod 2^32
  };
  return __ballot(!(zero == zero)) ? codes(std::true_type{}) : codes(std::false_type{});      // (groups without a scale)
}

// A wavefront takes U times four rows of a token (rows: KV heads' keys, their values, query heads), sixteen lanes a row, a lane
// the d/16 channels of a unit: accesses run along rows, and a group's extremes are a reduction over sixteen lanes.  U = 4 has
// four rows a lane in flight and reads the angles once for them; few tokens take U = 1, for more wavefronts.  Many tokens' queries
// go past the caches, their pages do not (2 / (G + 2) of it, and who attends or fetches reads them next).
// Bound by memory: 32k tokens of 32 and 8 heads of 128 bf16, 822 MB in 143.9 us (5.7 TB/s); into 4 bits by vector instructions too,
// ten a code: 8k tokens 183 MB in 36.7 us.  32 tokens of a decoding step 3.6 us, a chain of lengths, page and rows.
template <typename T, int D, bool Q4, bool VEC, int U, bool PAST>
__global__ __launch_bounds__(256) void k_append(Pages pg, const T* k, const T* v, char* k_pages, char* v_pages,
                                                uint32_t* k_scale, uint32_t* v_scale, const int32_t* __restrict__ positions,
                                                const float* __restrict__ cos, const float* __restrict__ sin, const T* q, T* q_out,
                                                int parts, int n_rows) {
  constexpr int UN = D / 16, NG = D / 32;
  const int lane = threadIdx.x & 63;
  const int64_t w = wide_block() * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  if (w >= (int64_t)pg.n_tokens * parts) return;
  const int t = (int)(w / parts), part = (int)(w % parts);
  // the sequence of token t: the last one that starts at or before it
  int s = 0;
  NewRows nr = {0, pg.max_new};
  if (pg.new_start) {
    for (int base = 0; base < pg.n_seqs && pg.n_seqs > 1; base += 64) {
      const int e = base + lane;
      const unsigned long long before = __ballot(e < pg.n_seqs && pg.new_start[e] <= t);
      if (before) s = base + 63 - __builtin_clzll(before);
      if (before != ~0ull) break;
    }
    const int a = min(max(uniform_load(pg.new_start + s), 0), pg.n_tokens);
    const int b = min(max(uniform_load(pg.new_start + s + 1), a), pg.n_tokens);
    nr = {a, min(b - a, pg.max_new)};
  } else {
    s = t / pg.max_new;
    nr.first = s * pg.max_new;
  }
  if (s >= pg.n_seqs) return;
  const int i = t - nr.first;
  if (i < 0 || i >= nr.n) return;
  const int u = lane & 15, c0 = u * UN;
  const bool turns = c0 < pg.rot;
  const int32_t* lens = pg.lens + s * pg.lens_ss;
  const int32_t* table = pg.table + s * pg.table_ss;
  // all that is read, asked for before any of it is used: rows (the last one again behind the last), angles, and where the
  // rows go
  int r[U];
  float x[U][UN], other[U][UN];
  // (what does not turn with its own neighbour has its partner eight lanes on if the whole row turns, else in memory)
  const bool far = pg.rot && !pg.rot_pairs && pg.rot != D;
#pragma unroll
  for (int c = 0; c < U; ++c) {
    r[c] = (part * U + c) * 4 + (lane >> 4);
    const int rc = min(r[c], n_rows - 1);
    const T* row = rc >= 2 * pg.Hkv ? q + t * pg.q_st + (rc - 2 * pg.Hkv) * pg.q_sh
                                    : (rc >= pg.Hkv ? v - pg.Hkv * pg.kv_sh : k) + t * pg.kv_st + rc * pg.kv_sh;
    load_unit<T, UN, VEC, PAST>(row + c0, x[c]);
    if (far && turns) load_unit<T, UN, VEC, false>(row + (c0 >= pg.rot >> 1 ? c0 - (pg.rot >> 1) : c0 + (pg.rot >> 1)), other[c]);
  }
  Turn<UN> turn;
  if (pg.rot) {
    const int pos = positions ? uniform_load(positions + t) : max(uniform_load(lens), 0) - nr.n + i;
    if (pos < 0 || pos >= pg.n_pos) return;        // (the whole token)
    if (turns) turn = angles<UN>(pg, c0, cos, sin, pos);
  }
  uint32_t slot[U];                                // where there is room
  bool room[U];
  if (!pg.lens_sh && !pg.table_sh) {
    const int at = max(uniform_load(lens), 0) - nr.n + i;
    const bool in = at >= 0 && at < pg.max_len;
    const int page = in ? uniform_load(table + (at >> pg.lg_ps)) : -1;
#pragma unroll
    for (int c = 0; c < U; ++c) {
      const int h = r[c] >= pg.Hkv ? r[c] - pg.Hkv : r[c];
      room[c] = page >= 0 && page < pg.n_pages;
      slot[c] = row_of(pg, page, h, at);
    }
  } else {
    int at[U];
#pragma unroll
    for (int c = 0; c < U; ++c) {
      const int h = min(r[c] >= pg.Hkv ? r[c] - pg.Hkv : r[c], pg.Hkv - 1);
      at[c] = max(lens[h * pg.lens_sh], 0) - nr.n + i;
    }
#pragma unroll
    for (int c = 0; c < U; ++c) {
      const int h = min(r[c] >= pg.Hkv ? r[c] - pg.Hkv : r[c], pg.Hkv - 1);
      const int page = at[c] >= 0 && at[c] < pg.max_len ? page_of(pg, s, h, at[c]) : -1;
      room[c] = page >= 0;
      slot[c] = row_of(pg, page, h, at[c]);
    }
  }
#pragma unroll
  for (int c = 0; c < U; ++c) {
    const bool is_q = r[c] >= 2 * pg.Hkv, is_v = !is_q && r[c] >= pg.Hkv;
    if (pg.rot && !is_v) {
      if (!far && !pg.rot_pairs)
#pragma unroll
        for (int m = 0; m < UN; ++m) other[c][m] = other_half(x[c][m]);
      if (turns) rotate_unit<UN>(pg, c0, turn, other[c], x[c]);
    }
    if (is_q) {
      if (r[c] < n_rows) store_unit<T, UN, VEC, U != 1>(q_out + t * pg.q_st + (r[c] - 2 * pg.Hkv) * pg.q_sh + c0, x[c]);
      continue;
    }
    if (!room[c]) continue;
    char* dst = is_v ? v_pages : k_pages;
    if constexpr (!Q4) {
      store_unit<T, UN, true, false>((T*)dst + (int64_t)slot[c] * D + c0, x[c]);
    } else {
      uint32_t scale[NG];
      const uint32_t code = unit_codes<UN>(x[c], u, scale);
      uint32_t* sc = (is_v ? v_scale : k_scale) + (int64_t)slot[c] * NG;
      if constexpr (UN == 8) {
        *(uint32_t*)(dst + (int64_t)slot[c] * (D / 2) + u * 4) = code;
        if (u == 0) *(uint4*)sc = make_uint4(scale[0], scale[1], scale[2], scale[3]);
      } else {
        *(uint16_t*)(dst + (int64_t)slot[c] * (D / 2) + u * 2) = (uint16_t)code;
        if (u == 0) *(uint2*)sc = make_uint2(scale[0], scale[1]);
      }
    }
  }
}

template <typename T, int D, bool Q4>
int run_append(const Pages& pg, const void* k, const void* v, void* k_pages, void* v_pages, void* k_scale, void* v_scale,
               const int32_t* positions, const float* cos, const float* sin, const void* q, void* q_out, hipStream_t st) {
  const int n_rows = 2 * pg.Hkv + (q ? pg.Hq : 0), chunks = (n_rows + 3) / 4;
  const int unit = D / 16 * (int)sizeof(T), mask = (unit < 16 ? unit : 16) - 1, el = (mask + 1) / (int)sizeof(T) - 1;
  const bool vec = !(((uintptr_t)k | (uintptr_t)v | (uintptr_t)q | (uintptr_t)q_out) & mask) &&
                   !((pg.kv_st | pg.kv_sh | (q ? pg.q_st | pg.q_sh : 0)) & el);
  // four groups of rows a wavefront where that leaves five wavefronts a unit (4 bits: sixteen).  One / four, us, tokens of 32 and 8
  // heads of 128: bf16 64 tokens 3.1 / 4.2, 512 5.4 / 4.9, 2048 13.1 / 9.5; 4 bits 512 5.8 / 7.1, 2048 14.5 / 13.1
  const bool few = (int64_t)pg.n_tokens * ((chunks + 3) / 4) < (int64_t)n_cu() * (Q4 ? 16 : 5);
  auto go = [&](auto kern, int U) {
    const int parts = (chunks + U - 1) / U;
    hipLaunchKernelGGL(kern, wide_grid(((int64_t)pg.n_tokens * parts + 3) / 4), dim3(256), 0, st, pg, (const T*)k, (const T*)v, (char*)k_pages,
                       (char*)v_pages, (uint32_t*)k_scale, (uint32_t*)v_scale, positions, cos, sin, (const T*)q, (T*)q_out, parts, n_rows);
  };
  // More than the last-level cache holds, each row once: read past the caches.  With the caches / past them, us, tokens of 32 and 8 heads
  // of 128 bf16, three inputs in turn: 24k tokens 110.6 / 104.9, 32k 145.9 / 145.3, 64k 286.9 / 289.1, 64k into 4 bits 274.7 / 267.5; what the
  // last call has read too, 32k 146.9 / 129.8, 64k 286.7 / 269.7, but 100 MB 36 / 40.
  const bool once = !(pg.rot && !pg.rot_pairs && pg.rot != D);
  const bool past = once && (int64_t)pg.n_tokens * n_rows * D * (int)sizeof(T) > (int64_t)256 << 20;
  if (!vec) go(k_append<T, D, Q4, false, 1, false>, 1);
  else if (few) go(k_append<T, D, Q4, true, 1, false>, 1);
  else if (past) go(k_append<T, D, Q4, true, 4, true>, 4);
  else go(k_append<T, D, Q4, true, 4, false>, 4);
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
