// Paged cache: what its kernels share (lengths and pages that only the device knows, 4-bit rows).
#pragma once

#include "score_common.hpp"

namespace restkv {

// Resolved cache description.  Device data that lies outside its bounds (lengths, counts, page numbers, positions) is
// brought inside or left out by the helpers below, so that no kernel touches memory that is not the caller's.
struct Pages {
  int n_seqs, Hq, Hkv, G, d, dtype, fmt, out_dtype;
  int lg_ps, n_pages, max_pages, max_len, max_new, n_tokens, causal, rot, rot_pairs, n_pos;
  float scale;
  int64_t page_s, head_s, tok_s;                              // in rows
  int64_t table_ss, table_sh, lens_ss, lens_sh;
  int64_t q_st, q_sh, kv_st, kv_sh, o_st, o_sh, lse_st, lse_sh;
  const int32_t* table;
  const int32_t* lens;
  const int32_t* new_start;
};

int resolve_cache(const restkv_cache* c, Pages* o);

int launch_append(const Pages& pg, const void* k, const void* v, void* k_pages, void* v_pages, void* k_scale, void* v_scale,
                  const int32_t* positions, const float* cos, const float* sin, const void* q, void* q_out, hipStream_t st);
int launch_fetch(const Pages& pg, const void* k_pages, const void* v_pages, const void* k_scale, const void* v_scale,
                 const int32_t* idx, int first, int n_rows, void* k_out, void* v_out, hipStream_t st);
size_t attend_ws_bytes(const Pages& pg);
int launch_attend(const Pages& pg, const void* q, const void* k_pages, const void* v_pages, const void* k_scale,
                  const void* v_scale, void* out, float* lse, char* ws, hipStream_t st);

// Wave-uniform reads of what the kernel does not write, through the scalar cache.
__device__ __forceinline__ int uniform_load(const int32_t* p) {
  return *(const __attribute__((address_space(4))) int32_t*)(uintptr_t)p;
}

// New tokens of sequence s: rows [first, first + n) of the packed tensors.
struct NewRows { int first, n; };
__device__ __forceinline__ NewRows new_rows(const Pages& pg, int s) {
  if (!pg.new_start) return {s * pg.max_new, pg.max_new};
  const int a = min(max(pg.new_start[s], 0), pg.n_tokens);
  const int b = min(max(pg.new_start[s + 1], a), pg.n_tokens);
  return {a, min(b - a, pg.max_new)};
}
// Cached tokens of (sequence, head) as the caller says, and how many of them there is room for.
__device__ __forceinline__ int told_len(const Pages& pg, int s, int h) {
  return max(pg.lens[s * pg.lens_ss + h * pg.lens_sh], 0);
}
__device__ __forceinline__ int cache_len(const Pages& pg, int s, int h) { return min(told_len(pg, s, h), pg.max_len); }
// Grids of many workgroups in two dimensions (the threads along one of them have to stay below 2^32).
constexpr int64_t GRID_X = 1 << 22;
inline dim3 wide_grid(int64_t n) { return dim3((unsigned)(n < GRID_X ? n : GRID_X), (unsigned)((n + GRID_X - 1) / GRID_X)); }
__device__ __forceinline__ int64_t wide_block() { return (int64_t)blockIdx.y * GRID_X + blockIdx.x; }
// Page that holds cache position t of (sequence, head), or -1; t must lie in [0, max_pages << lg_ps).
__device__ __forceinline__ int page_of(const Pages& pg, int s, int h, int t) {
  const int p = pg.table[s * pg.table_ss + h * pg.table_sh + (t >> pg.lg_ps)];
  return p >= 0 && p < pg.n_pages ? p : -1;
}
// Row of that position (rows of an array are counted in 32 bits: resolve_cache).
__device__ __forceinline__ uint32_t row_of(const Pages& pg, int page, int h, int t) {
  return (uint32_t)page * (uint32_t)pg.page_s + (uint32_t)h * (uint32_t)pg.head_s + (t & ((1 << pg.lg_ps) - 1)) * (uint32_t)pg.tok_s;
}

// Words of a store or load; PAST: past the caches (nontemporal), for what is more than they hold, a whole line at a time.  What is
// written so is on its way before the kernel's end flushes the L2s: append of 32k tokens, whose queries are two thirds of
// it, 157 -> 143 us, fetch of 4-bit rows (10 MB into 34) 10.8 -> 9.7, of 270 MB with loads as they were 106 -> 98.
typedef float f32x4 __attribute__((ext_vector_type(4)));
template <int N> struct WordsOf { typedef uint32_t type __attribute__((ext_vector_type(N))); };
template <> struct WordsOf<1> { typedef uint32_t type; };
template <int N> using Words = typename WordsOf<N>::type;
template <bool PAST, typename W>
__device__ __forceinline__ void put(void* p, W w) {
  if constexpr (PAST) __builtin_nontemporal_store(w, (W*)p);
  else *(W*)p = w;
}
template <bool PAST, typename W>
__device__ __forceinline__ W get(const void* p) {
  if constexpr (PAST) return __builtin_nontemporal_load((const W*)p);
  else return *(const W*)p;
}

// ---- 4-bit rows ---------------------------------------------------------------
// A row of d channels is 16 units of d/16 channels; group f holds the channels at places 2f and 2f+1 of every unit (32
// channels).  A group's values are zero + step * code, code 0 .. 15, zero and step bfloat16.  Why units: in the products of
// the attention a lane holds one unit of a value row (16 lanes a row) or four of a key row, and one matrix instruction takes
// the same place of every unit; so all it multiplies has one step per key.
__device__ __forceinline__ float bf16_below(float x) {       // largest bfloat16 that is not above x
  const uint32_t u = __float_as_uint(x), cut = u & 0xFFFF0000u;
  return __uint_as_float((u >> 31) && u != cut ? cut + 0x10000u : cut);
}

// Floats as integers of the same order, and back (a NaN lies beyond the infinities): least and greatest of integers take a
// lane shift in the same instruction, those of floats do not.
__device__ __forceinline__ int order_of(float x) {
  const int b = __float_as_int(x);
  return b ^ ((b >> 31) & 0x7FFFFFFF);
}
__device__ __forceinline__ float of_order(int k) { return __int_as_float(k ^ ((k >> 31) & 0x7FFFFFFF)); }
// Least and greatest over the sixteen lanes of a wavefront's row, in every lane.
template <int CTRL>
__device__ __forceinline__ int row_ror(int x) { return __builtin_amdgcn_mov_dpp(x, CTRL, 0xF, 0xF, true); }
__device__ __forceinline__ int row16_min(int x) {
  x = min(x, row_ror<0x121>(x));        // by 1, 2, 4 and 8 lanes
  x = min(x, row_ror<0x122>(x));
  x = min(x, row_ror<0x124>(x));
  return min(x, row_ror<0x128>(x));
}
__device__ __forceinline__ int row16_max(int x) {
  x = max(x, row_ror<0x121>(x));
  x = max(x, row_ror<0x122>(x));
  x = max(x, row_ror<0x124>(x));
  return max(x, row_ror<0x128>(x));
}

// Step and zero of a group from its extremes; inverse: 1/step, or 0.
__device__ __forceinline__ void group_scale(float low, float high, float& step, float& zero, float& inverse) {
#pragma clang fp contract(off)
  zero = bf16_below(low);
  const float spread = high - zero;
  step = -bf16_below(-(spread / 15.0f));
  step = spread > 0.f ? fmaxf(step, 0x1p-100f) : 0.f;
  // (a group with a NaN or an infinity has it for an extreme: these are looked at as they are, since the integers that round
  // a NaN may wrap to a finite number)
  if (!(__builtin_isfinite(low) && __builtin_isfinite(high) && __builtin_isfinite(spread) && __builtin_isfinite(step) && __builtin_isfinite(zero))) {
    step = 0.f;
    zero = __builtin_nanf("");
  }
  inverse = step > 0.f ? 1.0f / step : 0.f;
}

}  // namespace restkv
