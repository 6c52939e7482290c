// Attention of a sequence's newest tokens over its pages: the kernel, for each format of the pages.
//
// Rows are (new token, query head of the group) pairs of one KV head: softmax(scale q K^T) V in one pass over the keys with
// a running reference and sum.  Keys are cut into chunks by the real lengths, which only the device knows; a workgroup of
// four wavefronts takes a chunk for 16 R rows, its wavefronts every fourth tile of keys, and joins their sums in LDS.
// Everything is transposed (S^T = K Q^T, O^T = V^T P^T): a lane is a row, so its logits, statistics and weights stay in its
// registers, and the weights of two 16-key blocks are an operand of the second product as they come.  Keys and values go from
// memory into operand registers without LDS: a key operand is 16 bytes of a row, a value operand takes the same channel
// of eight keys, which a lane that has loaded a unit of d/16 channels of each of them holds already (one byte
// permute for two values).
// Bound by memory for bf16 (128k positions of 8 KV heads of 128, 537 MB in 89 us, 6.0 TB/s).  4 bits: by no one pipe (the same positions,
// 168 MB in 37.3 us: 4.5 TB/s, about 500 vector instructions a tile of 64 keys, which issue half of the time, matrix pipe 15 %) but by
// what two wavefronts a SIMD do not overlap, and by the longest chunk, nine passes of the loop where the mean is eight.  Short caches: by
// a chain of lengths, pages, keys.
#pragma once

#include "pages.hpp"

namespace restkv {

struct AttendArgs {
  Pages pg;
  const void* q;
  const char* k; const char* v;
  const uint32_t* ks; const uint32_t* vs;
  void* out; float* lse;
  int2* plan;                       // [entries] {first slot, chunks} of an entry (chunks < 2: the output is there already)
  float* part_m; float* part_l; float* part_o;   // [slots * Hy, rows] and [.., d]: chunks of entries that have several
  int entries, per_head, Hy;        // an entry is a sequence, or with lengths per head a (sequence, head); Hy heads share it
  int row_blocks, units, c_min, vec_q, vec_out;
  float chunks;                     // workgroups wanted of each head and row block
  // Beams (launch_attend_beams): entries 0 .. fronts-1 are the shared positions of groups of n_beams sequences (or of a group's
  // head), the rows of all its beams for them; then each sequence's own positions behind these.  An entry times a block of rows is a
  // part: front_blocks of each of the former, own_blocks of each of the latter.  plan[part] {first, last} slot (first > last: none);
  // front_*: [slots of fronts * Hy, rows of a block], part_*: [slots * Hy, rows of a sequence].  spread: parts are cut evenly over
  // the teams of workgroups of a head, of which there are `chunks` (cut_parts); else a workgroup takes a chunk of an entry
  // for a block of rows, and k_beams_list has written which: list[2 u], [2 u + 1] {entry (-1: none), tiles from, to, slot}, {positions, first
  // row, new tokens}, of up to front_chunks chunks of fronts, then up to own_chunks of the rest.
  const int32_t* shared;
  int4* list; int* tiles_of;
  int front_chunks, own_chunks;
  int n_beams, fronts, front_blocks, own_blocks, front_slots, spread, front_rows, own_rows, front_tiles, coarse;
  uint32_t part_cost;
  float first_more;
  float* front_m; float* front_l; float* front_o;
};

constexpr int ATT_TILE = 64;        // chunks are whole tiles of 64 keys

// The grid: x = 8 row blocks by 8 units, so that the row blocks of a unit (a chunk and a head) follow each other on one XCD, whose
// L2 then holds the chunk (workgroups go round eight XCDs); y and z the units by eight.
constexpr int GRID_Y = 32768;
inline dim3 unit_grid(const AttendArgs& a) {
  const unsigned n = ((unsigned)a.units + 7) / 8;
  return dim3(8u * a.row_blocks, n < GRID_Y ? n : GRID_Y, (n + GRID_Y - 1) / GRID_Y);
}
__device__ __forceinline__ int unit_of_block() { return (blockIdx.z * GRID_Y + blockIdx.y) * 8 + (blockIdx.x & 7); }

// Sum over the lanes up to this one.
__device__ __forceinline__ int wave_scan(int x) {
  x += __builtin_amdgcn_update_dpp(0, x, 0x111, 0xF, 0xF, false);   // row_shr:1
  x += __builtin_amdgcn_update_dpp(0, x, 0x112, 0xF, 0xF, false);   // row_shr:2
  x += __builtin_amdgcn_update_dpp(0, x, 0x114, 0xF, 0xF, false);   // row_shr:4
  x += __builtin_amdgcn_update_dpp(0, x, 0x118, 0xF, 0xF, false);   // row_shr:8
  x += __builtin_amdgcn_update_dpp(0, x, 0x142, 0xA, 0xF, false);   // lane 15 of rows 0, 2 to the rows behind them
  x += __builtin_amdgcn_update_dpp(0, x, 0x143, 0xC, 0xF, false);   // lane 31 to the upper half
  return x;
}

// What a workgroup takes.  An entry is cut into as few chunks of at most C tiles as it needs, with one C for all entries, so that a long
// sequence among short ones is cut as finely as the whole asks for, and C such that all chunks are fewer than the workgroups that the
// chip holds at a time (a few more would run alone at the end).  C is on the large side: an entry counts as half a chunk more than its tiles
// over C, in the mean, and one tile is added for the rounding.  So the longest chunk is above an even share, and takes the more
// passes: one sequence of 2048 tiles for 64 workgroups makes 63 chunks of up to 33, 24 sequences of 1 to 250 tiles (24.2 a workgroup) 61 of
// up to 35, 256 entries of 9 to 33 tiles 497 of up to 13 for 512 workgroups (9.3 each).  Up to 64 entries a wavefront works this out by
// itself, more are divided among the threads of the workgroup.
struct Chunk { int e, tile0, tile1, index, count, slot0, told, first, n; };
struct Entry { int told, first, n, tiles; };
__device__ __forceinline__ Entry read_entry(const AttendArgs& a, int e) {
  const Pages& pg = a.pg;
  Entry o = {0, 0, 0, 0};
  if (e < a.entries) {
    const int s = a.per_head ? e / pg.Hkv : e, h = a.per_head ? e - s * pg.Hkv : 0;
    o.told = told_len(pg, s, h);
    const NewRows nr = new_rows(pg, s);
    o.first = nr.first;
    o.n = nr.n;
    if (o.n) o.tiles = (min(o.told, pg.max_len) + ATT_TILE - 1) / ATT_TILE;
  }
  return o;
}
// Tiles of a chunk, from the tiles of all entries and how many entries have any: at least total / chunks, which the scratch is
// sized for (hence the rounding up).
__device__ __forceinline__ int chunk_tiles(const AttendArgs& a, float total, int active) {
  const float want = total / fmaxf(a.chunks - 0.5f * active, 0.25f * a.chunks) * (1.f + 0x1p-20f) + 1.f;
  return want < (float)a.c_min ? a.c_min : want > 0x1p25f ? 1 << 25 : (int)want;
}
__device__ __forceinline__ Chunk chunk_of(const Entry& x, int e, int index, int count, int slot0) {
  const int each = count == 1 ? x.tiles : (x.tiles + count - 1) / count, t0 = min(index * each, x.tiles);
  return {e, t0, min(t0 + each, x.tiles), index, count, slot0, x.told, x.first, x.n};
}
template <int NW = 4>
__device__ __forceinline__ bool find_chunk(const AttendArgs& a, int x, int* lds, Chunk& o) {
  const int lane = threadIdx.x & 63;
  if (a.entries <= 64) {
    const Entry en = read_entry(a, lane);
    int C = chunk_tiles(a, (float)wave_sum((uint32_t)en.tiles), __popcll(__ballot(en.tiles > 0)));
    int cnt = 0, inc = 0;
    for (int i = 0; i < 8; ++i) {       // (until they are fewer than the resident workgroups: a few too many cost a sixth of the time of 24 lengths)
      cnt = lane < a.entries ? max(1, (en.tiles + C - 1) / C) : 0;
      inc = wave_scan(cnt);
      if (__builtin_amdgcn_readlane(inc, 63) <= a.chunks || a.entries >= a.chunks) break;
      C += C / 16 + 1;
    }
    const int own = cnt > 1 ? cnt : 0, sl = wave_scan(own);
    const unsigned long long hit = __ballot(inc > x);
    if (!hit) return false;
    const int l = __builtin_ctzll(hit);
    auto of = [&](int v) { return __builtin_amdgcn_readlane(v, l); };
    const int count = of(cnt);
    o = chunk_of({of(en.told), of(en.first), of(en.n), of(en.tiles)}, l, x - of(inc) + count, count, of(sl - own));
    return true;
  }
  const int tid = threadIdx.x, wv = tid >> 6;
  Entry en = read_entry(a, tid);
  int64_t tiles = en.tiles;
  int active = en.tiles > 0;
  for (int e = tid + 64 * NW; e < a.entries; e += 64 * NW) {
    const int t = read_entry(a, e).tiles;
    tiles += t;
    active += t > 0;
  }
  // (a sum of 64 tiles of up to 2^24 entries' positions each may pass 32 bits: as a float)
  float ft = (float)tiles;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) ft += __shfl_xor(ft, d);
  active = (int)wave_sum((uint32_t)active);
  if (lane == 0) {
    lds[wv] = __float_as_int(ft);
    lds[NW + wv] = active;
  }
  __syncthreads();
  float total = 0.f;
  active = 0;
#pragma unroll
  for (int w = 0; w < NW; ++w) {
    total += __int_as_float(lds[w]);
    active += lds[NW + w];
  }
  const int C = chunk_tiles(a, total, active);
  int* const at = lds + 4 * NW;         // the chunk, once found
  int run = 0, slots = 0;
  for (int base = 0; base < a.entries; base += 64 * NW) {
    const int e = base + tid;
    if (base) en = read_entry(a, e);
    const int cnt = e < a.entries ? max(1, (en.tiles + C - 1) / C) : 0, own = cnt > 1 ? cnt : 0;
    int inc = wave_scan(cnt), sl = wave_scan(own);
    if (lane == 63) {
      lds[2 * NW + wv] = inc;
      lds[3 * NW + wv] = sl;
    }
    if (tid == 0) at[0] = -1;
    __syncthreads();
    int all = 0, all_slots = 0;
#pragma unroll
    for (int w = 0; w < NW; ++w) {
      if (w == wv) {
        inc += run + all;
        sl += slots + all_slots;
      }
      all += lds[2 * NW + w];
      all_slots += lds[3 * NW + w];
    }
    if (inc > x && inc - cnt <= x) {
      const Chunk c = chunk_of(en, e, x - inc + cnt, cnt, sl - own);
      at[0] = c.e; at[1] = c.tile0; at[2] = c.tile1; at[3] = c.index; at[4] = c.count; at[5] = c.slot0;
      at[6] = c.told; at[7] = c.first; at[8] = c.n;
    }
    run += all;
    slots += all_slots;
    __syncthreads();
    const bool found = at[0] >= 0;
    if (found) o = {at[0], at[1], at[2], at[3], at[4], at[5], at[6], at[7], at[8]};
    __syncthreads();                  // (the scratch is used for other things from here on, or for the next entries)
    if (found) return true;
  }
  return false;
}

// Over the four lanes (l, l ^ 16, l ^ 32, l ^ 48) that hold one row
__device__ __forceinline__ float quad_max(float x) {
  auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  x = fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
  r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float quad_sum(float x) {
  auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  x = __uint_as_float(r[0]) + __uint_as_float(r[1]);
  r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

__device__ __forceinline__ f32x4 mfma(uint4 a, uint4 b, f32x4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_bf16x8(a), as_bf16x8(b), c, 0, 0, 0);
}

// n consecutive channels of a query row as float32
template <typename T, int N>
__device__ __forceinline__ void load_row(const T* p, bool vec, float (&x)[N]) {
  if (vec) {
    constexpr int W = N * sizeof(T) / 16;
    uint4 r[W];
#pragma unroll
    for (int i = 0; i < W; ++i) r[i] = ((const uint4*)p)[i];
#pragma unroll
    for (int i = 0; i < N; ++i) {
      if constexpr (sizeof(T) == 4) {
        x[i] = __uint_as_float(((const uint32_t*)r)[i]);
      } else {
        const uint32_t w = ((const uint32_t*)r)[i / 2];
        x[i] = __uint_as_float(i & 1 ? w & 0xFFFF0000u : w << 16);
      }
    }
  } else {
#pragma unroll
    for (int i = 0; i < N; ++i) x[i] = to_float(p[i]);
  }
}

// Four channels of a row of the output from its sums, and its log-sum-exp.
__device__ __forceinline__ void store_out(const AttendArgs& a, int64_t t, int64_t head, int c, float4 x, float M, float L) {
  const Pages& pg = a.pg;
  const float f = L == 0.f ? 0.f : 1.f / L;
  x.x *= f; x.y *= f; x.z *= f; x.w *= f;
  if (L == 0.f) x = make_float4(0.f, 0.f, 0.f, 0.f);
  const int64_t at = t * pg.o_st + head * pg.o_sh + c;
  if (pg.out_dtype == RESTKV_F32) {
    float* o = (float*)a.out + at;
    if (a.vec_out) {
      *(float4*)o = x;
    } else {
      o[0] = x.x; o[1] = x.y; o[2] = x.z; o[3] = x.w;
    }
  } else {
    uint16_t* o = (uint16_t*)a.out + at;
    const uint32_t lo = __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{x.x, x.y}, bf16x2));
    const uint32_t hi = __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{x.z, x.w}, bf16x2));
    if (a.vec_out) {
      *(uint2*)o = make_uint2(lo, hi);
    } else {
      o[0] = (uint16_t)lo; o[1] = (uint16_t)(lo >> 16); o[2] = (uint16_t)hi; o[3] = (uint16_t)(hi >> 16);
    }
  }
  if (c == 0 && a.lse) a.lse[t * pg.lse_st + head * pg.lse_sh] = L == 0.f ? -INFINITY : (M + __builtin_amdgcn_logf(L)) * 0.693147180559945309f;
}

// Sums of a row's chunks joined into its output: a workgroup a row (new token, query head), 256 threads as 1024 / d
// groups that take every so manyeth chunk, four channels a thread.  A chain of two reads (where the chunks are, what they
// hold) and a launch: chunks are read four at a time, references with the sums.  3.6 to 5 us for decoding steps, 8.3 for the 33 MB of
// 256 queries a KV head.
struct Part { const float *m, *l, *o; };
struct Sums {
  float M = -INFINITY, L = 0.f;
  float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
  __device__ __forceinline__ void take(float m, float l, float4 y) {
    // (a chunk of which the row sees nothing has a reference of -inf and sums of 0)
    const float n = fmaxf(M, m);
    const float fo = M == n ? 1.f : __builtin_amdgcn_exp2f(M - n), fn = m == n ? 1.f : __builtin_amdgcn_exp2f(m - n);
    M = n;
    L = L * fo + l * fn;
    x.x = x.x * fo + y.x * fn; x.y = x.y * fo + y.y * fn; x.z = x.z * fo + y.z * fn; x.w = x.w * fo + y.w * fn;
  }
};
// Channels c to c + 3 of every `step`-th chunk from the first'th on, four chunks at a time.
template <typename F>
__device__ __forceinline__ Sums sum_chunks(int first, int step, int count, int c, F part) {
  constexpr int AHEAD = 4;
  Sums s;
  for (int k = first; k < count; k += step * AHEAD) {
    float m[AHEAD], l[AHEAD];
    float4 y[AHEAD];
#pragma unroll
    for (int u = 0; u < AHEAD; ++u) {
      const Part p = part(min(k + u * step, count - 1));
      m[u] = *p.m;
      l[u] = *p.l;
      y[u] = *(const float4*)(p.o + c);
    }
#pragma unroll
    for (int u = 0; u < AHEAD; ++u)
      if (k + u * step < count) s.take(m[u], l[u], y[u]);
  }
  return s;
}
template <int D, typename F>
__device__ __forceinline__ void join_chunks(const AttendArgs& a, int count, int64_t t, int head, F part) {
  constexpr int TPR = D / 4, NGR = 256 / TPR;
  __shared__ float4 sm_x[NGR][TPR];
  __shared__ float sm_m[NGR], sm_l[NGR];
  const int g = threadIdx.x / TPR, c = threadIdx.x % TPR;
  Sums s = sum_chunks(g, NGR, count, c * 4, part);
  sm_x[g][c] = s.x;
  if (c == 0) {
    sm_m[g] = s.M;
    sm_l[g] = s.L;
  }
  __syncthreads();
  if (g) return;
#pragma unroll
  for (int k = 1; k < NGR; ++k) s.take(sm_m[k], sm_l[k], sm_x[k][c]);
  store_out(a, t, head, c * 4, s.x, s.M, s.L);
}

enum { FMT_F32, FMT_BF16, FMT_Q4 };

// N words at a uniform address (held in scalar registers, so that the load adds the lane's 32-bit offset by itself).
template <int N, bool PAST = false>
__device__ __forceinline__ Words<N> load_words(const char* base, uint32_t off) {
  uint64_t u = (uint64_t)__builtin_amdgcn_readfirstlane((uint32_t)((uint64_t)base >> 32)) << 32 |
               (uint32_t)__builtin_amdgcn_readfirstlane((uint32_t)(uint64_t)base);
  asm("" : "+s"(u), "+v"(off));      // (the offset's extension stays beside the load)
  typedef const __attribute__((address_space(1))) char* global;
  if constexpr (PAST) return __builtin_nontemporal_load((const __attribute__((address_space(1))) Words<N>*)((global)u + off));
  else return *(const __attribute__((address_space(1))) Words<N>*)((global)u + off);
}
// A weight's three parts by cutting off the mantissa (8 bits each: exact), in two plain instructions a part: in a loop that the
// vector pipe bounds those of split8, one each, are slower (a window of 64 positions over 32k keys 89.9 -> 87.3 us).  Two
// parts are rounded, for the ninth bit.
template <int NP>
__device__ __forceinline__ Op<NP> weight_parts(const float (&x)[8]) {
  if constexpr (NP != 3) return split8<NP>(x);
  Op<NP> o;
  uint32_t w[NP][4];
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    float a = x[2 * e], b = x[2 * e + 1];
#pragma unroll
    for (int p = 0; p < NP; ++p) {
      w[p][e] = __builtin_amdgcn_perm(__float_as_uint(b), __float_as_uint(a), 0x07060302u);
      if (p + 1 < NP) {
        a -= __uint_as_float(__float_as_uint(a) & 0xFFFF0000u);
        b -= __uint_as_float(__float_as_uint(b) & 0xFFFF0000u);
      }
    }
  }
#pragma unroll
  for (int p = 0; p < NP; ++p) o.p[p] = make_uint4(w[p][0], w[p][1], w[p][2], w[p][3]);
  return o;
}
// NP parts of four weights, as split8 makes them of eight
template <int NP>
__device__ __forceinline__ void split4(const float (&x)[4], Words<2> (&o)[NP]) {
  const float y[8] = {x[0], x[1], x[2], x[3], 0.f, 0.f, 0.f, 0.f};
  const Op<NP> p = split8<NP>(y);
#pragma unroll
  for (int i = 0; i < NP; ++i) o[i] = Words<2>{p.p[i].x, p.p[i].y};
}

__device__ __forceinline__ uint32_t load_half(const char* base, uint32_t off) {
  uint64_t u = (uint64_t)__builtin_amdgcn_readfirstlane((uint32_t)((uint64_t)base >> 32)) << 32 |
               (uint32_t)__builtin_amdgcn_readfirstlane((uint32_t)(uint64_t)base);
  asm("" : "+s"(u), "+v"(off));
  typedef const __attribute__((address_space(1))) char* global;
  return *(const __attribute__((address_space(1))) uint16_t*)((global)u + off);
}

// A copy in a vector register, so that what it is made of stays in scalar ones.
__device__ __forceinline__ uint32_t vector(uint32_t x) {
  uint32_t y;
  asm("v_mov_b32 %0, %1" : "=v"(y) : "s"(__builtin_amdgcn_readfirstlane(x)));
  return y;
}
// Rare code works on copies that the compiler knows nothing of, so that none of it moves into the common path.
template <typename V, int N>
__device__ __forceinline__ void keep_here(V (&x)[N]) {
#pragma unroll
  for (int i = 0; i < N; ++i) asm volatile("" : "+v"(x[i]));
}
// Registers without a value from here on (where a load is left out, so that the old values need not be kept for it).
template <typename V, int N>
__device__ __forceinline__ void forget(V (&x)[N]) {
#pragma unroll
  for (int i = 0; i < N; ++i) asm("" : "=v"(x[i]));
}

// Nibble i of each half word as the bfloat16 16 + code: the code goes to the upper four of its seven mantissa bits.
__device__ __forceinline__ uint32_t sixteen_plus(uint32_t x, int i, uint32_t mask, uint32_t base) {
  return ((i == 0 ? x << 3 : x >> (4 * i - 3)) & mask) | base;
}

// The same as code - 8, for float32 output: its sums stay as small as what they stand for, where those of 16 + code are several
// times as large (error of the output over 75 to 120 positions against 64 bits 2e-6 -> 1.5e-7 of its norm, time over 32k
// positions in float32 27.8 -> 32.6 us).
template <bool CENTRED>
__device__ __forceinline__ uint32_t code_pair(uint32_t x, int i, uint32_t mask, uint32_t base) {
  const uint32_t w = sixteen_plus(x, i, mask, base);
  if constexpr (!CENTRED) return w;
  return __builtin_amdgcn_perm(__float_as_uint(__uint_as_float(w & 0xFFFF0000u) - 24.f), __float_as_uint(__uint_as_float(w << 16) - 24.f), 0x07060302u);
}

// Row of the token tensors for place `tok` of a group's new tokens, max_new for each beam from sequence s on (places that a beam does not
// have hold another's; nobody reads what comes of them).
__device__ __forceinline__ int front_token(const Pages& pg, int s, int tok) {
  const int b = tok / pg.max_new;
  const NewRows of = new_rows(pg, s + b);
  return min(of.first + min(tok - b * pg.max_new, max(of.n - 1, 0)), pg.n_tokens - 1);
}

// How a workgroup of a launch for beams comes by its work: parts cut evenly, one after the other, or one of a list.
enum { NO_BEAMS, BEAMS_PARTS, BEAMS_LIST };
struct BeamsWork {
  unsigned long long todo;       // parts (spread), or one
  int (*lds)[8];                 // of a part: positions, first row, new tokens, first and last tile of this workgroup (spread)
  int u, hy, team_rb, slot0;
};
// Parts (up to 64, a lane each; a front with all its blocks of rows is one) cut evenly: the rounds of all follow each other, with
// a.part_cost half rounds more for each part, which is what its beginning and end take.  Workgroups come in teams of front_blocks.  Some
// teams take the fronts, one front each and all about as many rounds, each of a team's workgroups the same tiles for a block of rows
// (at the same time on one XCD, whose L2 reads them once); the workgroups of the other teams cut what is left, one by one.  A round is
// what the wavefronts of a workgroup take at a time, a.c_min tiles.
// (What comes of it is in LDS, so that the loops between have the registers.)
// Quotients of small whole numbers (below 2^15), where a division of 32 bits would take forty instructions.
__device__ __forceinline__ int quotient(int x, float one_over) { return (int)(((float)x + 0.5f) * one_over); }
__device__ __forceinline__ bool cut_parts(const AttendArgs& a, BeamsWork& o) {
  const Pages& pg = a.pg;
  const int lane = threadIdx.x & 63, all_fronts = a.fronts * a.front_blocks;
  const int id = unit_of_block();
  if (id >= a.units) return false;
  const int rb = blockIdx.x >> 3;
  o.u = __builtin_amdgcn_readfirstlane(quotient(id, __builtin_amdgcn_rcpf((float)a.Hy)));
  const int hy = o.hy = id - o.u * a.Hy;
  __shared__ int s_parts[64][8];
  o.lds = s_parts;
  o.team_rb = rb;
  // lane = sequence (and head) first, then a part: what each sequence has in front of its new tokens, the least of each group
  const int owns = a.entries - a.fronts, parts = a.fronts + owns * a.own_blocks;
  const float one_beams = __builtin_amdgcn_rcpf((float)a.n_beams), one_heads = __builtin_amdgcn_rcpf((float)pg.Hkv);
  const int y = min(lane, owns - 1), s = a.per_head ? quotient(y, one_heads) : y;
  const int told = told_len(pg, s, a.per_head ? y - s * pg.Hkv : 0);
  const NewRows nr = new_rows(pg, s);
  const int want = max(a.shared[quotient(s, one_beams)], 0), room = !nr.n ? -1 : pg.causal ? max(told - nr.n, 0) : told;
  const bool is_front = lane < a.fronts;
  const int x = is_front ? lane : min(quotient(lane - a.fronts, __builtin_amdgcn_rcpf((float)a.own_blocks)), owns - 1);
  // first sequence (and head) of the part's group
  const int step = a.per_head ? pg.Hkv : 1, of = a.per_head ? quotient(x, one_heads) : x, h = x - of * step;
  const int group = is_front ? of : quotient(of, one_beams);
  const int seq0 = group * a.n_beams * step + h;
  int least = 0x7FFFFFFF;
#pragma unroll 4
  for (int b = 0; b < a.n_beams; ++b) {
    const int r = __shfl(room, seq0 + b * step);
    least = r >= 0 ? min(least, r) : least;
  }
  const int shared = (int)min((int64_t)__shfl(want, seq0) << pg.lg_ps, (int64_t)pg.max_len);
  const int tiles = least == 0x7FFFFFFF ? 0 : min(shared, least) / ATT_TILE;
  const int own = is_front ? 0 : x, t = __shfl(told, own), first = __shfl(nr.first, own), n = __shfl(nr.n, own);
  Entry en = {0, 0, 0, 0};
  if (lane < parts) {
    if (is_front) en = {tiles * ATT_TILE, 0, a.n_beams * pg.max_new, tiles};
    else en = {t, first, n, n ? (min(t, pg.max_len) + ATT_TILE - 1) / ATT_TILE - tiles : 0};
  }
  const int tile0 = is_front ? 0 : tiles;
  // (fronts of many rows go by tiles; of very long caches 2^coarse rounds are one)
  const uint32_t team = a.front_blocks, per = (uint32_t)(is_front ? a.front_tiles : a.c_min) << a.coarse;
  const uint32_t rounds = ((uint32_t)en.tiles + per - 1) / per, cost = rounds ? 2 * rounds + a.part_cost : 0;
  const uint32_t upto = (uint32_t)wave_scan((int)cost), all = __builtin_amdgcn_readlane(upto, 63);
  const uint32_t of_fronts = __builtin_amdgcn_readlane(upto, a.fronts - 1), of_own = all - of_fronts;
  // teams for fronts: as many as their cost asks for, and one each at least
  const uint32_t used = __popcll(__ballot(is_front && rounds > 0)), least_teams = used + (of_own > 0);
  const float weight = (float)of_fronts * team, every = weight + (float)of_own;      // (half rounds of all workgroups)
  const uint32_t teams = max(least_teams, (uint32_t)fminf(a.chunks, every * __builtin_amdgcn_rcpf((float)((a.part_cost + 2u) * team))));
  const float due = (float)teams * weight * __builtin_amdgcn_rcpf(fmaxf(every, 1.f));
  const uint32_t most = min(max((uint32_t)(due + 0.5f), used), teams - (of_own > 0 ? 1u : 0u));
  // the fewest rounds a team (sixteenths of them) for which those are enough
  const uint32_t of_front = is_front ? rounds : 0, all_rounds = wave_sum(of_front);
  uint32_t n_teams, upto_teams, front_teams;
  for (float each = fmaxf(1.f, 16.f * (float)all_rounds * __builtin_amdgcn_rcpf((float)max(most, 1u)));; each += each * 0.0625f + 1.f) {
    n_teams = min((uint32_t)(fmaxf(16.f * (float)of_front - 0.5f, 0.f) * __builtin_amdgcn_rcpf(each)) + (of_front > 0), of_front);
    upto_teams = (uint32_t)wave_scan((int)n_teams);
    front_teams = __builtin_amdgcn_readlane(upto_teams, 63);
    if (front_teams <= most) break;
  }
  if ((uint32_t)o.u >= max(teams, 1u)) return false;
  const bool at_fronts = (uint32_t)o.u < front_teams;
  uint32_t u = at_fronts ? o.u : (o.u - front_teams) * team + rb;
  int seg0 = 0, seg1 = 0;
  if (at_fronts) {
    // Of two workgroups of a compute unit the one that came first is served first, and ends first (4 bits: five rounds 23 us, then
    // 25 us): so it takes more.  Teams in the order first, second, first, .., then those whose second is no front's.
    const uint32_t firsts = (teams + 1) / 2, seconds = front_teams > firsts ? front_teams - firsts : 0;
    u = u >= firsts ? 2 * (u - firsts) + 1 : u < seconds ? 2 * u : u + seconds;
    auto upto_team = [&](uint32_t x) {
      return x < 2 * seconds ? (float)x + (x & 1 ? a.first_more : 0.f) : (float)x + (float)(x - 2 * seconds) * (seconds ? a.first_more : 0.f);
    };
    const uint32_t from = upto_teams - n_teams, i = u - from;
    if (is_front && i < n_teams) {
      const float base = upto_team(from), unit = (float)rounds * __builtin_amdgcn_rcpf(upto_team(from + n_teams) - base);
      // (of few rounds each takes as many, so that none is without)
      auto cut = [&](uint32_t k) {
        return k == n_teams ? rounds : rounds < 2 * n_teams ? (uint32_t)(((float)(k * rounds) + 0.5f) * __builtin_amdgcn_rcpf((float)n_teams)) : (uint32_t)((upto_team(from + k) - base) * unit);
      };
      seg0 = (int)min(cut(i) * per, (uint32_t)en.tiles);
      seg1 = (int)min(cut(i + 1) * per, (uint32_t)en.tiles);
    }
  } else if (!is_front && of_own) {
    // (a share of two half rounds at least: no workgroup between others of a part is without a tile of it)
    const uint32_t groups = max(1u, min((teams - front_teams) * team, of_own / 2)), q = of_own / groups, r = of_own % groups;
    const uint32_t at = u * q + min(u, r), end = at + q + (u < r ? 1 : 0), ends = upto - of_fronts, begins = ends - cost + a.part_cost;
    auto tile_of = [&](uint32_t c) { return c >= ends ? en.tiles : c <= begins ? 0 : (int)min((c - begins) / 2 * per, (uint32_t)en.tiles); };
    seg0 = tile_of(at);
    seg1 = tile_of(end);
  }
  const bool some = seg1 > seg0;
  o.todo = __ballot(some);
  o.slot0 = u + (at_fronts ? rb * a.front_slots : 0);
  if (hy == 0 && threadIdx.x < 64 && lane < parts) {
    int2* const plan = a.plan + (is_front ? lane * a.front_blocks + rb : all_fronts + lane - a.fronts);
    if (some && seg0 == 0) plan->x = o.slot0 + lane;
    if (some && seg1 == en.tiles) plan->y = o.slot0 + lane;
    if (o.u == 0 && en.tiles == 0 && (is_front || rb == 0)) *plan = make_int2(1, 0);
  }
  if (threadIdx.x < 64) {
    *(int4*)s_parts[lane] = make_int4(en.told, en.first, en.n, tile0 + seg0);
    s_parts[lane][4] = tile0 + seg1;
  }
  __syncthreads();
  return true;
}
// The next part: its chunk, whether it is a front, and the slot of its sums.
__device__ __forceinline__ void next_part(const AttendArgs& a, BeamsWork& o, Chunk& ch, int& rb, bool& front, int& slot) {
  const int l = __builtin_ctzll(o.todo);
  front = l < a.fronts;
  const int* p = o.lds[l];
  ch = {front ? l : a.fronts + (l - a.fronts) / a.own_blocks, p[3], p[4], 0, 0, 0, p[0], p[1], p[2]};
  slot = o.slot0 + l;
  rb = front ? o.team_rb : (l - a.fronts) % a.own_blocks;
  o.todo &= o.todo - 1;
}
// Of a workgroup in a launch by a list: the same, the head, and whether there is anything.
__device__ __forceinline__ bool listed_part(const AttendArgs& a, int& hy, Chunk& ch, int& rb, bool& front, int& slot) {
  const int id = unit_of_block();
  if (id >= a.units) return false;
  // blocks of eight units, all row blocks of theirs after each other (so on one XCD)
  const int front_ids = (a.front_chunks * a.Hy + 7) / 8 * 8 * a.front_blocks;
  front = id < front_ids;
  const int x = front ? id : id - front_ids, blocks = front ? a.front_blocks : a.own_blocks, eight = x / (8 * blocks);
  const int unit = eight * 8 + (x & 7), u = unit / a.Hy, at = front ? u : u + a.front_chunks;
  if (u >= (front ? a.front_chunks : a.own_chunks)) return false;
  const int4 p = a.list[2 * at], q = a.list[2 * at + 1];
  if (p.x < 0) return false;
  hy = unit - u * a.Hy;
  ch = {p.x, p.y, p.z, 0, 0, 0, q.x, q.y, q.z};
  rb = (x - eight * 8 * blocks) >> 3;
  slot = p.w + (front ? rb * a.front_slots : 0);
  return true;
}

// FMT: pages; T: queries; R: blocks of 16 rows of a wavefront; NP: bf16 parts of a softmax weight (products with float32 pages take
// the weight itself).  Three hold all its bits, for float32 output.  bf16 output has two, 2^-17 beside the 2^-8 of its own rounding: 0.2 % of
// its values (4 bits, 16 + code in place of the code: 1.5 %) are not the nearest bf16 but its neighbour, where sums in float32 leave 0.03 to 0.2 %,
// and the error against 64 bits is the same, 1.7e-3 of the norm.  Three parts there take up to 2 % more time with few rows of bf16 pages, 12 % with
// many, 3 to 15 % with 4 bits (and leave 0.8 %), centred codes 28 to 45 % (0.2 %).
// Of a tile the keys are loaded anew (for the next one) as soon as the logits are there, the
// values as soon as they are in the sums: a load has the other half's arithmetic, and other wavefronts', to come back,
// and costs no second set of registers.
// SP (4-bit pages, up to 16 / SP rows): the sixteen columns are SP copies of the rows, and copy x takes the 16-key blocks x,
// SP + x, ...: its queries are zeros in the products of other blocks, which add up in one set of registers, and its weights
// are zeros in those blocks' products with values.  The matrix pipe does as much as before, but a lane scales, exponentiates
// and splits 1 / SP of the keys, which is what bounds this format: four rows, 128k tokens 47.7 -> 39.2 us.
template <int FMT, typename T, int D, int NP, int R, int SP, int BEAMS>
__global__ __attribute__((amdgpu_flat_work_group_size(256, 256), amdgpu_waves_per_eu(2)))
void k_attend(AttendArgs a) {
  extern __shared__ __align__(16) float sm[];
  const int unit = unit_of_block();
  int rb = blockIdx.x >> 3, slot = 0;
  if (!BEAMS && unit >= a.units) return;
  int hy = BEAMS ? 0 : unit % a.Hy;
  bool front = false;
  Chunk ch;
  BeamsWork work;
  if constexpr (BEAMS == BEAMS_PARTS) {
    if (!cut_parts(a, work)) return;
    hy = work.hy;
  } else if constexpr (BEAMS == BEAMS_LIST) {
    if (!listed_part(a, hy, ch, rb, front, slot)) return;
  } else {
    if (!find_chunk(a, unit / a.Hy, (int*)sm, ch)) return;
  }
  do {
    if constexpr (BEAMS == BEAMS_PARTS) {
      if (!work.todo) return;
      next_part(a, work, ch, rb, front, slot);
    }
#include "attend_chunk.inc"
    if (BEAMS == BEAMS_PARTS) __syncthreads();          // (the sums of this part are read, before the next one's scales or sums come there)
  } while (BEAMS == BEAMS_PARTS);
}

// A chunk of what a beam has behind the shared positions, in a kernel that does other things too.
template <int FMT, typename T, int D, int NP, int R, int SP, int BEAMS>
__device__ __forceinline__ void attend_own(const AttendArgs& a, const Chunk& ch, int hy, int rb, int slot, float* sm) {
  constexpr bool front = false;
  do {
#include "attend_chunk.inc"
  } while (false);
}

template <int FMT, typename T, int D, int NP, int R, int SP = 1, int BEAMS = 0>
int run_attend(const AttendArgs& a, hipStream_t st) {
  constexpr size_t join = (8 * 16 * R + (size_t)4 * 16 * R * (D + 4)) * 4, scales = FMT == FMT_Q4 ? 4 * 4 * 64 * (D / 32) * 4 : 0;
  constexpr size_t lds = join > scales ? join : scales;
  auto kern = k_attend<FMT, T, D, NP, R, SP, BEAMS>;
  if constexpr (lds > 65536) {
    if (hipFuncSetAttribute((const void*)kern, hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds) != hipSuccess) return RESTKV_EHIP;
  }
  hipLaunchKernelGGL(kern, unit_grid(a), dim3(256), lds, st, a);
  return hip_status();
}

template <int FMT, typename T, int D, int NP, int R>
int run_attend_beams(const AttendArgs& a, hipStream_t st) {
  return a.spread ? run_attend<FMT, T, D, NP, R, 1, BEAMS_PARTS>(a, st) : run_attend<FMT, T, D, NP, R, 1, BEAMS_LIST>(a, st);
}

// by format, and for many rows (attend_*.hip); for beams (attend_beams_*.hip)
int run_attend_rows(const AttendArgs& a, int R, int waves, hipStream_t st);
int run_attend_f32(const AttendArgs& a, int R, hipStream_t st);
int run_attend_bf16(const AttendArgs& a, hipStream_t st);
int run_attend_q4(const AttendArgs& a, int R, hipStream_t st);
int run_attend_beams_f32(const AttendArgs& a, hipStream_t st);
int run_attend_beams_bf16(const AttendArgs& a, int R, hipStream_t st);
int run_attend_beams_q4(const AttendArgs& a, hipStream_t st);
int run_attend_beams_rows(const AttendArgs& a, hipStream_t st);
// What kernels and join share of the arguments.
AttendArgs attend_args(const Pages& pg, const void* q, const void* k_pages, const void* v_pages, const void* k_scale,
                       const void* v_scale, void* out, float* lse);

}  // namespace restkv
