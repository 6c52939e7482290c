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
template <int FMT, typename T, int D, int NP, int R, int SP>
__global__ __attribute__((amdgpu_flat_work_group_size(256, 256), amdgpu_waves_per_eu(2)))
void k_attend(AttendArgs a) {
  constexpr int UN = D / 16, NG = D / 32;
  constexpr int QP = FMT == FMT_Q4 ? planes_of<T> : 1;
  constexpr int TK = FMT == FMT_F32 ? 16 : FMT == FMT_BF16 ? 32 : 64, NB = TK / 16;
  constexpr int ROWB = FMT == FMT_F32 ? D * 4 : FMT == FMT_BF16 ? D * 2 : D / 2;
  constexpr bool CENTRED = NP == 3;
  constexpr float BASE = CENTRED ? 8.f : -16.f;    // of a code, from its operand
  constexpr int CW = 16 / SP, NBS = NB / SP;       // columns of a copy, blocks of a copy
  constexpr int LDO = D + 4, QC = FMT == FMT_F32 ? D / 16 : D / 32;
  extern __shared__ __align__(16) float sm[];
  const Pages& pg = a.pg;
  const int lane = threadIdx.x & 63, n = lane & 15, j = lane >> 4, copy = SP > 1 ? n / CW : 0;
  const int wv = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);

  const int unit = unit_of_block(), rb = blockIdx.x >> 3;
  if (unit >= a.units) return;
  const int hy = unit % a.Hy;
  Chunk ch;
  if (!find_chunk(a, unit / a.Hy, (int*)sm, ch)) return;
  const int e = __builtin_amdgcn_readfirstlane(ch.e);
  const int s = a.per_head ? e / pg.Hkv : e, h = a.per_head ? e - s * pg.Hkv : hy;
  const NewRows nr = {__builtin_amdgcn_readfirstlane(ch.first), __builtin_amdgcn_readfirstlane(ch.n)};
  const int rows = pg.G * nr.n, row0 = rb * 16 * R;
  if (row0 >= rows) return;
  if (a.plan && ch.index == 0 && hy == 0 && rb == 0 && threadIdx.x == 0) a.plan[e] = make_int2(ch.slot0, ch.count);

  const int told = __builtin_amdgcn_readfirstlane(ch.told), len = min(told, pg.max_len);
  auto limit = [&](int row) {       // positions that a row sees
    return pg.causal ? min(max(told - nr.n + row / pg.G + 1, 0), len) : len;
  };
  const int last_row = min(row0 + 16 * R, rows) - 1;
  const int k_end = __builtin_amdgcn_readfirstlane(min(ch.tile1 * ATT_TILE, limit(last_row)));
  const int lim_lo = __builtin_amdgcn_readfirstlane(limit(row0));
  const int k_begin = __builtin_amdgcn_readfirstlane(ch.tile0 * ATT_TILE) + wv * TK;
  const float sc = pg.scale * 1.44269504088896341f;

  f32x4 o[UN][R];
  float ref[R], l[R], corr[FMT == FMT_Q4 ? R : 1][NG];
#pragma unroll
  for (int cb = 0; cb < R; ++cb) {
#pragma unroll
    for (int i = 0; i < UN; ++i) o[i][cb] = f32x4{0.f, 0.f, 0.f, 0.f};
    ref[cb] = -INFINITY;
    l[cb] = 0.f;
    if constexpr (FMT == FMT_Q4)
#pragma unroll
      for (int f = 0; f < NG; ++f) corr[cb][f] = 0.f;
  }
  // of this wavefront's tile: {step, zero} of the keys as they are [64][NG], their steps [NG][64], the values' steps and
  // zeros + BASE steps [NG][64] each (a read takes four keys of a group)
  uint32_t* s_kz = (uint32_t*)sm + wv * (4 * 64 * NG);
  float* s_ks = (float*)s_kz + 64 * NG;
  float* s_vs = s_ks + 64 * NG;
  float* s_vz = s_vs + 64 * NG;
  float* s_rare = sm + wv * (UN * 4 * R * 64);       // the sums, for a moment (float32 and bfloat16 pages)

  // ---- tiles: where the 16-key blocks are (each lies in one page)
  const int32_t* table = pg.table + s * pg.table_ss + h * pg.table_sh;
  const int64_t tokb = pg.tok_s * ROWB;
  const char* const kh = a.k + h * pg.head_s * ROWB;
  const char* const vh = a.v + h * pg.head_s * ROWB;
  struct Where { uint32_t row[NB]; int ok; };    // first rows, and a bit for each block that has a page
  auto find = [&](int k0) {
    Where w;
    w.ok = 0;
#pragma unroll
    for (int b = 0; b < NB; ++b) {
      const int t = k0 + 16 * b;
      const int page = uniform_load(table + (min(t, k_end - 1) >> pg.lg_ps));
      const bool ok = (uint32_t)page < (uint32_t)pg.n_pages && t < k_end;
      w.row[b] = ok ? (uint32_t)page * (uint32_t)pg.page_s + (t & ((1 << pg.lg_ps) - 1)) * (uint32_t)pg.tok_s : 0u;
      w.ok |= ok ? 1 << b : 0;
    }
    return w;
  };
  // lane offsets of a block: key n, part j of its row; value row 4 j + r, unit n
  const uint32_t k_off = (uint32_t)(n * tokb) + j * (FMT == FMT_Q4 ? UN * 2 : 16);
  const uint32_t v_off = (uint32_t)(4 * j * tokb) + n * (ROWB / 16);
  constexpr int KV = FMT == FMT_Q4 ? UN / 2 : 4, KN = FMT == FMT_Q4 ? 1 : QC;      // words of a load, loads of a lane per block
  constexpr int VV = FMT == FMT_F32 ? 4 : FMT == FMT_BF16 ? UN / 2 : 1, VN = FMT == FMT_F32 ? UN / 4 : 1;
  Words<KV> kr[NB * KN];
  Words<VV> vr[NB * 4 * VN];
  Words<NG> sk[1], sv[1];
  // (Whole lines go past the caches, and leave them to the loads that take a line in parts: values of bf16 pages, whose keys come
  // half a line of sixteen rows at a time, 1 x 128k positions 99.6 -> 90.4 us a call, 32 sequences of 1k to 2k 38.9 -> 34.1;
  // keys of 4-bit pages, 128k positions 43.5 -> 41.2.  All loads so: 89.6, 37.4 and 40.8, f32 pages 47.4 -> 58.0.)
  auto load_keys = [&](const Where& w) {
#pragma unroll
    for (int b = 0; b < NB; ++b)
#pragma unroll
      for (int c = 0; c < KN; ++c) kr[b * KN + c] = load_words<KV, FMT == FMT_Q4>(kh + (uint64_t)w.row[b] * ROWB, k_off + c * 64);
  };
  auto load_values = [&](const Where& w) {
#pragma unroll
    for (int b = 0; b < NB; ++b)
#pragma unroll
      for (int r = 0; r < 4; ++r)
#pragma unroll
        for (int c = 0; c < VN; ++c) {
          const char* p = vh + ((uint64_t)w.row[b] * ROWB + r * tokb);
          if constexpr (FMT == FMT_Q4 && UN == 4) vr[b * 4 + r] = load_half(p, v_off);
          else vr[(b * 4 + r) * VN + c] = load_words<VV, FMT == FMT_BF16>(p, v_off + c * 16);
        }
  };
  auto scales_of = [&](const Where& w, const uint32_t* from) {       // lane = key of the tile
    uint32_t row0 = vector(w.row[0]);
#pragma unroll
    for (int b = 1; b < NB; ++b) row0 = j == b ? vector(w.row[b]) : row0;
    const uint64_t row = (row0 + (uint64_t)(h * pg.head_s + n * pg.tok_s)) * NG;
    return *(const Words<NG>*)(from + row);
  };
  auto load_scales = [&](const Where& w) {
    sk[0] = scales_of(w, a.ks);
    sv[0] = scales_of(w, a.vs);
  };

  Where at;
  if (k_begin < k_end) {
    at = find(k_begin);
    load_keys(at);
    if constexpr (FMT == FMT_Q4) load_scales(at);
    load_values(at);
  }
  int lim[R];
  // queries, as operands
  float4 qf[FMT == FMT_F32 ? R : 1][FMT == FMT_F32 ? QC : 1];
  Op<QP> qo[FMT == FMT_F32 ? 1 : R][FMT == FMT_F32 ? 1 : QC];
  uint4 qz[FMT == FMT_Q4 ? R : 1];
  uint32_t mine[SP];                 // all bits in the lanes of copy x
#pragma unroll
  for (int cb = 0; cb < R; ++cb) {
    const int row = min(row0 + cb * 16 + (SP > 1 ? n % CW : n), rows - 1);
    lim[cb] = limit(row);
    const int tok = row / pg.G;
    const T* p = (const T*)a.q + (nr.first + tok) * pg.q_st + (h * pg.G + row - tok * pg.G) * pg.q_sh;
    if constexpr (FMT == FMT_F32) {
#pragma unroll
      for (int c = 0; c < QC; ++c) {
        float x[4];
        load_row<T, 4>(p + c * 16 + j * 4, a.vec_q, x);
        qf[cb][c] = make_float4(x[0], x[1], x[2], x[3]);
      }
    } else if constexpr (FMT == FMT_BF16) {
#pragma unroll
      for (int c = 0; c < QC; ++c) {
        float x[8];
        load_row<T, 8>(p + c * 32 + j * 8, a.vec_q, x);
        qo[cb][c] = split8<1>(x);
      }
    } else {
      float x[4 * UN], z[8];         // units 4j .. 4j+3
      load_row<T, 4 * UN>(p + j * 4 * UN, a.vec_q, x);
#pragma unroll
      for (int i = 0; i < 8; ++i) z[i] = 0.f;
#pragma unroll
      for (int f = 0; f < NG; ++f) {
        float y[8], t = 0.f;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          y[i] = x[(i & 3) * UN + 2 * f + (i >> 2)];
          t += y[i];
        }
        qo[cb][f] = split8<QP>(y);
        t = quad_sum(t);
        if (j == f) z[0] = t;        // lane j: the sum of the group j that its eight places of the zeros' product stand for
      }
      // (zero, zero, zero, step, step, step, 0, 0) of a key times the sum's three parts h, m, l and BASE times them
      const Op<3> zp = split8<3>(z);
      const uint32_t zh = zp.p[0].x & 0xFFFFu, zm = zp.p[1].x & 0xFFFFu, zl = zp.p[2].x & 0xFFFFu;
      auto times = [](uint32_t b) {  // BASE times a bfloat16
        return __float_as_uint(BASE * __uint_as_float(b << 16)) >> 16;
      };
      qz[cb] = make_uint4(zh | zm << 16, zl | times(zh) << 16, times(zm) | times(zl) << 16, 0u);
    }
  }

  auto only = [](uint4 x, uint32_t m) { return make_uint4(x.x & m, x.y & m, x.z & m, x.w & m); };
  uint4 qm[SP > 1 ? SP : 1][SP > 1 ? NG : 1], qzm[SP];
#pragma unroll
  for (int x = 0; x < SP; ++x) {
    mine[x] = copy == x ? ~0u : 0u;
    if constexpr (SP > 1) {
      static_assert(QP == 1 && R == 1, "");
#pragma unroll
      for (int f = 0; f < NG; ++f) qm[x][f] = only(qo[0][f].p[0], mine[x]);
      qzm[x] = only(qz[0], mine[x]);
    }
  }
  uint32_t nib_mask = 0x00780078u, nib_base = 0x41804180u;
  if constexpr (FMT == FMT_Q4) asm("" : "+s"(nib_mask), "+v"(nib_base));      // (one of two constants may be scalar)

  for (int k0 = k_begin; k0 < k_end; k0 += 4 * TK) {
    const Where next = find(k0 + 4 * TK);
    const bool more = k0 + 4 * TK < k_end;
    f32x4 p[NBS][R];
    const bool masked = k0 + TK > min(k_end, lim_lo) || at.ok != (1 << NB) - 1;
    auto there = [&](int b) { return at.ok >> b & 1 ? min(k_end - (k0 + 16 * b), 16) : 0; };
    // key 16 b + 4 j + r of the tile is in register r of p[bb], b = bb SP + the lane's copy
    auto seen = [&](int bb, int r, int cb) {
      const int b = bb * SP + copy;
      return 4 * j + r < there(b) && k0 + 16 * b + 4 * j + r < lim[cb];
    };
    bool odd_scales = false;
    unsigned long long odd_keys = 0;

    // ---- logits
    if constexpr (FMT == FMT_F32) {
#pragma unroll
      for (int cb = 0; cb < R; ++cb) p[0][cb] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int c = 0; c < QC; ++c)
#pragma unroll
        for (int cb = 0; cb < R; ++cb) {
          const float y[4] = {qf[cb][c].x, qf[cb][c].y, qf[cb][c].z, qf[cb][c].w};
#pragma unroll
          for (int i = 0; i < 4; ++i)
            p[0][cb] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(kr[c][i]), y[i], p[0][cb], 0, 0, 0);
        }
    } else if constexpr (FMT == FMT_BF16) {
#pragma unroll
      for (int b = 0; b < NB; ++b)
#pragma unroll
        for (int cb = 0; cb < R; ++cb) p[b][cb] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int c = 0; c < QC; ++c)
#pragma unroll
        for (int b = 0; b < NB; ++b)
#pragma unroll
          for (int cb = 0; cb < R; ++cb) p[b][cb] = mfma(__builtin_bit_cast(uint4, kr[b * KN + c]), qo[cb][c].p[0], p[b][cb]);
    } else {
      if (masked) {                  // keys without a finite scale: zeros here, and NaN for the rows that see them below
        bool bad = false;
#pragma unroll
        for (int f = 0; f < NG; ++f) {
          const float x = __uint_as_float(sk[0][f] << 16), y = __uint_as_float(sk[0][f] & 0xFFFF0000u);
          bad = bad || !(x - x == 0.f && y - y == 0.f);
        }
        odd_keys = __ballot(bad);
        if (bad) sk[0] = Words<NG>{};
      }
      __builtin_amdgcn_wave_barrier();
      *(Words<NG>*)&s_kz[lane * NG] = sk[0];
      if (masked) {
        // Zeros stand for the values' scales of slots that nobody sees, and of keys that some rows see wherever what the
        // weights are multiplied with (zero + BASE step; not finite for finite steps of 2^124 too) would make NaN of a weight of 0.
        if (n >= there(j)) sv[0] = Words<NG>{};
#pragma unroll
        for (int f = 0; f < NG; ++f) {
          const float z = __builtin_fmaf(BASE, __uint_as_float(sv[0][f] << 16), __uint_as_float(sv[0][f] & 0xFFFF0000u));
          if (!(z - z == 0.f)) {
            sv[0][f] = 0u;
            odd_scales = true;
          }
        }
      }
#pragma unroll
      for (int f = 0; f < NG; ++f) {
        const float st = __uint_as_float(sv[0][f] << 16);
        s_ks[f * 64 + lane] = __uint_as_float(sk[0][f] << 16);
        s_vs[f * 64 + lane] = st;
        s_vz[f * 64 + lane] = __builtin_fmaf(BASE, st, __uint_as_float(sv[0][f] & 0xFFFF0000u));
      }
      odd_scales = __ballot(odd_scales);
      if (more) load_scales(next);
      else {
        forget(sk);
        forget(sv);
      }
      __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
      __builtin_amdgcn_wave_barrier();
      f32x4 copies[NG];               // of all copies: sums of q (code - BASE) of their blocks
#pragma unroll
      for (int b = 0; b < NB; ++b) {
        // sum over the groups of zero * (sum of q) + BASE step * (sum of q), as one product: lane j the group j
        uint32_t zw = s_kz[(16 * b + n) * NG + (NG == 4 ? j : (j & 1))];
        if (NG == 2 && j > 1) zw = 0u;
        const uint4 za = make_uint4(__builtin_amdgcn_perm(zw, zw, 0x07060706u), __builtin_amdgcn_perm(zw, zw, 0x05040706u),
                                    __builtin_amdgcn_perm(zw, zw, 0x05040504u), 0u);
        uint4 op[NG];                 // code - BASE as bf16, group by group
#pragma unroll
        for (int f = 0; f < NG; ++f) {
          uint32_t lo, hi;            // the half words of units (0, 1) and (2, 3) that hold the group
          if constexpr (UN == 8) {
            const uint32_t sel = f < 2 ? 0x05040100u : 0x07060302u;
            lo = __builtin_amdgcn_perm(kr[b][1], kr[b][0], sel);
            hi = __builtin_amdgcn_perm(kr[b][3], kr[b][2], sel);
          } else {
            lo = kr[b][0];
            hi = kr[b][1];
          }
          const int e0 = (2 * f) & 3;
          op[f] = make_uint4(code_pair<CENTRED>(lo, e0, nib_mask, nib_base), code_pair<CENTRED>(hi, e0, nib_mask, nib_base),
                             code_pair<CENTRED>(lo, e0 + 1, nib_mask, nib_base), code_pair<CENTRED>(hi, e0 + 1, nib_mask, nib_base));
        }
        if constexpr (SP == 1) {
          f32x4 st[NG];               // steps of keys 4 j .. 4 j + 3
#pragma unroll
          for (int f = 0; f < NG; ++f) st[f] = *(const f32x4*)&s_ks[f * 64 + 16 * b + 4 * j];
#pragma unroll
          for (int cb = 0; cb < R; ++cb) {
            p[b][cb] = mfma(za, qz[cb], f32x4{0.f, 0.f, 0.f, 0.f});
            f32x4 t[NG];
#pragma unroll
            for (int f = 0; f < NG; ++f) {
              t[f] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
              for (int pl = 0; pl < QP; ++pl) t[f] = mfma(op[f], qo[cb][f].p[pl], t[f]);
            }
#pragma unroll
            for (int f = 0; f < NG; ++f)
#pragma unroll
              for (int r = 0; r < 4; ++r) p[b][cb][r] = __builtin_fmaf(st[f][r], t[f][r], p[b][cb][r]);
          }
          // (one block at a time, finished here: else its sums are put off past the next loads, with all they are made of in
          // registers)
#pragma unroll
          for (int cb = 0; cb < R; ++cb) asm volatile("" : "+v"(p[b][cb]));
        } else {
          const int x = b % SP, bb = b / SP;
          p[bb][0] = mfma(za, qzm[x], x ? p[bb][0] : f32x4{0.f, 0.f, 0.f, 0.f});
#pragma unroll
          for (int f = 0; f < NG; ++f) copies[f] = mfma(op[f], qm[x][f], x ? copies[f] : f32x4{0.f, 0.f, 0.f, 0.f});
          if (x == SP - 1)
#pragma unroll
            for (int f = 0; f < NG; ++f) {
              const f32x4 st = *(const f32x4*)&s_ks[f * 64 + 16 * (bb * SP + copy) + 4 * j];
#pragma unroll
              for (int r = 0; r < 4; ++r) p[bb][0][r] = __builtin_fmaf(st[r], copies[f][r], p[bb][0][r]);
            }
          asm volatile("" : "+v"(p[bb][0]));
#pragma unroll
          for (int f = 0; f < NG; ++f) asm volatile("" : "+v"(copies[f]));
        }
        __builtin_amdgcn_sched_barrier(0);
      }
    }
    if (more) load_keys(next);
    else forget(kr);

    // ---- softmax: lane = row
    if (masked) {
      if (FMT == FMT_Q4 && odd_keys) {
#pragma unroll
        for (int cb = 0; cb < R; ++cb)
#pragma unroll
          for (int b = 0; b < NBS; ++b)
#pragma unroll
            for (int r = 0; r < 4; ++r)
              if (odd_keys >> (16 * (b * SP + copy) + 4 * j + r) & 1) p[b][cb][r] = __builtin_nanf("");
      }
#pragma unroll
      for (int cb = 0; cb < R; ++cb)
#pragma unroll
        for (int b = 0; b < NBS; ++b)
#pragma unroll
          for (int r = 0; r < 4; ++r) p[b][cb][r] = seen(b, r, cb) ? p[b][cb][r] : -INFINITY;
    }
    bool far = false;
    float top[R];
#pragma unroll
    for (int cb = 0; cb < R; ++cb) {
      float m = -INFINITY;
#pragma unroll
      for (int b = 0; b < NBS; ++b)
#pragma unroll
        for (int r = 0; r < 4; ++r) m = fmaxf(m, p[b][cb][r]);
      top[cb] = quad_max(m) * sc;
      far = far || top[cb] > ref[cb] + 8.f;
    }
    // the reference follows the largest logit when it is 2^8 behind: rarely
    if (__builtin_expect(__ballot(far) != 0, 0)) {
#pragma unroll
      for (int cb = 0; cb < R; ++cb) {
        const float m = fmaxf(ref[cb], top[cb]);
        const float f = ref[cb] == m ? 1.f : __builtin_amdgcn_exp2f(ref[cb] - m);
        ref[cb] = m;
        l[cb] *= f;
#pragma unroll
        for (int i = 0; i < UN; ++i) o[i][cb] *= f;
        if constexpr (FMT == FMT_Q4)
#pragma unroll
          for (int g = 0; g < NG; ++g) corr[cb][g] *= f;
      }
    }
#pragma unroll
    for (int cb = 0; cb < R; ++cb) {
      const float m = ref[cb] == -INFINITY ? 0.f : ref[cb];
#pragma unroll
      for (int b = 0; b < NBS; ++b)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          p[b][cb][r] = __builtin_amdgcn_exp2f(__builtin_fmaf(p[b][cb][r], sc, -m));
          l[cb] += p[b][cb][r];
        }
    }

    // Values that are not finite, in a tile where some rows do not see every key (0 times them would be NaN): each is added to
    // the sums of the rows that see its key, with the sums in LDS (rare, so kept out of the registers); zeros then take their
    // places in the products.
    auto odd_values = [&]() {
#pragma unroll
      for (int cb = 0; cb < R; ++cb)
#pragma unroll
        for (int i = 0; i < UN; ++i)
#pragma unroll
          for (int r = 0; r < 4; ++r) s_rare[((cb * UN + i) * 4 + r) * 64 + lane] = o[i][cb][r];
#pragma unroll 1
      for (int kk = 0; kk < TK; ++kk) {
        const int b = kk >> 4;
        uint32_t row = at.row[0];
        int have = there(0);
#pragma unroll
        for (int x = 1; x < NB; ++x)
          if (b == x) { row = at.row[x]; have = there(x); }
        if ((kk & 15) >= have) continue;
        float w[R];
#pragma unroll
        for (int cb = 0; cb < R; ++cb) {
          w[cb] = p[0][cb][0];
#pragma unroll
          for (int x = 1; x < NB * 4; ++x) w[cb] = x == b * 4 + (kk & 3) ? p[x >> 2][cb][x & 3] : w[cb];
          w[cb] = __shfl(w[cb], n + 16 * (kk >> 2 & 3));      // the lane that holds the key's weight
        }
        const char* vp = vh + (uint64_t)row * ROWB + (kk & 15) * tokb;
#pragma unroll 1
        for (int i = 0; i < UN; ++i) {
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            const int ch = (4 * j + r) * UN + i;
            const float v = FMT == FMT_F32 ? ((const float*)vp)[ch] : __uint_as_float((uint32_t)((const uint16_t*)vp)[ch] << 16);
#pragma unroll
            for (int cb = 0; cb < R; ++cb)
              if (!(v - v == 0.f) && k0 + kk < lim[cb]) s_rare[((cb * UN + i) * 4 + r) * 64 + lane] += w[cb] * v;
          }
        }
      }
#pragma unroll
      for (int cb = 0; cb < R; ++cb)
#pragma unroll
        for (int i = 0; i < UN; ++i)
#pragma unroll
          for (int r = 0; r < 4; ++r) o[i][cb][r] = s_rare[((cb * UN + i) * 4 + r) * 64 + lane];
    };

    // ---- O^T += V^T P^T
    if constexpr (FMT == FMT_F32) {
      auto val = [&](int r, int i) { return __uint_as_float(vr[r * VN + i / 4][i & 3]); };
      if (__builtin_expect(masked, 0)) {
        keep_here(vr);
        bool bad = false;
#pragma unroll
        for (int r = 0; r < 4; ++r)
#pragma unroll
          for (int i = 0; i < UN; ++i) {
            if (4 * j + r >= there(0)) vr[r * VN + i / 4][i & 3] = 0u;
            bad = bad || !(val(r, i) - val(r, i) == 0.f);
          }
        if (__builtin_expect(__ballot(bad) != 0, 0)) {
          odd_values();
#pragma unroll
          for (int r = 0; r < 4; ++r)
#pragma unroll
            for (int i = 0; i < UN; ++i)
              if (!(val(r, i) - val(r, i) == 0.f)) vr[r * VN + i / 4][i & 3] = 0u;
        }
      }
#pragma unroll
      for (int r = 0; r < 4; ++r)
#pragma unroll
        for (int i = 0; i < UN; ++i)
#pragma unroll
          for (int cb = 0; cb < R; ++cb) o[i][cb] = __builtin_amdgcn_mfma_f32_16x16x4f32(val(r, i), p[0][cb][r], o[i][cb], 0, 0, 0);
    } else if constexpr (FMT == FMT_BF16) {
      // eight keys of a lane: registers r of both blocks
      Op<NP> po[R];
#pragma unroll
      for (int cb = 0; cb < R; ++cb) {
        const float x[8] = {p[0][cb][0], p[0][cb][1], p[0][cb][2], p[0][cb][3], p[1][cb][0], p[1][cb][1], p[1][cb][2], p[1][cb][3]};
        po[cb] = split8<NP>(x);
      }
      auto operand = [&](int i) {      // place i of every unit, keys 0 .. 7
        const uint32_t sel = i & 1 ? 0x07060302u : 0x05040100u;
        return make_uint4(__builtin_amdgcn_perm(vr[1][i / 2], vr[0][i / 2], sel), __builtin_amdgcn_perm(vr[3][i / 2], vr[2][i / 2], sel),
                          __builtin_amdgcn_perm(vr[5][i / 2], vr[4][i / 2], sel), __builtin_amdgcn_perm(vr[7][i / 2], vr[6][i / 2], sel));
      };
      if (__builtin_expect(masked, 0)) {
        keep_here(vr);
        bool bad = false;
#pragma unroll
        for (int x = 0; x < 8; ++x)
#pragma unroll
          for (int i = 0; i < UN / 2; ++i) {
            if (4 * j + (x & 3) >= there(x >> 2)) vr[x][i] = 0u;
            bad = bad || (vr[x][i] & 0x7F80u) == 0x7F80u || (vr[x][i] & 0x7F800000u) == 0x7F800000u;
          }
        if (__builtin_expect(__ballot(bad) != 0, 0)) {
          odd_values();
#pragma unroll
          for (int x = 0; x < 8; ++x)
#pragma unroll
            for (int i = 0; i < UN / 2; ++i) {
              const uint32_t w = vr[x][i];
              vr[x][i] = w & ~(((w & 0x7F80u) == 0x7F80u ? 0xFFFFu : 0u) | ((w & 0x7F800000u) == 0x7F800000u ? 0xFFFF0000u : 0u));
            }
        }
      }
      // (two places at a time, the parts of a weight in turn: products that add to the same sums do not follow each other)
#pragma unroll
      for (int i = 0; i < UN; i += 2) {
        const uint4 x[2] = {operand(i), operand(i + 1)};
#pragma unroll
        for (int pl = NP - 1; pl >= 0; --pl)
#pragma unroll
          for (int cb = 0; cb < R; ++cb)
#pragma unroll
            for (int y = 0; y < 2; ++y) o[i + y][cb] = mfma(x[y], po[cb].p[pl], o[i + y][cb]);
      }
    } else {
      if (__builtin_expect(masked && odd_scales, 0)) {
        // scales for which zeros stand, in a tile where some rows do not see every key: here the rows that see the key get
        // what it adds to their groups
        const Words<NG> raw = scales_of(at, a.vs);
#pragma unroll 1
        for (int kk = 0; kk < 64; ++kk) {
          const int b = kk >> 4, r = kk & 3;
#pragma unroll
          for (int f = 0; f < NG; ++f) {
            const uint32_t w = __builtin_amdgcn_readlane(raw[f], kk);
            const float step = __uint_as_float(w << 16), zero = __uint_as_float(w & 0xFFFF0000u);
            float z = __builtin_fmaf(BASE, step, zero);
            if (z - z == 0.f) continue;
            z = step - step == 0.f ? z : __builtin_nanf("");
#pragma unroll
            for (int cb = 0; cb < R; ++cb) {
              float x = 0.f;
#pragma unroll
              for (int i = 0; i < NBS * 4; ++i) x = i == b / SP * 4 + r ? p[i >> 2][cb][i & 3] : x;
              if (copy == b % SP && j == (kk >> 2 & 3) && (kk & 15) < there(b) && k0 + kk < lim[cb]) corr[cb][f] = __builtin_fmaf(x, z, corr[cb][f]);
            }
          }
        }
      }
      // weights times the step of a group, in parts, for the lane's keys of p[bb]
      Words<2> pw[NG][NP];
      auto weights = [&](int bb, int f, Words<2> (&w)[NP]) {
        const int at = f * 64 + 16 * (bb * SP + copy) + 4 * j;
        const f32x4 st = *(const f32x4*)&s_vs[at], z = *(const f32x4*)&s_vz[at];
        float x[4];
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          x[r] = p[bb][0][r] * st[r];
          corr[0][f] = __builtin_fmaf(p[bb][0][r], z[r], corr[0][f]);
        }
        split4<NP>(x, w);
      };
#pragma unroll
      for (int hf = 0; hf < 2; ++hf) {
        if constexpr (SP > 1) {
          if (hf < NBS)
#pragma unroll
            for (int f = 0; f < NG; ++f) weights(hf, f, pw[f]);
        }
        // codes of keys (2 i, 2 i + 1), a half word of a unit each
        uint32_t pr[4][UN / 4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          pr[i][0] = __builtin_amdgcn_perm(vr[8 * hf + 2 * i + 1], vr[8 * hf + 2 * i], 0x05040100u);
          if constexpr (UN == 8) pr[i][1] = __builtin_amdgcn_perm(vr[8 * hf + 2 * i + 1], vr[8 * hf + 2 * i], 0x07060302u);
        }
#pragma unroll
        for (int f = 0; f < NG; ++f) {
          Op<NP> po[R];
          if constexpr (SP > 1) {
            const uint32_t m0 = mine[2 * hf % SP], m1 = mine[(2 * hf + 1) % SP];
#pragma unroll
            for (int pl = 0; pl < NP; ++pl) po[0].p[pl] = make_uint4(pw[f][pl][0] & m0, pw[f][pl][1] & m0, pw[f][pl][0] & m1, pw[f][pl][1] & m1);
          } else {
            f32x4 st[2], z[2];
#pragma unroll
            for (int b = 0; b < 2; ++b) {
              st[b] = *(const f32x4*)&s_vs[f * 64 + 32 * hf + 16 * b + 4 * j];
              z[b] = *(const f32x4*)&s_vz[f * 64 + 32 * hf + 16 * b + 4 * j];
            }
#pragma unroll
            for (int cb = 0; cb < R; ++cb) {
              float x[8];
#pragma unroll
              for (int i = 0; i < 8; ++i) {
                const float w = p[2 * hf + (i >> 2)][cb][i & 3];
                x[i] = w * st[i >> 2][i & 3];
                corr[cb][f] = __builtin_fmaf(w, z[i >> 2][i & 3], corr[cb][f]);
              }
              po[cb] = split8<NP>(x);
            }
          }
          uint4 c[2];
#pragma unroll
          for (int y = 0; y < 2; ++y) {
            const int i = 2 * f + y;
            c[y] = make_uint4(code_pair<CENTRED>(pr[0][i / 4], i & 3, nib_mask, nib_base), code_pair<CENTRED>(pr[1][i / 4], i & 3, nib_mask, nib_base),
                              code_pair<CENTRED>(pr[2][i / 4], i & 3, nib_mask, nib_base), code_pair<CENTRED>(pr[3][i / 4], i & 3, nib_mask, nib_base));
          }
#pragma unroll
          for (int pl = NP - 1; pl >= 0; --pl)
#pragma unroll
            for (int cb = 0; cb < R; ++cb)
#pragma unroll
              for (int y = 0; y < 2; ++y) o[2 * f + y][cb] = mfma(c[y], po[cb].p[pl], o[2 * f + y][cb]);
#pragma unroll
          for (int cb = 0; cb < R; ++cb) asm volatile("" : "+v"(o[2 * f][cb]), "+v"(o[2 * f + 1][cb]), "+v"(corr[cb][f]));      // (as above)
          __builtin_amdgcn_sched_barrier(0);
        }
      }
    }
    if (more) load_values(next);
    else forget(vr);
    at = next;
  }

  // ---- the four wavefronts' sums joined in LDS
  __syncthreads();                    // (the scales of the last tile lie in the same place)
  // (what the end takes of the arguments is read here, not held in scalar registers through the loop)
  auto* again = (const __attribute__((address_space(4))) AttendArgs*)__builtin_amdgcn_kernarg_segment_ptr();
  asm volatile("" : "+s"(again));
  const AttendArgs& z = *(const AttendArgs*)again;
  float* sm_m = sm;                   // [4][16 R]
  float* sm_l = sm + 4 * 16 * R;
  float* sm_o = sm + 8 * 16 * R;      // [4][16 R][LDO]
#pragma unroll
  for (int cb = 0; cb < R; ++cb) {
    const int at = wv * 16 * R + cb * 16 + n;
    const float total = quad_sum(l[cb]);
    if (j == 0) {
      sm_m[at] = ref[cb];
      sm_l[at] = total;
    }
    float add[NG];
#pragma unroll
    for (int f = 0; f < NG; ++f) {
      add[f] = 0.f;
      if constexpr (FMT == FMT_Q4) add[f] = quad_sum(corr[cb][f]);
    }
#pragma unroll
    for (int r = 0; r < 4; ++r)
#pragma unroll
      for (int i = 0; i < UN; i += 4)
        *(float4*)&sm_o[at * LDO + (4 * j + r) * UN + i] =
            make_float4(o[i][cb][r] + add[i / 2], o[i + 1][cb][r] + add[i / 2], o[i + 2][cb][r] + add[i / 2 + 1],
                        o[i + 3][cb][r] + add[i / 2 + 1]);
  }
  __syncthreads();
  const int valid = min(16 * R, rows - row0);      // (up to CW with copies)
  for (int it = threadIdx.x; it < valid * (D / 4); it += 256) {
    const int r = it / (D / 4), c = it % (D / 4) * 4;
    float M = -INFINITY;
    // (sums of four wavefronts, of each copy)
    auto part = [&](int w) { return SP == 1 ? w * 16 * R + r : w * CW + r; };
#pragma unroll
    for (int w = 0; w < 4 * SP; ++w) M = fmaxf(M, sm_m[part(w)]);
    float L = 0.f;
    float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
    for (int w = 0; w < 4 * SP; ++w) {
      const float m = sm_m[part(w)];
      const float f = m == M ? (M == -INFINITY ? 0.f : 1.f) : __builtin_amdgcn_exp2f(m - M);
      const float4 y = *(const float4*)&sm_o[part(w) * LDO + c];
      L = __builtin_fmaf(f, sm_l[part(w)], L);
      // (a wavefront without keys has sums of 0)
      x.x = __builtin_fmaf(f, y.x, x.x);
      x.y = __builtin_fmaf(f, y.y, x.y);
      x.z = __builtin_fmaf(f, y.z, x.z);
      x.w = __builtin_fmaf(f, y.w, x.w);
    }
    const int row = row0 + r;
    if (ch.count > 1) {
      const int64_t at = (int64_t)((ch.slot0 + ch.index) * z.Hy + hy) * ((int64_t)z.pg.G * z.pg.max_new) + row;
      *(float4*)&z.part_o[at * D + c] = x;
      if (c == 0) {
        z.part_m[at] = M;
        z.part_l[at] = L;
      }
    } else {
      const int tok = row / z.pg.G, head = h * z.pg.G + row - tok * z.pg.G;
      store_out(z, nr.first + tok, head, c, x, M, L);
    }
  }
}

template <int FMT, typename T, int D, int NP, int R, int SP = 1>
int run_attend(const AttendArgs& a, hipStream_t st) {
  constexpr size_t join = (8 * 16 * R + (size_t)4 * 16 * R * (D + 4)) * 4, scales = FMT == FMT_Q4 ? 4 * 4 * 64 * (D / 32) * 4 : 0;
  constexpr size_t lds = join > scales ? join : scales;
  auto kern = k_attend<FMT, T, D, NP, R, SP>;
  if constexpr (lds > 65536) {
    if (hipFuncSetAttribute((const void*)kern, hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds) != hipSuccess) return RESTKV_EHIP;
  }
  hipLaunchKernelGGL(kern, unit_grid(a), dim3(256), lds, st, a);
  return hip_status();
}

// by format, and for many rows (attend_*.hip)
int run_attend_rows(const AttendArgs& a, int R, int waves, hipStream_t st);
int run_attend_f32(const AttendArgs& a, int R, hipStream_t st);
int run_attend_bf16(const AttendArgs& a, hipStream_t st);
int run_attend_q4(const AttendArgs& a, int R, hipStream_t st);

}  // namespace restkv
