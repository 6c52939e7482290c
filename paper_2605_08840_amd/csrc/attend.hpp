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
  int row_blocks, units, c_min, target, vec_q, vec_out;
};

constexpr int ATT_TILE = 64;        // chunks are whole tiles of 64 keys

typedef float f32x4 __attribute__((ext_vector_type(4)));

// What a workgroup takes.  Chunks are of equal size C over all entries: enough for `target` workgroups in all, so that a
// long sequence among short ones is cut as finely as the whole asks for, and short batches not at all.
struct Chunk { int e, tile0, tile1, index, count, slot0; };
__device__ __forceinline__ bool find_chunk(const AttendArgs& a, int x, Chunk& o) {
  const Pages& pg = a.pg;
  const int lane = threadIdx.x & 63;
  auto tiles_of = [&](int e) {
    if (e >= a.entries) return 0;
    const int s = a.per_head ? e / pg.Hkv : e, h = a.per_head ? e - s * pg.Hkv : 0;
    const int n = pg.new_start ? pg.new_start[s + 1] > pg.new_start[s] : 1;
    return n ? (cache_len(pg, s, h) + ATT_TILE - 1) / ATT_TILE : 0;
  };
  int64_t total = 0;
  for (int base = 0; base < a.entries; base += 64) total += wave_sum((uint32_t)tiles_of(base + lane));
  const int64_t want = (total * (a.Hy * a.row_blocks) + a.target - 1) / a.target;
  const int C = (int)(want < a.c_min ? a.c_min : want > (1 << 25) ? (1 << 25) : want);
  int run = 0, slots = 0;
  for (int base = 0; base < a.entries; base += 64) {
    const int e = base + lane, tiles = tiles_of(e);
    const int cnt = e < a.entries ? max(1, (tiles + C - 1) / C) : 0;
    int inc = cnt, sl = cnt > 1 ? cnt : 0;
    const int own = sl;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
      const int p = __shfl_up(inc, d), q = __shfl_up(sl, d);
      if (lane >= d) { inc += p; sl += q; }
    }
    const unsigned long long hit = __ballot(run + inc > x);
    if (hit) {
      const int l = __builtin_ctzll(hit);
      o.e = base + l;
      o.count = __builtin_amdgcn_readlane(cnt, l);
      o.index = x - run - __builtin_amdgcn_readlane(inc, l) + o.count;
      o.slot0 = slots + __builtin_amdgcn_readlane(sl - own, l);
      const int t = __builtin_amdgcn_readlane(tiles, l), each = (t + o.count - 1) / o.count;
      o.tile0 = min(o.index * each, t);
      o.tile1 = min(o.tile0 + each, t);
      return true;
    }
    run += __builtin_amdgcn_readlane(inc, 63);
    slots += __builtin_amdgcn_readlane(sl, 63);
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

// FMT: pages; T: queries; NP: bf16 parts of a softmax weight (products with float32 pages take the weight itself); R: blocks
// of 16 rows of a wavefront.
template <int FMT, typename T, int D, int NP, int R>
__global__ __launch_bounds__(256) void k_attend(AttendArgs a) {
  constexpr int UN = D / 16, NG = D / 32;
  constexpr int QP = FMT == FMT_Q4 ? planes_of<T> : 1;
  constexpr int TK = FMT == FMT_F32 ? 16 : FMT == FMT_BF16 ? 32 : 64, NB = TK / 16;
  constexpr int64_t ROWB = FMT == FMT_F32 ? D * 4 : FMT == FMT_BF16 ? D * 2 : D / 2;
  constexpr int LDO = D + 4;
  extern __shared__ __align__(16) float sm[];
  const Pages& pg = a.pg;
  const int lane = threadIdx.x & 63, n = lane & 15, j = lane >> 4;
  const int wv = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);

  // row blocks of a chunk follow each other on one XCD, whose L2 then holds the chunk (workgroups go round eight XCDs)
  int unit, rb;
  if (a.row_blocks == 1) {
    unit = (int)wide_block();
    rb = 0;
  } else {
    const int64_t b = wide_block(), per = (int64_t)a.row_blocks * 8, in = b % per;
    unit = (int)(b / per * 8 + in % 8);
    rb = (int)(in / 8);
  }
  if (unit >= a.units) return;
  const int hy = unit % a.Hy;
  Chunk ch;
  if (!find_chunk(a, unit / a.Hy, ch)) return;
  const int e = __builtin_amdgcn_readfirstlane(ch.e);
  const int s = a.per_head ? e / pg.Hkv : e, h = a.per_head ? e - s * pg.Hkv : hy;
  const NewRows nr = new_rows(pg, s);
  const int rows = pg.G * nr.n, row0 = rb * 16 * R;
  if (row0 >= rows) return;
  if (a.plan && ch.index == 0 && hy == 0 && rb == 0 && threadIdx.x == 0) a.plan[e] = make_int2(ch.slot0, ch.count);

  const int told = told_len(pg, s, h), len = min(told, pg.max_len);
  auto limit = [&](int row) {       // positions that a row sees
    return pg.causal ? min(max(told - nr.n + row / pg.G + 1, 0), len) : len;
  };
  const int last_row = min(row0 + 16 * R, rows) - 1;
  const int k_end = __builtin_amdgcn_readfirstlane(min(ch.tile1 * ATT_TILE, limit(last_row)));
  const int lim_lo = __builtin_amdgcn_readfirstlane(limit(row0));
  const int k_begin = __builtin_amdgcn_readfirstlane(ch.tile0 * ATT_TILE);
  const float sc = pg.scale * 1.44269504088896341f;

  int lim[R];
  // queries, as operands
  constexpr int QC = FMT == FMT_F32 ? D / 16 : D / 32;
  float4 qf[FMT == FMT_F32 ? R : 1][FMT == FMT_F32 ? QC : 1];
  Op<QP> qo[FMT == FMT_F32 ? 1 : R][FMT == FMT_F32 ? 1 : QC];
  float qsum[FMT == FMT_Q4 ? R : 1][NG];
#pragma unroll
  for (int cb = 0; cb < R; ++cb) {
    const int row = min(row0 + cb * 16 + n, rows - 1);
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
      float x[4 * UN];               // units 4j .. 4j+3
      load_row<T, 4 * UN>(p + j * 4 * UN, a.vec_q, x);
#pragma unroll
      for (int f = 0; f < NG; ++f) {
        float y[8], t = 0.f;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          y[i] = x[(i & 3) * UN + 2 * f + (i >> 2)];
          t += y[i];
        }
        qo[cb][f] = split8<QP>(y);
        qsum[cb][f] = quad_sum(t);
      }
    }
  }

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
  float* scales = sm + wv * (2 * 64 * NG * 2);       // [K | V][64 keys][group]{step, zero - 16 step} of this wavefront's tile

  for (int k0 = k_begin + wv * TK; k0 < k_end; k0 += 4 * TK) {
    // the 16-key blocks of the tile: each lies in one page
    int64_t base[NB];
    int there[NB];
    bool whole = k0 + TK <= min(k_end, lim_lo);
#pragma unroll
    for (int b = 0; b < NB; ++b) {
      const int t = k0 + 16 * b;
      const int page = t < k_end ? page_of(pg, s, h, t) : -1;
      there[b] = page >= 0 ? min(k_end - t, 16) : 0;
      base[b] = page >= 0 ? row_of(pg, page, h, t) : 0;
      whole = whole && page >= 0;
    }
    const int tok = (int)pg.tok_s;

    f32x4 p[NB][R];
#pragma unroll
    for (int b = 0; b < NB; ++b)
#pragma unroll
      for (int cb = 0; cb < R; ++cb) p[b][cb] = f32x4{0.f, 0.f, 0.f, 0.f};

    // values, loaded ahead of their use
    uint32_t vw[FMT == FMT_F32 ? 1 : NB * 4][FMT == FMT_BF16 ? UN / 2 : 1];
    float vf[FMT == FMT_F32 ? 4 : 1][UN];
    if constexpr (FMT == FMT_F32) {
      float4 kr[QC];
      const char* kp = a.k + base[0] * ROWB + (int64_t)(min(n, max(there[0] - 1, 0)) * tok) * ROWB + j * 16;
#pragma unroll
      for (int c = 0; c < QC; ++c) kr[c] = *(const float4*)(kp + c * 64);
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const char* vp = a.v + base[0] * ROWB + (int64_t)(min(4 * j + r, max(there[0] - 1, 0)) * tok) * ROWB + n * (UN * 4);
#pragma unroll
        for (int i = 0; i < UN; i += 4) *(float4*)&vf[r][i] = *(const float4*)(vp + i * 4);
      }
#pragma unroll
      for (int c = 0; c < QC; ++c)
#pragma unroll
        for (int cb = 0; cb < R; ++cb) {
          p[0][cb] = __builtin_amdgcn_mfma_f32_16x16x4f32(kr[c].x, qf[cb][c].x, p[0][cb], 0, 0, 0);
          p[0][cb] = __builtin_amdgcn_mfma_f32_16x16x4f32(kr[c].y, qf[cb][c].y, p[0][cb], 0, 0, 0);
          p[0][cb] = __builtin_amdgcn_mfma_f32_16x16x4f32(kr[c].z, qf[cb][c].z, p[0][cb], 0, 0, 0);
          p[0][cb] = __builtin_amdgcn_mfma_f32_16x16x4f32(kr[c].w, qf[cb][c].w, p[0][cb], 0, 0, 0);
        }
    } else if constexpr (FMT == FMT_BF16) {
      uint4 kr[NB][QC];
#pragma unroll
      for (int b = 0; b < NB; ++b) {
        const char* kp = a.k + base[b] * ROWB + (int64_t)(n * tok) * ROWB + j * 16;
#pragma unroll
        for (int c = 0; c < QC; ++c) kr[b][c] = *(const uint4*)(kp + c * 64);
      }
#pragma unroll
      for (int b = 0; b < NB; ++b)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const char* vp = a.v + base[b] * ROWB + (int64_t)((4 * j + r) * tok) * ROWB + n * (UN * 2);
          if constexpr (UN == 8) *(uint4*)vw[b * 4 + r] = *(const uint4*)vp;
          else *(uint2*)vw[b * 4 + r] = *(const uint2*)vp;
        }
#pragma unroll
      for (int c = 0; c < QC; ++c)
#pragma unroll
        for (int b = 0; b < NB; ++b)
#pragma unroll
          for (int cb = 0; cb < R; ++cb) p[b][cb] = mfma(kr[b][c], qo[cb][c].p[0], p[b][cb]);
    } else {
      uint32_t kr[NB][UN / 2];       // units 4j .. 4j+3 of key n of each block
#pragma unroll
      for (int b = 0; b < NB; ++b) {
        const char* kp = a.k + base[b] * ROWB + (int64_t)(n * tok) * ROWB + j * (UN * 2);
        if constexpr (UN == 8) *(uint4*)kr[b] = *(const uint4*)kp;
        else *(uint2*)kr[b] = *(const uint2*)kp;
      }
#pragma unroll
      for (int b = 0; b < NB; ++b)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const char* vp = a.v + base[b] * ROWB + (int64_t)((4 * j + r) * tok) * ROWB + n * (UN / 2);
          vw[b * 4 + r][0] = UN == 8 ? *(const uint32_t*)vp : *(const uint16_t*)vp;
        }
      // steps and zeros: lane = key of the tile
      {
        int64_t row = base[0];
#pragma unroll
        for (int b = 1; b < NB; ++b) row = j == b ? base[b] : row;
        row = (row + (int64_t)(n * tok)) * NG;
        uint32_t w[2][NG];
        if constexpr (NG == 4) {
          *(uint4*)w[0] = *(const uint4*)(a.ks + row);
          *(uint4*)w[1] = *(const uint4*)(a.vs + row);
        } else {
          *(uint2*)w[0] = *(const uint2*)(a.ks + row);
          *(uint2*)w[1] = *(const uint2*)(a.vs + row);
        }
        __builtin_amdgcn_wave_barrier();
#pragma unroll
        for (int m = 0; m < 2; ++m) {
          float y[2 * NG];
#pragma unroll
          for (int f = 0; f < NG; ++f) {
            y[2 * f] = __uint_as_float(w[m][f] << 16);
            y[2 * f + 1] = __builtin_fmaf(-16.f, y[2 * f], __uint_as_float(w[m][f] & 0xFFFF0000u));
          }
#pragma unroll
          for (int f = 0; f < NG; f += 2)
            *(float4*)&scales[(m * 64 + lane) * (2 * NG) + 2 * f] = make_float4(y[2 * f], y[2 * f + 1], y[2 * f + 2], y[2 * f + 3]);
        }
        __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
        __builtin_amdgcn_wave_barrier();
      }
#pragma unroll
      for (int b = 0; b < NB; ++b) {
        uint4 op[NG];                 // 16 + code as bf16, group by group
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
          const int e0 = (2 * f) & 3;  // nibble of a half word; to bits 3 .. 6
          auto put = [](uint32_t x, int i) {
            return ((i == 0 ? x << 3 : x >> (4 * i - 3)) & 0x00780078u) | 0x41804180u;
          };
          op[f] = make_uint4(put(lo, e0), put(hi, e0), put(lo, e0 + 1), put(hi, e0 + 1));
        }
        float y[4][2 * NG];
#pragma unroll
        for (int r = 0; r < 4; ++r)
#pragma unroll
          for (int f = 0; f < 2 * NG; f += 4) *(float4*)&y[r][f] = *(const float4*)&scales[(16 * b + 4 * j + r) * (2 * NG) + f];
#pragma unroll
        for (int cb = 0; cb < R; ++cb)
#pragma unroll
          for (int f = 0; f < NG; ++f) {
            f32x4 t = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int pl = 0; pl < QP; ++pl) t = mfma(op[f], qo[cb][f].p[pl], t);
#pragma unroll
            for (int r = 0; r < 4; ++r) {
              const float z = __builtin_fmaf(y[r][2 * f + 1], qsum[cb][f], p[b][cb][r]);
              p[b][cb][r] = __builtin_fmaf(y[r][2 * f], t[r], z);
            }
          }
      }
    }

    // ---- softmax: lane = row, key 16 b + 4 j + r in register r of block b
    if (!whole) {
#pragma unroll
      for (int cb = 0; cb < R; ++cb)
#pragma unroll
        for (int b = 0; b < NB; ++b)
#pragma unroll
          for (int r = 0; r < 4; ++r)
            if (4 * j + r >= there[b] || k0 + 16 * b + 4 * j + r >= lim[cb]) p[b][cb][r] = -INFINITY;
    }
    bool far = false;
    float top[R];
#pragma unroll
    for (int cb = 0; cb < R; ++cb) {
      float m = -INFINITY;
#pragma unroll
      for (int b = 0; b < NB; ++b)
#pragma unroll
        for (int r = 0; r < 4; ++r) m = fmaxf(m, p[b][cb][r]);
      top[cb] = quad_max(m) * sc;
      far = far || top[cb] > ref[cb] + 8.f;
    }
    // the reference follows the largest logit when it is 2^8 behind: rarely
    if (__ballot(far)) {
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
      for (int b = 0; b < NB; ++b)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          p[b][cb][r] = __builtin_amdgcn_exp2f(__builtin_fmaf(p[b][cb][r], sc, -m));
          l[cb] += p[b][cb][r];
        }
    }

    // ---- O^T += V^T P^T
    if constexpr (FMT == FMT_F32) {
      bool bad = false;
      if (!whole) {
#pragma unroll
        for (int r = 0; r < 4; ++r)
#pragma unroll
          for (int i = 0; i < UN; ++i) {
            if (4 * j + r >= there[0]) vf[r][i] = 0.f;
            bad = bad || !(vf[r][i] - vf[r][i] == 0.f);
          }
      }
      if (__builtin_expect(__ballot(bad) != 0, 0)) {
        // values that are not finite, in a tile where some rows do not see every key (0 times them would be NaN): they come
        // first and key by key, a row that does not see the key keeps its sums, and zeros take their places below
        for (int kk = 0; kk < 16; ++kk) {
#pragma unroll
          for (int r = 0; r < 4; ++r)
            if (r == (kk & 3)) {
#pragma unroll
              for (int i = 0; i < UN; ++i) {
                const float x = j == kk >> 2 && !(vf[r][i] - vf[r][i] == 0.f) ? vf[r][i] : 0.f;
#pragma unroll
                for (int cb = 0; cb < R; ++cb) {
                  const f32x4 t = __builtin_amdgcn_mfma_f32_16x16x4f32(x, p[0][cb][r], o[i][cb], 0, 0, 0);
                  o[i][cb] = kk < there[0] && k0 + kk < lim[cb] ? t : o[i][cb];
                }
              }
            }
        }
#pragma unroll
        for (int r = 0; r < 4; ++r)
#pragma unroll
          for (int i = 0; i < UN; ++i) vf[r][i] = vf[r][i] - vf[r][i] == 0.f ? vf[r][i] : 0.f;
      }
#pragma unroll
      for (int r = 0; r < 4; ++r)
#pragma unroll
        for (int i = 0; i < UN; ++i)
#pragma unroll
          for (int cb = 0; cb < R; ++cb) o[i][cb] = __builtin_amdgcn_mfma_f32_16x16x4f32(vf[r][i], p[0][cb][r], o[i][cb], 0, 0, 0);
    } else if constexpr (FMT == FMT_BF16) {
      // eight keys of a lane: registers r of both blocks
      Op<NP> po[R];
#pragma unroll
      for (int cb = 0; cb < R; ++cb) {
        const float x[8] = {p[0][cb][0], p[0][cb][1], p[0][cb][2], p[0][cb][3], p[1][cb][0], p[1][cb][1], p[1][cb][2], p[1][cb][3]};
        po[cb] = split8<NP>(x);
      }
      auto operand = [](const uint32_t (&w)[8][UN / 2], int i) {      // place i of every unit, keys 0 .. 7
        const uint32_t sel = i & 1 ? 0x07060302u : 0x05040100u;
        return make_uint4(__builtin_amdgcn_perm(w[1][i / 2], w[0][i / 2], sel), __builtin_amdgcn_perm(w[3][i / 2], w[2][i / 2], sel),
                          __builtin_amdgcn_perm(w[5][i / 2], w[4][i / 2], sel), __builtin_amdgcn_perm(w[7][i / 2], w[6][i / 2], sel));
      };
      bool bad = false;
      if (!whole) {
#pragma unroll
        for (int x = 0; x < 8; ++x)
#pragma unroll
          for (int i = 0; i < UN / 2; ++i) {
            if (4 * j + (x & 3) >= there[x >> 2]) vw[x][i] = 0u;
            bad = bad || (vw[x][i] & 0x7F80u) == 0x7F80u || (vw[x][i] & 0x7F800000u) == 0x7F800000u;
          }
      }
      if (__builtin_expect(__ballot(bad) != 0, 0)) {       // as above
        auto odd = [](uint32_t w) {   // the halves that are not finite
          return ((w & 0x7F80u) == 0x7F80u ? 0xFFFFu : 0u) | ((w & 0x7F800000u) == 0x7F800000u ? 0xFFFF0000u : 0u);
        };
        for (int kk = 0; kk < 32; ++kk) {
          const int at = kk >> 4 << 2 | (kk & 3), have = kk >> 4 ? there[1] : there[0];
          const bool mine = j == (kk >> 2 & 3);
          uint32_t w1[8][UN / 2];
#pragma unroll
          for (int x = 0; x < 8; ++x)
#pragma unroll
            for (int i = 0; i < UN / 2; ++i) w1[x][i] = mine && x == at ? vw[x][i] & odd(vw[x][i]) : 0u;
#pragma unroll
          for (int i = 0; i < UN; ++i)
#pragma unroll
            for (int cb = 0; cb < R; ++cb) {
              // (the first part of a weight alone: parts of unlike sign would make a NaN of an infinity)
              const f32x4 t = mfma(operand(w1, i), po[cb].p[0], o[i][cb]);
              o[i][cb] = (kk & 15) < have && k0 + kk < lim[cb] ? t : o[i][cb];
            }
        }
#pragma unroll
        for (int x = 0; x < 8; ++x)
#pragma unroll
          for (int i = 0; i < UN / 2; ++i) vw[x][i] &= ~odd(vw[x][i]);
      }
#pragma unroll
      for (int i = 0; i < UN; ++i) {
        const uint4 x = operand(vw, i);
#pragma unroll
        for (int cb = 0; cb < R; ++cb)
#pragma unroll
          for (int pl = NP - 1; pl >= 0; --pl) o[i][cb] = mfma(x, po[cb].p[pl], o[i][cb]);
      }
    } else {
#pragma unroll
      for (int hf = 0; hf < 2; ++hf) {
        float y[8][2 * NG];           // {step, zero - 16 step} of the lane's eight keys
#pragma unroll
        for (int x = 0; x < 8; ++x)
#pragma unroll
          for (int f = 0; f < 2 * NG; f += 4)
            *(float4*)&y[x][f] = *(const float4*)&scales[(64 + 32 * hf + (x >> 2) * 16 + 4 * j + (x & 3)) * (2 * NG) + f];
        // codes of keys (2 i, 2 i + 1), a half word of a unit each
        uint32_t pr[4][UN / 4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          pr[i][0] = __builtin_amdgcn_perm(vw[8 * hf + 2 * i + 1][0], vw[8 * hf + 2 * i][0], 0x05040100u);
          if constexpr (UN == 8) pr[i][1] = __builtin_amdgcn_perm(vw[8 * hf + 2 * i + 1][0], vw[8 * hf + 2 * i][0], 0x07060302u);
        }
#pragma unroll
        for (int f = 0; f < NG; ++f) {
          Op<NP> po[R];
#pragma unroll
          for (int cb = 0; cb < R; ++cb) {
            float x[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
              const float w = p[2 * hf + (i >> 2)][cb][i & 3];
              float st = y[i][2 * f], z = y[i][2 * f + 1];
              // (a key that is not seen: its scale may hold anything, and 0 times it need not be 0)
              const int at = (i >> 2) * 16 + 4 * j + (i & 3);
              if (!whole && (4 * j + (i & 3) >= there[2 * hf + (i >> 2)] || k0 + 32 * hf + at >= lim[cb])) { st = 0.f; z = 0.f; }
              x[i] = w * st;
              corr[cb][f] = __builtin_fmaf(w, z, corr[cb][f]);
            }
            po[cb] = split8<NP>(x);
          }
#pragma unroll
          for (int i = 2 * f; i < 2 * f + 2; ++i) {
            const int nib = i & 3;
            auto put = [&](uint32_t x) {
              return ((nib == 0 ? x << 3 : x >> (4 * nib - 3)) & 0x00780078u) | 0x41804180u;
            };
            const uint4 x = make_uint4(put(pr[0][i / 4]), put(pr[1][i / 4]), put(pr[2][i / 4]), put(pr[3][i / 4]));
#pragma unroll
            for (int cb = 0; cb < R; ++cb)
#pragma unroll
              for (int pl = NP - 1; pl >= 0; --pl) o[i][cb] = mfma(x, po[cb].p[pl], o[i][cb]);
          }
        }
      }
    }
  }

  // ---- the four wavefronts' sums joined in LDS
  __syncthreads();                    // (the scales of the last tile lie in the same place)
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
  const int valid = min(16 * R, rows - row0);
  for (int it = threadIdx.x; it < valid * (D / 4); it += 256) {
    const int r = it / (D / 4), c = it % (D / 4) * 4;
    float M = -INFINITY;
#pragma unroll
    for (int w = 0; w < 4; ++w) M = fmaxf(M, sm_m[w * 16 * R + r]);
    float L = 0.f;
    float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      const float m = sm_m[w * 16 * R + r];
      const float f = m == M ? (M == -INFINITY ? 0.f : 1.f) : __builtin_amdgcn_exp2f(m - M);
      const float4 y = *(const float4*)&sm_o[(w * 16 * R + r) * LDO + c];
      L = __builtin_fmaf(f, sm_l[w * 16 * R + r], L);
      // (a wavefront without keys has sums of 0)
      x.x = __builtin_fmaf(f, y.x, x.x);
      x.y = __builtin_fmaf(f, y.y, x.y);
      x.z = __builtin_fmaf(f, y.z, x.z);
      x.w = __builtin_fmaf(f, y.w, x.w);
    }
    const int row = row0 + r;
    if (ch.count > 1) {
      const int64_t at = (int64_t)((ch.slot0 + ch.index) * a.Hy + hy) * ((int64_t)pg.G * pg.max_new) + row;
      *(float4*)&a.part_o[at * D + c] = x;
      if (c == 0) {
        a.part_m[at] = M;
        a.part_l[at] = L;
      }
    } else {
      const int tok = row / pg.G, head = h * pg.G + row - tok * pg.G;
      store_out(a, nr.first + tok, head, c, x, M, L);
    }
  }
}

template <int FMT, typename T, int D, int NP, int R>
int run_attend(const AttendArgs& a, hipStream_t st) {
  constexpr size_t join = (8 * 16 * R + (size_t)4 * 16 * R * (D + 4)) * 4, scales = FMT == FMT_Q4 ? 4 * 2 * 64 * (D / 32) * 2 * 4 : 0;
  constexpr size_t lds = join > scales ? join : scales;
  const int64_t blocks = a.row_blocks == 1 ? a.units : (int64_t)(a.units + 7) / 8 * 8 * a.row_blocks;
  auto kern = k_attend<FMT, T, D, NP, R>;
  if constexpr (lds > 65536) {
    if (hipFuncSetAttribute((const void*)kern, hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds) != hipSuccess) return RESTKV_EHIP;
  }
  hipLaunchKernelGGL(kern, wide_grid(blocks), dim3(256), lds, st, a);
  return hip_status();
}

// by format (attend_*.hip)
int run_attend_f32(const AttendArgs& a, int R, hipStream_t st);
int run_attend_bf16(const AttendArgs& a, int R, hipStream_t st);
int run_attend_q4(const AttendArgs& a, int R, hipStream_t st);

}  // namespace restkv
