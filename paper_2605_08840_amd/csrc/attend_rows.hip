// Attention over bfloat16 pages for many rows (the queries of an observation window, prompts): products and softmax take longer
// than memory, so a tile of 64 keys and values is copied to LDS once for the rows of a workgroup, 16 R for each of its four or
// eight wavefronts: 64 to 256.
#include "attend.hpp"

namespace restkv {

namespace {

// NW wavefronts of 16 R rows each share the tiles; otherwise the products and the softmax are those of k_attend.  Two tiles
// are in LDS: the next one is copied (each wavefront 64 / NW rows of it) while this one is used.  Rows lie unpadded, the 16-byte
// pieces of a row in the order piece ^ row, so that the reads of one piece of sixteen rows spread over the banks.
// 256 queries a KV head, 32k keys, d 128, float32 output (three parts of a weight: 69 GFLOP of products for 34), us a call with
// the join of its chunks, 83.4 now: four wavefronts 89.6, eight 87.2 (half the copies); two tiles a copy and a barrier 90.8.  Of that,
// without the copies 8 would go, without the second and third part of the weights 20, without the exponentials 3.  No pipe is full
// (matrix 36 % busy, vector issue 41 %): the two wavefronts of a SIMD do the same at the same time, behind one barrier a tile, so that products
// and softmax follow each other (a wavefront alone takes 4500 cycles a tile, 2048 of them products); 31 chunks of up to 17 tiles stand
// for 32 of 16, and 33 MB of chunk sums are written and read again.
template <int D, int NP, int R, int NW>
__global__ __attribute__((amdgpu_flat_work_group_size(64 * NW, 64 * NW), amdgpu_waves_per_eu(2)))
void k_attend_rows(AttendArgs a) {
  constexpr int UN = D / 16, QC = D / 32, ROWB = D * 2, TK = 64, NB = 4, CH = ROWB / 16, TILE = TK * ROWB;
  extern __shared__ __align__(16) char lds[];        // [2][keys | values][TILE]
  const Pages& pg = a.pg;
  const int lane = threadIdx.x & 63, n = lane & 15, j = lane >> 4;
  const int wv = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);

  const int unit = unit_of_block(), rb = blockIdx.x >> 3;
  if (unit >= a.units) return;
  const int hy = unit % a.Hy;
  Chunk ch;
  if (!find_chunk<NW>(a, unit / a.Hy, (int*)lds, ch)) return;
  ch.n = __builtin_amdgcn_readfirstlane(ch.n);
  ch.first = __builtin_amdgcn_readfirstlane(ch.first);
  const int e = __builtin_amdgcn_readfirstlane(ch.e);
  const int s = a.per_head ? e / pg.Hkv : e, h = a.per_head ? e - s * pg.Hkv : hy;
  const int rows = pg.G * ch.n, block0 = rb * 16 * NW * R, row0 = block0 + wv * 16 * R;
  if (block0 >= rows) return;
  if (a.plan && ch.index == 0 && hy == 0 && rb == 0 && threadIdx.x == 0) a.plan[e] = make_int2(ch.slot0, ch.count);

  const int told = __builtin_amdgcn_readfirstlane(ch.told), len = min(told, pg.max_len);
  auto limit = [&](int row) {       // positions that a row sees
    return pg.causal ? min(max(told - ch.n + row / pg.G + 1, 0), len) : len;
  };
  // of the workgroup, and of this wavefront (none, if it has no rows)
  const int k_begin = __builtin_amdgcn_readfirstlane(ch.tile0 * ATT_TILE);
  const int k_end = __builtin_amdgcn_readfirstlane(min(ch.tile1 * ATT_TILE, limit(min(block0 + 16 * NW * R, rows) - 1)));
  const int own_end = __builtin_amdgcn_readfirstlane(row0 < rows ? min(k_end, limit(min(row0 + 16 * R, rows) - 1)) : 0);
  const int lim_lo = __builtin_amdgcn_readfirstlane(limit(min(row0, rows - 1)));
  const float sc = pg.scale * 1.44269504088896341f;

  // ---- tiles
  const int32_t* table = pg.table + s * pg.table_ss + h * pg.table_sh;
  const uint32_t tokb = (uint32_t)pg.tok_s * ROWB;
  const char* const kh = a.k + h * pg.head_s * ROWB;
  const char* const vh = a.v + h * pg.head_s * ROWB;
  auto first_row = [&](int t, uint32_t& row) {       // of the 16-key block at t, and whether it has a page
    const int page = uniform_load(table + (min(t, k_end - 1) >> pg.lg_ps));
    const bool ok = (uint32_t)page < (uint32_t)pg.n_pages && t < k_end;
    row = ok ? (uint32_t)page * (uint32_t)pg.page_s + (t & ((1 << pg.lg_ps) - 1)) * (uint32_t)pg.tok_s : 0u;
    return ok;
  };
  // rows of a copy, a wavefront's rows of a tile and its copies of them
  constexpr int PER = 1024 / ROWB, OWN = TK / NW, PIECES = OWN / PER;
  static_assert(PIECES >= 1 && 16 % OWN == 0, "");
  const int own0 = wv * OWN, in_block = own0 & 15;
  uint32_t off[PIECES];
#pragma unroll
  for (int x = 0; x < PIECES; ++x) {
    const int r = in_block + x * PER + lane / CH;
    off[x] = r * tokb + ((lane % CH) ^ (r & (CH - 1))) * 16;
  }
  auto copy = [&](int k0, int buf) {                  // this wavefront's rows of the tile
    uint32_t row;
    first_row(k0 + (own0 & ~15), row);
    char* to = lds + buf * 2 * TILE + own0 * ROWB;
#pragma unroll
    for (int x = 0; x < PIECES; ++x) dma_1k(kh + (uint64_t)row * ROWB, off[x], to + x * 1024);
#pragma unroll
    for (int x = 0; x < PIECES; ++x) dma_1k(vh + (uint64_t)row * ROWB, off[x], to + TILE + x * 1024);
  };
  if (k_begin < k_end) copy(k_begin, 0);

  // ---- queries
  int lim[R];
  Op<1> qo[R][QC];
#pragma unroll
  for (int cb = 0; cb < R; ++cb) {
    const int row = min(row0 + cb * 16 + n, rows - 1);
    lim[cb] = limit(row);
    const int tok = row / pg.G;
    const bf16_t* p = (const bf16_t*)a.q + (ch.first + tok) * pg.q_st + (h * pg.G + row - tok * pg.G) * pg.q_sh;
#pragma unroll
    for (int c = 0; c < QC; ++c) {
      float x[8];
      load_row<bf16_t, 8>(p + c * 32 + j * 8, a.vec_q, x);
      qo[cb][c] = split8<1>(x);
    }
  }
  f32x4 o[UN][R];
  float ref[R], l[R];
#pragma unroll
  for (int cb = 0; cb < R; ++cb) {
#pragma unroll
    for (int i = 0; i < UN; ++i) o[i][cb] = f32x4{0.f, 0.f, 0.f, 0.f};
    ref[cb] = -INFINITY;
    l[cb] = 0.f;
  }

  int buf = 0;
  for (int k0 = k_begin; k0 < k_end; k0 += TK, buf ^= 1) {
    // this tile is there (every wavefront has waited for its own copies), and the other one is read by nobody any more
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
    if (k0 + TK < k_end) copy(k0 + TK, buf ^ 1);
    if (k0 >= own_end) continue;
    const char* kt = lds + buf * 2 * TILE;
    const char* vt = kt + TILE;
    int ok = 0;
#pragma unroll
    for (int b = 0; b < NB; ++b) {
      uint32_t row;
      ok |= first_row(k0 + 16 * b, row) ? 1 << b : 0;
    }
    const bool masked = k0 + TK > min(own_end, lim_lo) || ok != (1 << NB) - 1;
    auto there = [&](int b) { return ok >> b & 1 ? min(k_end - (k0 + 16 * b), 16) : 0; };

    // ---- logits
    f32x4 p[NB][R];
#pragma unroll
    for (int b = 0; b < NB; ++b) {
#pragma unroll
      for (int cb = 0; cb < R; ++cb) p[b][cb] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int c = 0; c < QC; ++c) {
        const uint4 x = *(const uint4*)(kt + (16 * b + n) * ROWB + ((4 * c + j) ^ (n & (CH - 1))) * 16);
#pragma unroll
        for (int cb = 0; cb < R; ++cb) p[b][cb] = mfma(x, qo[cb][c].p[0], p[b][cb]);
      }
    }
    // ---- softmax: lane = row, key 16 b + 4 j + r in register r of block b
    if (masked) {
#pragma unroll
      for (int cb = 0; cb < R; ++cb)
#pragma unroll
        for (int b = 0; b < NB; ++b)
#pragma unroll
          for (int r = 0; r < 4; ++r)
            p[b][cb][r] = 4 * j + r < there(b) && k0 + 16 * b + 4 * j + r < lim[cb] ? p[b][cb][r] : -INFINITY;
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
    if (__builtin_expect(__ballot(far) != 0, 0)) {
#pragma unroll
      for (int cb = 0; cb < R; ++cb) {
        const float m = fmaxf(ref[cb], top[cb]);
        const float f = ref[cb] == m ? 1.f : __builtin_amdgcn_exp2f(ref[cb] - m);
        ref[cb] = m;
        l[cb] *= f;
#pragma unroll
        for (int i = 0; i < UN; ++i) o[i][cb] *= f;
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
#pragma unroll
    for (int hf = 0; hf < 2; ++hf) {
      Words<UN / 2> vr[8];           // unit n of the lane's eight keys
#pragma unroll
      for (int x = 0; x < 8; ++x) {
        const int r = 4 * j + (x & 3);                // row of its block
        const char* row = vt + (32 * hf + (x >> 2) * 16 + r) * ROWB;
        vr[x] = *(const Words<UN / 2>*)(UN == 8 ? row + (n ^ (r & (CH - 1))) * 16 : row + ((n >> 1) ^ (r & (CH - 1))) * 16 + (n & 1) * 8);
      }
      Op<NP> po[R];
#pragma unroll
      for (int cb = 0; cb < R; ++cb) {
        const f32x4 u = p[2 * hf][cb], w = p[2 * hf + 1][cb];
        const float x[8] = {u[0], u[1], u[2], u[3], w[0], w[1], w[2], w[3]};
        po[cb] = weight_parts<NP>(x);
      }
      if (__builtin_expect(masked, 0)) {
        keep_here(vr);
        bool bad = false;
#pragma unroll
        for (int x = 0; x < 8; ++x)
#pragma unroll
          for (int i = 0; i < UN / 2; ++i) {
            if (4 * j + (x & 3) >= there(2 * hf + (x >> 2))) vr[x][i] = 0u;
            bad = bad || (vr[x][i] & 0x7F80u) == 0x7F80u || (vr[x][i] & 0x7F800000u) == 0x7F800000u;
          }
        if (__builtin_expect(__ballot(bad) != 0, 0)) {
          // Values that are not finite, where some rows do not see every key (0 times them would be NaN): each is added to the
          // sums of the rows that see its key; zeros then take their places in the products.
#pragma unroll 1
          for (int kk = 0; kk < 32; ++kk) {
            const int b = 2 * hf + (kk >> 4), r0 = kk & 15;
            if (r0 >= (kk >> 4 ? there(2 * hf + 1) : there(2 * hf))) continue;
            float w[R];
            uint32_t sees[R];
#pragma unroll
            for (int cb = 0; cb < R; ++cb) {
              sees[cb] = k0 + 16 * b + r0 < lim[cb] ? ~0u : 0u;
              w[cb] = p[2 * hf][cb][0];
#pragma unroll
              for (int x = 1; x < 8; ++x) w[cb] = x == (kk >> 4) * 4 + (kk & 3) ? p[2 * hf + (x >> 2)][cb][x & 3] : w[cb];
              w[cb] = __shfl(w[cb], n + 16 * (r0 >> 2));      // the lane that holds the key's weight
            }
#pragma unroll
            for (int i = 0; i < UN; ++i)
#pragma unroll
              for (int r = 0; r < 4; ++r) {
                const int piece = (4 * j + r) * UN * 2 / 16, in = (4 * j + r) * UN * 2 % 16 + 2 * i;
                const uint32_t x = *(const uint16_t*)(vt + (16 * b + r0) * ROWB + (piece ^ (r0 & (CH - 1))) * 16 + in);
                const uint32_t odd = (x << 16) & (0u - ((x & 0x7F80u) + 0x80u >> 15));      // 0 where it is finite
#pragma unroll
                for (int cb = 0; cb < R; ++cb) o[i][cb][r] = __builtin_fmaf(w[cb], __uint_as_float(odd & sees[cb]), o[i][cb][r]);
              }
          }
#pragma unroll
          for (int x = 0; x < 8; ++x)
#pragma unroll
            for (int i = 0; i < UN / 2; ++i) {
              const uint32_t w = vr[x][i];
              vr[x][i] = w & ~(((w & 0x7F80u) == 0x7F80u ? 0xFFFFu : 0u) | ((w & 0x7F800000u) == 0x7F800000u ? 0xFFFF0000u : 0u));
            }
        }
      }
#pragma unroll
      for (int i = 0; i < UN; ++i) {
        const uint32_t sel = i & 1 ? 0x07060302u : 0x05040100u;
        const uint4 x = make_uint4(__builtin_amdgcn_perm(vr[1][i / 2], vr[0][i / 2], sel), __builtin_amdgcn_perm(vr[3][i / 2], vr[2][i / 2], sel),
                                   __builtin_amdgcn_perm(vr[5][i / 2], vr[4][i / 2], sel), __builtin_amdgcn_perm(vr[7][i / 2], vr[6][i / 2], sel));
#pragma unroll
        for (int pl = NP - 1; pl >= 0; --pl)
#pragma unroll
          for (int cb = 0; cb < R; ++cb) o[i][cb] = mfma(x, po[cb].p[pl], o[i][cb]);
      }
    }
  }

  // ---- a lane has four units of its rows, 16 bytes at a time: by way of LDS to whole rows (where the tiles were), which are
  // stored 512 bytes at a time (256 queries a KV head over 32k keys 86.5 -> 83.4 us)
  __syncthreads();
  char* const own = lds + wv * (16 * D * 4);
  static_assert(NW * 16 * D * 4 <= 4 * TILE, "");
  constexpr int Q = D / 4;
#pragma unroll
  for (int cb = 0; cb < R; ++cb) {
    const float L = quad_sum(l[cb]);
#pragma unroll
    for (int r = 0; r < 4; ++r)
#pragma unroll
      for (int i = 0; i < UN; i += 4)
        *(f32x4*)(own + n * (D * 4) + (((4 * j + r) * (UN / 4) + i / 4) ^ n) * 16) = f32x4{o[i][cb][r], o[i + 1][cb][r], o[i + 2][cb][r], o[i + 3][cb][r]};
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
#pragma unroll
    for (int k = 0; k < 16 * Q / 64; ++k) {
      const int r = k * (64 / Q) + lane / Q, q = lane % Q, row = row0 + cb * 16 + r;
      const float4 x = *(const float4*)(own + r * (D * 4) + (q ^ r) * 16);
      const float m = __shfl(ref[cb], r), total = __shfl(L, r);
      if (row >= rows) continue;
      if (ch.count > 1) {
        const int64_t at = (int64_t)((ch.slot0 + ch.index) * a.Hy + hy) * ((int64_t)pg.G * pg.max_new) + row;
        *(float4*)&a.part_o[at * D + q * 4] = x;
        if (q == 0) {
          a.part_m[at] = m;
          a.part_l[at] = total;
        }
      } else {
        const int tok = row / pg.G;
        store_out(a, ch.first + tok, h * pg.G + row - tok * pg.G, q * 4, x, m, total);
      }
    }
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
  }
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
