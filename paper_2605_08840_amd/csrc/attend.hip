// Attention over pages: how the work is cut, and the join of the chunks of a sequence.
#include <algorithm>

#include "attend.hpp"

namespace restkv {

namespace {

template <int D>
__global__ __launch_bounds__(256) void k_attend_join(AttendArgs a) {
  const Pages& pg = a.pg;
  const int i = blockIdx.x / pg.Hq, head = blockIdx.x % pg.Hq, h = head / pg.G, s = blockIdx.y;
  const int2 pl = a.plan[a.per_head ? s * pg.Hkv + h : s];       // (of a sequence without new tokens: whatever it is, not used)
  const NewRows nr = new_rows(pg, s);
  if (i >= nr.n || pl.y < 2) return;
  const int hy = a.per_head ? 0 : h, row = i * pg.G + head - h * pg.G, rows = pg.G * pg.max_new;
  join_chunks<D>(a, pl.y, nr.first + i, head, [&](int k) {
    const int64_t at = (int64_t)((pl.x + k) * a.Hy + hy) * rows + row;
    return Part{a.part_m + at, a.part_l + at, a.part_o + at * D};
  });
}

struct AttendPlan { int R, many, waves, c_min, target; int64_t row_blocks, entries, Hy, chunks, slots; };
AttendPlan attend_plan(const Pages& pg) {
  AttendPlan p;
  // Up to 16 rows (32, where pages are not bfloat16) the four wavefronts of a workgroup share the rows and divide the keys; more
  // rows of bfloat16 pages are divided among them, with the keys in LDS.  The one / the other, us, 32k keys of 8 KV heads of 128:
  // 24 rows 32.4 / 31.6, 32 rows 33.5 / 31.7, 64 rows 41.1 / 34.4, 128 rows 62 / 46.
  const int64_t rows = (int64_t)pg.G * pg.max_new;
  p.many = pg.fmt == RESTKV_BF16 && rows > 16;
  // Two blocks of 16 rows a wavefront where one leaves rows for a second workgroup, which would read the tiles again.  One / two, us,
  // 32k keys of 8 KV heads of 128: bf16 64 rows 34.7 / 43.6, 96 rows 43.7 / 45.8, 256 rows 79.9 / 70.0 (16 caches of 2k keys,
  // 96 rows 59.4 / 57.9, 256 rows 88.8 / 120.5); 4 bits 32 rows 31.6 / 33.8, 64 rows 49.7 / 43.6, with float32 output 43.7 / 41.2,
  // 75.2 / 57.8 and 256 rows 290 / 188; f32 pages 32 rows 70.5 / 63.6, 64 rows 118 / 91, 256 rows 437 / 326.  But not for float32 queries over
  // 4 bits of 128 channels: two blocks of their three parts are more than the registers hold (32 rows 45.8 / 75.6, 64 rows 79 / 108,
  // 256 rows 304 / 322).
  const bool wide_q = pg.fmt == RESTKV_Q4 && pg.dtype == RESTKV_F32 && pg.d == 128;
  p.R = rows <= (p.many ? 64 : 16) || wide_q ? 1 : 2;
  const bool per_head = pg.lens_sh != 0;
  // eight wavefronts on one copy of a tile, where blocks of so many rows leave no more of them empty than those of four do
  p.waves = p.many && p.R == 2 && (rows + 127) / 128 % 2 == 0 ? 8 : 4;
  const int block = (p.many ? 16 * p.waves : 16) * p.R;
  p.row_blocks = (rows + block - 1) / block;
  p.entries = per_head ? (int64_t)pg.n_seqs * pg.Hkv : pg.n_seqs;
  p.Hy = per_head ? 1 : pg.Hkv;
  p.c_min = pg.fmt == RESTKV_Q4 ? 4 : 2;          // (a tile for each wavefront)
  // as many as are resident at a time, two wavefronts a SIMD (one / two / three, us: 24 sequences of 65 to 16000 4-bit positions
  // 84 / 42 / 52, 128k of them 54 / 43 / 48, 128k of bf16 98 / 100 / 108)
  p.target = n_cu() * 8 / p.waves;
  const int64_t tiles = (pg.max_len + ATT_TILE - 1) / ATT_TILE, each = p.Hy * p.row_blocks;
  // One chunk where a workgroup has read the longest cache before chunks would be joined.  One chunk / several, us, d 128, one
  // sequence of 2 KV heads with 2 rows each and one of 8 with 64 rows: bf16 192 keys 6.6 / 8.4 and 10.8 / 11.5, 384 keys 8.3 / 8.5
  // and 14.7 / 12.9, 512 keys 9.3 / 8.7; 4 bits 512 keys 9.2 / 10.0, 768 keys 11.4 / 9.9, 64 rows 384 keys 15.7 / 14.4;
  // f32 192 keys 8.3 / 9.8, 256 keys 9.9 / 9.9, 64 rows 192 keys 14.7 / 14.3.
  const int alone = rows > 16 ? (pg.fmt == RESTKV_F32 ? 2 : 4) : pg.fmt == RESTKV_F32 ? 3 : pg.fmt == RESTKV_BF16 ? 6 : 8;
  if (tiles <= alone) p.c_min = std::max(p.c_min, (int)tiles);
  // no entry has two chunks: chunks hold the sum of all tiles, or the longest entry fits the smallest chunk
  const bool single = each >= p.target || tiles <= p.c_min;
  const int64_t more = std::min<int64_t>(p.target / each + 1, p.entries * ((tiles + p.c_min - 1) / p.c_min));
  p.chunks = p.entries + (single ? 0 : more);
  p.slots = single ? 0 : std::min<int64_t>(2 * more, p.entries * ((tiles + p.c_min - 1) / p.c_min));
  return p;
}

struct AttendWs { size_t plan, m, l, o, bytes; };
AttendWs attend_ws(const Pages& pg, const AttendPlan& p) {
  AttendWs w = {};
  if (!p.slots) return w;
  size_t off = 0;
  auto take = [&](size_t bytes) { size_t o = off; off = align_up(off + bytes); return o; };
  const size_t rows = (size_t)p.slots * p.Hy * pg.G * pg.max_new;
  w.plan = take((size_t)p.entries * 8);
  w.m = take(rows * 4);
  w.l = take(rows * 4);
  w.o = take(rows * pg.d * 4);
  w.bytes = off;
  return w;
}

}  // namespace

size_t attend_ws_bytes(const Pages& pg) { return attend_ws(pg, attend_plan(pg)).bytes; }

AttendArgs attend_args(const Pages& pg, const void* q, const void* k_pages, const void* v_pages, const void* k_scale,
                       const void* v_scale, void* out, float* lse) {
  AttendArgs a = {};
  a.pg = pg;
  a.q = q; a.k = (const char*)k_pages; a.v = (const char*)v_pages;
  a.ks = (const uint32_t*)k_scale; a.vs = (const uint32_t*)v_scale;
  a.out = out; a.lse = lse;
  a.per_head = pg.lens_sh != 0;
  const int qel = pg.dtype == RESTKV_F32 ? 4 : 8;
  a.vec_q = !((uintptr_t)q & 15u) && !((pg.q_st | pg.q_sh) & (qel - 1));
  const int oal = pg.out_dtype == RESTKV_F32 ? 15 : 7;
  a.vec_out = !((uintptr_t)out & oal) && !((pg.o_st | pg.o_sh) & 3);
  return a;
}

int launch_attend(const Pages& pg, const void* q, const void* k_pages, const void* v_pages, const void* k_scale,
                  const void* v_scale, void* out, float* lse, char* ws, hipStream_t st) {
  const AttendPlan p = attend_plan(pg);
  const AttendWs lay = attend_ws(pg, p);
  if (p.chunks * p.Hy > (int64_t)1 << 30 || p.row_blocks * p.waves > (1 << 22) || (p.slots && (int64_t)pg.max_new * pg.Hq >= (1 << 24)))
    return RESTKV_EUNSUPPORTED;
  AttendArgs a = attend_args(pg, q, k_pages, v_pages, k_scale, v_scale, out, lse);
  if (p.slots) {
    a.plan = (int2*)(ws + lay.plan);
    a.part_m = (float*)(ws + lay.m); a.part_l = (float*)(ws + lay.l); a.part_o = (float*)(ws + lay.o);
  }
  a.entries = (int)p.entries; a.Hy = (int)p.Hy;
  a.row_blocks = (int)p.row_blocks; a.units = (int)(p.chunks * p.Hy);
  a.c_min = p.c_min; a.chunks = (float)((double)p.target / (double)(p.Hy * p.row_blocks) * (1 - 0x1p-23));
  const int rc = p.many ? run_attend_rows(a, p.R, p.waves, st) : pg.fmt == RESTKV_F32 ? run_attend_f32(a, p.R, st) : pg.fmt == RESTKV_BF16 ? run_attend_bf16(a, st) : run_attend_q4(a, p.R, st);
  if (rc || !p.slots) return rc;
  const dim3 grid(pg.max_new * pg.Hq, pg.n_seqs);
  if (pg.d == 128) hipLaunchKernelGGL(k_attend_join<128>, grid, dim3(256), 0, st, a);
  else hipLaunchKernelGGL(k_attend_join<64>, grid, dim3(256), 0, st, a);
  return hip_status();
}

}  // namespace restkv
