// Attention over pages that the beams of a group have in common in front: how the work is cut, and the join.
// The shared positions of a group are one entry, with the rows (beam, new token, query head) of all its beams; what a beam has behind
// them, to a whole tile, is another.  The kernels are those of attend.hpp, on chunks of both kinds in one launch, and a row's output is
// joined from the chunks of its group's entry and of its own.
#include <algorithm>
#include <atomic>

#include "attend.hpp"
#include "beams.hpp"

namespace restkv {

namespace {

// Where the chunks of a row are (new token i, query head `head` of sequence s).
struct RowParts {
  const AttendArgs& a;
  int n, count, of_group, row, first, own;       // chunks of the front, and of both
  int hy, rb;
  __device__ __forceinline__ RowParts(const AttendArgs& a, int s, int i, int head) : a(a) {
    const Pages& pg = a.pg;
    const int h = head / pg.G, g = s / a.n_beams, rows = pg.G * pg.max_new;
    hy = a.per_head ? 0 : h;
    row = i * pg.G + head - h * pg.G;
    of_group = (s - g * a.n_beams) * rows + row;
    rb = of_group / a.front_rows;
    const int2 pf = a.plan[(int64_t)(a.per_head ? g * pg.Hkv + h : g) * a.front_blocks + rb];
    const int2 pl = a.plan[(int64_t)a.fronts * a.front_blocks + (int64_t)(a.per_head ? s * pg.Hkv + h : s) * a.own_blocks + row / a.own_rows];
    n = pf.y - pf.x + 1;
    count = n + pl.y - pl.x + 1;
    first = pf.x;
    own = pl.x;
  }
  template <int D>
  __device__ __forceinline__ Part at(int k) const {
    const bool front = k < n;
    const int64_t slot = (int64_t)(front ? first + k : own + k - n) * a.Hy + hy;
    const int64_t at = front ? slot * a.front_rows + (of_group - rb * a.front_rows) : slot * (a.pg.G * a.pg.max_new) + row;
    return {(front ? a.front_m : a.part_m) + at, (front ? a.front_l : a.part_l) + at, (front ? a.front_o : a.part_o) + at * D};
  }
};

constexpr int FEW_CHUNKS = 8;
// A workgroup a row; or (ALONE, where there are many) as many rows as it has groups of d / 4 threads, each joined by one of these if
// none has many chunks.  256 groups of four beams, 32 heads of 128: 50 -> 19 us.
template <int D, bool ALONE>
__global__ __launch_bounds__(256) void k_beams_join(AttendArgs a) {
  constexpr int TPR = D / 4, NGR = 256 / TPR;
  const Pages& pg = a.pg;
  const int s = blockIdx.y, all = pg.max_new * pg.Hq;
  if constexpr (ALONE) {
    const int x = min((int)blockIdx.x * NGR + (int)threadIdx.x / TPR, all - 1), c = threadIdx.x % TPR * 4;
    const RowParts p(a, s, x / pg.Hq, x % pg.Hq);
    const NewRows nr = new_rows(pg, s);
    const bool there = (int)blockIdx.x * NGR + (int)threadIdx.x / TPR < all && x / pg.Hq < nr.n;
    if (!__syncthreads_or(there && p.count > FEW_CHUNKS)) {
      if (!there) return;
      const Sums sums = sum_chunks(0, 1, p.count, c, [&](int k) { return p.at<D>(k); });
      store_out(a, nr.first + x / pg.Hq, x % pg.Hq, c, sums.x, sums.M, sums.L);
      return;
    }
  }
  for (int x = blockIdx.x * (ALONE ? NGR : 1), end = ALONE ? min(x + NGR, all) : x + 1; x < end; ++x) {
    const int i = x / pg.Hq, head = x % pg.Hq;
    const RowParts p(a, s, i, head);
    const NewRows nr = new_rows(pg, s);
    if (i >= nr.n) return;
    join_chunks<D>(a, p.count, nr.first + i, head, [&](int k) { return p.at<D>(k); });
    if (ALONE) __syncthreads();
  }
}

// What a part's beginning and end take, in rounds (0 / 1 / 2, us: 20 groups of four beams over 4k positions 70.9 / 71.5 / 79.7, 16 over 1k 28.0 / 27.2 / 27.2).
constexpr int PART_ROUNDS = 1;
// Rounds of a chunk at the most: as many as the longest cache has tiles (2^30 positions), so that an entry is one chunk then.  Fewer would cut
// long entries into more chunks than there is room for, which is sized by even shares.
constexpr int MOST_ROUNDS = 1 << (30 - 6);
static_assert(ATT_TILE == 1 << 6, "");

// Sum over the workgroup; lds: 16 words, free to be written.
template <typename V>
__device__ __forceinline__ V block_sum(V x, V* lds) {
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) x += __shfl_xor(x, d);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = x;
  __syncthreads();
  x = lds[0];
  for (int w = 1; w < (int)blockDim.x / 64; ++w) x += lds[w];
  return x;
}

// Chunks of a list.  An entry of `tiles` tiles in `blocks` blocks of rows costs so many rounds of c_min tiles;
__host__ __device__ __forceinline__ long long list_cost(int tiles, int blocks, int c_min) {
  return tiles ? (long long)((tiles + c_min - 1) / c_min + PART_ROUNDS) * blocks : 0;
}
// a chunk has an even share of all rounds (so the chunks of entries, in all their blocks, are no more than at_a_time and one for each part)
__host__ __device__ __forceinline__ int list_rounds(long long cost, int at_a_time) {
  const long long even = (cost + at_a_time - 1) / at_a_time;
  return even < 1 ? 1 : even < MOST_ROUNDS ? (int)even : MOST_ROUNDS;
}
__host__ __device__ __forceinline__ int more_rounds(int rounds) { return rounds + rounds / 16 + 1; }
__host__ __device__ __forceinline__ int list_chunks(int tiles, int C) { return (tiles + C - 1) / C; }
// What is to be no more chunks than run at a time: the first so many entries (all, or where the parts alone are more the fronts).
__host__ __device__ __forceinline__ int list_fit(int fronts, int entries, int front_blocks, int parts, int at_a_time) {
  return parts <= at_a_time ? entries : (int64_t)fronts * front_blocks < at_a_time ? fronts : 0;
}

// Where there are many parts, or many rows: which workgroup takes what, worked out once, by one workgroup.  Entries are cut into chunks of at
// most C tiles, C being an even share of all rounds with what parts cost beside them, but more where the chunks would be more than
// run at a time (seven groups of eight beams, lengths per head, 536 chunks for 512 workgroups: 77 us, then 59); where the parts alone are more,
// the chunks of fronts.  Fronts come first: they are the long ones, and what the beams have of their own fills the end.
// (Each workgroup for itself, as restkv_attend has it, looks at all beams of all groups: 256 groups of four beams 472 us in place of 316.)
// 6 us for 16 groups of four beams, 10 for 256, 30 for 2048.
__global__ __launch_bounds__(1024) void k_beams_list(AttendArgs a, int at_a_time) {
  __shared__ long long s_sum[16];
  __shared__ int s_count[16];
  const Pages& pg = a.pg;
  const int tid = threadIdx.x, T = blockDim.x, lane = tid & 63, wv = tid >> 6, heads = a.per_head ? pg.Hkv : 1;
  // tiles that a group (and head) shares: `seg` lanes each, one a beam
  const int seg = 1 << (32 - __clz(a.n_beams - 1)), b = tid & (seg - 1);
  long long cost = 0;
  int parts = 0;
  for (int base = 0; base < a.fronts; base += T / seg) {
    const int x = base + tid / seg, y = min(x, a.fronts - 1), g = y / heads, h = y - g * heads, s = g * a.n_beams + min(b, a.n_beams - 1);
    const int told = told_len(pg, s, h), n = new_rows(pg, s).n;
    int least = !n ? 0x7FFFFFFF : pg.causal ? max(told - n, 0) : told;
    for (int d = 1; d < seg; d <<= 1) least = min(least, __shfl_xor(least, d));
    const int shared = (int)min((int64_t)max(a.shared[g], 0) << pg.lg_ps, (int64_t)pg.max_len);
    const int tiles = least == 0x7FFFFFFF ? 0 : min(shared, least) / ATT_TILE;
    if (x >= a.fronts || b >= a.n_beams) continue;
    if (b == 0) {
      a.tiles_of[x] = tiles;
      cost += list_cost(tiles, a.front_blocks, a.c_min);
      parts += tiles ? a.front_blocks : 0;
    }
    const int own = n ? (min(told, pg.max_len) + ATT_TILE - 1) / ATT_TILE - tiles : 0;
    a.tiles_of[a.fronts + s * heads + h] = own;
    cost += list_cost(own, a.own_blocks, a.c_min);
    parts += own ? a.own_blocks : 0;
  }
  cost = block_sum(cost, s_sum);       // (and tiles_of is there for the whole workgroup)
  const int active = block_sum(parts, s_count);
  int rounds = list_rounds(cost, at_a_time);
  const int fit = list_fit(a.fronts, a.entries, a.front_blocks, active, at_a_time);
  for (int i = 0; i < 16 && fit; ++i) {
    int chunks = 0;
    const int C = rounds * a.c_min;
    for (int x = tid; x < fit; x += T) chunks += list_chunks(a.tiles_of[x], C) * (x < a.fronts ? a.front_blocks : a.own_blocks);
    if (block_sum(chunks, s_count) <= at_a_time) break;
    rounds = more_rounds(rounds);
  }
  const int C = rounds * a.c_min;
  auto list = [&](bool front) {
    const int count = front ? a.fronts : a.entries - a.fronts, blocks = front ? a.front_blocks : a.own_blocks;
    int2* const plan = a.plan + (front ? 0 : (int64_t)a.fronts * a.front_blocks);
    int4* const to = a.list + (front ? 0 : 2 * (int64_t)a.front_chunks);
    int run = 0;
    for (int base = 0; base < count; base += T) {
      const int x = base + tid;
      int cnt = 0, tiles = 0, tile0 = 0, told = 0;
      NewRows nr = {0, a.n_beams * pg.max_new};
      if (x < count) {
        const int s = a.per_head ? x / pg.Hkv : x, h = a.per_head ? x - s * pg.Hkv : 0;
        tiles = a.tiles_of[front ? x : a.fronts + x];
        told = tiles * ATT_TILE;
        if (!front) {
          tile0 = a.tiles_of[s / a.n_beams * heads + h];
          told = told_len(pg, s, h);
          nr = new_rows(pg, s);
        }
        cnt = list_chunks(tiles, C);
      }
      const int inc = wave_scan(cnt);
      __syncthreads();
      if (lane == 63) s_count[wv] = inc;
      __syncthreads();
      int from = run + inc - cnt;
      for (int w = 0; w < T / 64; ++w) {
        from += w < wv ? s_count[w] : 0;
        run += s_count[w];
      }
      if (x >= count) continue;
      for (int rb = 0; rb < blocks; ++rb) {
        const int slot = from + (front ? rb * a.front_slots : 0);
        plan[(int64_t)x * blocks + rb] = cnt ? make_int2(slot, slot + cnt - 1) : make_int2(1, 0);
      }
      const int each = cnt > 1 ? (tiles + cnt - 1) / cnt : tiles;
      for (int i = 0; i < cnt; ++i) {
        const int t0 = min(i * each, tiles), u = from + i;
        to[2 * u] = make_int4(front ? x : a.fronts + x, tile0 + t0, tile0 + min(t0 + each, tiles), u);
        to[2 * u + 1] = make_int4(told, nr.first, nr.n, 0);
      }
    }
    for (int u = run + tid; u < (front ? a.front_chunks : a.own_chunks); u += T) to[2 * u] = make_int4(-1, 0, 0, 0);
  };
  list(true);
  list(false);
}

struct BeamsPlan {
  int many, R, front_rows, own_rows, c_min, target, spread, coarse;
  int64_t front_blocks, own_blocks, fronts, entries, parts, Hy, groups, at_a_time, slots, front_slots;
};
BeamsPlan beams_plan(const Pages& pg, int n_beams) {
  BeamsPlan p = {};
  const int64_t rows = (int64_t)pg.G * pg.max_new, of_group = rows * n_beams;
  const bool per_head = pg.lens_sh != 0, bf16 = pg.fmt == RESTKV_BF16;
  p.Hy = per_head ? 1 : pg.Hkv;
  p.fronts = (int64_t)(pg.n_seqs / n_beams) * (per_head ? pg.Hkv : 1);
  p.entries = p.fronts + (int64_t)pg.n_seqs * (per_head ? pg.Hkv : 1);
  p.c_min = pg.fmt == RESTKV_Q4 ? 4 : bf16 ? 2 : 1;      // (tiles of a round: one of the keys of each wavefront)
  p.target = n_cu() * 2;
  // Fronts of bf16 pages by tiles in LDS for 64 rows (many), or from memory for 16 R rows a wavefront; us, 32 query and 8 KV heads of 128: parts
  // cut evenly, 32 rows over two times 32k positions 62.3 (R = 2) / 67.5 (many), 48 rows over 16k 43.9 / 37.7, 64 rows 50.6 / 42.7; by a
  // list, 32 groups of 32 rows over 1k 56.8 / 51.7; R = 1 in place of 2 39 / 35.  Blocks of 64 / 128 rows
  // (many): parts cut evenly, 80 rows over 8k 25.4 / 29.5, 128 over 16k 40.7 / 43.8, two times 128 53.8 / 50.7; by a list, 32 groups of 80 rows over 1k
  // 99.4 / 89.9, 16 of 256 over 512 118 / 112, eight of 256 over 4k 130 / 96.7.
  // Other pages take R = 1: their kernels have no registers left for two blocks (R = 2 / 1: float32, 32 rows over 8k 43.9 / 38.8, 256 rows
  // 239 / 224; 4 bits, 32 rows over 16k 37.2 / 35.3, 32 groups of 64 rows over 1k 120 / 108, 256 rows over 4k 183 / 190).
  auto blocks_of = [&](int many) {       // rows of a block that go by tiles in LDS, or 0
    p.many = many != 0;
    p.R = !many && bf16 && of_group > 16 ? 2 : 1;
    p.front_rows = many ? many : 16 * p.R;
    p.own_rows = many ? 16 : 16 * p.R;
    p.front_blocks = (of_group + p.front_rows - 1) / p.front_rows;
    p.own_blocks = (rows + p.own_rows - 1) / p.own_rows;
    p.parts = p.fronts * p.front_blocks + (p.entries - p.fronts) * p.own_blocks;
    p.spread = p.fronts + (p.entries - p.fronts) * p.own_blocks <= 64 && (p.fronts + 1) * p.Hy * p.front_blocks <= p.target;
  };
  blocks_of(bf16 && of_group > 32 ? 64 : 0);
  if (!p.spread && bf16 && of_group > 16) {
    blocks_of(of_group > 64 ? 128 : 64);
    p.spread = 0;
  }
  p.coarse = 0;
  if (p.spread) {
    p.groups = p.target / (p.Hy * p.front_blocks);
    p.front_slots = p.groups + 64;
    p.slots = p.groups * p.front_blocks + 64;
    // (what 64 parts cost has to be below 2^32; of 2^30 positions it passes 2^31)
    while (((int64_t)(pg.max_len / ATT_TILE >> p.coarse) + 4) * 2 * 64 * p.front_blocks > (int64_t)1 << 31) ++p.coarse;
  } else {
    // chunks: one for each entry with tiles, and as many more as make up what runs at a time
    p.at_a_time = std::max<int64_t>(1, p.target / p.Hy);
    p.front_slots = p.fronts + p.at_a_time / p.front_blocks;
    p.slots = p.entries - p.fronts + p.at_a_time / p.own_blocks;
  }
  return p;
}

struct BeamsWs { size_t plan, list, tiles, m, l, o, fm, fl, fo, bytes; };
BeamsWs beams_ws(const Pages& pg, const BeamsPlan& p) {
  BeamsWs w = {};
  auto take = [&](size_t bytes) { size_t o = w.bytes; w.bytes = align_up(w.bytes + bytes); return o; };
  const size_t rows = (size_t)p.slots * p.Hy * pg.G * pg.max_new;
  const size_t front = (size_t)p.front_slots * p.front_blocks * p.Hy * p.front_rows;
  w.plan = take((size_t)p.parts * 8);
  w.list = take(p.spread ? 0 : (size_t)(p.front_slots + p.slots) * 32);
  w.tiles = take(p.spread ? 0 : (size_t)p.entries * 4);
  w.m = take(rows * 4);
  w.l = take(rows * 4);
  w.o = take(rows * pg.d * 4);
  w.fm = take(front * 4);
  w.fl = take(front * 4);
  w.fo = take(front * pg.d * 4);
  return w;
}

// Short caches are read as if nothing were shared: one launch where each is one chunk, and no join of two kinds of chunks.  By what all
// caches may hold together.  So / by parts, us, 8 KV heads of 128, pages that the last call has read too: bf16, 4 beams 33 MB 14.2 / 15.7
// and 64 MB 16.3 / 16.3, four groups of them 33 MB 13.7 / 14.8, 65 MB 16.3 / 16.4, 129 MB 23.6 / 17.4, two groups of 16 beams 66 MB 14.6 / 18.1, 130 MB
// 19.1 / 19.6; 4 bits 40 MB 19.4 / 21.1, 80 MB 28.5 / 21.7; float32 33 MB 15.9 / 17.0, 65 MB 19.3 / 17.2.  A list takes a launch, and 3 us
// for each 32 beams: so / by a list, MiB that the caches may hold: bf16, 12 beams with lengths per head 99 19.5 / 20.9, 32 136 22.0 / 23.2, 64 144
// 20.6 / 23.0 and 208 26.1 / 24.2, 80 180 25.0 / 26.4, 160 200 30.1 / 33.1 and 360 45.9 / 35.6; float32, 64 160 22.4 / 25.2 and 288 32.1 / 30.9; 4 bits,
// 32 42 19.9 / 23.1, 64 65 21.6 / 25.1, 80 106 36.2 / 30.2, 160 62 31.0 / 39.7 and 112 42.0 / 42.4.  Around the limit for 64 beams of 4 bits, 80 MiB, as
// 16 groups of four (as 32 of two, eight of eight or four of 16 within 2 us): 75 21.8 / 26.6, 80 22.1 / 26.7, 85 24.4 / 26.9, 100 25.0 / 29.0, 115 27.6 / 29.2: it
// is on the early side there, by up to 4 us; 160 beams 162 48.5 / 44.2.
std::atomic<int> g_force_shared{0};
bool as_if_alone(const Pages& pg, int n_beams, const BeamsPlan& p) {
  if (n_beams == 1 || g_force_shared) return n_beams == 1;
  const int64_t row = pg.fmt == RESTKV_Q4 ? pg.d / 2 + pg.d / 8 : pg.fmt == RESTKV_BF16 ? pg.d * 2 : pg.d * 4;
  const int64_t most = (p.spread ? 48 : 112 + (int64_t)pg.n_seqs * 3 / 4) << (!p.spread && pg.fmt == RESTKV_Q4 ? 19 : 20);
  return 2 * row * pg.Hkv * pg.n_seqs <= most / pg.max_len;
}

}  // namespace

// k_beams_list's numbers, from the tiles of every entry.
int beams_list(const Pages& pg, int n_beams, const int32_t* tiles, int32_t* chunks) {
  const BeamsPlan p = beams_plan(pg, n_beams);
  if (p.spread || as_if_alone(pg, n_beams, p) || p.parts > 1 << 30) return RESTKV_EUNSUPPORTED;
  const int fronts = (int)p.fronts, entries = (int)p.entries, at_a_time = (int)p.at_a_time;
  auto blocks = [&](int x) { return (int)(x < fronts ? p.front_blocks : p.own_blocks); };
  long long cost = 0;
  int parts = 0;
  for (int x = 0; x < entries; ++x) {
    if (tiles[x] < 0 || tiles[x] > (1 << 30) / ATT_TILE) return RESTKV_EINVAL;
    cost += list_cost(tiles[x], blocks(x), p.c_min);
    parts += tiles[x] ? blocks(x) : 0;
  }
  int rounds = list_rounds(cost, at_a_time);
  const int fit = list_fit(fronts, entries, (int)p.front_blocks, parts, at_a_time);
  for (int i = 0; i < 16 && fit; ++i) {
    int n = 0;
    for (int x = 0; x < fit; ++x) n += list_chunks(tiles[x], rounds * p.c_min) * blocks(x);
    if (n <= at_a_time) break;
    rounds = more_rounds(rounds);
  }
  chunks[0] = chunks[2] = 0;
  for (int x = 0; x < entries; ++x) chunks[x < fronts ? 0 : 2] += list_chunks(tiles[x], rounds * p.c_min);
  chunks[1] = (int)p.front_slots;
  chunks[3] = (int)p.slots;
  return RESTKV_OK;
}

void force_shared(bool on) { g_force_shared = on; }

size_t attend_beams_ws_bytes(const Pages& pg, int n_beams) {
  const BeamsPlan p = beams_plan(pg, n_beams);
  return as_if_alone(pg, n_beams, p) ? attend_ws_bytes(pg) : beams_ws(pg, p).bytes;
}

int launch_attend_beams(const Pages& pg, int n_beams, const int32_t* shared, const void* q, const void* k_pages, const void* v_pages,
                        const void* k_scale, const void* v_scale, void* out, float* lse, char* ws, hipStream_t st) {
  const BeamsPlan p = beams_plan(pg, n_beams);
  if (as_if_alone(pg, n_beams, p)) return launch_attend(pg, q, k_pages, v_pages, k_scale, v_scale, out, lse, ws, st);
  const BeamsWs lay = beams_ws(pg, p);
  const int64_t ids = p.spread ? p.groups * p.Hy : (p.front_slots * p.Hy + 7) / 8 * 8 * p.front_blocks + (p.slots * p.Hy + 7) / 8 * 8 * p.own_blocks;
  if (ids > (int64_t)1 << 30 || p.front_slots * p.front_blocks > (int64_t)1 << 30 || std::max(p.front_blocks, p.own_blocks) > (1 << 20) ||
      (int64_t)pg.max_new * pg.Hq >= (1 << 24))
    return RESTKV_EUNSUPPORTED;
  AttendArgs a = attend_args(pg, q, k_pages, v_pages, k_scale, v_scale, out, lse);
  a.plan = (int2*)(ws + lay.plan);
  a.list = (int4*)(ws + lay.list); a.tiles_of = (int*)(ws + lay.tiles);
  a.part_m = (float*)(ws + lay.m); a.part_l = (float*)(ws + lay.l); a.part_o = (float*)(ws + lay.o);
  a.front_m = (float*)(ws + lay.fm); a.front_l = (float*)(ws + lay.fl); a.front_o = (float*)(ws + lay.fo);
  a.entries = (int)p.entries; a.Hy = (int)p.Hy;
  a.shared = shared; a.n_beams = n_beams; a.fronts = (int)p.fronts;
  a.front_blocks = (int)p.front_blocks; a.own_blocks = (int)p.own_blocks; a.front_slots = (int)p.front_slots; a.spread = p.spread;
  a.front_rows = p.front_rows; a.own_rows = p.own_rows;
  // (half rounds that a part costs beside its own, 2 / 3 / 4, us: one group of 32 beams over 16k 46.7 / 41.8 / 40.2; two of eight over 32k 62.3 / 62.4 / 63.8;
  // 4 bits, four of four over 8k to 32k 37.2 / 37.3 / 40.0.  What is added for those served first, 0 / 0.05 / 0.1 / 0.2: the last 39.3 / 39.2 / 37.7 / 38.0,
  // over 32k 63.4 / 63.1 / 63.0 / 62.6)
  a.part_cost = p.many ? 4 : 3; a.front_tiles = p.many ? 1 : p.c_min; a.coarse = p.coarse;
  a.first_more = 0.1f;
  a.row_blocks = (int)(p.spread ? p.front_blocks : 1); a.units = (int)ids; a.c_min = p.c_min;
  a.chunks = (float)p.groups;
  if (!p.spread) {
    a.front_chunks = (int)p.front_slots; a.own_chunks = (int)p.slots;
    // (lanes for every beam of every group)
    const int64_t lanes = p.fronts << (32 - __builtin_clz(n_beams - 1)), threads = std::min<int64_t>(1024, (std::max(lanes, p.entries - p.fronts) + 63) / 64 * 64);
    hipLaunchKernelGGL(k_beams_list, dim3(1), dim3(threads), 0, st, a, (int)p.at_a_time);
  }
  const int rc = p.many ? run_attend_beams_rows(a, st) : pg.fmt == RESTKV_F32 ? run_attend_beams_f32(a, st) :
                 pg.fmt == RESTKV_BF16 ? run_attend_beams_bf16(a, p.R, st) : run_attend_beams_q4(a, st);
  if (rc) return rc;
  // (by the chunks that a front's row may have; one / eight rows a workgroup, bf16, us: one group of 64 beams over 16k 65.6 / 77.5, over 4k 36.6 / 34.6,
  // two groups of 33 beams with 8 query heads over 16k 47.1 / 62.7; 256 groups of four 316 / 287 when this came)
  const bool alone = !p.spread && p.at_a_time <= FEW_CHUNKS * p.fronts * p.front_blocks;
  const int each = alone ? 1024 / pg.d : 1;
  const dim3 grid((pg.max_new * pg.Hq + each - 1) / each, pg.n_seqs);
  auto join = [&](auto kern) { hipLaunchKernelGGL(kern, grid, dim3(256), 0, st, a); };
  if (pg.d == 128) alone ? join(k_beams_join<128, true>) : join(k_beams_join<128, false>);
  else alone ? join(k_beams_join<64, true>) : join(k_beams_join<64, false>);
  return hip_status();
}

}  // namespace restkv
