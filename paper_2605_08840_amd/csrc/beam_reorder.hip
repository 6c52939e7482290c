// Beams go on from other beams: page tables dealt anew, rows of the open columns copied (the definition stands in the header).
#include <algorithm>

#include "beams.hpp"

namespace restkv {

namespace {

constexpr int LAYERS = 64;             // of a launch (their addresses are arguments)

struct ReorderArgs {
  Pages pg;
  int n_beams, n_groups, n_layers;
  const int32_t* parents;
  int64_t parents_stride;
  int32_t* table_out;
  int64_t table_groups;      // workgroups that write tables
  int parts;                 // workgroups of a layer and group
};
struct LayerPages { restkv_layer_pages at[LAYERS]; };

// How a group's pages are dealt: lane = beam.
struct Deal {
  int parent;      // the beam that this one goes on from
  int giver;       // whose pages it gets in open columns: its parent's, or those of a beam without a child
  bool takes;      // the latter, so that the parent's rows are copied
};
__device__ __forceinline__ Deal deal_of(const ReorderArgs& a, int g) {
  const int lane = threadIdx.x & 63, B = a.n_beams;
  int p = lane < B ? a.parents[g * a.parents_stride + lane] : -1;
  if (p < 0 || p >= B) p = lane;
  const unsigned long long own = __ballot(lane < B && p == lane);
  unsigned long long have = 0;         // beams with a child
  bool later = false;                  // an earlier beam goes on from the same one
  for (int b = 0; b < B; ++b) {
    const int q = __builtin_amdgcn_readlane(p, b);
    have |= 1ull << q;
    later = later || (q == p && b < lane);
  }
  const bool takes = lane < B && p != lane && (later || (own >> p & 1));
  const int rank = __popcll(__ballot(takes) & ((1ull << lane) - 1));
  int giver = p, n = 0;
  for (int b = 0; b < B; ++b)
    if (!(have >> b & 1)) {
      if (takes && n == rank) giver = b;
      ++n;
    }
  return {p, giver, takes};
}

// Open columns of a group's tables (of a head's, where it has its own).
struct Open { int lo, hi; };
__device__ __forceinline__ Open open_columns(const Pages& pg, int s, int h) {
  int least = cache_len(pg, s, h), most = least;
  if (!pg.table_sh && pg.lens_sh) {
    for (int x = threadIdx.x & 63; x < pg.Hkv; x += 64) {
      const int n = cache_len(pg, s, x);
      least = min(least, n);
      most = max(most, n);
    }
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
      least = min(least, __shfl_xor(least, d));
      most = max(most, __shfl_xor(most, d));
    }
  }
  least = __builtin_amdgcn_readfirstlane(least);
  most = __builtin_amdgcn_readfirstlane(most);
  return {least >> pg.lg_ps, most ? (most - 1) >> pg.lg_ps : -1};
}
__device__ __forceinline__ int source(const Deal& d, const Open& open, int b, int col) {
  const int p = __builtin_amdgcn_readlane(d.parent, b), w = __builtin_amdgcn_readlane(d.giver, b);
  return col < open.lo ? p : col <= open.hi ? w : b;
}

// Rows: a wavefront takes, of one layer, a few rows (8 KB) of one head in an open column of one child that takes pages, keys or values, eight
// 16-byte loads a lane in flight.  What a group and layer has to copy is dealt over its a.parts workgroups.  Bound by memory, where it is
// short by the chain parents, pages, rows: 32 layers, eight groups that drop one beam of four, 78 MB in 17 us (4.5 TB/s; stores that stay in the
// caches 22.5, loads past them too 21.4).  The first a.table_groups workgroups write the new tables (which are others than the old ones).
template <int RB, int SB>
__global__ __launch_bounds__(256) void k_reorder(ReorderArgs a, LayerPages layers) {
  constexpr int U = 8, L = RB / 16, SEG = 8192 / RB;        // (lanes and rows of a piece)
  const Pages& pg = a.pg;
  const int lane = threadIdx.x & 63, wv = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  int64_t id = wide_block();
  if (id < a.table_groups) {
    const int heads = pg.table_sh ? pg.Hkv : 1, of = (pg.max_pages + 63) / 64, col = (int)(id % of) * 64 + lane;
    id /= of;
    const int h = (int)(id % heads), g = (int)(id / heads), s0 = g * a.n_beams;
    const Deal d = deal_of(a, g);
    const Open open = open_columns(pg, s0, h);
    for (int b = wv; b < a.n_beams; b += 4) {
      const int from = source(d, open, b, col);
      const int64_t at = h * pg.table_sh + col;
      if (col < pg.max_pages) a.table_out[(s0 + b) * pg.table_ss + at] = pg.table[(s0 + from) * pg.table_ss + at];
    }
    return;
  }
  // (32 bits: divisions of 64 take longer than the copies)
  uint32_t y = (uint32_t)(id - a.table_groups);
  const uint32_t part = y % (uint32_t)a.parts;
  y /= (uint32_t)a.parts;
  const int g = (int)(y % (uint32_t)a.n_groups), layer = (int)(y / (uint32_t)a.n_groups), s0 = g * a.n_beams;
  if (layer >= a.n_layers) return;
  const restkv_layer_pages at = layers.at[layer];
  const Open all = open_columns(pg, s0, 0);
  const Deal d = deal_of(a, g);
  const unsigned long long takes = __ballot(d.takes);
  // pieces of a (child, head, keys or values): `segs` of each of its columns; wavefronts share them where there are more than pairs
  const uint32_t segs = ((1u << pg.lg_ps) + SEG - 1) / SEG, pieces = (pg.table_sh ? 1u : (uint32_t)(all.hi - all.lo + 1)) * segs;
  const uint32_t pairs = (uint32_t)__popcll(takes) * 2 * pg.Hkv, waves = (uint32_t)a.parts * 4, w = part * 4 + wv;
  if (!pairs) return;
  const uint32_t share = waves > pairs ? waves / pairs : 1, turn = w / pairs;
  if (share > 1 && turn >= share) return;
  for (uint32_t pr = share > 1 ? w % pairs : w; pr < pairs; pr += share > 1 ? pairs : waves)
  for (uint32_t pc = share > 1 ? turn : 0; pc < pieces; pc += share) {
    const bool is_v = pr & 1;
    const int h = (int)((pr >> 1) % (uint32_t)pg.Hkv);
    const int seg = segs > 1 ? (int)(pc % segs) : 0;
    const int len = __builtin_amdgcn_readfirstlane(cache_len(pg, s0, h));
    const int col = pg.table_sh ? len >> pg.lg_ps : all.lo + (int)(segs > 1 ? pc / segs : pc);
    const int t0 = col << pg.lg_ps, n = min(len - t0, 1 << pg.lg_ps);
    if (len <= t0 || seg * SEG >= n) continue;
    unsigned long long left = takes;
    for (uint32_t i = (pr >> 1) / (uint32_t)pg.Hkv; i; --i) left &= left - 1;
    const int child = __builtin_ctzll(left), from = __builtin_amdgcn_readlane(d.parent, child), to = __builtin_amdgcn_readlane(d.giver, child);
    const int src = page_of(pg, s0 + from, h, t0), dst = page_of(pg, s0 + to, h, t0);
    if (src < 0 || dst < 0 || src == dst) continue;
    const int first = seg * SEG, end = min(n, first + SEG);
    char* const rows = (char*)(is_v ? at.v_pages : at.k_pages);
    const char* const in = rows + (uint64_t)row_of(pg, src, h, 0) * RB;
    char* const out = rows + (uint64_t)row_of(pg, dst, h, 0) * RB;
    const uint64_t hop = (uint64_t)pg.tok_s * RB;
    for (int i = first * L + lane; i < end * L; i += 64 * U) {
      Words<4> w[U];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int x = min(i + 64 * u, end * L - 1);
        w[u] = *(const Words<4>*)(in + x / L * hop + x % L * 16);
      }
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int x = i + 64 * u;
        if (x < end * L) put<true>(out + x / L * hop + x % L * 16, w[u]);
      }
    }
    if constexpr (SB != 0) {
      typedef Words<SB / 4> W;
      char* const scales = (char*)(is_v ? at.v_scale : at.k_scale);
      const W* const sin = (const W*)(scales + (uint64_t)row_of(pg, src, h, 0) * SB);
      W* const sout = (W*)(scales + (uint64_t)row_of(pg, dst, h, 0) * SB);
      for (int t = first + lane; t < end; t += 64) sout[t * pg.tok_s] = sin[t * pg.tok_s];
    }
  }
}

// A wavefront: 64 columns of the tables of one group (and head), in place: all entries are read before any is written, the columns on
// their own.
__global__ __launch_bounds__(64) void k_reorder_table(ReorderArgs a) {
  __shared__ int s_old[64][64];
  const Pages& pg = a.pg;
  const int lane = threadIdx.x, B = a.n_beams;
  const int heads = pg.table_sh ? pg.Hkv : 1, of = (pg.max_pages + 63) / 64;
  int64_t id = wide_block();
  const int col = (int)(id % of) * 64 + lane;
  id /= of;
  const int h = (int)(id % heads);
  id /= heads;
  if (id >= a.n_groups) return;
  const int g = (int)id, s0 = g * B;
  const Deal d = deal_of(a, g);
  const Open open = open_columns(pg, s0, h);
  const int64_t at = h * pg.table_sh + col;
  const bool in = col < pg.max_pages;
#pragma unroll 8
  for (int b = 0; b < B; ++b)
    if (in) s_old[b][lane] = pg.table[(s0 + b) * pg.table_ss + at];
  for (int b = 0; b < B; ++b) {
    const int from = source(d, open, b, col);
    if (in) a.table_out[(s0 + b) * pg.table_ss + at] = s_old[from][lane];
  }
}

}  // namespace

int launch_beam_reorder(const Pages& pg, int n_beams, const int32_t* parents, int64_t parents_stride, int32_t* table_out,
                        const restkv_layer_pages* layers, int n_layers, hipStream_t st) {
  ReorderArgs a = {};
  a.pg = pg;
  a.n_beams = n_beams; a.n_groups = pg.n_seqs / n_beams;
  a.parents = parents; a.parents_stride = parents_stride; a.table_out = table_out;
  const int64_t tables = (int64_t)a.n_groups * (pg.table_sh ? pg.Hkv : 1) * ((pg.max_pages + 63) / 64);
  const bool in_place = table_out == pg.table;
  // (one launch, if the tables are others and there are no more layers than it takes; the tables alone where nothing is copied)
  const int copied = n_beams > 1 ? n_layers : 0;
  for (int at = 0; at < copied || (at == 0 && !in_place); at += LAYERS) {
    LayerPages lp = {};
    a.n_layers = std::max(0, std::min(copied - at, LAYERS));
    for (int i = 0; i < a.n_layers; ++i) lp.at[i] = layers[at + i];
    a.table_groups = at || in_place ? 0 : tables;
    // workgroups for four on each compute unit (16 / 8 / 4, us: that 16.2 / 18.3 / 16.9, four layers with lengths per head 13.4 / 11.4 / 11.2), and no more than columns of a page, or eight where there may be more, have work for
    const int64_t most = ((int64_t)(n_beams - 1) * 2 * pg.Hkv * (pg.lens_sh ? 8 : 1) + 3) / 4, pairs = std::max<int64_t>(1, (int64_t)a.n_layers * a.n_groups);
    a.parts = (int)std::max<int64_t>(1, std::min(most, (4 * n_cu() + pairs - 1) / pairs));
    const dim3 grid = wide_grid(a.table_groups + (int64_t)a.n_layers * a.n_groups * a.parts);
    auto go = [&](auto kern) { hipLaunchKernelGGL(kern, grid, dim3(256), 0, st, a, lp); };
    const bool wide = pg.d == 128;
    if (pg.fmt == RESTKV_Q4) wide ? go(k_reorder<64, 16>) : go(k_reorder<32, 8>);
    else if (pg.fmt == RESTKV_BF16) wide ? go(k_reorder<256, 0>) : go(k_reorder<128, 0>);
    else wide ? go(k_reorder<512, 0>) : go(k_reorder<256, 0>);
    if (const int rc = hip_status()) return rc;
  }
  if (!in_place) return RESTKV_OK;
  hipLaunchKernelGGL(k_reorder_table, wide_grid(tables), dim3(64), 0, st, a);
  return hip_status();
}

}  // namespace restkv
