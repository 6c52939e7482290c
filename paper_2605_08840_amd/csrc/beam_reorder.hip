// Beams go on from other beams: page tables dealt anew, rows of the open columns copied (the definition stands in the header).
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
  if (!pg.table_sh && pg.lens_sh)
    for (int x = 0; x < pg.Hkv; ++x) {
      const int n = cache_len(pg, s, x);
      least = min(least, n);
      most = max(most, n);
    }
  return {least >> pg.lg_ps, most ? (most - 1) >> pg.lg_ps : -1};
}

// A workgroup: rows of one head in the open columns of one child that takes pages, of one layer, keys or values.
template <int RB, int SB>
__global__ __launch_bounds__(256) void k_reorder_rows(ReorderArgs a, LayerPages layers) {
  const Pages& pg = a.pg;
  int64_t id = wide_block();
  const bool is_v = id & 1;
  id >>= 1;
  const int h = (int)(id % pg.Hkv);
  id /= pg.Hkv;
  const int k = (int)(id % (a.n_beams - 1));
  id /= a.n_beams - 1;
  const int g = (int)(id % a.n_groups), layer = (int)(id / a.n_groups);
  if (layer >= a.n_layers) return;
  const Deal d = deal_of(a, g);
  unsigned long long takes = __ballot(d.takes);
  for (int i = 0; i < k; ++i) takes &= takes - 1;
  if (!takes) return;
  const int child = __builtin_ctzll(takes), from = __builtin_amdgcn_readlane(d.parent, child), to = __builtin_amdgcn_readlane(d.giver, child);
  const int s0 = g * a.n_beams, len = cache_len(pg, s0, h);
  const Open open = open_columns(pg, s0, h);
  const restkv_layer_pages& at = layers.at[layer];
  char* rows = (char*)(is_v ? at.v_pages : at.k_pages);
  char* scales = (char*)(is_v ? at.v_scale : at.k_scale);
  for (int col = open.lo; (int64_t)col << pg.lg_ps < len; ++col) {
    const int t0 = col << pg.lg_ps, n = min(len - t0, 1 << pg.lg_ps);
    const int src = page_of(pg, s0 + from, h, t0), dst = page_of(pg, s0 + to, h, t0);
    if (src < 0 || dst < 0 || src == dst) continue;
    constexpr int L = RB / 16;         // lanes of a row
    for (int i = threadIdx.x; i < n * L; i += 256) {
      const int t = i / L, c = i % L;
      *(uint4*)(rows + (uint64_t)row_of(pg, dst, h, t) * RB + c * 16) = *(const uint4*)(rows + (uint64_t)row_of(pg, src, h, t) * RB + c * 16);
    }
    if constexpr (SB)
      for (int t = threadIdx.x; t < n; t += 256) {
        typedef Words<SB / 4> W;
        *(W*)(scales + (uint64_t)row_of(pg, dst, h, t) * SB) = *(const W*)(scales + (uint64_t)row_of(pg, src, h, t) * SB);
      }
  }
}

// A wavefront: 64 columns of the tables of one group (and head).  All entries are read before any is written, the columns on
// their own, so that the tables may be dealt in place.
__global__ __launch_bounds__(64) void k_reorder_table(ReorderArgs a) {
  __shared__ int s_old[64][64];
  const Pages& pg = a.pg;
  const int lane = threadIdx.x, B = a.n_beams;
  const int heads = pg.table_sh ? pg.Hkv : 1, parts = (pg.max_pages + 63) / 64;
  int64_t id = wide_block();
  const int part = (int)(id % parts);
  id /= parts;
  const int h = (int)(id % heads);
  id /= heads;
  if (id >= a.n_groups) return;
  const int g = (int)id, s0 = g * B, col = part * 64 + lane;
  const Deal d = deal_of(a, g);
  const Open open = open_columns(pg, s0, h);
  const bool in = col < pg.max_pages;
  for (int b = 0; b < B; ++b)
    if (in) s_old[b][lane] = pg.table[(s0 + b) * pg.table_ss + h * pg.table_sh + col];
  for (int b = 0; b < B; ++b) {
    const int p = __builtin_amdgcn_readlane(d.parent, b), w = __builtin_amdgcn_readlane(d.giver, b);
    const int x = col < open.lo ? p : col <= open.hi ? w : b;
    if (in) a.table_out[(s0 + b) * pg.table_ss + h * pg.table_sh + col] = s_old[x][lane];
  }
}

}  // namespace

int launch_beam_reorder(const Pages& pg, int n_beams, const int32_t* parents, int64_t parents_stride, int32_t* table_out,
                        const restkv_layer_pages* layers, int n_layers, hipStream_t st) {
  ReorderArgs a = {};
  a.pg = pg;
  a.n_beams = n_beams; a.n_groups = pg.n_seqs / n_beams;
  a.parents = parents; a.parents_stride = parents_stride; a.table_out = table_out;
  for (int at = 0; at < n_layers && n_beams > 1; at += LAYERS) {
    LayerPages lp = {};
    a.n_layers = n_layers - at < LAYERS ? n_layers - at : LAYERS;
    for (int i = 0; i < a.n_layers; ++i) lp.at[i] = layers[at + i];
    const dim3 grid = wide_grid((int64_t)a.n_layers * a.n_groups * (n_beams - 1) * pg.Hkv * 2);
    auto go = [&](auto kern) { hipLaunchKernelGGL(kern, grid, dim3(256), 0, st, a, lp); };
    const bool wide = pg.d == 128;
    if (pg.fmt == RESTKV_Q4) wide ? go(k_reorder_rows<64, 16>) : go(k_reorder_rows<32, 8>);
    else if (pg.fmt == RESTKV_BF16) wide ? go(k_reorder_rows<256, 0>) : go(k_reorder_rows<128, 0>);
    else wide ? go(k_reorder_rows<512, 0>) : go(k_reorder_rows<256, 0>);
    if (const int rc = hip_status()) return rc;
  }
  const int64_t n = (int64_t)a.n_groups * (pg.table_sh ? pg.Hkv : 1) * ((pg.max_pages + 63) / 64);
  hipLaunchKernelGGL(k_reorder_table, wide_grid(n), dim3(64), 0, st, a);
  return hip_status();
}

}  // namespace restkv
