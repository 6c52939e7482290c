// The best continuations of each request's beams: score(b, v) = c[b] + (x[b, v] - m_b) - ln sum exp(x[b, .] - m_b).
// One pass over the logits: a workgroup takes a piece of a row and leaves its maximum, its sum of exponentials and its n_out best
// logits; a second launch joins the pieces of a request's rows.  Bound by memory, every logit read once.
#include <algorithm>

#include "beams.hpp"

namespace restkv {

namespace {

constexpr int SEL_THREADS = 256, SEL_VECS = 4;       // 16-byte blocks of a thread
constexpr int SEL_TILE = SEL_THREADS * SEL_VECS;

struct SelectArgs {
  Beams b;
  const void* logits;
  const float* scores; const int32_t* finished;
  float* new_scores; int32_t* parents; int32_t* tokens; int32_t* new_finished;
  int pieces, tiles;                                            // pieces of a row, tiles of a piece
  double* part_s; float* part_m; unsigned long long* keys;      // [row, piece], [row, piece], [row, piece, n_out]
};

// A candidate as a whole number: larger logit first, of equal ones the lower token; 0 is none (a logit of -inf, or NaN).
__device__ __forceinline__ unsigned long long key_of(float x, uint32_t token) {
  if (!(x > -INFINITY)) return 0;
  return (unsigned long long)float_key(x + 0.f) << 32 | ~token;         // (-0 counts as 0)
}
__device__ __forceinline__ float logit_of(unsigned long long key) {
  const uint32_t u = (uint32_t)(key >> 32);
  return __uint_as_float(u >> 31 ? u ^ 0x80000000u : ~u);
}
__device__ __forceinline__ uint32_t token_of(unsigned long long key) { return ~(uint32_t)key; }

template <typename V, typename F>
__device__ __forceinline__ V wave_join(V x, F f) {
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) x = f(x, __shfl_xor(x, d));
  return x;
}

// ---- lists of a wavefront's best logits, in LDS
constexpr int SEL_LIST = 256;                        // entries: n_out and what one step may add (64) at least
constexpr int SEL_OWN = SEL_LIST / 64;
// Logits as whole numbers have bits behind these that are all equal for a sign.
template <typename T> constexpr int SEL_LOW = sizeof(T) == 2 ? 16 : 0;

// The largest number t (in steps of 2^LOW) that at least K of the lanes' entries reach, or 0.
template <int LOW, int N>
__device__ __forceinline__ uint32_t kth(const uint32_t (&x)[N], int K) {
  uint32_t t = 0;
#pragma unroll 1
  for (int bit = 31; bit >= LOW; --bit) {
    const uint32_t u = t | 1u << bit;
    int n = 0;
#pragma unroll
    for (int j = 0; j < N; ++j) n += __popcll(__ballot(x[j] >= u));
    t = n >= K ? u : t;
  }
  return t;
}

// The K best of a list of n entries, to its front; n becomes min(n, K), the answer the K-th best (0: there are fewer).
template <int LOW>
__device__ __forceinline__ unsigned long long keep_best(unsigned long long* list, int& n, int K) {
  const int lane = threadIdx.x & 63;
  if (n < K) return 0;
  if (n <= 64) {                       // each entry's place by counting
    const unsigned long long e = lane < n ? list[lane] : 0;
    int rank = 0;
    for (int j = 0; j < n; ++j) rank += list[j] > e;
    __builtin_amdgcn_wave_barrier();
    if (lane < n && rank < K) list[rank] = e;
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    n = K;
    return list[K - 1];
  }
  uint32_t hi[SEL_OWN], lo[SEL_OWN];
#pragma unroll
  for (int j = 0; j < SEL_OWN; ++j) {
    const unsigned long long e = lane + 64 * j < n ? list[lane + 64 * j] : 0;
    hi[j] = (uint32_t)(e >> 32);
    lo[j] = (uint32_t)e;
  }
  const uint32_t t = kth<LOW>(hi, K), cut = t >> LOW;
  // those above t are in, of those at t the lowest tokens that there is room for
  uint32_t at[SEL_OWN];
  int above = 0, equal = 0;
#pragma unroll
  for (int j = 0; j < SEL_OWN; ++j) {
    above += __popcll(__ballot(hi[j] >> LOW > cut));
    equal += __popcll(__ballot(hi[j] >> LOW == cut));
    at[j] = hi[j] >> LOW == cut ? lo[j] : 0;
  }
  // (tokens are below 2^24, so that their complements have the upper bits set)
  uint32_t low = 0xFF000000u;
  if (above + equal > K) {
#pragma unroll 1
    for (int bit = 23; bit >= 0; --bit) {
      const uint32_t u = low | 1u << bit;
      int m = 0;
#pragma unroll
      for (int j = 0; j < SEL_OWN; ++j) m += __popcll(__ballot(at[j] >= u));
      low = above + m >= K ? u : low;
    }
  } else {
    // the K-th best itself: the highest token at t
    uint32_t least = 0xFFFFFFFFu;
#pragma unroll
    for (int j = 0; j < SEL_OWN; ++j) least = at[j] ? min(least, at[j]) : least;
    low = wave_join(least, [](uint32_t p, uint32_t q) { return min(p, q); });
  }
  int base = 0;
  uint32_t full = 0;                   // of an entry at t
  __builtin_amdgcn_wave_barrier();
#pragma unroll
  for (int j = 0; j < SEL_OWN; ++j) {
    const bool in = hi[j] >> LOW > cut || at[j] >= low;
    const unsigned long long mask = __ballot(in);
    if (in) list[base + __popcll(mask & ((1ull << lane) - 1))] = (unsigned long long)hi[j] << 32 | lo[j];
    base += __popcll(mask);
    const unsigned long long edge = __ballot(at[j] == low);
    if (edge) full = __builtin_amdgcn_readlane(hi[j], __builtin_ctzll(edge));
  }
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
  __builtin_amdgcn_wave_barrier();
  n = base;
  return (unsigned long long)full << 32 | low;
}

// A block of 16 bytes of a row, -inf where it lies outside the row; at: its first element, from the block of the row's start.
template <typename T>
__device__ __forceinline__ uint4 load_block(const T* p, int at, int skip, int V) {
  constexpr int VEC = 16 / sizeof(T);
  if (at >= skip && at + VEC <= skip + V) return *(const uint4*)(p + at);
  uint32_t w[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if constexpr (sizeof(T) == 4) {
      w[i] = at + i >= skip && at + i < skip + V ? __float_as_uint(p[at + i]) : 0xFF800000u;
    } else {
      w[i] = at + 2 * i >= skip && at + 2 * i < skip + V ? p[at + 2 * i].x : 0xFF80u;
      w[i] |= (at + 2 * i + 1 >= skip && at + 2 * i + 1 < skip + V ? p[at + 2 * i + 1].x : 0xFF80u) << 16;
    }
  }
  return make_uint4(w[0], w[1], w[2], w[3]);
}

// e^d for d <= 0 as 2^(d log2 e), with the second half of log2 e (its first alone is 1e-8 short).
__device__ __forceinline__ float exp_of(float d) {
  return __builtin_amdgcn_exp2f(__builtin_fmaf(d, 0x1.715476p+0f, d * 0x1.4ae0cp-26f));
}

// Maximum, sum and best logits of a piece of a row: a.tiles tiles of 1024 16-byte blocks.  Each wavefront keeps its best logits in a
// list, into which goes whatever is above the n_out-th best so far: of the first tile, above the n_out-th largest of the
// lanes' maxima (which as many logits reach).  A later block of a wavefront holds later tokens, so that a logit equal to the n_out-th best
// is not wanted any more and one comparison of a block's maximum decides.
template <typename T>
__global__ __launch_bounds__(SEL_THREADS) void k_select_rows(SelectArgs a) {
  constexpr int VEC = 16 / sizeof(T), NW = SEL_THREADS / 64, LOW = SEL_LOW<T>;
  __shared__ double s_sum[NW];
  __shared__ float s_max[NW];
  __shared__ int s_n[NW];
  __shared__ unsigned long long s_list[NW][SEL_LIST];
  const int64_t id = wide_block();
  const int64_t row = id / a.pieces;
  const int piece = (int)(id % a.pieces), V = a.b.n_vocab, K = a.b.n_out, tid = threadIdx.x, lane = tid & 63;
  const int wv = __builtin_amdgcn_readfirstlane(tid >> 6);
  if (row >= (int64_t)a.b.n_groups * a.b.n_beams || (a.finished && a.finished[row])) return;
  // blocks of 16 bytes as the memory has them; block 0 holds the row's first element, `skip` elements in
  const T* p = (const T*)a.logits + row * a.b.stride;
  const int skip = (int)((uintptr_t)p / sizeof(T) % VEC);
  p -= skip;
  unsigned long long* const list = s_list[wv];
  const int first = piece * a.tiles, last = min(first + a.tiles, (skip + V + SEL_TILE * VEC - 1) / (SEL_TILE * VEC));
  auto place = [&](int tile, int c) { return ((tile * SEL_VECS + c) * SEL_THREADS + tid) * VEC; };
  uint4 next[SEL_VECS];
#pragma unroll
  for (int c = 0; c < SEL_VECS; ++c) next[c] = load_block(p, place(first, c), skip, V);
  float m = -INFINITY, limit = 0.f;
  double sum = 0.0;
  int n = 0;
  unsigned long long bar = 0;          // the n_out-th best so far, 0: there are fewer
  for (int tile = first; tile < last; ++tile) {
    float x[SEL_VECS][VEC], top[SEL_VECS];
#pragma unroll
    for (int c = 0; c < SEL_VECS; ++c) {
      const uint32_t u[4] = {next[c].x, next[c].y, next[c].z, next[c].w};
      top[c] = -INFINITY;
#pragma unroll
      for (int i = 0; i < VEC; ++i) {
        if constexpr (sizeof(T) == 4) x[c][i] = __uint_as_float(u[i]);
        else x[c][i] = __uint_as_float(i & 1 ? u[i / 2] & 0xFFFF0000u : u[i / 2] << 16);
        top[c] = fmaxf(top[c], x[c][i]);
      }
    }
    if (tile + 1 < last)
#pragma unroll
      for (int c = 0; c < SEL_VECS; ++c) next[c] = load_block(p, place(tile + 1, c), skip, V);
    float mt = top[0];
#pragma unroll
    for (int c = 1; c < SEL_VECS; ++c) mt = fmaxf(mt, top[c]);
    if (mt > m) {
      sum *= m == -INFINITY ? 1.0 : (double)exp_of(m - mt);      // (a sum of 0, or NaN)
      m = mt;
    }
    const float ref = m == -INFINITY ? 0.f : m;
    float s = 0.f;
#pragma unroll
    for (int c = 0; c < SEL_VECS; ++c)
#pragma unroll
      for (int i = 0; i < VEC; ++i) {
        s += exp_of(x[c][i] - ref);
      }
    sum += (double)s;

    // ---- into the list
    bool any;
    if (tile == first) {
      const uint32_t t[1] = {mt > -INFINITY ? float_key(mt + 0.f) : 0u};
      bar = (unsigned long long)kth<16>(t, K) << 32;   // (its upper bits: below every logit that reaches it)
      limit = bar ? logit_of(bar) : -INFINITY;
      any = true;
    } else {
      any = mt > limit;
    }
    if (__ballot(any)) {
#pragma unroll
      for (int c = 0; c < SEL_VECS; ++c) {
        if (!__ballot(tile == first ? top[c] >= limit : top[c] > limit)) continue;
#pragma unroll
        for (int i = 0; i < VEC; ++i) {
          if (!__ballot(x[c][i] >= limit)) continue;
          const unsigned long long key = key_of(x[c][i], (uint32_t)(place(tile, c) - skip + i));
          unsigned long long mask = __ballot(key > bar);
          if (!mask) continue;
          if (n + __popcll(mask) > SEL_LIST) {
            bar = keep_best<LOW>(list, n, K);
            mask = __ballot(key > bar);
          }
          if (key > bar) list[n + __popcll(mask & ((1ull << lane) - 1))] = key;
          n += __popcll(mask);
          __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
          __builtin_amdgcn_wave_barrier();
        }
      }
      if (tile + 1 < last && (tile == first || n >= K + 64)) bar = keep_best<LOW>(list, n, K);
    }
    limit = bar ? logit_of(bar) : -INFINITY;
  }
  if (n > 64) keep_best<LOW>(list, n, K);
  const float wm = wave_join(m, [](float p, float q) { return fmaxf(p, q); });
  // (a thread of which everything is masked out has a sum of 0; a NaN stays one)
  sum *= m == wm ? 1.0 : (double)exp_of(m - wm);
  sum = wave_join(sum, [](double p, double q) { return p + q; });
  if (lane == 0) {
    s_max[wv] = wm;
    s_sum[wv] = sum;
    s_n[wv] = n;
  }
  __syncthreads();
  // ---- the wavefronts' sums joined, and the best of their lists (up to 64 entries each), an entry a thread
  const int64_t at = row * a.pieces + piece;
  if (tid == 0) {
    float M = s_max[0];
    for (int w = 1; w < NW; ++w) M = fmaxf(M, s_max[w]);
    double S = 0.0;
    for (int w = 0; w < NW; ++w) S += s_sum[w] * (s_max[w] == M ? 1.0 : (double)exp_of(s_max[w] - M));
    a.part_m[at] = M;
    a.part_s[at] = S;
  }
  const unsigned long long e = lane < n ? list[lane] : 0;
  int rank = 0, all = 0;
  for (int w = 0; w < NW; ++w) {
    const int nw = s_n[w];
    for (int j = 0; j < nw; ++j) rank += s_list[w][j] > e;
    all += nw;
  }
  if (lane < n && rank < K) a.keys[at * K + rank] = e;
  for (int k = all + tid; k < K; k += SEL_THREADS) a.keys[at * K + k] = 0;
}

// A continuation: larger first.
struct Cont { double score; int beam; unsigned long long key; };
__device__ __forceinline__ bool before(const Cont& x, const Cont& y) {
  return x.score > y.score || (x.score == y.score && (x.beam < y.beam || (x.beam == y.beam && x.key > y.key)));
}
__device__ __forceinline__ Cont better(const Cont& x, const Cont& y) { return before(x, y) ? x : y; }

// A workgroup a request, a wavefront a row or a part of one.  Of the continuations that the rows' pieces have left, those that reach a
// bound go into a list in LDS, and an entry's place in the answer is the number of entries before it.  The bound: of the wavefront that
// has the highest, the n_out-th largest of its lanes' maxima.  Where more reach it than the list holds (scores that are all equal) the answer is
// found one at a time.
constexpr int JOIN_WAVES = 16, JOIN_LIST = 64 * JOIN_WAVES, JOIN_AHEAD = 4;
__global__ __launch_bounds__(JOIN_LIST) void k_select_join(SelectArgs a) {
  constexpr int NW = JOIN_WAVES;
  __shared__ double s_score[64], s_log[64];
  __shared__ float s_top[64];
  __shared__ int s_end[64], s_count;
  __shared__ uint32_t s_bar[NW];
  __shared__ __align__(16) uint32_t s_floor[JOIN_LIST];
  __shared__ Cont s_list[JOIN_LIST];
  const int B = a.b.n_beams, K = a.b.n_out, C = a.pieces, tid = threadIdx.x, lane = tid & 63;
  const int wv = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int64_t g = blockIdx.x;
  const unsigned long long* const keys = a.keys + g * B * C * K;
  // rows of this wavefront: row0, row0 + NW, ..; of such a row every `parts`-th 64 keys
  const int parts = max(1, NW / B), row0 = wv / parts, part = wv % parts, per = C * K;
  const Cont none = {-INFINITY, 1 << 30, 0};
  // (none where the score is not finite)
  auto cont = [&](int b, unsigned long long key) {
    const Cont x = {s_score[b] + (((double)logit_of(key) - (double)s_top[b]) - s_log[b]), b, key};
    return key && x.score - x.score == 0.0 ? x : none;
  };
  auto ended = [&](int b) {
    const Cont x = {s_score[b], b, (unsigned long long)(uint32_t)~a.b.end_token};
    return x.score - x.score == 0.0 ? x : none;
  };
  // a score as a float that is not above it, as a whole number
  auto floor_of = [](double s) {
    const float f = (float)s;
    const uint32_t k = float_key(f);
    return s > -INFINITY ? ((double)f > s ? k - 1 : k) : 0u;
  };
  if (tid == 0) s_count = 0;
  uint32_t top[1] = {0};
  for (int b = row0; b < B; b += NW / parts) {
    const int64_t row = g * B + b;
    const bool end = a.finished && a.finished[row];
    unsigned long long key[JOIN_AHEAD];
#pragma unroll
    for (int u = 0; u < JOIN_AHEAD; ++u) {
      const int i = (u * parts + part) * 64 + lane;
      key[u] = !end && i < per ? keys[b * per + i] : 0;
    }
    double S = 0.0;
    float M = -INFINITY;
    const double score = a.scores[row];
    if (!end) {
      float m = lane < C ? a.part_m[row * C + lane] : -INFINITY;
      double s = lane < C ? a.part_s[row * C + lane] : 0.0;
      for (int c = lane + 64; c < C; c += 64) {
        const float mc = a.part_m[row * C + c], mx = fmaxf(m, mc);
        s = s * (m == mx ? 1.0 : (double)exp_of(m - mx)) + a.part_s[row * C + c] * (mc == mx ? 1.0 : (double)exp_of(mc - mx));
        m = mx;
      }
      M = wave_join(m, [](float p, float q) { return fmaxf(p, q); });
      S = wave_join(s * (m == M ? 1.0 : (double)exp_of(m - M)), [](double p, double q) { return p + q; });
    }
    if (lane == 0 && part == 0) {
      s_end[b] = end;
    }
    if (lane == 0) {                   // (all parts write the same)
      s_score[b] = score;
      s_log[b] = log(S);
      s_top[b] = M;
    }
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    if (end) {
      if (lane == 0) top[0] = max(top[0], floor_of(ended(b).score));
      continue;
    }
#pragma unroll
    for (int u = 0; u < JOIN_AHEAD; ++u) top[0] = max(top[0], floor_of(cont(b, key[u]).score));
    for (int i = (JOIN_AHEAD * parts + part) * 64 + lane; i < per; i += parts * 64) top[0] = max(top[0], floor_of(cont(b, keys[b * per + i]).score));
  }
  const uint32_t own = kth<12>(top, K);
  if (lane == 0) s_bar[wv] = own;
  __syncthreads();
  uint32_t bar = 1;
  for (int w = 0; w < NW; ++w) bar = max(bar, s_bar[w]);
  auto put_in = [&](const Cont& x) {
    const uint32_t f = floor_of(x.score);
    if (f < bar) return;
    const int at = atomicAdd(&s_count, 1);             // (in any order)
    if (at < JOIN_LIST) {
      s_list[at] = x;
      s_floor[at] = f;
    }
  };
  for (int b = row0; b < B; b += NW / parts) {
    if (s_end[b]) {
      if (part == 0 && lane == 0) put_in(ended(b));
      continue;
    }
    for (int i = part * 64 + lane; i < per; i += parts * 64) put_in(cont(b, keys[b * per + i]));
  }
  __syncthreads();
  const int n = s_count;
  auto give = [&](int k, const Cont& x) {
    const bool there = x.score > -INFINITY;
    const int token = there ? (int)token_of(x.key) : -1;
    a.new_scores[g * K + k] = (float)x.score;
    a.parents[g * K + k] = there ? x.beam : -1;
    a.tokens[g * K + k] = token;
    if (a.new_finished) a.new_finished[g * K + k] = !there || token == a.b.end_token || s_end[x.beam];
  };
  if (n <= JOIN_LIST) {
    // (whole floats first: only scores that are equal as such are compared in 64 bits)
    if (tid < n) {
      const uint32_t f = s_floor[tid];
      int rank = 0, equal = 0;
      for (int j = 0; j < n; ++j) {
        rank += s_floor[j] > f;
        equal += s_floor[j] == f;
      }
      const Cont x = s_list[tid];
      if (equal > 1)
        for (int j = 0; j < n; ++j) rank += s_floor[j] == f && before(s_list[j], x);
      if (rank < K) give(rank, x);
    }
    for (int k = n + tid; k < K; k += JOIN_LIST) give(k, none);
    return;
  }
  Cont last = {INFINITY, -1, ~0ull};
  Cont* const s_best = s_list;         // [2][NW]
  for (int k = 0; k < K; ++k) {
    Cont best = none;
    for (int b = row0; b < B; b += NW / parts) {
      if (s_end[b]) {
        const Cont x = ended(b);
        if (before(last, x)) best = better(best, x);
        continue;
      }
      for (int i = part * 64 + lane; i < per; i += parts * 64) {
        const Cont x = cont(b, keys[b * per + i]);
        if (before(last, x)) best = better(best, x);
      }
    }
    for (int d = 1; d < 64; d <<= 1) {
      const Cont o = {__shfl_xor(best.score, d), __shfl_xor(best.beam, d), __shfl_xor(best.key, d)};
      best = better(best, o);
    }
    if (lane == 0) s_best[(k & 1) * NW + wv] = best;
    __syncthreads();
    for (int w = 0; w < NW; ++w) best = better(best, s_best[(k & 1) * NW + w]);
    last = best;
    if (tid == 0) give(k, best);
  }
}

struct SelectPlan { int pieces, tiles; };
SelectPlan select_plan(const Beams& b) {
  const int vec = b.dtype == RESTKV_F32 ? 4 : 8;
  const int all = (b.n_vocab / vec + 2 + SEL_TILE - 1) / SEL_TILE;       // (blocks of 16 bytes that a row may touch)
  // workgroups for four on each compute unit, if there is as much
  const int64_t rows = (int64_t)b.n_groups * b.n_beams, want = 4 * n_cu();
  const int tiles = (int)std::max<int64_t>(1, rows * all / want);
  return {(all + tiles - 1) / tiles, tiles};
}
struct SelectWs { size_t s, m, keys, bytes; };
SelectWs select_ws(const Beams& b) {
  SelectWs w = {};
  const size_t n = (size_t)b.n_groups * b.n_beams * select_plan(b).pieces;
  auto take = [&](size_t bytes) { size_t o = w.bytes; w.bytes = align_up(w.bytes + bytes); return o; };
  w.s = take(n * 8);
  w.m = take(n * 4);
  w.keys = take(n * b.n_out * 8);
  return w;
}

}  // namespace

size_t beam_ws_bytes(const Beams& b) { return b.n_groups ? select_ws(b).bytes : 0; }

int launch_beam_select(const Beams& b, const void* logits, const float* scores, const int32_t* finished, float* new_scores,
                       int32_t* parents, int32_t* tokens, int32_t* new_finished, char* ws, hipStream_t st) {
  const SelectWs lay = select_ws(b);
  SelectArgs a = {};
  a.b = b;
  a.logits = logits; a.scores = scores; a.finished = finished;
  a.new_scores = new_scores; a.parents = parents; a.tokens = tokens; a.new_finished = new_finished;
  const SelectPlan plan = select_plan(b);
  a.pieces = plan.pieces; a.tiles = plan.tiles;
  a.part_s = (double*)(ws + lay.s); a.part_m = (float*)(ws + lay.m); a.keys = (unsigned long long*)(ws + lay.keys);
  const dim3 grid = wide_grid((int64_t)b.n_groups * b.n_beams * a.pieces);
  if (b.dtype == RESTKV_F32) hipLaunchKernelGGL(k_select_rows<float>, grid, dim3(SEL_THREADS), 0, st, a);
  else hipLaunchKernelGGL(k_select_rows<bf16_t>, grid, dim3(SEL_THREADS), 0, st, a);
  hipLaunchKernelGGL(k_select_join, dim3(b.n_groups), dim3(JOIN_LIST), 0, st, a);
  return hip_status();
}

}  // namespace restkv
