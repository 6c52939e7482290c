// The best continuations of each request's beams: score(b, v) = c[b] + (x[b, v] - m_b) - ln sum exp(x[b, .] - m_b).
// One pass over the logits: a workgroup takes a piece of a row and leaves its maximum, its sum of exponentials and its n_out best
// logits; a second launch joins the pieces of a request's rows.  Bound by memory, every logit read once.
#include <float.h>

#include <algorithm>

#include "beams.hpp"

namespace restkv {

namespace {

constexpr int SEL_THREADS = 256, SEL_VECS = 4;       // 16-byte blocks of a thread
constexpr int SEL_TILE = SEL_THREADS * SEL_VECS;
constexpr int MANY_OUT = 32;

struct SelectArgs {
  Beams b;
  const void* logits;
  const float* scores; const int32_t* finished;
  float* new_scores; int32_t* parents; int32_t* tokens; int32_t* new_finished;
  int pieces, blocks;                                           // pieces of a row, 16-byte blocks of a piece
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

// x of the lane that a data-parallel move names, for 32 and 64 bits.
template <int CTRL, typename V>
__device__ __forceinline__ V moved(V x) {
  if constexpr (sizeof(V) == 4) {
    return __builtin_bit_cast(V, __builtin_amdgcn_mov_dpp(__builtin_bit_cast(int, x), CTRL, 0xF, 0xF, true));
  } else {
    const int2 w = __builtin_bit_cast(int2, x);
    return __builtin_bit_cast(V, make_int2(moved<CTRL>(w.x), moved<CTRL>(w.y)));
  }
}
// f over 2, 4, 8, 16 or 64 neighbouring lanes, the answer in all of them.
template <int LANES, typename V, typename F>
__device__ __forceinline__ V lanes_join(V x, F f) {
  x = f(x, moved<0xB1>(x));            // neighbours, and pairs of them
  if constexpr (LANES >= 4) x = f(x, moved<0x4E>(x));
  if constexpr (LANES == 8) x = f(x, moved<0x141>(x));        // (the other four of eight)
  if constexpr (LANES >= 16) {
    x = f(x, moved<0x124>(x));         // round by 4 and by 8 of sixteen
    x = f(x, moved<0x128>(x));
  }
  if constexpr (LANES == 64) {
    x = f(x, __shfl_xor(x, 16));
    x = f(x, __shfl_xor(x, 32));
  }
  return x;
}
struct Max { template <typename V> __device__ __forceinline__ V operator()(V p, V q) const { return p > q ? p : q; } };
struct MaxF { __device__ __forceinline__ float operator()(float p, float q) const { return fmaxf(p, q); } };
struct Sum { template <typename V> __device__ __forceinline__ V operator()(V p, V q) const { return p + q; } };

// What the wavefront has written to LDS, to itself.
__device__ __forceinline__ void settle() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
  __builtin_amdgcn_wave_barrier();
}

// A number that at least K <= 64 of the workgroup's x reach (their lowest bits apart): the K-th largest of the maxima of GROUPS
// groups of threads.  lds: GROUPS + 1 words, 16-byte aligned; every thread has to come here.
template <int THREADS, int GROUPS>
__device__ __forceinline__ uint32_t bound_of(uint32_t x, int K, uint32_t* lds) {
  constexpr int L = THREADS / GROUPS, N = GROUPS / L / 4;        // threads of a group; each compares its maximum with 4 N others
  const int g = threadIdx.x / L, l = threadIdx.x % L;
  const uint32_t y = (lanes_join<L>(x, Max()) & ~(GROUPS - 1u)) | (GROUPS - 1 - g);
  if (l == 0) lds[g] = y;
  __syncthreads();
  int rank = 0;
#pragma unroll
  for (int u = 0; u < N; ++u) {
    const uint4 v = ((const uint4*)lds)[l * N + u];
    rank += (v.x > y) + (v.y > y) + (v.z > y) + (v.w > y);
  }
  rank = lanes_join<L>(rank, Sum());
  if (l == 0 && rank == K - 1) lds[GROUPS] = y;
  __syncthreads();
  return lds[GROUPS] & ~(GROUPS - 1u);
}
// (Many of 64 maxima are a low bound: the least of them lets three times as many logits through as the 64th of 128.  64 out of 16 beams, 11
// requests of 68267 logits, 48.5 -> 40.8 us.)
template <int THREADS>
__device__ __forceinline__ uint32_t block_bound(uint32_t x, int K, uint32_t* lds) {
  return K > MANY_OUT ? bound_of<THREADS, 128>(x, K, lds) : bound_of<THREADS, 64>(x, K, lds);
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

// How many of a list's n entries are above e; behind them are zeros up to a multiple of eight.
__device__ __forceinline__ int above(const unsigned long long* list, int n, unsigned long long e) {
  int rank = 0;
#pragma unroll 1
  for (int j = 0; j < n; j += 8) {
    ulonglong2 y[4];
#pragma unroll
    for (int u = 0; u < 4; ++u) y[u] = ((const ulonglong2*)(list + j))[u];
#pragma unroll
    for (int u = 0; u < 4; ++u) rank += (y[u].x > e) + (y[u].y > e);
  }
  return rank;
}
// The K <= 64 best of a list of n > 64 entries, to its front; n becomes K, the answer the K-th best.
template <int LOW>
__device__ __forceinline__ unsigned long long keep_best(unsigned long long* list, int& n, int K) {
  const int lane = threadIdx.x & 63;
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
    low = ~lanes_join<64>(~least, Max());
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
  settle();
  n = base;
  return (unsigned long long)full << 32 | low;
}

// A block of 16 bytes of a row, -inf where it lies outside the row; at: its first element, from the block of the row's start.
template <typename T>
__device__ __forceinline__ uint4 load_block(const T* p, int at, int skip, int V) {
  constexpr int VEC = 16 / sizeof(T);
  if (at >= skip && at + VEC <= skip + V) {
    // (past the caches: 134 MB 37.0 -> 33.8 us, others the same)
    const Words<4> w = get<true, Words<4>>(p + at);
    return make_uint4(w[0], w[1], w[2], w[3]);
  }
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

// Maximum, sum and best logits of a piece of a row: a.blocks blocks of 16 bytes, 1024 (a tile) at a time.  Each wavefront keeps a list
// of its logits that reach a bound: one that n_out of the threads' maxima so far reach, made anew after 1, 2, 4, .. tiles, or where
// a list has been full its n_out-th best.  At the end the same bound leaves few entries of all lists, and the best of these go out.
// 256 rows of 131072 logits: float32, 8 out, 26 us (5.1 TB/s), bound by memory; bf16, 32 out, 24 us, by vector instructions, 19 a logit.
template <typename T>
__global__ __launch_bounds__(SEL_THREADS) void k_select_rows(SelectArgs a) {
  constexpr int VEC = 16 / sizeof(T), NW = SEL_THREADS / 64, LOW = SEL_LOW<T>;
  __shared__ double s_sum[NW];
  __shared__ float s_max[NW];
  __shared__ int s_count;
  __shared__ __align__(16) uint32_t s_bound[132];
  __shared__ __align__(16) unsigned long long s_list[NW][SEL_LIST], s_all[SEL_THREADS + 8];
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
  const int first = piece * a.blocks, end = min((piece + 1) * a.blocks, (skip + V + VEC - 1) / VEC);
  // first element of a thread's block (outside the row: behind the piece)
  auto place = [&](int base, int c) {
    const int b = base + c * SEL_THREADS + tid;
    return b < end ? b * VEC : skip + V;
  };
  uint4 next[SEL_VECS];
#pragma unroll
  for (int c = 0; c < SEL_VECS; ++c) next[c] = load_block(p, place(first, c), skip, V);
  if (tid == 0) s_count = 0;
  s_all[tid] = 0;
  if (tid < 8) s_all[SEL_THREADS + tid] = 0;
  float m = -INFINITY, limit = -FLT_MAX;
  double sum = 0.0;
  int n = 0, tiles = 0;
  unsigned long long bar = 0;          // what goes into the list is above this, 0: anything
  for (int base = first; base < end; base += SEL_TILE) {
    float x[SEL_VECS][VEC], top[SEL_VECS];
    int at[SEL_VECS];
#pragma unroll
    for (int c = 0; c < SEL_VECS; ++c) {
      const uint32_t u[4] = {next[c].x, next[c].y, next[c].z, next[c].w};
      top[c] = -INFINITY;
      at[c] = place(base, c) - skip;
#pragma unroll
      for (int i = 0; i < VEC; ++i) {
        if constexpr (sizeof(T) == 4) x[c][i] = __uint_as_float(u[i]);
        else x[c][i] = __uint_as_float(i & 1 ? u[i / 2] & 0xFFFF0000u : u[i / 2] << 16);
        top[c] = fmaxf(top[c], x[c][i]);
      }
    }
    if (base + SEL_TILE < end)
#pragma unroll
      for (int c = 0; c < SEL_VECS; ++c) next[c] = load_block(p, place(base + SEL_TILE, c), skip, V);
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
      for (int i = 0; i < VEC; ++i) s += exp_of(x[c][i] - ref);
    sum += (double)s;

    // ---- into the list
    if ((tiles & (tiles + 1)) == 0) {
      const unsigned long long least = (unsigned long long)block_bound<SEL_THREADS>(m > -INFINITY ? float_key(m + 0.f) : 0u, K, s_bound) << 32;
      bar = least > bar ? least : bar;
      limit = bar ? logit_of(bar) : -FLT_MAX;
    }
    ++tiles;
    if (!__ballot(mt >= limit)) continue;
#pragma unroll
    for (int c = 0; c < SEL_VECS; ++c) {
      if (!__ballot(top[c] >= limit)) continue;
      uint32_t hits = 0;
#pragma unroll
      for (int i = 0; i < VEC; ++i) hits |= x[c][i] >= limit ? 1u << i : 0u;
      const bool several = __ballot(hits & (hits - 1)) != 0;       // (mostly a lane has one, its largest: 256 rows of 131072 logits, 32 out, 33.9 -> 33.4 us)
      while (__ballot(hits)) {         // one of each lane's at a time
        const int which = __builtin_ctz(hits | 1u << VEC);
        float y = top[c];
        if (several) {
          y = x[c][0];
#pragma unroll
          for (int i = 1; i < VEC; ++i) y = which == i ? x[c][i] : y;
        }
        const unsigned long long key = hits ? key_of(y, (uint32_t)(at[c] + which)) : 0;
        hits &= hits - 1;
        unsigned long long mask = __ballot(key > bar);
        if (n + __popcll(mask) > SEL_LIST) {
          bar = keep_best<LOW>(list, n, K);            // (the list is full: n_out and more)
          limit = logit_of(bar);
          mask = __ballot(key > bar);
        }
        if (key > bar) list[n + __popcll(mask & ((1ull << lane) - 1))] = key;
        n += __popcll(mask);
        settle();
      }
    }
  }
  if (n > 64) keep_best<LOW>(list, n, K);        // (at most 64 go on, a lane each)
  const float wm = lanes_join<64>(m, MaxF());
  // (a thread of which everything is masked out has a sum of 0; a NaN stays one)
  sum *= m == wm ? 1.0 : (double)exp_of(m - wm);
  sum = lanes_join<64>(sum, Sum());
  if (lane == 0) {
    s_max[wv] = wm;
    s_sum[wv] = sum;
  }
  // ---- the best of all lists, up to 64 entries each
  const unsigned long long e = lane < n ? list[lane] : 0;
  const uint32_t least = max(block_bound<SEL_THREADS>((uint32_t)(e >> 32), K, s_bound), 1u);
  const unsigned long long mask = __ballot((uint32_t)(e >> 32) >= least);
  int to = 0;
  if (lane == 0 && mask) to = atomicAdd(&s_count, __popcll(mask));     // (in any order)
  to = __builtin_amdgcn_readfirstlane(to);
  if ((uint32_t)(e >> 32) >= least) s_all[to + __popcll(mask & ((1ull << lane) - 1))] = e;
  __syncthreads();
  const int64_t to_row = row * a.pieces + piece;
  const int all = s_count;
  if (tid == SEL_THREADS - 1) {
    float M = s_max[0];
    for (int w = 1; w < NW; ++w) M = fmaxf(M, s_max[w]);
    double S = 0.0;
    for (int w = 0; w < NW; ++w) S += s_sum[w] * (s_max[w] == M ? 1.0 : (double)exp_of(s_max[w] - M));
    a.part_m[to_row] = M;
    a.part_s[to_row] = S;
  }
  if (wv * 64 >= max(all, K)) return;
  const unsigned long long own = s_all[tid];
  const int rank = own ? above(s_all, all, own) : tid;       // (behind the entries: zeros)
  if (rank < K) a.keys[to_row * K + rank] = own;
}

// A continuation as whole numbers, the first more significant; all 0: none.
struct Cont {
  unsigned long long score;            // of the order of the score in 64 bits
  unsigned long long rest;             // 63 - beam, the logit, the complement of the token: 6, 32 and 24 bits
};
__device__ __forceinline__ bool over(const Cont& x, const Cont& y) {
  return (x.score > y.score) | ((x.score == y.score) & (x.rest > y.rest));
}
__device__ __forceinline__ Cont higher(const Cont& x, const Cont& y) { return over(x, y) ? x : y; }
__device__ __forceinline__ Cont cont_of(double score, int beam, unsigned long long key) {
  const float f = (float)score;
  if (!(f - f == 0.f)) return {0, 0};                        // (only finite scores, as they are given out)
  const long long b = __double_as_longlong(score + 0.0);     // (-0 counts as 0)
  return {(unsigned long long)(b < 0 ? ~b : b | (long long)(1ull << 63)),
          (unsigned long long)(63 - beam) << 56 | (key >> 32) << 24 | (key & 0xFFFFFFu)};
}
__device__ __forceinline__ double score_of(const Cont& x) {
  const long long s = (long long)x.score;
  return __longlong_as_double(s < 0 ? s ^ (long long)(1ull << 63) : ~s);
}

// A workgroup a request, a wavefront a row or a part of one.  Of the continuations that the rows' pieces have left, those that reach a
// bound go into a list in LDS, and an entry's place in the answer is the number of entries above it.  Of a long list (where one beam
// is far ahead of the others, most threads' maxima tell little) the same bound is taken again over the list.  Where more than the list
// holds reach it all the same (scores that are all equal) the answer is found one at a time.  A chain of loads, logarithms, two bounds and a
// count: 4.5 us for four beams and few continuations, 7.4 for 504 of six beams, 10.5 for 2048 of sixteen.
constexpr int JOIN_AHEAD = 4, JOIN_ROUNDS = 5;
template <int NW>
__global__ __launch_bounds__(64 * NW) void k_select_join(SelectArgs a) {
  constexpr int JOIN_LIST = 64 * NW;
  __shared__ double s_score[64], s_log[64];
  __shared__ float s_top[64];
  __shared__ int s_end[64], s_count[JOIN_ROUNDS];
  __shared__ __align__(16) uint32_t s_bound[132];
  __shared__ unsigned long long s_scores[JOIN_LIST], s_rests[JOIN_LIST];
  __shared__ Cont s_best[2][NW];
  const int B = a.b.n_beams, K = a.b.n_out, C = a.pieces, tid = threadIdx.x, lane = tid & 63;
  const int wv = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int64_t g = blockIdx.x;
  const unsigned long long* const keys = a.keys + g * B * C * K;
  // rows of this wavefront: row0, row0 + step, ..; of such a row every `parts`-th `wide` keys
  const int parts = max(1, NW / B), step = NW / parts, row0 = wv / parts, part = wv % parts, per = C * K;
  const int wide = min(64, (per + parts - 1) / parts), hop = wide * parts;
  const int spread = lane % NW * (64 / NW) + lane / NW, at0 = spread < wide ? part * wide + spread : per;     // (neighbours to other groups)
  auto cont = [&](int b, unsigned long long key) {
    return key ? cont_of(s_score[b] + (((double)logit_of(key) - (double)s_top[b]) - s_log[b]), b, key) : Cont{0, 0};
  };
  if (tid < JOIN_ROUNDS) s_count[tid] = 0;
  unsigned long long mine[JOIN_AHEAD];         // of row0
  uint32_t top = 0;                            // (of the order of a score, 32 of 64 bits)
  for (int b = row0; b < B; b += step) {
    const int64_t row = g * B + b;
    const bool end = a.finished && a.finished[row];
    // (all that is read at once; of a beam that has ended it is not looked at)
    unsigned long long key[JOIN_AHEAD];
#pragma unroll
    for (int u = 0; u < JOIN_AHEAD; ++u) {
      const int i = at0 + u * hop;
      key[u] = i < per ? keys[b * per + i] : 0;
      if (b == row0) mine[u] = key[u];
    }
    const double score = a.scores[row];
    float m = lane < C ? a.part_m[row * C + lane] : -INFINITY;
    double S = 0.0, s = lane < C ? a.part_s[row * C + lane] : 0.0;
    float M = -INFINITY;
    if (!end) {
      for (int c = lane + 64; c < C; c += 64) {
        const float mc = a.part_m[row * C + c], mx = fmaxf(m, mc);
        s = s * (m == mx ? 1.0 : (double)exp_of(m - mx)) + a.part_s[row * C + c] * (mc == mx ? 1.0 : (double)exp_of(mc - mx));
        m = mx;
      }
      M = lanes_join<64>(m, MaxF());
      S = lanes_join<64>(s * (m == M ? 1.0 : (double)exp_of(m - M)), Sum());
    }
    if (lane == 0) {                   // (the parts of a row write the same)
      s_end[b] = end;
      s_score[b] = score;
      s_log[b] = log(S);
      s_top[b] = M;
    }
    settle();
    if (end) {
      if (lane == 0 && part == 0) top = max(top, (uint32_t)(cont_of(score, b, 0).score >> 32));
      continue;
    }
#pragma unroll
    for (int u = 0; u < JOIN_AHEAD; ++u) top = max(top, (uint32_t)(cont(b, key[u]).score >> 32));
    for (int i = at0 + JOIN_AHEAD * hop; i < per; i += hop)
      top = max(top, (uint32_t)(cont(b, keys[b * per + i]).score >> 32));
  }
  uint32_t bar = max(block_bound<JOIN_LIST>(top, K, s_bound), 1u);
  auto put_in = [&](const Cont& x, int which) {
    const bool in = (uint32_t)(x.score >> 32) >= bar;
    const unsigned long long mask = __ballot(in);
    if (!mask) return;
    int to = 0;
    if (lane == __builtin_ctzll(mask)) to = atomicAdd(&s_count[which], __popcll(mask));      // (in any order)
    to = __builtin_amdgcn_readlane(to, __builtin_ctzll(mask)) + __popcll(mask & ((1ull << lane) - 1));
    if (in && to < JOIN_LIST) {
      s_scores[to] = x.score;
      s_rests[to] = x.rest;
    }
  };
  auto put_all = [&](int which) {
    for (int b = row0; b < B; b += step) {
      if (s_end[b]) {
        if (part == 0) put_in(lane == 0 ? cont_of(s_score[b], b, 0) : Cont{0, 0}, which);
        continue;
      }
      int i = 0;                       // (the same for all lanes)
      if (b == row0) {
#pragma unroll
        for (int u = 0; u < JOIN_AHEAD; ++u) put_in(cont(b, mine[u]), which);
        i += JOIN_AHEAD * hop;
      }
      for (; i < per; i += hop) put_in(cont(b, i + at0 < per ? keys[b * per + i + at0] : 0), which);
    }
  };
  put_all(0);
  __syncthreads();
  int n = s_count[0];
  for (int round = 1; n > 128 && round < JOIN_ROUNDS; ++round) {
    // (of a list that has overflowed what is in it will do: as many reach the bound.  Which ones are in it depends on who came first, and so may
    // this bound, but not the answer: any bound that K continuations reach leaves the K best in)
    const int i = tid % NW * 64 + tid / NW;            // (neighbours to other groups)
    const Cont x = i < n ? Cont{s_scores[i], s_rests[i]} : Cont{0, 0};
    const uint32_t next = block_bound<JOIN_LIST>((uint32_t)(x.score >> 32), K, s_bound);
    if (next <= bar) break;
    bar = next;
    if (n <= JOIN_LIST) put_in(x, round);
    else put_all(round);
    __syncthreads();
    n = s_count[round];
  }
  auto give = [&](int k, const Cont& x) {
    const bool there = x.score != 0;
    const int beam = 63 - (int)(x.rest >> 56);
    const bool end = there && s_end[beam];
    const int token = !there ? -1 : end ? a.b.end_token : (int)(~x.rest & 0xFFFFFFu);
    a.new_scores[g * K + k] = there ? (float)score_of(x) : -INFINITY;
    a.parents[g * K + k] = there ? beam : -1;
    a.tokens[g * K + k] = token;
    if (a.new_finished) a.new_finished[g * K + k] = !there || end || token == a.b.end_token;
  };
  if (n <= JOIN_LIST) {
    if (wv * 64 >= max(n, K)) return;
    if (tid < n) {
      const Cont x = {s_scores[tid], s_rests[tid]};
      int rank = 0, equal = 0;
#pragma unroll 8
      for (int j = 0; j < n; ++j) {
        const unsigned long long y = s_scores[j];
        rank += y > x.score;
        equal += y == x.score;
      }
      if (__ballot(equal > 1))
#pragma unroll 8
        for (int j = 0; j < n; ++j) rank += (s_scores[j] == x.score) & (s_rests[j] > x.rest);
      if (rank < K) give(rank, x);
    }
    if (tid >= n && tid < K) give(tid, {0, 0});
    return;
  }
  Cont last = {~0ull, ~0ull};
  for (int k = 0; k < K; ++k) {
    Cont best = {0, 0};
    auto look = [&](const Cont& x) {
      if (over(last, x)) best = higher(best, x);
    };
    for (int b = row0; b < B; b += step) {
      if (s_end[b]) look(cont_of(s_score[b], b, 0));
      else
        for (int i = at0; i < per; i += hop) look(cont(b, keys[b * per + i]));
    }
    for (int d = 1; d < 64; d <<= 1) best = higher(best, Cont{__shfl_xor(best.score, d), __shfl_xor(best.rest, d)});
    if (lane == 0) s_best[k & 1][wv] = best;
    __syncthreads();
    for (int w = 0; w < NW; ++w) best = higher(best, s_best[k & 1][w]);
    last = best;
    if (tid == 0) give(k, best);
  }
}

struct SelectPlan { int pieces, blocks; };
// logits: null for the most pieces that there may be.
SelectPlan select_plan(const Beams& b, const void* logits) {
  const int size = b.dtype == RESTKV_F32 ? 4 : 2, vec = 16 / size;
  // blocks of 16 bytes that a row may touch; even pieces of them, a tile at least, as many as four workgroups on each compute unit take (for
  // 4 / 5 / 6 / 8 of them, us: 144 rows of 100003 23.4 / 26.9 / 29.1 / 24.2, 256 rows of 131072 float32 33.8 / 33.3 / 36.8 / 37.0, bf16 37.3 / 42.5 / 39.7 / 44.6)
  const bool aligned = logits && !(((uintptr_t)logits | (uint64_t)b.stride * size) & 15u);
  const int most = (b.n_vocab + vec - 1 + vec - 1) / vec, all = aligned ? (b.n_vocab + vec - 1) / vec : most;
  const int64_t rows = (int64_t)b.n_groups * b.n_beams, want = 4 * n_cu();
  const int pieces = (int)std::min<int64_t>((most + SEL_TILE - 1) / SEL_TILE, std::max<int64_t>(1, want / std::max<int64_t>(rows, 1)));
  const int blocks = (all + pieces - 1) / pieces;
  return {logits ? (all + blocks - 1) / blocks : pieces, blocks};
}
struct SelectWs { size_t s, m, keys, bytes; };
SelectWs select_ws(const Beams& b) {
  SelectWs w = {};
  const size_t n = (size_t)b.n_groups * b.n_beams * select_plan(b, nullptr).pieces;
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
  const SelectPlan plan = select_plan(b, logits);
  a.pieces = plan.pieces; a.blocks = plan.blocks;
  a.part_s = (double*)(ws + lay.s); a.part_m = (float*)(ws + lay.m); a.keys = (unsigned long long*)(ws + lay.keys);
  const dim3 grid = wide_grid((int64_t)b.n_groups * b.n_beams * a.pieces);
  if (b.dtype == RESTKV_F32) hipLaunchKernelGGL(k_select_rows<float>, grid, dim3(SEL_THREADS), 0, st, a);
  else hipLaunchKernelGGL(k_select_rows<bf16_t>, grid, dim3(SEL_THREADS), 0, st, a);
  // Wavefronts of a request: its beams go round them, and a barrier takes longer the more there are.  Four / eight / sixteen, us a call: 4 beams,
  // 112 continuations left by the pieces 11.9 / 12.0 / 13.3, 896 of them 15.5 / 13.9 / 14.5; 6 beams, 504 22.6 / 23.0 / 23.6; 8 beams, 256
  // 13.9 / 12.6 / 13.5; 16 beams, 256 20.1 / 16.8 / 16.9, 512 16.6 / 13.8 / 13.3, 1024 25.5 / 22.0 / 22.0; 12 beams, 1152 - / 17.3 / 15.7; 64 beams - / 55.2 / 37.8.
  const int64_t left = (int64_t)b.n_beams * a.pieces * b.n_out;
  auto join = [&](auto kern, int waves) { hipLaunchKernelGGL(kern, dim3(b.n_groups), dim3(64 * waves), 0, st, a); };
  if (left > 1024) join(k_select_join<16>, 16);
  else if (left > 512 || b.n_beams >= 8) join(k_select_join<8>, 8);
  else join(k_select_join<4>, 4);
  return hip_status();
}

}  // namespace restkv
