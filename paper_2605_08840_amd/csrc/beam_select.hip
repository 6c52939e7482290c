// The best continuations of each request's beams: score(b, v) = c[b] + (x[b, v] - m_b) - ln sum exp(x[b, .] - m_b).
// One pass over the logits: a workgroup takes a piece of a row and leaves its maximum, its sum of exponentials and its n_out best
// logits; a second launch joins the pieces of a request's rows.  Bound by memory, every logit read once.
#include "beams.hpp"

namespace restkv {

namespace {

constexpr int SEL_THREADS = 256, SEL_VECS = 4;       // 16-byte loads of a thread

struct SelectArgs {
  Beams b;
  const void* logits;
  const float* scores; const int32_t* finished;
  float* new_scores; int32_t* parents; int32_t* tokens; int32_t* new_finished;
  int pieces;
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

template <typename T>
__global__ __launch_bounds__(SEL_THREADS) void k_select_rows(SelectArgs a) {
  constexpr int VEC = 16 / sizeof(T), NW = SEL_THREADS / 64;
  __shared__ double s_sum[NW];
  __shared__ float s_max[NW];
  __shared__ unsigned long long s_best[2][NW];
  const int64_t id = wide_block();
  const int64_t row = id / a.pieces;
  const int piece = (int)(id % a.pieces), V = a.b.n_vocab, K = a.b.n_out, tid = threadIdx.x, wv = tid >> 6;
  if (row >= (int64_t)a.b.n_groups * a.b.n_beams || (a.finished && a.finished[row])) return;
  // blocks of 16 bytes as the memory has them; block 0 holds the row's first element, `skip` elements in
  const T* p = (const T*)a.logits + row * a.b.stride;
  const int skip = (int)((uintptr_t)p / sizeof(T) % VEC);
  p -= skip;
  float x[SEL_VECS][VEC];
  int first[SEL_VECS];
  float m = -INFINITY;
#pragma unroll
  for (int c = 0; c < SEL_VECS; ++c) {
    const int at = ((piece * SEL_VECS + c) * SEL_THREADS + tid) * VEC;       // element of the first block's start
    first[c] = at - skip;
    if (at >= skip && at + VEC <= skip + V) {
      const uint4 w = *(const uint4*)(p + at);
      const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
      for (int i = 0; i < VEC; ++i) {
        if constexpr (sizeof(T) == 4) x[c][i] = __uint_as_float(u[i]);
        else x[c][i] = __uint_as_float(i & 1 ? u[i / 2] & 0xFFFF0000u : u[i / 2] << 16);
      }
    } else {
#pragma unroll
      for (int i = 0; i < VEC; ++i) x[c][i] = at + i >= skip && at + i < skip + V ? to_float(p[at + i]) : -INFINITY;
    }
#pragma unroll
    for (int i = 0; i < VEC; ++i) m = fmaxf(m, x[c][i]);
  }
  float sum = 0.f;
  const float ref = m == -INFINITY ? 0.f : m;
#pragma unroll
  for (int c = 0; c < SEL_VECS; ++c)
#pragma unroll
    for (int i = 0; i < VEC; ++i) sum += expf(x[c][i] - ref);
  const float wm = wave_join(m, [](float p, float q) { return fmaxf(p, q); });
  // (a thread of which everything is masked out has a sum of 0; a NaN stays one)
  double s = (double)sum * exp(m == wm ? 0.0 : (double)m - (double)wm);
  s = wave_join(s, [](double p, double q) { return p + q; });
  if ((tid & 63) == 0) {
    s_max[wv] = wm;
    s_sum[wv] = s;
  }
  __syncthreads();
  const int64_t at = row * a.pieces + piece;
  if (tid == 0) {
    float M = s_max[0];
    for (int w = 1; w < NW; ++w) M = fmaxf(M, s_max[w]);
    double S = 0.0;
    for (int w = 0; w < NW; ++w) S += s_sum[w] * exp(s_max[w] == M ? 0.0 : (double)s_max[w] - (double)M);
    a.part_m[at] = M;
    a.part_s[at] = S;
  }
  // the best one at a time
  unsigned long long last = ~0ull;
  for (int k = 0; k < K; ++k) {
    unsigned long long best = 0;
    if (last)
#pragma unroll
      for (int c = 0; c < SEL_VECS; ++c)
#pragma unroll
        for (int i = 0; i < VEC; ++i) {
          const unsigned long long key = key_of(x[c][i], (uint32_t)(first[c] + i));
          best = key < last && key > best ? key : best;
        }
    best = wave_join(best, [](unsigned long long p, unsigned long long q) { return p > q ? p : q; });
    if ((tid & 63) == 0) s_best[k & 1][wv] = best;
    __syncthreads();
    for (int w = 0; w < NW; ++w) best = s_best[k & 1][w] > best ? s_best[k & 1][w] : best;
    if (tid == 0) a.keys[at * K + k] = best;
    last = best;
  }
}

// A continuation: larger first.
struct Cont { double score; int beam; unsigned long long key; };
__device__ __forceinline__ bool before(const Cont& x, const Cont& y) {
  return x.score > y.score || (x.score == y.score && (x.beam < y.beam || (x.beam == y.beam && x.key > y.key)));
}
__device__ __forceinline__ Cont better(const Cont& x, const Cont& y) { return before(x, y) ? x : y; }

__global__ __launch_bounds__(256) void k_select_join(SelectArgs a) {
  constexpr int NW = 4;
  __shared__ double s_score[64], s_log[64];
  __shared__ float s_top[64];
  __shared__ int s_end[64];
  __shared__ Cont s_best[2][NW];
  const int B = a.b.n_beams, K = a.b.n_out, C = a.pieces, tid = threadIdx.x, wv = tid >> 6, lane = tid & 63;
  const int64_t g = blockIdx.x;
  for (int b = wv; b < B; b += NW) {
    const int64_t row = g * B + b;
    const bool end = a.finished && a.finished[row];
    double S = 0.0;
    float M = -INFINITY;
    if (!end) {
      for (int c = lane; c < C; c += 64) M = fmaxf(M, a.part_m[row * C + c]);
      M = wave_join(M, [](float p, float q) { return fmaxf(p, q); });
      for (int c = lane; c < C; c += 64) {
        const float m = a.part_m[row * C + c];
        S += a.part_s[row * C + c] * exp(m == M ? 0.0 : (double)m - (double)M);
      }
      S = wave_join(S, [](double p, double q) { return p + q; });
    }
    if (lane == 0) {
      s_score[b] = a.scores[row];
      s_log[b] = log(S);
      s_top[b] = M;
      s_end[b] = end;
    }
  }
  __syncthreads();
  const Cont none = {-INFINITY, 1 << 30, 0};
  Cont last = {INFINITY, -1, ~0ull};
  for (int k = 0; k < K; ++k) {
    Cont best = none;
    for (int i = tid; i < B * C * K; i += 256) {
      const int b = i / (C * K);
      Cont x = {-INFINITY, b, 0};
      if (s_end[b]) {
        if (i == b * C * K) x = {s_score[b], b, (unsigned long long)(uint32_t)~a.b.end_token};
      } else if (const unsigned long long key = a.keys[(g * B) * C * K + i]) {
        x = {s_score[b] + (((double)logit_of(key) - (double)s_top[b]) - s_log[b]), b, key};
      }
      if (x.score - x.score == 0.0 && before(last, x)) best = better(best, x);
    }
    for (int d = 1; d < 64; d <<= 1) {
      const Cont o = {__shfl_xor(best.score, d), __shfl_xor(best.beam, d), __shfl_xor(best.key, d)};
      best = better(best, o);
    }
    if (lane == 0) s_best[k & 1][wv] = best;
    __syncthreads();
    for (int w = 0; w < NW; ++w) best = better(best, s_best[k & 1][w]);
    last = best;
    if (tid == 0) {
      const bool there = best.score > -INFINITY;
      const int token = there ? (int)token_of(best.key) : -1;
      a.new_scores[g * K + k] = (float)best.score;
      a.parents[g * K + k] = there ? best.beam : -1;
      a.tokens[g * K + k] = token;
      if (a.new_finished) a.new_finished[g * K + k] = !there || token == a.b.end_token || s_end[best.beam];
    }
  }
}

int pieces_of(const Beams& b) {
  const int vec = b.dtype == RESTKV_F32 ? 4 : 8, per = SEL_THREADS * SEL_VECS;
  return (b.n_vocab / vec + 2 + per - 1) / per;       // (blocks of 16 bytes that a row may touch)
}
struct SelectWs { size_t s, m, keys, bytes; };
SelectWs select_ws(const Beams& b) {
  SelectWs w = {};
  const size_t n = (size_t)b.n_groups * b.n_beams * pieces_of(b);
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
  a.pieces = pieces_of(b);
  a.part_s = (double*)(ws + lay.s); a.part_m = (float*)(ws + lay.m); a.keys = (unsigned long long*)(ws + lay.keys);
  const dim3 grid = wide_grid((int64_t)b.n_groups * b.n_beams * a.pieces);
  if (b.dtype == RESTKV_F32) hipLaunchKernelGGL(k_select_rows<float>, grid, dim3(SEL_THREADS), 0, st, a);
  else hipLaunchKernelGGL(k_select_rows<bf16_t>, grid, dim3(SEL_THREADS), 0, st, a);
  hipLaunchKernelGGL(k_select_join, dim3(b.n_groups), dim3(256), 0, st, a);
  return hip_status();
}

}  // namespace restkv
