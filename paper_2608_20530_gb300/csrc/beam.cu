// Beam search: the n best (beam, token) pairs of each request, and the beams' states moved to the
// beams that continue them.
//
// Selection from logits takes two launches.
//   (1) beam_stream_kernel reads every live row once, in chunks of 32 x 4 vectors of 16 bytes, one
//       warp a chunk, and leaves each chunk's largest logit and the row's sum of exponentials.
//   (2) beam_choose_kernel, one CTA a request, forms the rows' normalisers, takes the n chunks whose
//       largest totals (score + logit - normaliser) come first, reads those chunks again and ranks
//       their elements. No other chunk can hold one of the n best: each of the n chunks taken has an
//       element that goes before everything in a chunk not taken (a larger total, or an equal one at
//       a lower beam or id, chunks being runs of ids).
// So the pass over the vocabulary carries no candidates, only a maximum that the sum needs anyway.
// Totals are 64-bit sums and the normalisers good to about 1e-8: beams whose totals differ by less
// than an fp32 rounding of either normaliser are still told apart.
#include <math.h>

#include "internal.cuh"

namespace lilicorr {

namespace {

constexpr unsigned FULL = 0xffffffffu;
constexpr int BM_THREADS = 128;
constexpr int BM_CAND = LILICORR_MAX_BEAMS * LILICORR_MAX_K;
constexpr float LOG2E = 1.4426950408889634f;
constexpr float LOG2E_LO = 1.92596299e-8f;     // log2(e) - LOG2E

// Order-preserving image of a double that is not NaN; 0 is never one (it marks "no candidate").
__device__ __forceinline__ uint64_t ord64(double v) {
  const uint64_t b = (uint64_t)__double_as_longlong(v + 0.0);      // -0 to +0
  return (b >> 63) ? ~b : (b | (1ull << 63));
}
__device__ __forceinline__ double unord64(uint64_t o) {
  return __longlong_as_double((long long)((o >> 63) ? (o & ~(1ull << 63)) : ~o));
}
// a precedes b: larger total, then lower position
template <typename P>
__device__ __forceinline__ bool precedes(uint64_t ka, P pa, uint64_t kb, P pb) {
  return ka > kb || (ka == kb && pa < pb);
}

// The first n of `count` candidates in order: place(rank, key, position) for each; returns how many
// there are, up to n. near(i): candidate i's total in fp32, off by at most 2^-22 of |total| + `scale`,
// -inf for none; key(i) its 64-bit key (0: none).
//
// First a bound: 64 groups of threads put forward their best candidate (by near, one is as valid as
// another), and nothing below the n-th of those 64 can be among the first n. Only the few candidates
// that reach it get a 64-bit total (GB300 adds two of those a clock and SM) and are ranked against one
// another, four lanes a candidate. Where very many reach it (equal totals everywhere) the n are taken
// one after the other instead.
constexpr int RF_GROUPS = 64;
constexpr int RF_CAP = 1024;
struct RankShared {
  uint64_t key[RF_CAP], pos[RF_CAP];           // what reaches the bound
  uint64_t gkey[RF_GROUPS], gpos[RF_GROUPS];   // the groups' best
  uint64_t bound, bound_pos;
  int count;
};

template <int NT, class Near, class Key, class Pos, class Place>
__device__ __forceinline__ int rank_first(RankShared& sh, int count, int n, float scale, Near near,
                                          Key key, Pos pos, Place place) {
  constexpr int LPG = NT / RF_GROUPS;          // lanes a group
  static_assert(LPG >= 2 && LPG <= 32 && (LPG & (LPG - 1)) == 0 && RF_GROUPS >= LILICORR_MAX_K, "");
  const int tid = threadIdx.x;
  float floor = -INFINITY;
  uint64_t bound = 1ull, bound_pos = ~0ull;
  if (tid == 0) { sh.count = 0; sh.bound = 1ull; sh.bound_pos = ~0ull; }
  if (count > RF_GROUPS) {
    float best = -INFINITY;
    int at = -1;
    for (int i = tid; i < count; i += NT) {
      const float v = near(i);
      if (v > best) { best = v; at = i; }
    }
#pragma unroll
    for (int o = 1; o < LPG; o <<= 1) {
      const float v = __shfl_xor_sync(FULL, best, o);
      const int x = __shfl_xor_sync(FULL, at, o);
      if (v > best || (v == best && x > at)) { best = v; at = x; }
    }
    const int g = tid / LPG, in = tid % LPG;
    const uint64_t gk = at >= 0 ? key(at) : 0ull, gp = at >= 0 ? pos(at) : (uint64_t)g;
    if (in == 0) { sh.gkey[g] = gk; sh.gpos[g] = gp; }
    __syncthreads();
    int rank = 0;
#pragma unroll
    for (int j = 0; j < RF_GROUPS / LPG; ++j) {
      const int o = j * LPG + in;
      rank += precedes(sh.gkey[o], sh.gpos[o], gk, gp) ? 1 : 0;
    }
#pragma unroll
    for (int o = 1; o < LPG; o <<= 1) rank += __shfl_xor_sync(FULL, rank, o);
    if (in == 0 && gk && rank == n - 1) { sh.bound = gk; sh.bound_pos = gp; }
    __syncthreads();
    bound = sh.bound;
    bound_pos = sh.bound_pos;
    if (bound != 1ull) {
      const float b = (float)unord64(bound);
      floor = b - 0x1p-20f * (fabsf(b) + scale);
    }
  } else {
    __syncthreads();
  }
  for (int i = tid; i < count; i += NT) {
    const float v = near(i);
    if (!(v >= floor) || v == -INFINITY) continue;
    const uint64_t k = key(i), p = pos(i);
    if (!k || precedes(bound, bound_pos, k, p)) continue;
    const int at = atomicAdd(&sh.count, 1);
    if (at < RF_CAP) { sh.key[at] = k; sh.pos[at] = p; }
  }
  __syncthreads();
  const int m = sh.count;
  if (m <= RF_CAP) {
    const int in = tid & 3;
    for (int i0 = 0; i0 < m; i0 += NT / 4) {
      const int i = i0 + (tid >> 2);
      const uint64_t k = i < m ? sh.key[i] : ~0ull, p = i < m ? sh.pos[i] : 0ull;
      int rank = 0;
#pragma unroll 4
      for (int j = in; j < m; j += 4) rank += precedes(sh.key[j], sh.pos[j], k, p) ? 1 : 0;
      rank += __shfl_xor_sync(FULL, rank, 1);
      rank += __shfl_xor_sync(FULL, rank, 2);
      if (in == 0 && i < m && rank < n) place(rank, k, p);
    }
    return min(m, n);
  }
  uint64_t last = ~0ull, last_pos = 0ull;      // before every candidate
  for (int t = 0; t < n; ++t) {                // m > RF_CAP >= n: there is one each time
    uint64_t bk = 0ull, bp = ~0ull;
    for (int i = tid; i < count; i += NT) {
      if (near(i) == -INFINITY) continue;
      const uint64_t k = key(i), p = pos(i);
      if (k && precedes(last, last_pos, k, p) && precedes(k, p, bk, bp)) { bk = k; bp = p; }
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
      const uint64_t k = __shfl_xor_sync(FULL, bk, o), p = __shfl_xor_sync(FULL, bp, o);
      if (precedes(k, p, bk, bp)) { bk = k; bp = p; }
    }
    if ((tid & 31) == 0) { sh.gkey[tid >> 5] = bk; sh.gpos[tid >> 5] = bp; }
    __syncthreads();
    for (int w = 0; w < NT / 32; ++w)
      if (precedes(sh.gkey[w], sh.gpos[w], bk, bp)) { bk = sh.gkey[w]; bp = sh.gpos[w]; }
    if (tid == 0) place(t, bk, bp);
    last = bk;
    last_pos = bp;
    __syncthreads();
  }
  return n;
}

struct BeamOut {
  int32_t *tokens, *parents;
  float* next_scores;
  uint8_t* next_done;
  int32_t end_id;
  int n;
  __device__ void put(int r, int rank, uint64_t key, int w, int32_t token, bool over) const {
    const size_t at = (size_t)r * n + rank;
    tokens[at] = token;
    parents[at] = w;
    next_scores[at] = (float)unord64(key);
    if (next_done) next_done[at] = over || (end_id >= 0 && token == end_id);
  }
  __device__ void none(int r, int rank) const {
    const size_t at = (size_t)r * n + rank;
    tokens[at] = -1;
    parents[at] = -1;
    next_scores[at] = -INFINITY;
    if (next_done) next_done[at] = 0;
  }
};

// A total's key: 0 (and `bad`) for NaN and +inf, 0 for -inf.
__device__ __forceinline__ uint64_t total_key(double total, bool& bad) {
  if (!(total < INFINITY)) { bad = true; return 0ull; }
  return total > -INFINITY ? ord64(total) : 0ull;
}

// Candidate lists: one CTA a request.
__global__ void __launch_bounds__(BM_THREADS)
beam_merge_kernel(const int32_t* __restrict__ ids, const float* __restrict__ logp, int W, int K,
                  const float* __restrict__ scores, const uint8_t* __restrict__ done, BeamOut out,
                  uint32_t* status) {
  pdl_wait();
  __shared__ uint64_t s_key[BM_CAND];
  __shared__ float s_near[BM_CAND];
  __shared__ RankShared sh;
  const int tid = threadIdx.x, r = blockIdx.x, M = W * K;
  const size_t row0 = (size_t)r * W;
  bool bad = false;
  for (int i = tid; i < M; i += BM_THREADS) {
    const int w = i / K;
    const float sc = scores[row0 + w], lp = logp[row0 * K + i];
    double total = -INFINITY;
    if (done && done[row0 + w]) {
      if (i == w * K) total = (double)sc;
    } else if (sc != -INFINITY) {
      total = (double)sc + (double)lp;
    }
    const uint64_t key = total_key(total, bad);
    s_key[i] = key;
    s_near[i] = key ? (float)total : -INFINITY;
  }
  if (bad) set_status(status, LILICORR_ERR_NONFINITE);
  // (a thread reads back what it wrote, but for its group's best)
  __syncthreads();
  const int m = rank_first<BM_THREADS>(
      sh, M, out.n, 0.f, [&](int i) { return s_near[i]; }, [&](int i) { return s_key[i]; },
      [&](int i) { return (uint64_t)i; },
      [&](int rank, uint64_t key, uint64_t p) {
        const int w = (int)p / K;
        const bool over = done && done[row0 + w];
        out.put(r, rank, key, w, over ? out.end_id : ids[row0 * K + p], over);
      });
  for (int i = m + tid; i < out.n; i += BM_THREADS) out.none(r, i);      // fewer candidates than n
}

// ---------------------------------------------------------------------------- from logits
constexpr int BS_THREADS = 256;                // of the streaming kernel
constexpr int BS_U = 4;                        // 16-byte vectors per lane and chunk
constexpr int BC_THREADS = 256;                // of the choosing kernel

// How rows are cut: chunk 0 of a row holds the ids before its first 16-byte boundary where rows need
// not start on one (`odd`), the others runs of `size` ids; warp i of the streaming kernel takes the
// chunks [i * per_warp, (i + 1) * per_warp) of all rows, and leaves a record for each row among them.
struct BeamCut {
  int V, vec, size, odd, chunks;               // chunks per row
  int per_warp, slots;                         // records per row
  __host__ __device__ int head(size_t row) const {
    if (!odd) return 0;
    const int h = (int)((vec - (row * (size_t)V) % vec) % vec);
    return h < V ? h : V;
  }
  // ids [begin, end) of chunk c
  __host__ __device__ void range(size_t row, int c, int& begin, int& end) const {
    const int h = head(row);
    if (odd && c == 0) { begin = 0; end = h; return; }
    const long long b = h + (long long)(c - odd) * size, e = b + size;
    begin = b < V ? (int)b : V;
    end = e < V ? (int)e : V;
  }
};

BeamCut beam_cut(int rows, int V, lilicorr_dtype_t dt) {
  BeamCut c;
  c.V = V;
  c.vec = dt == LILICORR_BF16 ? 8 : 4;
  c.size = 32 * BS_U * c.vec;
  c.odd = V % c.vec != 0;
  c.chunks = ceil_div(V, c.size) + c.odd;
  // one wave of 32 warps an SM
  const long long total = (long long)rows * c.chunks, warps = 32ll * num_sms();
  c.per_warp = (int)((total + warps - 1) / warps);
  if (c.per_warp < 1) c.per_warp = 1;
  c.slots = (c.chunks + c.per_warp - 1) / c.per_warp + 1;
  return c;
}

// A row's sum of exponentials over some chunks: s in units of 2^e, e a whole number (-inf: nothing
// but -inf was met, s 0, or NaN). A whole power of two as the reference makes every rescale exact.
struct SumRec {
  double s;
  float e;
  float pad;
};

// 2^d of a whole number d <= 0 (0 below the normal range and for -inf)
__device__ __forceinline__ float pow2_whole(float d) {
  return d < -126.f ? 0.f : __int_as_float((127 + (int)d) << 23);
}
__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ uint64_t pack2(float lo, float hi) {
  uint64_t r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(lo), "f"(hi));
  return r;
}
__device__ __forceinline__ void unpack2(uint64_t v, float& lo, float& hi) {
  asm("mov.b64 {%0, %1}, %2;" : "=f"(lo), "=f"(hi) : "l"(v));
}
__device__ __forceinline__ uint64_t fma2(uint64_t a, uint64_t b, uint64_t c) {
  uint64_t d;
  asm("fma.rn.ftz.f32x2 %0, %1, %2, %3;" : "=l"(d) : "l"(a), "l"(b), "l"(c));
  return d;
}
__device__ __forceinline__ uint64_t add2(uint64_t a, uint64_t b) {
  uint64_t d;
  asm("add.rn.ftz.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
  return d;
}
// order-preserving 32-bit image of a float (-0 below +0)
__device__ __forceinline__ uint32_t ord32(float v) {
  const uint32_t b = __float_as_uint(v);
  return (b & 0x80000000u) ? ~b : (b | 0x80000000u);
}
__device__ __forceinline__ float unord32(uint32_t o) {
  return __uint_as_float((o & 0x80000000u) ? (o & 0x7FFFFFFFu) : ~o);
}

// One vector of logits as words: bf16 pairs or floats.
template <typename T> struct Elem;
template <> struct Elem<uint16_t> {
  static constexpr int N = 8;
  static constexpr uint32_t NONE = 0xFF80FF80u;
  __device__ static void pair(const uint4& v, int i, float& a, float& b) {
    const uint32_t w = i == 0 ? v.x : i == 1 ? v.y : i == 2 ? v.z : v.w;
    a = __uint_as_float(w << 16);
    b = __uint_as_float(w & 0xFFFF0000u);
  }
  __device__ static float vmax(const uint4& v) {           // NaN ignored
    uint32_t m, n;
    asm("max.bf16x2 %0, %1, %2;" : "=r"(m) : "r"(v.x), "r"(v.y));
    asm("max.bf16x2 %0, %1, %2;" : "=r"(n) : "r"(v.z), "r"(v.w));
    asm("max.bf16x2 %0, %1, %2;" : "=r"(m) : "r"(m), "r"(n));
    return fmaxf(__uint_as_float(m << 16), __uint_as_float(m & 0xFFFF0000u));
  }
  __device__ static uint4 gather(const uint16_t* p, int live) {      // the first `live` of a vector
    uint32_t w[4] = {NONE, NONE, NONE, NONE};
#pragma unroll
    for (int j = 0; j < 8; ++j)
      if (j < live) {
        const uint32_t x = p[j];
        w[j >> 1] = (j & 1) ? (w[j >> 1] & 0xFFFFu) | (x << 16) : (w[j >> 1] & 0xFFFF0000u) | x;
      }
    return make_uint4(w[0], w[1], w[2], w[3]);
  }
};
template <> struct Elem<float> {
  static constexpr int N = 4;
  static constexpr uint32_t NONE = 0xFF800000u;
  __device__ static void pair(const uint4& v, int i, float& a, float& b) {
    a = __uint_as_float(i == 0 ? v.x : v.z);
    b = __uint_as_float(i == 0 ? v.y : v.w);
  }
  __device__ static float vmax(const uint4& v) {
    return fmaxf(fmaxf(__uint_as_float(v.x), __uint_as_float(v.y)),
                 fmaxf(__uint_as_float(v.z), __uint_as_float(v.w)));
  }
  __device__ static uint4 gather(const float* p, int live) {
    uint32_t w[4] = {NONE, NONE, NONE, NONE};
#pragma unroll
    for (int j = 0; j < 4; ++j)
      if (j < live) w[j] = __float_as_uint(p[j]);
    return make_uint4(w[0], w[1], w[2], w[3]);
  }
};

// A warp's share of ids [begin, end) of a row, -inf past the end. Vectors start on 16-byte
// boundaries, but for the row's head, which one lane takes.
template <typename T>
__device__ __forceinline__ void load_chunk(const T* __restrict__ row, int begin, int end, int lane,
                                           uint4 (&raw)[BS_U]) {
  constexpr int N = Elem<T>::N;
  constexpr uint32_t NI = Elem<T>::NONE;
  if (end - begin == 32 * BS_U * N) {
    const uint4* p = reinterpret_cast<const uint4*>(row + begin) + lane;
#pragma unroll
    for (int u = 0; u < BS_U; ++u) raw[u] = __ldcs(p + 32 * u);
    return;
  }
#pragma unroll
  for (int u = 0; u < BS_U; ++u) {
    const int at = begin + (u * 32 + lane) * N;
    raw[u] = make_uint4(NI, NI, NI, NI);
    if (at + N <= end) raw[u] = __ldcs(reinterpret_cast<const uint4*>(row + at));
    else if (at < end) raw[u] = Elem<T>::gather(row + at, end - at);
  }
}

// Bound by HBM: 16 bytes a lane and load, the next chunk's four in flight while this one is summed;
// no shared memory, no barrier.
template <typename T>
__global__ void __launch_bounds__(BS_THREADS, 1024 / BS_THREADS)
beam_stream_kernel(const T* __restrict__ logits, int rows, const float* __restrict__ scores,
                   const uint8_t* __restrict__ done, BeamCut cut, float* __restrict__ maxima,
                   SumRec* __restrict__ sums) {
  pdl_wait();
  const int lane = threadIdx.x & 31;
  const long long wid = (long long)blockIdx.x * (BS_THREADS / 32) + (threadIdx.x >> 5);
  const long long total = (long long)rows * cut.chunks;
  long long at = wid * cut.per_warp;
  const long long stop = min(total, at + cut.per_warp);
  while (at < stop) {
    const int row = (int)(at / cut.chunks);
    const int c0 = (int)(at - (long long)row * cut.chunks);
    const int c1 = (int)min((long long)cut.chunks, c0 + (stop - at));
    at += c1 - c0;
    if (!(scores[row] > -INFINITY) || (done && done[row])) continue;
    const T* rp = logits + (size_t)row * cut.V;
    float s = 0.f, lost = 0.f, e = -INFINITY;         // e is the same in all lanes
    uint4 cur[BS_U], nxt[BS_U];
    int b, en;
    cut.range(row, c0, b, en);
    load_chunk<T>(rp, b, en, lane, cur);
    for (int c = c0; c < c1; ++c) {
      if (c + 1 < c1) {
        cut.range(row, c + 1, b, en);
        load_chunk<T>(rp, b, en, lane, nxt);
      }
      float m = Elem<T>::vmax(cur[0]);
#pragma unroll
      for (int u = 1; u < BS_U; ++u) m = fmaxf(m, Elem<T>::vmax(cur[u]));
      m = unord32(__reduce_max_sync(FULL, ord32(m)));
      if (lane == 0) maxima[(size_t)row * cut.chunks + c] = m;
      const float ce = ceilf(m * LOG2E);
      if (ce > e) {
        const float f = e == -INFINITY ? 1.f : pow2_whole(e - ce);   // before: 0, or NaN
        s *= f;
        lost *= f;
        e = ce;
      }
      // arguments x log2(e) - e with log2(e) in two parts; -inf adds 0, NaN stays
      const float ref = e == -INFINITY ? 0.f : e;
      const uint64_t hi = pack2(LOG2E, LOG2E), lo = pack2(LOG2E_LO, LOG2E_LO), nm = pack2(-ref, -ref);
      uint64_t a0 = pack2(0.f, 0.f), a1 = a0;
#pragma unroll
      for (int u = 0; u < BS_U; ++u)
#pragma unroll
        for (int i = 0; i < Elem<T>::N / 2; ++i) {
          float x0, x1;
          Elem<T>::pair(cur[u], i, x0, x1);
          const uint64_t x = pack2(x0, x1);
          unpack2(fma2(x, lo, fma2(x, hi, nm)), x0, x1);
          const uint64_t p = pack2(ex2(x0), ex2(x1));
          if (i & 1) a1 = add2(a1, p); else a0 = add2(a0, p);
        }
      float p0, p1, p2, p3;
      unpack2(a0, p0, p1);
      unpack2(a1, p2, p3);
      // what the running sum's additions lose is kept beside it
      const float add = (p0 + p1) + (p2 + p3), t = s + add, bb = t - s;
      lost += (s - (t - bb)) + (add - bb);
      s = t;
#pragma unroll
      for (int u = 0; u < BS_U; ++u) cur[u] = nxt[u];
    }
    double d = (double)s + (double)lost;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) d += __shfl_xor_sync(FULL, d, o);
    if (lane == 0) {
      const long long first = (long long)row * cut.chunks / cut.per_warp;
      SumRec* rec = sums + (size_t)row * cut.slots + (wid - first);
      rec->s = d;
      rec->e = e;
    }
  }
}

// One CTA a request: normalisers, the n chunks to look at, their elements, the n best.
template <typename T>
__global__ void __launch_bounds__(BC_THREADS)
beam_choose_kernel(const T* __restrict__ logits, int W, const float* __restrict__ scores,
                   const uint8_t* __restrict__ done, BeamCut cut, const float* __restrict__ maxima,
                   const SumRec* __restrict__ sums, BeamOut out, uint32_t* status) {
  pdl_wait();
  constexpr int N = Elem<T>::N;
  constexpr int NW = BC_THREADS / 32;
  constexpr int CAND = LILICORR_MAX_K * LILICORR_MAX_K;
  __shared__ double s_lse[LILICORR_MAX_BEAMS];
  __shared__ float s_score[LILICORR_MAX_BEAMS];
  __shared__ uint8_t s_kind[LILICORR_MAX_BEAMS];        // 0 absent, 1 live, 2 done
  __shared__ float s_base[LILICORR_MAX_BEAMS];          // score - lse, to fp32
  __shared__ RankShared sh;
  __shared__ uint64_t s_ckey[LILICORR_MAX_K], s_cpos[LILICORR_MAX_K];
  __shared__ uint64_t s_key[CAND], s_at[CAND];
  __shared__ int s_cand;
  __shared__ uint32_t s_scale;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, r = blockIdx.x;
  const size_t row0 = (size_t)r * W;
  if (tid == 0) { s_cand = 0; s_scale = 0u; }
  __syncthreads();

  for (int w = warp; w < W; w += NW) {
    const float sc = scores[row0 + w];
    const size_t row = row0 + w;
    int kind = !(sc > -INFINITY) ? 0 : (done && done[row]) ? 2 : 1;
    bool bad = sc != sc || sc == INFINITY;
    double lse = 0.0;
    if (kind == 1) {
      const long long first = (long long)row * cut.chunks / cut.per_warp;
      const int count = (int)(((long long)(row + 1) * cut.chunks - 1) / cut.per_warp - first) + 1;
      float e = -INFINITY;
      double s = 0.0;
      for (int i = lane; i < count; i += 32) {
        const SumRec x = sums[row * cut.slots + i];
        const float big = fmaxf(e, x.e);
        s = (e == -INFINITY ? s : s * (double)pow2_whole(e - big)) +
            (x.e == -INFINITY ? x.s : x.s * (double)pow2_whole(x.e - big));
        e = big;
      }
      const float E = warp_max(e);
      s = e == -INFINITY ? s : s * (double)pow2_whole(e - E);
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(FULL, s, o);
      lse = (double)E * 0.69314718055994530942 + log(s);
      if (!isfinite(lse)) bad = true;
    }
    if (bad) kind = 0;
    if (lane == 0) {
      if (bad) set_status(status, LILICORR_ERR_NONFINITE);
      const float base = kind == 0 ? -INFINITY : (float)((double)sc - lse);
      s_lse[w] = lse;
      s_score[w] = sc;
      s_base[w] = base;
      s_kind[w] = (uint8_t)kind;
      if (kind) atomicMax(&s_scale, __float_as_uint(fabsf(base)));
    }
  }
  __syncthreads();

  // the first n chunks, by their largest total; a done beam is one chunk of one candidate
  const int M = W * cut.chunks;
  const float* mx = maxima + row0 * cut.chunks;
  bool ignore = false;
  const int taken = rank_first<BC_THREADS>(
      sh, M, out.n, __uint_as_float(s_scale),
      [&](int i) {
        const int w = i / cut.chunks;
        if (s_kind[w] == 2) return i == w * cut.chunks ? s_base[w] : -INFINITY;
        return s_kind[w] ? s_base[w] + mx[i] : -INFINITY;
      },
      [&](int i) -> uint64_t {
        const int w = i / cut.chunks;
        if (s_kind[w] == 2) return total_key((double)s_score[w], ignore);
        return total_key((double)s_score[w] + ((double)mx[i] - s_lse[w]), ignore);
      },
      [&](int i) { return (uint64_t)i; },
      [&](int rank, uint64_t key, uint64_t p) {
        s_ckey[rank] = key;
        s_cpos[rank] = p;
      });
  __syncthreads();
  const double least = taken == out.n ? unord64(s_ckey[taken - 1]) : -INFINITY;
  for (int c = warp; c < taken; c += NW) {
    const int i = (int)s_cpos[c], w = i / cut.chunks;
    const size_t row = row0 + w;
    if (s_kind[w] == 2) {
      if (lane == 0) {
        const int at = atomicAdd(&s_cand, 1);
        s_key[at] = s_ckey[c];
        s_at[at] = ((uint64_t)w << 32) | (uint32_t)out.end_id;
      }
      continue;
    }
    int b, en;
    cut.range(row, i - w * cut.chunks, b, en);
    uint4 raw[BS_U];
    load_chunk<T>(logits + row * cut.V, b, en, lane, raw);
    const double sc = (double)s_score[w], lse = s_lse[w];
    // an element whose total reaches `least`, by its logit with a margin for the rounding
    const double x0 = least - sc + lse;
    const float thr = x0 == -INFINITY ? -INFINITY : (float)(x0 - 1e-5 * (1.0 + fabs(x0)));
    uint32_t hot = 0;                                   // element j of vector u: bit u * N + j
#pragma unroll
    for (int u = 0; u < BS_U; ++u)
#pragma unroll
      for (int j = 0; j < N / 2; ++j) {
        float a, d;
        Elem<T>::pair(raw[u], j, a, d);
        hot |= (a >= thr && a > -INFINITY ? 1u : 0u) << (u * N + 2 * j);
        hot |= (d >= thr && d > -INFINITY ? 1u : 0u) << (u * N + 2 * j + 1);
      }
    auto value = [&](int bit) {
      float v = 0.f;
#pragma unroll
      for (int u = 0; u < BS_U; ++u)
#pragma unroll
        for (int j = 0; j < N / 2; ++j) {
          float a, d;
          Elem<T>::pair(raw[u], j, a, d);
          if (bit == u * N + 2 * j) v = a;
          if (bit == u * N + 2 * j + 1) v = d;
        }
      return v + 0.f;                                   // -0 to +0
    };
    const int hits = __reduce_add_sync(FULL, __popc(hot));
    if (hits > out.n) {
      // more than n in one chunk (equal logits, or a row that falls steadily): its n first, by a
      // search over the bits of the n-th largest value; of those equal to it the lowest ids
      uint32_t nth = 0;
      for (int bit = 31; bit >= 0; --bit) {
        const uint32_t t = nth | (1u << bit);
        int cnt = 0;
        for (uint32_t h = hot; h; h &= h - 1) cnt += ord32(value(__ffs(h) - 1)) >= t ? 1 : 0;
        if (__reduce_add_sync(FULL, cnt) >= out.n) nth = t;
      }
      uint32_t above = 0, equal = 0;
      for (uint32_t h = hot; h; h &= h - 1) {
        const int j = __ffs(h) - 1;
        const uint32_t o = ord32(value(j));
        if (o > nth) above |= 1u << j;
        if (o == nth) equal |= 1u << j;
      }
      int room = out.n - __reduce_add_sync(FULL, __popc(above));
      for (int u = 0; u < BS_U; ++u) {
        const uint32_t mask = ((N == 8 ? 0xFFu : 0xFu) << (u * N));
        const int mine = __popc(equal & mask);
        int before = mine;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
          const int x = __shfl_up_sync(FULL, before, o);
          if (lane >= o) before += x;
        }
        const int all = __shfl_sync(FULL, before, 31);
        int left = room - (before - mine);
        for (uint32_t h = equal & mask; h; h &= h - 1, --left)
          if (left <= 0) equal &= ~(1u << (__ffs(h) - 1));
        room -= all;
      }
      hot = above | equal;
    }
    for (uint32_t h = hot; h; h &= h - 1) {
      const int j = __ffs(h) - 1;
      const int at = atomicAdd(&s_cand, 1);
      bool no = false;
      s_key[at] = total_key(sc + ((double)value(j) - lse), no);
      s_at[at] = ((uint64_t)w << 32) | (uint32_t)(b + ((j / N) * 32 + lane) * N + j % N);
    }
  }
  __syncthreads();
  const int found = rank_first<BC_THREADS>(
      sh, s_cand, out.n, 0.f, [&](int i) { return (float)unord64(s_key[i]); },
      [&](int i) { return s_key[i]; }, [&](int i) { return s_at[i]; },
      [&](int rank, uint64_t key, uint64_t p) {
        const int w = (int)(p >> 32);
        out.put(r, rank, key, w, (int32_t)(uint32_t)p, s_kind[w] == 2);
      });
  for (int i = found + tid; i < out.n; i += BC_THREADS) out.none(r, i);  // fewer candidates than n
}

// ---------------------------------------------------------------------------- states
constexpr int BR_THREADS = 256;
constexpr int BR_STATES = 64;            // arrays per launch

struct Reorder {
  unsigned char* state[BR_STATES];
  int W, positions, heads;
  uint32_t pieces;                       // vectors per row
  int64_t s_req, s_beam, s_pos, s_head;
  const int32_t* parents;
  const int32_t* lengths;
};

// One (array, request) per grid row. A thread owns one vector-wide column of all W beams: it loads
// every beam that moves from its parent, then stores, so the move is in place without a second
// buffer and without a barrier: nobody else reads or writes its column.
template <typename V, int WMAX>
__global__ void __launch_bounds__(BR_THREADS)
beam_reorder_kernel(const __grid_constant__ Reorder a) {
  pdl_wait();
  __shared__ int s_parent[LILICORR_MAX_BEAMS];
  const int tid = threadIdx.x, r = blockIdx.y;
  if (tid < a.W) {
    const int p = a.parents[(size_t)r * a.W + tid];
    s_parent[tid] = (p < 0 || p >= a.W) ? tid : p;
  }
  __syncthreads();
  int len = a.positions;
  if (a.lengths) len = min(max(a.lengths[r], 0), a.positions);
  const uint32_t per_pos = (uint32_t)a.heads * a.pieces, total = (uint32_t)len * per_pos;
  unsigned char* base = a.state[blockIdx.z] + (int64_t)r * a.s_req;
  for (uint32_t u = blockIdx.x * BR_THREADS + tid; u < total; u += gridDim.x * BR_THREADS) {
    const uint32_t pos = u / per_pos, in = u - pos * per_pos, h = in / a.pieces, c = in - h * a.pieces;
    unsigned char* col = base + (int64_t)pos * a.s_pos + (int64_t)h * a.s_head + (int64_t)c * sizeof(V);
    V v[WMAX];
#pragma unroll
    for (int w = 0; w < WMAX; ++w)
      if (w < a.W && s_parent[w] != w)
        v[w] = *reinterpret_cast<const V*>(col + (int64_t)s_parent[w] * a.s_beam);
#pragma unroll
    for (int w = 0; w < WMAX; ++w)
      if (w < a.W && s_parent[w] != w) *reinterpret_cast<V*>(col + (int64_t)w * a.s_beam) = v[w];
  }
}

template <typename V>
lilicorr_status_t launch_reorder(const Reorder& a, int count, int requests, cudaStream_t st) {
  // CTAs for about four waves over all (array, request) pairs; the rest by the loop
  const long long most = (long long)a.positions * a.heads * a.pieces;
  const long long pairs = (long long)count * requests;
  long long x = (most + BR_THREADS - 1) / BR_THREADS;
  const long long want = (16ll * num_sms() + pairs - 1) / pairs;
  if (x > want) x = want;
  if (x < 1) x = 1;
  const dim3 grid((unsigned)x, (unsigned)requests, (unsigned)count);
  if (a.W <= 4) return launch_k(beam_reorder_kernel<V, 4>, grid, BR_THREADS, 0, st, a);
  if (a.W <= 8) return launch_k(beam_reorder_kernel<V, 8>, grid, BR_THREADS, 0, st, a);
  if (a.W <= 16) return launch_k(beam_reorder_kernel<V, 16>, grid, BR_THREADS, 0, st, a);
  if constexpr (sizeof(V) <= 8)
    if (a.W <= 32) return launch_k(beam_reorder_kernel<V, 32>, grid, BR_THREADS, 0, st, a);
  if constexpr (sizeof(V) <= 4)
    return launch_k(beam_reorder_kernel<V, 64>, grid, BR_THREADS, 0, st, a);
  return LILICORR_ERR_SHAPE;
}

size_t select_ws_bytes(int rows, int V, lilicorr_dtype_t dt) {
  const BeamCut c = beam_cut(rows, V, dt);
  return 256 + align_up((size_t)rows * c.chunks * sizeof(float), 256) +
         align_up((size_t)rows * c.slots * sizeof(SumRec), 256);
}

template <typename T>
lilicorr_status_t run_select(const T* logits, lilicorr_dtype_t dt, int requests, int W, int V,
                             const float* scores, const uint8_t* done, const BeamOut& out, void* ws,
                             cudaStream_t st) {
  const int rows = requests * W;
  const BeamCut cut = beam_cut(rows, V, dt);
  unsigned char* w = static_cast<unsigned char*>(ws);
  float* maxima = reinterpret_cast<float*>(w + 256);
  SumRec* sums = reinterpret_cast<SumRec*>(
      w + 256 + align_up((size_t)rows * cut.chunks * sizeof(float), 256));
  const long long warps = ((long long)rows * cut.chunks + cut.per_warp - 1) / cut.per_warp;
  LL_TRY(launch_k(beam_stream_kernel<T>, ceil_div(warps, BS_THREADS / 32), BS_THREADS, 0, st, logits,
                  rows, scores, done, cut, maxima, sums));
  return launch_k(beam_choose_kernel<T>, requests, BC_THREADS, 0, st, logits, W, scores, done, cut,
                  maxima, sums, out, reinterpret_cast<uint32_t*>(w));
}

bool beam_shape_ok(int requests, int beams, int n) {
  return requests >= 0 && beams >= 1 && beams <= LILICORR_MAX_BEAMS && n >= 1 && n <= LILICORR_MAX_K;
}

}  // namespace
}  // namespace lilicorr

using namespace lilicorr;

extern "C" {

size_t lilicorr_beam_select_workspace_bytes(int requests, int beams, int V, int n) {
  if (!beam_shape_ok(requests, beams, n) || V <= 0 || n > (long long)beams * V) return 0;
  const long long rows = (long long)requests * beams;
  if (rows > 65535) return 0;
  const size_t a = select_ws_bytes((int)rows, V, LILICORR_F32);
  const size_t b = select_ws_bytes((int)rows, V, LILICORR_BF16);
  return a > b ? a : b;
}

lilicorr_status_t lilicorr_beam_select(const void* logits, lilicorr_dtype_t dtype, int requests,
                                       int beams, int V, int n, const float* scores,
                                       const uint8_t* done, int32_t end_id, int32_t* tokens,
                                       int32_t* parents, float* next_scores, uint8_t* next_done,
                                       void* ws, size_t ws_bytes, cudaStream_t stream) {
  if (dtype != LILICORR_F32 && dtype != LILICORR_BF16) return LILICORR_ERR_DTYPE;
  const size_t need = lilicorr_beam_select_workspace_bytes(requests, beams, V, n);
  if (need == 0) return LILICORR_ERR_SHAPE;
  if (end_id < -1 || end_id >= V || (done && end_id < 0)) return LILICORR_ERR_ARG;
  if (requests == 0) return LILICORR_OK;
  if (!logits || !scores || !tokens || !parents || !next_scores || !ws) return LILICORR_ERR_ARG;
  if (!aligned16(logits) || !aligned16(ws)) return LILICORR_ERR_ARG;
  if (ws_bytes < need) return LILICORR_ERR_WORKSPACE;
  const BeamOut out{tokens, parents, next_scores, next_done, end_id, n};
  if (dtype == LILICORR_BF16)
    return run_select(static_cast<const uint16_t*>(logits), dtype, requests, beams, V, scores, done,
                      out, ws, stream);
  return run_select(static_cast<const float*>(logits), dtype, requests, beams, V, scores, done, out,
                    ws, stream);
}

lilicorr_status_t lilicorr_beam_merge(const int32_t* ids, const float* logp, int requests, int beams,
                                      int K, int n, const float* scores, const uint8_t* done,
                                      int32_t end_id, int32_t* tokens, int32_t* parents,
                                      float* next_scores, uint8_t* next_done, uint32_t* status,
                                      cudaStream_t stream) {
  if (!beam_shape_ok(requests, beams, n) || K < 1 || K > LILICORR_MAX_K || n > beams * K)
    return LILICORR_ERR_SHAPE;
  if (end_id < -1 || (done && end_id < 0)) return LILICORR_ERR_ARG;
  if (requests == 0) return LILICORR_OK;
  if (!ids || !logp || !scores || !tokens || !parents || !next_scores) return LILICORR_ERR_ARG;
  const BeamOut out{tokens, parents, next_scores, next_done, end_id, n};
  return launch_k(beam_merge_kernel, requests, BM_THREADS, 0, stream, ids, logp, beams, K, scores,
                  done, out, status);
}

lilicorr_status_t lilicorr_beam_reorder(void* const* host_states, int n_states, int requests,
                                        int beams, int positions, int heads, size_t row_bytes,
                                        int64_t stride_request, int64_t stride_beam,
                                        int64_t stride_position, int64_t stride_head,
                                        const int32_t* parents, const int32_t* lengths,
                                        cudaStream_t stream) {
  if (n_states < 0 || requests < 0 || requests > 65535 || positions < 0 || heads < 0 || beams < 1 ||
      beams > LILICORR_MAX_BEAMS)
    return LILICORR_ERR_SHAPE;
  if (n_states == 0 || requests == 0 || positions == 0 || heads == 0 || row_bytes == 0)
    return LILICORR_OK;
  if (!host_states || !parents) return LILICORR_ERR_ARG;
  if (row_bytes > (1ull << 31) || (double)positions * heads * (double)row_bytes >= 16.0 * 2147483648.0)
    return LILICORR_ERR_SHAPE;
  // heads that follow one another are one longer row
  if (heads > 1 && stride_head == (int64_t)row_bytes) {
    row_bytes *= heads;
    heads = 1;
  }
  // the widest vector that every row starts at and fills, and that W beams leave registers for
  uint64_t bits = row_bytes | (requests > 1 ? (uint64_t)stride_request : 0) |
                  (beams > 1 ? (uint64_t)stride_beam : 0) |
                  (positions > 1 ? (uint64_t)stride_position : 0) |
                  (heads > 1 ? (uint64_t)stride_head : 0);
  for (int i = 0; i < n_states; ++i) {
    if (!host_states[i]) return LILICORR_ERR_ARG;
    bits |= reinterpret_cast<uintptr_t>(host_states[i]);
  }
  int vec = beams <= 16 ? 16 : beams <= 32 ? 8 : 4;
  while (bits & (uint64_t)(vec - 1)) vec >>= 1;
  if ((double)positions * heads * (double)(row_bytes / vec) >= 2147483648.0) return LILICORR_ERR_SHAPE;
  Reorder a;
  a.W = beams;
  a.positions = positions;
  a.heads = heads;
  a.pieces = (uint32_t)(row_bytes / vec);
  a.s_req = stride_request;
  a.s_beam = stride_beam;
  a.s_pos = stride_position;
  a.s_head = stride_head;
  a.parents = parents;
  a.lengths = lengths;
  for (int i0 = 0; i0 < n_states; i0 += BR_STATES) {
    const int count = n_states - i0 < BR_STATES ? n_states - i0 : BR_STATES;
    for (int i = 0; i < BR_STATES; ++i)
      a.state[i] = i < count ? static_cast<unsigned char*>(host_states[i0 + i]) : nullptr;
    switch (vec) {
      case 16: LL_TRY(launch_reorder<uint4>(a, count, requests, stream)); break;
      case 8: LL_TRY(launch_reorder<uint2>(a, count, requests, stream)); break;
      case 4: LL_TRY(launch_reorder<uint32_t>(a, count, requests, stream)); break;
      case 2: LL_TRY(launch_reorder<uint16_t>(a, count, requests, stream)); break;
      default: LL_TRY(launch_reorder<uint8_t>(a, count, requests, stream)); break;
    }
  }
  return LILICORR_OK;
}

}  // extern "C"
