// Beam search: the n best (beam, token) pairs of each request, and the beams' states moved to the
// beams that continue them.
//
// Selection from logits takes two launches. (In one, the CTA that finishes a request choosing for it, the
// choosing ran beside warps that still stream and behind their fences: 34 us for 32 x 8 rows, when two took 30.)
//   (1) beam_stream_kernel reads every live row once, in chunks of 32 x 8 vectors of 16 bytes, one
//       warp a chunk, and leaves each chunk's largest logit m and the sum of exp(x - m).
//   (2) beam_choose_kernel, one CTA a request, forms the rows' normalisers, takes the n chunks whose
//       largest totals come first, reads those chunks again and ranks their elements. No other chunk
//       can hold one of the n best: each of the n chunks taken has an element that goes before
//       everything in a chunk not taken (a larger total, or an equal one at a lower beam or id, chunks
//       being runs of ids).
// So the pass over the vocabulary carries no candidates, only a maximum that the sum needs anyway.
// A total is (score - log S) + (x - M), M the row's largest logit and S the sum of exp(x - M): whatever the
// logits' size, x - M keeps what tells them apart. S is at least 1 (the largest logit's own term is 1 exactly),
// so that no total lies above its score. Totals are sums of 48 bits of inputs that are not: ex2.approx is good
// to 2^-22 and its argument to half a step, 2^-20 from 16 log2 units on, so that log S is good to 2^-20 at worst for V
// up to 151,936 (terms 11 nats below M, half of S together), to 2^-19 at any V, and to some 1e-8 where many
// unlike terms share the sum.
// Beams of one content tie: the sums have one order, and rows that are cut alike (V a multiple of a vector) the
// same bits. Where rows start off their 16-byte boundaries their chunks differ, and with them the roundings;
// there the pass also adds up the logits' bits (-0 as +0) as whole numbers, which no order changes, and rows of
// a request with the same M, the same such sum and normalisers within 2^-18 (twice the above) take the lower
// beam's.
#include <math.h>

#include "internal.cuh"

namespace lilicorr {

namespace {

constexpr unsigned FULL = 0xffffffffu;
constexpr int BM_THREADS = 128;
constexpr float LOG2E = 1.4426950408889634f;

// order-preserving 32-bit image of a float (-0 below +0)
__device__ __forceinline__ uint32_t ord32(float v) {
  const uint32_t b = __float_as_uint(v);
  return (b & 0x80000000u) ? ~b : (b | 0x80000000u);
}
__device__ __forceinline__ float unord32(uint32_t o) {
  return __uint_as_float((o & 0x80000000u) ? (o & 0x7FFFFFFFu) : ~o);
}
// s + c and s2 + c2 to s + c, the rounding of s + s2 kept in c
__device__ __forceinline__ void add_pair(float& s, float& c, float s2, float c2) {
  const float t = s + s2, bb = t - s;
  c = (c + c2) + ((s - (t - bb)) + (s2 - bb));
  s = t;
}
// Key of a total s + c (|c| at most half a step of s): order-preserving, 0 for -inf, NaN and +inf. Two
// fp32 numbers carry 48 bits; GB300 would take 16 clocks a warp for any one operation in FP64.
__device__ __forceinline__ uint64_t pair_key(float s, float c) {
  if (!(s > -INFINITY && s < INFINITY)) return 0ull;
  return ((uint64_t)ord32(s + 0.f) << 32) | ord32(c + 0.f);          // -0 to +0
}
__device__ __forceinline__ float key_score(uint64_t key) { return unord32((uint32_t)(key >> 32)); }
// A row's totals: (hi + lo) + (x - top) for its logits x <= top.
struct Base {
  float hi, lo, top;
};
__device__ __forceinline__ uint64_t sum_key(const Base& b, float x) {
  float d = x, rest = 0.f, hi = b.hi, lo = b.lo;
  add_pair(d, rest, -b.top, 0.f);
  add_pair(hi, lo, d, rest);
  const float s = hi + lo;
  return pair_key(s, lo - (s - hi));
}
// No logit below this reaches a total of `need`: by fp32, with a margin for its roundings.
__device__ __forceinline__ float logit_floor(const Base& b, float need) {
  const float d = (need - b.hi) - 0x1p-20f * (fabsf(need) + fabsf(b.hi));
  return (b.top + d) - 0x1p-22f * fabsf(b.top);
}
// log(s + c) of s >= 1 as hi + lo, to about 1e-9. log m = 2 atanh((m - 1) / (m + 1)) for s
// scaled to m in [0.7, 1.42): the quotient as a pair, the series' further terms (below 0.004) in fp32.
__device__ __forceinline__ void log_pair(float s, float c, float& hi, float& lo) {
  // s = m 2^k
  const int bits = __float_as_int(s);
  int k = ((bits >> 23) & 255) - 127;
  float m = __int_as_float((bits & 0x7FFFFF) | 0x3F800000);
  if (m > 1.41421356f) { m *= 0.5f; ++k; }
  const float mc = c * __int_as_float((127 - k) << 23);
  const float num = m - 1.f, den = m + 1.f;          // num exact; den off by at most 2^-24
  const float dl = m - (den - 1.f);
  const float z = __fdividef(num, den);
  const float zl = __fdividef(fmaf(-z, den, num) + mc - z * (dl + mc), den);
  const float q = z * z;
  const float rest = z * q * (0.66666667f + q * (0.4f + q * (0.28571429f + q * (0.22222222f + q * 0.18181818f))));
  const float n = (float)k, l = 0.69314718f, ll = -1.9046543e-9f;   // log 2 = l + ll + ...
  hi = n * l;
  lo = fmaf(n, l, -hi) + n * ll;
  add_pair(hi, lo, 2.f * z, 2.f * zl);
  add_pair(hi, lo, rest, 0.f);
  const float t = hi + lo;
  lo -= t - hi;
  hi = t;
}
// a precedes b: larger total, then lower position
template <typename P>
__device__ __forceinline__ bool precedes(uint64_t ka, P pa, uint64_t kb, P pb) {
  return ka > kb || (ka == kb && pa < pb);
}

// The first n of many candidates in order. First a bound: 64 groups of threads put forward their best
// candidate (best as far as fp32 tells, one is as valid as another), and nothing below the n-th of
// those 64 can be among the first n. The few candidates that reach it are kept and ranked against one
// another, four lanes a candidate. Where very many reach it (equal totals everywhere) the n are taken
// one after the other instead. Keys are order-preserving, 0 for no candidate.
constexpr int RF_GROUPS = 64;
constexpr int RF_CAP = 1024;
struct RankShared {
  uint64_t key[RF_CAP], pos[RF_CAP];           // what reaches the bound
  uint64_t gkey[RF_GROUPS], gpos[RF_GROUPS];   // the groups' best
  uint64_t bound, bound_pos;
  int count;
};

// The threads' best candidates (key 0: none) to sh.bound: all NT threads, LPG = NT / 64 lanes a group.
template <int NT>
__device__ __forceinline__ void rank_bound(RankShared& sh, int n, uint64_t key, uint64_t pos) {
  constexpr int LPG = NT / RF_GROUPS;
  static_assert(LPG >= 2 && LPG <= 32 && (LPG & (LPG - 1)) == 0 && RF_GROUPS >= LILICORR_MAX_K, "");
  const int tid = threadIdx.x;
#pragma unroll
  for (int o = 1; o < LPG; o <<= 1) {
    const uint64_t k = __shfl_xor_sync(FULL, key, o), p = __shfl_xor_sync(FULL, pos, o);
    if (precedes(k, p, key, pos)) { key = k; pos = p; }
  }
  const int g = tid / LPG, in = tid % LPG;
  if (in == 0) { sh.gkey[g] = key; sh.gpos[g] = pos; }
  if (tid == 0) { sh.count = 0; sh.bound = 1ull; sh.bound_pos = ~0ull; }
  __syncthreads();
  int rank = 0;
#pragma unroll
  for (int j = 0; j < RF_GROUPS / LPG; ++j) {
    const int o = j * LPG + in;
    rank += precedes(sh.gkey[o], sh.gpos[o], key, pos) ? 1 : 0;
  }
#pragma unroll
  for (int o = 1; o < LPG; o <<= 1) rank += __shfl_xor_sync(FULL, rank, o);
  if (in == 0 && key && rank == n - 1) { sh.bound = key; sh.bound_pos = pos; }
  __syncthreads();
}
__device__ __forceinline__ void rank_keep(RankShared& sh, uint64_t k, uint64_t p) {
  if (!k || precedes(sh.bound, sh.bound_pos, k, p)) return;
  const int at = atomicAdd(&sh.count, 1);
  if (at < RF_CAP) { sh.key[at] = k; sh.pos[at] = p; }
}
// place(rank, key, position) for the first n of what was kept; how many there are, up to n, or -1
// where more were kept than fit. After a barrier.
template <int NT, class Place>
__device__ __forceinline__ int rank_kept(RankShared& sh, int n, Place place) {
  const int m = sh.count;
  if (m > RF_CAP) return -1;
  const int tid = threadIdx.x, in = tid & 3;
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
// The same from all `count` candidates, one after the other; at least n of them have a key.
template <int NT, class Key, class Pos, class Place>
__device__ __noinline__ void rank_rounds(RankShared& sh, int count, int n, Key key_of, Pos pos_of,
                                         Place place) {
  const int tid = threadIdx.x;
  uint64_t last = ~0ull, last_pos = 0ull;      // before every candidate
  for (int t = 0; t < n; ++t) {
    uint64_t bk = 0ull, bp = ~0ull;
    for (int i = tid; i < count; i += NT) {
      const uint64_t k = key_of(i), p = pos_of(i);
      if (k && precedes(last, last_pos, k, p) && precedes(k, p, bk, bp)) { bk = k; bp = p; }
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
      const uint64_t k = __shfl_xor_sync(FULL, bk, o), p = __shfl_xor_sync(FULL, bp, o);
      if (precedes(k, p, bk, bp)) { bk = k; bp = p; }
    }
    __syncthreads();
    if ((tid & 31) == 0) { sh.gkey[tid >> 5] = bk; sh.gpos[tid >> 5] = bp; }
    __syncthreads();
    for (int w = 0; w < NT / 32; ++w)
      if (precedes(sh.gkey[w], sh.gpos[w], bk, bp)) { bk = sh.gkey[w]; bp = sh.gpos[w]; }
    if (tid == 0) place(t, bk, bp);
    last = bk;
    last_pos = bp;
  }
}
// All of it for keys that lie in shared memory (written before a barrier), no more than fit.
template <int NT, int CAP, class Pos, class Place>
__device__ __forceinline__ int rank_first(RankShared& sh, const uint64_t (&keys)[CAP], int count, int n,
                                          Pos pos_of, Place place) {
  static_assert(CAP <= RF_CAP, "");
  const int tid = threadIdx.x;
  if (count > RF_GROUPS) {
    uint64_t best = 0ull, best_p = ~0ull;
    for (int i = tid; i < count; i += NT) {
      const uint64_t k = keys[i];
      if (k < best) continue;
      const uint64_t p = pos_of(i);
      if (precedes(k, p, best, best_p)) { best = k; best_p = p; }
    }
    rank_bound<NT>(sh, n, best, best_p);
  } else {
    if (tid == 0) { sh.count = 0; sh.bound = 1ull; sh.bound_pos = ~0ull; }
    __syncthreads();
  }
  const uint64_t least = sh.bound;
  for (int i = tid; i < count; i += NT)
    if (keys[i] >= least) rank_keep(sh, keys[i], pos_of(i));
  __syncthreads();
  return rank_kept<NT>(sh, n, place);
}

struct BeamOut {
  int32_t *tokens, *parents;
  float* next_scores;
  uint8_t* next_done;
  int32_t end_id;
  int n;
  __device__ void put(int r, int rank, float score, int w, int32_t token, bool over) const {
    const size_t at = (size_t)r * n + rank;
    tokens[at] = token;
    parents[at] = w;
    next_scores[at] = score;
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

// Candidate lists: one CTA a request, a warp a list at a time (lane = rank), each warp keeping the 32
// first it has seen in order. Two runs of 32 in order merge in six steps: the larger of a[i] and
// b[31 - i] are the 32 first, and a bitonic sequence. Lists that do not come in order are sorted first.
constexpr int BM_WARPS = BM_THREADS / 32;

struct Cand { uint64_t key; int pos; };
__device__ __forceinline__ Cand cand_xor(const Cand& a, int o) {
  Cand b;
  b.key = __shfl_xor_sync(FULL, a.key, o);
  b.pos = __shfl_xor_sync(FULL, a.pos, o);
  return b;
}
// the earlier (or, with `later`, the later) of the two
__device__ __forceinline__ Cand cand_pick(const Cand& a, const Cand& b, bool later) {
  return precedes(a.key, a.pos, b.key, b.pos) != later ? a : b;
}
__device__ __forceinline__ void cand_bitonic(Cand& a, int lane) {      // a bitonic run to one in order
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) a = cand_pick(a, cand_xor(a, o), (lane & o) != 0);
}
__device__ __noinline__ Cand cand_sort(Cand a, int lane) {
  for (int size = 2; size <= 32; size <<= 1)
    for (int o = size >> 1; o > 0; o >>= 1)
      a = cand_pick(a, cand_xor(a, o), ((lane & o) != 0) != ((lane & size) != 0));
  return a;
}
__device__ __forceinline__ void cand_merge(Cand& a, const Cand& b, int lane) {
  a = cand_pick(a, cand_xor(b, 31), false);
  cand_bitonic(a, lane);
}

__global__ void __launch_bounds__(BM_THREADS)
beam_merge_kernel(const int32_t* __restrict__ ids, const float* __restrict__ logp, int W, int K,
                  const float* __restrict__ scores, const uint8_t* __restrict__ done, BeamOut out,
                  uint32_t* status) {
  pdl_wait();
  __shared__ uint64_t s_key[BM_WARPS - 1][32];
  __shared__ int s_pos[BM_WARPS - 1][32];
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, r = blockIdx.x;
  const size_t row0 = (size_t)r * W;
  Cand top{0ull, 0x7FFFFFFF};
  bool bad = false;
  constexpr int AHEAD = 4;                             // lists whose loads go out together
  for (int w0 = warp; w0 < W; w0 += AHEAD * BM_WARPS) {
    float sc[AHEAD], lp[AHEAD];
    bool over[AHEAD];
#pragma unroll
    for (int u = 0; u < AHEAD; ++u) {
      const int w = w0 + u * BM_WARPS;
      sc[u] = lp[u] = -INFINITY;
      over[u] = false;
      if (w >= W) continue;
      sc[u] = scores[row0 + w];
      if (done) over[u] = done[row0 + w] != 0;
      if (lane < K) lp[u] = logp[(row0 + w) * K + lane];
    }
#pragma unroll
    for (int u = 0; u < AHEAD; ++u) {
      const int w = w0 + u * BM_WARPS;
      if (w >= W) break;
      // the exact sum as its rounding to fp32 and what that lost
      float total = -INFINITY, lost = 0.f;
      if (over[u]) {
        if (lane == 0) total = sc[u];
      } else if (sc[u] != -INFINITY && lane < K) {
        total = sc[u];
        add_pair(total, lost, lp[u], 0.f);
      }
      if (!(total < INFINITY)) bad = true;             // NaN, +inf
      Cand c{pair_key(total, lost), w * K + lane};
      const uint64_t after = __shfl_down_sync(FULL, c.key, 1);
      if (!__all_sync(FULL, lane == 31 || c.key >= after)) c = cand_sort(c, lane);
      if (w == warp) top = c;
      else cand_merge(top, c, lane);
    }
  }
  if (bad) set_status(status, LILICORR_ERR_NONFINITE);
  // the warps' runs, two and two
#pragma unroll
  for (int half = BM_WARPS / 2; half > 0; half >>= 1) {
    if (warp >= half && warp < 2 * half) {
      s_key[warp - 1][lane] = top.key;
      s_pos[warp - 1][lane] = top.pos;
    }
    __syncthreads();
    if (warp < half && warp + half < W)
      cand_merge(top, Cand{s_key[warp + half - 1][lane], s_pos[warp + half - 1][lane]}, lane);
  }
  if (warp == 0 && lane < out.n) {
    if (top.key == 0ull) {
      out.none(r, lane);                               // fewer candidates than n
    } else {
      const int w = top.pos / K;
      const bool over = done && done[row0 + w];
      out.put(r, lane, key_score(top.key), w, over ? out.end_id : ids[row0 * K + top.pos], over);
    }
  }
}

// ---------------------------------------------------------------------------- from logits
// The streaming kernel: vectors of 16 bytes per lane and chunk, chunks of a warp in flight or in use, CTAs an
// SM. The call on 32 x 8 bf16 rows of 151,936 and on 24 x 5 fp32 rows of 128,257, device us: (8, 3, 2) 23.8 and
// 20.6; (8, 2, 3) 23.9 and 19.8; (4, 4, 3) 26.9 and 23.1, (4, 6, 2) 27.9 and 24.7, (4, 4, 2) 29.3 and 24.6. What is
// in flight (96 KB an SM in the second and the last, 128 to 160 in the others) matters less than what each chunk
// costs besides its elements.
constexpr int BS_THREADS = 256;
constexpr int BS_U = 8, BS_STAGES = 3, BS_CTAS = 2;
constexpr int BC_THREADS = 512;                // of the choosing kernel

// How rows are cut: chunk 0 of a row holds the ids before its first 16-byte boundary where rows need
// not start on one (`odd`), the others runs of `size` ids; warp i of the streaming kernel takes the
// chunks [i * per_warp, (i + 1) * per_warp) of all rows.
struct BeamCut {
  int V, vec, size, odd, chunks;               // chunks per row
  int per_warp;
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
  // one wave of CTAs
  const long long total = (long long)rows * c.chunks;
  const long long warps = (long long)BS_CTAS * (BS_THREADS / 32) * num_sms();
  c.per_warp = (int)((total + warps - 1) / warps);
  if (c.per_warp < 1) c.per_warp = 1;
  return c;
}

__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
// One vector of logits as words: bf16 pairs or floats.
template <typename T> struct Elem;
template <> struct Elem<uint16_t> {
  static constexpr int N = 8;
  __device__ static float value(uint16_t x) { return bf16_to_f32(x); }
  static constexpr uint32_t NONE = 0xFF80FF80u;
  static constexpr int BITS = 16;
  // the sum of bits with those of both halves, -0 as +0
  __device__ static uint32_t mark(uint32_t w, uint32_t sum) {
    const __nv_bfloat162 x = __hadd2(*reinterpret_cast<const __nv_bfloat162*>(&w), __float2bfloat162_rn(0.f));
    return __dp2a_lo(*reinterpret_cast<const uint32_t*>(&x), 0x0101u, sum);
  }
  static constexpr uint32_t MARK_NONE = 0xFF80u;           // of one element that is not there
  // the value whose ord32 begins with these 16 bits, and how many of a lane's share reach it
  __device__ static float image(uint32_t code) { return unord32((code >> 31) ? code : code | 0xFFFFu); }
  __device__ static int at_least(const uint4 (&v)[BS_U], uint32_t code) {
    const __nv_bfloat162 t = __float2bfloat162_rn(image(code));          // (exact)
    auto reach = [&](uint32_t w) {
      return __popc(__hge2_mask(*reinterpret_cast<const __nv_bfloat162*>(&w), t));
    };
    int n = 0;
#pragma unroll
    for (int u = 0; u < BS_U; ++u) n += (reach(v[u].x) + reach(v[u].y)) + (reach(v[u].z) + reach(v[u].w));
    return n >> 4;
  }
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
  __device__ static float vmax(const uint4 (&v)[BS_U]) {
    uint32_t m = NONE, n = NONE;
#pragma unroll
    for (int u = 0; u < BS_U; ++u) {
      asm("max.bf16x2 %0, %0, %1;" : "+r"(m) : "r"(v[u].x));
      asm("max.bf16x2 %0, %0, %1;" : "+r"(n) : "r"(v[u].y));
      asm("max.bf16x2 %0, %0, %1;" : "+r"(m) : "r"(v[u].z));
      asm("max.bf16x2 %0, %0, %1;" : "+r"(n) : "r"(v[u].w));
    }
    asm("max.bf16x2 %0, %0, %1;" : "+r"(m) : "r"(n));
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
  __device__ static float value(float x) { return x; }
  static constexpr uint32_t NONE = 0xFF800000u;
  static constexpr int BITS = 32;
  __device__ static uint32_t mark(uint32_t w, uint32_t sum) {
    return sum + __float_as_uint(__uint_as_float(w) + 0.f);
  }
  static constexpr uint32_t MARK_NONE = NONE;
  __device__ static float image(uint32_t code) { return unord32(code); }
  __device__ static int at_least(const uint4 (&v)[BS_U], uint32_t code) {
    const float t = image(code);
    int n = 0;
#pragma unroll
    for (int u = 0; u < BS_U; ++u)
      n += ((__uint_as_float(v[u].x) >= t) + (__uint_as_float(v[u].y) >= t)) +
           ((__uint_as_float(v[u].z) >= t) + (__uint_as_float(v[u].w) >= t));
    return n;
  }
  __device__ static void pair(const uint4& v, int i, float& a, float& b) {
    a = __uint_as_float(i == 0 ? v.x : v.z);
    b = __uint_as_float(i == 0 ? v.y : v.w);
  }
  __device__ static float vmax(const uint4& v) {
    return fmaxf(fmaxf(__uint_as_float(v.x), __uint_as_float(v.y)),
                 fmaxf(__uint_as_float(v.z), __uint_as_float(v.w)));
  }
  __device__ static float vmax(const uint4 (&v)[BS_U]) {
    float m = vmax(v[0]);
#pragma unroll
    for (int u = 1; u < BS_U; ++u) m = fmaxf(m, vmax(v[u]));
    return m;
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
    const unsigned at = (unsigned)begin + (u * 32 + lane) * N;     // (may pass 2^31 - 1, as V may come near it)
    raw[u] = make_uint4(NI, NI, NI, NI);
    if (at + N <= (unsigned)end) raw[u] = __ldcs(reinterpret_cast<const uint4*>(row + at));
    else if (at < (unsigned)end) raw[u] = Elem<T>::gather(row + at, end - (int)at);
  }
}

// Bound by HBM. A warp's chunks lie one after the other; each lane copies its own 128 bytes of a chunk
// into its own part of a ring in shared memory, two chunks ahead, and reads back only what it copied:
// 128 KB a SM in flight, no registers for it and no barrier.
// ODD: as in the cut; the chunks' sums of bits go to `marks`.
template <typename T, bool ODD>
__global__ void __launch_bounds__(BS_THREADS, BS_CTAS)
beam_stream_kernel(const T* __restrict__ logits, unsigned rows, const float* __restrict__ scores,
                   const uint8_t* __restrict__ done, const BeamCut cut, float* __restrict__ maxima,
                   float* __restrict__ sums, uint32_t* __restrict__ marks) {
  pdl_wait();
  constexpr int N = Elem<T>::N;
  constexpr unsigned STAGE = BS_U * 32;
  extern __shared__ uint4 ring[];
  const int lane = threadIdx.x & 31;
  uint4* mine = ring + (threadIdx.x >> 5) * (BS_STAGES * STAGE) + lane;
  const unsigned wid = blockIdx.x * (BS_THREADS / 32) + (threadIdx.x >> 5);
  const unsigned chunks = (unsigned)cut.chunks, total = rows * chunks;
  const unsigned begin = wid * (unsigned)cut.per_warp, stop = min(total, begin + (unsigned)cut.per_warp);
  if (begin >= total) return;

  // A row as a run of chunks: its first full chunk's logits, and how many full ones follow (shorter
  // ones, at the row's ends, are loaded when they are summed).
  struct Row {
    const T* full;
    unsigned first, count;
    bool live;
  };
  auto open = [&](unsigned row) {
    Row x;
    const int h = cut.head(row);
    x.live = scores[row] > -INFINITY && !(done && done[row]);
    x.full = logits + (size_t)row * cut.V + h;
    x.first = (unsigned)cut.odd;
    x.count = (unsigned)(cut.V - h) / (unsigned)cut.size;
    return x;
  };
  unsigned row = begin / chunks, c = begin - row * chunks;
  Row here = open(row);

  // the copying side, ahead of the summing one
  unsigned at = begin, crow = row, cc = c, cstage = 0;
  Row ahead = here;
  const T* src = ahead.full + (size_t)(cc < ahead.first ? 0u : cc - ahead.first) * cut.size + lane * N;
  // (sure: the row is live, or that is not known yet and the copy does not wait for it)
  auto copy = [&](bool sure) {
    if (at < stop) {
      if (cc - ahead.first < ahead.count && (sure || ahead.live)) {
        const uint32_t dst = (uint32_t)__cvta_generic_to_shared(mine + cstage * STAGE);
#pragma unroll
        for (int u = 0; u < BS_U; ++u)
          asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst + u * 512),
                       "l"(src + u * 32 * N)
                       : "memory");
      }
      if (cc >= ahead.first) src += cut.size;
      ++at;
      if (++cc == chunks) {
        cc = 0;
        if (at < stop) {
          ahead = open(++crow);
          src = ahead.full + lane * N;
        }
      }
    }
    cstage = cstage + 1 == BS_STAGES ? 0 : cstage + 1;
    asm volatile("cp.async.commit_group;" ::: "memory");
  };
#pragma unroll
  for (int i = 0; i < BS_STAGES - 1; ++i) copy(true);

  unsigned stage = 0;
  for (unsigned i = begin; i < stop; ++i) {
    copy(false);
    asm volatile("cp.async.wait_group %0;" ::"n"(BS_STAGES - 1) : "memory");
    if (here.live) {
      uint4 raw[BS_U];
      int missing = 0;                                  // elements that a short chunk lacks
      if (c - here.first < here.count) {
#pragma unroll
        for (int u = 0; u < BS_U; ++u) raw[u] = mine[stage * STAGE + u * 32];
      } else {
        int b, en;
        cut.range(row, (int)c, b, en);
        load_chunk<T>(logits + (size_t)row * cut.V, b, en, lane, raw);
        missing = 32 * BS_U * N - (en - b);
      }
      const float m = unord32(__reduce_max_sync(FULL, ord32(Elem<T>::vmax(raw))));
      // terms exp(x - m): -inf adds 0 (in a chunk of nothing else too), NaN stays. The difference first, which
      // is exact for what counts, whatever the size of m.
      const float ref = m == -INFINITY ? 0.f : m;
      float p0 = 0.f, p1 = 0.f, p2 = 0.f, p3 = 0.f;
#pragma unroll
      for (int u = 0; u < BS_U; ++u)
#pragma unroll
        for (int k = 0; k < N / 2; ++k) {
          float x0, x1;
          Elem<T>::pair(raw[u], k, x0, x1);
          x0 = ex2((x0 - ref) * LOG2E);
          x1 = ex2((x1 - ref) * LOG2E);
          if (k & 1) { p2 += x0; p3 += x1; } else { p0 += x0; p1 += x1; }
        }
      const float sum = warp_sum((p0 + p1) + (p2 + p3));
      if (lane == 0) {
        maxima[i] = m;
        sums[i] = sum;
      }
      if constexpr (ODD) {
        uint32_t mark = 0;
#pragma unroll
        for (int u = 0; u < BS_U; ++u) {
          mark = Elem<T>::mark(raw[u].y, Elem<T>::mark(raw[u].x, mark));
          mark = Elem<T>::mark(raw[u].w, Elem<T>::mark(raw[u].z, mark));
        }
        mark = __reduce_add_sync(FULL, mark) - (uint32_t)missing * Elem<T>::MARK_NONE;
        if (lane == 0) marks[i] = mark;
      }
    }
    stage = stage + 1 == BS_STAGES ? 0 : stage + 1;
    if (++c == chunks) {
      c = 0;
      if (i + 1 < stop) here = open(++row);
    }
  }
}

// More than n of a chunk's elements reach the bound (few chunks for n, equal logits, a row that falls
// steadily): its first n, by a search over the bits of the n-th largest value, in registers; of those
// equal to it the lowest ids. hot: this lane's elements (element j of vector u: bit u * N + j). What lies
// below the bound does not change a count that is compared with n.
template <typename T>
__device__ __forceinline__ uint64_t chunk_first(const uint4 (&raw)[BS_U], uint64_t hot, int n, int lane) {
  constexpr int N = Elem<T>::N;
  uint32_t nth = 0;
  for (int b = 31; b >= 32 - Elem<T>::BITS; --b) {
    const uint32_t t = nth | (1u << b);
    if (__reduce_add_sync(FULL, Elem<T>::at_least(raw, t)) >= n) nth = t;
  }
  const float v = Elem<T>::image(nth);
  uint64_t above = 0, equal = 0;
#pragma unroll
  for (int u = 0; u < BS_U; ++u)
#pragma unroll
    for (int j = 0; j < N / 2; ++j) {
      float x0, x1;
      Elem<T>::pair(raw[u], j, x0, x1);
      above |= (x0 > v ? 1ull : 0ull) << (u * N + 2 * j) | (x1 > v ? 1ull : 0ull) << (u * N + 2 * j + 1);
      equal |= (x0 == v ? 1ull : 0ull) << (u * N + 2 * j) | (x1 == v ? 1ull : 0ull) << (u * N + 2 * j + 1);
    }
  above &= hot;
  equal &= hot;
  int room = n - __reduce_add_sync(FULL, __popcll(above));
  for (int u = 0; u < BS_U; ++u) {
    const uint64_t mask = (N == 8 ? 0xFFull : 0xFull) << (u * N);
    const int mine = __popcll(equal & mask);
    int before = mine;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int x = __shfl_up_sync(FULL, before, o);
      if (lane >= o) before += x;
    }
    const int all = __shfl_sync(FULL, before, 31);
    int left = room - (before - mine);
    for (uint64_t h = equal & mask; h; h &= h - 1, --left)
      if (left <= 0) equal &= ~(1ull << (__ffsll((long long)h) - 1));
    room -= all;
  }
  return above | equal;
}

constexpr int BC_MAX = 4;                      // maxima of a lane loaded together

__device__ __forceinline__ void load_maxima(const float* __restrict__ p, int c0, int chunks,
                                            float (&v)[BC_MAX]) {
#pragma unroll
  for (int u = 0; u < BC_MAX; ++u) v[u] = c0 + 32 * u < chunks ? p[c0 + 32 * u] : -INFINITY;
}

// One CTA a request: normalisers, the n chunks to look at, their elements, the n best. Bound by
// latency: what the phases cost is loads one after the other, barriers and instructions first met.
template <typename T>
__global__ void __launch_bounds__(BC_THREADS)
beam_choose_kernel(const T* __restrict__ logits, int W, const float* __restrict__ scores,
                   const uint8_t* __restrict__ done, BeamCut cut, const float* __restrict__ maxima,
                   const float* __restrict__ sums, const uint32_t* __restrict__ marks, BeamOut out,
                   uint32_t* status) {
  pdl_wait();
  constexpr int N = Elem<T>::N;
  constexpr int NW = BC_THREADS / 32;
  constexpr int CAND = LILICORR_MAX_K * LILICORR_MAX_K;
  __shared__ Base s_base[LILICORR_MAX_BEAMS];           // (score - log S, as a pair; M)
  __shared__ float2 s_norm[LILICORR_MAX_BEAMS];         // log S, as a pair (+inf: none)
  __shared__ uint32_t s_mark[LILICORR_MAX_BEAMS];       // the rows' sums of bits (odd cuts)
  __shared__ uint8_t s_kind[LILICORR_MAX_BEAMS];        // 0 absent, 1 live, 2 done
  // a lane's largest chunk maximum of a row and where it is, while chunks are chosen; the candidates
  // after that
  __shared__ union {
    struct { float top[LILICORR_MAX_BEAMS][32]; int at[LILICORR_MAX_BEAMS][32]; } lanes;
    struct { uint64_t key[CAND], at[CAND]; } cand;
  } s_u;
  auto& s_lane = s_u.lanes.top;
  auto& s_lane_at = s_u.lanes.at;
  auto& s_key = s_u.cand.key;
  auto& s_at = s_u.cand.at;
  __shared__ RankShared sh;
  __shared__ uint64_t s_ckey[LILICORR_MAX_K], s_cpos[LILICORR_MAX_K];
  __shared__ int s_cand;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, r = blockIdx.x;
  const size_t row0 = (size_t)r * W;
  const float* mx = maxima + row0 * cut.chunks;
  if (tid == 0) s_cand = 0;

  // a warp a row: its normaliser from the chunks' sums, and each lane's best chunk
  for (int w = warp; w < W; w += NW) {
    const size_t row = row0 + w;
    // every load at once: what a row that is not live left there is not used
    const float sc = scores[row];
    const bool over = done && done[row];
    const float* rm = mx + (size_t)w * cut.chunks;
    const float* rs = sums + row * cut.chunks;
    float v[BC_MAX], part[BC_MAX];
    load_maxima(rm, lane, cut.chunks, v);
#pragma unroll
    for (int u = 0; u < BC_MAX; ++u) part[u] = lane + 32 * u < cut.chunks ? rs[lane + 32 * u] : 0.f;
    uint32_t mark = 0;
    if (cut.odd) {
#pragma unroll
      for (int u = 0; u < BC_MAX; ++u)
        if (lane + 32 * u < cut.chunks) mark += marks[row * cut.chunks + lane + 32 * u];
    }
    float best = -INFINITY;
    int at = 0;
#pragma unroll
    for (int u = 0; u < BC_MAX; ++u)
      if (v[u] > best) { best = v[u]; at = lane + 32 * u; }
    for (int c = lane + 32 * BC_MAX; c < cut.chunks; c += 32)
      if (rm[c] > best) { best = rm[c]; at = c; }
    float2 norm = make_float2(INFINITY, 0.f);
    float top = 0.f;
    int kind = !(sc > -INFINITY) ? 0 : over ? 2 : 1;
    bool bad = sc != sc || sc == INFINITY;
    if (kind == 1) {
      // S in an order of its own: whatever warps met the chunks, the same bits
      top = warp_max(best);
      float s = 0.f, c = 0.f;
#pragma unroll
      for (int u = 0; u < BC_MAX; ++u) add_pair(s, c, part[u] * ex2((v[u] - top) * LOG2E), 0.f);
      for (int i = lane + 32 * BC_MAX; i < cut.chunks; i += 32)
        add_pair(s, c, rs[i] * ex2((rm[i] - top) * LOG2E), 0.f);
#pragma unroll
      for (int o = 16; o > 0; o >>= 1)
        add_pair(s, c, __shfl_xor_sync(FULL, s, o), __shfl_xor_sync(FULL, c, o));
      // (no finite logit: NaN, as from one)
      if (!(s >= 1.f && s < INFINITY)) bad = true;
      if (cut.odd) {
        for (int i = lane + 32 * BC_MAX; i < cut.chunks; i += 32) mark += marks[row * cut.chunks + i];
        mark = __reduce_add_sync(FULL, mark);
        if (lane == 0) s_mark[w] = mark;
      }
      log_pair(s, c, norm.x, norm.y);
      if (norm.x < 0.f) norm = make_float2(0.f, 0.f);     // (a rounding of the sum's second half)
    } else {
      best = kind == 2 && lane == 0 ? 0.f : -INFINITY;  // the one candidate of a beam that is done
      at = 0;
    }
    if (bad) kind = 0;
    if (kind == 0) best = -INFINITY;
    s_lane[w][lane] = best;
    s_lane_at[w][lane] = at;
    if (lane == 0) {
      if (bad) set_status(status, LILICORR_ERR_NONFINITE);
      s_norm[w] = kind == 1 ? norm : make_float2(INFINITY, 0.f);
      s_base[w] = Base{sc, 0.f, top};
      s_kind[w] = (uint8_t)kind;
    }
  }
  __syncthreads();

  // Rows of one content take one normaliser (see above). Then each row's base, and of all its rows this
  // thread's best.
  uint64_t best_key = 0ull, best_pos = ~0ull;
  for (int w = warp; w < W; w += NW) {
    const float best = s_lane[w][lane];
    Base base = s_base[w];
    if (s_kind[w] == 1) {
      float2 norm = s_norm[w];
      for (int w0 = 0; cut.odd && w0 < w; w0 += 32) {
        const int v = w0 + lane;
        const float2 x = v < w ? s_norm[v] : make_float2(INFINITY, 0.f);       // (+inf: not live)
        const unsigned same = __ballot_sync(
            FULL, fabsf((x.x - norm.x) + (x.y - norm.y)) <= 0x1p-18f && s_base[v].top == base.top &&
                      s_mark[v] == s_mark[w]);
        if (same) {
          norm = s_norm[w0 + __ffs(same) - 1];
          break;
        }
      }
      add_pair(base.hi, base.lo, -norm.x, -norm.y);
    }
    if (lane == 0) {                                     // (others read its top meanwhile, which stays)
      s_base[w].hi = base.hi;
      s_base[w].lo = base.lo;
    }
    const uint64_t key = best == -INFINITY ? 0ull : sum_key(base, best);
    const uint64_t pos = ((uint64_t)w << 32) | (uint32_t)s_lane_at[w][lane];
    if (precedes(key, pos, best_key, best_pos)) { best_key = key; best_pos = pos; }
  }

  // the first n chunks, by their largest total; a done beam is one chunk of one candidate
  rank_bound<BC_THREADS>(sh, out.n, best_key, best_pos);
  // Few groups have a row of their own where beams are few, and many chunks reach the n-th of them where
  // beams differ: the n-th of all lanes' best instead
  for (int w = warp; w < W; w += NW) {
    const float v = s_lane[w][lane];
    if (v == -INFINITY) continue;
    rank_keep(sh, sum_key(s_base[w], v), ((uint64_t)w << 32) | (uint32_t)s_lane_at[w][lane]);
  }
  __syncthreads();
  uint64_t nth = 0ull, nth_pos = 0ull;
  rank_kept<BC_THREADS>(sh, out.n, [&](int rank, uint64_t key, uint64_t p) {
    if (rank == out.n - 1) { nth = key; nth_pos = p; }
  });
  __syncthreads();
  if (nth) { sh.bound = nth; sh.bound_pos = nth_pos; }
  if (tid == 0) sh.count = 0;
  __syncthreads();
  const uint64_t bound = sh.bound;
  for (int w = warp; w < W; w += NW) {
    const Base base = s_base[w];
    const float v = s_lane[w][lane];
    const float thr = bound == 1ull ? -INFINITY : logit_floor(base, key_score(bound));
    if (v == -INFINITY || v < thr) continue;             // nor any other of the lane's
    const uint64_t pos = (uint64_t)w << 32;
    if (s_kind[w] == 2) {
      rank_keep(sh, sum_key(base, 0.f), pos);
      continue;
    }
    for (int c0 = lane; c0 < cut.chunks; c0 += 32 * BC_MAX) {
      float x[BC_MAX];
      load_maxima(mx + (size_t)w * cut.chunks, c0, cut.chunks, x);
#pragma unroll
      for (int u = 0; u < BC_MAX; ++u) {
        if (x[u] >= thr && x[u] > -INFINITY)
          rank_keep(sh, sum_key(base, x[u]), pos | (uint32_t)(c0 + 32 * u));
      }
    }
  }
  __syncthreads();
  auto take = [&](int rank, uint64_t key, uint64_t p) {
    s_ckey[rank] = key;
    s_cpos[rank] = p;
  };
  int taken = rank_kept<BC_THREADS>(sh, out.n, take);
  if (taken < 0) {
    rank_rounds<BC_THREADS>(
        sh, W * cut.chunks, out.n,
        [&](int i) -> uint64_t {
          const int w = i / cut.chunks;
          if (s_kind[w] == 0 || (s_kind[w] == 2 && i != w * cut.chunks)) return 0ull;
          const float x = s_kind[w] == 2 ? 0.f : mx[i];
          return x > -INFINITY ? sum_key(s_base[w], x) : 0ull;
        },
        [&](int i) { return ((uint64_t)(i / cut.chunks) << 32) | (uint32_t)(i % cut.chunks); }, take);
    taken = out.n;
  }
  __syncthreads();
  uint64_t least = taken == out.n ? s_ckey[taken - 1] : 1ull;
  // The chunks' elements, and a bound from the groups' best of them where a row has no more chunks than n: with
  // one beam ahead of the others the n chunks are then all of its own and more, and most of them lies above
  // the last one's maximum. Without and with the step, one beam far ahead / beams near one another, us: 44 x 15
  // rows of 16,000 bf16 (8 chunks), n 4 13.3 14.4 / 13.0 14.2, n 8 19.8 15.1 / 13.5 14.7, n 32 39 30 / 19.7 18.5;
  // fp32 (16 chunks), n 12 17.2 18.4 / 16.8 17.9, n 16 21.6 18.8 / 17.2 18.3, n 32 39 24 / 23 24; 16 x 2 rows of
  // 50,000 (25 chunks), n 16 10.1 11.1 / 9.9 11.0, n 24 14.4 12.8 / 11.4 12.7, n 32 35 13.5 / 12.9 13.4; 32 x 8 rows of
  // 151,936 (75 chunks), n 8 23.4 25.0 / 23.1 24.4, n 32 30.4 33.1 / 29.7 32.1. 64 x 16 rows of 2,000 (1 chunk),
  // n 1 15.9 16.8 / 14.0 15.0, n 4 16.4 17.6 / 16.1 15.1, n 16 25 19 / 24 19.
  constexpr int MINE = (LILICORR_MAX_K + NW - 1) / NW;
  uint4 raw[MINE][BS_U];
  int from[MINE];                                       // a chunk's first id, or -1
  best_key = 0ull;
  best_pos = ~0ull;
#pragma unroll
  for (int i = 0; i < MINE; ++i) {
    const int c = warp + i * NW;
    from[i] = -1;
    if (c >= taken) continue;
    const uint64_t cpos = s_cpos[c];
    const int w = (int)(cpos >> 32);
    if (s_kind[w] == 2) {
      if (lane == 0 && precedes(s_ckey[c], cpos, best_key, best_pos)) { best_key = s_ckey[c]; best_pos = cpos; }
      continue;
    }
    int en;
    cut.range(row0 + w, (int)(uint32_t)cpos, from[i], en);
    load_chunk<T>(logits + (row0 + w) * cut.V, from[i], en, lane, raw[i]);
  }
  if (out.n > 1 && cut.chunks <= out.n) {
#pragma unroll
    for (int i = 0; i < MINE; ++i) {
      if (from[i] < 0) continue;
      const int c = warp + i * NW;
      const float top = Elem<T>::vmax(raw[i]);
      if (top == -INFINITY) continue;
      const uint64_t key = sum_key(s_base[(int)(s_cpos[c] >> 32)], top), pos = (uint64_t)(c * 32 + lane);
      if (precedes(key, pos, best_key, best_pos)) { best_key = key; best_pos = pos; }
    }
    rank_bound<BC_THREADS>(sh, out.n, best_key, best_pos);
    if (sh.bound > least) least = sh.bound;
  }
#pragma unroll
  for (int i = 0; i < MINE; ++i) {
    const int c = warp + i * NW;
    if (c >= taken) continue;
    const int w = (int)(s_cpos[c] >> 32);
    if (s_kind[w] == 2) {
      if (lane == 0 && s_ckey[c] >= least) {
        const int at = atomicAdd(&s_cand, 1);
        s_key[at] = s_ckey[c];
        s_at[at] = ((uint64_t)w << 32) | (uint32_t)out.end_id;
      }
      continue;
    }
    const T* rp = logits + (row0 + w) * cut.V;
    const Base base = s_base[w];
    // elements whose total may reach `least`
    const float thr = least == 1ull ? -INFINITY : logit_floor(base, key_score(least));
    uint64_t hot = 0;                                   // element j of vector u: bit u * N + j
#pragma unroll
    for (int u = 0; u < BS_U; ++u) {
      if (!__any_sync(FULL, Elem<T>::vmax(raw[i][u]) >= thr)) continue;
#pragma unroll
      for (int j = 0; j < N / 2; ++j) {
        float x0, x1;
        Elem<T>::pair(raw[i][u], j, x0, x1);
        hot |= (x0 >= thr && x0 > -INFINITY ? 1ull : 0ull) << (u * N + 2 * j);
        hot |= (x1 >= thr && x1 > -INFINITY ? 1ull : 0ull) << (u * N + 2 * j + 1);
      }
    }
    if (__reduce_add_sync(FULL, __popcll(hot)) > out.n) hot = chunk_first<T>(raw[i], hot, out.n, lane);
    for (uint64_t h = hot; h; h &= h - 1) {
      const int j = __ffsll((long long)h) - 1, id = from[i] + ((j / N) * 32 + lane) * N + j % N;
      const uint64_t key = sum_key(base, Elem<T>::value(rp[id]));
      if (key < least) continue;
      const int at = atomicAdd(&s_cand, 1);
      s_key[at] = key;
      s_at[at] = ((uint64_t)w << 32) | (uint32_t)id;
    }
  }
  __syncthreads();
  const int found = rank_first<BC_THREADS>(
      sh, s_key, s_cand, out.n, [&](int i) { return s_at[i]; },
      [&](int rank, uint64_t key, uint64_t p) {
        const int w = (int)(p >> 32);
        out.put(r, rank, key_score(key), w, (int32_t)(uint32_t)p, s_kind[w] == 2);
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
// buffer and without a barrier: nobody else reads or writes its column. Bound by HBM: loads and stores
// past the caches (nothing is read twice but a parent of several beams, by one thread) and many CTAs,
// so that the run that a CTA takes of each beam is a few KB at a time: 32 x 8 beams of 4 x 512 x 2 KB,
// 0.9 GB moved, 6.5 TB/s; 19 CTAs a pair instead of 76 6.1, cached accesses 5.6.
// DENSE: the positions of a head follow one another, and the grid has the heads: no divisions. 8 requests
// of 512 positions x 2 KB x 4 arrays: 32 beams 266 us, with the divisions 376; 16 beams 129 and 137; 4
// beams 33 and 32.
template <typename V, int WMAX, bool DENSE>
__global__ void __launch_bounds__(BR_THREADS)
beam_reorder_kernel(const __grid_constant__ Reorder a) {
  pdl_wait();
  __shared__ int s_parent[LILICORR_MAX_BEAMS];
  const int tid = threadIdx.x, r = blockIdx.y;
  if (tid < a.W) {
    const int p = a.parents[(size_t)r * a.W + tid];
    s_parent[tid] = (p < 0 || p >= a.W) ? tid : p;
  }
  int len = a.positions;
  if (a.lengths) len = min(max(a.lengths[r], 0), a.positions);
  __syncthreads();
  const uint32_t per_pos = DENSE ? a.pieces : (uint32_t)a.heads * a.pieces;
  const uint32_t total = (uint32_t)len * per_pos;
  const int st = DENSE ? blockIdx.z / a.heads : blockIdx.z;
  unsigned char* base = a.state[st] + (int64_t)r * a.s_req;
  if (DENSE) base += (int64_t)(blockIdx.z - st * a.heads) * a.s_head;
  for (uint32_t u = blockIdx.x * BR_THREADS + tid; u < total; u += gridDim.x * BR_THREADS) {
    unsigned char* col = base + (int64_t)u * sizeof(V);
    if (!DENSE) {
      const uint32_t pos = u / per_pos, in = u - pos * per_pos, h = in / a.pieces, c = in - h * a.pieces;
      col = base + (int64_t)pos * a.s_pos + (int64_t)h * a.s_head + (int64_t)c * sizeof(V);
    }
    V v[WMAX];
#pragma unroll
    for (int w = 0; w < WMAX; ++w)
      if (w < a.W && s_parent[w] != w)
        v[w] = __ldcs(reinterpret_cast<const V*>(col + (int64_t)s_parent[w] * a.s_beam));
#pragma unroll
    for (int w = 0; w < WMAX; ++w)
      if (w < a.W && s_parent[w] != w) __stcs(reinterpret_cast<V*>(col + (int64_t)w * a.s_beam), v[w]);
  }
}

template <typename V, bool DENSE>
lilicorr_status_t launch_reorder_form(const Reorder& a, int count, int requests, cudaStream_t st) {
  const long long most = (long long)a.positions * a.pieces * (DENSE ? 1 : a.heads);
  const long long z = (long long)count * (DENSE ? a.heads : 1), pairs = z * requests;
  long long x = (most + BR_THREADS - 1) / BR_THREADS;
  const long long want = (64ll * num_sms() + pairs - 1) / pairs;     // the rest by the loop
  if (x > want) x = want;
  if (x < 1) x = 1;
  const dim3 grid((unsigned)x, (unsigned)requests, (unsigned)z);
  if (a.W <= 4) return launch_k(beam_reorder_kernel<V, 4, DENSE>, grid, BR_THREADS, 0, st, a);
  if (a.W <= 8) return launch_k(beam_reorder_kernel<V, 8, DENSE>, grid, BR_THREADS, 0, st, a);
  if (a.W <= 16) return launch_k(beam_reorder_kernel<V, 16, DENSE>, grid, BR_THREADS, 0, st, a);
  if constexpr (sizeof(V) <= 8)
    if (a.W <= 32) return launch_k(beam_reorder_kernel<V, 32, DENSE>, grid, BR_THREADS, 0, st, a);
  if constexpr (sizeof(V) <= 4)
    return launch_k(beam_reorder_kernel<V, 64, DENSE>, grid, BR_THREADS, 0, st, a);
  return LILICORR_ERR_SHAPE;
}

template <typename V>
lilicorr_status_t launch_reorder(const Reorder& a, int count, int requests, cudaStream_t st) {
  if ((a.positions == 1 || a.s_pos == (int64_t)a.pieces * (int64_t)sizeof(V)) &&
      (long long)count * a.heads <= 65535)
    return launch_reorder_form<V, true>(a, count, requests, st);
  return launch_reorder_form<V, false>(a, count, requests, st);
}

size_t select_ws_bytes(int rows, int V, lilicorr_dtype_t dt) {
  const BeamCut c = beam_cut(rows, V, dt);
  return 256 + (c.odd ? 3 : 2) * align_up((size_t)rows * c.chunks * sizeof(float), 256);
}

template <typename T, bool ODD>
lilicorr_status_t launch_stream(const T* logits, int rows, const float* scores, const uint8_t* done,
                                const BeamCut& cut, float* maxima, float* sums, uint32_t* marks,
                                cudaStream_t st) {
  const long long warps = ((long long)rows * cut.chunks + cut.per_warp - 1) / cut.per_warp;
  static bool configured[64] = {false};
  auto* kernel = beam_stream_kernel<T, ODD>;
  LL_TRY(allow_max_dynamic_smem(kernel, configured));
  return launch_k(kernel, ceil_div(warps, BS_THREADS / 32), BS_THREADS,
                  (size_t)BS_THREADS * BS_STAGES * BS_U * sizeof(uint4), st, logits, (unsigned)rows,
                  scores, done, cut, maxima, sums, marks);
}

template <typename T>
lilicorr_status_t run_select(const T* logits, lilicorr_dtype_t dt, int requests, int W, int V,
                             const float* scores, const uint8_t* done, const BeamOut& out, void* ws,
                             cudaStream_t st) {
  const int rows = requests * W;
  const BeamCut cut = beam_cut(rows, V, dt);
  unsigned char* w = static_cast<unsigned char*>(ws);
  const size_t each = align_up((size_t)rows * cut.chunks * sizeof(float), 256);
  float* maxima = reinterpret_cast<float*>(w + 256);
  float* sums = reinterpret_cast<float*>(w + 256 + each);
  uint32_t* marks = cut.odd ? reinterpret_cast<uint32_t*>(w + 256 + 2 * each) : nullptr;
  if (cut.odd) LL_TRY((launch_stream<T, true>(logits, rows, scores, done, cut, maxima, sums, marks, st)));
  else LL_TRY((launch_stream<T, false>(logits, rows, scores, done, cut, maxima, sums, marks, st)));
  return launch_k(beam_choose_kernel<T>, requests, BC_THREADS, 0, st, logits, W, scores, done, cut,
                  maxima, sums, marks, out, reinterpret_cast<uint32_t*>(w));
}

// The checks of one layout but for overlaps, and how its arrays are moved: all of `a` but the arrays, parents
// and lengths, and the bytes a thread takes at a time (0: there is nothing to move).
lilicorr_status_t reorder_layout(const lilicorr_beam_states& s, int requests, int beams,
                                 const int32_t* parents, Reorder* a, int* bytes) {
  *bytes = 0;
  if (s.n_states < 0 || s.positions < 0 || s.heads < 0) return LILICORR_ERR_SHAPE;
  if (s.n_states == 0 || requests == 0 || s.positions == 0 || s.heads == 0 || s.row_bytes == 0)
    return LILICORR_OK;
  if (!s.host_states || !parents) return LILICORR_ERR_ARG;
  if (s.row_bytes > (1ull << 31) ||
      (double)s.positions * s.heads * (double)s.row_bytes >= 16.0 * 2147483648.0)
    return LILICORR_ERR_SHAPE;
  for (int i = 0; i < s.n_states; ++i)
    if (!s.host_states[i]) return LILICORR_ERR_ARG;
  // heads that follow one another are one longer row
  size_t row_bytes = s.row_bytes;
  int heads = s.heads;
  if (heads > 1 && s.stride_head == (int64_t)row_bytes) {
    row_bytes *= heads;
    heads = 1;
  }
  // the widest vector that every row starts at and fills, and that W beams leave registers for. (8
  // requests of 512 positions x 2 KB x 4 arrays, 16, 8 and 4 bytes: 4 beams 33, 41 and 50 us, 16 beams 129,
  // 130 and 305; 32 beams 266 in 8 bytes and 312 in 4)
  uint64_t bits = row_bytes | (requests > 1 ? (uint64_t)s.stride_request : 0) |
                  (beams > 1 ? (uint64_t)s.stride_beam : 0) |
                  (s.positions > 1 ? (uint64_t)s.stride_position : 0) |
                  (heads > 1 ? (uint64_t)s.stride_head : 0);
  for (int i = 0; i < s.n_states; ++i) bits |= reinterpret_cast<uintptr_t>(s.host_states[i]);
  int vec = beams <= 16 ? 16 : beams <= 32 ? 8 : 4;
  while (bits & (uint64_t)(vec - 1)) vec >>= 1;
  if ((double)s.positions * heads * (double)(row_bytes / vec) >= 2147483648.0) return LILICORR_ERR_SHAPE;
  a->W = beams;
  a->positions = s.positions;
  a->heads = heads;
  a->pieces = (uint32_t)(row_bytes / vec);
  a->s_req = s.stride_request;
  a->s_beam = s.stride_beam;
  a->s_pos = s.stride_position;
  a->s_head = s.stride_head;
  *bytes = vec;
  return LILICORR_OK;
}

// Rows that share bytes would race: a column of the beams is moved by one thread.
bool states_overlap(void* const* states, int n, const int64_t* strides, const int64_t* extents,
                    int64_t row_bytes) {
  const StrideNest nest(strides, extents, 4, row_bytes);
  if (!nest.nests()) return true;
  for (int i = 1; i < n; ++i)
    for (int j = 0; j < i; ++j)
      if (nest.meets((__int128)reinterpret_cast<intptr_t>(states[i]) - reinterpret_cast<intptr_t>(states[j])))
        return true;
  return false;
}

// Do two arrays of different layouts share a byte? The distance of two of their rows is the bases' and a
// whole multiple of each stride that occurs, the multiple an index of the one, the other, or a difference of
// both; from the largest stride down, only multiples that the smaller ones can make up for are followed.
// Layouts cut from one buffer share their strides, and few multiples are left. `steps` bounds the search
// where layouts have nothing in common; past it the answer is yes.
struct RowDistance {
  struct Term { __int128 stride; int64_t lo, hi; };
  int n = 0;
  Term term[8];
  __int128 lo[9], hi[9];                   // what the terms from here on can add
  int64_t row_a, row_b;                    // bytes of a row
  __int128 shift = 0;                      // of the bases, from rows at negative strides
  void add(int64_t stride, int64_t extent, bool second) {
    if (extent <= 1) return;
    __int128 s = stride;
    if (s < 0) {                           // counted from its lowest row
      shift += (second ? s : -s) * (extent - 1);
      s = -s;
    }
    int i = 0;
    while (i < n && term[i].stride > s) ++i;
    if (i == n || term[i].stride != s) {
      for (int j = n; j > i; --j) term[j] = term[j - 1];
      term[i] = {s, 0, 0};
      ++n;
    }
    if (second) term[i].hi += extent - 1;
    else term[i].lo -= extent - 1;
  }
  void close(int64_t a, int64_t b) {
    row_a = a;
    row_b = b;
    lo[n] = hi[n] = 0;
    for (int i = n - 1; i >= 0; --i) {
      lo[i] = lo[i + 1] + term[i].lo * term[i].stride;
      hi[i] = hi[i + 1] + term[i].hi * term[i].stride;
    }
  }
  // second row - first row = d so far
  bool meets(__int128 d, long long* steps, int i = 0) const {
    if (d + lo[i] >= row_a || d + hi[i] <= -row_b) return false;
    if (i == n || --*steps <= 0) return true;
    const __int128 s = term[i].stride;
    // -row_b < d + c s + hi[i + 1] and d + c s + lo[i + 1] < row_a (s > 0: no layout has equal rows)
    const __int128 from = -row_b - d - hi[i + 1], to = row_a - d - lo[i + 1];
    const __int128 least = from >= 0 ? from / s + 1 : 1 - (-from + s - 1) / s;
    const __int128 most = to > 0 ? (to - 1) / s : -((s - to) / s);
    const __int128 c0 = least > term[i].lo ? least : term[i].lo, c1 = most < term[i].hi ? most : term[i].hi;
    for (__int128 c = c0; c <= c1; ++c)
      if (meets(d + c * s, steps, i + 1)) return true;
    return false;
  }
};

// All arrays of a call, of layouts that passed reorder_layout.
constexpr long long OVERLAP_STEPS = 1 << 20;         // some 10 ms of the host
bool layouts_overlap(const lilicorr_beam_states* layouts, int n, int requests, int beams) {
  long long steps = OVERLAP_STEPS;
  auto empty = [](const lilicorr_beam_states& s) {
    return s.n_states == 0 || s.positions == 0 || s.heads == 0 || s.row_bytes == 0;
  };
  for (int i = 0; i < n; ++i) {
    const lilicorr_beam_states& b = layouts[i];
    if (empty(b)) continue;
    const int64_t strides[4] = {b.stride_request, b.stride_beam, b.stride_position, b.stride_head};
    const int64_t extents[4] = {requests, beams, b.positions, b.heads};
    if (states_overlap(b.host_states, b.n_states, strides, extents, (int64_t)b.row_bytes)) return true;
    for (int j = 0; j < i; ++j) {
      const lilicorr_beam_states& a = layouts[j];
      if (empty(a)) continue;
      RowDistance dist;
      const int64_t strides_a[4] = {a.stride_request, a.stride_beam, a.stride_position, a.stride_head};
      const int64_t extents_a[4] = {requests, beams, a.positions, a.heads};
      for (int d = 0; d < 4; ++d) {
        dist.add(strides_a[d], extents_a[d], false);
        dist.add(strides[d], extents[d], true);
      }
      dist.close((int64_t)a.row_bytes, (int64_t)b.row_bytes);
      for (int x = 0; x < a.n_states; ++x)
        for (int y = 0; y < b.n_states; ++y) {
          const __int128 d = (__int128)reinterpret_cast<intptr_t>(b.host_states[y]) -
                             reinterpret_cast<intptr_t>(a.host_states[x]);
          if (dist.meets(d + dist.shift, &steps)) return true;
        }
    }
  }
  return false;
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
  // (chunks of 4 KB: 2^31 of them are more than the device holds)
  if (rows > 65535 || rows * (V / 1024 + 2ll) >= 0x7FFFFFFFll) return 0;
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

lilicorr_status_t lilicorr_beam_reorder_layouts(const lilicorr_beam_states* host_layouts, int n_layouts,
                                               int requests, int beams, const int32_t* parents,
                                               const int32_t* lengths, cudaStream_t stream) {
  if (n_layouts < 0 || requests < 0 || requests > 65535 || beams < 1 || beams > LILICORR_MAX_BEAMS)
    return LILICORR_ERR_SHAPE;
  if (n_layouts > 0 && !host_layouts) return LILICORR_ERR_ARG;
  // every layout is looked at before the first array is moved
  Reorder a;
  int vec;
  for (int i = 0; i < n_layouts; ++i)
    LL_TRY(reorder_layout(host_layouts[i], requests, beams, parents, &a, &vec));
  if (requests > 0 && layouts_overlap(host_layouts, n_layouts, requests, beams)) return LILICORR_ERR_ARG;
  a.parents = parents;
  a.lengths = lengths;
  for (int i = 0; i < n_layouts; ++i) {
    const lilicorr_beam_states& s = host_layouts[i];
    LL_TRY(reorder_layout(s, requests, beams, parents, &a, &vec));
    if (vec == 0) continue;
    for (int i0 = 0; i0 < s.n_states; i0 += BR_STATES) {
      const int count = s.n_states - i0 < BR_STATES ? s.n_states - i0 : BR_STATES;
      for (int j = 0; j < BR_STATES; ++j)
        a.state[j] = j < count ? static_cast<unsigned char*>(s.host_states[i0 + j]) : nullptr;
      switch (vec) {
        case 16: LL_TRY(launch_reorder<uint4>(a, count, requests, stream)); break;
        case 8: LL_TRY(launch_reorder<uint2>(a, count, requests, stream)); break;
        case 4: LL_TRY(launch_reorder<uint32_t>(a, count, requests, stream)); break;
        case 2: LL_TRY(launch_reorder<uint16_t>(a, count, requests, stream)); break;
        default: LL_TRY(launch_reorder<uint8_t>(a, count, requests, stream)); break;
      }
    }
  }
  return LILICORR_OK;
}

lilicorr_status_t lilicorr_beam_reorder(void* const* host_states, int n_states, int requests,
                                        int beams, int positions, int heads, size_t row_bytes,
                                        int64_t stride_request, int64_t stride_beam,
                                        int64_t stride_position, int64_t stride_head,
                                        const int32_t* parents, const int32_t* lengths,
                                        cudaStream_t stream) {
  const lilicorr_beam_states one = {host_states, n_states, positions, heads, row_bytes, stride_request,
                                    stride_beam, stride_position, stride_head};
  return lilicorr_beam_reorder_layouts(&one, 1, requests, beams, parents, lengths, stream);
}

int lilicorr_test_states_overlap(void* const* host_states, int n_states, const int64_t* strides,
                                 const int64_t* extents, size_t row_bytes) {
  return states_overlap(host_states, n_states, strides, extents, (int64_t)row_bytes);
}

int lilicorr_test_layouts_overlap(const lilicorr_beam_states* host_layouts, int n_layouts, int requests,
                                  int beams) {
  return layouts_overlap(host_layouts, n_layouts, requests, beams);
}

}  // extern "C"
