// A decoding cache held in 4 bits: new tokens rounded into it, read back, and the keys of least weight
// evicted.
#include "cache.cuh"

namespace lilicorr {

// ------------------------------------------------------------------------------- checks
namespace {
bool unit_ok(float u) {
  uint32_t b;
  memcpy(&b, &u, 4);
  return !(b & 0x807FFFFFu) && u >= 0x1p-60f && u <= 0x1p60f;      // a power of two
}
}  // namespace

lilicorr_status_t cache_shape(const lilicorr_cache_desc* d) {
  if (!d) return LILICORR_ERR_ARG;
  if (d->sequences < 0 || d->capacity < 0 || d->capacity > (1 << 30) || d->kv_heads < 1)
    return LILICORR_ERR_SHAPE;
  if (d->head_dim < 16 || d->head_dim > 128 || d->head_dim % 16) return LILICORR_ERR_SHAPE;
  if ((int64_t)d->sequences * d->kv_heads > 0x7FFFFFFFll) return LILICORR_ERR_SHAPE;
  return unit_ok(d->k_unit) && unit_ok(d->v_unit) ? LILICORR_OK : LILICORR_ERR_ARG;
}

bool cache_rows_ok(const int64_t* s, const int64_t (&e)[3], int per16, int row, bool written) {
  for (int i = 0; i < 3; ++i)
    if (e[i] > 1 && (s[i] < 0 || s[i] % per16 || s[i] > (1ll << 40))) return false;
  return !written || StrideNest(s, e, 3, row).nests();
}

lilicorr_status_t cache_view(const lilicorr_cache_desc* d, const void* cache, bool written, CacheView* v) {
  if (d->sequences && d->capacity && (!cache || !aligned16(cache))) return LILICORR_ERR_ARG;
  const int64_t e[3] = {d->sequences, d->capacity, d->kv_heads};
  if (!cache_rows_ok(d->stride, e, 16, cache_record_bytes(d->head_dim), written)) return LILICORR_ERR_ARG;
  if (e[1] > 1 && d->stride[1] >= (1 << 28)) return LILICORR_ERR_ARG;        // 16 positions in 32 bits
  v->p = static_cast<unsigned char*>(const_cast<void*>(cache));
  for (int i = 0; i < 3; ++i) v->s[i] = e[i] > 1 ? d->stride[i] : 0;
  v->N = d->sequences;
  v->S = d->capacity;
  v->H = d->kv_heads;
  v->d = d->head_dim;
  v->k_unit = d->k_unit;
  v->v_unit = d->v_unit;
  return LILICORR_OK;
}

namespace {

// ------------------------------------------------------------------------------- append and read
// x / d of whole numbers x < 2^31 by a product: with 2^s >= d and m = ceil(2^(31 + s) / d) below 2^32,
// m x / 2^(31 + s) exceeds x / d by less than 1 / d (Granlund and Montgomery, 1994).
struct Quotient {
  uint32_t d, m, s;
  void set(uint32_t by) {
    d = by;
    for (s = 0; (1ull << s) < by; ++s) {}
    m = (uint32_t)(((1ull << (31 + s)) + by - 1) / by);
  }
  __device__ __forceinline__ uint32_t of(uint32_t x) const { return (uint32_t)(((uint64_t)x * m) >> 31) >> s; }
};

struct CacheTokens {
  const void* k;               // read: written
  const void* v;
  int64_t k_s[3], v_s[3];      // elements: sequence, token, head
  int T;
  const int32_t* seq_len;
  float* weights;
  uint32_t total;              // threads that have work
  int wide;                    // all groups start at multiples of 32 bytes: a load or store of 32 each
  Quotient by_row, by_head, by_T;
};

__device__ __forceinline__ float max_nan(float a, float b) {
  float r;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
  return r;
}
// two values as codes, lo in the low half of the byte; ties to the even code, cut at 6
__device__ __forceinline__ uint32_t codes2(float lo, float hi) {
  uint32_t r;
  asm("{\n .reg .b8 t;\n cvt.rn.satfinite.e2m1x2.f32 t, %2, %1;\n cvt.u32.u8 %0, t;\n}"
      : "=r"(r) : "f"(lo), "f"(hi));
  return r;
}
// a scale's byte of a value >= 0: to the nearest, ties to even, cut at 448; NaN becomes 127
__device__ __forceinline__ uint32_t scale_byte(float x) {
  uint16_t r;
  asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(r) : "f"(0.f), "f"(x));
  return r & 0x7Fu;
}
__device__ __forceinline__ float scale_value(uint32_t byte) {
  uint32_t r;
  asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(r) : "h"((uint16_t)byte));
  float f;
  asm("{\n .reg .b16 lo, hi;\n mov.b32 {lo, hi}, %1;\n cvt.f32.f16 %0, lo;\n}" : "=f"(f) : "r"(r));
  return f;
}
// the eight codes of a word
__device__ __forceinline__ void code_values(uint32_t w, float* x) {
  uint32_t r[4];
  asm("{\n .reg .b8 a, b, c, d;\n mov.b32 {a, b, c, d}, %4;\n cvt.rn.f16x2.e2m1x2 %0, a;\n"
      " cvt.rn.f16x2.e2m1x2 %1, b;\n cvt.rn.f16x2.e2m1x2 %2, c;\n cvt.rn.f16x2.e2m1x2 %3, d;\n}"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(w));
#pragma unroll
  for (int i = 0; i < 4; ++i)
    asm("{\n .reg .b16 l, h;\n mov.b32 {l, h}, %2;\n cvt.f32.f16 %0, l;\n cvt.f32.f16 %1, h;\n}"
        : "=f"(x[2 * i]), "=f"(x[2 * i + 1]) : "r"(r[i]));
}

// 32 bytes, in one piece (a whole sector a lane) or in two
__device__ __forceinline__ void load32(const void* p, int wide, uint32_t* u) {
  if (wide) {
    asm volatile("ld.global.v8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                 : "=r"(u[0]), "=r"(u[1]), "=r"(u[2]), "=r"(u[3]), "=r"(u[4]), "=r"(u[5]), "=r"(u[6]), "=r"(u[7])
                 : "l"(p));
  } else {
    const uint4 x = __ldcs(static_cast<const uint4*>(p)), y = __ldcs(static_cast<const uint4*>(p) + 1);
    u[0] = x.x; u[1] = x.y; u[2] = x.z; u[3] = x.w;
    u[4] = y.x; u[5] = y.y; u[6] = y.z; u[7] = y.w;
  }
}
__device__ __forceinline__ void store32(void* p, int wide, const uint32_t* u) {
  if (wide) {
    asm volatile("st.global.v8.b32 [%8], {%0, %1, %2, %3, %4, %5, %6, %7};" ::"r"(u[0]), "r"(u[1]), "r"(u[2]),
                 "r"(u[3]), "r"(u[4]), "r"(u[5]), "r"(u[6]), "r"(u[7]), "l"(p)
                 : "memory");
  } else {
    static_cast<uint4*>(p)[0] = make_uint4(u[0], u[1], u[2], u[3]);
    static_cast<uint4*>(p)[1] = make_uint4(u[4], u[5], u[6], u[7]);
  }
}
__device__ __forceinline__ void store16(__nv_bfloat16* p, int wide, const float (&x)[16]) {
  uint32_t u[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) u[i] = bf16_pack2(x[2 * i], x[2 * i + 1]);
  store32(p, wide, u);
}
__device__ __forceinline__ void store16(float* p, int wide, const float (&x)[16]) {
  store32(p, wide, reinterpret_cast<const uint32_t*>(x));
  store32(p + 8, wide, reinterpret_cast<const uint32_t*>(x) + 8);
}

// The byte of the scale nearest to top / (6 unit). The quotient's rounding to fp32 must not put it on the
// border between two scales where it is beside it: what it lost, found exactly by one fused multiply and
// subtract, becomes its last bit.
__device__ __forceinline__ uint32_t group_scale(float top, float inv_unit) {
  const float a = top * inv_unit;                    // exact, or far outside the scales
  float q = a / 6.f;
  if (q > 0x1p-20f && q < 0x1p20f) {
    const float rest = fmaf(-6.f, q, a);
    if (rest != 0.f) q = __uint_as_float((__float_as_uint(q) - (rest < 0.f)) | 1u);
  }
  const uint32_t b = scale_byte(q);
  return b == 0 ? 1 : b;
}

// The codes of 16 elements x, whose bits are u and whose scale times the unit is su. In bf16 x / su is a border
// between two codes or at least 2^-10 away from it, so that the product with the rounded inverse, rounded to
// multiples of 2^-12, falls on the same side; fp32 elements are compared with the borders, which are exact products.
// Either way a code has its element's sign, that of a zero too, and codes of a NaN group have nothing else.
__device__ __forceinline__ uint2 group_codes(const float (&x)[16], const uint32_t (&u)[8], float su) {
  const float inv = 1.f / su, big = 0x1.8p11f;
  uint32_t w[2];
#pragma unroll
  for (int j = 0; j < 2; ++j) {
    w[j] = 0;
#pragma unroll
    for (int i = 0; i < 8; i += 2) {
      const float lo = fmaf(x[8 * j + i], inv, big) - big, hi = fmaf(x[8 * j + i + 1], inv, big) - big;
      w[j] |= codes2(lo, hi) << (4 * i);
    }
    if (!(su == su)) w[j] = 0;
    // what rounds to zero comes out as +0: the bytes that hold the signs of the even and of the odd elements
    const uint32_t a = __byte_perm(u[4 * j], u[4 * j + 1], 0x7351), b = __byte_perm(u[4 * j + 2], u[4 * j + 3], 0x7351);
    const uint32_t even = __byte_perm(a, b, 0x5410), odd = __byte_perm(a, b, 0x7632);
    w[j] |= (even >> 4 & 0x08080808u) | (odd & 0x80808080u);
  }
  return make_uint2(w[0], w[1]);
}
__device__ __forceinline__ uint2 group_codes(const float (&x)[16], const uint32_t (&)[16], float su) {
  uint32_t w[2] = {0, 0};
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    const float a = fabsf(x[i]);
    const uint32_t c = (a > 0.25f * su) + (a >= 0.75f * su) + (a > 1.25f * su) + (a >= 1.75f * su) +
                       (a > 2.5f * su) + (a >= 3.5f * su) + (a > 5.f * su);
    w[i / 8] |= (c | (__float_as_uint(x[i]) >> 31 << 3)) << (i % 8 * 4);
  }
  return make_uint2(w[0], w[1]);
}

// A thread has a group of 16 elements of the key and of the value; groups in the order (token, head, group).
struct CacheGroup { int n, t, h, g, pos; };
__device__ __forceinline__ bool cache_group(const CacheView& c, const CacheTokens& a, CacheGroup* x) {
  uint32_t i = blockIdx.x * blockDim.x + threadIdx.x;
  if (i >= a.total) return false;
  const uint32_t row = a.by_row.of(i);
  i -= row * a.by_row.d;
  x->h = a.by_head.of(i);
  x->g = i - x->h * a.by_head.d;
  x->n = a.by_T.of(row);
  x->t = row - x->n * a.T;
  const int len = a.seq_len[x->n];
  x->pos = len < 0 ? -1 : len - a.T + x->t;
  return true;
}

// A group, and its max |x|: NaN where there is one
__device__ __forceinline__ void group_load(const __nv_bfloat16* p, int wide, uint32_t (&u)[8]) { load32(p, wide, u); }
__device__ __forceinline__ void group_load(const float* p, int wide, uint32_t (&u)[16]) {
  load32(p, wide, u);
  load32(p + 8, wide, u + 8);
}
__device__ __forceinline__ float group_top(const uint32_t (&u)[8], float (&x)[16]) {
  uint32_t top = u[0] & 0x7FFF7FFFu;                 // two maxima side by side
#pragma unroll
  for (int i = 1; i < 8; ++i)
    asm("max.NaN.bf16x2 %0, %0, %1;" : "+r"(top) : "r"(u[i] & 0x7FFF7FFFu));
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    x[2 * i] = __uint_as_float(u[i] << 16);
    x[2 * i + 1] = __uint_as_float(u[i] & 0xFFFF0000u);
  }
  return max_nan(__uint_as_float(top << 16), __uint_as_float(top & 0xFFFF0000u));
}
__device__ __forceinline__ float group_top(const uint32_t (&u)[16], float (&x)[16]) {
  float top = 0.f;
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    x[i] = __uint_as_float(u[i]);
    top = max_nan(top, fabsf(x[i]));
  }
  return top;
}

// Bytes should bound both kernels (bf16: 2.56 an element); neither they (DRAM 48 and 50 % under a profiler) nor issue
// (67 and 56 % of the slots; about 160 and 110 instructions a thread's group of the key and of the value) do: what is
// left is the way of a thread's two loads, all that it has under way. Up to 8,192 tokens of four sequences, 8 heads
// of 128: append and read together 51.5 us in a graph, 260 MB at 5.0 TB/s (under the profiler 29.2 and 25.8). Loads and
// stores of 32 bytes, a whole sector a lane, and products for the divisions took them there from 72.
template <typename E>
__global__ void __launch_bounds__(256) cache_append_kernel(const CacheView c, const CacheTokens a) {
  pdl_wait();
  CacheGroup x;
  if (!cache_group(c, a, &x) || x.pos < 0 || x.pos >= c.S) return;
  uint32_t u[2][4 * sizeof(E)];
  group_load(static_cast<const E*>(a.k) + (x.n * a.k_s[0] + x.t * a.k_s[1] + x.h * a.k_s[2] + x.g * 16), a.wide,
             u[0]);
  group_load(static_cast<const E*>(a.v) + (x.n * a.v_s[0] + x.t * a.v_s[1] + x.h * a.v_s[2] + x.g * 16), a.wide,
             u[1]);
  unsigned char* rec = c.at(x.n, x.pos, x.h);
#pragma unroll
  for (int kv = 0; kv < 2; ++kv) {
    const float unit = kv ? c.v_unit : c.k_unit;
    float e[16];
    const float top = group_top(u[kv], e);
    const uint32_t b = group_scale(top, 1.f / unit);
    unsigned char* to = rec + kv * cache_half_bytes(c.d);
    *reinterpret_cast<uint2*>(to + x.g * 8) = group_codes(e, u[kv], scale_value(b) * unit);
    to[c.d / 2 + x.g] = (unsigned char)b;
    if (x.g == 0)                                    // scales that no group has
      for (int i = c.d / 16; i < 8; ++i) to[c.d / 2 + i] = 0;
  }
  if (a.weights && x.g == 0) a.weights[((size_t)x.n * c.H + x.h) * c.S + x.pos] = 0.f;
}

template <typename E>
__global__ void __launch_bounds__(256) cache_read_kernel(const CacheView c, const CacheTokens a) {
  pdl_wait();
  CacheGroup x;
  if (!cache_group(c, a, &x)) return;
  uint2 w[2] = {make_uint2(0, 0), make_uint2(0, 0)};
  uint32_t b[2] = {0, 0};
  if (x.pos >= 0 && x.pos < c.S) {
    const unsigned char* rec = c.at(x.n, x.pos, x.h);
#pragma unroll
    for (int kv = 0; kv < 2; ++kv) {
      w[kv] = *reinterpret_cast<const uint2*>(rec + kv * cache_half_bytes(c.d) + x.g * 8);
      b[kv] = rec[kv * cache_half_bytes(c.d) + c.d / 2 + x.g];
    }
  }
#pragma unroll
  for (int kv = 0; kv < 2; ++kv) {
    const float su = scale_value(b[kv]) * (kv ? c.v_unit : c.k_unit);
    float e[16];
    code_values(w[kv].x, e);
    code_values(w[kv].y, e + 8);
#pragma unroll
    for (int i = 0; i < 16; ++i) e[i] *= su;
    E* dst = static_cast<E*>(const_cast<void*>(kv ? a.v : a.k));
    const int64_t* s = kv ? a.v_s : a.k_s;
    store16(dst + (x.n * s[0] + x.t * s[1] + x.h * s[2] + x.g * 16), a.wide, e);
  }
}

lilicorr_status_t run_tokens(const lilicorr_cache_desc* desc, const void* cache, lilicorr_dtype_t dtype,
                             int tokens, const void* k, const int64_t* ks, const void* v,
                             const int64_t* vs, const int32_t* seq_len, float* weights, bool append,
                             cudaStream_t st) {
  LL_TRY(cache_shape(desc));
  if (dtype != LILICORR_F32 && dtype != LILICORR_BF16) return LILICORR_ERR_DTYPE;
  if (tokens < 0) return LILICORR_ERR_SHAPE;
  const double groups = (double)desc->sequences * tokens * desc->kv_heads * (desc->head_dim / 16);
  if (groups >= 2147483648.0) return LILICORR_ERR_SHAPE;
  CacheView c;
  LL_TRY(cache_view(desc, cache, append, &c));
  if (groups == 0) return LILICORR_OK;
  if (!k || !v || !ks || !vs || !seq_len || !aligned16(k) || !aligned16(v)) return LILICORR_ERR_ARG;
  const int64_t e[3] = {desc->sequences, tokens, desc->kv_heads};
  const int per16 = dtype == LILICORR_BF16 ? 8 : 4;
  if (!cache_rows_ok(ks, e, per16, c.d, !append) || !cache_rows_ok(vs, e, per16, c.d, !append))
    return LILICORR_ERR_ARG;
  CacheTokens a;
  a.k = k;
  a.v = v;
  for (int i = 0; i < 3; ++i) {
    a.k_s[i] = e[i] > 1 ? ks[i] : 0;
    a.v_s[i] = e[i] > 1 ? vs[i] : 0;
  }
  a.T = tokens;
  a.seq_len = seq_len;
  a.weights = weights;
  a.total = (uint32_t)groups;
  const int per32 = 2 * per16;
  a.wide = !(((uintptr_t)k | (uintptr_t)v) & 31);
  for (int i = 0; i < 3; ++i) a.wide &= a.k_s[i] % per32 == 0 && a.v_s[i] % per32 == 0;
  a.by_row.set(c.H * (c.d / 16));
  a.by_head.set(c.d / 16);
  a.by_T.set(tokens);
  const unsigned grid = (unsigned)(((int64_t)groups + 255) / 256);
  if (append)
    return dtype == LILICORR_BF16 ? launch_k(cache_append_kernel<__nv_bfloat16>, grid, 256, 0, st, c, a)
                                  : launch_k(cache_append_kernel<float>, grid, 256, 0, st, c, a);
  return dtype == LILICORR_BF16 ? launch_k(cache_read_kernel<__nv_bfloat16>, grid, 256, 0, st, c, a)
                                : launch_k(cache_read_kernel<float>, grid, 256, 0, st, c, a);
}

// ------------------------------------------------------------------------------- eviction
struct EvictArgs {
  CacheView from, to;
  float* w;                    // [N, H, from.S]
  float* to_w;                 // [N, H, to.S]
  const int32_t* seq_len;
  int budget, recent, first, in_place;
  int32_t* kept;               // [N, H, budget]
  int32_t* new_len;            // [N]
};

// Weights in the order of whole numbers: NaN below all, -0 as +0.
__device__ __forceinline__ uint32_t weight_key(float w) {
  uint32_t b = __float_as_uint(w);
  if (w != w) return 0;
  if ((b << 1) == 0u) b = 0u;
  return (b & 0x80000000u) ? ~b : (b | 0x80000000u);
}

// A cluster of CTAs has one (sequence, kv head). Which positions stay is found by each of them for itself where
// there are few (a barrier of the cluster costs as much as a pass), else each looks at a stretch of them. The
// records that stay are moved by all of them together.
// What bounds it: for one sequence its chain, of 22 thousand clocks 10 in the move (one turn's loads and stores), 2.6 a
// round (count, barriers, prefix sum, barrier), 3 each for the ranking and the places; for many the rounds, then the
// records, a turn after the other (DRAM 27 %, waits for loads). 8 heads cut from 2,304 to 2,048 11.3 us in a graph
// (one CTA that read weights from memory each round: 55), 256 heads of up to 4,160 to 2,048 40.4 (records read and
// written 19 at the copy rate), 16 heads of up to 65,536 to 4,096 31.8.
// CTAs of 1,024 threads, one an SM, took 17 and 58 for the first two's 13 and 36 of then.
constexpr int EV_THREADS = 512, EV_WARPS = EV_THREADS / 32;
constexpr int EV_BINS = 2048;  // 11 bits a round
constexpr int EV_COPIES = 4;   // of the counts: weights are alike in their upper bits, and lanes would queue
constexpr int EV_KEYS = 8192;  // of a stretch, kept in shared memory; longer ones are read again each time
constexpr int EV_RANKED = 384; // so many on the border are compared with one another
constexpr int EV_VECS = 8;     // 16-byte pieces that a thread moves at a time

struct EvictSmem {
  union {
    int hist[EV_BINS * EV_COPIES];
    int kept[EV_KEYS];                       // the list, where every CTA has all of it; else positions in hand
  };
  int sum[3][EV_BINS];                       // of rounds in turn; the first CTA's are the cluster's
  int total;                                 // of this CTA's stretch, read by the others
  int warp[EV_WARPS];
  int found[3];
  int place[EV_WARPS][EV_WARPS];
  int cands;
  uint64_t border;
  uint64_t cand[EV_RANKED];
  uint32_t keys[EV_KEYS];
};

__device__ __forceinline__ uint32_t cluster_rank() {
  uint32_t r;
  asm("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
  return r;
}
__device__ __forceinline__ uint32_t cluster_size() {
  uint32_t r;
  asm("mov.u32 %0, %%cluster_nctaid.x;" : "=r"(r));
  return r;
}
__device__ __forceinline__ void cluster_sync() {
  asm volatile("barrier.cluster.arrive.release.aligned;\nbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
__device__ __forceinline__ uint32_t peer(const int* p, uint32_t rank) {   // the same variable of another CTA
  uint32_t to;
  asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(to) : "r"((uint32_t)__cvta_generic_to_shared(p)), "r"(rank));
  return to;
}
__device__ __forceinline__ int peer_int(const int* p, uint32_t rank) {
  int v;
  asm volatile("ld.shared::cluster.s32 %0, [%1];" : "=r"(v) : "r"(peer(p, rank)) : "memory");
  return v;
}
__device__ __forceinline__ int4 peer_int4(const int* p, uint32_t rank) {
  int4 v;
  asm volatile("ld.shared::cluster.v4.s32 {%0, %1, %2, %3}, [%4];"
               : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(peer(p, rank)) : "memory");
  return v;
}
__device__ __forceinline__ void peer_add(int* p, uint32_t rank, int v) {
  asm volatile("red.relaxed.cluster.shared::cluster.add.s32 [%0], %1;" ::"r"(peer(p, rank)), "r"(v) : "memory");
}

// Sum over the block, to all threads.
__device__ __forceinline__ int block_sum(int v, int* warp) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  __syncthreads();
  if ((threadIdx.x & 31) == 0) warp[threadIdx.x >> 5] = v;
  __syncthreads();
  int t = 0;
#pragma unroll
  for (int w = 0; w < EV_WARPS; ++w) t += warp[w];
  return t;
}

__global__ void __launch_bounds__(EV_THREADS, 2) cache_evict_kernel(const EvictArgs a) {
  pdl_wait();
  extern __shared__ __align__(16) unsigned char sm[];
  EvictSmem& x = *reinterpret_cast<EvictSmem*>(sm);
  const uint32_t C = cluster_size(), rank = cluster_rank();
  const int item = blockIdx.x / C, n = item / a.from.H, h = item - n * a.from.H;
  const int tid = threadIdx.x, lane = tid & 31, wid = tid >> 5;
  const int raw = a.seq_len[n], L = cache_len(raw, a.from.S), stay = min(L, a.budget);
  const float* w = a.w + (size_t)item * a.from.S;
  float* to_w = a.to_w + (size_t)item * a.to.S;
  int32_t* kept = a.kept + (size_t)item * a.budget;
  if (h == 0 && rank == 0 && tid == 0) a.new_len[n] = raw < 0 ? raw : stay;
  for (int j = stay + rank * EV_THREADS + tid; j < a.budget; j += C * EV_THREADS) kept[j] = -1;
  const bool all = L <= a.budget;
  if (all)
    for (int j = rank * EV_THREADS + tid; j < L; j += C * EV_THREADS) kept[j] = j;
  if (stay == 0 || (all && a.in_place)) return;      // (all CTAs of the cluster)
  const bool whole = L <= EV_KEYS;                   // each CTA has all positions, and the whole list
  if (!all) {
    const bool split = !whole && C > 1;
    const int chunk = split ? (int)(((int64_t)L + C - 1) / C + EV_THREADS - 1) / EV_THREADS * EV_THREADS : L;
    const int p0 = split ? min((int64_t)L, (int64_t)rank * chunk) : 0, p1 = min((int64_t)L, (int64_t)p0 + chunk);
    const int lo = a.first, hi = L - a.recent, c0 = max(p0, lo), c1 = min(p1, hi);
    const bool cached = chunk <= EV_KEYS;
    if (cached) {                                    // (eight loads under way at a time)
#pragma unroll 8
      for (int i = p0 + tid; i < p1; i += EV_THREADS) x.keys[i - p0] = weight_key(w[i]);
    }
    auto key = [&](int i) { return cached ? x.keys[i - p0] : weight_key(w[i]); };
    // Larger weights first, then lower positions: the order of weight << 32 | ~position.
    auto order = [&](int i) { return (uint64_t)key(i) << 32 | (uint32_t)~i; };
    int left = a.budget - a.first - a.recent;        // to be found among [lo, hi)
    uint64_t border = ~0ull;                         // of them, the last in this order that stays
    if (left > 0) {
      for (int i = tid; i < EV_BINS * EV_COPIES / 4; i += EV_THREADS)
        reinterpret_cast<int4*>(x.hist)[i] = make_int4(0, 0, 0, 0);
      if (tid == 0) x.cands = 0;
      if (split) {
        for (int i = tid; i < 3 * EV_BINS / 4; i += EV_THREADS)
          reinterpret_cast<int4*>(&x.sum[0][0])[i] = make_int4(0, 0, 0, 0);
        cluster_sync();
      }
      __syncthreads();
      // eleven bits a round from the top, those of positions only where weights are equal
      border = 0;
#pragma unroll 1
      for (int round = 0; round < 6; ++round) {
        const int shift = 64 - 11 * (round + 1) > 0 ? 64 - 11 * (round + 1) : 0;
        const uint64_t known = round == 0 ? 0ull : ~0ull << (64 - 11 * round);
        const uint32_t digits = shift ? 2047 : (1 << (64 - 55)) - 1;
#pragma unroll 4
        for (int i = c0 + tid; i < c1; i += EV_THREADS) {
          const uint64_t k = order(i);
          if (((k ^ border) & known) == 0)
            atomicAdd(&x.hist[((uint32_t)(k >> shift) & digits) * EV_COPIES + (lane & (EV_COPIES - 1))], 1);
        }
        __syncthreads();
        // each thread EV_BINS / EV_THREADS = 4 bins, the largest digits first
        const int b0 = EV_BINS - 4 - 4 * tid;
        int part[4];
        int* sum = x.sum[round % 3];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int4 v = reinterpret_cast<const int4*>(x.hist)[b0 + i];
          part[i] = v.x + v.y + v.z + v.w;
          if (part[i]) {
            reinterpret_cast<int4*>(x.hist)[b0 + i] = make_int4(0, 0, 0, 0);
            if (split) peer_add(&sum[b0 + i], 0, part[i]);
          }
        }
        if (split) {
          cluster_sync();
          const int4 t = peer_int4(&sum[b0], 0);
          part[0] = t.x; part[1] = t.y; part[2] = t.z; part[3] = t.w;
          // last read before this barrier, next written after the one to come
          reinterpret_cast<int4*>(x.sum[(round + 2) % 3])[tid] = make_int4(0, 0, 0, 0);
        }
        const int mine = part[0] + part[1] + part[2] + part[3];
        int before = mine;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
          const int y = __shfl_up_sync(0xffffffffu, before, o);
          if (lane >= o) before += y;
        }
        if (lane == 31) x.warp[wid] = before;
        __syncthreads();
        before -= mine;
#pragma unroll
        for (int v = 0; v < EV_WARPS; ++v)
          if (v < wid) before += x.warp[v];
#pragma unroll
        for (int i = 3; i >= 0; --i) {
          if (before < left && left <= before + part[i]) {     // one bin of one thread
            x.found[0] = b0 + i;
            x.found[1] = left - before;
            x.found[2] = part[i];
          }
          before += part[i];
        }
        __syncthreads();
        border |= (uint64_t)x.found[0] << shift;
        left = x.found[1];
        const int cands = x.found[2];
        if (left == cands) break;                    // all that begin so stay
        if (whole && cands <= EV_RANKED) {
          const uint64_t same = ~0ull << shift;
          for (int i = c0 + tid; i < c1; i += EV_THREADS) {
            const uint64_t k = order(i);
            if (((k ^ border) & same) == 0) x.cand[atomicAdd(&x.cands, 1)] = k;
          }
          __syncthreads();
          if (tid < cands) {
            const uint64_t k = x.cand[tid];
            int larger = 0;
#pragma unroll 8
            for (int i = 0; i < cands; ++i) larger += x.cand[i] > k;
            if (larger == left - 1) x.border = k;
          }
          __syncthreads();
          border = x.border;
          break;
        }
      }
    }
    __syncthreads();
    // ---- each one's place, in order of position
    auto stays = [&](int i) { return i < lo || i >= hi || order(i) >= border; };
    int places = 0;                          // before this stretch
    if (split) {
      int m = 0;
#pragma unroll 4
      for (int i = p0 + tid; i < p1; i += EV_THREADS) m += stays(i);
      m = block_sum(m, x.warp);
      if (tid == 0) x.total = m;
      cluster_sync();
      for (uint32_t r = 0; r < rank; ++r) places += peer_int(&x.total, r);
    }
    int32_t* list = whole ? x.kept : kept;
#pragma unroll 1
    for (int i0 = p0; i0 < p1; i0 += EV_THREADS * EV_WARPS) {
      // sixteen positions a thread, EV_THREADS apart: counts of each 32 neighbours, then their sums
      uint32_t ma[EV_WARPS];
#pragma unroll
      for (int u = 0; u < EV_WARPS; ++u) {
        ma[u] = 0;
        if (i0 + u * EV_THREADS < p1) {
          const int i = i0 + u * EV_THREADS + tid;
          ma[u] = __ballot_sync(0xffffffffu, i < p1 && stays(i));
        }
        if (lane == 0) x.place[u][wid] = __popc(ma[u]);
      }
      __syncthreads();
      if (wid == 0) {                        // exclusive sums in order of (u, warp), eight entries a lane
        int* p = &x.place[0][0] + lane * 8;
        int v[8], t = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          v[i] = t;
          t += p[i];
        }
        int sum = t;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
          const int y = __shfl_up_sync(0xffffffffu, sum, o);
          if (lane >= o) sum += y;
        }
        if (lane == 31) x.found[0] = sum;
#pragma unroll
        for (int i = 0; i < 8; ++i) p[i] = sum - t + v[i];
      }
      __syncthreads();
      const uint32_t below = (1u << lane) - 1u;
#pragma unroll
      for (int u = 0; u < EV_WARPS; ++u)
        if (ma[u] >> lane & 1) list[places + x.place[u][wid] + __popc(ma[u] & below)] = i0 + u * EV_THREADS + tid;
      places += x.found[0];
      __syncthreads();
    }
    if (whole) {
      for (int j = rank * EV_THREADS + tid; j < stay; j += C * EV_THREADS) kept[j] = x.kept[j];
    } else {
      cluster_sync();                        // the list is whole
    }
  }

  // ---- records and weights that stay, in order, EV_VECS pieces a thread at a time. In place a record moves to
  // its own or a lower position, past all that later ones come from: what is in hand is read by all CTAs before
  // any of it is written.
  const int vecs = cache_record_bytes(a.from.d) / 16;
  int mine = EV_THREADS * EV_VECS / vecs;            // records of a CTA at a time: 455 of 144 bytes
  if (C > 1) {                                       // as many turns, but as many records for each of the cluster
    const uint32_t turns = (stay + C * mine - 1) / (C * mine);
    mine = (stay + C * turns - 1) / (C * turns);
  }
  const int step = EV_THREADS / vecs, rest = EV_THREADS - step * vecs;
  const int jt = tid / vecs, pt = tid - jt * vecs;
  const unsigned char* from = a.from.at(n, 0, h);
  unsigned char* to = a.to.at(n, 0, h);
  const uint32_t from_s = (uint32_t)a.from.s[1], to_s = (uint32_t)a.to.s[1];
#pragma unroll 1
  for (int64_t r0 = 0; r0 < stay; r0 += (int64_t)C * mine) {
    const int64_t j0 = r0 + (int64_t)rank * mine;
    const int m = (int)max((int64_t)0, min((int64_t)mine, stay - j0));
    const int* list = whole && !all ? x.kept + j0 : x.kept;
    if (all || !whole) {
      __syncthreads();
      for (int j = tid; j < m; j += EV_THREADS) x.kept[j] = all ? (int)j0 + j : __ldcg(&kept[j0 + j]);
      __syncthreads();
    }
    uint4 v[EV_VECS];
    float wv[4];                             // (narrow records: up to 2,048 of them)
    int j = jt, part = pt;
#pragma unroll
    for (int u = 0; u < EV_VECS; ++u) {
      if (j < m) v[u] = __ldcs(reinterpret_cast<const uint4*>(from + (uint64_t)(uint32_t)list[j] * from_s) + part);
      j += step;
      part += rest;
      if (part >= vecs) {
        part -= vecs;
        ++j;
      }
    }
#pragma unroll
    for (int u = 0; u < 4; ++u)
      if (tid + u * EV_THREADS < m) wv[u] = w[list[tid + u * EV_THREADS]];
    if (a.in_place) {
      if (C > 1) cluster_sync();
      else __syncthreads();
    }
    unsigned char* dst = to + (uint64_t)(uint32_t)j0 * to_s;
    j = jt;
    part = pt;
#pragma unroll
    for (int u = 0; u < EV_VECS; ++u) {
      if (j < m) reinterpret_cast<uint4*>(dst + (uint64_t)(uint32_t)j * to_s)[part] = v[u];
      j += step;
      part += rest;
      if (part >= vecs) {
        part -= vecs;
        ++j;
      }
    }
#pragma unroll
    for (int u = 0; u < 4; ++u)
      if (tid + u * EV_THREADS < m) to_w[j0 + tid + u * EV_THREADS] = wv[u];
  }
  if (C > 1 && !whole) cluster_sync();       // nobody leaves while its counts may be read
}

// [first byte, last byte] of a cache's records, as offsets from 0
void span(const lilicorr_cache_desc* d, const void* p, __int128* lo, __int128* hi) {
  const int64_t e[3] = {d->sequences, d->capacity, d->kv_heads};
  *lo = (__int128)(uintptr_t)p;
  *hi = *lo + cache_record_bytes(d->head_dim);
  for (int i = 0; i < 3; ++i)
    if (e[i] > 1) *hi += (__int128)(e[i] - 1) * d->stride[i];
}

lilicorr_status_t run_evict(const lilicorr_cache_desc* desc, void* cache, float* weights,
                            const int32_t* seq_len, int budget, int recent, int first,
                            const lilicorr_cache_desc* into, void* into_cache, float* into_weights,
                            int32_t* kept, int32_t* new_len, cudaStream_t st) {
  LL_TRY(cache_shape(desc));
  if (budget < 1 || recent < 0 || first < 0 || (int64_t)recent + first > budget) return LILICORR_ERR_ARG;
  if (budget > (1 << 30)) return LILICORR_ERR_SHAPE;           // (places are counted in 32 bits)
  EvictArgs a;
  LL_TRY(cache_view(desc, cache, into == nullptr, &a.from));   // in place it is written
  a.to = a.from;
  if (into) {
    LL_TRY(cache_shape(into));
    if (into->sequences != desc->sequences || into->kv_heads != desc->kv_heads ||
        into->head_dim != desc->head_dim || into->capacity < budget)
      return LILICORR_ERR_SHAPE;
    if (into->k_unit != desc->k_unit || into->v_unit != desc->v_unit) return LILICORR_ERR_ARG;
    LL_TRY(cache_view(into, into_cache, true, &a.to));
  } else if (into_cache || into_weights) {
    return LILICORR_ERR_ARG;
  }
  if (desc->sequences == 0) return LILICORR_OK;
  if (!seq_len || !kept || !new_len || (desc->capacity && !weights) || (into && !into_weights))
    return LILICORR_ERR_ARG;
  // every head's CTAs read the lengths
  if (seq_len < new_len + desc->sequences && new_len < seq_len + desc->sequences) return LILICORR_ERR_ARG;
  if (into && desc->capacity) {
    __int128 lo[2], hi[2];
    span(desc, cache, &lo[0], &hi[0]);
    span(into, into_cache, &lo[1], &hi[1]);
    if (lo[0] < hi[1] && lo[1] < hi[0]) return LILICORR_ERR_ARG;
    const size_t rows = (size_t)desc->sequences * desc->kv_heads;
    if (weights < into_weights + rows * into->capacity && into_weights < weights + rows * desc->capacity)
      return LILICORR_ERR_ARG;
  }
  a.w = weights;
  a.to_w = into ? into_weights : weights;
  a.seq_len = seq_len;
  a.budget = budget;
  a.recent = recent;
  a.first = first;
  a.in_place = into == nullptr;
  a.kept = kept;
  a.new_len = new_len;
  // as many CTAs an item as keep two an SM busy, up to eight
  const int64_t items = (int64_t)desc->sequences * desc->kv_heads;
  int cluster = 8;
  while (cluster > 1 && items * cluster > 2 * num_sms()) cluster /= 2;
  if (items * cluster > 0x7FFFFFFFll) return LILICORR_ERR_SHAPE;
  static bool configured[64] = {false};
  LL_TRY(allow_max_dynamic_smem(cache_evict_kernel, configured));
  return launch_cluster_k(cache_evict_kernel, (unsigned)(items * cluster), EV_THREADS, sizeof(EvictSmem), cluster,
                          st, a);
}

}  // namespace
}  // namespace lilicorr

using namespace lilicorr;

extern "C" {

size_t lilicorr_cache_record_bytes(int head_dim) {
  return head_dim < 16 || head_dim > 128 || head_dim % 16 ? 0 : (size_t)cache_record_bytes(head_dim);
}

lilicorr_status_t lilicorr_cache_append(const lilicorr_cache_desc* desc, void* cache,
                                        lilicorr_dtype_t dtype, int tokens, const void* k,
                                        const int64_t host_k_stride[3], const void* v,
                                        const int64_t host_v_stride[3], const int32_t* seq_len,
                                        float* weights, cudaStream_t stream) {
  return run_tokens(desc, cache, dtype, tokens, k, host_k_stride, v, host_v_stride, seq_len, weights, true,
                    stream);
}

lilicorr_status_t lilicorr_cache_read(const lilicorr_cache_desc* desc, const void* cache,
                                      lilicorr_dtype_t dtype, int tokens, void* k,
                                      const int64_t host_k_stride[3], void* v,
                                      const int64_t host_v_stride[3], const int32_t* seq_len,
                                      cudaStream_t stream) {
  return run_tokens(desc, cache, dtype, tokens, k, host_k_stride, v, host_v_stride, seq_len, nullptr, false,
                    stream);
}

lilicorr_status_t lilicorr_cache_evict(const lilicorr_cache_desc* desc, void* cache, float* weights,
                                       const int32_t* seq_len, int budget, int recent, int first,
                                       const lilicorr_cache_desc* into, void* into_cache,
                                       float* into_weights, int32_t* kept, int32_t* new_len,
                                       cudaStream_t stream) {
  return run_evict(desc, cache, weights, seq_len, budget, recent, first, into, into_cache, into_weights, kept,
                   new_len, stream);
}

}  // extern "C"
