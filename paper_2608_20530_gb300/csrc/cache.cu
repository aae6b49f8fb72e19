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
struct CacheTokens {
  const void* k;               // read: written
  const void* v;
  int64_t k_s[3], v_s[3];      // elements: sequence, token, head
  int T;
  const int32_t* seq_len;
  float* weights;
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
// the two codes of a byte
__device__ __forceinline__ float2 code_values(uint32_t byte) {
  float2 f;
  asm("{\n .reg .b8 t;\n .reg .b32 w;\n .reg .b16 lo, hi;\n cvt.u8.u32 t, %2;\n cvt.rn.f16x2.e2m1x2 w, t;\n"
      " mov.b32 {lo, hi}, w;\n cvt.f32.f16 %0, lo;\n cvt.f32.f16 %1, hi;\n}"
      : "=f"(f.x), "=f"(f.y) : "r"(byte));
  return f;
}

__device__ __forceinline__ void load16(const __nv_bfloat16* p, float (&x)[16]) {
  uint4 w[2] = {reinterpret_cast<const uint4*>(p)[0], reinterpret_cast<const uint4*>(p)[1]};
  const uint32_t* u = reinterpret_cast<const uint32_t*>(w);
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    x[2 * i] = __uint_as_float(u[i] << 16);
    x[2 * i + 1] = __uint_as_float(u[i] & 0xFFFF0000u);
  }
}
__device__ __forceinline__ void load16(const float* p, float (&x)[16]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) reinterpret_cast<float4*>(x)[i] = reinterpret_cast<const float4*>(p)[i];
}
__device__ __forceinline__ void store16(__nv_bfloat16* p, const float (&x)[16]) {
  uint32_t u[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) u[i] = bf16_pack2(x[2 * i], x[2 * i + 1]);
  reinterpret_cast<uint4*>(p)[0] = *reinterpret_cast<uint4*>(u);
  reinterpret_cast<uint4*>(p)[1] = *reinterpret_cast<uint4*>(u + 4);
}
__device__ __forceinline__ void store16(float* p, const float (&x)[16]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) reinterpret_cast<float4*>(p)[i] = reinterpret_cast<const float4*>(x)[i];
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

// The codes of 16 elements whose scale times the unit is su. In bf16 x / su is a border between two codes or
// at least 2^-10 away from it, so that the product with the rounded inverse, rounded to multiples of 2^-12,
// falls on the same side; fp32 elements are compared with the borders, which are exact products.
__device__ __forceinline__ uint2 group_codes(const float (&x)[16], float su, __nv_bfloat16) {
  const float inv = 1.f / su, big = 0x1.8p11f;
  uint32_t w[2] = {0, 0};
#pragma unroll
  for (int i = 0; i < 16; i += 2)
    w[i / 8] |= codes2(fmaf(x[i], inv, big) - big, fmaf(x[i + 1], inv, big) - big) << (i % 8 * 4);
  return make_uint2(w[0], w[1]);
}
__device__ __forceinline__ uint2 group_codes(const float (&x)[16], float su, float) {
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

// A thread has one group of 16 elements; groups in the order (token, head, key or value, group).
struct CacheGroup { int n, t, h, kv, g, pos; };
__device__ __forceinline__ bool cache_group(const CacheView& c, const CacheTokens& a, CacheGroup* x) {
  uint32_t i = blockIdx.x * blockDim.x + threadIdx.x;
  const uint32_t G = c.d / 16, per = 2 * G * c.H, total = per * (uint32_t)a.T * (uint32_t)c.N;
  if (i >= total) return false;
  const uint32_t row = i / per;
  i -= row * per;
  x->n = row / a.T;
  x->t = row - x->n * a.T;
  x->h = i / (2 * G);
  i -= x->h * 2 * G;
  x->kv = i >= G;
  x->g = i - x->kv * G;
  const int len = a.seq_len[x->n];
  x->pos = len < 0 ? -1 : len - a.T + x->t;
  return true;
}

template <typename E>
__global__ void __launch_bounds__(256) cache_append_kernel(const CacheView c, const CacheTokens a) {
  pdl_wait();
  CacheGroup x;
  if (!cache_group(c, a, &x) || x.pos < 0 || x.pos >= c.S) return;
  const E* src = static_cast<const E*>(x.kv ? a.v : a.k);
  const int64_t* s = x.kv ? a.v_s : a.k_s;
  float e[16];
  load16(src + (x.n * s[0] + x.t * s[1] + x.h * s[2] + x.g * 16), e);
  float top = 0.f;
#pragma unroll
  for (int i = 0; i < 16; ++i) top = max_nan(top, fabsf(e[i]));
  const float unit = x.kv ? c.v_unit : c.k_unit;
  const uint32_t b = group_scale(top, 1.f / unit);
  unsigned char* rec = c.at(x.n, x.pos, x.h) + x.kv * cache_half_bytes(c.d);
  *reinterpret_cast<uint2*>(rec + x.g * 8) = group_codes(e, scale_value(b) * unit, E());
  rec[c.d / 2 + x.g] = (unsigned char)b;
  if (x.g == 0)                                      // scales that no group has
    for (int i = c.d / 16; i < 8; ++i) rec[c.d / 2 + i] = 0;
  if (a.weights && x.g == 0 && !x.kv) a.weights[((size_t)x.n * c.H + x.h) * c.S + x.pos] = 0.f;
}

template <typename E>
__global__ void __launch_bounds__(256) cache_read_kernel(const CacheView c, const CacheTokens a) {
  pdl_wait();
  CacheGroup x;
  if (!cache_group(c, a, &x)) return;
  float e[16];
#pragma unroll
  for (int i = 0; i < 16; ++i) e[i] = 0.f;
  if (x.pos >= 0 && x.pos < c.S) {
    const unsigned char* rec = c.at(x.n, x.pos, x.h) + x.kv * cache_half_bytes(c.d);
    const uint2 w = *reinterpret_cast<const uint2*>(rec + x.g * 8);
    const float su = scale_value(rec[c.d / 2 + x.g]) * (x.kv ? c.v_unit : c.k_unit);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float2 f = code_values(((i < 4 ? w.x : w.y) >> (i % 4 * 8)) & 0xFFu);
      e[2 * i] = f.x * su;
      e[2 * i + 1] = f.y * su;
    }
  }
  E* dst = static_cast<E*>(const_cast<void*>(x.kv ? a.v : a.k));
  const int64_t* s = x.kv ? a.v_s : a.k_s;
  store16(dst + (x.n * s[0] + x.t * s[1] + x.h * s[2] + x.g * 16), e);
}

lilicorr_status_t run_tokens(const lilicorr_cache_desc* desc, const void* cache, lilicorr_dtype_t dtype,
                             int tokens, const void* k, const int64_t* ks, const void* v,
                             const int64_t* vs, const int32_t* seq_len, float* weights, bool append,
                             cudaStream_t st) {
  LL_TRY(cache_shape(desc));
  if (dtype != LILICORR_F32 && dtype != LILICORR_BF16) return LILICORR_ERR_DTYPE;
  if (tokens < 0) return LILICORR_ERR_SHAPE;
  const double groups = (double)desc->sequences * tokens * desc->kv_heads * (desc->head_dim / 8);
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

constexpr int EV_THREADS = 1024;

// Exclusive sums of two flags over the block; `sums`: 64 words.
__device__ __forceinline__ void scan2(bool a, bool b, int* sums, int& ra, int& rb, int& ta, int& tb) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const uint32_t ba = __ballot_sync(0xffffffffu, a), bb = __ballot_sync(0xffffffffu, b);
  const uint32_t below = (1u << lane) - 1u;
  __syncthreads();
  if (lane == 0) {
    sums[warp] = __popc(ba);
    sums[32 + warp] = __popc(bb);
  }
  __syncthreads();
  ra = __popc(ba & below);
  rb = __popc(bb & below);
  ta = tb = 0;
  for (int i = 0; i < EV_THREADS / 32; ++i) {
    const int x = sums[i], y = sums[32 + i];
    if (i < warp) { ra += x; rb += y; }
    ta += x;
    tb += y;
  }
}

// The positions that stay, a CTA a (sequence, head): the weight of the last one that does, digit by digit
// from the top, then all positions in order.
__global__ void __launch_bounds__(EV_THREADS) cache_choose_kernel(const EvictArgs a) {
  pdl_wait();
  __shared__ int hist[256], sums[64], found[2];
  const int n = blockIdx.x / a.from.H, tid = threadIdx.x;
  const int raw = a.seq_len[n], L = cache_len(raw, a.from.S);
  const float* w = a.w + (size_t)blockIdx.x * a.from.S;
  int32_t* kept = a.kept + (size_t)blockIdx.x * a.budget;
  if (blockIdx.x % a.from.H == 0 && tid == 0) a.new_len[n] = raw < 0 ? raw : min(L, a.budget);
  if (L <= a.budget) {
    for (int i = tid; i < a.budget; i += EV_THREADS) kept[i] = i < L ? i : -1;
    return;
  }
  const int lo = a.first, hi = L - a.recent;
  int left = a.budget - a.first - a.recent;          // to be found among [lo, hi)
  uint32_t top = 0;                                  // the digits known so far
  const bool some = left > 0;
  if (some)
    for (int shift = 24; shift >= 0; shift -= 8) {
      for (int i = tid; i < 256; i += EV_THREADS) hist[i] = 0;
      __syncthreads();
      for (int i = lo + tid; i < hi; i += EV_THREADS) {
        const uint32_t k = weight_key(w[i]);
        if (shift == 24 || k >> (shift + 8) == top >> (shift + 8)) atomicAdd(&hist[(k >> shift) & 255], 1);
      }
      __syncthreads();
      if (tid == 0) {
        int b = 255, need = left;
        while (b > 0 && hist[b] < need) need -= hist[b--];
        found[0] = b;
        found[1] = need;
      }
      __syncthreads();
      top |= (uint32_t)found[0] << shift;
      left = found[1];
    }
  // of the weights equal to `top`, `left` stay
  int at = 0, equal = 0;
  for (int i0 = 0; i0 < L; i0 += EV_THREADS) {
    const int i = i0 + tid;
    const bool there = i < L, fixed = i < lo || i >= hi;
    const uint32_t k = there && !fixed ? weight_key(w[i]) : 0;
    const bool same = there && !fixed && some && k == top;
    int r_same, r_keep, t_same, t_keep;
    scan2(same, false, sums, r_same, r_keep, t_same, t_keep);
    const bool keep = there && (fixed || (some && (k > top || (same && equal + r_same < left))));
    equal += t_same;
    scan2(keep, false, sums, r_keep, r_same, t_keep, t_same);
    if (keep) kept[at + r_keep] = i;
    at += t_keep;
  }
}

constexpr int EV_STAGE = 128;  // records that move at a time

// The records and weights that stay, moved to the front, a CTA a (sequence, head). In place a record moves to
// its own or a lower position, past all that later ones come from, so records go in order, EV_STAGE at a
// time, all of them read before any of them is written.
__global__ void __launch_bounds__(256) cache_move_kernel(const EvictArgs a) {
  pdl_wait();
  __shared__ __align__(16) unsigned char stage[EV_STAGE * cache_record_bytes(128)];
  __shared__ float sw[EV_STAGE];
  const int n = blockIdx.x / a.from.H, h = blockIdx.x % a.from.H, tid = threadIdx.x;
  const int L = cache_len(a.seq_len[n], a.from.S), keep = min(L, a.budget);
  if (a.in_place && L <= a.budget) return;
  const int32_t* kept = a.kept + (size_t)blockIdx.x * a.budget;
  const float* w = a.w + (size_t)blockIdx.x * a.from.S;
  float* to_w = a.to_w + (size_t)blockIdx.x * a.to.S;
  const int vecs = cache_record_bytes(a.from.d) / 16;
  for (int j0 = 0; j0 < keep; j0 += EV_STAGE) {
    const int m = min(EV_STAGE, keep - j0);
    for (int i = tid; i < m * vecs; i += 256) {
      const int j = i / vecs, v = i - j * vecs;
      reinterpret_cast<uint4*>(stage)[i] = reinterpret_cast<const uint4*>(a.from.at(n, kept[j0 + j], h))[v];
    }
    if (tid < m) sw[tid] = w[kept[j0 + tid]];
    __syncthreads();
    for (int i = tid; i < m * vecs; i += 256) {
      const int j = i / vecs, v = i - j * vecs;
      reinterpret_cast<uint4*>(a.to.at(n, j0 + j, h))[v] = reinterpret_cast<const uint4*>(stage)[i];
    }
    if (tid < m) to_w[j0 + tid] = sw[tid];
    __syncthreads();
  }
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
  if ((double)desc->sequences * desc->kv_heads * budget >= 9e18) return LILICORR_ERR_SHAPE;
  EvictArgs a;
  LL_TRY(cache_view(desc, cache, true, &a.from));
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
  const unsigned grid = (unsigned)(desc->sequences * desc->kv_heads);
  LL_TRY(launch_k(cache_choose_kernel, grid, EV_THREADS, 0, st, a));
  return launch_k(cache_move_kernel, grid, 256, 0, st, a);
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
