// Attention over a cache held in 4 bits.
#include "cache.cuh"

namespace lilicorr {
namespace {

struct CaArgs {
  CacheView c;
  const void* q;
  int64_t q_s[3];              // elements: sequence, token, head
  void* out;
  int64_t o_s[3];
  float* lse;                  // [N, T, Hq]
  const int32_t* seq_len;
  float* weights;              // [N, H, S] or null
  int T, Hq, rep;
  float scale;
};

__device__ __forceinline__ float ca_element(const unsigned char* half, int d, int i) {
  const uint32_t c = (half[i / 2] >> (i % 2 * 4)) & 15u, s = half[d / 2 + i / 16];
  const uint32_t e = (c >> 1) & 3u, f = c & 1u;
  float x = e == 0 ? 0.5f * f : (1.f + 0.5f * f) * (float)(1 << (e - 1));
  if (c & 8u) x = -x;
  const uint32_t se = s >> 3, sf = s & 7u;
  const float y = s == 127 ? NAN : se == 0 ? sf * 0x1p-9f : (8.f + sf) * exp2f((float)se - 10.f);
  return x * y;
}

// A warp a row: four elements of each key a lane, one key after the other. Then, where weights are asked
// for, the scores once more.
template <typename E>
__global__ void __launch_bounds__(32) ca_simple_kernel(const CaArgs a) {
  pdl_wait();
  const int lane = threadIdx.x, d = a.c.d;
  const int hq = blockIdx.x % a.Hq, nt = blockIdx.x / a.Hq, t = nt % a.T, n = nt / a.T, h = hq / a.rep;
  const int raw = a.seq_len[n];
  if (raw < 0) return;
  const int seen = max(0, cache_len(raw, a.c.S) - (a.T - 1 - t));
  const E* q = static_cast<const E*>(a.q) + n * a.q_s[0] + t * a.q_s[1] + hq * a.q_s[2];
  float x[4], o[4] = {0.f, 0.f, 0.f, 0.f}, m = -INFINITY, l = 0.f;
  for (int i = 0; i < 4; ++i) x[i] = lane * 4 + i < d ? ld_elem(q, lane * 4 + i) : 0.f;
  auto score = [&](int j) {
    const unsigned char* rec = a.c.at(n, j, h);
    float s = 0.f;
    for (int i = 0; i < 4; ++i)
      if (lane * 4 + i < d) s = fmaf(x[i], ca_element(rec, d, lane * 4 + i), s);
    return warp_sum(s) * (a.scale * a.c.k_unit);
  };
  for (int j = 0; j < seen; ++j) {
    const float s = score(j), top = s > m ? s : m, f = expf(m - top), p = expf(s - top);
    const unsigned char* rec = a.c.at(n, j, h) + cache_half_bytes(d);
    l = l * f + p;
    m = top;
    for (int i = 0; i < 4; ++i)
      if (lane * 4 + i < d) o[i] = o[i] * f + p * ca_element(rec, d, lane * 4 + i);
  }
  E* out = static_cast<E*>(a.out) + n * a.o_s[0] + t * a.o_s[1] + hq * a.o_s[2];
  for (int i = 0; i < 4; ++i)
    if (lane * 4 + i < d) st_elem(out, lane * 4 + i, seen ? o[i] / l * a.c.v_unit : 0.f);
  const float lse = seen ? m + logf(l) : -INFINITY;
  if (lane == 0) a.lse[(size_t)nt * a.Hq + hq] = lse;
}

__global__ void __launch_bounds__(256) ca_simple_weights_kernel(const CaArgs a, int bf16) {
  pdl_wait();
  const size_t i = (size_t)blockIdx.x * 256 + threadIdx.x;
  if (i >= (size_t)a.c.N * a.c.H * a.c.S) return;
  const int j = i % a.c.S, h = i / a.c.S % a.c.H, n = i / a.c.S / a.c.H, d = a.c.d;
  const int raw = a.seq_len[n], L = cache_len(raw, a.c.S);
  if (raw < 0 || j >= L) return;
  const unsigned char* rec = a.c.at(n, j, h);
  float sum = 0.f;
  for (int t = max(0, a.T - L + j); t < a.T; ++t)
    for (int r = 0; r < a.rep; ++r) {
      const int64_t at = n * a.q_s[0] + t * a.q_s[1] + (h * a.rep + r) * a.q_s[2];
      float s = 0.f;
      for (int e = 0; e < d; ++e)
        s = fmaf(bf16 ? ld_elem(static_cast<const __nv_bfloat16*>(a.q), at + e)
                      : ld_elem(static_cast<const float*>(a.q), at + e), ca_element(rec, d, e), s);
      const float lse = a.lse[((size_t)n * a.T + t) * a.Hq + h * a.rep + r];
      if (fabsf(lse) < INFINITY) sum += expf(s * (a.scale * a.c.k_unit) - lse);
    }
  a.weights[i] += sum;
}

lilicorr_status_t ca_shape(const lilicorr_cache_attention_desc* d) {
  if (!d) return LILICORR_ERR_ARG;
  LL_TRY(cache_shape(&d->cache));
  if (d->dtype != LILICORR_F32 && d->dtype != LILICORR_BF16) return LILICORR_ERR_DTYPE;
  if (d->tokens < 1 || d->q_heads < 1 || d->q_heads % d->cache.kv_heads) return LILICORR_ERR_SHAPE;
  if ((double)d->cache.sequences * d->tokens * d->q_heads >= 2147483648.0) return LILICORR_ERR_SHAPE;
  return LILICORR_OK;
}

}  // namespace
}  // namespace lilicorr

using namespace lilicorr;

extern "C" {

size_t lilicorr_cache_attention_workspace_bytes(const lilicorr_cache_attention_desc* desc) {
  return ca_shape(desc) == LILICORR_OK ? 256 : 0;
}

lilicorr_status_t lilicorr_cache_attention(const lilicorr_cache_attention_desc* desc, const void* q,
                                           const void* cache, const int32_t* seq_len, void* out,
                                           float* lse, float* weights, void* ws, size_t ws_bytes,
                                           cudaStream_t stream) {
  LL_TRY(ca_shape(desc));
  const float scale = desc->scale;
  if (!(scale > 0.f) || !((double)scale * desc->cache.k_unit < 0x1p100)) return LILICORR_ERR_ARG;
  CaArgs a;
  memset(&a, 0, sizeof(a));
  LL_TRY(cache_view(&desc->cache, cache, false, &a.c));
  if (desc->cache.sequences == 0) return LILICORR_OK;
  if (!q || !out || !lse || !ws || !seq_len) return LILICORR_ERR_ARG;
  if (!aligned16(q) || !aligned16(out) || !aligned16(ws)) return LILICORR_ERR_ARG;
  const int64_t e[3] = {desc->cache.sequences, desc->tokens, desc->q_heads};
  const int per16 = desc->dtype == LILICORR_BF16 ? 8 : 4;
  if (!cache_rows_ok(desc->q_stride, e, per16, a.c.d, false) ||
      !cache_rows_ok(desc->out_stride, e, per16, a.c.d, true))
    return LILICORR_ERR_ARG;
  if (ws_bytes < 256) return LILICORR_ERR_WORKSPACE;
  a.q = q;
  a.out = out;
  for (int i = 0; i < 3; ++i) {
    a.q_s[i] = e[i] > 1 ? desc->q_stride[i] : 0;
    a.o_s[i] = e[i] > 1 ? desc->out_stride[i] : 0;
  }
  a.lse = lse;
  a.seq_len = seq_len;
  a.weights = weights;
  a.T = desc->tokens;
  a.Hq = desc->q_heads;
  a.rep = desc->q_heads / a.c.H;
  a.scale = scale;
  const bool bf = desc->dtype == LILICORR_BF16;
  const unsigned grid = (unsigned)(e[0] * e[1] * e[2]);
  if (bf) LL_TRY(launch_k(ca_simple_kernel<__nv_bfloat16>, grid, 32, 0, stream, a));
  else LL_TRY(launch_k(ca_simple_kernel<float>, grid, 32, 0, stream, a));
  const size_t keys = (size_t)a.c.N * a.c.H * a.c.S;
  if (!weights || !keys) return LILICORR_OK;
  if ((keys + 255) / 256 > 0x7FFFFFFFull) return LILICORR_ERR_SHAPE;
  return launch_k(ca_simple_weights_kernel, (unsigned)((keys + 255) / 256), 256, 0, stream, a, (int)bf);
}

}  // extern "C"
