// Attention over a cache held in 4 bits: the call, and the kernels for the usual widths.
#include "cache_attention_kernels.cuh"

namespace lilicorr {

extern template lilicorr_status_t ca_launch_rows<32, 0>(const CaArgs&, const CaPlan&, cudaStream_t);
extern template lilicorr_status_t ca_launch_rows<64, 0>(const CaArgs&, const CaPlan&, cudaStream_t);
extern template lilicorr_status_t ca_launch_rows<128, 0>(const CaArgs&, const CaPlan&, cudaStream_t);
template lilicorr_status_t ca_launch_rows<64, 64>(const CaArgs&, const CaPlan&, cudaStream_t);
template lilicorr_status_t ca_launch_rows<128, 128>(const CaArgs&, const CaPlan&, cudaStream_t);

namespace {

int g_ca_path = 0;             // test hook: 1 the tensor-core kernel for all bf16 queries, 2 for none

lilicorr_status_t ca_plan(const lilicorr_cache_attention_desc* d, CaPlan* p) {
  if (!d) return LILICORR_ERR_ARG;
  LL_TRY(cache_shape(&d->cache));
  if (d->dtype != LILICORR_F32 && d->dtype != LILICORR_BF16) return LILICORR_ERR_DTYPE;
  const lilicorr_cache_desc& c = d->cache;
  if (d->tokens < 1 || d->q_heads < 1 || d->q_heads % c.kv_heads) return LILICORR_ERR_SHAPE;
  const double all = (double)c.sequences * d->tokens * d->q_heads;
  if (all > 0x1p30 || (double)d->tokens * d->q_heads > 0x1p30) return LILICORR_ERR_SHAPE;
  const int rows = d->tokens * (d->q_heads / c.kv_heads);
  p->dp = c.head_dim <= 32 ? 32 : c.head_dim <= 64 ? 64 : 128;
  p->pieces = d->dtype == LILICORR_BF16 ? 1 : 3;
  // More than 32 rows go to the 5th-generation tensor cores, 128 at a time, fewer to mma.sync, where each 16 keys
  // cost a matrix instruction for every 8 rows: 32 sequences of 8,192 keys, d = 128, 16 rows a kv head 101 us (on
  // tcgen05 135), 32 rows 147 (141; d = 64 100 and 115), 48 rows 270 (144), 64 rows 275 (148). Few short contexts
  // stay on mma.sync: 8 of 384 keys, 64 rows 13 us (25), 64 of 256 69 (46).
  const int64_t small = (int64_t)c.sequences * c.kv_heads * ((rows + 31) / 32);
  p->tc = p->pieces == 1 && (g_ca_path ? g_ca_path == 1 : rows > 32 && (c.capacity > 512 || small > num_sms()));
  if (p->tc && p->dp < 64) p->dp = 64;
  p->nt = rows <= 8 ? 1 : rows <= 16 || p->pieces > 1 ? 2 : 4;
  const int per_block = p->tc ? 128 : 8 * p->nt;
  p->blocks = (rows + per_block - 1) / per_block;
  p->items = (size_t)c.sequences * c.kv_heads * p->blocks;
  // An item a CTA where there is little to share out, or where many items balance by themselves: no list to find
  // one's place in, no parts to join. 64 items of 640 keys 7.4 us (cut evenly 8.8), of 1,024 8.9 (9.0), of
  // 2,048 13.9 (11.5); 128 items of 2,048 keys 14.0 (15.9), 512 40.5 (44.0), 2,048 130 (133).
  p->whole = !p->tc && (c.capacity <= 1024 || (c.capacity <= 2048 && p->items >= (size_t)num_sms() * 3 / 4));
  if ((double)p->items * (c.capacity / 128 + 1) >= 2147483648.0) return LILICORR_ERR_SHAPE;
  // the widest team of at most 16: all heads of a position where there are so few. Measured for 8 heads whose records
  // lie side by side (32 sequences of 8,192: 193 MB read for 259 one head after the other); caches by head, where heads
  // share no line, and 11 or more heads, which leave up to 9 SMs without a CTA, take the same rule unmeasured.
  p->team = 1;
  for (int i = 2; i <= 16; ++i)
    if (c.kv_heads % i == 0) p->team = i;
  p->ctas = num_sms() * (p->tc || p->nt * p->pieces > 3 || p->nt > 2 ? 1 : 2) / p->team * p->team;
  const size_t parts = p->whole ? 0 : (size_t)2 * p->ctas * per_block;
  p->pad = rows <= 16 ? (rows + 1) / 2 * 2 : 0;
  const size_t keys = (size_t)c.sequences * c.kv_heads * c.capacity;
  // the counts of parts keep their place in every call's layout: nothing else is ever written there
  p->left_off = 256;
  p->ml_off = p->left_off + align_up((size_t)4 * num_sms() * sizeof(uint32_t), 256);
  p->po_off = p->ml_off + align_up(parts * sizeof(float2), 256);
  p->rows_off = p->po_off + parts * p->dp * sizeof(float);
  p->factors_off = p->rows_off + align_up((size_t)all * sizeof(float2), 256);
  p->scores_off = p->factors_off + align_up((size_t)all * sizeof(float), 256);
  p->total = p->scores_off + align_up(keys * p->pad * sizeof(float), 256);
  return LILICORR_OK;
}

lilicorr_status_t run_cache_attention(const lilicorr_cache_attention_desc* desc, const void* q,
                                      const void* cache, const int32_t* seq_len, void* out, float* lse,
                                      float* weights, void* ws, size_t ws_bytes, cudaStream_t stream,
                                      long long wait_limit, int starve) {
  CaPlan p;
  LL_TRY(ca_plan(desc, &p));
  const double scale = (double)desc->scale * desc->cache.k_unit;
  if (!(scale > 0.0) || !(scale < 0x1p100)) return LILICORR_ERR_ARG;
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
  if (ws_bytes < p.total) return LILICORR_ERR_WORKSPACE;
  if (starve && (starve == 3 ? p.pieces > 1 || p.pad : !p.tc)) return LILICORR_ERR_SHAPE;
  unsigned char* w = static_cast<unsigned char*>(ws);
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
  a.blocks = p.blocks;
  a.team = p.team;
  a.whole = p.whole;
  const double log2e = 1.4426950408889634 * scale;
  a.scale = (float)log2e;
  a.scale_rest = (float)(log2e - a.scale);
  a.rest_ratio = (float)((log2e - a.scale) / log2e);
  a.left = reinterpret_cast<uint32_t*>(w + p.left_off);
  a.ml = reinterpret_cast<float2*>(w + p.ml_off);
  a.po = reinterpret_cast<float*>(w + p.po_off);
  a.status = reinterpret_cast<uint32_t*>(w);
  a.wait_limit = wait_limit;
  a.test_starve = starve;
  a.rows = reinterpret_cast<float2*>(w + p.rows_off);
  a.factors = reinterpret_cast<float*>(w + p.factors_off);
  a.scores = weights && p.pad ? reinterpret_cast<float*>(w + p.scores_off) : nullptr;
  a.pad = p.pad;
  if (a.c.d == 128) return ca_launch_rows<128, 128>(a, p, stream);
  if (a.c.d == 64) return ca_launch_rows<64, 64>(a, p, stream);
  return p.dp == 32   ? ca_launch_rows<32, 0>(a, p, stream)
         : p.dp == 64 ? ca_launch_rows<64, 0>(a, p, stream)
                      : ca_launch_rows<128, 0>(a, p, stream);
}

}  // namespace
}  // namespace lilicorr

using namespace lilicorr;

extern "C" {

size_t lilicorr_cache_attention_workspace_bytes(const lilicorr_cache_attention_desc* desc) {
  CaPlan p;
  return ca_plan(desc, &p) == LILICORR_OK ? p.total : 0;
}

lilicorr_status_t lilicorr_cache_attention(const lilicorr_cache_attention_desc* desc, const void* q,
                                           const void* cache, const int32_t* seq_len, void* out,
                                           float* lse, float* weights, void* ws, size_t ws_bytes,
                                           cudaStream_t stream) {
  return run_cache_attention(desc, q, cache, seq_len, out, lse, weights, ws, ws_bytes, stream, CA_WAIT, 0);
}

int lilicorr_test_cache_attention_path(int mode) {
  const int prev = g_ca_path;
  g_ca_path = mode < 0 ? 0 : mode > 2 ? 2 : mode;
  return prev;
}

lilicorr_status_t lilicorr_test_cache_attention_timeout(const lilicorr_cache_attention_desc* desc, const void* q,
                                                        const void* cache, const int32_t* seq_len, void* out,
                                                        float* lse, float* weights, void* ws,
                                                        size_t ws_bytes, long long wait_cycles, int which,
                                                        cudaStream_t stream) {
  if (wait_cycles < 100000 || wait_cycles > CA_WAIT || which < 1 || which > 3 || (which == 3) != (weights != nullptr))
    return LILICORR_ERR_ARG;
  return run_cache_attention(desc, q, cache, seq_len, out, lse, weights, ws, ws_bytes, stream, wait_cycles,
                             which);
}

}  // extern "C"
