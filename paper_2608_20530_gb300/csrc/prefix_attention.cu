// Attention of sequences that share a prefix: beams of a request, or drafted blocks under
// verification, each with a short cache of its own behind the request's.
//
//   out = sum_j softmax_j(scale q . k_j) v_j  over the prefix's keys and the sequence's own
//
// The softmax over the two key sets splits: with (m, l, o) = (max s, sum 2^(s - m), sum 2^(s - m) v)
// of each piece of the keys, the whole is sum 2^(m_i - M) o_i / sum 2^(m_i - M) l_i, M = max m_i. So
// the rows of ALL sequences of a group meet the prefix as one product (its keys are read once for
// all), each sequence's own keys are a second, and one pass joins the pieces. Scores, maxima, sums and
// o are fp32; on bf16 inputs the probabilities are rounded to bf16 for the second product, whose operands
// have one type with V (each term off by at most 2^-8 of itself, of either sign, where the output is
// rounded to 2^-8 as a whole); their sum is of the unrounded ones.
#include "prefix_attention.cuh"

#include "lilicorr_testing.h"

namespace lilicorr {

namespace {

constexpr int PM_STAGES = 3;
constexpr float LN2 = 0.69314718f, LN2_REST = -1.9046543e-9f;      // ln 2 = LN2 + LN2_REST

__device__ __forceinline__ uint32_t sm_addr(const void* p) {
  return static_cast<uint32_t>(__cvta_generic_to_shared(p));
}
__device__ __forceinline__ void ldsm4(uint32_t addr, uint32_t (&r)[4]) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0, %1, %2, %3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
               : "r"(addr));
}
__device__ __forceinline__ void ldsm4_t(uint32_t addr, uint32_t (&r)[4]) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
               : "r"(addr));
}
__device__ __forceinline__ void mma_16x8x16(float (&c)[4], const uint32_t (&a)[4], uint32_t b0,
                                            uint32_t b1) {
  asm volatile(
      "mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, "
      "{%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
      : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
      : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
// 16 bytes to shared memory, zeros where `live` is false (the source is not read then)
__device__ __forceinline__ void copy16(void* dst, const void* src, bool live) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(sm_addr(dst)), "l"(src),
               "r"(live ? 16 : 0)
               : "memory");
}
__device__ __forceinline__ void copy_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void copy_wait() {
  asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory");
}

// Stage keys [key0, key0 + KT) of one (group or sequence, head): rows of `row_bytes` live bytes in
// smem rows of ld bytes, zeros past `held` keys and past the head's width, so that whatever the cache
// holds behind its last token (NaN too) meets its zero probability as a zero.
template <int KT, int PIECES, int NT>
__device__ __forceinline__ void stage_rows(unsigned char* dst, const unsigned char* src, int64_t s_pos,
                                           int ld, int key0, int held, int pieces, int tid) {
#pragma unroll 4
  for (int i = tid; i < KT * PIECES; i += NT) {
    const int j = i / PIECES, p = i % PIECES;
    const bool live = key0 + j < held && p < pieces;
    copy16(dst + j * ld + p * 16, live ? src + (int64_t)(key0 + j) * s_pos + p * 16 : src, live);
  }
}
// the same, keys from `front` on up to `held` from a second place
template <int KT, int PIECES, int NT>
__device__ __forceinline__ void stage_rows(unsigned char* dst, const unsigned char* src, int64_t s_pos,
                                           int ld, int key0, int front, int pieces, int tid,
                                           const unsigned char* src2, int64_t s_pos2, int held) {
#pragma unroll 4
  for (int i = tid; i < KT * PIECES; i += NT) {
    const int key = key0 + i / PIECES, p = i % PIECES;
    const bool live = key < held && p < pieces;
    const unsigned char* at = key < front ? src + (int64_t)key * s_pos : src2 + (int64_t)key * s_pos2;
    copy16(dst + i / PIECES * ld + p * 16, live ? at + p * 16 : src, live);
  }
}

// A row's result from its maximum, its sum and its sums of V, four columns a lane, to out and lse. A row that
// saw no key has the sum 0 (any other's is positive, or NaN, which stays; maxima pass over NaN).
template <typename T>
__device__ __forceinline__ void write_row(const PaArgs& a, const PaRow& w, float m, float l, const float4& o,
                                          int lane) {
  const float inv = l == 0.f ? 0.f : 1.0f / l;
  T* out = static_cast<T*>(a.out) + (int64_t)w.n * a.o_s[0] + (int64_t)w.t * a.o_s[1] +
           (int64_t)w.h * a.o_s[2];
  if (lane * 4 < a.d) {
    const float4 y = make_float4(o.x * inv, o.y * inv, o.z * inv, o.w * inv);
    if constexpr (sizeof(T) == 4)
      *reinterpret_cast<float4*>(out + lane * 4) = y;
    else
      *reinterpret_cast<uint2*>(out + lane * 4) = make_uint2(bf16_pack2(y.x, y.y), bf16_pack2(y.z, y.w));
  }
  if (lane == 0)
    a.lse[pa_index(a, w)] = l == 0.f ? -INFINITY : fmaf(m, LN2, fmaf(m, LN2_REST, logf(l)));
}

// Join the rows' pieces, the prefix's segments and the slots, where no kernel of the own keys writes the result:
// one warp a row, the sums of four pieces on their way together.
template <typename T>
__global__ void __launch_bounds__(128, 8)
pa_combine_kernel(const PaArgs a) {
  pdl_wait();
  const size_t rows = a.rows(), row = (size_t)blockIdx.x * 4 + (threadIdx.x >> 5);
  const int lane = threadIdx.x & 31;
  if (row >= rows) return;
  PaRow w;
  w.h = (int)(row % a.Hq);
  const size_t nt = row / a.Hq;
  w.t = (int)(nt % a.T);
  w.n = (int)(nt / a.T);
  if (a.seq_len[w.n] < 0) return;                   // no such sequence: its rows stay as they are
  int segs = 0, step = PA_BLOCK;
  size_t seg0 = 0;
  if (a.seg_ctas) {
    const uint32_t hb = (uint32_t)a.Hkv * a.seg_blocks;
    const uint32_t per = pa_per_cta(a.seg_start[a.G] * hb, a.seg_ctas);
    const int g = w.n / a.W, hk = w.h / a.rep;
    const int r = ((w.n - g * a.W) * a.T + w.t) * a.rep + (w.h - hk * a.rep);
    const uint32_t before = a.seg_start[g], tiles = a.seg_start[g + 1] - before;
    if (tiles) {
      const uint32_t in = (uint32_t)hk * a.seg_blocks + r / PA_BLOCK;
      const uint32_t first = before * hb + in * tiles;
      const uint32_t c0 = first / per, c1 = (first + tiles - 1) / per;
      // in halves of a block: one a segment where the block has two row tiles, else two pieces a segment
      const bool two = a.seg_rows - r / PA_BLOCK * PA_BLOCK > 128;
      step = two ? PA_BLOCK : PA_BLOCK / 2;
      segs = ((int)(c1 - c0) + 1) * (two ? 1 : 2);
      seg0 = ((size_t)c0 + (size_t)g * hb + in) * PA_BLOCK + r % PA_BLOCK;
    }
  }
  const int all = segs + a.slots;
  float m = -INFINITY, l = 0.f;
  float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
  constexpr int U = 4;
  for (int s0 = 0; s0 < all; s0 += 32) {
    const int mine = s0 + lane;
    float2 ml = make_float2(-INFINITY, 0.f);
    if (mine < all)
      ml = mine < segs ? a.seg_ml[seg0 + (size_t)mine * step] : a.ml[(size_t)(mine - segs) * rows + row];
    const float M = fmaxf(m, warp_max(ml.x)), u = M == -INFINITY ? 0.f : M;
    const float keep = pa_ex2(m - u), f = pa_ex2(ml.x - u);
    m = M;
    l = l * keep + warp_sum(f * ml.y);
    o.x *= keep; o.y *= keep; o.z *= keep; o.w *= keep;
    const unsigned there = __ballot_sync(0xffffffffu, ml.y != 0.f);             // others wrote no sums
    const int n = min(32, all - s0);
    for (int j0 = 0; j0 < n; j0 += U) {
      float4 p[U];
#pragma unroll
      for (int v = 0; v < U; ++v) {
        const int s = s0 + j0 + v;
        p[v] = make_float4(0.f, 0.f, 0.f, 0.f);
        if (j0 + v < n && (there >> (j0 + v) & 1u) && lane * 4 < a.d)
          p[v] = *reinterpret_cast<const float4*>(
              (s < segs ? a.seg_po + (seg0 + (size_t)s * step) * a.d
                        : a.po + ((size_t)(s - segs) * rows + row) * a.d) + lane * 4);
      }
#pragma unroll
      for (int v = 0; v < U; ++v) {
        const float x = __shfl_sync(0xffffffffu, f, (j0 + v) & 31);     // (0 with p: nothing there)
        o.x = fmaf(x, p[v].x, o.x);
        o.y = fmaf(x, p[v].y, o.y);
        o.z = fmaf(x, p[v].z, o.z);
        o.w = fmaf(x, p[v].w, o.w);
      }
    }
  }
  write_row<T>(a, w, m, l, o, lane);
}

// What one CTA of the warp-level kernels has: a piece of the keys of one (group or sequence, key head) and
// a block of the rows that meet them.
struct PaPlace {
  int block, hk, b, slot;
  int own;                     // the sequence's own length as given
  int front, held, k0, k1;     // keys of the prefix in front, all keys, this piece
};
template <bool JOIN>
__device__ __forceinline__ PaPlace pa_place(const PaArgs& a, const PaKeys& kk, int blocks) {
  PaPlace p;
  int x = blockIdx.x;
  p.block = x % blocks; x /= blocks;
  p.hk = x % a.Hkv; x /= a.Hkv;
  const int sets = kk.own ? a.G * a.W : a.G;
  p.b = x % sets;
  const int split = x / sets;
  p.own = kk.len[p.b];
  p.front = JOIN && kk.front ? min(max(kk.front_len[p.b / a.W], 0), kk.front_capacity) : 0;
  p.held = p.front + min(max(p.own, 0), kk.capacity);
  pa_piece(p.held, kk.splits, split, p.k0, p.k1);
  p.slot = kk.slot0 + split;
  return p;
}
// Where the keys of a place lie: its own from key `front` on, before that the prefix's.
struct PaSource {
  const unsigned char *k, *v, *fk, *fv;
  int64_t k_s, v_s, fk_s, fv_s;                      // bytes from key to key
};
__device__ __forceinline__ PaSource pa_source(const PaArgs& a, const PaKeys& kk, const PaPlace& p, int es) {
  PaSource s;
  s.k_s = kk.k_s[1] * es;
  s.v_s = kk.v_s[1] * es;
  s.k = static_cast<const unsigned char*>(kk.k) +
        es * ((int64_t)p.b * kk.k_s[0] + (int64_t)p.hk * kk.k_s[2]) - p.front * s.k_s;
  s.v = static_cast<const unsigned char*>(kk.v) +
        es * ((int64_t)p.b * kk.v_s[0] + (int64_t)p.hk * kk.v_s[2]) - p.front * s.v_s;
  s.fk = s.k;
  s.fv = s.v;
  s.fk_s = s.fv_s = 0;
  if (p.front) {
    s.fk_s = kk.front_k_s[1] * es;
    s.fv_s = kk.front_v_s[1] * es;
    s.fk = static_cast<const unsigned char*>(kk.front_k) +
           es * ((int64_t)(p.b / a.W) * kk.front_k_s[0] + (int64_t)p.hk * kk.front_k_s[2]);
    s.fv = static_cast<const unsigned char*>(kk.front_v) +
           es * ((int64_t)(p.b / a.W) * kk.front_v_s[0] + (int64_t)p.hk * kk.front_v_s[2]);
  }
  return s;
}
// Stage keys [key, key + KT) of K at dst and of V behind it.
template <int KT, int PIECES, int NT>
__device__ __forceinline__ void stage_tile(unsigned char* dst, const PaSource& s, const PaPlace& p, int ld,
                                           int key, int pieces, int tid) {
  if (p.front) {
    stage_rows<KT, PIECES, NT>(dst, s.fk, s.fk_s, ld, key, min(p.k1, p.front), pieces, tid, s.k, s.k_s, p.k1);
    stage_rows<KT, PIECES, NT>(dst + KT * ld, s.fv, s.fv_s, ld, key, min(p.k1, p.front), pieces, tid, s.v,
                               s.v_s, p.k1);
  } else {
    stage_rows<KT, PIECES, NT>(dst, s.k, s.k_s, ld, key, p.k1, pieces, tid);
    stage_rows<KT, PIECES, NT>(dst + KT * ld, s.v, s.v_s, ld, key, p.k1, pieces, tid);
  }
}
// Rows [r0, r0 + n) of a place have no key: said in their slot.
template <int NT>
__device__ __forceinline__ void no_keys(const PaArgs& a, const PaKeys& kk, const PaPlace& p, int r0, int n,
                                        int rows, int tid) {
  for (int r = r0 + tid; r < min(rows, r0 + n); r += NT)
    a.ml[(size_t)p.slot * a.rows() + pa_index(a, pa_row(a, kk.own, p.b, p.hk, r))] =
        make_float2(-INFINITY, 0.f);
}
// Queries [r0, r0 + n) to shared memory, zeros behind the rows and the head's width.
template <int N, int PIECES, int NT>
__device__ __forceinline__ void stage_queries(unsigned char* dst, const PaArgs& a, const PaKeys& kk,
                                              const PaPlace& p, int ld, int r0, int rows, int pieces,
                                              int tid) {
  for (int i = tid; i < N * PIECES; i += NT) {
    const int r = r0 + i / PIECES, c = i % PIECES;
    const bool live = r < rows && c < pieces;
    const __nv_bfloat16* src = static_cast<const __nv_bfloat16*>(a.q);
    if (live) {
      const PaRow w = pa_row(a, kk.own, p.b, p.hk, r);
      src += (int64_t)w.n * a.q_s[0] + (int64_t)w.t * a.q_s[1] + (int64_t)w.h * a.q_s[2] + c * 8;
    }
    copy16(dst + i / PIECES * ld + c * 16, src, live);
  }
}

// bf16, up to 8 rows a (group or sequence, key head): the products turned round, keys and columns of V as
// the 16-row operand and the queries as the 8-wide one, S^T = K Q^T and O^T = V^T P^T, which halves the
// instructions and the registers of 16-row tiles that are half empty: 4 rows, 512 own keys, 64 ranges
// 10.4 us, in 16-row tiles 14.4; 512 ranges 33 both (bytes); 2,048 ranges 84 and 101. Four warps, 16 keys
// of a stage each. Short caches are waits more than work: both stages are asked for before anything is waited for,
// and three CTAs share an SM. The caller's `behind`: the launch before is of the same call and has waited
// for everything before it, so that the inputs may be read at once; it is waited for at the end.
constexpr int PF_THREADS = 128, PF_KT = 64, PF_STAGES = 2;
template <int DP>
struct PfCfg {
  static constexpr int LD = (DP + 8) * 2, STAGE = 2 * PF_KT * LD;
  static constexpr size_t SMEM = (size_t)PF_STAGES * STAGE + 8 * LD;
};
__device__ __forceinline__ uint32_t transpose8(uint32_t x) {
  uint32_t y;
  asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
  return y;
}
template <int DP, bool JOIN>
__global__ void __launch_bounds__(PF_THREADS, 3)
pa_few_kernel(const PaArgs a, const PaKeys kk, int rows) {
  if (JOIN || !kk.behind) pdl_wait();
  using Cfg = PfCfg<DP>;
  constexpr int LD = Cfg::LD, KS = DP / 16, NT = PF_THREADS;
  extern __shared__ __align__(16) unsigned char sm[];
  unsigned char* sq = sm + PF_STAGES * Cfg::STAGE;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const PaPlace p = pa_place<JOIN>(a, kk, 1);
  if (JOIN && p.own < 0) return;                     // no such sequence
  if (!JOIN && p.k0 >= p.k1) {
    if (kk.behind) pdl_wait();
    no_keys<NT>(a, kk, p, 0, rows, rows, tid);
    return;
  }
  const PaSource src = pa_source(a, kk, p, 2);
  const int pieces = a.d / 8, tiles = (p.k1 - p.k0 + PF_KT - 1) / PF_KT;
  auto stage = [&](int t) {
    if (t < tiles)
      stage_tile<PF_KT, DP / 8, NT>(sm + (t % PF_STAGES) * Cfg::STAGE, src, p, LD, p.k0 + t * PF_KT, pieces,
                                    tid);
    copy_commit();
  };
  stage_queries<8, DP / 8, NT>(sq, a, kk, p, LD, 0, rows, pieces, tid);
  copy_commit();
#pragma unroll
  for (int t = 0; t < PF_STAGES; ++t) stage(t);
  copy_wait<PF_STAGES>();
  __syncthreads();
  uint32_t qb[KS][2];
#pragma unroll
  for (int ks = 0; ks < KS; ks += 2) {
    uint32_t x[4];
    ldsm4(sm_addr(sq + (lane & 7) * LD + (ks * 16 + (lane >> 3) * 8) * 2), x);
    qb[ks][0] = x[0];
    qb[ks][1] = x[1];
    qb[ks + 1][0] = x[2];
    qb[ks + 1][1] = x[3];
  }
  // this thread's two rows, 2 c and 2 c + 1, and how many keys each may see
  const int g = lane >> 2, c = lane & 3;
  int lim[2];
#pragma unroll
  for (int e = 0; e < 2; ++e)
    lim[e] = kk.own ? min(p.k1, max(p.front, p.held - (a.T - 1 - (2 * c + e) / a.rep))) : p.k1;
  float m[2] = {-INFINITY, -INFINITY}, l[2] = {0.f, 0.f};
  float o[KS][4];
#pragma unroll
  for (int i = 0; i < KS; ++i) o[i][0] = o[i][1] = o[i][2] = o[i][3] = 0.f;

  for (int t = 0; t < tiles; ++t) {
    copy_wait<PF_STAGES - 1>();
    __syncthreads();                                 // tile t landed
    const unsigned char* sk = sm + (t % PF_STAGES) * Cfg::STAGE + warp * 16 * LD;
    const unsigned char* sv = sk + PF_KT * LD;
    const int key = p.k0 + t * PF_KT + warp * 16 + g;
    float s[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
      uint32_t ka[4];
      ldsm4(sm_addr(sk + (lane & 15) * LD + (ks * 16 + (lane >> 4) * 8) * 2), ka);
      mma_16x8x16(s, ka, qb[ks][0], qb[ks][1]);
    }
    uint32_t pb[2];
    float f[2], pr[4];
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      const float s0 = key < lim[e] ? s[e] * a.scale_log2 : -INFINITY;
      const float s1 = key + 8 < lim[e] ? s[2 + e] * a.scale_log2 : -INFINITY;
      float top = fmaxf(s0, s1);
      top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 4));
      top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 8));
      top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 16));
      const float n = fmaxf(m[e], top);
      // a row that has seen no key yet keeps maximum -inf; its terms are taken against 0
      const float u = n == -INFINITY ? 0.f : n;
      f[e] = pa_ex2(m[e] - u);
      m[e] = n;
      pr[e] = pa_ex2(s0 - u);
      pr[2 + e] = pa_ex2(s1 - u);
      l[e] = l[e] * f[e] + (pr[e] + pr[2 + e]);      // this thread's keys
    }
    pb[0] = transpose8(bf16_pack2(pr[0], pr[1]));
    pb[1] = transpose8(bf16_pack2(pr[2], pr[3]));
#pragma unroll
    for (int i = 0; i < KS; ++i) {
      o[i][0] *= f[0]; o[i][1] *= f[1];
      o[i][2] *= f[0]; o[i][3] *= f[1];
      uint32_t va[4];
      ldsm4_t(sm_addr(sv + ((lane & 7) + ((lane >> 4) << 3)) * LD + (i * 16 + ((lane >> 3) & 1) * 8) * 2), va);
      mma_16x8x16(o[i], va, pb[0], pb[1]);
    }
    __syncthreads();                                 // the tile's space is free
    stage(t + PF_STAGES);
  }
#pragma unroll
  for (int e = 0; e < 2; ++e) {
    l[e] += __shfl_xor_sync(0xffffffffu, l[e], 4);
    l[e] += __shfl_xor_sync(0xffffffffu, l[e], 8);
    l[e] += __shfl_xor_sync(0xffffffffu, l[e], 16);
  }
  // the warps' parts of the keys, a warp a row
  copy_wait<0>();
  __syncthreads();
  constexpr int XL = DP + 4;
  float* xo = reinterpret_cast<float*>(sm);          // [warp][row][XL]
  float2* xm = reinterpret_cast<float2*>(xo + 4 * 8 * XL);
  if (g == 0) {
    xm[warp * 8 + 2 * c] = make_float2(m[0], l[0]);
    xm[warp * 8 + 2 * c + 1] = make_float2(m[1], l[1]);
  }
#pragma unroll
  for (int i = 0; i < KS; ++i)
#pragma unroll
    for (int e = 0; e < 4; ++e)
      xo[(warp * 8 + 2 * c + (e & 1)) * XL + i * 16 + g + (e >> 1) * 8] = o[i][e];
  __syncthreads();
  if (!JOIN && kk.behind) pdl_wait();
#pragma unroll 1
  for (int r = warp; r < rows; r += 4) {
    float M = -INFINITY;
#pragma unroll
    for (int w = 0; w < 4; ++w) M = fmaxf(M, xm[w * 8 + r].x);
    const float u = M == -INFINITY ? 0.f : M;
    float L = 0.f;
    float4 y = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      const float2 ml = xm[w * 8 + r];
      const float x = pa_ex2(ml.x - u);
      L += x * ml.y;
      if (lane < DP / 4) {
        const float4 z = *reinterpret_cast<const float4*>(xo + (w * 8 + r) * XL + lane * 4);
        y.x = fmaf(x, z.x, y.x);
        y.y = fmaf(x, z.y, y.y);
        y.z = fmaf(x, z.z, y.z);
        y.w = fmaf(x, z.w, y.w);
      }
    }
    const PaRow w = pa_row(a, kk.own, p.b, p.hk, r);
    if constexpr (JOIN) {
      write_row<__nv_bfloat16>(a, w, M, L, y, lane);
    } else {
      const size_t at = (size_t)p.slot * a.rows() + pa_index(a, w);
      if (lane == 0) a.ml[at] = make_float2(M, L);
      if (lane * 4 < a.d) *reinterpret_cast<float4*>(a.po + at * a.d + lane * 4) = y;
    }
  }
}

// bf16: RB of the CTA's warps over 16 query rows each, the others over the keys of a stage, KW keys a warp
// (warp-level products; the pieces of the keys meet in shared memory at the end). RB follows the rows: 256
// ranges of 1,024 keys, 16 rows 29.6 us, in tiles of 32 rows 30.9, of 64 43; 32 rows 33, in tiles of 64 45.
// JOIN: the own keys in one piece, and the kernel writes the result: there is no prefix, or (`front`) its
// keys come before the own ones in the kernel's own walk, and there is no other launch.
template <int DP, int RB>
struct PmCfg {
  static constexpr int WARPS = 4, PH = WARPS / RB, KW = 64 / PH;
  static constexpr int THREADS = 32 * WARPS, KT = PH * KW;
  static constexpr int LD = (DP + 8) * 2;            // bytes of a staged row
  static constexpr int STAGE = 2 * KT * LD;
  static constexpr size_t SMEM = (size_t)PM_STAGES * STAGE;
};
template <int DP, int RB, bool JOIN>
__global__ void __launch_bounds__(32 * PmCfg<DP, RB>::WARPS, 12 / PmCfg<DP, RB>::WARPS)
pa_mma_kernel(const PaArgs a, const PaKeys kk, int rows, int blocks) {
  if (JOIN || !kk.behind) pdl_wait();
  using Cfg = PmCfg<DP, RB>;
  constexpr int LD = Cfg::LD, PH = Cfg::PH, KW = Cfg::KW, KT = Cfg::KT, NT = Cfg::THREADS;
  constexpr int KS = DP / 16, NB = KW / 8, OB = DP / 8, STAGE = Cfg::STAGE;
  extern __shared__ __align__(16) unsigned char sm[];
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int rb = warp % RB, ph = warp / RB;

  const PaPlace p = pa_place<JOIN>(a, kk, blocks);
  const int hk = p.hk, b = p.b, front = p.front, held = p.held, k0 = p.k0, k1 = p.k1, slot = p.slot;
  const int r0 = p.block * 16 * RB;
  if (JOIN && p.own < 0) return;                   // no such sequence
  if (!JOIN && k0 >= k1) {
    if (kk.behind) pdl_wait();
    no_keys<NT>(a, kk, p, r0, 16 * RB, rows, tid);
    return;
  }
  const PaSource src = pa_source(a, kk, p, 2);
  const int pieces = a.d / 8, tiles = (k1 - k0 + KT - 1) / KT;
  auto stage = [&](int t) {
    if (t < tiles)
      stage_tile<KT, DP / 8, NT>(sm + (t % PM_STAGES) * STAGE, src, p, LD, k0 + t * KT, pieces, tid);
    copy_commit();
  };
  // the queries pass through the last stage's space
  unsigned char* sq = sm + (PM_STAGES - 1) * STAGE;
  stage_queries<16 * RB, DP / 8, NT>(sq, a, kk, p, LD, r0, rows, pieces, tid);
  copy_commit();
#pragma unroll
  for (int t = 0; t < PM_STAGES - 1; ++t) stage(t);
  copy_wait<PM_STAGES - 1>();
  __syncthreads();
  uint32_t qa[KS][4];
#pragma unroll
  for (int ks = 0; ks < KS; ++ks)
    ldsm4(sm_addr(sq + (rb * 16 + (lane & 15)) * LD + (ks * 16 + (lane >> 4) * 8) * 2), qa[ks]);

  // the two query rows of this thread, and how many keys each may see
  const int g = lane >> 2, c = lane & 3;
  int lim0 = k1, lim1 = k1;
  if (kk.own) {
    const int t0 = (r0 + rb * 16 + g) / a.rep, t1 = (r0 + rb * 16 + g + 8) / a.rep;
    lim0 = min(k1, max(front, held - (a.T - 1 - t0)));
    lim1 = min(k1, max(front, held - (a.T - 1 - t1)));
  }
  float m0 = -INFINITY, m1 = -INFINITY, l0 = 0.f, l1 = 0.f;
  float o[OB][4];
#pragma unroll
  for (int i = 0; i < OB; ++i) o[i][0] = o[i][1] = o[i][2] = o[i][3] = 0.f;

  for (int t = 0; t < tiles; ++t) {
    copy_wait<PM_STAGES - 2>();
    __syncthreads();                               // tile t landed; tile t - 1's space is free
    stage(t + PM_STAGES - 1);
    const unsigned char* sk = sm + (t % PM_STAGES) * STAGE + ph * KW * LD;
    const unsigned char* sv = sk + KT * LD;
    const int key0 = k0 + t * KT + ph * KW;
    float s[NB][4];
#pragma unroll
    for (int i = 0; i < NB; ++i) s[i][0] = s[i][1] = s[i][2] = s[i][3] = 0.f;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks)
#pragma unroll
      for (int nb = 0; nb < NB; nb += 2) {
        uint32_t bf[4];
        const int key = nb * 8 + (lane & 7) + ((lane >> 4) << 3);
        ldsm4(sm_addr(sk + key * LD + (ks * 16 + ((lane >> 3) & 1) * 8) * 2), bf);
        mma_16x8x16(s[nb], qa[ks], bf[0], bf[1]);
        mma_16x8x16(s[nb + 1], qa[ks], bf[2], bf[3]);
      }
    float b0 = -INFINITY, b1 = -INFINITY;
#pragma unroll
    for (int nb = 0; nb < NB; ++nb)
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const int key = key0 + nb * 8 + 2 * c + e;
        s[nb][e] = key < lim0 ? s[nb][e] * a.scale_log2 : -INFINITY;
        s[nb][2 + e] = key < lim1 ? s[nb][2 + e] * a.scale_log2 : -INFINITY;
        b0 = fmaxf(b0, s[nb][e]);
        b1 = fmaxf(b1, s[nb][2 + e]);
      }
    b0 = fmaxf(b0, __shfl_xor_sync(0xffffffffu, b0, 1));
    b0 = fmaxf(b0, __shfl_xor_sync(0xffffffffu, b0, 2));
    b1 = fmaxf(b1, __shfl_xor_sync(0xffffffffu, b1, 1));
    b1 = fmaxf(b1, __shfl_xor_sync(0xffffffffu, b1, 2));
    const float n0 = fmaxf(m0, b0), n1 = fmaxf(m1, b1);
    // a row that has seen no key yet keeps maximum -inf; its terms are taken against 0
    const float u0 = n0 == -INFINITY ? 0.f : n0, u1 = n1 == -INFINITY ? 0.f : n1;
    const float c0 = pa_ex2(m0 - u0), c1 = pa_ex2(m1 - u1);
    m0 = n0;
    m1 = n1;
    l0 *= c0;
    l1 *= c1;
#pragma unroll
    for (int i = 0; i < OB; ++i) {
      o[i][0] *= c0; o[i][1] *= c0;
      o[i][2] *= c1; o[i][3] *= c1;
    }
    uint32_t pa[NB / 2][4];
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) {
      const float p0 = pa_ex2(s[nb][0] - u0), p1 = pa_ex2(s[nb][1] - u0);
      const float p2 = pa_ex2(s[nb][2] - u1), p3 = pa_ex2(s[nb][3] - u1);
      l0 += p0 + p1;
      l1 += p2 + p3;
      pa[nb >> 1][(nb & 1) * 2] = bf16_pack2(p0, p1);
      pa[nb >> 1][(nb & 1) * 2 + 1] = bf16_pack2(p2, p3);
    }
#pragma unroll
    for (int ks = 0; ks < NB / 2; ++ks)
#pragma unroll
      for (int ob = 0; ob < OB; ob += 2) {
        uint32_t vf[4];
        const int key = ks * 16 + (lane & 7) + ((lane >> 3) & 1) * 8;
        ldsm4_t(sm_addr(sv + key * LD + (ob * 8 + (lane >> 4) * 8) * 2), vf);
        mma_16x8x16(o[ob], pa[ks], vf[0], vf[1]);
        mma_16x8x16(o[ob + 1], pa[ks], vf[2], vf[3]);
      }
  }
  l0 += __shfl_xor_sync(0xffffffffu, l0, 1);
  l0 += __shfl_xor_sync(0xffffffffu, l0, 2);
  l1 += __shfl_xor_sync(0xffffffffu, l1, 1);
  l1 += __shfl_xor_sync(0xffffffffu, l1, 2);

  // join the key phases of each row: phase ph > 0 leaves its state in shared memory
  if constexpr (PH > 1) {
    copy_wait<0>();
    __syncthreads();
    float* xo = reinterpret_cast<float*>(sm);
    constexpr int XL = DP + 4;
    float* xm = xo + (size_t)(PH - 1) * RB * 16 * XL;
    if (ph > 0) {
      const int row = ((ph - 1) * RB + rb) * 16 + g;
      if (c == 0) {
        xm[2 * row] = m0; xm[2 * row + 1] = l0;
        xm[2 * (row + 8)] = m1; xm[2 * (row + 8) + 1] = l1;
      }
#pragma unroll
      for (int i = 0; i < OB; ++i) {
        *reinterpret_cast<float2*>(xo + (size_t)row * XL + i * 8 + 2 * c) = make_float2(o[i][0], o[i][1]);
        *reinterpret_cast<float2*>(xo + (size_t)(row + 8) * XL + i * 8 + 2 * c) =
            make_float2(o[i][2], o[i][3]);
      }
    }
    __syncthreads();
    if (!JOIN && ph > 0) {
      if (kk.behind) pdl_wait();
      return;
    }
#pragma unroll
    for (int p = 0; p < PH - 1; ++p) {
      if (ph > 0) break;
      const int row = (p * RB + rb) * 16 + g;
      const float pm0 = xm[2 * row], pl0 = xm[2 * row + 1];
      const float pm1 = xm[2 * (row + 8)], pl1 = xm[2 * (row + 8) + 1];
      const float n0 = fmaxf(m0, pm0), n1 = fmaxf(m1, pm1);
      const float u0 = n0 == -INFINITY ? 0.f : n0, u1 = n1 == -INFINITY ? 0.f : n1;
      const float c0 = pa_ex2(m0 - u0), c1 = pa_ex2(m1 - u1);
      const float e0 = pa_ex2(pm0 - u0), e1 = pa_ex2(pm1 - u1);
      m0 = n0; m1 = n1;
      l0 = l0 * c0 + pl0 * e0;
      l1 = l1 * c1 + pl1 * e1;
#pragma unroll
      for (int i = 0; i < OB; ++i) {
        const float2 q0 = *reinterpret_cast<const float2*>(xo + (size_t)row * XL + i * 8 + 2 * c);
        const float2 q1 = *reinterpret_cast<const float2*>(xo + (size_t)(row + 8) * XL + i * 8 + 2 * c);
        o[i][0] = o[i][0] * c0 + q0.x * e0;
        o[i][1] = o[i][1] * c0 + q0.y * e0;
        o[i][2] = o[i][2] * c1 + q1.x * e1;
        o[i][3] = o[i][3] * c1 + q1.y * e1;
      }
    }
  }
  if constexpr (JOIN) {
    // the rows as they are to shared memory, then a warp a row
    if constexpr (PH == 1) copy_wait<0>();
    __syncthreads();
    float* xr = reinterpret_cast<float*>(sm);
    constexpr int XL = DP + 4;
    float* xm = xr + (size_t)RB * 16 * XL;
    if (ph == 0) {
      const int row = rb * 16 + g;
      if (c == 0) {
        xm[2 * row] = m0; xm[2 * row + 1] = l0;
        xm[2 * (row + 8)] = m1; xm[2 * (row + 8) + 1] = l1;
      }
#pragma unroll
      for (int i = 0; i < OB; ++i) {
        *reinterpret_cast<float2*>(xr + (size_t)row * XL + i * 8 + 2 * c) = make_float2(o[i][0], o[i][1]);
        *reinterpret_cast<float2*>(xr + (size_t)(row + 8) * XL + i * 8 + 2 * c) =
            make_float2(o[i][2], o[i][3]);
      }
    }
    __syncthreads();
    const int here = min(16 * RB, rows - r0);
    constexpr int R = 4;                             // rows of a warp at a time: their divisions side by side
    for (int r = warp * R; r < here; r += R * Cfg::WARPS)
#pragma unroll
      for (int y = r; y < r + R; ++y)
        if (y < here)
          write_row<__nv_bfloat16>(a, pa_row(a, kk.own, b, hk, r0 + y), xm[2 * y], xm[2 * y + 1],
                                   lane < DP / 4 ? *reinterpret_cast<const float4*>(xr + (size_t)y * XL + lane * 4)
                                                 : make_float4(0.f, 0.f, 0.f, 0.f), lane);
    return;
  }
  if (kk.behind) pdl_wait();
  const int ra = r0 + rb * 16 + g;
#pragma unroll
  for (int half = 0; half < 2; ++half) {
    const int r = ra + half * 8;
    if (r >= rows) continue;
    const size_t at = (size_t)slot * a.rows() + pa_index(a, pa_row(a, kk.own, b, hk, r));
    if (c == 0) a.ml[at] = half ? make_float2(m1, l1) : make_float2(m0, l0);
#pragma unroll
    for (int i = 0; i < OB; ++i)
      if (i * 8 < a.d)
        *reinterpret_cast<float2*>(a.po + at * a.d + i * 8 + 2 * c) =
            half ? make_float2(o[i][2], o[i][3]) : make_float2(o[i][0], o[i][1]);
  }
}

// fp32 on the CUDA cores: each of four warps owns four query rows, a lane a key of the stage's 32 for
// the scores and four columns of V for the sums.
constexpr int PS_THREADS = 128;
constexpr int PS_ROWS = 16;
constexpr int PS_KT = 32;
constexpr int PS_STAGES = 2;

template <int DP>
__global__ void __launch_bounds__(PS_THREADS)
pa_simt_kernel(const PaArgs a, const PaKeys kk, int rows, int blocks) {
  if (!kk.behind) pdl_wait();
  constexpr int LD = (DP + 4) * 4;
  constexpr int STAGE = 2 * PS_KT * LD;
  extern __shared__ __align__(16) unsigned char sm[];
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const PaPlace p = pa_place<false>(a, kk, blocks);
  const int hk = p.hk, b = p.b, held = p.held, k0 = p.k0, k1 = p.k1, slot = p.slot;
  const int r0 = p.block * PS_ROWS;
  if (k0 >= k1) {
    if (kk.behind) pdl_wait();
    no_keys<PS_THREADS>(a, kk, p, r0, PS_ROWS, rows, tid);
    return;
  }
  const PaSource from = pa_source(a, kk, p, 4);
  const int pieces = a.d / 4, tiles = (k1 - k0 + PS_KT - 1) / PS_KT;
  float* sq = reinterpret_cast<float*>(sm + PS_STAGES * STAGE);          // [16][DP]
  auto stage = [&](int t) {
    if (t < tiles)
      stage_tile<PS_KT, DP / 4, PS_THREADS>(sm + (t % PS_STAGES) * STAGE, from, p, LD, k0 + t * PS_KT,
                                            pieces, tid);
    copy_commit();
  };
  for (int i = tid; i < PS_ROWS * (DP / 4); i += PS_THREADS) {
    const int r = r0 + i / (DP / 4), c = i % (DP / 4);
    const bool live = r < rows && c < pieces;
    const float* src = static_cast<const float*>(a.q);
    if (live) {
      const PaRow w = pa_row(a, kk.own, b, hk, r);
      src += (int64_t)w.n * a.q_s[0] + (int64_t)w.t * a.q_s[1] + (int64_t)w.h * a.q_s[2] + c * 4;
    }
    copy16(sq + i * 4, src, live);
  }
  stage(0);
  const int rw = r0 + warp * 4;                   // this warp's first row
  int lim[4];
  float m[4], l[4];
  float4 o[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    lim[i] = kk.own ? min(k1, held - (a.T - 1 - (rw + i) / a.rep)) : k1;
    m[i] = -INFINITY;
    l[i] = 0.f;
    o[i] = make_float4(0.f, 0.f, 0.f, 0.f);
  }
  for (int t = 0; t < tiles; ++t) {
    copy_wait<0>();
    __syncthreads();
    stage(t + 1);
    if (rw >= rows) continue;
    const unsigned char* sk = sm + (t % PS_STAGES) * STAGE;
    const unsigned char* sv = sk + PS_KT * LD;
    const int key = k0 + t * PS_KT + lane;
    float s[4] = {0.f, 0.f, 0.f, 0.f}, odd[4] = {0.f, 0.f, 0.f, 0.f};      // two shorter chains of roundings
#pragma unroll 4
    for (int c = 0; c < DP / 4; c += 2) {
      const float4 kv = *reinterpret_cast<const float4*>(sk + lane * LD + c * 16);
      const float4 kw = *reinterpret_cast<const float4*>(sk + lane * LD + c * 16 + 16);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float* q = sq + (warp * 4 + i) * DP + c * 4;
        s[i] = dot4(*reinterpret_cast<const float4*>(q), kv, s[i]);
        odd[i] = dot4(*reinterpret_cast<const float4*>(q + 4), kw, odd[i]);
      }
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      s[i] += odd[i];
      // (the product with the scale is exact beside u, and what the scale's own rounding left is added to that
      // small difference, where it counts: scores of 20 would leave 1e-6 of a term otherwise)
      const bool seen = key < lim[i];
      const float n = fmaxf(m[i], warp_max(seen ? s[i] * a.scale_log2 : -INFINITY));
      const float u = n == -INFINITY ? 0.f : n;
      const float f = pa_ex2(m[i] - u);
      m[i] = n;
      s[i] = seen ? pa_ex2(fmaf(s[i], a.scale_rest, fmaf(s[i], a.scale_log2, -u))) : 0.f;
      l[i] = l[i] * f + s[i];                     // this lane's share of the sum
      o[i].x *= f; o[i].y *= f; o[i].z *= f; o[i].w *= f;
    }
#pragma unroll 8
    for (int j = 0; j < PS_KT; ++j) {
      const float4 v = *reinterpret_cast<const float4*>(sv + j * LD + (lane % (DP / 4)) * 16);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float x = __shfl_sync(0xffffffffu, s[i], j);
        o[i].x = fmaf(x, v.x, o[i].x);
        o[i].y = fmaf(x, v.y, o[i].y);
        o[i].z = fmaf(x, v.z, o[i].z);
        o[i].w = fmaf(x, v.w, o[i].w);
      }
    }
  }
  if (kk.behind) pdl_wait();
  if (rw >= rows) return;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float sum = warp_sum(l[i]);
    if (rw + i >= rows) continue;
    const size_t at = (size_t)slot * a.rows() + pa_index(a, pa_row(a, kk.own, b, hk, rw + i));
    if (lane == 0) a.ml[at] = make_float2(m[i], sum);
    if (lane < DP / 4 && lane * 4 < a.d) *reinterpret_cast<float4*>(a.po + at * a.d + lane * 4) = o[i];
  }
}

int key_sets(const PaArgs& a, const PaKeys& k) { return k.own ? a.G * a.W : a.G; }
int key_rows(const PaArgs& a, const PaKeys& k) { return (k.own ? 1 : a.W) * a.T * a.rep; }

template <int DP, int RB, bool JOIN>
lilicorr_status_t launch_mma(const PaArgs& a, const PaKeys& k, cudaStream_t st) {
  static bool configured[64] = {false};
  auto* kernel = pa_mma_kernel<DP, RB, JOIN>;
  LL_TRY(allow_max_dynamic_smem(kernel, configured));
  const int rows = key_rows(a, k), blocks = ceil_div(rows, 16 * RB);
  const size_t grid = (size_t)key_sets(a, k) * a.Hkv * blocks * k.splits;
  if (grid > 0x7FFFFFFFull) return LILICORR_ERR_SHAPE;
  return launch_k(kernel, (unsigned)grid, PmCfg<DP, RB>::THREADS, PmCfg<DP, RB>::SMEM, st, a, k, rows,
                  blocks);
}

template <int DP, bool JOIN>
lilicorr_status_t launch_mma_rows(const PaArgs& a, const PaKeys& k, cudaStream_t st) {
  const int rows = key_rows(a, k);
  if (rows <= 8) {
    static bool configured[64] = {false};
    auto* kernel = pa_few_kernel<DP, JOIN>;
    LL_TRY(allow_max_dynamic_smem(kernel, configured));
    const size_t grid = (size_t)key_sets(a, k) * a.Hkv * k.splits;
    if (grid > 0x7FFFFFFFull) return LILICORR_ERR_SHAPE;
    return launch_k(kernel, (unsigned)grid, PF_THREADS, PfCfg<DP>::SMEM, st, a, k, rows);
  }
  if (rows <= 16) return launch_mma<DP, 1, JOIN>(a, k, st);
  if (rows <= 32) return launch_mma<DP, 2, JOIN>(a, k, st);
  return launch_mma<DP, 4, JOIN>(a, k, st);
}

template <int DP>
lilicorr_status_t launch_simt(const PaArgs& a, const PaKeys& k, cudaStream_t st) {
  static bool configured[64] = {false};
  LL_TRY(allow_max_dynamic_smem(pa_simt_kernel<DP>, configured));
  const int rows = key_rows(a, k), blocks = ceil_div(rows, PS_ROWS);
  const size_t smem = (size_t)PS_STAGES * 2 * PS_KT * (DP + 4) * 4 + PS_ROWS * DP * 4;
  const size_t grid = (size_t)key_sets(a, k) * a.Hkv * blocks * k.splits;
  if (grid > 0x7FFFFFFFull) return LILICORR_ERR_SHAPE;
  return launch_k(pa_simt_kernel<DP>, (unsigned)grid, PS_THREADS, smem, st, a, k, rows, blocks);
}

}  // namespace

lilicorr_status_t launch_pa_mma(const PaArgs& a, const PaKeys& k, cudaStream_t st) {
  if (k.join) return a.d <= 64 ? launch_mma_rows<64, true>(a, k, st) : launch_mma_rows<128, true>(a, k, st);
  return a.d <= 64 ? launch_mma_rows<64, false>(a, k, st) : launch_mma_rows<128, false>(a, k, st);
}

lilicorr_status_t launch_pa_simt(const PaArgs& a, const PaKeys& k, cudaStream_t st) {
  return a.d <= 64 ? launch_simt<64>(a, k, st) : launch_simt<128>(a, k, st);
}

lilicorr_status_t launch_pa_combine(const PaArgs& a, lilicorr_dtype_t dt, cudaStream_t st) {
  const size_t grid = (a.rows() + 3) / 4;
  if (dt == LILICORR_BF16) return launch_k(pa_combine_kernel<__nv_bfloat16>, (unsigned)grid, 128, 0, st, a);
  return launch_k(pa_combine_kernel<float>, (unsigned)grid, 128, 0, st, a);
}

// ---------------------------------------------------------------------------- the call
namespace {

int g_pa_path = 0;             // test hook: 1 the tensor-core kernel for every bf16 prefix, 2 for none

struct PaPlan {
  bool front, tc;              // how the prefix is taken: by the own keys' kernel, by the tensor-core kernel
  int psplits, ssplits;        // psplits 0: the prefix's pieces are segments
  int seg_ctas, seg_blocks;
  size_t rows, ml_off, po_off, start_off, seg_ml_off, seg_po_off, total;
};

bool stride_ok(const int64_t (&s)[3], const int (&extent)[3], int per16) {
  for (int i = 0; i < 3; ++i)
    if (extent[i] > 1 && (s[i] < 0 || s[i] % per16 || s[i] > (1ll << 40))) return false;
  return true;
}

bool pa_plan(const lilicorr_prefix_attention_desc* d, PaPlan* p) {
  if (!d || (d->dtype != LILICORR_F32 && d->dtype != LILICORR_BF16)) return false;
  if (d->groups < 0 || d->beams < 1 || d->tokens < 1 || d->q_heads < 1 || d->kv_heads < 1) return false;
  if (d->q_heads % d->kv_heads || d->head_dim < 8 || d->head_dim > 128 || d->head_dim % 8) return false;
  if (d->prefix_capacity < 0 || d->own_capacity < 0) return false;
  if (d->prefix_capacity > (1 << 30) || d->own_capacity > (1 << 30)) return false;
  const double rows = (double)d->groups * d->beams * d->tokens * d->q_heads;
  if (rows >= 2147483648.0 || (double)d->groups * d->beams * d->kv_heads >= 2147483648.0) return false;
  const int sms = num_sms();
  const int rep = d->q_heads / d->kv_heads;
  const bool f32 = d->dtype == LILICORR_F32;
  const long long prow = (long long)d->beams * d->tokens * rep, orow = (long long)d->tokens * rep;
  const long long pranges = (long long)d->groups * d->kv_heads, oranges = pranges * d->beams;
  const long long octas = oranges * ((orow + 63) / 64);    // the own keys' CTAs in one piece
  const bool whole = octas >= sms, half = 2 * octas >= sms;

  // Pieces of a key range, of which a kernel takes per_block rows: one and a half CTAs an SM over all
  // ranges, no piece below 128 keys. More pieces cost more in the join than they save: 128 ranges of 768
  // keys, 16 rows, 24.6 us, at three CTAs an SM 28.6; 128 of 4,096 own keys 49 and 61. Pieces of 256 keys
  // at least: 8 ranges of 768 keys, 64 rows, 15.2 -> 18.5 us; 8 of 8,192 the same.
  // fp32: three CTAs an SM, 64 keys, which a stage of 32 on the CUDA cores takes as long for as a bf16 tile
  // of 128: 32 sequences behind 4,096 keys 44 us, at one and a half 52; 15 behind 1,777 keys 24.7, at 256
  // keys 36.
  const int least = f32 ? 64 : 128, per_block = f32 ? 16 : 64;
  const long long wave = f32 ? 3ll * sms : 3ll * sms / 2;
  auto pieces = [&](long long ranges, long long rows, int cap) {
    ranges *= (rows + per_block - 1) / per_block;
    const long long want = ranges > 0 ? (wave + ranges - 1) / ranges : 1;
    const long long most = (cap + least - 1) / least;
    long long n = want < most ? want : most;
    return (int)(n < 1 ? 1 : n > 128 ? 128 : n);
  };

  // A short prefix that few sequences share is read again by each of them, in the walk over their own keys,
  // which then writes the result: one launch for three. Own keys of 64, 32 CTAs: a prefix of 64 keys 6.9 us,
  // beside it 11; of 512 12.4 and 12.3. 512 CTAs: 64 keys 12.4 and 16, 256 20 and 18, 512 27 and 21; with
  // four tokens 256 keys 24.7 and 27.5. 4,096 CTAs: 64 keys 50 and 55, 128 63 and 57. CTAs that leave
  // most SMs idle walk at most 512 keys: 8 CTAs, 384 keys 10.3 and 10.4, 576 12.4 and 11.0.
  p->front = !f32 && g_pa_path == 0 && d->prefix_capacity && d->own_capacity && d->prefix_capacity <= 512 &&
             octas * d->prefix_capacity <= 1024ll * sms &&
             (whole || (long long)d->prefix_capacity + d->own_capacity <= (half ? 768 : 512));

  // The tensor-core kernel pays 6-8 us for its start and its segments' sums, so that small products are
  // faster on mma.sync, in pieces: 8 ranges, 4 rows, 2,048 keys 18.5 us and 12.4 there; 32 ranges, 32 rows,
  // 2,048 keys 24.7 and 22; at 4,096 keys 30.9 and 27; 64 rows 36.3 and 37; 128 rows 44.5 and 62; 256 rows
  // 60 and 106. At d = 64, 32 ranges, 4,096 keys, 64 rows 26.8 and 24; at 8,192 34.4 and 32; 128 rows 31 and
  // 38. Each range costs it 4 us or more besides: 2,048 ranges of 256 keys, 4 rows 106 us and 70; 256 of 256,
  // 64 rows 62 and 56; 512 of 2,048, 16 rows 119 and 114; 512 of 1,024, 64 rows 142 and 157; 256 of 256, 256
  // rows 181 and 197. And at d = 64 up to 16 rows never fill it: 512 ranges of 2,048 keys 91 and 68.
  // (Heads of 72 to 120 are computed as 128 wide by either, and counted so.)
  const long long blocks = (prow + PA_BLOCK - 1) / PA_BLOCK;
  const double tiles = (double)pranges * blocks * ((double)d->prefix_capacity / PA_TILE + 1);
  const double item = (double)d->prefix_capacity / PA_TILE * (prow < 16 ? 16 : prow) *
                      (d->head_dim <= 64 ? 64 : 128);
  p->tc = !f32 && d->prefix_capacity && !p->front &&
          (g_pa_path ? g_pa_path == 1
                     : pranges * item > 4.0 * 1048576.0 && item > 32768.0 && (prow > 16 || d->head_dim > 64));
  if (p->tc && tiles >= 2147483648.0) return false;      // (they are counted in 32 bits)
  p->seg_ctas = p->tc ? sms : 0;
  p->seg_blocks = p->tc ? (int)blocks : 0;
  p->psplits = d->prefix_capacity ? pieces(pranges, prow, d->prefix_capacity) : 0;
  // bf16 own keys: one piece where that is a wave of CTAs (behind a prefix, 256 ranges of 512 keys 26.6 us,
  // in pieces 28.9; 128 ranges 24.9 and 20.5), or where, alone, they need no join then (32 ranges of 256 keys
  // 8.3 us, in pieces 9.0; of 512 11.0 and 8.9; 128 ranges of 512 12.3 and 13.2).
  p->ssplits = !d->own_capacity ? 0
               : p->front || (!f32 && (whole || (!d->prefix_capacity && d->own_capacity <= (half ? 512 : 256))))
                   ? 1 : pieces(oranges, orow, d->own_capacity);
  p->rows = (size_t)rows;
  const size_t slots = (size_t)p->psplits + p->ssplits;
  const size_t segs = p->tc ? (size_t)sms + (size_t)pranges * blocks : 0;
  p->ml_off = 256;
  p->po_off = p->ml_off + align_up(slots * p->rows * sizeof(float2), 256);
  p->start_off = p->po_off + align_up(slots * p->rows * d->head_dim * sizeof(float), 256);
  p->seg_ml_off = p->start_off + align_up(((size_t)d->groups + 1) * sizeof(uint32_t), 256);
  p->seg_po_off = p->seg_ml_off + align_up(segs * PA_BLOCK * sizeof(float2), 256);
  p->total = p->seg_po_off + align_up(segs * PA_BLOCK * d->head_dim * sizeof(float), 256);
  return true;
}

lilicorr_status_t run_prefix_attention(const lilicorr_prefix_attention_desc* desc, const void* q,
                                       const void* prefix_k, const void* prefix_v,
                                       const int32_t* prefix_len, const void* k, const void* v,
                                       const int32_t* seq_len, void* out, float* lse, void* ws,
                                       size_t ws_bytes, cudaStream_t stream, long long wait_limit,
                                       int starve) {
  if (!desc) return LILICORR_ERR_ARG;
  if (desc->dtype != LILICORR_F32 && desc->dtype != LILICORR_BF16) return LILICORR_ERR_DTYPE;
  PaPlan p;
  if (!pa_plan(desc, &p)) return LILICORR_ERR_SHAPE;
  if (!(desc->scale > 0.f) || !(desc->scale < 0x1p127f)) return LILICORR_ERR_ARG;      // (times log2(e): finite)
  if (desc->groups == 0) return LILICORR_OK;
  const bool has_p = desc->prefix_capacity > 0, has_s = desc->own_capacity > 0;
  if (!q || !out || !lse || !ws || !seq_len) return LILICORR_ERR_ARG;
  if (has_p && (!prefix_k || !prefix_v || !prefix_len)) return LILICORR_ERR_ARG;
  if (has_s && (!k || !v)) return LILICORR_ERR_ARG;
  if (!aligned16(q) || !aligned16(out) || !aligned16(ws)) return LILICORR_ERR_ARG;
  if (has_p && (!aligned16(prefix_k) || !aligned16(prefix_v))) return LILICORR_ERR_ARG;
  if (has_s && (!aligned16(k) || !aligned16(v))) return LILICORR_ERR_ARG;
  const int N = desc->groups * desc->beams, per16 = desc->dtype == LILICORR_BF16 ? 8 : 4;
  const int rows_e[3] = {N, desc->tokens, desc->q_heads};
  const int pre_e[3] = {desc->groups, desc->prefix_capacity, desc->kv_heads};
  const int own_e[3] = {N, desc->own_capacity, desc->kv_heads};
  if (!stride_ok(desc->q_stride, rows_e, per16) || !stride_ok(desc->out_stride, rows_e, per16) ||
      (has_p && (!stride_ok(desc->prefix_k_stride, pre_e, per16) ||
                 !stride_ok(desc->prefix_v_stride, pre_e, per16))) ||
      (has_s && (!stride_ok(desc->k_stride, own_e, per16) || !stride_ok(desc->v_stride, own_e, per16))))
    return LILICORR_ERR_ARG;
  const int64_t out_e[3] = {N, desc->tokens, desc->q_heads};
  if (!StrideNest(desc->out_stride, out_e, 3, desc->head_dim).nests()) return LILICORR_ERR_ARG;
  if (ws_bytes < p.total) return LILICORR_ERR_WORKSPACE;

  unsigned char* w = static_cast<unsigned char*>(ws);
  PaArgs a;
  memset(&a, 0, sizeof(a));
  a.q = q;
  a.out = out;
  a.lse = lse;
  a.seq_len = seq_len;
  a.G = desc->groups; a.W = desc->beams; a.T = desc->tokens;
  a.Hq = desc->q_heads; a.Hkv = desc->kv_heads; a.rep = desc->q_heads / desc->kv_heads;
  a.d = desc->head_dim;
  const double scale = (double)desc->scale * 1.4426950408889634;       // log2(e)
  a.scale_log2 = (float)scale;
  a.scale_rest = (float)(scale - a.scale_log2);
  a.seg_ctas = p.seg_ctas;
  a.seg_blocks = p.seg_blocks;
  a.seg_rows = a.W * a.T * a.rep;
  a.seg_start = reinterpret_cast<uint32_t*>(w + p.start_off);
  a.seg_ml = reinterpret_cast<float2*>(w + p.seg_ml_off);
  a.seg_po = reinterpret_cast<float*>(w + p.seg_po_off);
  a.status = reinterpret_cast<uint32_t*>(w);
  a.wait_limit = wait_limit;
  a.test_starve = starve;
  a.ml = reinterpret_cast<float2*>(w + p.ml_off);
  a.po = reinterpret_cast<float*>(w + p.po_off);
  PaKeys pre, own;
  memset(&pre, 0, sizeof(pre));
  memset(&own, 0, sizeof(own));
  for (int i = 0; i < 3; ++i) {                    // a dimension of one has no stride to speak of
    a.q_s[i] = rows_e[i] > 1 ? desc->q_stride[i] : 0;
    a.o_s[i] = rows_e[i] > 1 ? desc->out_stride[i] : 0;
    pre.k_s[i] = pre_e[i] > 1 ? desc->prefix_k_stride[i] : 0;
    pre.v_s[i] = pre_e[i] > 1 ? desc->prefix_v_stride[i] : 0;
    own.k_s[i] = own_e[i] > 1 ? desc->k_stride[i] : 0;
    own.v_s[i] = own_e[i] > 1 ? desc->v_stride[i] : 0;
  }
  pre.k = prefix_k; pre.v = prefix_v; pre.len = prefix_len;
  pre.capacity = desc->prefix_capacity; pre.splits = p.psplits; pre.slot0 = 0; pre.own = 0;
  own.k = k; own.v = v; own.len = seq_len;
  own.capacity = desc->own_capacity; own.splits = p.ssplits; own.own = 1;
  const bool bf = desc->dtype == LILICORR_BF16;
  // no prefix, or one that the own keys' kernel walks through first: one launch
  own.join = bf && own.splits == 1 && (!has_p || p.front);
  a.slots = 0;
  if (starve && (!has_p || own.join || !bf)) return LILICORR_ERR_SHAPE;
  if (p.front) {
    own.front = 1;
    own.front_k = pre.k;
    own.front_v = pre.v;
    for (int i = 0; i < 3; ++i) { own.front_k_s[i] = pre.k_s[i]; own.front_v_s[i] = pre.v_s[i]; }
    own.front_len = pre.len;
    own.front_capacity = pre.capacity;
    return launch_pa_mma(a, own, stream);
  }
  PaMaps maps;
  const bool tc = p.tc && pa_tc_maps(a, pre, &maps);
  if (starve && !tc) return LILICORR_ERR_SHAPE;
  if (!tc) a.seg_ctas = 0;
  else pre.splits = 0;
  own.slot0 = pre.splits;
  a.slots = own.join ? 0 : pre.splits + own.splits;
  own.behind = has_p;
  if (tc) LL_TRY(launch_pa_tc(a, pre, maps, stream));
  else if (has_p) LL_TRY(bf ? launch_pa_mma(a, pre, stream) : launch_pa_simt(a, pre, stream));
  if (has_s) LL_TRY(bf ? launch_pa_mma(a, own, stream) : launch_pa_simt(a, own, stream));
  return own.join ? LILICORR_OK : launch_pa_combine(a, desc->dtype, stream);
}

}  // namespace
}  // namespace lilicorr

using namespace lilicorr;

extern "C" {

size_t lilicorr_prefix_attention_workspace_bytes(const lilicorr_prefix_attention_desc* desc) {
  PaPlan p;
  return pa_plan(desc, &p) ? p.total : 0;
}

lilicorr_status_t lilicorr_prefix_attention(const lilicorr_prefix_attention_desc* desc, const void* q,
                                            const void* prefix_k, const void* prefix_v,
                                            const int32_t* prefix_len, const void* k, const void* v,
                                            const int32_t* seq_len, void* out, float* lse, void* ws,
                                            size_t ws_bytes, cudaStream_t stream) {
  return run_prefix_attention(desc, q, prefix_k, prefix_v, prefix_len, k, v, seq_len, out, lse, ws,
                              ws_bytes, stream, PA_WAIT, 0);
}

int lilicorr_test_prefix_path(int mode) {
  const int prev = g_pa_path;
  g_pa_path = mode < 0 ? 0 : mode > 2 ? 2 : mode;
  return prev;
}

lilicorr_status_t lilicorr_test_prefix_attention_timeout(
    const lilicorr_prefix_attention_desc* desc, const void* q, const void* prefix_k,
    const void* prefix_v, const int32_t* prefix_len, const void* k, const void* v,
    const int32_t* seq_len, void* out, float* lse, void* ws, size_t ws_bytes, long long wait_cycles,
    int which, cudaStream_t stream) {
  if (wait_cycles < 100000 || wait_cycles > PA_WAIT || which < 1 || which > 2) return LILICORR_ERR_ARG;
  return run_prefix_attention(desc, q, prefix_k, prefix_v, prefix_len, k, v, seq_len, out, lse, ws,
                              ws_bytes, stream, wait_cycles, which);
}

}  // extern "C"
