// Attention over a cache held in 4 bits: what each key gets from more rows than scores are kept for, bf16 queries.
//
// Scores are computed once more, on the 5th-generation tensor cores with the product turned round:
//   S^T = K Q^T   (M 128 keys, N up to 128 rows)
// so that a thread has a key, and its weight is a sum along the thread's own columns, in their order:
//   weight += sum over rows of 2^(factor s - reference) / sum,
// the rows' references and sums being those of the attention before. One CTA an SM: two warps copy the keys' half of the
// records, two times four warps expand them in turn, a thread a key, one issues, and two streams of four warps take
// pairs of tiles in turn, so that what a thread reads of a row serves two keys. More than 128 rows come one block
// after the other, with the keys again.
//
// What bounds it: for few rows the way of a tile through copies, expansion and product, for more the rows' figures that
// the streams read from shared memory (12 bytes a row and warp), beside the products that read there. 8 sequences of
// 16,384, 8 heads of 128: 64 rows 46.5 us behind an attention of 82, with a tile a stream at a time 55; 32 rows 41.5
// (on mma.sync, 32 rows at a time, 129 and 82).
#include "cache_attention_tc.cuh"

namespace lilicorr {
namespace {

constexpr uint32_t CW_TMEM = 512;
constexpr int CW_RAW = 4;                            // tiles of keys under way
constexpr int CW_SOFT = 256, CW_MMA_WARP = 8, CW_COPY_WARP = 9, CW_FIRST = 11, CW_THREADS = 32 * 19;

template <int DP>
struct CwCfg {
  static constexpr int CH = DP / 64;
  static constexpr uint32_t TILE = CH * CT_CHUNK, RAW = CT_KEYS * (DP / 2 + 16);
  static constexpr size_t SMEM = 1024 + 3 * TILE + CW_RAW * RAW;
};

template <int DP, int DIM>
__global__ void __launch_bounds__(CW_THREADS, 1) cache_attention_tc_weights_kernel(const CaArgs a) {
  using Cfg = CwCfg<DP>;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* sQ = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) &
                                           ~static_cast<uintptr_t>(1023));
  uint8_t* sK = sQ + Cfg::TILE;
  uint8_t* sR = sK + 2 * Cfg::TILE;
  __shared__ __align__(8) uint64_t k_full[2], k_empty[2], r_full[CW_RAW], r_empty[CW_RAW], s_ready[2], s_free[2], drain;
  __shared__ uint32_t tmem_base;
  __shared__ volatile int abort_flag;
  // a row's factor, what its reference adds, 1 / sum (0: it adds nothing), keys that it sees
  __shared__ __align__(16) float s_factor[CT_ROWS], s_add[CT_ROWS], s_inv[CT_ROWS];
  __shared__ int s_seen[CT_ROWS];

  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int d = DIM ? DIM : a.c.d, R = (cache_half_bytes(d) + 15) / 16 * 16, rows = a.T * a.rep;
  if (tid == 0) {
    for (int i = 0; i < 2; ++i) {
      mbar_init(&k_full[i], 4);
      mbar_init(&k_empty[i], 1);
      mbar_init(&s_ready[i], 1);
      mbar_init(&s_free[i], 4);
    }
    for (int i = 0; i < CW_RAW; ++i) { mbar_init(&r_full[i], 64); mbar_init(&r_empty[i], 4); }
    mbar_init(&drain, 1);
    abort_flag = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == CW_MMA_WARP) tmem_alloc(&tmem_base, CW_TMEM);
  pdl_wait();
  CaCursor<CT_KEYS> at = {};
  uint32_t first = 0, per = 1;
  const uint32_t count = ca_range<CT_KEYS>(a, 1, &at, &first, &per);
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = tmem_base;
  auto wait = [&](uint64_t* bar, uint32_t parity) {  // for a whole warp: all lanes go on, or none
    if (__all_sync(0xffffffffu, mbar_try_wait(bar, parity))) return true;
    return __all_sync(0xffffffffu, wait_long(bar, parity, a.wait_limit, &abort_flag)) != 0;
  };
  uint32_t done = 0;                                 // tiles of the list behind this warp
  uint32_t g = 0, pairs = 0;                         // tiles so far, whose place is g % 2; pairs of them: their stream
  // f(tile0, tiles, r0) for each block of rows of each item's tiles here
  auto walk = [&](auto f) {
    while (done < count) {
      const int here = min((uint32_t)(at.tiles - at.tile), count - done);
      for (int r0 = 0; r0 < rows; r0 += CT_ROWS) {
        f(at.tile, here, r0);
        g += here;
        pairs += (here + 1) / 2;
      }
      done += here;
      if (done < count) at.next(a, 1);
    }
  };

  if (warp >= CW_COPY_WARP && warp < CW_FIRST) {
    const int x = tid - 32 * CW_COPY_WARP, vecs = R / 16;
    const int step = 64 / vecs, rest = 64 - step * vecs, first_k = x / vecs, first_v = x - first_k * vecs;
    const int64_t stride = a.c.s[1];
    bool ok = true;
    walk([&](int tile0, int here, int) {
      const unsigned char* src = a.c.at(at.n, tile0 * CT_KEYS, at.h);
      for (int t = 0; t < here && ok; ++t) {
        const uint32_t i = g + t, into = i % CW_RAW;
        if (!wait(&r_empty[into], (i / CW_RAW & 1u) ^ 1u)) { ok = false; break; }
        const int there = min(CT_KEYS, at.len - (tile0 + t) * CT_KEYS);
        int k = first_k, v = first_v;
        const unsigned char* from = src + first_k * stride + first_v * 16;
        uint32_t to = smem_u32(sR + into * Cfg::RAW) + x * 16;
#pragma unroll 5
        for (int u = 0; u < vecs * 2; ++u) {
          if (k < there) copy16(to, from, true);
          to += 64 * 16;
          k += step;
          v += rest;
          from += step * stride + rest * 16;
          if (v >= vecs) {
            v -= vecs;
            ++k;
            from += stride - vecs * 16;
          }
        }
        asm volatile("cp.async.mbarrier.arrive.noinc.shared::cta.b64 [%0];" ::"r"(smem_u32(&r_full[into]))
                     : "memory");
        src += CT_KEYS * stride;
      }
    });
    copy_commit();
    copy_wait<0>();
  } else if (warp >= CW_FIRST) {
    const int x = tid - 32 * CW_FIRST, key = x & 127;
    const uint32_t mine = x >> 7;                    // of each two tiles
    bool ok = a.test_starve != 3;
    walk([&](int tile0, int here, int) {
      for (int t = (g ^ mine) & 1u; t < here && ok; t += 2) {
        const uint32_t i = g + t, raw = i % CW_RAW;
        ok = wait(&r_full[raw], i / CW_RAW & 1u) && wait(&k_empty[mine], (i >> 1 & 1u) ^ 1u);
        if (!ok) break;
        expand<DP, DIM>(smem_u32(sR) + raw * Cfg::RAW + key * R, (tile0 + t) * CT_KEYS + key < at.len, d,
                        smem_u32(sK) + mine * Cfg::TILE, key);
        fence_async_shared();
        __syncwarp();
        if (lane == 0) {
          mbar_arrive(&k_full[mine]);
          mbar_arrive(&r_empty[raw]);
        }
      }
    });
  } else if (warp == CW_MMA_WARP) {
    const bool leader = elect_one();
    const uint64_t q_desc = smem_desc(sQ), k_desc = smem_desc(sK);
    bool ok = true;
    walk([&](int, int here, int r0) {
      const uint32_t idesc = instr_desc_f16(128, min(CT_ROWS, (rows - r0 + 31) / 32 * 32));
      named_bar(1, CW_SOFT + 32);                    // Q is there
      tc_fence_after();
      for (int t = 0; t < here && ok; ++t) {
        const uint32_t i = g + t, k = i & 1u, pair = pairs + t / 2, s = pair & 1u;
        ok = wait(&k_full[k], i >> 1 & 1u) && (t & 1 || wait(&s_free[s], (pair >> 1 & 1u) ^ 1u));
        if (!ok) break;
        tc_fence_after();
        const uint64_t kd = k_desc + k * (Cfg::TILE >> 4);
        if (leader) {
#pragma unroll
          for (int c = 0; c < Cfg::CH; ++c)
#pragma unroll
            for (int j = 0; j < 4; ++j)
              mma_bf16(tmem + s * 256 + (t & 1) * 128, kd + c * (CT_CHUNK >> 4) + 2 * j,
                       q_desc + c * (CT_CHUNK >> 4) + 2 * j, idesc, (c | j) > 0);
          mma_commit(&k_empty[k]);
          if (t & 1 || t + 1 == here) mma_commit(&s_ready[s]);
        }
        __syncwarp();
      }
    });
    if (abort_flag) {                                // products under way, before their memory goes
      if (leader) mma_commit(&drain);
      mbar_wait(&drain, 0, a.wait_limit);
      __syncwarp();
    }
  } else {
    const uint32_t s = warp >> 2;
    const int key = (warp & 3) * 32 + lane;
    const uint32_t scores = tmem + s * 256 + ((uint32_t)((warp & 3) * 32) << 16);
    bool ok = true;
    walk([&](int tile0, int here, int r0) {
      // the block's queries and its rows' figures, a row two threads
      {
        const int row = tid & 127, r = r0 + row, tok = r / a.rep, hq = at.h * a.rep + (r - tok * a.rep);
        float2 ml = make_float2(0.f, 0.f);
        if (r < rows) ml = a.rows[((size_t)at.n * a.T + tok) * a.Hq + hq];
        // rows without keys, or without a finite sum, add nothing
        const bool there = ml.y > 0.f && ml.y < INFINITY && fabsf(ml.x) < INFINITY;
        const __nv_bfloat16* q = static_cast<const __nv_bfloat16*>(a.q) + at.n * a.q_s[0] + tok * a.q_s[1] +
                                 hq * a.q_s[2];
        auto piece = [&](int p) {
          return there && p * 8 < d ? __ldg(reinterpret_cast<const uint4*>(q + p * 8)) : make_uint4(0, 0, 0, 0);
        };
        float top = 0.f;
#pragma unroll 4
        for (int p = 0; p < DP / 8; ++p) {
          const uint4 v = piece(p);
          const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
          for (int i = 0; i < 4; ++i)
            top = fmaxf(top, fmaxf(fabsf(__uint_as_float(w[i] << 16)), fabsf(__uint_as_float(w[i] & 0xFFFF0000u))));
        }
        const int up = query_shift(top);
        const float by = pow2(up);
#pragma unroll 4
        for (int i = 0; i < DP / 16; ++i) {          // (again, from the cache)
          const int p = (tid >> 7) * (DP / 16) + i;
          const uint4 v = piece(p);
          uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
          for (int j = 0; j < 4; ++j)
            w[j] = half2_of(__uint_as_float(w[j] << 16) * by, __uint_as_float(w[j] & 0xFFFF0000u) * by);
          sts16(smem_u32(sQ) + (p >> 3) * CT_CHUNK + swz(row, p & 7), w[0], w[1], w[2], w[3]);
        }
        if (tid < CT_ROWS) {
          s_factor[row] = there ? row_factor(a, up) : 0.f;
          s_add[row] = there ? CA_UP - ml.x : 0.f;
          s_inv[row] = there ? 1.f / ml.y : 0.f;
          s_seen[row] = there ? max(0, at.seen(a, tok)) : 0;
        }
        fence_async_shared();
      }
      named_bar(1, CW_SOFT + 32);
      const int cols = min(CT_ROWS, rows - r0);
      // a row that adds nothing may be one that has met a key that is not finite
      bool all = true;
      for (int r = lane; r < cols; r += 32) all &= s_inv[r] > 0.f;
      all = __all_sync(0xffffffffu, all);
      for (int t = 2 * ((pairs ^ s) & 1u); t < here && ok; t += 4) {
        const uint32_t pair = pairs + t / 2;
        const int k = (tile0 + t) * CT_KEYS + key;   // and the key 128 behind it
        float* to = a.weights + ((size_t)at.n * a.c.H + at.h) * a.c.S + k;
        float w[2] = {0.f, 0.f};
#pragma unroll
        for (int u = 0; u < 2; ++u)
          if (t + u < here && k + u * CT_KEYS < at.len) w[u] = to[u * CT_KEYS];
        if (!wait(&s_ready[s], pair >> 1 & 1u)) { ok = false; break; }
        tc_fence_after();
        // some row does not see all of them, or may not take their products
        const bool masked = !all || (tile0 + t + 2) * CT_KEYS > at.len - (a.T - 1);
        uint64_t sum[2] = {0ull, 0ull};
        auto add = [&](auto some) {                  // (some: not all of them)
#pragma unroll 1
          for (int c = 0; c < cols; c += 16) {
            uint32_t x[2][16];
            tmem_ld16_nowait(scores + c, x[0]);
            tmem_ld16(scores + 128 + c, x[1]);       // (without a second tile: what lies there, for nobody)
#pragma unroll
            for (int e = 0; e < 16; e += 8)          // nothing that uses the first moves above the second's wait
              asm volatile("" : "+r"(x[0][e]), "+r"(x[0][e + 1]), "+r"(x[0][e + 2]), "+r"(x[0][e + 3]),
                                "+r"(x[0][e + 4]), "+r"(x[0][e + 5]), "+r"(x[0][e + 6]), "+r"(x[0][e + 7]));
#pragma unroll
            for (int e = 0; e < 16; e += 4) {        // (columns past the last: queries of 0, 1 / sum of 0)
              const float4 f = *reinterpret_cast<const float4*>(s_factor + c + e);
              const float4 b = *reinterpret_cast<const float4*>(s_add + c + e);
              const float4 y = *reinterpret_cast<const float4*>(s_inv + c + e);
#pragma unroll
              for (int u = 0; u < 2; ++u) {
                float p[4];
                halves(fma_pair(pair_of(__uint_as_float(x[u][e]), __uint_as_float(x[u][e + 1])), pair_of(f.x, f.y),
                                pair_of(b.x, b.y)), p[0], p[1]);
                halves(fma_pair(pair_of(__uint_as_float(x[u][e + 2]), __uint_as_float(x[u][e + 3])),
                                pair_of(f.z, f.w), pair_of(b.z, b.w)), p[2], p[3]);
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                  p[i] = ex2(p[i]);
                  if (decltype(some)::value && k + u * CT_KEYS >= s_seen[c + e + i]) p[i] = 0.f;
                }
                sum[u] = fma_pair(pair_of(p[0], p[1]), pair_of(y.x, y.y), sum[u]);
                sum[u] = fma_pair(pair_of(p[2], p[3]), pair_of(y.z, y.w), sum[u]);
              }
            }
          }
        };
        if (masked) add(std::true_type{});
        else add(std::false_type{});
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(&s_free[s]);
#pragma unroll
        for (int u = 0; u < 2; ++u) {
          float even, odd;
          halves(sum[u], even, odd);
          if (t + u < here && k + u * CT_KEYS < at.len) to[u * CT_KEYS] = w[u] + (even + odd);
        }
      }
      named_bar(3, CW_SOFT);                         // every product with these queries is done
    });
  }
  tc_fence_before();
  __syncthreads();
  if (abort_flag && tid == 0) set_status(a.status, LILICORR_ERR_TIMEOUT);
  if (warp == CW_MMA_WARP) {
    tc_fence_after();
    tmem_dealloc(tmem, CW_TMEM);
  }
}

template <int DP, int DIM>
lilicorr_status_t launch(const CaArgs& a, const CaPlan& p, cudaStream_t st) {
  static bool configured[64] = {false};
  auto* kernel = cache_attention_tc_weights_kernel<DP, DIM>;
  LL_TRY(allow_max_dynamic_smem(kernel, configured));
  return launch_k(kernel, (unsigned)(num_sms() / p.team * p.team), CW_THREADS, CwCfg<DP>::SMEM, st, a);
}

}  // namespace

lilicorr_status_t launch_ca_tc_weights(const CaArgs& a, const CaPlan& p, cudaStream_t st) {
  if (a.c.d == 128) return launch<128, 128>(a, p, st);
  if (a.c.d == 64) return launch<64, 64>(a, p, st);
  return a.c.d < 64 ? launch<64, 0>(a, p, st) : launch<128, 0>(a, p, st);
}

}  // namespace lilicorr
