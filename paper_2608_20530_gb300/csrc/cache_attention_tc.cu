// Attention over a cache held in 4 bits on the 5th-generation tensor cores: bf16 queries of more rows than one
// matrix instruction has columns (drafted blocks under verification, wide groups of heads), 128 rows at a time
// against tiles of 128 keys.
//
// One CTA an SM. Two warps copy records to shared memory; eight expand them, a thread half a record, to fp16 (exact:
// six significant bits) in the swizzled layout that the tensor cores read, four of them keys, four values. One warp
// issues
//   S = Q K^T   (M 128, N 128)   into tensor memory, and
//   O += P V    (M 128, N d)     with P read from tensor memory, V as the MN-major operand.
// The first warps are two streams, a thread a row, that take the key tiles in turn: while one is at its
// exponentials the tensor cores work for the other. Queries are brought to fp16 by a power of two of their row,
// as on mma.sync (cache_attention_kernels.cuh). Each stream has its own references and sums, whole numbers
// m that move only when a score passes them by 8; at an item's end the two come together.
//
// What bounds it: 8 sequences of 4,096 to 16,384 positions, 8 heads of 128, 64 rows: 63.5 us. A tile more costs an SM
// 0.97 us, some 1,850 clocks: 1,060 of the tensor pipe (its operands are 96 KB of shared memory), 1,900 of a stream's
// two passes over its scores (128 exponentials a thread are 1,024 of them) and the way from one to the other, for
// two tiles at a time. None of them alone: half of the matrix work, half of the stores of expanded records, no
// copies, or no exponentials leave 95, 94, 95 and 94 % of the time. 26 us are start, first tile, a change of item, parts and
// their join (14 where every CTA has one item). Tried: a thread half of a row's scores of a tile (its softmax in half
// the time, 63 us for 64), a warp that issues for each stream (65), both (67), half tiles of 64 keys (73).
#include "cache_attention_tc.cuh"

namespace lilicorr {
namespace {

constexpr uint32_t CT_TMEM = 512;
constexpr int CT_RAW = 3;                            // tiles of records under way

// HALF: blocks of 64 rows or fewer. Q lies in the tile twice, so that scores of all rows lie in tensor memory twice,
// and each stream has the half whose quarters its warps can read: warps 0 and 1, 2 and 3, a scheduler each, and
// more registers a thread (both streams on the first two quarters: 79 us for 63).
template <int DP, bool HALF>
struct CtCfg {
  static constexpr int QUARTERS = HALF ? 2 : 4, SOFT = 2 * 32 * QUARTERS;      // warps of a stream; threads of both
  static constexpr int MMA_WARP = SOFT / 32, COPY_WARP = MMA_WARP + 1, FIRST = MMA_WARP + 2;   // FIRST to expand
  static constexpr int WARPS = FIRST + 9, THREADS = 32 * WARPS;    // (the last one copies, too)
  static constexpr int CH = DP / 64;                 // 64-column chunks of a row
  static constexpr uint32_t TILE = CH * CT_CHUNK;
  static constexpr int NK = 2, NV = 2;
  static constexpr uint32_t RAW = CT_KEYS * (DP + 16);
  static constexpr size_t SMEM = 1024 + (1 + NK + NV) * TILE + CT_RAW * RAW;
  // tensor-memory columns: scores, output, and the probabilities of keys [16 k, 16 k + 16), at d = 128 over
  // the scores, which their thread has read: the next scores of the stream are issued behind the product that
  // reads them
  __device__ static constexpr uint32_t S(int s) { return s * 128; }
  __device__ static constexpr uint32_t O(int s) { return 256 + s * DP; }
  __device__ static constexpr uint32_t P(int s, int k) { return (DP == 128 ? S(s) : 384 + s * 64) + k * 8; }
};

// A of the product from tensor memory
__device__ __forceinline__ void mma_ta(uint32_t tmem_d, uint32_t tmem_a, uint64_t b, uint32_t idesc,
                                       uint32_t accumulate) {
  asm volatile(
      "{\n .reg .pred p;\n setp.ne.b32 p, %4, 0;\n"
      " tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n}" ::"r"(tmem_d),
      "r"(tmem_a), "l"(b), "r"(idesc), "r"(accumulate));
}
// MN-major operand of 128-byte-swizzled rows: 64-column chunks CT_CHUNK bytes apart, 8-row groups 1024
__device__ __forceinline__ uint64_t smem_desc_mn(const void* tile) {
  return smem_desc(tile) & ~(0x3FFFull << 16) | ((uint64_t)(CT_CHUNK >> 4) << 16);
}
__device__ __forceinline__ uint64_t add_pairs(uint64_t a, uint64_t b) {
  uint64_t d;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
  return d;
}
// Nothing that uses these registers moves above this point (a load from tensor memory fills them until its wait).
__device__ __forceinline__ void pin(uint32_t (&r)[32]) {
#pragma unroll
  for (int i = 0; i < 32; i += 8)
    asm volatile("" : "+r"(r[i]), "+r"(r[i + 1]), "+r"(r[i + 2]), "+r"(r[i + 3]), "+r"(r[i + 4]),
                      "+r"(r[i + 5]), "+r"(r[i + 6]), "+r"(r[i + 7]));
}
// 2^d of a whole number d <= 0 (0 below the normal range, and for -inf)
__device__ __forceinline__ float pow2_down(float d) {
  return d < -126.f ? 0.f : __int_as_float((127 + (int)d) << 23);
}
template <int DP, int DIM, bool HALF>
__global__ void __launch_bounds__((CtCfg<DP, HALF>::THREADS), 1) cache_attention_tc_kernel(const CaArgs a) {
  using Cfg = CtCfg<DP, HALF>;
  using E = __nv_bfloat16;
  constexpr int NK = Cfg::NK, NV = Cfg::NV;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* sQ = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) &
                                           ~static_cast<uintptr_t>(1023));
  uint8_t* sK = sQ + Cfg::TILE;
  uint8_t* sV = sK + NK * Cfg::TILE;
  uint8_t* sR = sV + NV * Cfg::TILE;
  __shared__ __align__(8) uint64_t k_full[NK], k_empty[NK], v_full[NV], v_empty[NV];
  __shared__ __align__(8) uint64_t r_full[CT_RAW], r_empty[CT_RAW], s_ready[2], p_ready[2], o_ready[2], drain;
  __shared__ uint32_t tmem_base;
  __shared__ volatile int abort_flag;
  __shared__ float s_factor[CT_ROWS];
  __shared__ float2 s_ml[2][CT_ROWS];

  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int d = DIM ? DIM : a.c.d, R = cache_record_bytes(d), rows = a.T * a.rep;
  if (tid == 0) {
    for (int i = 0; i < NK; ++i) { mbar_init(&k_full[i], 4); mbar_init(&k_empty[i], 1); }
    for (int i = 0; i < NV; ++i) { mbar_init(&v_full[i], 4); mbar_init(&v_empty[i], 1); }
    for (int i = 0; i < CT_RAW; ++i) { mbar_init(&r_full[i], 64); mbar_init(&r_empty[i], 8); }
    for (int i = 0; i < 2; ++i) {
      mbar_init(&s_ready[i], 1);
      mbar_init(&p_ready[i], Cfg::QUARTERS);
      mbar_init(&o_ready[i], 1);
    }
    mbar_init(&drain, 1);
    abort_flag = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == Cfg::MMA_WARP) tmem_alloc(&tmem_base, CT_TMEM);
  pdl_wait();
  CaCursor<CT_KEYS> at = {};
  uint32_t first = 0, per = 1;
  const uint32_t count = ca_range<CT_KEYS>(a, a.blocks, &at, &first, &per);
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = tmem_base;
  auto wait = [&](uint64_t* bar, uint32_t parity) {  // for a whole warp: all lanes go on, or none
    if (__all_sync(0xffffffffu, mbar_try_wait(bar, parity))) return true;
    return __all_sync(0xffffffffu, wait_long(bar, parity, a.wait_limit, &abort_flag)) != 0;
  };
  uint32_t done = 0;                                 // tiles of the list behind this warp

  if (warp == Cfg::COPY_WARP || warp == Cfg::WARPS - 1) {
    // ---- records: CT_RAW tiles ahead, 16 bytes a lane (one bulk copy a record takes 58 clocks each)
    const int x = lane + (warp == Cfg::COPY_WARP ? 0 : 32), vecs = R / 16;
    const int step = 64 / vecs, rest = 64 - step * vecs, first_k = x / vecs, first_v = x - first_k * vecs;
    const int64_t stride = a.c.s[1];
    uint32_t into = 0, parity = 1;
    bool ok = true;
    while (done < count && ok) {
      const int tile1 = min((uint32_t)at.tiles, at.tile + (count - done));
      const unsigned char* src = a.c.at(at.n, at.tile * CT_KEYS, at.h);
      done += tile1 - at.tile;
      for (; at.tile < tile1 && ok; ++at.tile) {
        if (!wait(&r_empty[into], parity)) { ok = false; break; }
        const int there = min(CT_KEYS, at.len - at.tile * CT_KEYS);
        int k = first_k, v = first_v;
        const unsigned char* from = src + first_k * stride + first_v * 16;
        uint32_t to = smem_u32(sR + into * Cfg::RAW) + x * 16;
#pragma unroll 6
        for (int i = 0; i < vecs * 2; ++i) {
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
        if (++into == CT_RAW) { into = 0; parity ^= 1u; }
      }
      if (done < count && ok) at.next(a, a.blocks);
    }
    copy_commit();
    copy_wait<0>();
  } else if (warp >= Cfg::FIRST) {
    // ---- records expanded, when their tile and its new place are there: four warps keys, four values
    const int x = tid - 32 * Cfg::FIRST, key = x & 127, is_v = x >> 7;
    uint64_t* full = is_v ? v_full : k_full;
    uint64_t* empty = is_v ? v_empty : k_empty;
    const uint32_t ring = smem_u32(is_v ? sV : sK);
    const uint32_t source = smem_u32(sR) + key * R + is_v * cache_half_bytes(d);
    uint32_t slot = 0, parity = 1, raw = 0, raw_parity = 0;
    bool ok = a.test_starve != is_v + 1;
    while (done < count && ok) {
      const int tile1 = min((uint32_t)at.tiles, at.tile + (count - done));
      done += tile1 - at.tile;
      for (; at.tile < tile1 && ok; ++at.tile) {
        ok = wait(&r_full[raw], raw_parity) && wait(&empty[slot], parity);
        if (!ok) break;
        expand<DP, DIM>(source + raw * Cfg::RAW, at.tile * CT_KEYS + key < at.len, d, ring + slot * Cfg::TILE, key);
        fence_async_shared();
        __syncwarp();
        if (lane == 0) {
          mbar_arrive(&full[slot]);
          mbar_arrive(&r_empty[raw]);
        }
        if (++raw == CT_RAW) { raw = 0; raw_parity ^= 1u; }
        if (++slot == (is_v ? NV : NK)) { slot = 0; parity ^= 1u; }
      }
      if (done < count && ok) at.next(a, a.blocks);
    }
  } else if (warp == Cfg::MMA_WARP) {
    // ---- products. The whole warp walks, one lane issues.
    constexpr uint32_t idesc_s = instr_desc_f16(128, 128);
    constexpr uint32_t idesc_o = instr_desc_f16(128, DP) | (1u << 16);      // V MN-major
    const bool leader = elect_one();
    const uint64_t q_desc = smem_desc(sQ), k_desc = smem_desc(sK), v_desc = smem_desc_mn(sV);
    uint32_t ki = 0, kp = 0, vi = 0, vp = 0;         // the rings' next slots and their parities
    uint32_t pp[2] = {0, 0};                         // parity of the streams' probabilities
    while (done < count) {
      const uint32_t here = min((uint32_t)(at.tiles - at.tile), count - done);
      const int end = at.len - at.tile * CT_KEYS;    // keys from here on
      named_bar(1, Cfg::SOFT + 32);                  // Q is there
      tc_fence_after();
      bool ok = true;
      auto scores = [&](int s) {
        if (!wait(&k_full[ki], kp)) { ok = false; return; }
        tc_fence_after();
        const uint64_t kd = k_desc + ki * (Cfg::TILE >> 4);
        if (leader) {
#pragma unroll
          for (int c = 0; c < Cfg::CH; ++c)
#pragma unroll
            for (int k = 0; k < 4; ++k)
              mma_bf16(tmem + Cfg::S(s), q_desc + c * (CT_CHUNK >> 4) + 2 * k, kd + c * (CT_CHUNK >> 4) + 2 * k,
                       idesc_s, (c | k) > 0);
          mma_commit(&s_ready[s]);
          mma_commit(&k_empty[ki]);
        }
        __syncwarp();
        if (++ki == NK) { ki = 0; kp ^= 1u; }
      };
      auto sums = [&](int s, int keys, bool fresh, bool last) {
        if (!wait(&p_ready[s], pp[s])) { ok = false; return; }
        pp[s] ^= 1u;
        if (!wait(&v_full[vi], vp)) { ok = false; return; }
        tc_fence_after();
        const uint64_t vd = v_desc + vi * (Cfg::TILE >> 4);
        if (leader) {
          const int ks = keys >= CT_KEYS ? CT_KEYS / 16 : max(1, (keys + 15) / 16);
          if (ks == CT_KEYS / 16) {
#pragma unroll
            for (int k = 0; k < CT_KEYS / 16; ++k)
              mma_ta(tmem + Cfg::O(s), tmem + Cfg::P(s, k), vd + k * 128, idesc_o, !fresh || k > 0);
          } else {
#pragma unroll 1
            for (int k = 0; k < ks; ++k)
              mma_ta(tmem + Cfg::O(s), tmem + Cfg::P(s, k), vd + k * 128, idesc_o, !fresh || k > 0);
          }
          mma_commit(&v_empty[vi]);
          if (last) mma_commit(&o_ready[s]);
        }
        __syncwarp();
        if (++vi == NV) { vi = 0; vp ^= 1u; }
      };
      scores(0);
      if (ok && here > 1) scores(1);
      for (uint32_t t = 0; t < here && ok; ++t) {
        const int s = (int)(t & 1u);
        sums(s, end - (int)t * CT_KEYS, t < 2, t + 2 >= here);
        if (ok && t + 2 < here) scores(s);
      }
      named_bar(2, Cfg::SOFT + 32);                  // the item is done with
      done += here;
      if (done < count) at.next(a, a.blocks);
    }
    if (abort_flag) {                                // products under way, before their memory goes
      if (leader) mma_commit(&drain);
      mbar_wait(&drain, 0, a.wait_limit);
      __syncwarp();
    }
  } else {
    // ---- the streams: a thread a row
    const int s = warp / Cfg::QUARTERS, row = warp % Cfg::QUARTERS * 32 + lane;
    const uint32_t lane_base = tmem + ((uint32_t)((warp & 3) * 32) << 16);
    uint32_t sn = 0, on = 0;                         // scores and outputs met so far
    while (done < count) {
      const int tile0 = at.tile, tile1 = min((uint32_t)at.tiles, tile0 + (count - done));
      const uint32_t here = tile1 - tile0;
      const int tile_rows = min(CT_ROWS, rows - at.rb * CT_ROWS);
      const int r = at.rb * CT_ROWS + row, tok = r / a.rep, hq = at.h * a.rep + (r - tok * a.rep);
      const bool mine = row < tile_rows;
      // the block's queries, a row a thread: the first stream's, or with HALF either's of its own
      if (HALF || s == 0) {
        const E* q = static_cast<const E*>(a.q) + at.n * a.q_s[0] + tok * a.q_s[1] + hq * a.q_s[2];
        auto piece = [&](int p) {
          return mine && p * 8 < d ? __ldg(reinterpret_cast<const uint4*>(q + p * 8)) : make_uint4(0, 0, 0, 0);
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
        for (int p = 0; p < DP / 8; ++p) {           // (again, from the cache)
          const uint4 v = piece(p);
          uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
          for (int i = 0; i < 4; ++i)
            w[i] = half2_of(__uint_as_float(w[i] << 16) * by, __uint_as_float(w[i] & 0xFFFF0000u) * by);
          sts16(smem_u32(sQ) + (p >> 3) * CT_CHUNK + swz(HALF ? s * 64 + row : row, p & 7), w[0], w[1], w[2], w[3]);
        }
        const float factor = row_factor(a, up);
        if (s == 0) s_factor[row] = factor;
        fence_async_shared();
        if (a.scores && s == 0 && mine) a.factors[((size_t)at.n * a.T + tok) * a.Hq + hq] = factor;
      }
      named_bar(1, Cfg::SOFT + 32);
      const float f = s_factor[row];
      const bool idle = warp % Cfg::QUARTERS * 32 >= tile_rows;
      const int lim = mine ? at.seen(a, tok) : 0;      // keys that the row sees
      float m = -INFINITY, l = 0.f;
      bool ok = true;
      for (uint32_t t = s; t < here; t += 2) {
        if (!wait(&s_ready[s], sn & 1u)) { ok = false; break; }
        ++sn;
        if (idle) {                                  // (what P holds for its rows reaches no other row)
          if (lane == 0) mbar_arrive(&p_ready[s]);
          continue;
        }
        tc_fence_after();
        const int k0 = (tile0 + (int)t) * CT_KEYS, seen = lim - k0;
        const bool masked = k0 + CT_KEYS > at.len - (a.T - 1);   // some row does not see all of them
        if (masked) {                                // scores of keys that the row does not see: -infinity
#pragma unroll 1
          for (int c = 0; c < 4; ++c) {
            uint32_t x[32];
            tmem_ld32(lane_base + Cfg::S(s) + 32 * c, x);
#pragma unroll
            for (int e = 0; e < 32; ++e)
              if (32 * c + e >= seen) x[e] = 0xFF800000u;
            tmem_st32(lane_base + Cfg::S(s) + 32 * c, x);
          }
          tmem_wait_st();
        }
        // 32 scores at a time; HALF: the next ones are read while these are worked on
        uint32_t xs[HALF ? 2 : 1][32];
        auto scores = [&](int c) -> uint32_t (&)[32] {
          if (HALF) {
            if (c == 0) tmem_ld32_nowait(lane_base + Cfg::S(s), xs[0]);
            tmem_wait_ld();
            pin(xs[HALF ? c & 1 : 0]);
            if (c < 3) tmem_ld32_nowait(lane_base + Cfg::S(s) + 32 * (c + 1), xs[HALF ? (c + 1) & 1 : 0]);
          } else {
            tmem_ld32(lane_base + Cfg::S(s) + 32 * c, xs[0]);
          }
          return xs[HALF ? c & 1 : 0];
        };
        float mx[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
        for (int c = 0; c < 4; ++c) {
          uint32_t (&x)[32] = scores(c);
          if (a.scores && mine) {                    // for what each key gets: 32 rows of a key side by side
            float* to = a.scores + (((size_t)at.n * a.c.H + at.h) * a.c.S + k0 + 32 * c) * a.pad + r;
#pragma unroll
            for (int e = 0; e < 32; ++e)
              if (k0 + 32 * c + e < at.len) to[(size_t)e * a.pad] = __uint_as_float(x[e]);
          }
#pragma unroll
          for (int e = 0; e < 32; e += 8)
#pragma unroll
            for (int i = 0; i < 4; ++i)
              mx[i] = fmaxf(fmaxf(mx[i], __uint_as_float(x[e + i])), __uint_as_float(x[e + 4 + i]));
        }
        const float top = fmaxf(fmaxf(mx[0], mx[1]), fmaxf(mx[2], mx[3])) * f;
        if (t == (uint32_t)s) {
          m = ceilf(top);
        } else if (__any_sync(0xffffffffu, top > m + CA_SLACK)) {
          // the sums so far to the new reference, by a whole power of two (their product is complete: the
          // scores came behind it)
          const float to = fmaxf(m, ceilf(top)), y = pow2_down(m - to);
          m = to;
          l *= y;
#pragma unroll 1
          for (int i = 0; i < DP / 16; ++i) {
            uint32_t o[16];
            tmem_ld16(lane_base + Cfg::O(s) + 16 * i, o);
#pragma unroll
            for (int e = 0; e < 16; ++e) o[e] = __float_as_uint(__uint_as_float(o[e]) * y);
            tmem_st16(lane_base + Cfg::O(s) + 16 * i, o);
          }
        }
        // once more, for the probabilities: no branch in this pass, so that one's exponentials run beside
        // another's reads and writes
        const uint64_t f2 = pair_of(f, f);
        const float base = CA_UP - (m == -INFINITY ? 0.f : m);
        const uint64_t base2 = pair_of(base, base);
        uint64_t sum[2] = {0ull, 0ull};
#pragma unroll
        for (int c = 0; c < 4; ++c) {
          uint32_t (&x)[32] = scores(c);
          uint32_t p[16];
#pragma unroll
          for (int e = 0; e < 16; ++e) {
            float p0, p1;
            halves(fma_pair(pair_of(__uint_as_float(x[2 * e]), __uint_as_float(x[2 * e + 1])), f2, base2), p0, p1);
            p0 = ex2(p0);
            p1 = ex2(p1);
            sum[e & 1] = add_pairs(sum[e & 1], pair_of(p0, p1));
            p[e] = half2_of(p0, p1);
          }
          tmem_st16(lane_base + Cfg::P(s, 2 * c), p);
        }
        float l0, l1;
        halves(add_pairs(sum[0], sum[1]), l0, l1);
        l += l0 + l1;
        tmem_wait_st();
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(&p_ready[s]);
      }
      if (ok && (uint32_t)s < here) {
        if (!wait(&o_ready[s], on & 1u)) ok = false;
        ++on;
        tc_fence_after();
      }
      done += here;
      // ---- the two streams' sums come together: with HALF the second's come over by the queries' space (every
      // product with them is done), else each stream takes half of the columns of both
      s_ml[s][row] = make_float2(m, l);
      named_bar(3, Cfg::SOFT);
      const float2 z0 = s_ml[0][row], z1 = s_ml[1][row];
      const float M = fmaxf(fmaxf(z0.x, z1.x), -FLT_MAX);
      const float f0 = ex2(z0.x - M), f1 = here > 1 ? ex2(z1.x - M) : 0.f, L = z0.y * f0 + z1.y * f1;
      const bool complete = tile0 == 0 && tile1 == at.tiles;
      const uint32_t s0 = first + done - tile1;
      const int head = blockIdx.x % a.team;
      auto part = [&](uint32_t team) { return 2 * ((size_t)team * a.team + head) + (team * per < s0); };
      const size_t place = part(blockIdx.x / a.team) * CT_ROWS + row;
      const float by = L == 0.f ? 0.f : a.c.v_unit / L;
      auto leave = [&](int c, const float (&y)[16]) {            // 16 columns of the row
        if (!mine || c * 16 >= d) return;
        if (complete) {
          E* out = static_cast<E*>(a.out) + at.n * a.o_s[0] + tok * a.o_s[1] + hq * a.o_s[2] + c * 16;
#pragma unroll
          for (int e = 0; e < 16; e += 8)
            if (L == 0.f)
              *reinterpret_cast<uint4*>(out + e) = make_uint4(0, 0, 0, 0);
            else
              *reinterpret_cast<uint4*>(out + e) =
                  make_uint4(bf16_pack2(y[e] * by, y[e + 1] * by), bf16_pack2(y[e + 2] * by, y[e + 3] * by),
                             bf16_pack2(y[e + 4] * by, y[e + 5] * by), bf16_pack2(y[e + 6] * by, y[e + 7] * by));
        } else {
          float* po = a.po + place * DP + c * 16;
#pragma unroll
          for (int e = 0; e < 16; e += 4)
            *reinterpret_cast<float4*>(po + e) = make_float4(y[e], y[e + 1], y[e + 2], y[e + 3]);
        }
      };
      if constexpr (HALF) {
        float4* box = reinterpret_cast<float4*>(sQ) + row * (DP / 4);        // 16-byte pieces, turned by the row
        if (s == 1 && here > 1 && !idle) {
#pragma unroll 1
          for (int c = 0; c < DP / 16; ++c) {
            uint32_t o[16];
            tmem_ld16(lane_base + Cfg::O(1) + 16 * c, o);
#pragma unroll
            for (int i = 0; i < 4; ++i)
              box[(4 * c + i) ^ (row & 7)] =
                  make_float4(__uint_as_float(o[4 * i]) * f1, __uint_as_float(o[4 * i + 1]) * f1,
                              __uint_as_float(o[4 * i + 2]) * f1, __uint_as_float(o[4 * i + 3]) * f1);
          }
        }
        named_bar(3, Cfg::SOFT);
        if (s == 0 && !idle) {
#pragma unroll 1
          for (int c = 0; c < DP / 16; ++c) {
            uint32_t o[16];
            tmem_ld16(lane_base + Cfg::O(0) + 16 * c, o);
            float y[16];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
              if (here > 1) v = box[(4 * c + i) ^ (row & 7)];
              y[4 * i] = fmaf(__uint_as_float(o[4 * i]), f0, v.x);
              y[4 * i + 1] = fmaf(__uint_as_float(o[4 * i + 1]), f0, v.y);
              y[4 * i + 2] = fmaf(__uint_as_float(o[4 * i + 2]), f0, v.z);
              y[4 * i + 3] = fmaf(__uint_as_float(o[4 * i + 3]), f0, v.w);
            }
            leave(c, y);
          }
        }
      } else if (!idle) {
#pragma unroll 1
        for (int c = s * (DP / 32); c < (s + 1) * (DP / 32); ++c) {
          uint32_t o[16], o1[16];
          tmem_ld16(lane_base + Cfg::O(0) + 16 * c, o);
          if (here > 1) tmem_ld16(lane_base + Cfg::O(1) + 16 * c, o1);
          float y[16];
#pragma unroll
          for (int e = 0; e < 16; ++e) {
            y[e] = __uint_as_float(o[e]) * f0;
            if (here > 1) y[e] = fmaf(__uint_as_float(o1[e]), f1, y[e]);
          }
          leave(c, y);
        }
      }
      if (s == 0 && mine) {
        if (complete) ca_write_row(a, at.n, tok, hq, M, L);
        else a.ml[place] = make_float2(M, L);
      }
      tc_fence_before();
      named_bar(2, Cfg::SOFT + 32);
      tc_fence_after();
      if (done < count) at.next(a, a.blocks);
    }
  }
  tc_fence_before();
  __syncthreads();
  if (abort_flag && tid == 0) set_status(a.status, LILICORR_ERR_TIMEOUT);
  if (warp == Cfg::MMA_WARP) {
    tc_fence_after();
    tmem_dealloc(tmem, CT_TMEM);
  }
}

// The items that several CTAs have parts of, in a launch of its own: up to 128 rows of 512 bytes a part are too much
// for the last CTA alone. A block has CJ_ROWS rows, a warp each, of the item at a border between two teams' parts of
// the list, if that is the item's first border.
constexpr int CJ_ROWS = 8;
template <int DP>
__global__ void __launch_bounds__(32 * CJ_ROWS) cache_attention_tc_join_kernel(const CaArgs a, int pieces) {
  pdl_wait();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const uint32_t id = blockIdx.x / pieces, border = id / a.team;
  const int head = id - border * a.team, rows = a.T * a.rep;
  const uint32_t teams = gridDim.x / pieces / a.team + 1;
  CaCursor<CT_KEYS> at;
  uint32_t per;
  const uint32_t total =
      ca_locate<CT_KEYS>(a, a.blocks, teams, [&](uint32_t p) { return (border + 1) * p; }, &at, &per);
  const uint32_t x = (border + 1) * per, s0 = x - at.tile;
  if (x >= total || at.tile == 0 || s0 / per != border) return;
  const uint32_t last = (s0 + at.tiles - 1) / per;
  const int i = (blockIdx.x - id * pieces) * CJ_ROWS + warp, r = at.rb * CT_ROWS + i;
  if (i >= CT_ROWS || r >= rows) return;
  auto part = [&](uint32_t team) { return (2 * ((size_t)team * a.team + head) + (team * per < s0)) * CT_ROWS + i; };
  float M = -FLT_MAX, L = 0.f;
  float4 y = make_float4(0.f, 0.f, 0.f, 0.f);
  for (uint32_t t0 = border; t0 <= last; t0 += 32) { // 32 parts: references and sums are all asked for at once
    const int parts = min(32u, last - t0 + 1);
    const float2 z = lane < parts ? a.ml[part(t0 + lane)] : make_float2(-FLT_MAX, 0.f);
    float4 v[8];
    auto ask = [&](int j) {
#pragma unroll
      for (int k = 0; k < 8; ++k)
        if (j + k < parts && lane < DP / 4)
          v[k] = *reinterpret_cast<const float4*>(a.po + part(t0 + j + k) * DP + lane * 4);
    };
    ask(0);
    const float to = fmaxf(M, warp_max(z.x)), x0 = ex2(M - to), f = ex2(z.x - to);
    M = to;
    L = L * x0 + warp_sum(f * z.y);
    y.x *= x0; y.y *= x0; y.z *= x0; y.w *= x0;
    for (int j = 0; j < parts; j += 8) {
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        const float g = __shfl_sync(0xffffffffu, f, (j + k) & 31);
        if (j + k < parts && lane < DP / 4) {
          y.x = fmaf(g, v[k].x, y.x);
          y.y = fmaf(g, v[k].y, y.y);
          y.z = fmaf(g, v[k].z, y.z);
          y.w = fmaf(g, v[k].w, y.w);
        }
      }
      ask(j + 8);
    }
  }
  const int t = r / a.rep;
  ca_write<__nv_bfloat16>(a, at.n, t, (at.h + head) * a.rep + (r - t * a.rep), M, L, y, lane);
}

template <int DP, int DIM, bool HALF>
lilicorr_status_t launch_tc(const CaArgs& a, const CaPlan& p, cudaStream_t st) {
  using Cfg = CtCfg<DP, HALF>;
  static bool configured[64] = {false};
  auto* kernel = cache_attention_tc_kernel<DP, DIM, HALF>;
  LL_TRY(allow_max_dynamic_smem(kernel, configured));
  LL_TRY(launch_k(kernel, (unsigned)p.ctas, Cfg::THREADS, Cfg::SMEM, st, a));
  if (p.ctas <= a.team) return LILICORR_OK;
  const int pieces = (min(CT_ROWS, a.T * a.rep) + CJ_ROWS - 1) / CJ_ROWS;
  return launch_k(cache_attention_tc_join_kernel<DP>, (unsigned)((p.ctas - a.team) * pieces),
                  32 * CJ_ROWS, 0, st, a, pieces);
}
template <int DP, int DIM>
lilicorr_status_t launch_rows(const CaArgs& a, const CaPlan& p, cudaStream_t st) {
  return a.T * a.rep <= 64 ? launch_tc<DP, DIM, true>(a, p, st) : launch_tc<DP, DIM, false>(a, p, st);
}

}  // namespace

lilicorr_status_t launch_ca_tc(const CaArgs& a, const CaPlan& p, cudaStream_t st) {
  if (a.c.d == 128) return launch_rows<128, 128>(a, p, st);
  if (a.c.d == 64) return launch_rows<64, 64>(a, p, st);
  return a.c.d < 64 ? launch_rows<64, 0>(a, p, st) : launch_rows<128, 0>(a, p, st);
}

}  // namespace lilicorr
