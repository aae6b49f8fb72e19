// Attention over a cache held in 4 bits on the 5th-generation tensor cores: bf16 queries of more rows than one
// matrix instruction has columns (drafted blocks under verification, wide groups of heads), 128 rows at a time
// against tiles of 128 keys.
//
// One CTA an SM. Warps 9-16 copy records to shared memory and expand them, a thread half a record, to fp16 (exact:
// six significant bits) in the swizzled layout that the tensor cores read: warps 9-12 keys, 13-16 values.
// Warp 8 issues
//   S = Q K^T   (M 128, N 128)   into tensor memory, and
//   O += P V    (M 128, N d)     with P read from tensor memory, V as the MN-major operand.
// Warps 0-3 and 4-7 are two streams, a thread a row, that take the key tiles in turn: while one is at its
// exponentials the tensor cores work for the other. Queries are brought to fp16 by a power of two of their row,
// as on mma.sync (cache_attention_kernels.cuh). Each stream has its own references and sums, whole numbers
// m that move only when a score passes them by 8; at an item's end the two come together.
//
// What bounds it: 1,024 clocks a tile for the two products at d = 128, whatever the number of rows, beside 480 issue
// slots for the expansion and 64 KB written to and 96 KB read from shared memory.
#include "cache_attention_kernels.cuh"
#include "tc_ptx.cuh"

namespace lilicorr {
namespace {
using namespace tc;

constexpr int CT_SOFT = 256, CT_EXPAND = 256, CT_THREADS = CT_SOFT + 32 + CT_EXPAND;
constexpr int CT_KEYS = 128, CT_ROWS = 128;
constexpr uint32_t CT_CHUNK = 128 * 128;             // 128 rows of 128 bytes
constexpr uint32_t CT_TMEM = 512;
constexpr int CT_RAW = 3;                            // tiles of records under way

template <int DP>
struct CtCfg {
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

// fp16 operands, fp32 sums
__host__ __device__ constexpr uint32_t instr_desc_f16(int m, int n) {
  return (1u << 4) | ((uint32_t)(n >> 3) << 17) | ((uint32_t)(m >> 4) << 24);
}
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
__device__ __forceinline__ bool elect_one() {        // one lane of a converged warp
  uint32_t r;
  asm volatile("{\n .reg .pred p;\n elect.sync _|p, 0xffffffff;\n selp.u32 %0, 1, 0, p;\n}" : "=r"(r));
  return r != 0;
}
// 2^d of a whole number d <= 0 (0 below the normal range, and for -inf)
__device__ __forceinline__ float pow2_down(float d) {
  return d < -126.f ? 0.f : __int_as_float((127 + (int)d) << 23);
}
// A wait that did not end at once: false after `limit` SM cycles, or when another warp gave up.
__device__ __noinline__ bool wait_long(uint64_t* bar, uint32_t parity, long long limit,
                                       volatile int* abort_flag) {
  const long long t0 = clock64();
  while (!mbar_try_wait(bar, parity)) {
    if (*abort_flag) return false;
    if (clock64() - t0 > limit) {
      *abort_flag = 1;
      return false;
    }
  }
  return true;
}

// Half a record at `rec` (or zeros) as row `key` of a tile: DP columns of fp16, zeros past the head's width.
template <int DP, int DIM>
__device__ __forceinline__ void expand(const unsigned char* rec, bool there, int d, uint8_t* tile, int key) {
  const uint32_t zero = there ? 0xFFu : 0u;          // (a scale of 0: codes are finite whatever they are)
#pragma unroll
  for (int g = 0; g < DP / 16; ++g) {
    uint4 v[2] = {make_uint4(0, 0, 0, 0), make_uint4(0, 0, 0, 0)};
    if (DIM || g * 16 < d) {
      const uint2 w = *reinterpret_cast<const uint2*>(rec + g * 8);
      const uint32_t b = rec[d / 2 + g] & zero, f = scales(b | b << 8);
      uint32_t r[4];
      codes(w.x, r);
      v[0] = make_uint4(mul2(r[0], f), mul2(r[1], f), mul2(r[2], f), mul2(r[3], f));
      codes(w.y, r);
      v[1] = make_uint4(mul2(r[0], f), mul2(r[1], f), mul2(r[2], f), mul2(r[3], f));
    }
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int p = 2 * g + i;
      *reinterpret_cast<uint4*>(tile + (p >> 3) * CT_CHUNK + swz(key, p & 7)) = v[i];
    }
  }
}

template <int DP, int DIM>
__global__ void __launch_bounds__(CT_THREADS, 1) cache_attention_tc_kernel(const CaArgs a) {
  using Cfg = CtCfg<DP>;
  using E = __nv_bfloat16;
  constexpr int NK = Cfg::NK, NV = Cfg::NV;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* sQ = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) &
                                           ~static_cast<uintptr_t>(1023));
  uint8_t* sK = sQ + Cfg::TILE;
  uint8_t* sV = sK + NK * Cfg::TILE;
  uint8_t* sR = sV + NV * Cfg::TILE;
  __shared__ __align__(8) uint64_t k_full[NK], k_empty[NK], v_full[NV], v_empty[NV];
  __shared__ __align__(8) uint64_t s_ready[2], p_ready[2], o_ready[2], drain;
  __shared__ uint32_t tmem_base;
  __shared__ volatile int abort_flag;
  __shared__ float s_factor[CT_ROWS];
  __shared__ float2 s_ml[2][CT_ROWS];
  __shared__ bool joins;

  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int d = DIM ? DIM : a.c.d, R = cache_record_bytes(d), rows = a.T * a.rep;
  if (tid == 0) {
    for (int i = 0; i < NK; ++i) { mbar_init(&k_full[i], 4); mbar_init(&k_empty[i], 1); }
    for (int i = 0; i < NV; ++i) { mbar_init(&v_full[i], 4); mbar_init(&v_empty[i], 1); }
    for (int i = 0; i < 2; ++i) {
      mbar_init(&s_ready[i], 1);
      mbar_init(&p_ready[i], 4);
      mbar_init(&o_ready[i], 1);
    }
    mbar_init(&drain, 1);
    abort_flag = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == 8) tmem_alloc(&tmem_base, CT_TMEM);
  pdl_wait();
  CaCursor<CT_KEYS> at;
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

  if (warp > 8) {
    // ---- records: copied two tiles ahead, expanded when both their tile and its place are there
    const int x = tid - CT_SOFT - 32, key = x & 127, is_v = x >> 7;
    const int vecs = R / 16;
    CaCursor<CT_KEYS> ahead = at;
    uint32_t copied = 0;
    auto copy_next = [&] {
      if (copied < count) {
        uint8_t* dst = sR + copied % CT_RAW * Cfg::RAW;
        const int k0 = ahead.tile * CT_KEYS, there = ahead.len - k0;
        const unsigned char* src = a.c.at(ahead.n, k0, ahead.h);
        for (int i = x; i < CT_KEYS * vecs; i += CT_EXPAND) {
          const int k = i / vecs;
          if (k < there) copy16(smem_u32(dst + i * 16), src + k * a.c.s[1] + (i - k * vecs) * 16, true);
        }
        if (++ahead.tile == ahead.tiles && copied + 1 < count) ahead.next(a, a.blocks);
      }
      ++copied;
      copy_commit();
    };
    copy_next();
    copy_next();
    uint64_t* full = is_v ? v_full : k_full;
    uint64_t* empty = is_v ? v_empty : k_empty;
    uint8_t* ring = is_v ? sV : sK;
    uint32_t slot = 0, parity = 1;
    bool ok = true;
    for (; done < count; ++done) {
      copy_wait<1>();
      named_bar(4, CT_EXPAND);                       // this tile is there for all, the one before it used up
      copy_next();
      if (ok && a.test_starve != is_v + 1) {
        ok = wait(&empty[slot], parity);
        if (ok) {
          const unsigned char* rec = sR + done % CT_RAW * Cfg::RAW + key * R + is_v * cache_half_bytes(d);
          expand<DP, DIM>(rec, at.tile * CT_KEYS + key < at.len, d, ring + slot * Cfg::TILE, key);
          fence_async_shared();
          __syncwarp();
          if (lane == 0) mbar_arrive(&full[slot]);
        }
      }
      if (++slot == (is_v ? NV : NK)) { slot = 0; parity ^= 1u; }
      if (++at.tile == at.tiles && done + 1 < count) at.next(a, a.blocks);
    }
    copy_wait<0>();
  } else if (warp == 8) {
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
      named_bar(1, CT_SOFT + 32);                    // Q is there
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
      named_bar(2, CT_SOFT + 32);                    // the item is done with
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
    const int s = warp >> 2, row = (warp & 3) * 32 + lane;
    const uint32_t lane_base = tmem + ((uint32_t)((warp & 3) * 32) << 16);
    uint32_t sn = 0, on = 0;                         // scores and outputs met so far
    while (done < count) {
      const int tile0 = at.tile, tile1 = min((uint32_t)at.tiles, tile0 + (count - done));
      const uint32_t here = tile1 - tile0;
      const int tile_rows = min(CT_ROWS, rows - at.rb * CT_ROWS);
      const int r = at.rb * CT_ROWS + row, tok = r / a.rep, hq = at.h * a.rep + (r - tok * a.rep);
      const bool mine = row < tile_rows;
      // the block's queries: the first stream a row a thread
      if (s == 0) {
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
          *reinterpret_cast<uint4*>(sQ + (p >> 3) * CT_CHUNK + swz(row, p & 7)) = make_uint4(w[0], w[1], w[2], w[3]);
        }
        s_factor[row] = a.scale * pow2(-up);
        fence_async_shared();
        if (a.scores && mine) a.factors[((size_t)at.n * a.T + tok) * a.Hq + hq] = a.scale * pow2(-up);
      }
      named_bar(1, CT_SOFT + 32);
      const float f = s_factor[row];
      const bool idle = (warp & 3) * 32 >= tile_rows;
      const int lim = mine ? at.len - (a.T - 1 - tok) : 0;     // keys that the row sees
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
        uint32_t x[32];
        float mx[2] = {-INFINITY, -INFINITY};
#pragma unroll
        for (int c = 0; c < 4; ++c) {
          tmem_ld32(lane_base + Cfg::S(s) + 32 * c, x);
          if (masked)
#pragma unroll
            for (int e = 0; e < 32; ++e)
              if (32 * c + e >= seen) x[e] = 0xFF800000u;        // -inf
#pragma unroll
          for (int e = 0; e < 32; e += 4) {
            mx[0] = fmaxf(fmaxf(mx[0], __uint_as_float(x[e])), __uint_as_float(x[e + 1]));
            mx[1] = fmaxf(fmaxf(mx[1], __uint_as_float(x[e + 2])), __uint_as_float(x[e + 3]));
          }
          if (a.scores && mine) {                    // for what each key gets: 32 rows of a key side by side
            float* to = a.scores + (((size_t)at.n * a.c.H + at.h) * a.c.S + k0 + 32 * c) * a.pad + r;
#pragma unroll
            for (int e = 0; e < 32; ++e)
              if (k0 + 32 * c + e < at.len) to[(size_t)e * a.pad] = __uint_as_float(x[e]);
          }
        }
        const float top = fmaxf(mx[0], mx[1]) * f;
        if (t == (uint32_t)s) {
          m = ceilf(top);
        } else if (__any_sync(0xffffffffu, top > m + CA_SLACK)) {
          // the sums so far to the new reference, by a whole power of two (their product is complete: the
          // scores came behind it)
          const float to = fmaxf(m, ceilf(top)), y = pow2_down(m - to);
          m = to;
          l *= y;
#pragma unroll 1
          for (int c = 0; c < DP / 16; ++c) {
            uint32_t o[16];
            tmem_ld16(lane_base + Cfg::O(s) + 16 * c, o);
#pragma unroll
            for (int e = 0; e < 16; ++e) o[e] = __float_as_uint(__uint_as_float(o[e]) * y);
            tmem_st16(lane_base + Cfg::O(s) + 16 * c, o);
          }
        }
        const float base = CA_UP - (m == -INFINITY ? 0.f : m);
#pragma unroll
        for (int c = 0; c < 4; ++c) {
          tmem_ld32(lane_base + Cfg::S(s) + 32 * c, x);
          uint32_t p[16];
          float sum[2] = {0.f, 0.f};
#pragma unroll
          for (int e = 0; e < 32; e += 2) {
            float p0 = ex2(fmaf(__uint_as_float(x[e]), f, base)), p1 = ex2(fmaf(__uint_as_float(x[e + 1]), f, base));
            if (masked) {
              if (32 * c + e >= seen) p0 = 0.f;
              if (32 * c + e + 1 >= seen) p1 = 0.f;
            }
            sum[0] += p0;
            sum[1] += p1;
            p[e / 2] = half2_of(p0, p1);
          }
          l += sum[0] + sum[1];
          tmem_st16(lane_base + Cfg::P(s, 2 * c), p);
        }
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
      // ---- the two streams' sums come together: each takes half of the columns
      s_ml[s][row] = make_float2(m, l);
      named_bar(3, CT_SOFT);
      const float2 z0 = s_ml[0][row], z1 = s_ml[1][row];
      const float M = fmaxf(fmaxf(z0.x, z1.x), -FLT_MAX);
      const float f0 = ex2(z0.x - M), f1 = here > 1 ? ex2(z1.x - M) : 0.f, L = z0.y * f0 + z1.y * f1;
      const bool complete = tile0 == 0 && tile1 == at.tiles;
      const uint32_t s0 = first + done - tile1, team0 = s0 / per, team1 = (s0 + at.tiles - 1) / per;
      const int head = blockIdx.x % a.team;
      auto part = [&](uint32_t team) { return 2 * ((size_t)team * a.team + head) + (team * per < s0); };
      const size_t place = part(blockIdx.x / a.team) * CT_ROWS + row;
      const float by = L == 0.f ? 0.f : a.c.v_unit / L;
      if (!idle) {
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
          if (!mine || c * 16 >= d) continue;
          if (complete) {
            E* out = static_cast<E*>(a.out) + at.n * a.o_s[0] + tok * a.o_s[1] + hq * a.o_s[2] + c * 16;
#pragma unroll
            for (int e = 0; e < 16; e += 8)
              *reinterpret_cast<uint4*>(out + e) =
                  L == 0.f ? make_uint4(0, 0, 0, 0)
                           : make_uint4(bf16_pack2(y[e] * by, y[e + 1] * by), bf16_pack2(y[e + 2] * by, y[e + 3] * by),
                                        bf16_pack2(y[e + 4] * by, y[e + 5] * by), bf16_pack2(y[e + 6] * by, y[e + 7] * by));
          } else {
            float* po = a.po + place * DP + c * 16;
#pragma unroll
            for (int e = 0; e < 16; e += 4) *reinterpret_cast<float4*>(po + e) = make_float4(y[e], y[e + 1], y[e + 2], y[e + 3]);
          }
        }
      }
      if (s == 0 && mine) {
        if (complete) ca_write_row(a, at.n, tok, hq, M, L);
        else a.ml[place] = make_float2(M, L);
      }
      if (!complete) {
        named_bar(3, CT_SOFT);
        if (tid == 0) {
          __threadfence();
          uint32_t* left = a.left + part(team0);
          joins = atomicAdd(left, 1u) == team1 - team0;
          if (joins) *left = 0;
          __threadfence();
        }
        named_bar(3, CT_SOFT);
        if (joins)
          for (int i0 = warp * 4; i0 < tile_rows; i0 += 32) {  // four rows a warp, a part of each at a time
            float jm[4], jl[4];
            float4 y[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
              jm[j] = -FLT_MAX;
              jl[j] = 0.f;
              y[j] = make_float4(0.f, 0.f, 0.f, 0.f);
            }
#pragma unroll 1
            for (uint32_t team = team0; team <= team1; ++team) {
              const size_t at_part = part(team) * CT_ROWS;
              float2 z[4];
              float4 v[4];
#pragma unroll
              for (int j = 0; j < 4; ++j) {
                const int i = min(i0 + j, tile_rows - 1);
                z[j] = __ldcg(&a.ml[at_part + i]);
                v[j] = lane < DP / 4 ? __ldcg(reinterpret_cast<const float4*>(a.po + (at_part + i) * DP + lane * 4))
                                     : make_float4(0.f, 0.f, 0.f, 0.f);
              }
#pragma unroll
              for (int j = 0; j < 4; ++j) {
                const float to = fmaxf(jm[j], z[j].x), x0 = ex2(jm[j] - to), x1 = ex2(z[j].x - to);
                jm[j] = to;
                jl[j] = jl[j] * x0 + z[j].y * x1;
                y[j].x = y[j].x * x0 + v[j].x * x1;
                y[j].y = y[j].y * x0 + v[j].y * x1;
                y[j].z = y[j].z * x0 + v[j].z * x1;
                y[j].w = y[j].w * x0 + v[j].w * x1;
              }
            }
#pragma unroll
            for (int j = 0; j < 4; ++j)
              if (i0 + j < tile_rows) {
                const int rr = at.rb * CT_ROWS + i0 + j, t = rr / a.rep;
                ca_write<E>(a, at.n, t, at.h * a.rep + (rr - t * a.rep), jm[j], jl[j], y[j], lane);
              }
          }
      }
      tc_fence_before();
      named_bar(2, CT_SOFT + 32);
      tc_fence_after();
      if (done < count) at.next(a, a.blocks);
    }
  }
  tc_fence_before();
  __syncthreads();
  if (abort_flag && tid == 0) set_status(a.status, LILICORR_ERR_TIMEOUT);
  if (warp == 8) {
    tc_fence_after();
    tmem_dealloc(tmem, CT_TMEM);
  }
}

template <int DP, int DIM>
lilicorr_status_t launch_tc(const CaArgs& a, const CaPlan& p, cudaStream_t st) {
  static bool configured[64] = {false};
  auto* kernel = cache_attention_tc_kernel<DP, DIM>;
  LL_TRY(allow_max_dynamic_smem(kernel, configured));
  return launch_k(kernel, (unsigned)p.ctas, CT_THREADS, CtCfg<DP>::SMEM, st, a);
}

}  // namespace

lilicorr_status_t launch_ca_tc(const CaArgs& a, const CaPlan& p, cudaStream_t st) {
  if (a.c.d == 128) return launch_tc<128, 128>(a, p, st);
  if (a.c.d == 64) return launch_tc<64, 64>(a, p, st);
  return a.c.d < 64 ? launch_tc<64, 0>(a, p, st) : launch_tc<128, 0>(a, p, st);
}

}  // namespace lilicorr
