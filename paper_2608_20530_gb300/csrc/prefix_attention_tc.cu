// The shared prefix on the 5th-generation tensor cores (bf16): the rows of all sequences of a group
// (PA_BLOCK at a time, two tiles of 128) against tiles of 128 of its keys.
//
// One CTA an SM. Warps 8 and 10 feed K and V tiles by TMA into two rings. Warp 9 issues
//   S = Q K^T   (M 128, N 128)   into tensor memory, and
//   O += P V    (M 128, N d)     with P read from tensor memory, V as the MN-major operand.
// Warps 0-3 and 4-7 are two streams, a thread a row: it reads the row's scores 64 at a time (all 128 at
// once spill), takes the running maximum, writes P = 2^(s - m) as bf16 and keeps the row's sum. While one
// stream is at its exponentials the tensor cores work for the other. With two row tiles the streams share
// each key tile; with one they take the key tiles in turn, and each leaves its own sums. Warps without a row
// do nothing but keep the count of arrivals.
//
// O is not rescaled whenever a maximum grows: m, a whole number, is what a row's sums are taken against, and
// it moves only when a score would pass it by 8, so that terms stay below 2^8 and sums exact to fp32.
//
// What bounds it: bytes of K and V for up to about 256 rows a group (each is read from HBM once and
// from L2 by the further row blocks), beyond that the two products (512 clocks each of an SM's tensor
// cores a 128 x 128 tile at d = 128) beside 16,384 exponentials (512 clocks at 32 a clock).
#include "prefix_attention.cuh"
#include "tc_ptx.cuh"

namespace lilicorr {

namespace {
using namespace tc;

constexpr int PT_THREADS = 352;
constexpr int PT_SOFT = 256;                         // of them in the streams
constexpr uint32_t PT_CHUNK = 128 * 128;             // 128 rows of 128 bytes
constexpr uint32_t PT_TMEM = 512;

// ONE: no group has more than 128 rows: one row tile, and the second's space goes to the rings, which
// then hold three tiles of K and of V (d = 128) where two row tiles leave room for three and two. The
// bytes under way are what bounds few rows: 8 groups behind 5,120 keys of 8 heads, d = 64, 32 rows 36.7 ->
// 35.0 us, 128 rows 52.3 -> 50.6; d = 128, 32 rows 51.6 -> 50.9, 128 rows the same (72).
template <int DP, bool ONE>
struct PtCfg {
  static constexpr int CH = DP / 64;                 // 64-column chunks of a row
  static constexpr uint32_t TILE = CH * PT_CHUNK;    // bytes of a K, V or Q tile
  static constexpr int NQ = ONE ? 1 : 2;
  static constexpr int NK = DP == 128 ? 3 : 6, NV = DP == 128 ? (ONE ? 3 : 2) : 6;
  static constexpr size_t QBYTES = NQ * TILE < 32768 ? 32768 : NQ * TILE;      // (and the rows' way out)
  static constexpr size_t SMEM = 1024 + QBYTES + (size_t)(NK + NV) * TILE;
  // tensor-memory columns: scores, output, and the probabilities of keys [16 k, 16 k + 16). At d = 128
  // those lie over the scores, which their thread has read: the next scores of the stream are issued
  // behind the product that reads them, and products of one shape run in the order of issue. At d = 64 the
  // two products differ in shape, and there is room elsewhere.
  __device__ static constexpr uint32_t S(int s) { return s * 128; }
  __device__ static constexpr uint32_t O(int s) { return 256 + s * DP; }
  __device__ static constexpr uint32_t P(int s, int k) {
    return (DP == 128 ? S(s) : 384 + s * 64) + k * 8;
  }
};

// A of the product from tensor memory
__device__ __forceinline__ void mma_bf16_ta(uint32_t tmem_d, uint32_t tmem_a, uint64_t b, uint32_t idesc,
                                            uint32_t accumulate) {
  asm volatile(
      "{\n .reg .pred p;\n setp.ne.b32 p, %4, 0;\n"
      " tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n}" ::"r"(tmem_d),
      "r"(tmem_a), "l"(b), "r"(idesc), "r"(accumulate));
}
// MN-major operand of 128-byte-swizzled rows: 64-column chunks PT_CHUNK bytes apart, 8-row groups 1024
__device__ __forceinline__ uint64_t smem_desc_mn(const void* tile) {
  return smem_desc(tile) & ~(0x3FFFull << 16) | ((uint64_t)(PT_CHUNK >> 4) << 16);
}

// one lane of a converged warp
__device__ __forceinline__ bool elect_one() {
  uint32_t r;
  asm volatile("{\n .reg .pred p;\n elect.sync _|p, 0xffffffff;\n selp.u32 %0, 1, 0, p;\n}" : "=r"(r));
  return r != 0;
}
// packed fp32 pairs: one instruction for both halves (a tensor-memory load leaves its columns in
// neighbouring registers, so no moves pair them up)
__device__ __forceinline__ uint64_t pair_of(uint32_t lo, uint32_t hi) {
  uint64_t r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "r"(lo), "r"(hi));
  return r;
}
__device__ __forceinline__ void halves(uint64_t v, float& lo, float& hi) {
  asm("mov.b64 {%0, %1}, %2;" : "=f"(lo), "=f"(hi) : "l"(v));
}
__device__ __forceinline__ uint64_t fma_pair(uint64_t a, uint64_t b, uint64_t c) {
  uint64_t d;
  asm("fma.rn.ftz.f32x2 %0, %1, %2, %3;" : "=l"(d) : "l"(a), "l"(b), "l"(c));
  return d;
}
__device__ __forceinline__ uint64_t add_pairs(uint64_t a, uint64_t b) {
  uint64_t d;
  asm("add.rn.ftz.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
  return d;
}

// Nothing that uses these registers moves above this point (a load from tensor memory fills them until
// its wait).
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

// Where a CTA is in the list of tiles.
struct Cursor {
  int g;                       // group
  uint32_t item;               // key head * blocks + block
  uint32_t tile;               // of the item
  uint32_t left;               // tiles of this CTA from here on
};
__device__ __forceinline__ int pt_len(const PaKeys& k, int g) {
  return min(max(k.len[g], 0), k.capacity);
}
__device__ __forceinline__ uint32_t pt_tiles(const PaKeys& k, int g) {
  return (uint32_t)(pt_len(k, g) + PA_TILE - 1) / PA_TILE;
}
// The tiles of the segment that starts here; `next` moves behind them.
__device__ __forceinline__ uint32_t pt_here(const PaKeys& k, const Cursor& c) {
  return min(c.left, pt_tiles(k, c.g) - c.tile);
}
__device__ __forceinline__ void pt_next(const PaArgs& a, const PaKeys& k, Cursor& c, uint32_t here) {
  c.left -= here;
  c.tile = 0;
  if (c.left == 0) return;
  if (++c.item == (uint32_t)a.Hkv * a.seg_blocks) {
    c.item = 0;
    do ++c.g;
    while (pt_tiles(k, c.g) == 0);
  }
}

template <int DP, bool ONE>
__global__ void __launch_bounds__(PT_THREADS, 1)
pa_tc_kernel(const __grid_constant__ CUtensorMap map_k, const __grid_constant__ CUtensorMap map_v,
             int copies, const PaArgs a, const PaKeys kk, int rows) {
  using Cfg = PtCfg<DP, ONE>;
  constexpr int NK = Cfg::NK, NV = Cfg::NV;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>(
      (reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~static_cast<uintptr_t>(1023));
  uint8_t* sQ = smem;
  uint8_t* sK = smem + Cfg::QBYTES;
  uint8_t* sV = sK + NK * Cfg::TILE;
  uint32_t* s_sum = reinterpret_cast<uint32_t*>(sQ);             // before the first Q
  __shared__ __align__(8) uint64_t k_full[NK], k_empty[NK], v_full[NV], v_empty[NV];
  __shared__ __align__(8) uint64_t s_ready[2], p_ready[2], o_ready[2], drain;
  __shared__ uint32_t tmem_base;
  __shared__ volatile int abort_flag;
  __shared__ Cursor s_cur;

  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  if (tid == 0) {
    for (int i = 0; i < NK; ++i) { mbar_init(&k_full[i], 1); mbar_init(&k_empty[i], 1); }
    for (int i = 0; i < NV; ++i) { mbar_init(&v_full[i], 1); mbar_init(&v_empty[i], 1); }
    for (int i = 0; i < 2; ++i) {
      mbar_init(&s_ready[i], 1);
      mbar_init(&p_ready[i], 4);
      mbar_init(&o_ready[i], 1);
    }
    mbar_init(&drain, 1);
    abort_flag = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == 9) tmem_alloc(&tmem_base, PT_TMEM);
  pdl_wait();

  // ---- this CTA's part of the list: tiles of each thread's run of groups, their scan
  const uint32_t hb = (uint32_t)a.Hkv * a.seg_blocks;
  const int run = (a.G + PT_THREADS - 1) / PT_THREADS;
  const int ga = min(a.G, tid * run), gb = min(a.G, ga + run);
  uint32_t mine = 0;
  for (int g = ga; g < gb; ++g) mine += pt_tiles(kk, g);
  s_sum[tid] = mine;
  if (tid == 0) s_cur.left = 0;
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  uint32_t before = 0, total = 0;
  const int used = (a.G + run - 1) / run;            // threads that have groups
  for (int i = 0; i < used; ++i) {
    if (i == tid) before = total;
    total += s_sum[i];
  }
  const uint32_t all = total * hb, per = pa_per_cta(all, a.seg_ctas);
  const uint32_t from = min(all, blockIdx.x * per), to = min(all, from + per);
  uint32_t at = before;
  for (int g = ga; g < gb; ++g) {
    const uint32_t n = pt_tiles(kk, g);
    if (blockIdx.x == 0) a.seg_start[g] = at;
    if (from < to && from >= at * hb && from < (at + n) * hb) {
      const uint32_t in = from - at * hb;
      s_cur.g = g;
      s_cur.item = in / n;
      s_cur.tile = in % n;
      s_cur.left = to - from;
    }
    at += n;
  }
  if (blockIdx.x == 0 && tid == 0) a.seg_start[a.G] = total;
  __syncthreads();
  Cursor cur = s_cur;
  const uint32_t tmem = tmem_base;
  auto wait = [&](uint64_t* bar, uint32_t parity) {
    return mbar_try_wait(bar, parity) || wait_long(bar, parity, a.wait_limit, &abort_flag);
  };
  // the same for a whole warp: all lanes go on, or none
  auto wait_all = [&](uint64_t* bar, uint32_t parity) {
    if (__all_sync(0xffffffffu, mbar_try_wait(bar, parity))) return true;
    return __all_sync(0xffffffffu, wait_long(bar, parity, a.wait_limit, &abort_flag)) != 0;
  };

  if (warp == 8 || warp == 10) {
    // ---- copies, K by one warp and V by the other: a K tile's place is free as soon as its scores are
    // there, long before V's, and waits for no V tile. The first queries are asked for first: everything
    // waits for them, and they would queue behind the 24 MB of tiles that all SMs ask for at once.
    if (cur.left) named_bar(4, PT_SOFT + 64);
    if (lane == 0) {
      const bool is_k = warp == 8;
      const CUtensorMap* map = is_k ? &map_k : &map_v;
      uint64_t* full = is_k ? k_full : v_full;
      uint64_t* empty = is_k ? k_empty : v_empty;
      uint8_t* ring = is_k ? sK : sV;
      const uint32_t slots = is_k ? NK : NV;
      uint32_t slot = 0, parity = 1, issued = 0;
      bool ok = true;
      const bool starve = a.test_starve == (is_k ? 1 : 2);
      while (cur.left && ok && !starve) {
        const uint32_t here = pt_here(kk, cur);
        const int hk = (int)(cur.item / a.seg_blocks);
        for (uint32_t t = 0; t < here; ++t) {
          if (!wait(&empty[slot], parity)) { ok = false; break; }
          mbar_expect_tx(&full[slot], Cfg::TILE);
          for (int c = 0; c < copies; ++c)
            tma_load_5d(ring + slot * Cfg::TILE + c * PT_CHUNK, map, &full[slot], c * 64,
                        (int)(cur.tile + t) * PA_TILE, 0, hk, cur.g);
          ++issued;
          if (++slot == slots) { slot = 0; parity ^= 1u; }
        }
        pt_next(a, kk, cur, here);
      }
      if (!ok)                                       // given up: the copies under way land before the
        for (uint32_t x = issued > slots ? issued - slots : 0; x < issued; ++x)      // CTA's memory goes
          mbar_wait(&full[x % slots], (x / slots) & 1u, a.wait_limit);
    }
    __syncwarp();
  } else if (warp == 9) {
    // ---- products. The whole warp walks, one lane issues: a single thread's own loop, with its
    // descriptors formed one by one, took 80 clocks a product and was what everything waited for.
    constexpr uint32_t idesc_s = instr_desc(128, 128);
    constexpr uint32_t idesc_o = instr_desc(128, DP) | (1u << 16);       // V MN-major
    const bool leader = elect_one();
    const uint64_t q_desc = smem_desc(sQ), k_desc = smem_desc(sK), v_desc = smem_desc_mn(sV);
    uint32_t ki = 0, kp = 0, vi = 0, vp = 0;         // the rings' next slots and their parities
    uint32_t pp[2] = {0, 0};                         // parity of the streams' probabilities
    while (cur.left) {
      const uint32_t here = pt_here(kk, cur);
      const int block = (int)(cur.item % a.seg_blocks);
      const bool two = !ONE && rows - block * PA_BLOCK > 128;
      const int end = pt_len(kk, cur.g) - (int)cur.tile * PA_TILE;       // keys from this segment on
      named_bar(1, PT_SOFT + 32);                    // Q is there
      tc_fence_after();
      bool ok = true;
      // S of stream s from the K tile in the ring's next slot; last: the slot's last use
      auto scores = [&](int s, bool first, bool last) {
        if (first) {
          if (!wait_all(&k_full[ki], kp)) { ok = false; return; }
          tc_fence_after();
        }
        const uint64_t qd = q_desc + (two ? s : 0) * (Cfg::TILE >> 4), kd = k_desc + ki * (Cfg::TILE >> 4);
        if (leader) {
#pragma unroll
          for (int c = 0; c < Cfg::CH; ++c)
#pragma unroll
            for (int k = 0; k < 4; ++k)
              mma_bf16(tmem + Cfg::S(s), qd + c * (PT_CHUNK >> 4) + 2 * k, kd + c * (PT_CHUNK >> 4) + 2 * k,
                       idesc_s, (c | k) > 0);
          mma_commit(&s_ready[s]);
          if (last) mma_commit(&k_empty[ki]);
        }
        __syncwarp();
        if (last && ++ki == NK) { ki = 0; kp ^= 1u; }
      };
      // O += P V of stream s and the key tile `keys` long in the V ring's next slot
      auto sums = [&](int s, int keys, bool fresh, bool first, bool last, bool done) {
        if (!wait_all(&p_ready[s], pp[s])) { ok = false; return; }
        pp[s] ^= 1u;
        if (first && !wait_all(&v_full[vi], vp)) { ok = false; return; }
        tc_fence_after();
        const uint64_t vd = v_desc + vi * (Cfg::TILE >> 4);
        if (leader) {
          if (keys >= PA_TILE) {
#pragma unroll
            for (int k = 0; k < PA_TILE / 16; ++k)
              mma_bf16_ta(tmem + Cfg::O(s), tmem + Cfg::P(s, k), vd + k * 128, idesc_o, !fresh || k > 0);
          } else {
#pragma unroll 1
            for (int k = 0; k * 16 < keys; ++k)
              mma_bf16_ta(tmem + Cfg::O(s), tmem + Cfg::P(s, k), vd + k * 128, idesc_o, !fresh || k > 0);
          }
          if (last) mma_commit(&v_empty[vi]);
          if (done) mma_commit(&o_ready[s]);
        }
        __syncwarp();
        if (last && ++vi == NV) { vi = 0; vp ^= 1u; }
      };
      if (two) {
        scores(0, true, false);
        if (ok) scores(1, false, true);
        for (uint32_t t = 0; t < here && ok; ++t) {
          const int keys = end - (int)t * PA_TILE;
          const bool more = t + 1 < here;
          sums(0, keys, t == 0, true, false, !more);
          if (ok && more) scores(0, true, false);
          if (ok) sums(1, keys, t == 0, false, true, !more);
          if (ok && more) scores(1, false, true);
        }
      } else {
        scores(0, true, true);
        if (ok && here > 1) scores(1, true, true);
        for (uint32_t t = 0; t < here && ok; ++t) {
          const int s = (int)(t & 1u);
          sums(s, end - (int)t * PA_TILE, t < 2, true, true, t + 2 >= here);
          if (ok && t + 2 < here) scores(s, true, true);
        }
      }
      named_bar(2, PT_SOFT + 32);                    // the segment is done with
      pt_next(a, kk, cur, here);
    }
    if (abort_flag) {                                // products under way, before their memory goes
      if (leader) mma_commit(&drain);
      mbar_wait(&drain, 0, a.wait_limit);
      __syncwarp();
    }
  } else if (warp < 8) {
    // ---- the streams: a thread a row
    const int s = warp >> 2, row = (warp & 3) * 32 + lane;
    const uint32_t lane_base = tmem + ((uint32_t)((warp & 3) * 32) << 16);
    uint32_t sn = 0, on = 0;                         // scores and outputs met so far
    uint32_t i0 = 0;
    while (cur.left) {
      const uint32_t here = pt_here(kk, cur);
      const int block = (int)(cur.item % a.seg_blocks), hk = (int)(cur.item / a.seg_blocks);
      const bool two = !ONE && rows - block * PA_BLOCK > 128;
      const int end = pt_len(kk, cur.g) - (int)cur.tile * PA_TILE;
      // Q of the block: 16-byte pieces in swizzled rows, zeros past the rows and the head's width. A lane
      // finds the place of one row, the warp copies its 32 (or 16) rows one or two at a time.
      {
        constexpr int PIECES = DP / 8, AT_ONCE = 32 / PIECES;
        const int per_warp = two ? 32 : 16, r0 = warp * per_warp;
        int64_t off = -1;
        if (lane < per_warp && block * PA_BLOCK + r0 + lane < rows) {
          const PaRow w = pa_row(a, 0, cur.g, hk, block * PA_BLOCK + r0 + lane);
          off = (int64_t)w.n * a.q_s[0] + (int64_t)w.t * a.q_s[1] + (int64_t)w.h * a.q_s[2];
        }
        const int p = lane % PIECES;
        for (int x = 0; x < per_warp; x += AT_ONCE) {
          const int r = r0 + x + lane / PIECES;
          const int64_t at = __shfl_sync(0xffffffffu, off, x + lane / PIECES);
          const bool there = at >= 0 && p * 8 < a.d;
          const __nv_bfloat16* src = static_cast<const __nv_bfloat16*>(a.q) + (there ? at + p * 8 : 0);
          const uint32_t dst = smem_u32(sQ + (r >> 7) * Cfg::TILE + (p >> 3) * PT_CHUNK + swz(r & 127, p & 7));
          asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src),
                       "r"(there ? 16 : 0)
                       : "memory");
        }
        if (i0 == 0) named_bar(4, PT_SOFT + 64);       // the first segment's: the tiles may follow
        asm volatile("cp.async.commit_group;\n cp.async.wait_group 0;" ::: "memory");
        fence_async_shared();
      }
      named_bar(1, PT_SOFT + 32);
      const int tile_rows = min(128, rows - block * PA_BLOCK - (two ? s * 128 : 0));
      const int warps = (tile_rows + 31) / 32;       // of the stream's that have rows
      const bool idle = (warp & 3) >= warps;
      float m = -INFINITY, l = 0.f;
      bool ok = true;
      const uint32_t first = two ? 0 : (uint32_t)s, step = two ? 1 : 2;
      for (uint32_t t = first; t < here; t += step) {
        if (!wait_all(&s_ready[s], sn & 1u)) { ok = false; break; }
        ++sn;
        if (idle) {                                  // (what P holds for its rows reaches no other row)
          if (lane == 0) mbar_arrive(&p_ready[s]);
          continue;
        }
        tc_fence_after();
        const int keys = end - (int)t * PA_TILE;
        // 64 scores at a time, a step of the running maximum each: the second half's are read while the
        // first's exponentials run (all 128 at once spill beside the rest)
        uint32_t x[2][32];
        auto load = [&](int quarter) {
          tmem_ld32_nowait(lane_base + Cfg::S(s) + 32 * quarter, x[quarter & 1]);
        };
        auto landed = [&]() {
          tmem_wait_ld();
          pin(x[0]);
          pin(x[1]);
        };
        load(0);
        load(1);
        landed();
        if (keys < PA_TILE) {
          // V behind the last key: zeros, whatever the cache holds there (to the product's 16)
          const uint32_t i = i0 + t;
          if (!wait_all(&v_full[i % NV], (i / NV) & 1u)) { ok = false; break; }
          uint8_t* v = sV + (i % NV) * Cfg::TILE;
          const int up = (keys + 15) / 16 * 16;
          for (int z = row; z < (up - keys) * (DP / 8); z += warps * 32) {
            const int vr = keys + z / (DP / 8), p = z % (DP / 8);
            *reinterpret_cast<uint4*>(v + (p >> 3) * PT_CHUNK + vr * 128 + (p & 7) * 16) =
                make_uint4(0, 0, 0, 0);
          }
          fence_async_shared();
          __syncwarp();
        }
#pragma unroll
        for (int half = 0; half < 2; ++half) {
          if (keys < PA_TILE) {
#pragma unroll
            for (int c = 0; c < 2; ++c)
#pragma unroll
              for (int e = 0; e < 32; ++e)
                if (64 * half + 32 * c + e >= keys) x[c][e] = 0xFF800000u;         // -inf
          }
          float mx[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
          for (int e = 0; e < 32; e += 4)              // three at a time
#pragma unroll
            for (int c = 0; c < 2; ++c) {
              mx[c] = fmaxf(fmaxf(mx[c], __uint_as_float(x[c][e])), __uint_as_float(x[c][e + 1]));
              mx[2 + c] = fmaxf(fmaxf(mx[2 + c], __uint_as_float(x[c][e + 2])), __uint_as_float(x[c][e + 3]));
            }
          const float top = fmaxf(fmaxf(mx[0], mx[1]), fmaxf(mx[2], mx[3])) * a.scale_log2;
          if (half == 0 && t == first) {
            m = ceilf(top);
          } else if (__any_sync(0xffffffffu, top > m + 8.f)) {
            // the sums so far, and the first half's probabilities, to the new maximum: by a whole power
            // of two, which rounds nothing that 2^-118 of the row's largest term would show (their product is
            // complete: the scores came behind it)
            const float to = fmaxf(m, ceilf(top)), f = pow2_down(m - to);
            m = to;
            l *= f;
            if (half == 1) tmem_wait_st();             // the first half's stores, of O too where it moved
            if (t != first) {
#pragma unroll 1
              for (int c = 0; c < DP / 16; ++c) {
                uint32_t o[16];
                tmem_ld16(lane_base + Cfg::O(s) + 16 * c, o);
#pragma unroll
                for (int e = 0; e < 16; ++e) o[e] = __float_as_uint(__uint_as_float(o[e]) * f);
                tmem_st16(lane_base + Cfg::O(s) + 16 * c, o);
              }
            }
            if (half == 1) {
#pragma unroll 1
              for (int c = 0; c < 2; ++c) {
                uint32_t p[16];
                tmem_ld16(lane_base + Cfg::P(s, 2 * c), p);
#pragma unroll
                for (int e = 0; e < 16; ++e)
                  p[e] = pack_bf16x2(__uint_as_float(p[e] << 16) * f, __uint_as_float(p[e] & 0xFFFF0000u) * f);
                tmem_st16(lane_base + Cfg::P(s, 2 * c), p);
              }
            }
          }
          const float base = m == -INFINITY ? 0.f : m;
          uint64_t sum0 = 0ull, sum1 = 0ull;
          const uint64_t sc2 = pair_of(__float_as_uint(a.scale_log2), __float_as_uint(a.scale_log2));
          const uint64_t nb2 = pair_of(__float_as_uint(-base), __float_as_uint(-base));
#pragma unroll
          for (int c = 0; c < 2; ++c) {
            uint32_t p[16];
#pragma unroll
            for (int e = 0; e < 16; ++e) {
              float p0, p1;
              halves(fma_pair(pair_of(x[c][2 * e], x[c][2 * e + 1]), sc2, nb2), p0, p1);
              p0 = pa_ex2(p0);
              p1 = pa_ex2(p1);
              const uint64_t pp = pair_of(__float_as_uint(p0), __float_as_uint(p1));
              if (e & 1) sum1 = add_pairs(sum1, pp);
              else sum0 = add_pairs(sum0, pp);
              p[e] = pack_bf16x2(p0, p1);
            }
            if (half == 0) load(2 + c);
            tmem_st16(lane_base + Cfg::P(s, 4 * half + 2 * c), p);
          }
          float l0, l1;
          halves(add_pairs(sum0, sum1), l0, l1);
          l += l0 + l1;
          if (half == 0) landed();
        }
        tmem_wait_st();
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(&p_ready[s]);
      }
      if (ok && first < here) {
        if (!wait_all(&o_ready[s], on & 1u)) ok = false;
        ++on;
        tc_fence_after();
      }
      const uint32_t item = (uint32_t)cur.g * hb + cur.item;
      const size_t seg = ((size_t)blockIdx.x + item) * PA_BLOCK;
      // the rows' sums to memory, 32 columns at a time by way of the warp's 4 KB of Q's space (every
      // product with Q is done): a lane has a row there, and 128 bytes of a row leave together. With one
      // row tile the second stream's part of the keys takes the place of the second tile's rows.
      named_bar(3, PT_SOFT);
      const int place = s * 128 + (warp & 3) * 32;   // the warp's first row of the segment
      uint8_t* box = sQ + warp * 4096;
      auto piece = [&](int rr, int p) { return rr * 128 + ((p ^ (rr & 7)) << 4); };
      if (!idle && first < here) {
#pragma unroll 1
        for (int c = 0; 32 * c < a.d; ++c) {
          uint32_t o[32];
          tmem_ld32(lane_base + Cfg::O(s) + 32 * c, o);
          __syncwarp();
#pragma unroll
          for (int p = 0; p < 8; ++p)
            *reinterpret_cast<uint4*>(box + piece(lane, p)) =
                make_uint4(o[4 * p], o[4 * p + 1], o[4 * p + 2], o[4 * p + 3]);
          __syncwarp();
          const int col = 32 * c + 4 * (lane & 7);
          float* dst = a.seg_po + (seg + place) * a.d + col;
#pragma unroll
          for (int x = 0; x < 32; x += 4) {
            const int rr = x + (lane >> 3);
            if (ok && col < a.d && (warp & 3) * 32 + rr < tile_rows)
              *reinterpret_cast<float4*>(dst + (size_t)rr * a.d) =
                  *reinterpret_cast<const float4*>(box + piece(rr, lane & 7));
          }
        }
      }
      if (row < tile_rows) a.seg_ml[seg + place + lane] = make_float2(m, l);
      i0 += here;
      tc_fence_before();
      named_bar(2, PT_SOFT + 32);
      tc_fence_after();
      pt_next(a, kk, cur, here);
    }
  }
  if (abort_flag && tid == 0) set_status(a.status, LILICORR_ERR_TIMEOUT);
  tc_fence_before();
  __syncthreads();
  if (warp == 9) {
    tc_fence_after();
    tmem_dealloc(tmem, PT_TMEM);
  }
}

// K or V as (64 columns, position, 64-column block, head, group): one copy a tile where the width is a
// multiple of 64; else blocks by the first coordinate, zeros past the width.
bool pt_map(CUtensorMap* map, const void* base, const int64_t (&s)[3], const PaArgs& a, int capacity,
            int* copies) {
  const bool whole = a.d % 64 == 0;
  const uint64_t dims[5] = {whole ? 64u : (uint64_t)a.d, (uint64_t)capacity,
                            whole ? (uint64_t)a.d / 64 : 1u, (uint64_t)a.Hkv, (uint64_t)a.G};
  // (a dimension of one has stride 0 here, which a map does not take)
  auto bytes = [&](int64_t stride, int extent) {
    return extent > 1 ? (uint64_t)stride * 2 : (uint64_t)16 * ((a.d + 7) / 8);
  };
  const uint64_t strides[5] = {2, bytes(s[1], capacity), whole ? 128u : bytes(0, 1), bytes(s[2], a.Hkv),
                               bytes(s[0], a.G)};
  for (int i = 1; i < 5; ++i)
    if (strides[i] == 0) return false;               // an expanded dimension
  const uint32_t box[5] = {64, PA_TILE, whole ? (uint32_t)a.d / 64 : 1u, 1, 1};
  *copies = whole ? 1 : (a.d + 63) / 64;
  return make_map_nd(map, base, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 5, dims, strides, box);
}

template <int DP, bool ONE>
lilicorr_status_t launch_tc(const PaArgs& a, const PaKeys& k, const PaMaps& m, cudaStream_t st) {
  static bool configured[64] = {false};
  auto* kernel = pa_tc_kernel<DP, ONE>;
  LL_TRY(allow_max_dynamic_smem(kernel, configured));
  return launch_k(kernel, a.seg_ctas, PT_THREADS, PtCfg<DP, ONE>::SMEM, st, m.k, m.v, m.copies, a, k,
                  a.seg_rows);
}

}  // namespace

bool pa_tc_maps(const PaArgs& a, const PaKeys& k, PaMaps* m) {
  return encode_fn() != nullptr && pt_map(&m->k, k.k, k.k_s, a, k.capacity, &m->copies) &&
         pt_map(&m->v, k.v, k.v_s, a, k.capacity, &m->copies);
}

lilicorr_status_t launch_pa_tc(const PaArgs& a, const PaKeys& k, const PaMaps& m, cudaStream_t st) {
  if (a.seg_rows <= 128)
    return a.d <= 64 ? launch_tc<64, true>(a, k, m, st) : launch_tc<128, true>(a, k, m, st);
  return a.d <= 64 ? launch_tc<64, false>(a, k, m, st) : launch_tc<128, false>(a, k, m, st);
}

}  // namespace lilicorr
