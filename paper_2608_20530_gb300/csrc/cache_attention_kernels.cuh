// Attention over a cache held in 4 bits: the kernels.
//
// A record's elements are products of 2 and 4 significant bits: exact in fp16. So both products run on fp16
// matrix instructions with fp32 sums, without a rounding of keys or values: queries are brought to fp16 by a
// power of two of their row (bf16: exact to 2^-38 of the row's largest; fp32: as three fp16 numbers that add
// up to it), the probabilities are rounded to fp16 (for fp32 queries, kept as three numbers again).
//
// Products are turned round: keys (of the second product, elements) are the 16 rows of a matrix instruction,
// query rows its 8 columns, so the few rows of a decoding step fill it, and what is read from the cache is
// expanded once, in the registers that the instruction reads, whatever the number of rows.
//
// What bounds it: bytes by the cache's rate, 32 sequences of 2,048 to 8,192 positions, 8 heads of 128, 4 rows each:
// 49.8 us, 3.9 TB/s of records; one of 131,072: 38.9. A key more costs as much as at 5.3 to 6.1 TB/s, and 12 to 14 us
// are start, first bytes, parts and their join. On the way 16 keys cost a warp some 320 instructions, 54 % of all
// issue slots (alu pipe 45 %: unpacking codes). Tried: 16 warps a CTA that share a tile (a barrier each: 50 -> 66 us), three CTAs
// an SM at 80 registers (49 -> 54), shorter shares for the CTAs that start last (no better).
#pragma once
#include <float.h>

#include "cache_attention.cuh"

namespace lilicorr {
namespace {

constexpr int CA_WARPS = 8;                  // of a CTA, each with its own keys of a tile
constexpr int CA_THREADS = 32 * CA_WARPS;
// Probabilities are 2^(s - m + CA_UP) with the row's reference m. Only where a score is more than CA_SLACK above
// it does it move, to CA_ROOM above the largest so far, so that few steps have sums to rescale. The largest is
// then between 2^6 and 2^15, and fp16 numbers have their full precision down to 2^-20 of it. (Up to scores of 2^24 in
// log2 units: their sums with the reference round by at most 1/2 there, and 2^15.5 is still an fp16 number.)
constexpr float CA_UP = 7.f, CA_SLACK = 8.f, CA_ROOM = 1.f;

// The work is the list of all (sequence, team of kv heads, row block, tile of KEYS keys), in that order, cut
// evenly over the teams of CTAs: team g takes tiles [g * per, (g + 1) * per), each of its CTAs for its own head.
// So the heads of a position, which may lie side by side in 64 bytes that memory reads at once, are read
// at about the same time. An item is one (sequence, kv head, row block). A CTA leaves at most two parts of items
// that other CTAs have parts of: of its first item (place 2 b) and of its last (2 b + 1). Of the CTAs that have parts
// of an item, the last to leave its own joins them, in the order of the list (a launch of its own for that: 43 us for
// 41). One head after the other, records of 144 bytes 8 heads apart, read 259 MB for 193 (lines of 128 bytes that
// two heads share).
__device__ __forceinline__ uint32_t ca_per_team(uint32_t tiles, uint32_t teams) {
  return max(1u, (tiles + teams - 1) / teams);
}
// tiles of a row block of a sequence: one even where there is no key, none where there is no sequence
template <int KEYS>
__device__ __forceinline__ int ca_tiles(int raw, int S) {
  return raw < 0 ? 0 : max(1, (min(raw, S) + KEYS - 1) / KEYS);
}

// A place in the list.
template <int KEYS>
struct CaCursor {
  int n, h, rb, tile, tiles, len;            // len: what the cache holds of the sequence
  __device__ __forceinline__ void set(const CaArgs& a, int at, int raw) {
    n = at;
    len = cache_len(raw, a.c.S);
    tiles = ca_tiles<KEYS>(raw, a.c.S);
  }
  // positions that token t sees: up to its own, seq_len - T + t, as far as the cache holds them; all tokens see the
  // first len - (T - 1). (Rows past the last token: len. The length itself is read again, where it matters: held,
  // it cost decoding steps 0.3 us.)
  __device__ __forceinline__ int seen(const CaArgs& a, int t) const {
    return a.T == 1 ? len : min(len, a.seq_len[n] - max(a.T - 1 - t, 0));
  }
  __device__ __forceinline__ void sequence(const CaArgs& a, int at) { set(a, at, a.seq_len[at]); }
  // the next item; there has to be one
  __device__ __forceinline__ void next(const CaArgs& a, int blocks) {
    tile = 0;
    if (++rb < blocks) return;
    rb = 0;
    h += a.team;
    if (h < a.c.H) return;
    h -= a.c.H;
    do sequence(a, n + 1); while (tiles == 0);
  }
};

// The list cut over `teams` teams: `per` tiles each. `want` (of `per`) says which place of the list `at` becomes,
// which head of the team apart; the number of places. Each warp finds it for itself.
template <int KEYS, typename F>
__device__ __forceinline__ uint32_t ca_locate(const CaArgs& a, int blocks, uint32_t teams, F want,
                                              CaCursor<KEYS>* at, uint32_t* per) {
  const int lane = threadIdx.x & 31, N = a.c.N, chunk = (N + 31) / 32;
  const int n0 = min(N, lane * chunk), n1 = min(N, n0 + chunk);
  const uint32_t per_tile = (uint32_t)(a.c.H / a.team) * blocks;
  int raw = -1;                                      // of n0, the only one up to 32 sequences
  if (n0 < n1) raw = a.seq_len[n0];
  uint32_t mine = ca_tiles<KEYS>(raw, a.c.S);
#pragma unroll 4
  for (int n = n0 + 1; n < n1; ++n) mine += ca_tiles<KEYS>(a.seq_len[n], a.c.S);
  mine *= per_tile;
  uint32_t upto = mine;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const uint32_t x = __shfl_up_sync(0xffffffffu, upto, o);
    if (lane >= o) upto += x;
  }
  const uint32_t total = __shfl_sync(0xffffffffu, upto, 31);
  *per = ca_per_team(total, teams);
  const uint32_t wanted = want(*per);
  if (wanted >= total) return total;
  const int owner = __ffs(__ballot_sync(0xffffffffu, wanted < upto)) - 1;
  uint32_t b = upto - mine;
  int n = n0;
  if (lane == owner && chunk > 1)
    while (true) {
      const uint32_t t = ca_tiles<KEYS>(raw, a.c.S) * per_tile;
      if (wanted < b + t) break;
      b += t;
      raw = a.seq_len[++n];
    }
  at->set(a, __shfl_sync(0xffffffffu, n, owner), __shfl_sync(0xffffffffu, raw, owner));
  const uint32_t place = wanted - __shfl_sync(0xffffffffu, b, owner), item = place / at->tiles;
  at->tile = place - item * at->tiles;
  at->h = item / blocks;
  at->rb = item - at->h * blocks;
  at->h *= a.team;
  return total;
}
// This CTA's part of the list: as many tiles as it returns, from `at` on, which is place `first` of the list.
template <int KEYS>
__device__ __forceinline__ uint32_t ca_range(const CaArgs& a, int blocks, CaCursor<KEYS>* at, uint32_t* first,
                                             uint32_t* per) {
  const uint32_t g = blockIdx.x / a.team;
  const uint32_t total = ca_locate<KEYS>(a, blocks, gridDim.x / a.team, [&](uint32_t p) { return g * p; }, at, per);
  *first = g * *per;
  if (*first >= total) return 0;
  at->h += blockIdx.x - g * a.team;
  return min(*per, total - *first);
}

// ------------------------------------------------------------------------------- small pieces
__device__ __forceinline__ uint32_t smem_u32(const void* p) { return (uint32_t)__cvta_generic_to_shared(p); }
// 16 bytes to shared memory, zeros where !there
__device__ __forceinline__ void copy16(uint32_t dst, const void* src, bool there) {
  asm volatile("cp.async.cg.shared.global.L2::128B [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(there ? 16 : 0)
               : "memory");
}
__device__ __forceinline__ void copy_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void copy_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }
__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ void mma(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
      : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
      : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t transpose8(uint32_t x) {   // an 8 x 8 matrix of 16-bit elements
  uint32_t y;
  asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
  return y;
}
__device__ __forceinline__ uint32_t half2_of(float lo, float hi) {
  uint32_t r;
  asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  return r;
}
__device__ __forceinline__ void half2_sub(uint32_t h, float& lo, float& hi) {   // what rounding to h left
  float a, b;
  asm("{\n .reg .b16 l, h;\n mov.b32 {l, h}, %2;\n cvt.f32.f16 %0, l;\n cvt.f32.f16 %1, h;\n}"
      : "=f"(a), "=f"(b) : "r"(h));
  lo -= a;
  hi -= b;
}
__device__ __forceinline__ float pow2(int e) { return __uint_as_float((uint32_t)(e + 127) << 23); }   // |e| < 127
__device__ __forceinline__ uint32_t mul2(uint32_t a, uint32_t b) {
  uint32_t r;
  asm("mul.rn.f16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
  return r;
}
// the two codes of each byte of w
__device__ __forceinline__ void codes(uint32_t w, uint32_t (&r)[4]) {
  asm("{\n .reg .b8 a, b, c, d;\n mov.b32 {a, b, c, d}, %4;\n cvt.rn.f16x2.e2m1x2 %0, a;\n"
      " cvt.rn.f16x2.e2m1x2 %1, b;\n cvt.rn.f16x2.e2m1x2 %2, c;\n cvt.rn.f16x2.e2m1x2 %3, d;\n}"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(w));
}
__device__ __forceinline__ uint32_t scales(uint32_t two) {     // of two bytes
  uint32_t r;
  asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(r) : "h"((uint16_t)two));
  return r;
}

// The key of row r, r < 8, of a matrix instruction; row r + 8 is the key behind it. In this order neither the
// reads of keys (8 or 16 bytes a lane, four lanes a record) nor those of values (4 or 8 bytes a lane, eight
// lanes a record, of every second key of the order) meet in a bank, for records of 80 and 144 bytes.
__device__ __forceinline__ int key_of(int r) {
  const int j = r >> 1, hi = j >> 1;
  return 2 * (j & 1) + 8 * hi + 4 * ((r & 1) ^ hi);
}

template <typename F, int... I>
__device__ __forceinline__ void steps(F& f, std::integer_sequence<int, I...>) {
  (f(std::integral_constant<int, I>{}), ...);
}

template <int DP>
struct CaCfg {
  static constexpr int KS = DP / 16;         // matrix steps of a score; tiles of 16 elements of the output
  static constexpr int KB = DP / 8;          // key bytes a lane: elements [c * DP / 4, (c + 1) * DP / 4)
  static constexpr int CH = (16 * (DP + 16) / 16 + 31) / 32;   // 16-byte pieces a lane of 16 records
  static constexpr int XL = DP + 4;
};

// A lane's 16-byte pieces of 16 records (of their first `bytes` bytes).
template <int DP>
struct CaLane {
  uint32_t off[CaCfg<DP>::CH];               // in the cache
  int pieces, per;                           // 16-byte pieces: of 16 records, of one
  __device__ __forceinline__ CaLane(const CaArgs& a, int bytes, int lane) {
    per = bytes / 16;
    pieces = 16 * per;
#pragma unroll
    for (int u = 0; u < CaCfg<DP>::CH; ++u) {
      const int i = lane + 32 * u, key = i / per;
      off[u] = (uint32_t)key * (uint32_t)a.c.s[1] + (i - key * per) * 16;
    }
  }
  // the 16 records at src, of which `there` are held (any number)
  __device__ __forceinline__ void copy(const CaArgs& a, const unsigned char* src, int there, uint32_t dst,
                                       int lane) const {
    if (there >= 16) {
#pragma unroll
      for (int u = 0; u < CaCfg<DP>::CH; ++u)
        if (lane + 32 * u < pieces) copy16(dst + (lane + 32 * u) * 16, src + off[u], true);
    } else {
#pragma unroll
      for (int u = 0; u < CaCfg<DP>::CH; ++u)
        if (lane + 32 * u < pieces) {
          const bool held = (lane + 32 * u) / per < there;
          copy16(dst + (lane + 32 * u) * 16, held ? static_cast<const void*>(src + off[u]) : a.q, held);
        }
    }
  }
};

// A lane's part of the keys of a matrix instruction: rows g and g + 8, all steps.
template <int DP>
struct CaKeyPart {
  uint32_t w[2][DP / 32 < 1 ? 1 : DP / 32];  // codes, 8 a word
  uint32_t s[2];                             // scales as fp16: DP 128 of two groups, else of one, twice
  __device__ __forceinline__ void load(const unsigned char* rec, int R, int d, int c, uint32_t mask) {
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      const unsigned char* p = rec + e * R + c * CaCfg<DP>::KB;
      if constexpr (DP == 128) {
        const uint4 x = *reinterpret_cast<const uint4*>(p);
        w[e][0] = x.x; w[e][1] = x.y; w[e][2] = x.z; w[e][3] = x.w;
        s[e] = scales(*reinterpret_cast<const uint16_t*>(rec + e * R + d / 2 + 2 * c) & mask);
      } else {
        if constexpr (DP == 64) {
          const uint2 x = *reinterpret_cast<const uint2*>(p);
          w[e][0] = x.x; w[e][1] = x.y;
        } else {
          w[e][0] = *reinterpret_cast<const uint32_t*>(p);
        }
        const uint32_t b = rec[e * R + d / 2 + (DP == 64 ? c : c >> 1)] & mask;
        s[e] = scales(b | b << 8);
      }
    }
  }
  // the operands of steps 2 i and 2 i + 1: a[0], a[2] of row g, a[1], a[3] of row g + 8
  template <int i>
  __device__ __forceinline__ void operands(uint32_t (&a)[2][4]) const {
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      uint32_t f = s[e], r[4];
      if constexpr (DP == 128) f = __byte_perm(f, f, i < 2 ? 0x1010 : 0x3232);
      codes(w[e][i], r);
      a[0][e] = mul2(r[0], f);
      a[0][e + 2] = mul2(r[1], f);
      a[1][e] = mul2(r[2], f);
      a[1][e + 2] = mul2(r[3], f);
    }
  }
};
// bytes of a lane's key scales that exist
template <int DP>
__device__ __forceinline__ uint32_t key_scale_mask(int d, int c) {
  const int G = d / 16;
  if (DP == 128) return (2 * c < G ? 0xFFu : 0u) | (2 * c + 1 < G ? 0xFF00u : 0u);
  return (DP == 64 ? c : c >> 1) < G ? 0xFFu : 0u;
}

__device__ __forceinline__ void load16b(const float* p, float* x) {
  const float4 v = *reinterpret_cast<const float4*>(p);
  x[0] = v.x; x[1] = v.y; x[2] = v.z; x[3] = v.w;
}
__device__ __forceinline__ void load16b(const __nv_bfloat16* p, float* x) {
  const uint4 v = *reinterpret_cast<const uint4*>(p);
  const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    x[2 * i] = __uint_as_float(w[i] << 16);
    x[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
  }
}
// The power of two that takes a row's largest element to [2^13, 2^14); an infinity or a row of zeros stays as it is,
// and numbers that no power of two in fp32 brings so far (below 2^-113) go as far as it does.
__device__ __forceinline__ int query_shift(float top) {
  return top > 0.f && top < INFINITY ? min(140 - (int)(__float_as_uint(top) >> 23), 126) : 0;
}
// What takes the products of a row shifted by `up` to scores in log2 units; never 0, which would make NaN of the
// -infinity that stands for a key that is not seen.
__device__ __forceinline__ float row_factor(const CaArgs& a, int up) {
  return fmaxf(a.scale * pow2(-up), 0x1p-149f);
}
// Queries as the second operand: of column g (row `row` of the item, or none) elements c * DP / 4 ..,
// brought to fp16 by 2^(the result) of their row, in PIECES numbers that add up to them.
template <int DP, int PIECES, typename E>
__device__ __forceinline__ int load_query(const E* q, int d, int c, uint32_t (*b)[CaCfg<DP>::KS][2]) {
  float x[DP / 4];
  float top = 0.f;
#pragma unroll
  for (int i = 0; i < DP / 4; i += 16 / (int)sizeof(E)) {
    const int at = c * (DP / 4) + i;
    if (q && at < d) {
      load16b(q + at, x + i);
    } else {
#pragma unroll
      for (int j = 0; j < 16 / (int)sizeof(E); ++j) x[i + j] = 0.f;
    }
  }
#pragma unroll
  for (int i = 0; i < DP / 4; ++i) top = fmaxf(top, fabsf(x[i]));
  top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 1));
  top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 2));
  const int up = query_shift(top);
  const float by = pow2(up);
#pragma unroll
  for (int i = 0; i < DP / 4; i += 2) {
    float lo = x[i] * by, hi = x[i + 1] * by;
#pragma unroll
    for (int p = 0; p < PIECES; ++p) {
      const uint32_t h = half2_of(lo, hi);
      b[p][i / 4][i / 2 % 2] = h;
      half2_sub(h, lo, hi);
    }
  }
  return up;
}

// ------------------------------------------------------------------------------- the kernel
template <int DP, int NT, int PIECES>
struct CaSmem {
  static constexpr bool QS = NT * PIECES > 1;            // queries in shared memory
  static constexpr int SUB = NT == 2 || PIECES > 1 ? 1 : 2;   // 16 keys each, of a warp's step
  static constexpr int KEYS = 16 * SUB * CA_WARPS;       // of a tile
  static constexpr int STAGES = SUB > 1 ? 2 : 3;
  static constexpr int STAGE = 16 * SUB * (DP + 16);     // bytes of a warp's records
  static constexpr int XO = CA_WARPS * 8 * CaCfg<DP>::XL * 4;
  static constexpr int XM = CA_WARPS * 8 * 8;
  static constexpr int Q = QS ? NT * PIECES * CaCfg<DP>::KS * 256 : 0;
  static constexpr int AT_XO = CA_WARPS * STAGES * STAGE + 64;   // (lanes past a narrow record's end read on)
  static constexpr int AT_XM = AT_XO + XO;
  static constexpr int AT_Q = AT_XM + XM;
  static constexpr int TOTAL = AT_Q + Q;
};

template <typename E>
__device__ __forceinline__ void store4(E* p, const float4& v) {
  if constexpr (sizeof(E) == 4) *reinterpret_cast<float4*>(p) = v;
  else *reinterpret_cast<uint2*>(p) = make_uint2(bf16_pack2(v.x, v.y), bf16_pack2(v.z, v.w));
}
__device__ __forceinline__ void named_barrier(int id, int threads) {
  asm volatile("bar.sync %0, %1;" ::"r"(id), "r"(threads) : "memory");
}
// a row's normaliser from its reference and sum
__device__ __forceinline__ void ca_write_row(const CaArgs& a, int n, int t, int hq, float m, float l) {
  // the scores were taken in units that their factor's rounding moved
  const size_t row = ((size_t)n * a.T + t) * a.Hq + hq;
  a.lse[row] = l == 0.f ? -INFINITY
                        : fmaf(fmaf(m, a.rest_ratio, m), 0.69314718f, fmaf(-CA_UP, 0.69314718f, logf(l)));
  if (a.weights) a.rows[row] = make_float2(m, l);
}
// a row's result from these and the lane's four sums of p V
template <typename E>
__device__ __forceinline__ void ca_write(const CaArgs& a, int n, int t, int hq, float m, float l, float4 o,
                                         int lane) {
  E* out = static_cast<E*>(a.out) + n * a.o_s[0] + t * a.o_s[1] + hq * a.o_s[2];
  const float f = l == 0.f ? 0.f : a.c.v_unit / l;
  if (lane * 4 < a.c.d) store4(out + lane * 4, make_float4(o.x * f, o.y * f, o.z * f, o.w * f));
  if (lane == 0) ca_write_row(a, n, t, hq, m, l);
}

// DIM: head_dim where it is DP, which makes all places in a record constants, else 0.
template <int DP, int DIM, int NT, int PIECES, typename E>
__global__ void __launch_bounds__(CA_THREADS, NT * PIECES > 3 || NT > 2 ? 1 : 2)
cache_attention_kernel(const CaArgs a) {
  pdl_wait();
  using Cfg = CaCfg<DP>;
  using Sm = CaSmem<DP, NT, PIECES>;
  constexpr int KS = Cfg::KS, ST = Sm::STAGES, SUB = Sm::SUB, KEYS = Sm::KEYS, ROWS = 8 * NT;
  extern __shared__ __align__(16) unsigned char sm[];
  __shared__ bool joins;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, g = lane >> 2, c = lane & 3;
  const int d = DIM ? DIM : a.c.d, R = cache_record_bytes(d), half = cache_half_bytes(d), rows = a.T * a.rep;

  CaCursor<KEYS> at;
  uint32_t first = 0, per = 0, count;
  if (a.whole) {
    const int item = blockIdx.x / a.c.H;
    at.sequence(a, item / a.blocks);
    at.h = blockIdx.x - item * a.c.H;
    at.rb = item % a.blocks;
    at.tile = 0;
    count = at.tiles;
  } else {
    count = ca_range<KEYS>(a, a.blocks, &at, &first, &per);
  }
  if (count == 0) return;

  const CaLane<DP> mine(a, R, lane);
  unsigned char* stage = sm + warp * ST * Sm::STAGE;
  CaCursor<KEYS> ahead = at;                         // of the copies
  const unsigned char* src;
  int held;                                          // keys from src on
  const int64_t tile_bytes = KEYS * a.c.s[1];
  uint32_t copied = 0;
  auto seek = [&] {
    const int k = ahead.tile * KEYS + warp * (16 * SUB);
    src = a.c.at(ahead.n, k, ahead.h);
    held = ahead.len - k;
  };
  seek();
  auto copy_next = [&](int place) {
    if (copied < count) {
      const uint32_t dst = smem_u32(stage + place * Sm::STAGE);
#pragma unroll
      for (int i = 0; i < SUB; ++i) mine.copy(a, src + i * 16 * a.c.s[1], held - 16 * i, dst + i * 16 * R, lane);
      if (++copied < count) {
        if (++ahead.tile < ahead.tiles) {
          src += tile_bytes;
          held -= KEYS;
        } else {
          ahead.next(a, a.blocks);
          seek();
        }
      }
    }
    copy_commit();
  };
#pragma unroll
  for (int i = 0; i < ST; ++i) copy_next(i);

  // where this lane's keys and values lie in 16 records
  const int key = key_of(g), va = key_of(2 * c), vb = key_of(2 * c + 1);
  const uint32_t kmask = key_scale_mask<DP>(d, c);
  const int vg = DP == 128 ? g : DP == 64 ? g >> 1 : g >> 2;   // the scale group of its values
  const bool vthere = vg < d / 16;
  const int vbyte = vthere ? g * (DP / 16) : 0;

  uint32_t qr[Sm::QS ? 1 : PIECES][KS][2];
  uint2* qs = reinterpret_cast<uint2*>(sm + Sm::AT_Q);         // [NT][PIECES][KS][lane]
  float m[NT][2], l[NT][2], f[NT][2], fr[NT][2];               // f: a row's factor; fr: what it lacks
  float o[KS][NT][4];
  uint32_t done = 0;
  int place = 0;
  while (true) {
    // an item begins
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      const int r = at.rb * ROWS + nt * 8 + g, t = r / a.rep;
      const E* q = r < rows ? static_cast<const E*>(a.q) + at.n * a.q_s[0] + t * a.q_s[1] +
                                  (at.h * a.rep + (r - t * a.rep)) * a.q_s[2]
                            : nullptr;
      uint32_t qb[PIECES][KS][2];
      const int up = load_query<DP, PIECES, E>(q, d, c, qb);
      if constexpr (Sm::QS) {
        if (warp == 0)
#pragma unroll
          for (int p = 0; p < PIECES; ++p)
#pragma unroll
            for (int i = 0; i < KS; ++i)
              qs[((nt * PIECES + p) * KS + i) * 32 + lane] = make_uint2(qb[p][i][0], qb[p][i][1]);
      } else {
#pragma unroll
        for (int i = 0; i < KS; ++i) { qr[0][i][0] = qb[0][i][0]; qr[0][i][1] = qb[0][i][1]; }
      }
#pragma unroll
      for (int e = 0; e < 2; ++e) {                // this lane's columns
        const int u = __shfl_sync(0xffffffffu, up, (2 * c + e) * 4);
        f[nt][e] = row_factor(a, u);
        fr[nt][e] = a.scale_rest * pow2(-u);
        m[nt][e] = -FLT_MAX;
        l[nt][e] = 0.f;
        const int r = at.rb * ROWS + nt * 8 + 2 * c + e, t = r / a.rep;
        if (a.scores && warp == 0 && g == 0 && r < rows)
          a.factors[((size_t)at.n * a.T + t) * a.Hq + at.h * a.rep + (r - t * a.rep)] = f[nt][e];
      }
    }
#pragma unroll
    for (int i = 0; i < KS; ++i)
#pragma unroll
      for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int e = 0; e < 4; ++e) o[i][nt][e] = 0.f;
    if constexpr (Sm::QS) __syncthreads();
    // its tiles here, and the first place in the list behind the last of them
    const int tile0 = at.tile, tile1 = min((uint32_t)at.tiles, tile0 + (count - done));
#pragma unroll 1
    for (int tile = tile0; tile < tile1; ++tile) {
      copy_wait<ST - 1>();
      __syncwarp();
      const unsigned char* rec = stage + place * Sm::STAGE;

      // ---- scores
      float s[SUB][NT][4];
#pragma unroll
      for (int u = 0; u < SUB; ++u) {
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) s[u][nt][0] = s[u][nt][1] = s[u][nt][2] = s[u][nt][3] = 0.f;
        CaKeyPart<DP> kp;
        kp.load(rec + (16 * u + key) * R, R, d, c, kmask);
        auto step = [&](auto is) {
          constexpr int i = decltype(is)::value;
          uint32_t ka[2][4];
          kp.template operands<i>(ka);
#pragma unroll
          for (int j = 0; j < 2; ++j)
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
              for (int p = PIECES - 1; p >= 0; --p) {  // the smallest parts first
                if constexpr (Sm::QS) {
                  const uint2 b = qs[((nt * PIECES + p) * KS + 2 * i + j) * 32 + lane];
                  mma(s[u][nt], ka[j], b.x, b.y);
                } else {
                  mma(s[u][nt], ka[j], qr[p][2 * i + j][0], qr[p][2 * i + j][1]);
                }
              }
        };
        steps(step, std::make_integer_sequence<int, KS / 2>{});
      }
      const int k0 = tile * KEYS + warp * (16 * SUB);
      if (k0 + 16 * SUB > at.len - (a.T - 1)) {        // some row may not see all of these keys
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            const int r = at.rb * ROWS + nt * 8 + 2 * c + e;
            const int seen = at.seen(a, r / a.rep) - k0 - key;
#pragma unroll
            for (int u = 0; u < SUB; ++u) {
              if (16 * u >= seen) s[u][nt][e] = -INFINITY;
              if (16 * u + 1 >= seen) s[u][nt][e + 2] = -INFINITY;
            }
          }
      }
      if (a.scores) {                                  // for what each key gets
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
          if (nt * 8 + 2 * c < a.pad)
#pragma unroll
            for (int u = 0; u < SUB; ++u)
#pragma unroll
              for (int e = 0; e < 2; ++e) {
                const int k = k0 + 16 * u + key + e;
                if (k < at.len)
                  *reinterpret_cast<float2*>(a.scores + (((size_t)at.n * a.c.H + at.h) * a.c.S + k) * a.pad +
                                             nt * 8 + 2 * c) = make_float2(s[u][nt][2 * e], s[u][nt][2 * e + 1]);
              }
      }
      // ---- probabilities: the reference moves when some row of the warp's has left it behind
      float top[NT][2];
      bool up = false;
#pragma unroll
      for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          top[nt][e] = fmaxf(s[0][nt][e], s[0][nt][e + 2]);
#pragma unroll
          for (int u = 1; u < SUB; ++u) top[nt][e] = fmaxf(top[nt][e], fmaxf(s[u][nt][e], s[u][nt][e + 2]));
          up |= fmaf(top[nt][e], f[nt][e], -m[nt][e]) > CA_SLACK;
        }
      if (__any_sync(0xffffffffu, up)) {
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            float t = top[nt][e];
            t = fmaxf(t, __shfl_xor_sync(0xffffffffu, t, 4));
            t = fmaxf(t, __shfl_xor_sync(0xffffffffu, t, 8));
            t = fmaxf(t, __shfl_xor_sync(0xffffffffu, t, 16));
            const float to = fmaxf(m[nt][e], fmaf(t, f[nt][e], CA_ROOM)), x = ex2(m[nt][e] - to);
            m[nt][e] = to;
            l[nt][e] *= x;
#pragma unroll
            for (int i = 0; i < KS; ++i) {
              o[i][nt][e] *= x;
              o[i][nt][e + 2] *= x;
            }
          }
      }
#pragma unroll
      for (int u = 0; u < SUB; ++u) {
        uint32_t pb[NT][PIECES][2];
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
          float p[4];
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            float x = CA_UP - m[nt][e & 1];
            // (a key that is not seen has -infinity, which no number of either sign may meet: without one that is
            // seen the reference is -FLT_MAX, and anything above FLT_MAX would make NaN of it)
            if (PIECES > 1) x = s[u][nt][e] > -INFINITY ? fmaf(s[u][nt][e], fr[nt][e & 1], x) : x;
            p[e] = ex2(fmaf(s[u][nt][e], f[nt][e & 1], x));
          }
          l[nt][0] += p[0] + p[2];
          l[nt][1] += p[1] + p[3];
#pragma unroll
          for (int i = 0; i < PIECES; ++i) {
            const uint32_t x = half2_of(p[0], p[1]), y = half2_of(p[2], p[3]);
            pb[nt][i][0] = transpose8(x);
            pb[nt][i][1] = transpose8(y);
            if (PIECES > 1) {
              half2_sub(x, p[0], p[1]);
              half2_sub(y, p[2], p[3]);
            }
          }
        }
        // ---- sums of p V: two keys a register, so the codes of two records go together, byte by byte
        const unsigned char* v = rec + 16 * u * R + half;
        uint32_t fs[2], w[4][DP / 128 < 1 ? 1 : 2];
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const unsigned char *pa = v + (va + e) * R, *pb2 = v + (vb + e) * R;
          if constexpr (DP == 128) {
            const uint2 x = *reinterpret_cast<const uint2*>(pa + vbyte);
            const uint2 y = *reinterpret_cast<const uint2*>(pb2 + vbyte);
            w[2 * e][0] = x.x; w[2 * e][1] = x.y;
            w[2 * e + 1][0] = y.x; w[2 * e + 1][1] = y.y;
          } else if constexpr (DP == 64) {
            w[2 * e][0] = *reinterpret_cast<const uint32_t*>(pa + vbyte);
            w[2 * e + 1][0] = *reinterpret_cast<const uint32_t*>(pb2 + vbyte);
          } else {
            w[2 * e][0] = *reinterpret_cast<const uint16_t*>(pa + vbyte);
            w[2 * e + 1][0] = *reinterpret_cast<const uint16_t*>(pb2 + vbyte);
          }
          uint32_t b = pa[d / 2 + vg] | (uint32_t)pb2[d / 2 + vg] << 8;
          if (!vthere) b = 0;
          fs[e] = scales(b);
        }
        auto step = [&](auto is) {
          constexpr int i = decltype(is)::value;       // four tiles of 16 elements (DP 32: two)
          constexpr int tiles = KS < 4 ? KS : 4;
          uint32_t oa[4][4];
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            const uint32_t x = w[2 * e][i], y = w[2 * e + 1][i];
            uint32_t even[4], odd[4];
            codes((x & 0x0F0F0F0Fu) | ((y << 4) & 0xF0F0F0F0u), even);
            codes(((x >> 4) & 0x0F0F0F0Fu) | (y & 0xF0F0F0F0u), odd);
#pragma unroll
            for (int j = 0; j < tiles; ++j) {
              oa[j][2 * e] = mul2(even[j], fs[e]);
              oa[j][2 * e + 1] = mul2(odd[j], fs[e]);
            }
          }
#pragma unroll
          for (int j = 0; j < tiles; ++j)
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
              for (int p = PIECES - 1; p >= 0; --p) mma(o[4 * i + j][nt], oa[j], pb[nt][p][0], pb[nt][p][1]);
        };
        steps(step, std::make_integer_sequence<int, DP == 128 ? 2 : 1>{});
      }
      __syncwarp();                                    // the records' place is free
      copy_next(place);
      place = place + 1 == ST ? 0 : place + 1;
    }
    done += tile1 - tile0;

    // ---- the warps' parts of an item come together, 8 rows at a time, a warp a row
    const bool complete = tile0 == 0 && tile1 == at.tiles;
    float* xo = reinterpret_cast<float*>(sm + Sm::AT_XO);      // [warp][row][XL]
    float2* xm = reinterpret_cast<float2*>(sm + Sm::AT_XM);
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      __syncthreads();
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        float x = l[nt][e];
        x += __shfl_xor_sync(0xffffffffu, x, 4);
        x += __shfl_xor_sync(0xffffffffu, x, 8);
        x += __shfl_xor_sync(0xffffffffu, x, 16);
        if (g == 0) xm[warp * 8 + 2 * c + e] = make_float2(m[nt][e], x);
        float* y = xo + (warp * 8 + 2 * c + e) * Cfg::XL + g * (DP / 8);
#pragma unroll
        for (int i = 0; i < KS; i += 2)
          *reinterpret_cast<float4*>(y + 2 * i) =
              make_float4(o[i][nt][e], o[i][nt][e + 2], o[i + 1][nt][e], o[i + 1][nt][e + 2]);
      }
      __syncthreads();
      const int r = at.rb * ROWS + nt * 8 + warp;
      if (r < rows) {
        float M = -FLT_MAX, L = 0.f;
#pragma unroll
        for (int w = 0; w < CA_WARPS; ++w) M = fmaxf(M, xm[w * 8 + warp].x);
        float4 y = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
        for (int w = 0; w < CA_WARPS; ++w) {
          const float2 z = xm[w * 8 + warp];
          const float x = ex2(z.x - M);
          L = fmaf(x, z.y, L);
          if (lane < DP / 4) {
            const float4 v = *reinterpret_cast<const float4*>(xo + (w * 8 + warp) * Cfg::XL + lane * 4);
            y.x = fmaf(x, v.x, y.x);
            y.y = fmaf(x, v.y, y.y);
            y.z = fmaf(x, v.z, y.z);
            y.w = fmaf(x, v.w, y.w);
          }
        }
        if (complete) {
          const int t = r / a.rep;
          ca_write<E>(a, at.n, t, at.h * a.rep + (r - t * a.rep), M, L, y, lane);
        } else {
          const size_t part =
              ((size_t)2 * blockIdx.x + (tile0 == 0 && done > (uint32_t)tile1)) * ROWS + nt * 8 + warp;
          if (lane == 0) a.ml[part] = make_float2(M, L);
          if (lane < DP / 4) *reinterpret_cast<float4*>(a.po + part * DP + lane * 4) = y;
        }
      }
    }
    if (!complete) {
      // the item's places in the list, and the teams that have parts of it
      const uint32_t s0 = first + done - tile1, team0 = s0 / per, team1 = (s0 + at.tiles - 1) / per;
      const int head = blockIdx.x % a.team;
      auto part = [&](uint32_t t) { return 2 * ((size_t)t * a.team + head) + (t * per < s0); };
      __syncthreads();
      if (tid == 0) {
        __threadfence();
        uint32_t* left = a.left + part(team0);
        joins = atomicAdd(left, 1u) == team1 - team0;
        if (joins) *left = 0;                        // as it was, for the next call
        __threadfence();
      }
      __syncthreads();
      if (joins) {
        // a warp a row, or two where there are so few: then the second has every second four parts (38 parts of
        // 131,072 positions: 41.4 -> 39.0 us; eight or more in hand at a time cost the kernel its registers)
        const bool two = NT == 1 && rows <= CA_WARPS / 2 && team1 - team0 >= 4;
        const uint32_t step = two ? 8 : 4;
        for (int i = two ? warp % (CA_WARPS / 2) : warp; i < ROWS && at.rb * ROWS + i < rows; i += CA_WARPS) {
          float M = -FLT_MAX, L = 0.f;
          float4 y = make_float4(0.f, 0.f, 0.f, 0.f);
          for (uint32_t t0 = team0 + (two ? warp & 4 : 0); t0 <= team1; t0 += step) {   // four parts at a time
            float2 z[4];
            float4 v[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
              z[j] = make_float2(-FLT_MAX, 0.f);
              v[j] = make_float4(0.f, 0.f, 0.f, 0.f);
              if (t0 + j <= team1) {
                const size_t p = part(t0 + j) * ROWS + i;
                z[j] = __ldcg(&a.ml[p]);
                if (lane < DP / 4) v[j] = __ldcg(reinterpret_cast<const float4*>(a.po + p * DP + lane * 4));
              }
            }
            const float to = fmaxf(fmaxf(fmaxf(z[0].x, z[1].x), fmaxf(z[2].x, z[3].x)), M), x0 = ex2(M - to);
            M = to;
            L *= x0;
            y.x *= x0; y.y *= x0; y.z *= x0; y.w *= x0;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
              const float x = ex2(z[j].x - to);
              L = fmaf(x, z[j].y, L);
              y.x = fmaf(x, v[j].x, y.x);
              y.y = fmaf(x, v[j].y, y.y);
              y.z = fmaf(x, v[j].z, y.z);
              y.w = fmaf(x, v[j].w, y.w);
            }
          }
          if (two) {
            if (warp & 4) {
              xm[i] = make_float2(M, L);
              if (lane < DP / 4) *reinterpret_cast<float4*>(xo + i * Cfg::XL + lane * 4) = y;
            }
            named_barrier(1 + i, 64);
            if (warp & 4) break;
            const float2 z = xm[i];
            const float to = fmaxf(M, z.x), x0 = ex2(M - to), x1 = ex2(z.x - to);
            float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
            if (lane < DP / 4) v = *reinterpret_cast<const float4*>(xo + i * Cfg::XL + lane * 4);
            M = to;
            L = fmaf(x1, z.y, L * x0);
            y = make_float4(fmaf(x1, v.x, y.x * x0), fmaf(x1, v.y, y.y * x0), fmaf(x1, v.z, y.z * x0),
                            fmaf(x1, v.w, y.w * x0));
          }
          const int r = at.rb * ROWS + i, t = r / a.rep;
          ca_write<E>(a, at.n, t, at.h * a.rep + (r - t * a.rep), M, L, y, lane);
        }
      }
    }
    if (done == count) break;
    at.next(a, a.blocks);
    if constexpr (Sm::QS) __syncthreads();
  }
  copy_wait<0>();
}

// What each key gets, from the scores that the kernel left, against their rows' references and sums; a thread a
// key, and a block CS_KEYS keys of one kv head. Bytes bound it: 4 bytes a row and key written and read again, from L2
// where they are few, for 8 of the weight itself. 16 sequences of 8,192, 8 heads, 4 rows: 52 us with the attention,
// which alone takes 41.
constexpr int CS_KEYS = 512;
template <int PIECES>
__global__ void __launch_bounds__(256) cache_attention_spread_kernel(const CaArgs a, int pieces) {
  pdl_wait();
  __shared__ float4 row[16];                         // reference, 1 / sum, factor, what it lacks
  const int nh = blockIdx.x / pieces, k0 = (blockIdx.x - nh * pieces) * CS_KEYS;
  const int n = nh / a.c.H, h = nh - n * a.c.H, rows = a.T * a.rep, len = cache_len(a.seq_len[n], a.c.S);
  if (k0 >= len) return;
  const size_t base = ((size_t)n * a.c.H + h) * a.c.S;
  constexpr int PER = CS_KEYS / 256;
  float w[PER];
  float2 s[PER];                                     // the first two rows' products: asked for before the rows' sums
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    const int k = k0 + i * 256 + threadIdx.x;
    if (k < len) {
      w[i] = a.weights[base + k];
      s[i] = __ldcs(reinterpret_cast<const float2*>(a.scores + (base + k) * a.pad));
    }
  }
  if (threadIdx.x < a.pad) {
    float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
    if (threadIdx.x < rows) {
      const int t = threadIdx.x / a.rep;
      const size_t at = ((size_t)n * a.T + t) * a.Hq + h * a.rep + (threadIdx.x - t * a.rep);
      const float2 ml = a.rows[at];
      const float f = a.factors[at];
      // rows without keys, or without a finite sum, add nothing
      if (ml.y > 0.f && ml.y < INFINITY && fabsf(ml.x) < INFINITY)
        x = make_float4(CA_UP - ml.x, 1.f / ml.y, f, f * a.rest_ratio);
    }
    row[threadIdx.x] = x;
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    const int k = k0 + i * 256 + threadIdx.x;
    if (k >= len) break;
    float sum = 0.f;
    for (int r = 0; r < a.pad; r += 2) {
      float2 next = s[i];
      if (r + 2 < a.pad) next = __ldcs(reinterpret_cast<const float2*>(a.scores + (base + k) * a.pad + r + 2));
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const float4 x = row[r + e];
        const float v = e ? s[i].y : s[i].x;
        if (x.y > 0.f && v > -INFINITY) {            // (a row that may not see the key has -infinity there)
          float t = x.x;
          if (PIECES > 1) t = fmaf(v, x.w, t);
          sum = fmaf(ex2(fmaf(v, x.z, t)), x.y, sum);
        }
      }
      s[i] = next;
    }
    a.weights[base + k] = w[i] + sum;
  }
}

// The same for more rows of fp32 queries than scores are kept for: computed once more, a warp 16 keys; rows go
// through shared memory 8 NT at a time, and each key's weight is read and written by one lane, once for each
// 8 NT rows. (bf16: cache_attention_tc_weights.cu.)
template <int DP, int DIM>
__global__ void __launch_bounds__(CA_THREADS, 2) cache_attention_weights_kernel(const CaArgs a) {
  pdl_wait();
  using E = float;
  constexpr int NT = 1, PIECES = 3, KS = CaCfg<DP>::KS, ST = 4, ROWS = 8 * NT, STAGE = 16 * (DP / 2 + 16);
  constexpr int KEYS = 16 * CA_WARPS;
  extern __shared__ __align__(16) unsigned char sm[];
  uint2* qs = reinterpret_cast<uint2*>(sm + CA_WARPS * ST * STAGE);      // [NT][PIECES][KS][lane]
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, g = lane >> 2, c = lane & 3;
  const int d = DIM ? DIM : a.c.d, R = (cache_half_bytes(d) + 15) / 16 * 16, rows = a.T * a.rep;
  CaCursor<KEYS> at;
  uint32_t first, per;
  uint32_t count = ca_range<KEYS>(a, 1, &at, &first, &per);
  const CaLane<DP> mine(a, R, lane);
  unsigned char* stage = sm + warp * ST * STAGE;
  const int key = key_of(g);
  const uint32_t kmask = key_scale_mask<DP>(d, c);
  while (count > 0) {
    const int tile0 = at.tile, tile1 = min((uint32_t)at.tiles, tile0 + count);
    for (int r0 = 0; r0 < rows; r0 += ROWS) {
      __syncthreads();
      float f[NT][2], fr[NT][2], ref[NT][2], inv[NT][2];
      int lim[NT][2];
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
        const int r = r0 + nt * 8 + g, t = r / a.rep, hq = at.h * a.rep + (r - t * a.rep);
        float2 ml = make_float2(0.f, 0.f);
        if (r < rows) ml = a.rows[((size_t)at.n * a.T + t) * a.Hq + hq];
        // rows without keys, or without a finite sum, add nothing
        const bool there = ml.y > 0.f && ml.y < INFINITY && fabsf(ml.x) < INFINITY;
        uint32_t qb[PIECES][KS][2];
        const int up = load_query<DP, PIECES, E>(
            there ? static_cast<const E*>(a.q) + at.n * a.q_s[0] + t * a.q_s[1] + hq * a.q_s[2] : nullptr, d, c,
            qb);
        if (warp == nt % CA_WARPS)
#pragma unroll
          for (int p = 0; p < PIECES; ++p)
#pragma unroll
            for (int i = 0; i < KS; ++i)
              qs[((nt * PIECES + p) * KS + i) * 32 + lane] = make_uint2(qb[p][i][0], qb[p][i][1]);
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const int col = 2 * c + e, rr = r0 + nt * 8 + col;
          const int u = __shfl_sync(0xffffffffu, up, col * 4);
          const float m = __shfl_sync(0xffffffffu, ml.x, col * 4);
          const bool ok = __shfl_sync(0xffffffffu, there, col * 4);
          const float l = __shfl_sync(0xffffffffu, ml.y, col * 4);
          f[nt][e] = row_factor(a, u);
          fr[nt][e] = a.scale_rest * pow2(-u);
          ref[nt][e] = CA_UP - m;
          inv[nt][e] = 1.f / l;
          lim[nt][e] = ok ? max(0, at.seen(a, rr / a.rep)) : 0;
        }
      }
      int ahead = tile0;
      auto copy_next = [&] {
        if (ahead < tile1)
          mine.copy(a, a.c.at(at.n, ahead * KEYS + warp * 16, at.h), at.len - (ahead * KEYS + warp * 16),
                    smem_u32(stage + ahead % ST * STAGE), lane);
        ++ahead;
        copy_commit();
      };
#pragma unroll
      for (int i = 0; i < ST - 1; ++i) copy_next();
      __syncthreads();
      for (int tile = tile0; tile < tile1; ++tile) {
        copy_wait<ST - 2>();
        __syncwarp();
        const int k0 = tile * KEYS + warp * 16;
        float s[NT][4];
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) s[nt][0] = s[nt][1] = s[nt][2] = s[nt][3] = 0.f;
        CaKeyPart<DP> kp;
        kp.load(stage + tile % ST * STAGE + key * R, R, d, c, kmask);
        auto step = [&](auto ks) {
          constexpr int i = decltype(ks)::value;
          uint32_t ka[2][4];
          kp.template operands<i>(ka);
#pragma unroll
          for (int j = 0; j < 2; ++j)
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
              for (int p = PIECES - 1; p >= 0; --p) {
                const uint2 b = qs[((nt * PIECES + p) * KS + 2 * i + j) * 32 + lane];
                mma(s[nt], ka[j], b.x, b.y);
              }
        };
        steps(step, std::make_integer_sequence<int, KS / 2>{});
        float sum[2] = {0.f, 0.f};
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            float x = ref[nt][e & 1];
            if (PIECES > 1) x = fmaf(s[nt][e], fr[nt][e & 1], x);
            const float p = ex2(fmaf(s[nt][e], f[nt][e & 1], x));
            if (k0 + key + (e >> 1) < lim[nt][e & 1]) sum[e >> 1] = fmaf(p, inv[nt][e & 1], sum[e >> 1]);
          }
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          sum[e] += __shfl_xor_sync(0xffffffffu, sum[e], 1);
          sum[e] += __shfl_xor_sync(0xffffffffu, sum[e], 2);
        }
        if (c < 2 && k0 + key + c < at.len)
          a.weights[((size_t)at.n * a.c.H + at.h) * a.c.S + k0 + key + c] += c ? sum[1] : sum[0];
        __syncwarp();
        copy_next();
      }
      copy_wait<0>();
    }
    count -= tile1 - tile0;
    if (count > 0) {
      at.next(a, 1);
    }
  }
}

// What each key gets, behind the rows' results.
template <int DP, int DIM, int PIECES>
lilicorr_status_t ca_launch_weights(const CaArgs& a, const CaPlan& p, cudaStream_t st) {
  if (!a.weights || a.c.S == 0) return LILICORR_OK;
  if (a.scores) {
    const int pieces = (a.c.S + CS_KEYS - 1) / CS_KEYS;
    return launch_k(cache_attention_spread_kernel<PIECES>, (unsigned)(a.c.N * a.c.H * pieces), 256, 0, st, a, pieces);
  }
  if constexpr (PIECES == 1) {
    return launch_ca_tc_weights(a, p, st);
  } else {
    static bool configured[64] = {false};
    auto* weights = cache_attention_weights_kernel<DP, DIM>;
    LL_TRY(allow_max_dynamic_smem(weights, configured));
    const size_t smem = CA_WARPS * 4 * 16 * (DP / 2 + 16) + 3 * (DP / 16) * 256;
    return launch_k(weights, (unsigned)(2 * num_sms() / p.team * p.team), CA_THREADS, smem, st, a);
  }
}

template <int DP, int DIM, int NT, int PIECES, typename E>
lilicorr_status_t ca_launch(const CaArgs& a, const CaPlan& p, cudaStream_t st) {
  static bool configured[64] = {false};
  auto* kernel = cache_attention_kernel<DP, DIM, NT, PIECES, E>;
  LL_TRY(allow_max_dynamic_smem(kernel, configured));
  LL_TRY(launch_k(kernel, p.whole ? (unsigned)p.items : (unsigned)p.ctas, CA_THREADS,
                  CaSmem<DP, NT, PIECES>::TOTAL, st, a));
  return ca_launch_weights<DP, DIM, PIECES>(a, p, st);
}

}  // namespace

template <int DP, int DIM>
lilicorr_status_t ca_launch_rows(const CaArgs& a, const CaPlan& p, cudaStream_t st) {
  if (p.pieces > 1)
    return p.nt == 1 ? ca_launch<DP, DIM, 1, 3, float>(a, p, st) : ca_launch<DP, DIM, 2, 3, float>(a, p, st);
  if (p.tc) {
    LL_TRY(launch_ca_tc(a, p, st));
    return ca_launch_weights<DP, DIM, 1>(a, p, st);
  }
  return p.nt == 1   ? ca_launch<DP, DIM, 1, 1, __nv_bfloat16>(a, p, st)
         : p.nt == 2 ? ca_launch<DP, DIM, 2, 1, __nv_bfloat16>(a, p, st)
                     : ca_launch<DP, DIM, 4, 1, __nv_bfloat16>(a, p, st);
}

}  // namespace lilicorr
