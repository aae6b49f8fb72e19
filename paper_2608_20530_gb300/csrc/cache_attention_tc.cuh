// Attention over a cache held in 4 bits on the 5th-generation tensor cores: what its kernels have in common.
#pragma once
#include "cache_attention_kernels.cuh"
#include "tc_ptx.cuh"

namespace lilicorr {
namespace {
using namespace tc;

constexpr int CT_KEYS = 128, CT_ROWS = 128;
constexpr uint32_t CT_CHUNK = 128 * 128;             // 128 rows of 128 bytes

// fp16 operands, fp32 sums
__host__ __device__ constexpr uint32_t instr_desc_f16(int m, int n) {
  return (1u << 4) | ((uint32_t)(n >> 3) << 17) | ((uint32_t)(m >> 4) << 24);
}
__device__ __forceinline__ bool elect_one() {        // one lane of a converged warp
  uint32_t r;
  asm volatile("{\n .reg .pred p;\n elect.sync _|p, 0xffffffff;\n selp.u32 %0, 1, 0, p;\n}" : "=r"(r));
  return r != 0;
}
// packed fp32 pairs: one instruction for both halves
__device__ __forceinline__ uint64_t pair_of(float lo, float hi) {
  uint64_t r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(lo), "f"(hi));
  return r;
}
__device__ __forceinline__ void halves(uint64_t v, float& lo, float& hi) {
  asm("mov.b64 {%0, %1}, %2;" : "=f"(lo), "=f"(hi) : "l"(v));
}
__device__ __forceinline__ uint64_t fma_pair(uint64_t a, uint64_t b, uint64_t c) {
  uint64_t d;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(d) : "l"(a), "l"(b), "l"(c));
  return d;
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

// shared memory by its address (which ring a pointer is in is not known where it is compiled)
__device__ __forceinline__ uint2 lds8(uint32_t at) {
  uint2 v;
  asm volatile("ld.shared.v2.u32 {%0, %1}, [%2];" : "=r"(v.x), "=r"(v.y) : "r"(at) : "memory");
  return v;
}
__device__ __forceinline__ void sts16(uint32_t at, uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
  asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(at), "r"(a), "r"(b), "r"(c), "r"(d) : "memory");
}

// Half a record at `rec` (or zeros) as row `key` of a tile: DP columns of fp16, zeros past the head's width.
template <int DP, int DIM>
__device__ __forceinline__ void expand(uint32_t rec, bool there, int d, uint32_t tile, int key) {
  // Everything is read first: the place may be given back while it is expanded. Records of 144 bytes start at every
  // second pair of banks, so keys of the upper half of 16 read their groups in another order than the lower.
  const int turn = DIM ? key >> 3 & 1 : 0;
  uint2 w[DP / 16], b = lds8(rec + d / 2);
#pragma unroll
  for (int g = 0; g < DP / 16; ++g) {
    w[g] = make_uint2(0, 0);
    if (DIM || g * 16 < d) w[g] = lds8(rec + (g ^ turn) * 8);
  }
  // scales of 0 where there is no key (codes are finite whatever they are), or no such group
  if (!there) b = make_uint2(0, 0);
  const uint32_t row = tile + key * 128, x = key & 7;
#pragma unroll
  for (int g = 0; g < DP / 16; ++g) {
    const uint32_t two = __byte_perm(b.x, b.y, ((g & 7) ^ turn) * 0x11), f = scales(DIM || g * 16 < d ? two : 0u);
    uint32_t r[4];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const uint32_t p = 2 * (g ^ turn) + i;
      codes(i ? w[g].y : w[g].x, r);
      sts16(row + (2 * g + i >> 3) * CT_CHUNK + (((p & 7) ^ x) << 4), mul2(r[0], f), mul2(r[1], f), mul2(r[2], f),
            mul2(r[3], f));
    }
  }
}

}  // namespace
}  // namespace lilicorr
