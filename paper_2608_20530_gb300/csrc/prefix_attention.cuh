// Attention of sequences that share their request's prefix: what its kernels have in common.
#pragma once
#include <cuda.h>

#include "internal.cuh"


namespace lilicorr {

// One side of the keys: the prefix of each group (shared by its sequences), or each sequence's own.
struct PaKeys {
  const void* k;
  const void* v;
  int64_t k_s[3], v_s[3];      // strides in elements: group or sequence, position, head
  const int32_t* len;          // [groups] or [sequences]
  int capacity;
  int splits;                  // pieces that each key range is cut into
  int slot0;                   // first partial slot
  int own;                     // 0: prefix, 1: the sequences' own keys (causal over the T tokens)
  int join;                    // the kernel of these keys writes the result
  int behind;                  // the launch before it is the prefix's of the same call
  int front;                   // the prefix's keys come first in its own walk
  const void* front_k;
  const void* front_v;
  int64_t front_k_s[3], front_v_s[3];
  const int32_t* front_len;    // [groups]
  int front_capacity;
};

struct PaArgs {
  const void* q;
  int64_t q_s[3];              // sequence, token, head
  void* out;
  int64_t o_s[3];
  float* lse;                  // [N, T, Hq]
  const int32_t* seq_len;      // [N]
  int G, W, T, Hq, Hkv, rep, d;
  float scale_log2;            // scale * log2(e): scores in log2 units
  float scale_rest;            // what its rounding left
  // partial results of a piece of the keys: (maximum, sum of 2^(s - maximum)) and the sums of
  // 2^(s - maximum) V, fp32; a sum of 0: no keys, and no sums of V were written
  int slots;                   // pieces per row that are kept by row
  float2* ml;                  // [slots][rows]
  float* po;                   // [slots][rows][d]
  // the prefix's pieces of the tensor-core kernel, kept by segment (PaSegments)
  int seg_ctas;                // its CTAs (0: the prefix's pieces are among the slots)
  int seg_blocks;              // blocks of PA_BLOCK rows per (group, key head)
  int seg_rows;                // rows per (group, key head)
  float2* seg_ml;              // [segments][PA_BLOCK]
  float* seg_po;               // [segments][PA_BLOCK][d]
  uint32_t* seg_start;         // [G + 1] tiles before each group (of one key head and row block)
  uint32_t* status;
  long long wait_limit;        // SM cycles per bounded wait of the tensor-core kernel
  int test_starve;             // test hook only: it issues no copies of K (1) or V (2)
  __device__ __host__ size_t rows() const { return (size_t)G * W * T * Hq; }
};

// The tensor-core kernel's work is the list of all (group, key head, block of PA_BLOCK rows, tile of
// PA_TILE keys), in that order, cut evenly among its CTAs: CTA b takes tiles [b * per, (b + 1) * per). A
// segment is what one CTA has of one (group, key head, block) = item; its number is CTA + item, which
// no other segment has, the list being walked in order. A block of 128 rows or fewer leaves two pieces a
// segment, the second in the places of the rows from 128 on.
constexpr int PA_BLOCK = 256;
constexpr int PA_TILE = 128;
// At least two tiles of a CTA, so that short lists leave fewer segments to join: 8 heads of 2,048 keys, 64
// rows, 21.5 -> 18.8 us (four at least: 19.3); from about 300 tiles on there is no difference.
constexpr int PA_MIN_TILES = 2;
__host__ __device__ __forceinline__ uint32_t pa_per_cta(uint32_t tiles, int ctas) {
  const uint32_t per = (tiles + ctas - 1) / ctas;
  return per < PA_MIN_TILES ? PA_MIN_TILES : per;
}

constexpr long long PA_WAIT = 4000000000ll;          // about 2 s

// Rows that share a key range: (sequence of the group, token, query head of the key head), in that
// order. Row r of (group or sequence b, key head h) as (sequence, token, query head).
struct PaRow { int n, t, h; };
__device__ __forceinline__ PaRow pa_row(const PaArgs& a, int own, int b, int hk, int r) {
  const int per = a.T * a.rep, w = own ? 0 : r / per, in = own ? r : r - w * per;
  PaRow x;
  x.n = own ? b : b * a.W + w;
  x.t = in / a.rep;
  x.h = hk * a.rep + (in - x.t * a.rep);
  return x;
}
__device__ __forceinline__ size_t pa_index(const PaArgs& a, const PaRow& x) {
  return ((size_t)x.n * a.T + x.t) * a.Hq + x.h;
}
// Piece `split` of a key range of length len: [k0, k1), starts at multiples of 64.
__device__ __forceinline__ void pa_piece(int len, int splits, int split, int& k0, int& k1) {
  const int chunk = ((len + splits - 1) / splits + 63) / 64 * 64;
  k0 = min((long long)len, (long long)split * chunk);
  k1 = min((long long)len, (long long)k0 + chunk);
}
__device__ __forceinline__ float pa_ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

// the prefix on the 5th-generation tensor cores (prefix_attention_tc.cu): false where the driver makes no
// tensor maps of these keys (an expanded dimension)
struct PaMaps {
  CUtensorMap k, v;
  int copies;                  // of a tile
};
bool pa_tc_maps(const PaArgs& a, const PaKeys& k, PaMaps* maps);
lilicorr_status_t launch_pa_tc(const PaArgs& a, const PaKeys& k, const PaMaps& maps, cudaStream_t st);
lilicorr_status_t launch_pa_mma(const PaArgs& a, const PaKeys& k, cudaStream_t st);
lilicorr_status_t launch_pa_simt(const PaArgs& a, const PaKeys& k, cudaStream_t st);
lilicorr_status_t launch_pa_combine(const PaArgs& a, lilicorr_dtype_t dt, cudaStream_t st);

}  // namespace lilicorr
