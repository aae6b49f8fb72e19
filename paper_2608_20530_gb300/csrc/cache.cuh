// A decoding cache held in 4 bits: records, their checks, and what the kernels on them have in common.
#pragma once
#include "internal.cuh"

namespace lilicorr {

// A record: key codes [d / 2], key scales [8], value codes [d / 2], value scales [8] (see lilicorr.h).
__host__ __device__ constexpr int cache_half_bytes(int d) { return d / 2 + 8; }
__host__ __device__ constexpr int cache_record_bytes(int d) { return d + 16; }

// The records as kernels get them: strides in bytes, 0 for a dimension of one.
struct CacheView {
  unsigned char* p;
  int64_t s[3];                // sequence, position, head
  int N, S, H, d;              // sequences, capacity, kv heads, head_dim
  float k_unit, v_unit;
  __device__ __forceinline__ unsigned char* at(int n, int pos, int h) const {
    return p + (n * s[0] + pos * s[1] + h * s[2]);
  }
};

// Shapes and units (ERR_SHAPE, ERR_ARG), then the pointer and the strides; `written`: no two records overlap.
lilicorr_status_t cache_shape(const lilicorr_cache_desc* d);
lilicorr_status_t cache_view(const lilicorr_cache_desc* d, const void* cache, bool written, CacheView* v);
// Rows [e0, e1, e2] of `row` units at these strides: multiples of per16, not negative, disjoint if `written`.
bool cache_rows_ok(const int64_t* s, const int64_t (&e)[3], int per16, int row, bool written);

// min(max(len, 0), S)
__device__ __forceinline__ int cache_len(int len, int S) { return min(max(len, 0), S); }

}  // namespace lilicorr
