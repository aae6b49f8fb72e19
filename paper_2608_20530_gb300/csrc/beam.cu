// Beam search: the n best (beam, token) pairs of each request, and the beams' states moved to the
// beams that continue them.
//
// Selection. A request's answer is among its beams' n best tokens each (in a beam the order of
// totals is the order of logits), so the pass over the logits is the top-K pass of topk_lse.cu with
// normalisers in 64 bits, and what remains is the n largest of W * n totals. Totals are double sums:
// beams whose totals differ by less than an fp32 rounding of either normaliser are still told apart,
// and the order does not depend on how a row was split.
#include <math.h>

#include "internal.cuh"

namespace lilicorr {

namespace {

constexpr int BM_THREADS = 128;
constexpr int BM_CAND = LILICORR_MAX_BEAMS * LILICORR_MAX_K;

// Order-preserving image of a double that is not NaN; 0 is never one (it marks "no candidate").
__device__ __forceinline__ uint64_t ord64(double v) {
  const uint64_t b = (uint64_t)__double_as_longlong(v + 0.0);      // -0 to +0
  return (b >> 63) ? ~b : (b | (1ull << 63));
}
__device__ __forceinline__ double unord64(uint64_t o) {
  return __longlong_as_double((long long)((o >> 63) ? (o & ~(1ull << 63)) : ~o));
}

struct BeamPick {
  int W, K, n;
  const float* scores;
  const uint8_t* done;
  int32_t end_id;
  // candidates: lists (ids, logp), or the records of launch_beam_rows
  const int32_t* ids;
  const float* logp;
  const unsigned char* records;
  int32_t *tokens, *parents;
  float* next_scores;
  uint8_t* next_done;
  uint32_t* status;
};

// a precedes b: larger total, then lower position
__device__ __forceinline__ bool precedes(uint64_t ka, int pa, uint64_t kb, int pb) {
  return ka > kb || (ka == kb && pa < pb);
}

// One CTA a request. Each thread's best candidate first: the n-th of those bounds the answer from
// below, so that only the few candidates at or above it are ranked against one another.
__global__ void __launch_bounds__(BM_THREADS)
beam_pick_kernel(const BeamPick a) {
  pdl_wait();
  __shared__ uint64_t s_key[BM_CAND];
  __shared__ uint64_t s_best[BM_THREADS];
  __shared__ int s_at[BM_THREADS];
  __shared__ uint64_t s_bound;
  __shared__ int s_bound_at, s_count;
  __shared__ int s_surv[BM_CAND];
  const int tid = threadIdx.x, r = blockIdx.x;
  const int M = a.W * a.K;
  const float* scores = a.scores + (size_t)r * a.W;
  const uint8_t* done = a.done ? a.done + (size_t)r * a.W : nullptr;

  uint64_t best = 0ull;
  int best_at = 0;
  bool bad = false;
  for (int i = tid; i < M; i += BM_THREADS) {
    const int w = i / a.K, k = i - w * a.K;
    const float sc = scores[w];
    double total = -INFINITY;
    if (done && done[w]) {
      if (k == 0) total = (double)sc;
    } else if (sc != -INFINITY) {
      const size_t row = (size_t)r * a.W + w;
      if (a.records) {
        const unsigned char* rec = a.records + row * beam_record_bytes(a.K);
        const float* vals = reinterpret_cast<const float*>(rec + 8);
        // a row without a finite normaliser has set the status already
        const double lse = *reinterpret_cast<const double*>(rec);
        if (isfinite(lse) && reinterpret_cast<const int32_t*>(vals)[a.K + k] >= 0)
          total = (double)sc + ((double)vals[k] - lse);
      } else {
        total = (double)sc + (double)a.logp[row * a.K + k];
      }
    }
    uint64_t key = 0ull;
    if (!(total < INFINITY)) bad = true;               // NaN or +inf
    else if (total > -INFINITY) key = ord64(total);
    s_key[i] = key;
    if (key > best) { best = key; best_at = i; }
  }
  if (bad) set_status(a.status, LILICORR_ERR_NONFINITE);
  s_best[tid] = best;
  s_at[tid] = best_at;
  if (tid == 0) { s_bound = 1ull; s_bound_at = BM_CAND; s_count = 0; }
  __syncthreads();
  if (best) {
    int rank = 0;
    for (int j = 0; j < BM_THREADS; ++j) rank += precedes(s_best[j], s_at[j], best, best_at) ? 1 : 0;
    if (rank == a.n - 1) { s_bound = best; s_bound_at = best_at; }
  }
  __syncthreads();
  const uint64_t bound = s_bound;
  const int bound_at = s_bound_at;
  for (int i = tid; i < M; i += BM_THREADS)
    if (!precedes(bound, bound_at, s_key[i], i)) s_surv[atomicAdd(&s_count, 1)] = i;
  __syncthreads();
  const int count = s_count;
  for (int i = tid; i < count; i += BM_THREADS) {
    const int at = s_surv[i];
    const uint64_t key = s_key[at];
    int rank = 0;
    for (int j = 0; j < count; ++j) {
      const int o = s_surv[j];
      rank += precedes(s_key[o], o, key, at) ? 1 : 0;
    }
    if (rank >= a.n) continue;
    const int w = at / a.K, k = at - w * a.K;
    const bool over = done && done[w];
    const size_t row = (size_t)r * a.W + w, dst = (size_t)r * a.n + rank;
    int32_t token = a.end_id;
    if (!over)
      token = a.records ? reinterpret_cast<const int32_t*>(
                              a.records + row * beam_record_bytes(a.K) + 8)[a.K + k]
                        : a.ids[row * a.K + k];
    a.tokens[dst] = token;
    a.parents[dst] = w;
    a.next_scores[dst] = (float)unord64(key);
    if (a.next_done) a.next_done[dst] = over || (a.end_id >= 0 && token == a.end_id);
  }
  for (int i = count + tid; i < a.n; i += BM_THREADS) {      // fewer than n candidates
    const size_t dst = (size_t)r * a.n + i;
    a.tokens[dst] = -1;
    a.parents[dst] = -1;
    a.next_scores[dst] = -INFINITY;
    if (a.next_done) a.next_done[dst] = 0;
  }
}

// ---------------------------------------------------------------------------- states
constexpr int BR_THREADS = 256;
constexpr int BR_STATES = 64;            // arrays per launch

struct Reorder {
  unsigned char* state[BR_STATES];
  int W, positions, heads;
  uint32_t pieces;                       // vectors per row
  int64_t s_req, s_beam, s_pos, s_head;
  const int32_t* parents;
  const int32_t* lengths;
};

// One (array, request) per grid row. A thread owns one vector-wide column of all W beams: it loads
// every beam that moves from its parent, then stores, so the move is in place without a second
// buffer and without a barrier: nobody else reads or writes its column.
template <typename V, int WMAX>
__global__ void __launch_bounds__(BR_THREADS)
beam_reorder_kernel(const __grid_constant__ Reorder a) {
  pdl_wait();
  __shared__ int s_parent[LILICORR_MAX_BEAMS];
  const int tid = threadIdx.x, r = blockIdx.y;
  if (tid < a.W) {
    const int p = a.parents[(size_t)r * a.W + tid];
    s_parent[tid] = (p < 0 || p >= a.W) ? tid : p;
  }
  __syncthreads();
  int len = a.positions;
  if (a.lengths) len = min(max(a.lengths[r], 0), a.positions);
  const uint32_t per_pos = (uint32_t)a.heads * a.pieces, total = (uint32_t)len * per_pos;
  unsigned char* base = a.state[blockIdx.z] + (int64_t)r * a.s_req;
  for (uint32_t u = blockIdx.x * BR_THREADS + tid; u < total; u += gridDim.x * BR_THREADS) {
    const uint32_t pos = u / per_pos, in = u - pos * per_pos, h = in / a.pieces, c = in - h * a.pieces;
    unsigned char* col = base + (int64_t)pos * a.s_pos + (int64_t)h * a.s_head + (int64_t)c * sizeof(V);
    V v[WMAX];
#pragma unroll
    for (int w = 0; w < WMAX; ++w)
      if (w < a.W && s_parent[w] != w)
        v[w] = *reinterpret_cast<const V*>(col + (int64_t)s_parent[w] * a.s_beam);
#pragma unroll
    for (int w = 0; w < WMAX; ++w)
      if (w < a.W && s_parent[w] != w) *reinterpret_cast<V*>(col + (int64_t)w * a.s_beam) = v[w];
  }
}

template <typename V>
lilicorr_status_t launch_reorder(const Reorder& a, int count, int requests, cudaStream_t st) {
  // CTAs for about four waves over all (array, request) pairs; the rest by the loop
  const long long most = (long long)a.positions * a.heads * a.pieces;
  const long long pairs = (long long)count * requests;
  long long x = (most + BR_THREADS - 1) / BR_THREADS;
  const long long want = (16ll * num_sms() + pairs - 1) / pairs;
  if (x > want) x = want;
  if (x < 1) x = 1;
  const dim3 grid((unsigned)x, (unsigned)requests, (unsigned)count);
  if (a.W <= 4) return launch_k(beam_reorder_kernel<V, 4>, grid, BR_THREADS, 0, st, a);
  if (a.W <= 8) return launch_k(beam_reorder_kernel<V, 8>, grid, BR_THREADS, 0, st, a);
  if (a.W <= 16) return launch_k(beam_reorder_kernel<V, 16>, grid, BR_THREADS, 0, st, a);
  if constexpr (sizeof(V) <= 8)
    if (a.W <= 32) return launch_k(beam_reorder_kernel<V, 32>, grid, BR_THREADS, 0, st, a);
  if constexpr (sizeof(V) <= 4)
    return launch_k(beam_reorder_kernel<V, 64>, grid, BR_THREADS, 0, st, a);
  return LILICORR_ERR_SHAPE;
}

bool beam_shape_ok(int requests, int beams, int n) {
  return requests >= 0 && beams >= 1 && beams <= LILICORR_MAX_BEAMS && n >= 1 && n <= LILICORR_MAX_K;
}

}  // namespace
}  // namespace lilicorr

using namespace lilicorr;

extern "C" {

size_t lilicorr_beam_select_workspace_bytes(int requests, int beams, int V, int n) {
  if (!beam_shape_ok(requests, beams, n) || V <= 0 || n > (long long)beams * V) return 0;
  const long long rows = (long long)requests * beams;
  if (rows > 65535) return 0;
  const int K = n < V ? n : V;
  const size_t a = beam_rows_ws_bytes((int)rows, V, K, LILICORR_F32);
  const size_t b = beam_rows_ws_bytes((int)rows, V, K, LILICORR_BF16);
  return 256 + align_up((size_t)rows * beam_record_bytes(K), 256) + (a > b ? a : b);
}

lilicorr_status_t lilicorr_beam_select(const void* logits, lilicorr_dtype_t dtype, int requests,
                                       int beams, int V, int n, const float* scores,
                                       const uint8_t* done, int32_t end_id, int32_t* tokens,
                                       int32_t* parents, float* next_scores, uint8_t* next_done,
                                       void* ws, size_t ws_bytes, cudaStream_t stream) {
  if (dtype != LILICORR_F32 && dtype != LILICORR_BF16) return LILICORR_ERR_DTYPE;
  const size_t need = lilicorr_beam_select_workspace_bytes(requests, beams, V, n);
  if (need == 0) return LILICORR_ERR_SHAPE;
  if (end_id < -1 || end_id >= V || (done && end_id < 0)) return LILICORR_ERR_ARG;
  if (requests == 0) return LILICORR_OK;
  if (!logits || !scores || !tokens || !parents || !next_scores || !ws) return LILICORR_ERR_ARG;
  if (!aligned16(logits) || !aligned16(ws)) return LILICORR_ERR_ARG;
  if (ws_bytes < need) return LILICORR_ERR_WORKSPACE;
  const int rows = requests * beams, K = n < V ? n : V;
  unsigned char* w = static_cast<unsigned char*>(ws);
  unsigned char* records = w + 256;
  uint32_t* status = reinterpret_cast<uint32_t*>(w);
  LL_TRY(launch_beam_rows(logits, dtype, rows, V, K, scores, done, records, status,
                          records + align_up((size_t)rows * beam_record_bytes(K), 256), stream));
  const BeamPick a{beams, K, n, scores, done, end_id, nullptr, nullptr, records,
                   tokens, parents, next_scores, next_done, status};
  return launch_k(beam_pick_kernel, requests, BM_THREADS, 0, stream, a);
}

lilicorr_status_t lilicorr_beam_merge(const int32_t* ids, const float* logp, int requests, int beams,
                                      int K, int n, const float* scores, const uint8_t* done,
                                      int32_t end_id, int32_t* tokens, int32_t* parents,
                                      float* next_scores, uint8_t* next_done, uint32_t* status,
                                      cudaStream_t stream) {
  if (!beam_shape_ok(requests, beams, n) || K < 1 || K > LILICORR_MAX_K || n > beams * K)
    return LILICORR_ERR_SHAPE;
  if (end_id < -1 || (done && end_id < 0)) return LILICORR_ERR_ARG;
  if (requests == 0) return LILICORR_OK;
  if (!ids || !logp || !scores || !tokens || !parents || !next_scores) return LILICORR_ERR_ARG;
  const BeamPick a{beams, K, n, scores, done, end_id, ids, logp, nullptr,
                   tokens, parents, next_scores, next_done, status};
  return launch_k(beam_pick_kernel, requests, BM_THREADS, 0, stream, a);
}

lilicorr_status_t lilicorr_beam_reorder(void* const* host_states, int n_states, int requests,
                                        int beams, int positions, int heads, size_t row_bytes,
                                        int64_t stride_request, int64_t stride_beam,
                                        int64_t stride_position, int64_t stride_head,
                                        const int32_t* parents, const int32_t* lengths,
                                        cudaStream_t stream) {
  if (n_states < 0 || requests < 0 || requests > 65535 || positions < 0 || heads < 0 || beams < 1 ||
      beams > LILICORR_MAX_BEAMS)
    return LILICORR_ERR_SHAPE;
  if (n_states == 0 || requests == 0 || positions == 0 || heads == 0 || row_bytes == 0)
    return LILICORR_OK;
  if (!host_states || !parents) return LILICORR_ERR_ARG;
  if (row_bytes > (1ull << 31) || (double)positions * heads * (double)row_bytes >= 16.0 * 2147483648.0)
    return LILICORR_ERR_SHAPE;
  // heads that follow one another are one longer row
  if (heads > 1 && stride_head == (int64_t)row_bytes) {
    row_bytes *= heads;
    heads = 1;
  }
  // the widest vector that every row starts at and fills, and that W beams leave registers for
  uint64_t bits = row_bytes | (requests > 1 ? (uint64_t)stride_request : 0) |
                  (beams > 1 ? (uint64_t)stride_beam : 0) |
                  (positions > 1 ? (uint64_t)stride_position : 0) |
                  (heads > 1 ? (uint64_t)stride_head : 0);
  for (int i = 0; i < n_states; ++i) {
    if (!host_states[i]) return LILICORR_ERR_ARG;
    bits |= reinterpret_cast<uintptr_t>(host_states[i]);
  }
  int vec = beams <= 16 ? 16 : beams <= 32 ? 8 : 4;
  while (bits & (uint64_t)(vec - 1)) vec >>= 1;
  if ((double)positions * heads * (double)(row_bytes / vec) >= 2147483648.0) return LILICORR_ERR_SHAPE;
  Reorder a;
  a.W = beams;
  a.positions = positions;
  a.heads = heads;
  a.pieces = (uint32_t)(row_bytes / vec);
  a.s_req = stride_request;
  a.s_beam = stride_beam;
  a.s_pos = stride_position;
  a.s_head = stride_head;
  a.parents = parents;
  a.lengths = lengths;
  for (int i0 = 0; i0 < n_states; i0 += BR_STATES) {
    const int count = n_states - i0 < BR_STATES ? n_states - i0 : BR_STATES;
    for (int i = 0; i < BR_STATES; ++i)
      a.state[i] = i < count ? static_cast<unsigned char*>(host_states[i0 + i]) : nullptr;
    switch (vec) {
      case 16: LL_TRY(launch_reorder<uint4>(a, count, requests, stream)); break;
      case 8: LL_TRY(launch_reorder<uint2>(a, count, requests, stream)); break;
      case 4: LL_TRY(launch_reorder<uint32_t>(a, count, requests, stream)); break;
      case 2: LL_TRY(launch_reorder<uint16_t>(a, count, requests, stream)); break;
      default: LL_TRY(launch_reorder<uint8_t>(a, count, requests, stream)); break;
    }
  }
  return LILICORR_OK;
}

}  // extern "C"
