// Attention over a cache held in 4 bits: what its kernels and the call have in common.
#pragma once
#include "cache.cuh"

namespace lilicorr {

struct CaArgs {
  CacheView c;
  const void* q;
  int64_t q_s[3];              // elements: sequence, token, head
  void* out;
  int64_t o_s[3];
  float* lse;                  // [N, T, Hq]
  const int32_t* seq_len;
  float* weights;              // [N, H, S] or null
  int T, Hq, rep;
  int blocks;                  // row blocks of a (sequence, kv head)
  int team;                    // CTAs that take the same tiles, of as many kv heads; divides H
  int whole;                   // a CTA an item (else the list of all tiles is cut evenly)
  float scale;                 // scale * k_unit * log2(e): scores in log2 units
  float scale_rest;            // what its rounding left
  float rest_ratio;            // scale_rest / scale
  uint32_t* left;              // [2 * CTAs] parts that an item's CTAs have left; 0 between calls
  float2* ml;                  // [2 * CTAs][rows of a block]: reference and sum of an item's part
  float* po;                   // [2 * CTAs][rows of a block][DP]: its sum of p V
  float2* rows;                // [N, T, Hq] reference and sum of whole rows, for the weights
  float* factors;              // [N, T, Hq] what takes a row's products to scores in log2 units
  float* scores;               // [N, H, S, pad] the products themselves, or null: computed again
  int pad;                     // rows, even
  uint32_t* status;
  long long wait_limit;        // SM cycles per bounded wait of the tensor-core kernel
  int test_starve;             // test hook only: no keys (1), values (2) or keys for the weights (3)
};

struct CaPlan {
  int dp, nt, pieces, blocks, ctas, team;
  bool tc, whole;
  int pad;                     // rows whose products are kept (0: none)
  size_t items, left_off, ml_off, po_off, rows_off, factors_off, scores_off, total;
};

// The launches of a call, for widths up to DP (cache_attention_any.cu), or for DP itself.
template <int DP, int DIM>
lilicorr_status_t ca_launch_rows(const CaArgs& a, const CaPlan& p, cudaStream_t st);

// bf16 queries on the 5th-generation tensor cores (cache_attention_tc.cu)
lilicorr_status_t launch_ca_tc(const CaArgs& a, const CaPlan& p, cudaStream_t st);
// what each key gets from bf16 queries whose scores were not kept (cache_attention_tc_weights.cu)
lilicorr_status_t launch_ca_tc_weights(const CaArgs& a, const CaPlan& p, cudaStream_t st);

constexpr long long CA_WAIT = 4000000000ll;          // about 2 s

}  // namespace lilicorr
