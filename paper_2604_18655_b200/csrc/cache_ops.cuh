// The operators around a bounded KV cache (kernel-level calls): rotary append, attention that totals the keys' softmax
// weights, eviction by those totals.  Argument blocks and launch interface between mlora.cu and the kernels.
#pragma once
#include "common.cuh"

namespace mlora {

struct RopeArgs {
  const void *q, *k, *v;           // rows of fp16 or fp32; null: that part is left out (k and v together)
  long long q_stride, k_stride, v_stride;   // elements between rows
  const int32_t* positions;        // dev [n * T]
  const double* freq;              // dev [rotary / 2] radians per position
  float gain;                      // factor on cos and sin
  int in_fp32, interleaved, rotary;
  int n, T, Hq, Hkv, hd, cap;
  __half *q_out, *own_k, *own_v;   // [n * T][Hq][hd], [n][Hkv][cap][hd]
  const int32_t* suffix_len;       // dev [n]
  float* own_weight;               // [n][Hkv][cap] or null
  int32_t* own_position;           // [n][Hkv][cap] or null
  int* status;
};
cudaError_t launch_rope_append(const RopeArgs& a, cudaStream_t st);

struct ScoredArgs {
  const __half *q, *prefix_k, *prefix_v, *own_k, *own_v;
  const int32_t *suffix_len, *parent;   // parent null: the pass's rows form a chain
  int P, n, T, Hq, Hkv, hd, cap, suffix_bound;
  __half* out;
  float *own_weight, *prefix_weight;    // [n][Hkv][cap], [Hkv][P]
  int* status;
  // set by scored_plan
  int prefix_chunk, n_prefix_chunks, own_chunk, n_own_chunks;   // keys, multiples of 64
  int rt_prefix, rt_own;                // 16-row tiles of all rows / of one stream's rows
  int ld_prefix, ld_own;                // keys a row of the score scratch has room for
  // scratch
  float *part_o, *part_ml, *sc_prefix, *sc_own;
  int tc;                               // many rows a KV head: the tcgen05 kernels
  AttnArgs attn;                        // ... their attention
  float2* row_ml;                       // ... scratch: the rows' (maximum, 1 / sum)
  unsigned long long* anc;              // ... scratch: ancestor masks
};
cudaError_t init_scored();              // per device, once
void scored_plan(ScoredArgs& a, int sm_count);
size_t scored_workspace_floats(const ScoredArgs& a);       // of a planned call
size_t scored_workspace_most(const ScoredArgs& a, int sm_count);   // of any call with this suffix_bound or a smaller one
void scored_carve(ScoredArgs& a, float* ws);
cudaError_t launch_attention_scored(const ScoredArgs& a, cudaStream_t st);

struct EvictArgs {
  __half *own_k, *own_v;           // [n][Hkv][cap][hd]
  const float* weight;             // [n][Hkv][cap]
  const int32_t* position;         // [n][Hkv][cap] or null
  float* out_weight;
  int32_t* out_position;
  const int32_t *suffix_len, *newest;   // dev [n]
  int32_t* out_len;                // dev [n]
  int32_t* out_source;             // [n][Hkv][budget] or null
  int n, Hkv, hd, cap, bound, budget, recent;
  int32_t* counts;                 // scratch: [n * Hkv] moves
  int2* moves;                     // scratch: [n * Hkv][max_moves] (from, to)
  int max_moves;
  int past_l2;                     // set by launch_kv_evict: the rows that move may not fit in L2
  int* status;
};
cudaError_t launch_kv_evict(const EvictArgs& a, cudaStream_t st);

}  // namespace mlora
