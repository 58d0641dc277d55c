// Attention over caches that the caller holds: what the host code and the kernels of attn_scored and decode_attn_prefix share.
//
// A stream is one KV head's cache of at most `cap` rows, the first len of which are in use, and a set of query rows that attend it.
// Logits are kept in base 2: x = <k, q> log2(e) / sqrt d + log2 w.
#pragma once

#include "common.cuh"

namespace bkv {

constexpr int kAttnSms = 148;                 // split factors and workspaces follow from sizes alone
constexpr int kAttnMaxSplits = 64;
constexpr int kFewRows = 8;                   // query rows of a stream that the one-pass decode kernels take

struct AttnRows {
  const void *K, *V;        // [n_streams, cap, d]
  const int32_t* lens;      // [n_streams / lens_div] rows in use; null: cap
  const float* w;           // [n_streams, cap] weights of the rows; null: 1
  int32_t n_streams, cap, lens_div;
  // Query rows.  Row r of stream s sits at s q_stream + (r / q_inner) q_outer + (r % q_inner), in rows of d elements, and so does
  // its output; that is also its number among the call's rows.
  const void* q;
  void* out;
  int32_t n_rows;           // of a stream
  int32_t q_stream, q_inner, q_outer;
  int32_t n_queries;        // row r is the query r % n_queries: it sees the first len - n_queries + r % n_queries + 1 rows
  int32_t total_rows;       // of the call
  float scale;              // log2(e) / sqrt d
  // Partial results: slot0 + split of n_slots; one slot: the results themselves.
  int32_t splits, slot0, n_slots;
  float* part;              // [n_slots, total_rows, d] sums of 2^(x - max) v
  float2* part_ml;          // [n_slots, total_rows] maximum of x, sum of 2^(x - max)
  float* lse;               // [total_rows] log2 of the sum of 2^x (+inf: the row sees nothing); null: not asked for
};

__host__ __device__ inline int64_t attn_row(const AttnRows& A, int s, int r) {
  return (int64_t)s * A.q_stream + (int64_t)(r / A.q_inner) * A.q_outer + r % A.q_inner;
}
__device__ inline int attn_len(const AttnRows& A, int s) {
  return A.lens ? max(0, min(A.lens[s / A.lens_div], A.cap)) : A.cap;
}
// Rows that query row r of a stream of len rows sees.
__device__ inline int attn_limit(const AttnRows& A, int len, int r) {
  return max(0, min(len, len - A.n_queries + r % A.n_queries + 1));
}

// The sums of what every row received: score_out = decay score_in + sum over heads and the newest n_scored queries of 2^(x - lse).
struct ScoreArgs {
  const float* in;          // [n_streams, cap]; null: zeros
  float* out;               // [n_streams, cap]; rows behind the last keep what they hold
  float decay;
  int32_t n_scored;
};
__device__ inline void score_put(const ScoreArgs& S, int64_t at, float sum) {
  S.out[at] = S.in ? fmaf(S.decay, S.in[at], sum) : sum;
}

cudaError_t launch_attn_simt(const AttnRows& A, int d, int is_bf16, cudaStream_t st);
cudaError_t launch_attn_combine(const AttnRows& A, int d, int is_bf16, cudaStream_t st);
cudaError_t launch_score_simt(const AttnRows& A, const ScoreArgs& S, int d, int is_bf16, cudaStream_t st);

struct EvictArgs {
  const void *K, *V;
  const float* score;
  const int32_t *pos, *lens;      // null: the row's number; every row in use
  void *K_out, *V_out;
  float* score_out;
  int32_t *pos_out, *lens_out;    // null: not wanted
  int32_t n_streams, cap, cap_out, keep, n_first, n_recent;
  int32_t row_bytes;
  int32_t in_place;               // K_out == K and so on: only the rows that fill a hole move
  int32_t* moves;                 // workspace: [n_streams][2][list] holes and what fills them
  int32_t* n_moves;               // [n_streams]
  int32_t list;
};
cudaError_t launch_evict(const EvictArgs& E, cudaStream_t st);

}  // namespace bkv
