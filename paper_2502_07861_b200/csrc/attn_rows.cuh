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

// A warp per query row: the slots' sums brought to one maximum and added, in the order of the slots.
template <bool kBf16, int D>
__device__ inline void join_splits(const AttnRows& A, int64_t row, int lane) {
  float top = -INFINITY;
  for (int i = lane; i < A.n_slots; i += 32) top = fmaxf(top, A.part_ml[(int64_t)i * A.total_rows + row].x);
  top = warp_max(top);
  const float base = top == -INFINITY ? 0.f : top;
  constexpr int kPer = D / 32;
  float sum = 0.f, acc[kPer] = {};
#pragma unroll 4
  for (int i = 0; i < A.n_slots; ++i) {
    const int64_t at = (int64_t)i * A.total_rows + row;
    const float2 ml = A.part_ml[at];
    const float f = exp2f(ml.x - base);
    sum = fmaf(ml.y, f, sum);
#pragma unroll
    for (int c = 0; c < kPer; c += 2) {
      const float2 v = *reinterpret_cast<const float2*>(A.part + at * D + kPer * lane + c);
      acc[c] = fmaf(v.x, f, acc[c]);
      acc[c + 1] = fmaf(v.y, f, acc[c + 1]);
    }
  }
  const float inv = sum == 0.f ? 0.f : 1.f / sum;
  if (A.lse && lane == 0) A.lse[row] = sum == 0.f ? INFINITY : base + log2f(sum);
#pragma unroll
  for (int c = 0; c < kPer; c += 2) {
    if constexpr (kBf16)
      *reinterpret_cast<__nv_bfloat162*>(static_cast<__nv_bfloat16*>(A.out) + row * D + kPer * lane + c) = __floats2bfloat162_rn(acc[c] * inv, acc[c + 1] * inv);
    else
      *reinterpret_cast<float2*>(static_cast<float*>(A.out) + row * D + kPer * lane + c) = make_float2(acc[c] * inv, acc[c + 1] * inv);
  }
}

cudaError_t launch_attn_simt(const AttnRows& A, int d, int is_bf16, cudaStream_t st);
cudaError_t launch_attn_combine(const AttnRows& A, int d, int is_bf16, cudaStream_t st);
cudaError_t launch_score_simt(const AttnRows& A, const ScoreArgs& S, int d, int is_bf16, cudaStream_t st);

int few_splits(int64_t streams, int cap);
int64_t few_pitch(int cap);
cudaError_t launch_attn_few(const AttnRows& A, float* x, int d, int is_bf16, cudaStream_t st);
int few_cluster(int64_t streams, int cap, int n_rows, int d, int is_bf16);
cudaError_t launch_attn_few_cluster(const AttnRows& A, const ScoreArgs& S, int C, int d, int is_bf16, cudaStream_t st);
cudaError_t launch_few_end(const AttnRows& A, float* x, const ScoreArgs& S, int d, int is_bf16, cudaStream_t st);

int attn_tc_splits(const AttnRows& A);
cudaError_t launch_attn_tc(const AttnRows& A, int d, cudaStream_t st);
cudaError_t launch_score_tc(const AttnRows& A, const ScoreArgs& S, int d, cudaStream_t st);

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
