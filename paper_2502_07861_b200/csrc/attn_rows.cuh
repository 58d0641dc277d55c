// Attention over caches that the caller holds: what the host code and the kernels of attn_scored and decode_attn_prefix share.
//
// A stream is one KV head's cache of at most `cap` rows, the first len of which are in use, and a set of query rows that attend it.
// Logits are kept in base 2: x = <k, q> log2(e) / sqrt d + log2 w.
#pragma once

#include <atomic>

#include "common.cuh"

namespace bkv {

// A kernel's dynamic shared memory, set once per device: 0.4 us of every call otherwise.
template <class Kern>
cudaError_t kernel_limits(Kern kern, size_t smem, std::atomic<unsigned long long>& devices) {
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  const unsigned long long bit = dev < 64 ? 1ull << dev : 0;
  if (devices.load(std::memory_order_acquire) & bit) return cudaSuccess;
  e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
  if (e == cudaSuccess) devices.fetch_or(bit, std::memory_order_release);
  return e;
}

constexpr int kAttnSms = 148;                 // split factors and workspaces follow from sizes alone
constexpr int kAttnMaxSplits = 64;
constexpr int kFewRows = 8;                   // query rows that a CTA of the one-pass decode kernels takes

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
// Some kernels read lens, queries and old scores before they wait for the kernel ahead of them, which has waited for what wrote these:
// past L1, whose lines may be older than that.
__device__ inline int attn_len(const AttnRows& A, int s) {
  return A.lens ? max(0, min(__ldcg(A.lens + s / A.lens_div), A.cap)) : A.cap;
}
// Rows that query row r of a stream of len rows sees.
__device__ inline int attn_limit(const AttnRows& A, int len, int r) {
  return max(0, min(len, len - A.n_queries + r % A.n_queries + 1));
}

// The sums over `kG` neighbouring lanes of a[0], .., a[kG - 1], that of a[i] to the lane i of them: kG - 1 exchanges.
template <int kG>
__device__ inline float sum_scatter(float (&a)[kG], int lane) {
#pragma unroll
  for (int off = kG / 2; off > 0; off /= 2) {
    const bool upper = lane & off;
#pragma unroll
    for (int i = 0; i < off; ++i) {
      const float give = upper ? a[i] : a[i + off], keep = upper ? a[i + off] : a[i];
      a[i] = keep + __shfl_xor_sync(0xffffffffu, give, off);
    }
  }
  return a[0];
}

// The sums of what every row received: score_out = decay score_in + sum over heads and the newest n_scored queries of 2^(x - lse).
struct ScoreArgs {
  const float* in;          // [n_streams, cap]; null: zeros
  float* out;               // [n_streams, cap]; rows behind the last keep what they hold
  float decay;
  int32_t n_scored;
};
__device__ inline float score_old(const ScoreArgs& S, int64_t at) { return S.in ? __ldcg(S.in + at) : 0.f; }
__device__ inline void score_put(const ScoreArgs& S, int64_t at, float old, float sum) { S.out[at] = S.in ? fmaf(S.decay, old, sum) : sum; }
__device__ inline void score_put(const ScoreArgs& S, int64_t at, float sum) { score_put(S, at, score_old(S, at), sum); }

// Joining the slots of query rows: their sums brought to one maximum and added.  A CTA of eight warps takes eight rows, or, of more than
// eight slots, two rows with four warps each, which add every fourth slot up and then one another's sums: the order depends on sizes alone.
constexpr int kJoinThreads = 256, kJoinMaxSlots = 2 * kAttnMaxSplits;
__host__ __device__ inline int join_rows(const AttnRows& A) { return A.n_slots > 8 ? 2 : 8; }
inline int join_ctas(const AttnRows& A) { return (A.total_rows + join_rows(A) - 1) / join_rows(A); }
template <int D>
struct JoinShared {
  float acc[kJoinThreads / 32][D];
};
// kAhead: slots that a warp asks for at once.
template <bool kBf16, int D, int kAhead>
__device__ inline void join_splits(const AttnRows& A, int cta, JoinShared<D>& sh) {
  constexpr int kPer = D / 32, kChunks = kJoinMaxSlots / 32;
  const int warp = threadIdx.x / 32, lane = threadIdx.x % 32, rows = join_rows(A), ways = kJoinThreads / 32 / rows, way = warp % ways;
  const int64_t row = (int64_t)cta * rows + warp / ways;
  const bool held = row < A.total_rows;
  float acc[kPer] = {}, sum = 0.f, base = 0.f;
  if (held) {
    float2 ml[kChunks];
    float top = -INFINITY, f[kChunks];
#pragma unroll
    for (int k = 0; k < kChunks; ++k) {
      ml[k] = lane + 32 * k < A.n_slots ? A.part_ml[(int64_t)(lane + 32 * k) * A.total_rows + row] : make_float2(-INFINITY, 0.f);
      top = fmaxf(top, ml[k].x);
    }
    top = warp_max(top);
    base = top == -INFINITY ? 0.f : top;
#pragma unroll
    for (int k = 0; k < kChunks; ++k) {
      f[k] = exp2f(ml[k].x - base);
      sum = fmaf(ml[k].y, f[k], sum);
    }
    sum = warp_sum(sum);
#pragma unroll
    for (int k = 0; k < kChunks; ++k) {
      for (int i0 = 32 * k + way; i0 < min(32 * k + 32, A.n_slots); i0 += kAhead * ways) {
        float v[kAhead][kPer];
#pragma unroll
        for (int j = 0; j < kAhead; ++j) {
          const int i = i0 + j * ways;
          const float* from = A.part + ((int64_t)i * A.total_rows + row) * D + kPer * lane;
          const bool in = i < min(32 * k + 32, A.n_slots);
#pragma unroll
          for (int c = 0; c < kPer; c += 2) {
            const float2 x = in ? *reinterpret_cast<const float2*>(from + c) : make_float2(0.f, 0.f);
            v[j][c] = x.x;
            v[j][c + 1] = x.y;
          }
        }
#pragma unroll
        for (int j = 0; j < kAhead; ++j) {
          const float w = __shfl_sync(0xffffffffu, f[k], i0 + j * ways & 31);
          if (i0 + j * ways >= min(32 * k + 32, A.n_slots)) break;
          if (w == 0.f) continue;                // an empty slot, whose sums are not written
#pragma unroll
          for (int c = 0; c < kPer; ++c) acc[c] = fmaf(v[j][c], w, acc[c]);
        }
      }
    }
  }
  if (ways > 1) {
#pragma unroll
    for (int c = 0; c < kPer; ++c) sh.acc[warp][kPer * lane + c] = acc[c];
    __syncthreads();
    if (way != 0) return;
#pragma unroll
    for (int c = 0; c < kPer; ++c) {
      acc[c] = 0.f;
      for (int w = 0; w < ways; ++w) acc[c] += sh.acc[warp + w][kPer * lane + c];
    }
  }
  if (!held) return;
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

int simt_row_tiles(int n_rows);
cudaError_t launch_attn_simt(const AttnRows& A, int d, cudaStream_t st);      // fp32
cudaError_t launch_attn_combine(const AttnRows& A, int d, int is_bf16, cudaStream_t st);
cudaError_t launch_score_simt(const AttnRows& A, const ScoreArgs& S, int d, cudaStream_t st);      // fp32

int few_splits(int64_t streams, int cap, int n_rows, int d, int is_bf16);
int64_t few_pitch(int cap);
// How a launch of the one-pass kernel stands to the launch before it: behind it; behind it, to finish its outputs (one split, which joins the slots
// before its own); beside it, on the SMs that it leaves.
enum FewOrder { kFewAlone, kFewFinish, kFewBeside };
cudaError_t launch_attn_few(const AttnRows& A, float* x, const AttnRows* also, FewOrder order, int d, int is_bf16, cudaStream_t st);
int few_cluster(int64_t streams, int cap, int n_rows, int d, int is_bf16);
int64_t few_cluster_sums(const AttnRows& A);
cudaError_t launch_attn_few_cluster(const AttnRows& A, const ScoreArgs& S, int C, float* sums, int d, int is_bf16, cudaStream_t st);
cudaError_t launch_few_end(const AttnRows& A, float* x, const ScoreArgs& S, int d, int is_bf16, cudaStream_t st);

int attn_tc_splits(const AttnRows& A);
int attn_tc_blocks(const AttnRows& A);         // CTAs of a split, of all streams
bool attn_tc_by_keys(const AttnRows& A);
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
