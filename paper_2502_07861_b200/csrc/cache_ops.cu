// balancekv_attn_scored, balancekv_cache_evict, balancekv_decode_attn_prefix: operators on caches that the caller holds.
// Arguments are checked here and workspaces are laid out; everything else runs in the kernels.
#include <algorithm>
#include <climits>
#include <cmath>
#include <cstdio>

#include "../../include/balancekv.h"
#include "attn_rows.cuh"

using namespace bkv;

namespace {

constexpr int64_t kMostRows = (int64_t)1 << 30;        // rows and tiles are numbered in 32 bits

bool aligned(const void* p, uintptr_t to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) == 0; }
bool shape_ok(int head_dim, int dtype) { return (head_dim == 64 || head_dim == 128) && (dtype == 0 || dtype == 1); }

// Pieces of a workspace, 256 bytes aligned.  Without a base it counts.
struct Pieces {
  char* base;
  size_t used = 0;
  template <class T>
  T* take(int64_t n) {
    T* p = base ? reinterpret_cast<T*>(base + used) : nullptr;
    used += ((size_t)n * sizeof(T) + 255) & ~(size_t)255;
    return p;
  }
};

int report(const char* what, cudaError_t e) {
  if (e == cudaSuccess) return BALANCEKV_OK;
  std::fprintf(stderr, "%s: launch failed: %s\n", what, cudaGetErrorString(e));
  return e == cudaErrorMemoryAllocation ? BALANCEKV_E_NOMEM : BALANCEKV_E_CUDA;
}

// CTAs that share the keys of a tile of query rows on CUDA cores: two waves of them at most, two tiles of keys each at least.
int simt_splits(int64_t row_tiles, int cap) {
  const int64_t key_tiles = (cap + 63) / 64, want = 2 * kAttnSms / row_tiles;
  return (int)std::max<int64_t>(1, std::min<int64_t>({want, key_tiles / 2, (int64_t)kAttnMaxSplits}));
}

void take_parts(AttnRows& A, Pieces& ws, int d) {
  if (A.n_slots == 1) return;
  A.part = ws.take<float>((int64_t)A.n_slots * A.total_rows * d);
  A.part_ml = ws.take<float2>((int64_t)A.n_slots * A.total_rows);
}

// ---- attn_scored

// CTAs of a cluster where clusters serve the call, else 0.
int cluster_of(const AttnRows& A, int n_scored, int head_dim, int dtype) {
  return n_scored ? few_cluster(A.n_streams, A.cap, A.n_rows, head_dim, dtype) : 0;
}

// x: what the one-pass kernels leave for the scores.
int plan_scored(AttnRows& A, float*& x, Pieces& ws, int n_streams, int capacity, int n_queries, int group, int head_dim, int dtype, int n_scored) {
  if (n_streams < 1 || capacity < 1 || n_queries < 1 || group < 1 || group > kMaxGroup || !shape_ok(head_dim, dtype)) return BALANCEKV_E_INVAL;
  if (n_scored < 0 || n_scored > n_queries) return BALANCEKV_E_INVAL;
  const int64_t rows = (int64_t)group * n_queries;
  if (rows > kMostRows / n_streams || (int64_t)n_streams * ((capacity + 63) / 64) > kMostRows) return BALANCEKV_E_INVAL;
  A.n_streams = n_streams;
  A.cap = capacity;
  A.lens_div = 1;
  A.n_rows = A.q_stream = A.q_inner = (int)rows;
  A.q_outer = 0;
  A.n_queries = n_queries;
  A.total_rows = (int)rows * n_streams;
  A.scale = (float)(1.4426950408889634 / std::sqrt((double)head_dim));
  const bool few = rows <= kFewRows;
  if (cluster_of(A, n_scored, head_dim, dtype)) {        // nothing leaves the chip but what groups of query rows add up
    x = ws.take<float>(few_cluster_sums(A));
    return BALANCEKV_OK;
  }
  A.splits = few ? few_splits(n_streams, capacity, (int)rows, head_dim, dtype) : dtype ? attn_tc_splits(A) : simt_splits((int64_t)simt_row_tiles((int)rows) * n_streams, capacity);
  A.n_slots = A.splits;
  take_parts(A, ws, head_dim);
  if (n_scored) A.lse = ws.take<float>(A.total_rows);
  x = n_scored && few ? ws.take<float>(A.total_rows * few_pitch(capacity)) : nullptr;
  return BALANCEKV_OK;
}

// ---- decode_attn_prefix

// Whether the one-pass kernels take the prefix, eight query rows to a CTA: fp32 has no tensor cores to go to, and its tiles of 128 query
// rows pay only when there are a few of them.
bool prefix_by_few(const AttnRows& P, int dtype) { return P.n_rows <= (dtype ? kFewRows : 128); }

// Whether the sequences' own rows are read beside the tensor-core kernel's work on the prefix, which then leaves them SMs, and by how many splits
// that works.  Times in us: a pair of query tiles with a tile of keys takes 1.7, a tile of keys by itself 1.55 (it waits for memory); the one-pass
// kernel reads 6 MB and a wave of its CTAs takes 4.5.  The SMs are shared out by these times, the tensor-core kernel's counted half as long
// again, since others now read too, the own rows' at half of their capacity, which is what they fill on the way; three quarters at most (128 x 8 x 4
// behind 16384 rows, 300 own each: 66 to 71 us by 112 CTAs, 84 by 128, 74 one after the other; up to 300: 64, 68, 62).  Calls one behind the
// other, on three sets of inputs in turn: 256 sequences x 5 heads x 8 behind 8192 rows with 1024 own rows each 220 us one after the other, 193 so,
// with up to 1024 147 and 137, with 256 113 and 104, with up to 256 96 and 101.
// It costs a launch that joins, unless the own rows need one anyway: short ones finish the outputs themselves instead (64 x 4 x 8 behind 32768
// rows, 200 own: 60 us against 62 beside), and where the tensor-core kernel waits for memory too, so do all that are not most of the work (32 x 4 x 8
// behind 32768, 512 own: 45 against 51 beside; 2048 own: 85 against 75).
bool prefix_beside(const AttnRows& P, const AttnRows& A, int head_dim, int& splits) {
  const bool by_keys = attn_tc_by_keys(P);
  const int64_t blocks = attn_tc_blocks(P), tiles = (P.cap + 127) / 128;
  const double prefix = (double)blocks * tiles * (by_keys ? 1.55 : 1.7) / kAttnSms;
  const int64_t waves = ((int64_t)A.n_streams * A.splits + 2 * kAttnSms - 1) / (2 * kAttnSms);
  const double bytes = (double)A.n_streams * A.cap * head_dim * 4, own = std::max(bytes / 6e6, 4.5 * waves), usual = std::max(bytes / 12e6, 4.5 * waves);
  if (A.splits == 1 && (own < 10 || (by_keys && own < 1.5 * prefix))) return false;
  const double sms = kAttnSms * std::min(0.75, 1.5 * prefix / (1.5 * prefix + usual));
  splits = (int)std::max<int64_t>(1, std::min<int64_t>({(int64_t)std::ceil(sms / blocks), tiles / 2, kAttnMaxSplits}));
  return true;
}

int plan_prefix(AttnRows& P, AttnRows& A, bool& beside, Pieces& ws, int prefix_len, int capacity, int n_seqs, int n_kv_heads, int group, int head_dim, int dtype) {
  if (prefix_len < 1 || capacity < 0 || n_seqs < 1 || n_kv_heads < 1 || group < 1 || group > kMaxGroup || !shape_ok(head_dim, dtype)) return BALANCEKV_E_INVAL;
  const int64_t streams = (int64_t)n_seqs * n_kv_heads;
  if (streams > kMostRows / group || streams * ((capacity + 63) / 64) > kMostRows || (int64_t)n_kv_heads * ((prefix_len + 63) / 64) > kMostRows)
    return BALANCEKV_E_INVAL;
  P.total_rows = A.total_rows = (int)streams * group;
  P.scale = A.scale = (float)(1.4426950408889634 / std::sqrt((double)head_dim));
  P.n_queries = A.n_queries = 1;
  P.lens_div = 1;
  P.n_streams = n_kv_heads;                    // a KV head's prefix and the query heads of all sequences
  P.cap = prefix_len;
  P.n_rows = n_seqs * group;
  P.q_stream = P.q_inner = group;
  P.q_outer = n_kv_heads * group;
  const bool few = prefix_by_few(P, dtype);
  P.splits = few ? few_splits(n_kv_heads, prefix_len, P.n_rows, head_dim, dtype) : dtype ? attn_tc_splits(P) : simt_splits((int64_t)simt_row_tiles(P.n_rows) * n_kv_heads, prefix_len);
  A.n_streams = (int)streams;                  // a sequence's own rows
  A.lens_div = n_kv_heads;
  A.cap = capacity;
  A.n_rows = A.q_stream = A.q_inner = group;
  A.splits = capacity ? few_splits(streams, capacity, group, head_dim, dtype) : 0;
  beside = capacity && dtype && !few && prefix_beside(P, A, head_dim, P.splits);
  A.slot0 = P.splits;
  P.n_slots = A.n_slots = A.slot0 + A.splits;
  take_parts(P, ws, head_dim);
  A.part = P.part;
  A.part_ml = P.part_ml;
  return BALANCEKV_OK;
}

// ---- cache_evict

int plan_evict(EvictArgs& E, Pieces& ws, int n_streams, int capacity, int n_keep, int head_dim, int dtype, int in_place) {
  if (n_streams < 1 || capacity < 1 || n_keep < 1 || !shape_ok(head_dim, dtype)) return BALANCEKV_E_INVAL;
  if ((int64_t)n_streams * capacity > ((int64_t)1 << 40) || capacity > (1 << 30) || (int64_t)n_streams * ((capacity + 31) / 32) > kMostRows)
    return BALANCEKV_E_INVAL;
  E.n_streams = n_streams;
  E.cap = capacity;
  E.keep = std::min(n_keep, capacity);
  E.list = std::min(E.keep, capacity - E.keep);
  E.in_place = in_place;
  E.row_bytes = head_dim * (dtype ? 2 : 4);
  E.moves = ws.take<int>((int64_t)n_streams * (2 * (int64_t)E.list + (in_place ? 0 : E.keep)));
  E.n_moves = ws.take<int>(n_streams);
  return BALANCEKV_OK;
}

}  // namespace

extern "C" int balancekv_attn_scored_workspace(int n_streams, int capacity, int n_queries, int group, int head_dim, int dtype, int n_scored,
                                               size_t* bytes) {
  if (!bytes) return BALANCEKV_E_INVAL;
  AttnRows A{};
  float* x;
  Pieces ws{nullptr};
  const int rc = plan_scored(A, x, ws, n_streams, capacity, n_queries, group, head_dim, dtype, n_scored);
  if (rc == BALANCEKV_OK) *bytes = ws.used;
  return rc;
}

extern "C" int balancekv_attn_scored(const void* K, const void* V, const int32_t* lens, int n_streams, int capacity, const void* q, void* out,
                                     int n_queries, int group, int head_dim, int dtype, const float* score_in, float* score_out, int n_scored,
                                     float decay, void* workspace, size_t workspace_bytes, void* stream) {
  if (!K || !V || !q || !out || (n_scored != 0 && !score_out)) return BALANCEKV_E_INVAL;
  if (!aligned(K, 16) || !aligned(V, 16) || !aligned(q, 16) || !aligned(out, 16) || !aligned(lens, 4) || !aligned(score_in, 4) || !aligned(score_out, 4) ||
      !aligned(workspace, 256))
    return BALANCEKV_E_INVAL;
  AttnRows A{};
  float* x;
  Pieces ws{static_cast<char*>(workspace)};
  if (const int rc = plan_scored(A, x, ws, n_streams, capacity, n_queries, group, head_dim, dtype, n_scored)) return rc;
  if (ws.used && !workspace) return BALANCEKV_E_INVAL;
  if (workspace_bytes < ws.used) return BALANCEKV_E_NOMEM;
  A.K = K;
  A.V = V;
  A.lens = lens;
  A.q = q;
  A.out = out;
  const cudaStream_t st = static_cast<cudaStream_t>(stream);
  const ScoreArgs S{score_in, score_out, decay, n_scored};
  cudaError_t e;
  if (const int C = cluster_of(A, n_scored, head_dim, dtype)) {
    e = launch_attn_few_cluster(A, S, C, x, head_dim, dtype, st);
  } else if (A.n_rows <= kFewRows) {
    e = launch_attn_few(A, x, nullptr, kFewAlone, head_dim, dtype, st);
    if (e == cudaSuccess && n_scored) e = launch_few_end(A, x, S, head_dim, dtype, st);
    else if (e == cudaSuccess && A.n_slots > 1) e = launch_attn_combine(A, head_dim, dtype, st);
  } else {
    e = dtype ? launch_attn_tc(A, head_dim, st) : launch_attn_simt(A, head_dim, st);
    if (e == cudaSuccess && A.n_slots > 1) e = launch_attn_combine(A, head_dim, dtype, st);
    if (e == cudaSuccess && n_scored) e = dtype ? launch_score_tc(A, S, head_dim, st) : launch_score_simt(A, S, head_dim, st);
  }
  return report("balancekv_attn_scored", e);
}

extern "C" int balancekv_decode_attn_prefix_workspace(int prefix_len, int capacity, int n_seqs, int n_kv_heads, int group, int head_dim, int dtype,
                                                      size_t* bytes) {
  if (!bytes) return BALANCEKV_E_INVAL;
  AttnRows P{}, A{};
  bool beside;
  Pieces ws{nullptr};
  const int rc = plan_prefix(P, A, beside, ws, prefix_len, capacity, n_seqs, n_kv_heads, group, head_dim, dtype);
  if (rc == BALANCEKV_OK) *bytes = ws.used;
  return rc;
}

extern "C" int balancekv_decode_attn_prefix(const void* K_prefix, const void* V_prefix, const float* w_prefix, int prefix_len, const void* K,
                                            const void* V, const int32_t* lens, int capacity, const void* q, void* out, int n_seqs, int n_kv_heads,
                                            int group, int head_dim, int dtype, void* workspace, size_t workspace_bytes, void* stream) {
  if (!K_prefix || !V_prefix || !q || !out || (capacity != 0 && (!K || !V))) return BALANCEKV_E_INVAL;
  if (!aligned(K_prefix, 16) || !aligned(V_prefix, 16) || !aligned(K, 16) || !aligned(V, 16) || !aligned(q, 16) || !aligned(out, 16) ||
      !aligned(w_prefix, 4) || !aligned(lens, 4) || !aligned(workspace, 256))
    return BALANCEKV_E_INVAL;
  AttnRows P{}, A{};
  bool beside;
  Pieces ws{static_cast<char*>(workspace)};
  if (const int rc = plan_prefix(P, A, beside, ws, prefix_len, capacity, n_seqs, n_kv_heads, group, head_dim, dtype)) return rc;
  if (ws.used && !workspace) return BALANCEKV_E_INVAL;
  if (workspace_bytes < ws.used) return BALANCEKV_E_NOMEM;
  P.K = K_prefix;
  P.V = V_prefix;
  P.w = w_prefix;
  A.K = K;
  A.V = V;
  A.lens = lens;
  P.q = A.q = q;
  P.out = A.out = out;
  const cudaStream_t st = static_cast<cudaStream_t>(stream);
  // Own rows of one split join the prefix's slots themselves, unless they are read beside its launch.
  const bool few = prefix_by_few(P, dtype), finish = !few && A.splits == 1 && !beside && A.slot0 <= kAttnMaxSplits;
  cudaError_t e;
  if (few) {
    e = launch_attn_few(P, nullptr, A.splits ? &A : nullptr, kFewAlone, head_dim, dtype, st);
  } else {
    e = dtype ? launch_attn_tc(P, head_dim, st) : launch_attn_simt(P, head_dim, st);
    if (e == cudaSuccess && A.splits) e = launch_attn_few(A, nullptr, nullptr, finish ? kFewFinish : beside ? kFewBeside : kFewAlone, head_dim, dtype, st);
  }
  if (e == cudaSuccess && P.n_slots > 1 && !finish) e = launch_attn_combine(P, head_dim, dtype, st);
  return report("balancekv_decode_attn_prefix", e);
}

extern "C" int balancekv_cache_evict_workspace(int n_streams, int capacity, int n_keep, int head_dim, int dtype, int in_place, size_t* bytes) {
  if (!bytes) return BALANCEKV_E_INVAL;
  EvictArgs E{};
  Pieces ws{nullptr};
  const int rc = plan_evict(E, ws, n_streams, capacity, n_keep, head_dim, dtype, in_place != 0);
  if (rc == BALANCEKV_OK) *bytes = ws.used;
  return rc;
}

extern "C" int balancekv_cache_evict(const void* K, const void* V, const float* score, const int32_t* pos, const int32_t* lens, int n_streams,
                                     int capacity, void* K_out, void* V_out, float* score_out, int32_t* pos_out, int32_t* lens_out, int capacity_out,
                                     int n_keep, int n_first, int n_recent, int head_dim, int dtype, void* workspace, size_t workspace_bytes,
                                     void* stream) {
  if (!K || !V || !score || !K_out || !V_out || !score_out) return BALANCEKV_E_INVAL;
  // all of the cache in place, or none of it
  const int same = (K_out == K) + (V_out == V) + (score_out == score);
  const bool in_place = same == 3;
  if ((same != 0 && !in_place) || (in_place ? pos_out != pos || capacity_out != capacity : pos_out && pos_out == pos)) return BALANCEKV_E_INVAL;
  if (!aligned(K, 16) || !aligned(V, 16) || !aligned(K_out, 16) || !aligned(V_out, 16) || !aligned(score, 4) || !aligned(score_out, 4) ||
      !aligned(pos, 4) || !aligned(pos_out, 4) || !aligned(lens, 4) || !aligned(lens_out, 4) || !aligned(workspace, 256))
    return BALANCEKV_E_INVAL;
  EvictArgs E{};
  Pieces ws{static_cast<char*>(workspace)};
  if (const int rc = plan_evict(E, ws, n_streams, capacity, n_keep, head_dim, dtype, in_place)) return rc;
  if (n_first < 0 || n_recent < 0 || (int64_t)n_first + n_recent > n_keep || capacity_out < E.keep) return BALANCEKV_E_INVAL;
  if (ws.used && !workspace) return BALANCEKV_E_INVAL;
  if (workspace_bytes < ws.used) return BALANCEKV_E_NOMEM;
  E.K = K;
  E.V = V;
  E.score = score;
  E.pos = pos;
  E.lens = lens;
  E.K_out = K_out;
  E.V_out = V_out;
  E.score_out = score_out;
  E.pos_out = pos_out;
  E.lens_out = lens_out;
  E.cap_out = capacity_out;
  E.n_first = n_first;
  E.n_recent = n_recent;
  return report("balancekv_cache_evict", launch_evict(E, static_cast<cudaStream_t>(stream)));
}
