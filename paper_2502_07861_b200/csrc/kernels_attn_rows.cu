// Attention of many query rows over a caller-held fp32 cache, its score pass, and the kernel that joins splits.
//
//   x_{r,i} = <q_r, k_i> log2(e) / sqrt d + log2 w_i,   out_r = sum_i 2^(x_{r,i} - m_r) v_i / sum_i 2^(x_{r,i} - m_r)
//
// over the rows that r sees, with a maximum m_r that follows when it would grow by more than 8, so that the cache is read once.  A CTA of 256
// threads takes 128 query rows and walks its share of the keys in tiles of 64; a thread forms 8 x 4 logits, then 8 rows x d / 16 columns of
// the outputs, by packed FFMA from tiles in shared memory.  The next tile of K comes in (cp.async) while this one's weights and outputs are formed, the
// next of V under the logits.  What bounds it are the FMAs: 64 of them per 16-byte load of a thread's rows and keys keep the loads at half of
// shared memory's rate.
#include "attn_rows.cuh"

namespace bkv {

namespace {

constexpr int kRows = 128, kKeys = 64, kThreads = 256;
constexpr int kMine = kRows / 16;                // query rows of a thread: ty + 16 a
constexpr float kGrow = 8.f;                     // a maximum follows when it would grow by more: weights stay below 2^8

template <int D>
struct Tile {
  static constexpr int kPitch = D + 4;           // floats: rows 16 bytes aligned, neighbours in other banks
  static constexpr int kPPitch = kKeys + 16;
  static constexpr size_t kSmem = sizeof(float) * (size_t)(kRows * kPitch + 2 * kKeys * kPitch + kRows * kPPitch + kKeys);
};

// rows x D of a tile on their way into shared memory; row i of the tile is row at(i) of base, or zeros where at(i) < 0.
template <int D, class At>
__device__ inline void ask_tile(float* sm, const void* base, int rows, At at) {
  for (int i = threadIdx.x; i < rows * (D / 4); i += kThreads) {
    const int row = i / (D / 4), e = i % (D / 4) * 4;
    const int64_t from = at(row);
    const float* src = static_cast<const float*>(base) + (from < 0 ? 0 : from * D + e);
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;"
                 ::"r"((uint32_t)__cvta_generic_to_shared(sm + row * Tile<D>::kPitch + e)), "l"(src), "r"(from < 0 ? 0 : 16) : "memory");
  }
}
__device__ inline void commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int kPending>
__device__ inline void arrived() { asm volatile("cp.async.wait_group %0;" ::"n"(kPending) : "memory"); }

// <X row ty + 16 a, Y row tx + 16 b>
template <int D>
__device__ inline void dots(const float* X, const float* Y, int ty, int tx, float (&out)[kMine][4]) {
  float2 acc[kMine][4];
#pragma unroll
  for (int a = 0; a < kMine; ++a)
#pragma unroll
    for (int b = 0; b < 4; ++b) acc[a][b] = make_float2(0.f, 0.f);
#pragma unroll 4
  for (int e = 0; e < D; e += 4) {
    float4 y[4];
#pragma unroll
    for (int b = 0; b < 4; ++b) y[b] = *reinterpret_cast<const float4*>(Y + (tx + 16 * b) * Tile<D>::kPitch + e);
#pragma unroll
    for (int a = 0; a < kMine; ++a) {
      const float4 x = *reinterpret_cast<const float4*>(X + (ty + 16 * a) * Tile<D>::kPitch + e);
#pragma unroll
      for (int b = 0; b < 4; ++b) {
        acc[a][b] = __ffma2_rn(make_float2(x.x, x.y), make_float2(y[b].x, y[b].y), acc[a][b]);
        acc[a][b] = __ffma2_rn(make_float2(x.z, x.w), make_float2(y[b].z, y[b].w), acc[a][b]);
      }
    }
  }
#pragma unroll
  for (int a = 0; a < kMine; ++a)
#pragma unroll
    for (int b = 0; b < 4; ++b) out[a][b] = acc[a][b].x + acc[a][b].y;
}

__device__ inline float half_warp_max(float v) {
#pragma unroll
  for (int o = 8; o > 0; o >>= 1) v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, o));
  return v;
}
__device__ inline float half_warp_sum(float v) {
#pragma unroll
  for (int o = 8; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}

template <int D>
__global__ void __launch_bounds__(kThreads) attn_simt_kernel(const AttnRows A, int row_tiles) {
  constexpr int kPitch = Tile<D>::kPitch, kPPitch = Tile<D>::kPPitch, kC = D / 64;      // 16-byte pieces of a thread's columns: 4 tx + 64 c
  extern __shared__ __align__(16) float smem[];
  float *Qs = smem, *Ks = Qs + kRows * kPitch, *Vs = Ks + kKeys * kPitch, *Ps = Vs + kKeys * kPitch, *lw = Ps + kRows * kPPitch;
  const int tid = threadIdx.x, ty = tid / 16, tx = tid % 16;
  const int s = blockIdx.x / row_tiles, r0 = (row_tiles - 1 - (int)blockIdx.x % row_tiles) * kRows, split = blockIdx.y;
  grid_wait_and_release();
  const int len = attn_len(A, s);
  const int last = min(r0 + kRows, A.n_rows) - 1;
  const int most = r0 / A.n_queries != last / A.n_queries ? len : attn_limit(A, len, last);      // of the tile's rows
  const int tiles = (most + kKeys - 1) / kKeys;
  const int t0 = (int)((int64_t)tiles * split / A.splits), t1 = (int)((int64_t)tiles * (split + 1) / A.splits);
  const int64_t first = (int64_t)s * A.cap;
  auto ask_keys = [&](int t) {
    if (t < t1) ask_tile<D>(Ks, A.K, kKeys, [&](int i) { return t * kKeys + i < len ? first + t * kKeys + i : (int64_t)-1; });
    commit();
  };
  // a row of weight zero counts as absent, whatever it holds
  auto ask_values = [&](int t) {
    if (t < t1)
      ask_tile<D>(Vs, A.V, kKeys, [&](int i) {
        const int64_t row = first + t * kKeys + i;
        return t * kKeys + i < len && !(A.w && A.w[row] == 0.f) ? row : (int64_t)-1;
      });
    commit();
  };
  auto weight = [&](int t) { return A.w && t < t1 && t * kKeys + tid < len ? A.w[first + t * kKeys + tid] : 1.f; };      // tid < kKeys
  ask_tile<D>(Qs, A.q, kRows, [&](int i) { return r0 + i < A.n_rows ? attn_row(A, s, r0 + i) : (int64_t)-1; });
  ask_keys(t0);
  ask_values(t0);
  float w = tid < kKeys ? weight(t0) : 1.f;
  int limit[kMine];
  float m[kMine], l[kMine];
  float2 acc[kMine][kC][2];
#pragma unroll
  for (int a = 0; a < kMine; ++a) {
    limit[a] = attn_limit(A, len, min(r0 + ty + 16 * a, A.n_rows - 1));
    m[a] = -INFINITY;
    l[a] = 0.f;
#pragma unroll
    for (int c = 0; c < kC; ++c) acc[a][c][0] = acc[a][c][1] = make_float2(0.f, 0.f);
  }
  for (int t = t0; t < t1; ++t) {
    const int k0 = t * kKeys;
    arrived<1>();                                // K (and Q); V may still be on its way
    if (tid < kKeys) {
      lw[tid] = log2f(w);
      w = weight(t + 1);
    }
    __syncthreads();
    float x[kMine][4];
    dots<D>(Qs, Ks, ty, tx, x);
    float add[4];
#pragma unroll
    for (int b = 0; b < 4; ++b) add[b] = lw[tx + 16 * b];
    __syncthreads();
    ask_keys(t + 1);
    bool more = false;
#pragma unroll
    for (int a = 0; a < kMine; ++a)
#pragma unroll
      for (int b = 0; b < 4; ++b) {
        x[a][b] = k0 + tx + 16 * b < limit[a] && add[b] != -INFINITY ? fmaf(x[a][b], A.scale, add[b]) : -INFINITY;
        more = more || x[a][b] > m[a] + kGrow;
      }
    if (__any_sync(0xffffffffu, more)) {
#pragma unroll
      for (int a = 0; a < kMine; ++a) {
        const float mn = fmaxf(m[a], half_warp_max(fmaxf(fmaxf(x[a][0], x[a][1]), fmaxf(x[a][2], x[a][3]))));
        const float shrink = mn == -INFINITY ? 0.f : exp2f(m[a] - mn);
        m[a] = mn;
        l[a] *= shrink;
#pragma unroll
        for (int c = 0; c < kC; ++c)
#pragma unroll
          for (int i = 0; i < 2; ++i) acc[a][c][i] = __fmul2_rn(acc[a][c][i], make_float2(shrink, shrink));
      }
    }
#pragma unroll
    for (int a = 0; a < kMine; ++a) {
      const float base = m[a] == -INFINITY ? 0.f : m[a];
#pragma unroll
      for (int b = 0; b < 4; ++b) {
        const float p = exp2f(x[a][b] - base);
        l[a] += p;
        Ps[(ty + 16 * a) * kPPitch + tx + 16 * b] = p;     // written and read by one half warp
      }
    }
    arrived<1>();                                // V; the next K may still be on its way
    __syncthreads();
#pragma unroll 2
    for (int i = 0; i < kKeys; i += 4) {
      float4 v[4][kC];
#pragma unroll
      for (int j = 0; j < 4; ++j)
#pragma unroll
        for (int c = 0; c < kC; ++c) v[j][c] = *reinterpret_cast<const float4*>(Vs + (i + j) * kPitch + 4 * tx + 64 * c);
#pragma unroll
      for (int a = 0; a < kMine; ++a) {
        const float4 p4 = *reinterpret_cast<const float4*>(Ps + (ty + 16 * a) * kPPitch + i);
        const float p[4] = {p4.x, p4.y, p4.z, p4.w};
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
          for (int c = 0; c < kC; ++c) {
            acc[a][c][0] = __ffma2_rn(make_float2(v[j][c].x, v[j][c].y), make_float2(p[j], p[j]), acc[a][c][0]);
            acc[a][c][1] = __ffma2_rn(make_float2(v[j][c].z, v[j][c].w), make_float2(p[j], p[j]), acc[a][c][1]);
          }
      }
    }
    __syncthreads();
    ask_values(t + 1);
  }
  arrived<0>();
#pragma unroll
  for (int a = 0; a < kMine; ++a) {
    const float sum = half_warp_sum(l[a]);
    const int r = r0 + ty + 16 * a;
    if (r >= A.n_rows) continue;
    const int64_t row = attn_row(A, s, r), at = (int64_t)(A.slot0 + split) * A.total_rows + row;
    const bool parts = A.n_slots > 1;
    const float inv = parts ? 1.f : sum == 0.f ? 0.f : 1.f / sum;
    if (parts && tx == 0) A.part_ml[at] = make_float2(m[a], sum);
    if (!parts && A.lse && tx == 0) A.lse[row] = sum == 0.f ? INFINITY : m[a] + log2f(sum);
    float* to = parts ? A.part + at * D : static_cast<float*>(A.out) + row * D;
#pragma unroll
    for (int c = 0; c < kC; ++c)
      *reinterpret_cast<float4*>(to + 4 * tx + 64 * c) = make_float4(acc[a][c][0].x * inv, acc[a][c][0].y * inv, acc[a][c][1].x * inv, acc[a][c][1].y * inv);
  }
}

template <bool kBf16, int D>
__global__ void __launch_bounds__(kThreads) attn_combine_kernel(const AttnRows A) {
  static_assert(kThreads == kJoinThreads, "");
  __shared__ JoinShared<D> sh;
  grid_wait_and_release();
  join_splits<kBf16, D, 8>(A, blockIdx.x, sh);
}

// 64 keys of a stream: their logits again, against every scored query that sees them, and the weights' sums.  The next tile of queries
// comes in while this one's weights are added up.
template <int D>
__global__ void __launch_bounds__(kThreads) score_simt_kernel(const AttnRows A, const ScoreArgs S, int key_tiles) {
  constexpr int kPitch = Tile<D>::kPitch;
  extern __shared__ __align__(16) float smem[];
  float *Qs = smem, *Ks = Qs + kRows * kPitch, *red = Ks + kKeys * kPitch, *lse = red + 16 * kKeys;
  __shared__ int limit[kRows];
  const int tid = threadIdx.x, ty = tid / 16, tx = tid % 16;
  const int s = blockIdx.x / key_tiles, k0 = blockIdx.x % key_tiles * kKeys;
  grid_wait_and_release();
  const int len = attn_len(A, s);
  if (k0 >= len) return;
  const int64_t first = (int64_t)s * A.cap;
  ask_tile<D>(Ks, A.K, kKeys, [&](int i) { return k0 + i < len ? first + k0 + i : (int64_t)-1; });
  commit();
  // scored row i of a stream: head i / n_scored, query n_queries - n_scored + i % n_scored
  const int rows = A.n_rows / A.n_queries * S.n_scored;
  auto query_row = [&](int i) { return i / S.n_scored * A.n_queries + A.n_queries - S.n_scored + i % S.n_scored; };
  auto next_tile = [&](int r0) {                 // the next one of which some row sees the keys
    for (; r0 < rows; r0 += kRows) {
      const int last = min(r0 + kRows, rows) - 1;
      if (r0 / S.n_scored != last / S.n_scored || attn_limit(A, len, query_row(last)) > k0) break;
    }
    return r0;
  };
  float see_lse = 0.f;
  int see = 0;
  auto ask = [&](int r0) {                       // and what thread r < kRows puts down for row r
    if (r0 < rows) {
      const int last = min(r0 + kRows, rows) - 1;
      ask_tile<D>(Qs, A.q, kRows, [&](int i) { return r0 + i <= last ? attn_row(A, s, query_row(r0 + i)) : (int64_t)-1; });
      if (tid < kRows) {
        const int r = query_row(min(r0 + tid, last));
        see = r0 + tid <= last ? attn_limit(A, len, r) : 0;
        see_lse = A.lse[attn_row(A, s, r)];
      }
    }
    commit();
  };
  float sum[4] = {0.f, 0.f, 0.f, 0.f};
  int r0 = next_tile(0);
  ask(r0);
  while (r0 < rows) {
    if (tid < kRows) {
      limit[tid] = see;
      lse[tid] = see_lse;
    }
    arrived<0>();
    __syncthreads();
    float x[kMine][4], part[4] = {0.f, 0.f, 0.f, 0.f}, off[kMine];
    int lim[kMine];
    dots<D>(Qs, Ks, ty, tx, x);
#pragma unroll
    for (int a = 0; a < kMine; ++a) {
      off[a] = lse[ty + 16 * a];
      lim[a] = limit[ty + 16 * a];
    }
    __syncthreads();
    r0 = next_tile(r0 + kRows);
    ask(r0);
#pragma unroll
    for (int a = 0; a < kMine; ++a)
#pragma unroll
      for (int b = 0; b < 4; ++b) part[b] += k0 + tx + 16 * b < lim[a] ? exp2f(fmaf(x[a][b], A.scale, -off[a])) : 0.f;
#pragma unroll
    for (int b = 0; b < 4; ++b) sum[b] += part[b];
  }
  arrived<0>();
#pragma unroll
  for (int b = 0; b < 4; ++b) red[ty * kKeys + tx + 16 * b] = sum[b];
  __syncthreads();
  if (tid < kKeys && k0 + tid < len) {
    float all = 0.f;
    for (int y = 0; y < 16; ++y) all += red[y * kKeys + tid];
    score_put(S, first + k0 + tid, all);
  }
}

template <class Kern, class... Args>
cudaError_t launch(Kern kern, std::atomic<unsigned long long>& devices, dim3 grid, size_t smem, cudaStream_t st, const Args&... args) {
  const cudaError_t e = kernel_limits(kern, smem, devices);
  if (e != cudaSuccess) return e;
  const PdlConfig pc(grid, kThreads, smem, st);
  return cudaLaunchKernelEx(&pc.cfg, kern, args...);
}
template <int D>
cudaError_t attn(const AttnRows& A, cudaStream_t st) {
  static std::atomic<unsigned long long> devices{0};
  const int tiles = simt_row_tiles(A.n_rows);
  return launch(attn_simt_kernel<D>, devices, dim3((unsigned)tiles * A.n_streams, A.splits), Tile<D>::kSmem, st, A, tiles);
}
template <int D>
cudaError_t score(const AttnRows& A, const ScoreArgs& S, cudaStream_t st) {
  static std::atomic<unsigned long long> devices{0};
  const int tiles = (A.cap + kKeys - 1) / kKeys;
  return launch(score_simt_kernel<D>, devices, dim3((unsigned)tiles * A.n_streams), Tile<D>::kSmem, st, A, S, tiles);
}
template <bool kBf16, int D>
cudaError_t combine(const AttnRows& A, cudaStream_t st) {
  const PdlConfig pc(dim3(join_ctas(A)), kThreads, 0, st);
  return cudaLaunchKernelEx(&pc.cfg, attn_combine_kernel<kBf16, D>, A);
}

}  // namespace

int simt_row_tiles(int n_rows) { return (n_rows + kRows - 1) / kRows; }

cudaError_t launch_attn_simt(const AttnRows& A, int d, cudaStream_t st) { return d == 128 ? attn<128>(A, st) : attn<64>(A, st); }

cudaError_t launch_attn_combine(const AttnRows& A, int d, int is_bf16, cudaStream_t st) {
  if (d == 128) return is_bf16 ? combine<true, 128>(A, st) : combine<false, 128>(A, st);
  return is_bf16 ? combine<true, 64>(A, st) : combine<false, 64>(A, st);
}

cudaError_t launch_score_simt(const AttnRows& A, const ScoreArgs& S, int d, cudaStream_t st) { return d == 128 ? score<128>(A, S, st) : score<64>(A, S, st); }

}  // namespace bkv
