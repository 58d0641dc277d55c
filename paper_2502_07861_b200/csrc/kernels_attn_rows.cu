// Attention of any number of query rows over a caller-held cache on CUDA cores, its score pass, and the kernel that joins splits.
//
//   x_{r,i} = <q_r, k_i> log2(e) / sqrt d + log2 w_i,   out_r = sum_i 2^(x_{r,i} - m_r) v_i / sum_i 2^(x_{r,i} - m_r)
//
// over the rows that r sees, with a running maximum m_r, so that the cache is read once.  A CTA of 256 threads takes 64 query rows
// and walks its share of the keys in tiles of 64; a thread forms 4 x 4 logits, then 4 rows x d / 16 columns of the outputs, both
// from tiles in shared memory in fp32.
#include "attn_rows.cuh"

namespace bkv {

namespace {

constexpr int kRows = 64, kKeys = 64, kThreads = 256;

template <int D>
struct Tile {
  static constexpr int kPitch = D + 4;       // floats: rows 16 bytes aligned, neighbours in other banks
  static constexpr int kPPitch = kKeys + 4;
  static constexpr size_t kSmem = sizeof(float) * (size_t)(kRows * kPitch + 2 * kKeys * kPitch + kRows * kPPitch + kKeys);
};

template <bool kBf16>
__device__ inline const void* row_ptr(const void* base, int64_t row, int d) {
  return static_cast<const char*>(base) + row * d * (kBf16 ? 2 : 4);
}

// rows x D of a tile into shared memory as fp32; row i of the tile is row at(i) of base, or zeros where at(i) < 0.
template <bool kBf16, int D, class At>
__device__ inline void load_tile(float* sm, const void* base, int rows, At at) {
  for (int i = threadIdx.x; i < rows * (D / 8); i += kThreads) {
    const int row = i / (D / 8), e = i % (D / 8) * 8;
    float v[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    const int64_t from = at(row);
    if (from >= 0) load8<kBf16>(row_ptr<kBf16>(base, from, D), e, v);
    float4* to = reinterpret_cast<float4*>(sm + row * Tile<D>::kPitch + e);
    to[0] = make_float4(v[0], v[1], v[2], v[3]);
    to[1] = make_float4(v[4], v[5], v[6], v[7]);
  }
}

// acc[a][b] += <X row ty + 16 a, Y row tx + 16 b>
template <int D>
__device__ inline void dots(const float* X, const float* Y, int ty, int tx, float (&acc)[4][4]) {
#pragma unroll 4
  for (int e = 0; e < D; e += 4) {
    float4 x[4], y[4];
#pragma unroll
    for (int a = 0; a < 4; ++a) x[a] = *reinterpret_cast<const float4*>(X + (ty + 16 * a) * Tile<D>::kPitch + e);
#pragma unroll
    for (int b = 0; b < 4; ++b) y[b] = *reinterpret_cast<const float4*>(Y + (tx + 16 * b) * Tile<D>::kPitch + e);
#pragma unroll
    for (int a = 0; a < 4; ++a)
#pragma unroll
      for (int b = 0; b < 4; ++b)
        acc[a][b] = fmaf(x[a].x, y[b].x, fmaf(x[a].y, y[b].y, fmaf(x[a].z, y[b].z, fmaf(x[a].w, y[b].w, acc[a][b]))));
  }
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

template <bool kBf16, int D>
__global__ void __launch_bounds__(kThreads) attn_simt_kernel(const AttnRows A, int row_tiles) {
  constexpr int kPitch = Tile<D>::kPitch, kPPitch = Tile<D>::kPPitch, kCols = D / 16;
  extern __shared__ __align__(16) float smem[];
  float *Qs = smem, *Ks = Qs + kRows * kPitch, *Vs = Ks + kKeys * kPitch, *Ps = Vs + kKeys * kPitch, *lw = Ps + kRows * kPPitch;
  const int tid = threadIdx.x, ty = tid / 16, tx = tid % 16;
  const int s = blockIdx.x / row_tiles, r0 = blockIdx.x % row_tiles * kRows, split = blockIdx.y;
  grid_wait_and_release();
  const int len = attn_len(A, s);
  const int last = min(r0 + kRows, A.n_rows) - 1;
  const int most = r0 / A.n_queries != last / A.n_queries ? len : attn_limit(A, len, last);      // of the tile's rows
  const int tiles = (most + kKeys - 1) / kKeys;
  const int t0 = (int)((int64_t)tiles * split / A.splits), t1 = (int)((int64_t)tiles * (split + 1) / A.splits);
  load_tile<kBf16, D>(Qs, A.q, kRows, [&](int i) { return r0 + i < A.n_rows ? attn_row(A, s, r0 + i) : (int64_t)-1; });
  int limit[4];
  float m[4], l[4], acc[4][kCols];
#pragma unroll
  for (int a = 0; a < 4; ++a) {
    limit[a] = attn_limit(A, len, min(r0 + ty + 16 * a, A.n_rows - 1));
    m[a] = -INFINITY;
    l[a] = 0.f;
#pragma unroll
    for (int c = 0; c < kCols; ++c) acc[a][c] = 0.f;
  }
  const int64_t first = (int64_t)s * A.cap;
  for (int t = t0; t < t1; ++t) {
    const int k0 = t * kKeys;
    __syncthreads();
    if (tid < kKeys) lw[tid] = A.w && k0 + tid < len ? log2f(A.w[first + k0 + tid]) : 0.f;
    load_tile<kBf16, D>(Ks, A.K, kKeys, [&](int i) { return k0 + i < len ? first + k0 + i : (int64_t)-1; });
    // a row of weight zero counts as absent, whatever it holds
    load_tile<kBf16, D>(Vs, A.V, kKeys, [&](int i) { return k0 + i < len && !(A.w && A.w[first + k0 + i] == 0.f) ? first + k0 + i : (int64_t)-1; });
    __syncthreads();
    float x[4][4] = {};
    dots<D>(Qs, Ks, ty, tx, x);
#pragma unroll
    for (int a = 0; a < 4; ++a) {
      float top = -INFINITY;
#pragma unroll
      for (int b = 0; b < 4; ++b) {
        const float add = lw[tx + 16 * b];
        x[a][b] = k0 + tx + 16 * b < limit[a] && add != -INFINITY ? fmaf(x[a][b], A.scale, add) : -INFINITY;
        top = fmaxf(top, x[a][b]);
      }
      const float mn = fmaxf(m[a], half_warp_max(top)), base = mn == -INFINITY ? 0.f : mn;
      const float shrink = exp2f(m[a] - base);
      float sum = 0.f;
#pragma unroll
      for (int b = 0; b < 4; ++b) {
        const float p = exp2f(x[a][b] - base);
        sum += p;
        Ps[(ty + 16 * a) * kPPitch + tx + 16 * b] = p;
      }
      l[a] = fmaf(l[a], shrink, half_warp_sum(sum));
      m[a] = mn;
#pragma unroll
      for (int c = 0; c < kCols; ++c) acc[a][c] *= shrink;
    }
    __syncwarp();                            // a row of P is written and read by one half warp
#pragma unroll 4
    for (int i = 0; i < kKeys; ++i) {
      float4 v[kCols / 4];
#pragma unroll
      for (int c = 0; c < kCols / 4; ++c) v[c] = *reinterpret_cast<const float4*>(Vs + i * kPitch + 4 * tx + 64 * c);
#pragma unroll
      for (int a = 0; a < 4; ++a) {
        const float p = Ps[(ty + 16 * a) * kPPitch + i];
#pragma unroll
        for (int c = 0; c < kCols / 4; ++c) {
          acc[a][4 * c] = fmaf(p, v[c].x, acc[a][4 * c]);
          acc[a][4 * c + 1] = fmaf(p, v[c].y, acc[a][4 * c + 1]);
          acc[a][4 * c + 2] = fmaf(p, v[c].z, acc[a][4 * c + 2]);
          acc[a][4 * c + 3] = fmaf(p, v[c].w, acc[a][4 * c + 3]);
        }
      }
    }
  }
#pragma unroll
  for (int a = 0; a < 4; ++a) {
    const int r = r0 + ty + 16 * a;
    if (r >= A.n_rows) continue;
    const int64_t row = attn_row(A, s, r);
    if (A.n_slots > 1) {
      const int64_t at = (int64_t)(A.slot0 + split) * A.total_rows + row;
      if (tx == 0) A.part_ml[at] = make_float2(m[a], l[a]);
#pragma unroll
      for (int c = 0; c < kCols / 4; ++c)
        *reinterpret_cast<float4*>(A.part + at * D + 4 * tx + 64 * c) = make_float4(acc[a][4 * c], acc[a][4 * c + 1], acc[a][4 * c + 2], acc[a][4 * c + 3]);
      continue;
    }
    const float inv = l[a] == 0.f ? 0.f : 1.f / l[a];
    if (A.lse && tx == 0) A.lse[row] = l[a] == 0.f ? INFINITY : m[a] + log2f(l[a]);
#pragma unroll
    for (int c = 0; c < kCols; c += 4) {
      const int at = 4 * tx + 16 * c;
      if constexpr (kBf16) {
        __nv_bfloat162* to = reinterpret_cast<__nv_bfloat162*>(static_cast<__nv_bfloat16*>(A.out) + row * D + at);
        to[0] = __floats2bfloat162_rn(acc[a][c] * inv, acc[a][c + 1] * inv);
        to[1] = __floats2bfloat162_rn(acc[a][c + 2] * inv, acc[a][c + 3] * inv);
      } else {
        *reinterpret_cast<float4*>(static_cast<float*>(A.out) + row * D + at) =
            make_float4(acc[a][c] * inv, acc[a][c + 1] * inv, acc[a][c + 2] * inv, acc[a][c + 3] * inv);
      }
    }
  }
}

template <bool kBf16, int D>
__global__ void __launch_bounds__(kThreads) attn_combine_kernel(const AttnRows A) {
  static_assert(kThreads == kJoinThreads, "");
  __shared__ JoinShared<D> sh;
  grid_wait_and_release();
  join_splits<kBf16, D, 8>(A, blockIdx.x, sh);
}

// 64 keys of a stream: their logits again, against every scored query that sees them, and the weights' sums.
template <bool kBf16, int D>
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
  load_tile<kBf16, D>(Ks, A.K, kKeys, [&](int i) { return k0 + i < len ? first + k0 + i : (int64_t)-1; });
  // scored row i of a stream: head i / n_scored, query n_queries - n_scored + i % n_scored
  const int rows = A.n_rows / A.n_queries * S.n_scored;
  auto query_row = [&](int i) { return i / S.n_scored * A.n_queries + A.n_queries - S.n_scored + i % S.n_scored; };
  float sum[4] = {0.f, 0.f, 0.f, 0.f};
  for (int r0 = 0; r0 < rows; r0 += kRows) {
    const int last = min(r0 + kRows, rows) - 1;
    if (r0 / S.n_scored == last / S.n_scored && attn_limit(A, len, query_row(last)) <= k0) continue;
    __syncthreads();
    if (tid < kRows) {
      const int r = query_row(min(r0 + tid, last));
      limit[tid] = r0 + tid <= last ? attn_limit(A, len, r) : 0;
      lse[tid] = A.lse[attn_row(A, s, r)];
    }
    load_tile<kBf16, D>(Qs, A.q, kRows, [&](int i) { return r0 + i <= last ? attn_row(A, s, query_row(r0 + i)) : (int64_t)-1; });
    __syncthreads();
    float x[4][4] = {}, part[4] = {0.f, 0.f, 0.f, 0.f};
    dots<D>(Qs, Ks, ty, tx, x);
#pragma unroll
    for (int a = 0; a < 4; ++a)
#pragma unroll
      for (int b = 0; b < 4; ++b)
        part[b] += k0 + tx + 16 * b < limit[ty + 16 * a] ? exp2f(fmaf(x[a][b], A.scale, -lse[ty + 16 * a])) : 0.f;
#pragma unroll
    for (int b = 0; b < 4; ++b) sum[b] += part[b];
  }
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
template <bool kBf16, int D>
cudaError_t attn(const AttnRows& A, dim3 grid, int tiles, cudaStream_t st) {
  static std::atomic<unsigned long long> devices{0};
  return launch(attn_simt_kernel<kBf16, D>, devices, grid, Tile<D>::kSmem, st, A, tiles);
}
template <bool kBf16, int D>
cudaError_t score(const AttnRows& A, const ScoreArgs& S, dim3 grid, int tiles, cudaStream_t st) {
  static std::atomic<unsigned long long> devices{0};
  return launch(score_simt_kernel<kBf16, D>, devices, grid, Tile<D>::kSmem, st, A, S, tiles);
}
template <bool kBf16, int D>
cudaError_t combine(const AttnRows& A, cudaStream_t st) {
  const PdlConfig pc(dim3(join_ctas(A)), kThreads, 0, st);
  return cudaLaunchKernelEx(&pc.cfg, attn_combine_kernel<kBf16, D>, A);
}

}  // namespace

cudaError_t launch_attn_simt(const AttnRows& A, int d, int is_bf16, cudaStream_t st) {
  const int tiles = (A.n_rows + kRows - 1) / kRows;
  const dim3 grid((unsigned)tiles * A.n_streams, A.splits);
  if (d == 128) return is_bf16 ? attn<true, 128>(A, grid, tiles, st) : attn<false, 128>(A, grid, tiles, st);
  return is_bf16 ? attn<true, 64>(A, grid, tiles, st) : attn<false, 64>(A, grid, tiles, st);
}

cudaError_t launch_attn_combine(const AttnRows& A, int d, int is_bf16, cudaStream_t st) {
  if (d == 128) return is_bf16 ? combine<true, 128>(A, st) : combine<false, 128>(A, st);
  return is_bf16 ? combine<true, 64>(A, st) : combine<false, 64>(A, st);
}

cudaError_t launch_score_simt(const AttnRows& A, const ScoreArgs& S, int d, int is_bf16, cudaStream_t st) {
  const int tiles = (A.cap + kKeys - 1) / kKeys;
  const dim3 grid((unsigned)tiles * A.n_streams);
  if (d == 128) return is_bf16 ? score<true, 128>(A, S, grid, tiles, st) : score<false, 128>(A, S, grid, tiles, st);
  return is_bf16 ? score<true, 64>(A, S, grid, tiles, st) : score<false, 64>(A, S, grid, tiles, st);
}

}  // namespace bkv
