// The weight that every row of a bf16 cache receives from many queries, on the 5th-generation tensor cores:
//
//   score_out_i = decay score_in_i + sum_r 2^(x_{r,i} - lse_r),   x_{r,i} = <q_r, k_i> log2(e) / sqrt d,
//
// over the counted query rows r that see row i, lse_r from the attention kernel's finished sums.  The logits are formed again (they
// would be 4 bytes per pair to keep, 2 d operations to form), transposed: S^T = K Q^T has the cached rows as TMEM lanes, so that a thread
// adds up one row's weights and no sum crosses threads.
//
// A CTA keeps 256 cached rows in shared memory (two tiles, two warpgroups each, which take half of a tile's queries, two buffers of
// 128 x 128 logits per tile) and walks
// the queries in tiles of 128, head by head, from the first tile that sees its rows on.  What bounds it are the exponentials: 32768 per
// tile of queries are 2048 cycles of the special-function unit against 1024 of products (d = 128), so a larger share of them than in the attention
// kernel is formed by FMAs.
// Warps: 0-7 and 8-15 the rows of the two tiles, 16 asks for K and the Q tiles (TMA) and loads their lse, 17 issues the MMAs.
// Every wait is bounded; one that gives up makes the scores NaN.
#include "attn_tc.cuh"

namespace bkv {

namespace {

using namespace tc;
using namespace mma;

constexpr int kThreads = 640;
// Registers of a thread at launch, and what the warps go on with: 16 x 104 + 4 x 56 <= 20 x 96.
constexpr int kRegs = 96, kRegsRows = 104, kRegsOther = 56;
static_assert(16 * kRegsRows + 4 * kRegsOther <= 20 * kRegs && kThreads * kRegs <= 65536, "a register split beyond the launch's waits forever");

template <int D>
struct Shape {
  static constexpr uint32_t kBox = 128 * 128;
  static constexpr uint32_t kTile = (D / 64) * kBox;
  static constexpr int kRing = D == 128 ? 4 : 8;
  static constexpr int kLse = 16;                // tiles of lse: more than the ring and the buffers of logits hold
  static constexpr size_t kSmem = 1024 + (2 + kRing) * (size_t)kTile;
};

template <int D>
__global__ void __maxnreg__(kRegs)
score_tc_kernel(const __grid_constant__ AttnRows A, const ScoreArgs C, int blocks, const __grid_constant__ CUtensorMap mq, const __grid_constant__ CUtensorMap mk) {
  using Sh = Shape<D>;
  constexpr int kRing = Sh::kRing;
  extern __shared__ unsigned char smem_raw[];
  __shared__ uint64_t k_full, q_full[kRing], q_empty[kRing], lse_full[Sh::kLse], s_full[2][2], s_empty[2][2], drained;
  __shared__ uint32_t tmem_s;
  __shared__ int abort_flag;
  __shared__ __align__(16) float lse[Sh::kLse][kTcRows];      // negative
  __shared__ float half[2][kTcKeys];
  unsigned char* sm = smem_raw + (-smem_u32(smem_raw) & 1023u);
  unsigned char* ring = sm + 2 * Sh::kTile;
  const int tid = threadIdx.x, warp = __shfl_sync(0xffffffffu, tid / 32, 0), lane = tid % 32;
  if (tid == 0) {
    mbar_init(&k_full, 1);
    mbar_init(&drained, 1);
    for (int i = 0; i < kRing; ++i) { mbar_init(q_full + i, 1); mbar_init(q_empty + i, 1); }
    for (int i = 0; i < Sh::kLse; ++i) mbar_init(lse_full + i, 32);
    for (int i = 0; i < 4; ++i) { mbar_init(&s_full[0][0] + i, 1); mbar_init(&s_empty[0][0] + i, 256); }
    abort_flag = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
  }
  if (warp == 17) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&tmem_s)), "r"(512u) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  grid_wait_and_release();
  // the first cached rows, which the most queries see, first
  const int s = blockIdx.x % A.n_streams, key0 = blockIdx.x / A.n_streams * 2 * kTcKeys;
  const int len = attn_len(A, s), m = A.n_queries, heads = A.n_rows / m;
  // query j sees row i if i <= len - m + j: the tiles of a head start behind the queries that see no row of the CTA's
  const int first = m - C.n_scored, skip = max(0, key0 - (len - m) - first) / kTcRows * kTcRows;
  const int start = first + skip, per_head = max(0, (m - start + kTcRows - 1) / kTcRows);
  const int n = key0 < len ? heads * per_head : 0;
  const int tiles = key0 + kTcKeys < len ? 2 : 1;
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = __shfl_sync(0xffffffffu, tmem_s, 0);

  if (warp >= 16) {
    regs_down<kRegsOther>();
    if (warp == 16 && n > 0) {
      bool ok = true;
      if (lane == 0) {
        mbar_expect_tx(&k_full, tiles * Sh::kTile);
        for (int t = 0; t < tiles; ++t)
          for (int b = 0; b < D / 64; ++b) tma_load_3d(sm + t * Sh::kTile + b * Sh::kBox, &mk, 64 * b, key0 + t * kTcKeys, s, &k_full);
      }
      int i = 0;
      for (; i < n; ++i) {
        const int slot = i % kRing, head = i / per_head, j = start + i % per_head * kTcRows;
        if (i >= kRing) ok = wait_bar(q_empty + slot, (uint32_t)(i / kRing - 1) & 1u, &abort_flag);
        if (!__all_sync(0xffffffffu, ok)) break;
        if (lane == 0) {
          mbar_expect_tx(q_full + slot, Sh::kTile);
          for (int b = 0; b < D / 64; ++b) tma_load_3d(ring + slot * Sh::kTile + b * Sh::kBox, &mq, 64 * b, j, s * heads + head, q_full + slot);
        }
        // rows behind the head's last are zeros, of weight zero.  (The place's last readers are done: the entry kRing before has been
        // multiplied, and so the logits two before that read.)
        float* to = lse[i % Sh::kLse];
#pragma unroll
        for (int c = 0; c < kTcRows / 32; ++c) {
          const int q = j + lane + 32 * c;
          to[lane + 32 * c] = q < m ? -A.lse[((int64_t)s * heads + head) * m + q] : -INFINITY;
        }
        mbar_arrive(lse_full + i % Sh::kLse);
        __syncwarp();
      }
      if (i < n && lane == 0) {                  // gave up: the copies in flight, within limits
        const long long t0 = clock64();
        while (!mbar_try_wait(&k_full, 0) && clock64() - t0 < kWaitCycles) {}
        for (int e = max(0, i - kRing); e < i; ++e)
          while (!mbar_try_wait(q_full + e % kRing, (uint32_t)(e / kRing) & 1u) && clock64() - t0 < kWaitCycles) {}
      }
    } else if (warp == 17 && n > 0) {
      bool ok = true;
      auto wait = [&](uint64_t* bar, uint32_t parity) { ok = ok && __all_sync(0xffffffffu, wait_bar(bar, parity, &abort_flag)); };
      wait(&k_full, 0);
      for (int i = 0; i < n && ok; ++i) {
        wait(q_full + i % kRing, (uint32_t)(i / kRing) & 1u);
        for (int t = 0; t < tiles && ok; ++t) {
          if (i > 1) wait(&s_empty[t][i & 1], (uint32_t)(i / 2 - 1) & 1u);
          tc_fence_after();
          if (ok && elect_one()) {
            const uint32_t a = umma_desc_lo(smem_u32(sm + t * Sh::kTile)), b = umma_desc_lo(smem_u32(ring + i % kRing * Sh::kTile));
            const uint32_t d = tmem + 256 * t + 128 * (i & 1);
#pragma unroll
            for (int k = 0; k < D / 16; ++k) {
              const uint32_t at = (uint32_t)(k / 4) * (Sh::kBox >> 4) + 2 * (k % 4);
              if (k == 0) umma_bf16<0>(d, a + at, b + at);
              else umma_bf16<1>(d, a + at, b + at);
            }
            umma_commit(&s_full[t][i & 1]);
            if (t == tiles - 1) umma_commit(q_empty + i % kRing);
          }
          __syncwarp();
        }
      }
      if (!ok) {                                 // gave up: the products in flight, within limits
        if (elect_one()) umma_commit(&drained);
        st_release(&abort_flag, 1);
        const long long t0 = clock64();
        while (!mbar_try_wait(&drained, 0) && clock64() - t0 < kWaitCycles) {}
      }
    }
  } else {
    regs_up<kRegsRows>();
    const int t = warp / 8, h = warp / 4 % 2, lanes = 32 * (warp % 4), key = key0 + t * kTcKeys + lanes + lane;
    const uint32_t S = tmem + ((uint32_t)lanes << 16) + 256 * t + 64 * h;
    const float2 scale2 = make_float2(A.scale, A.scale);
    float sum = 0.f;
    bool ok = true;
    if (t < tiles) {
      for (int i = 0; i < n; ++i) {
        ok = __all_sync(0xffffffffu, wait_bar(&s_full[t][i & 1], (uint32_t)(i / 2) & 1u, &abort_flag) && wait_bar(lse_full + i % Sh::kLse, (uint32_t)(i / Sh::kLse) & 1u, &abort_flag));
        if (!ok) break;
        tc_fence_after();
        float x[2][32];
#pragma unroll
        for (int c = 0; c < 2; ++c) tmem_ld32(S + 128 * (i & 1) + 32 * c, x[c]);
        tmem_ld_wait();
        tc_fence_before();
        mbar_arrive(&s_empty[t][i & 1]);
        const int j = start + i % per_head * kTcRows + 64 * h;
        const int from = key - (len - m) - j;    // the half tile's first query that sees the row
        const bool masked = key0 + (t + 1) * kTcKeys - 1 > len - m + j;
        const float4* l4 = reinterpret_cast<const float4*>(lse[i % Sh::kLse] + 64 * h);
        float2 part[2] = {};
        auto weights = [&](auto mask) {
#pragma unroll
          for (int c = 0; c < 2; ++c)
#pragma unroll
            for (int k = 0; k < 32; k += 4) {
              const float4 l = l4[(32 * c + k) / 4];
              const float2 lo = __ffma2_rn(make_float2(x[c][k], x[c][k + 1]), scale2, make_float2(l.x, l.y));
              const float2 hi = __ffma2_rn(make_float2(x[c][k + 2], x[c][k + 3]), scale2, make_float2(l.z, l.w));
              if constexpr (decltype(mask)::value) {
                const int q = 32 * c + k;
                part[0].x += (q >= from ? ex2(lo.x) : 0.f) + (q + 2 >= from ? ex2(hi.x) : 0.f);
                part[0].y += (q + 1 >= from ? ex2(lo.y) : 0.f) + (q + 3 >= from ? ex2(hi.y) : 0.f);
              } else {
                part[0] = __fadd2_rn(part[0], make_float2(ex2(lo.x), ex2(lo.y)));
                part[1] = __fadd2_rn(part[1], (k / 4) % 4 != 3 ? make_float2(ex2(hi.x), ex2(hi.y)) : exp2_fma(hi));    // an eighth of the pairs
              }
            }
        };
        if (masked) weights(std::true_type{});
        else weights(std::false_type{});
        sum += (part[0].x + part[0].y) + (part[1].x + part[1].y);
      }
    }
    if (!ok) sum = NAN;
    if (h == 1) half[t][lanes + lane] = sum;
    asm volatile("bar.sync 1, 512;" ::: "memory");         // the row warps
    if (h == 0 && key < len) score_put(C, (int64_t)s * A.cap + key, sum + half[t][lanes + lane]);
    tc_fence_before();
  }
  __syncthreads();
  tc_fence_after();
  if (warp == 17) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512u) : "memory");
}

template <int D>
cudaError_t launch(const AttnRows& A, const ScoreArgs& S, cudaStream_t st) {
  CUtensorMap mq, mk;
  cudaError_t e = cache_map(&mq, A.q, true, D, A.n_queries, A.total_rows / A.n_queries, kTcRows);
  if (e == cudaSuccess) e = cache_map(&mk, A.K, true, D, A.cap, A.n_streams, kTcKeys);
  static std::atomic<unsigned long long> devices{0};
  if (e == cudaSuccess) e = kernel_limits(score_tc_kernel<D>, Shape<D>::kSmem, false, devices);
  if (e != cudaSuccess) return e;
  const int blocks = (A.cap + 2 * kTcKeys - 1) / (2 * kTcKeys);
  const PdlConfig pc(dim3((unsigned)blocks * A.n_streams), kThreads, Shape<D>::kSmem, st);
  return cudaLaunchKernelEx(&pc.cfg, score_tc_kernel<D>, A, S, blocks, mq, mk);
}

}  // namespace

cudaError_t launch_score_tc(const AttnRows& A, const ScoreArgs& S, int d, cudaStream_t st) {
  return d == 128 ? launch<128>(A, S, st) : launch<64>(A, S, st);
}

}  // namespace bkv
