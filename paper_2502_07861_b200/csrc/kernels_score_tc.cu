// The weight that every row of a bf16 cache receives from many queries, on the 5th-generation tensor cores:
//
//   score_out_i = decay score_in_i + sum_r 2^(x_{r,i} - lse_r),   x_{r,i} = <q_r, k_i> log2(e) / sqrt d,
//
// over the counted query rows r that see row i, lse_r from the attention kernel's finished sums.  The logits are formed again: kept,
// they would be 4 bytes per pair to write and to read, formed again they are 2 d operations.
//
// score_tc_kernel: a CTA keeps 128 cached rows in shared memory and walks the queries in tiles of 128, head by head, from the first tile
// that sees its rows on; where at most 64 queries of more heads count, a tile has several heads'.  S = Q K^T has the queries as TMEM lanes, so that a
// thread has one query, its lse is a register and its weights are added to 128 sums of its own, which meet the other threads' only at
// the end: a pair costs a multiply-add, an exponential and an addition.  (With the cached rows as lanes every pair also needs its
// query's lse from shared memory, whose loads share a queue with the exponentials: 345 us for a prompt of 8192 queries and 32 heads, 321 so.)
// Two pairs of warpgroups take tiles in turn, half of the cached rows each, from four buffers of 128 x 128 logits in TMEM.
// Where there are few CTAs the tiles are shared out to a cluster, whose sums meet in shared memory.
// No pipe bounds it (40 streams of 8192 rows, 512 queries x 4 heads: exponentials take 52 % of theirs, products 32 %, instructions issue in half of
// the cycles): the row warps wait for TMEM, of which one load of 8 columns is on its way; registers hold no more beside the sums.  A quarter
// of the exponentials is formed by FMAs, which saves a little of the special-function unit's queue (a prompt of 8192 queries and 32 heads with its
// attention: 866 us so, 874 without).
// Warps: 0-7 and 8-15 the queries of even and odd tiles, 16 asks for K and the Q tiles (TMA), 17 issues the MMAs.
// Every wait is bounded; one that gives up makes the scores NaN.
#include <cooperative_groups.h>

#include <algorithm>
#include <type_traits>

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
  static constexpr int kRing = D == 128 ? 5 : 8;
  static constexpr size_t kSmem = 1024 + (1 + kRing) * (size_t)kTile;
};

template <int D>
__global__ void __maxnreg__(kRegs)
score_tc_kernel(const __grid_constant__ AttnRows A, const ScoreArgs C, int box_rows, const __grid_constant__ CUtensorMap mq, const __grid_constant__ CUtensorMap mk) {
  namespace cg = cooperative_groups;
  using Sh = Shape<D>;
  constexpr int kRing = Sh::kRing;
  extern __shared__ unsigned char smem_raw[];
  __shared__ uint64_t k_full, q_full[kRing], q_empty[kRing], s_full[4], s_empty[4], drained;
  __shared__ uint32_t tmem_s;
  __shared__ int abort_flag;
  __shared__ float sums[8][kTcKeys];             // of the row warps' queries
  __shared__ float total[kTcKeys];               // of the CTA
  unsigned char* sm = smem_raw + (-smem_u32(smem_raw) & 1023u);
  unsigned char* ring = sm + Sh::kTile;
  cg::cluster_group cluster = cg::this_cluster();
  const int tid = threadIdx.x, warp = __shfl_sync(0xffffffffu, tid / 32, 0), lane = tid % 32;
  const int pack = kTcRows / box_rows;           // heads of a tile
  if (tid == 0) {
    mbar_init(&k_full, 1);
    mbar_init(&drained, 1);
    for (int i = 0; i < kRing; ++i) { mbar_init(q_full + i, 1); mbar_init(q_empty + i, 1); }
    for (int i = 0; i < 4; ++i) { mbar_init(s_full + i, 1); mbar_init(s_empty + i, 256); }
    abort_flag = 0;
    asm volatile("prefetch.tensormap [%0];" ::"l"(&mq) : "memory");
    asm volatile("prefetch.tensormap [%0];" ::"l"(&mk) : "memory");
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
  }
  if (warp == 17) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&tmem_s)), "r"(512u) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  // The first loads do not wait for the attention kernel to end: it writes lse alone of what is read here, and what came before it is
  // complete.  (Before a wait that hangs on the row warps, whose limit the attention kernel's time would count towards, everybody does.)
  const int s = blockIdx.x % A.n_streams, key0 = blockIdx.x / A.n_streams * kTcKeys;             // the first cached rows, which the most queries see, first
  const int len = attn_len(A, s), m = A.n_queries, heads = A.n_rows / m;
  // Query j sees row i if i <= len - m + j: the tiles of a head start behind the queries that see no row of the CTA's.
  const int first = m - C.n_scored, skip = pack > 1 ? 0 : max(0, key0 - (len - m) - first) / kTcRows * kTcRows;
  const int start = first + skip, per_head = max(0, (m - start + box_rows - 1) / box_rows);
  const int n_all = key0 < len ? pack > 1 ? (heads + pack - 1) / pack : heads * per_head : 0;
  const int i0 = (int)((int64_t)n_all * blockIdx.y / gridDim.y), n = (int)((int64_t)n_all * (blockIdx.y + 1) / gridDim.y) - i0;      // this CTA's
  // Of the CTA's tiles, one after the other: the first head and its first query.
  struct Walk {
    int head, query, start, end, pack;
    __device__ void next() {
      if (pack > 1) head += pack;
      else if ((query += kTcRows) >= end) { query = start; ++head; }
    }
  };
  auto walk = [&]() { return pack > 1 ? Walk{i0 * pack, start, start, m, pack} : Walk{n ? i0 / per_head : 0, n ? start + i0 % per_head * kTcRows : 0, start, m, 1}; };
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = __shfl_sync(0xffffffffu, tmem_s, 0);

  if (warp >= 16) {
    regs_down<kRegsOther>();
    if (warp == 16 && n > 0) {
      bool ok = true;
      if (lane == 0) {
        mbar_expect_tx(&k_full, Sh::kTile);
        for (int b = 0; b < D / 64; ++b) tma_load_3d(sm + b * Sh::kBox, &mk, 64 * b, key0, s, &k_full);
      }
      Walk at = walk();
      int i = 0;
      for (; i < n; ++i, at.next()) {
        const int slot = i % kRing;
        if (i == kRing) grid_wait_and_release();
        if (i >= kRing) ok = wait_bar(q_empty + slot, (uint32_t)(i / kRing - 1) & 1u, &abort_flag);
        if (!__all_sync(0xffffffffu, ok)) break;
        if (lane == 0) {
          const int boxes = min(pack, heads - at.head);      // (lanes that no head's queries fill are not read)
          mbar_expect_tx(q_full + slot, (uint32_t)boxes * box_rows * 2 * D);
          for (int h = 0; h < boxes; ++h)
            for (int b = 0; b < D / 64; ++b)
              tma_load_3d(ring + slot * Sh::kTile + b * Sh::kBox + h * box_rows * 128, &mq, 64 * b, at.query, s * heads + at.head + h, q_full + slot);
        }
        __syncwarp();
      }
      if (lane == 0) {
        copy_landed(&k_full);
        copies_landed(q_full, i);
      }
    } else if (warp == 17 && n > 0) {
      bool ok = true;
      auto wait = [&](uint64_t* bar, uint32_t parity) { ok = ok && __all_sync(0xffffffffu, wait_bar(bar, parity, &abort_flag)); };
      grid_wait_and_release();
      wait(&k_full, 0);
      for (int i = 0; i < n && ok; ++i) {
        wait(q_full + i % kRing, (uint32_t)(i / kRing) & 1u);
        if (i > 3) wait(s_empty + (i & 3), (uint32_t)(i / 4 - 1) & 1u);
        tc_fence_after();
        if (ok && elect_one()) {
          const uint32_t a = umma_desc_lo(smem_u32(ring + i % kRing * Sh::kTile)), b = umma_desc_lo(smem_u32(sm)), d = tmem + 128 * (i & 3);
#pragma unroll
          for (int k = 0; k < D / 16; ++k) {
            const uint32_t at = (uint32_t)(k / 4) * (Sh::kBox >> 4) + 2 * (k % 4);
            if (k == 0) umma_bf16<0>(d, a + at, b + at);
            else umma_bf16<1>(d, a + at, b + at);
          }
          umma_commit(s_full + (i & 3));
          umma_commit(q_empty + i % kRing);
        }
        __syncwarp();
      }
      if (!ok) st_release(&abort_flag, 1);
      products_done(&drained);
    }
  } else {
    regs_up<kRegsRows>();
    constexpr int kMine = kTcKeys / 2;           // columns of a warp
    const int turn = warp / 8, half = warp / 4 % 2, lanes = 32 * (warp % 4), r = lanes + lane;
    const int in_head = pack > 1 ? r / box_rows : 0, in_query = pack > 1 ? r % box_rows : r;
    const uint32_t S = tmem + ((uint32_t)lanes << 16) + kMine * half;
    const float2 scale2 = make_float2(A.scale, A.scale);
    float2 acc[kMine / 2];                       // this thread's queries' weights of the warp's half of the CTA's rows
#pragma unroll
    for (int c = 0; c < kMine / 2; ++c) acc[c] = make_float2(0.f, 0.f);
    grid_wait_and_release();
    // of this thread's query in a tile: lse, and how many of the warp's rows it sees.  (Nothing is done with lse before it is used, a tile
    // later: its sign changed here kept every tile waiting for it, 460 of 2530 cycles.)
    auto look = [&](const Walk& at, bool held, float& raw, int& sees) {
      const int h = at.head + in_head, q = at.query + in_query;
      const bool counts = held && in_head < pack && h < heads && q < m;
      raw = INFINITY;
      if (counts) raw = A.lse[((int64_t)s * heads + h) * m + q];
      sees = counts ? len - m + q + 1 - key0 - kMine * half : 0;
    };
    Walk at = walk();
    if (turn) at.next();
    float next_lse;
    int next_sees;
    look(at, turn < n, next_lse, next_sees);
    // A tile is taken 8 columns at a time, the next ones on their way from TMEM while these are worked on -- behind the last ones, those of
    // the warpgroup's next tile.
    constexpr int kChunk = 8, kChunks = kMine / kChunk;
    float x[2][kChunk];
    auto begin = [&](int i) {
      const bool ok = __all_sync(0xffffffffu, wait_bar(s_full + (i & 3), (uint32_t)(i / 4) & 1u, &abort_flag));
      if (ok) {
        tc_fence_after();
        tmem_ld8(S + 128 * (i & 3), x[0]);
      }
      return ok;
    };
    bool ok = turn >= n || begin(turn);
    for (int i = turn; i < n && ok; i += 2) {
      const float off = -next_lse;
      const int sees = next_sees;
      at.next();
      at.next();
      look(at, i + 2 < n, next_lse, next_sees);  // (a tile ahead)
      const float2 off2 = make_float2(off, off);
      auto weights = [&](auto mask) {
#pragma unroll
        for (int c = 0; c < kChunks; ++c) {
          tmem_ld_wait();
          if (c + 1 < kChunks) {
            tmem_ld8(S + 128 * (i & 3) + kChunk * (c + 1), x[(c + 1) & 1]);
          } else {
            tc_fence_before();
            mbar_arrive(s_empty + (i & 3));
            if (i + 2 < n) ok = begin(i + 2);
          }
#pragma unroll
          for (int k = 0; k < kChunk; k += 2) {
            const float2 y = __ffma2_rn(make_float2(x[c & 1][k], x[c & 1][k + 1]), scale2, off2);
            float2 p;
            if constexpr (decltype(mask)::value) {
              p = make_float2(ex2(y.x), ex2(y.y));
              p = make_float2(kChunk * c + k < sees ? p.x : 0.f, kChunk * c + k + 1 < sees ? p.y : 0.f);
            } else if (k % 8 == 6) {             // a quarter of the pairs
              p = exp2_fma(y);
            } else {
              p = make_float2(ex2(y.x), ex2(y.y));
            }
            acc[(kChunk * c + k) / 2] = __fadd2_rn(acc[(kChunk * c + k) / 2], p);
          }
        }
      };
      // masked: some query does not see all of the rows, or a lane has no query that counts, whatever it holds; or its lse is not a number, which
      // exp2_fma would make one
      if (__any_sync(0xffffffffu, sees < kMine || !(off > -INFINITY))) weights(std::true_type{});
      else weights(std::false_type{});
    }
    // over the warp's queries: 32 of the rows at a time, row `lane` of them to a lane
#pragma unroll
    for (int g = 0; g < kMine / 32; ++g) {
      float a[32];
#pragma unroll
      for (int k = 0; k < 16; ++k) {
        a[2 * k] = acc[16 * g + k].x;
        a[2 * k + 1] = acc[16 * g + k].y;
      }
      const float sum = sum_scatter<32>(a, lane);
      sums[4 * turn + warp % 4][kMine * half + 32 * g + lane] = ok ? sum : NAN;
    }
    asm volatile("bar.sync 1, 512;" ::: "memory");         // the row warps
    if (tid < kTcKeys) {
      float sum = 0.f;
#pragma unroll
      for (int w = 0; w < 8; ++w) sum += sums[w][tid];
      if (gridDim.y > 1) total[tid] = sum;
      else if (key0 + tid < len) score_put(C, (int64_t)s * A.cap + key0 + tid, sum);
    }
    tc_fence_before();
  }
  if (gridDim.y > 1) {                           // the cluster's sums: every CTA adds up its part of the rows, in the order of the CTAs
    cluster.sync();
    const int row = tid * (int)gridDim.y + (int)blockIdx.y;
    if (warp < 16 && row < kTcKeys && key0 + row < len) {             // (the row warps, which have the registers)
      float sum = 0.f;
      for (int b = 0; b < (int)gridDim.y; ++b) sum += cluster.map_shared_rank(&total[0], b)[row];
      score_put(C, (int64_t)s * A.cap + key0 + row, sum);
    }
    cluster.sync();
  }
  __syncthreads();
  tc_fence_after();
  if (warp == 17) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512u) : "memory");
}

// The same where the counted queries of a stream fill one or two tiles: they stay in shared memory and the cached rows go by, a CTA's
// share of the stream's tiles of 128 rows.  A tile of queries has `cols` rows, as few 32s as hold its heads' boxes: the products and
// exponentials of the others are saved.  S^T = K Q^T has the cached rows as lanes here, so that a thread adds up one row's weights; two
// warpgroups take 32 queries in turn, and every tile's rows are written at once.
constexpr int kStreamThreads = 384;

template <int D>
struct StreamShape {
  static constexpr uint32_t kBox = 128 * 128;
  static constexpr uint32_t kTile = (D / 64) * kBox;
  static constexpr int kRing = D == 128 ? 4 : 8;
  static constexpr size_t kSmem = 1024 + (2 + kRing) * (size_t)kTile;
};
template <int D>
__global__ void __launch_bounds__(kStreamThreads, 1)
score_stream_kernel(const __grid_constant__ AttnRows A, const ScoreArgs C, int box_rows, int q_tiles, int cols, const __grid_constant__ CUtensorMap mq, const __grid_constant__ CUtensorMap mk) {
  using Sh = StreamShape<D>;
  constexpr int kRing = Sh::kRing;
  extern __shared__ unsigned char smem_raw[];
  __shared__ uint64_t q_full, k_full[kRing], k_empty[kRing], s_full[4], s_empty[4], drained;
  __shared__ uint32_t tmem_s;
  __shared__ int abort_flag;
  __shared__ __align__(16) float lse[2][kTcRows];             // negative
  __shared__ __align__(16) int query[2][kTcRows];             // of a head
  __shared__ float total[2][kTcKeys];            // the second warpgroup's sums of a tile
  unsigned char* sm = smem_raw + (-smem_u32(smem_raw) & 1023u);
  unsigned char* ring = sm + 2 * Sh::kTile;
  const int tid = threadIdx.x, warp = __shfl_sync(0xffffffffu, tid / 32, 0), lane = tid % 32;
  const int pack = kTcRows / box_rows;           // heads of a tile
  if (tid == 0) {
    mbar_init(&q_full, 1);
    mbar_init(&drained, 1);
    for (int i = 0; i < kRing; ++i) { mbar_init(k_full + i, 1); mbar_init(k_empty + i, 1); }
    for (int i = 0; i < 4; ++i) { mbar_init(s_full + i, 1); mbar_init(s_empty + i, 256); }
    abort_flag = 0;
    asm volatile("prefetch.tensormap [%0];" ::"l"(&mq) : "memory");
    asm volatile("prefetch.tensormap [%0];" ::"l"(&mk) : "memory");
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (box_rows < kTcRows)                        // what no head's queries fill is zero, so that its weights are
    for (int i = tid; i < 2 * (int)Sh::kTile / 16; i += kStreamThreads) reinterpret_cast<uint4*>(sm)[i] = make_uint4(0, 0, 0, 0);
  asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
  if (warp == 9) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&tmem_s)), "r"(512u) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  const int s = blockIdx.x, len = attn_len(A, s), m = A.n_queries, heads = A.n_rows / m, start = m - C.n_scored;
  const int all = (len + kTcKeys - 1) / kTcKeys;
  const int t0 = (int)((int64_t)all * blockIdx.y / gridDim.y), n = (int)((int64_t)all * (blockIdx.y + 1) / gridDim.y) - t0;      // this CTA's
  // The queries and the first cached rows come in before the attention kernel has ended, whose lse alone is waited for.
  auto ask_keys = [&](int i) {
    mbar_expect_tx(k_full + i % kRing, Sh::kTile);
    for (int b = 0; b < D / 64; ++b) tma_load_3d(ring + i % kRing * Sh::kTile + b * Sh::kBox, &mk, 64 * b, (t0 + i) * kTcKeys, s, k_full + i % kRing);
  };
  __syncthreads();
  if (tid == 8 * 32 && n > 0) {
    mbar_expect_tx(&q_full, (uint32_t)heads * box_rows * 2 * D);
    for (int h = 0; h < heads; ++h)
      for (int b = 0; b < D / 64; ++b)
        tma_load_3d(sm + h / pack * Sh::kTile + b * Sh::kBox + h % pack * box_rows * 128, &mq, 64 * b, start, s * heads + h, &q_full);
    for (int i = 0; i < min(kRing, n); ++i) ask_keys(i);
  }
  grid_wait_and_release();
  // query row r of tile t: head and query (box_rows = 128: a head to a tile)
  if (n > 0)
    for (int i = tid; i < 2 * kTcRows; i += kStreamThreads) {
      const int t = i / kTcRows, r = i % kTcRows, h = t * pack + r / box_rows, q = start + r % box_rows;
      lse[t][r] = t < q_tiles && r < pack * box_rows && h < heads && q < m ? -A.lse[((int64_t)s * heads + h) * m + q] : -INFINITY;
      query[t][r] = q;
    }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = __shfl_sync(0xffffffffu, tmem_s, 0);

  if (warp == 8 && n > 0) {
    bool ok = true;
    int i = min(kRing, n);
    for (; i < n; ++i) {
      ok = wait_bar(k_empty + i % kRing, (uint32_t)(i / kRing - 1) & 1u, &abort_flag);
      if (!__all_sync(0xffffffffu, ok)) break;
      if (lane == 0) ask_keys(i);
      __syncwarp();
    }
    if (lane == 0) {
      copy_landed(&q_full);
      copies_landed(k_full, i);
    }
  } else if (warp == 9 && n > 0) {
    bool ok = true;
    auto wait = [&](uint64_t* bar, uint32_t parity) { ok = ok && __all_sync(0xffffffffu, wait_bar(bar, parity, &abort_flag)); };
    const uint32_t instr = (kInstrBf16<kTcRows> & ~(63u << 17)) | (uint32_t)(cols >> 3) << 17;
    wait(&q_full, 0);
    int u = 0;                                   // products so far: the buffer u % 4 of logits
    for (int i = 0; i < n && ok; ++i) {
      wait(k_full + i % kRing, (uint32_t)(i / kRing) & 1u);
      for (int t = 0; t < q_tiles; ++t, ++u) {
        if (u > 3) wait(s_empty + (u & 3), (uint32_t)(u / 4 - 1) & 1u);
        tc_fence_after();
        if (ok && elect_one()) {
          const uint32_t a = umma_desc_lo(smem_u32(ring + i % kRing * Sh::kTile)), b = umma_desc_lo(smem_u32(sm + t * Sh::kTile)), d = tmem + 128 * (u & 3);
#pragma unroll
          for (int k = 0; k < D / 16; ++k) {
            const uint32_t at = (uint32_t)(k / 4) * (Sh::kBox >> 4) + 2 * (k % 4);
            umma_n(d, a + at, b + at, instr, k > 0);
          }
          umma_commit(s_full + (u & 3));
          if (t == q_tiles - 1) umma_commit(k_empty + i % kRing);
        }
        __syncwarp();
      }
    }
    if (!ok) st_release(&abort_flag, 1);
    products_done(&drained);
  } else if (warp < 8) {
    const int h = warp / 4, lanes = 32 * (warp % 4);
    const uint32_t S = tmem + ((uint32_t)lanes << 16);
    const float2 scale2 = make_float2(A.scale, A.scale);
    bool ok = true;
    int u = 0;
    for (int i = 0; i < n; ++i) {
      const int key0 = (t0 + i) * kTcKeys, key = key0 + lanes + lane, from = key - (len - m);      // the first query that sees the row
      const int64_t at = (int64_t)s * A.cap + key;
      const float old = h == 0 && key < len ? score_old(C, at) : 0.f;
      const bool masked = key0 + kTcKeys - 1 > len - m + start;
      float2 part[2] = {};
      for (int t = 0; t < q_tiles; ++t, ++u) {
        ok = ok && __all_sync(0xffffffffu, wait_bar(s_full + (u & 3), (uint32_t)(u / 4) & 1u, &abort_flag));
        if (!ok) break;
        tc_fence_after();
        for (int c = 32 * h; c < cols; c += 64) {          // the warpgroups take 32 columns in turn
          float x[32];
          tmem_ld32(S + 128 * (u & 3) + c, x);
          tmem_ld_wait();
          const float4* l4 = reinterpret_cast<const float4*>(lse[t] + c);
          const int4* q4 = reinterpret_cast<const int4*>(query[t] + c);
          auto weights = [&](auto mask) {
#pragma unroll
            for (int k = 0; k < 32; k += 4) {
              const float4 l = l4[k / 4];
              const float2 lo = __ffma2_rn(make_float2(x[k], x[k + 1]), scale2, make_float2(l.x, l.y));
              const float2 hi = __ffma2_rn(make_float2(x[k + 2], x[k + 3]), scale2, make_float2(l.z, l.w));
              float2 a = make_float2(ex2(lo.x), ex2(lo.y)), b = make_float2(ex2(hi.x), ex2(hi.y));
              if constexpr (decltype(mask)::value) {
                const int4 q = q4[k / 4];
                a = make_float2(q.x >= from ? a.x : 0.f, q.y >= from ? a.y : 0.f);
                b = make_float2(q.z >= from ? b.x : 0.f, q.w >= from ? b.y : 0.f);
              }
              part[0] = __fadd2_rn(part[0], a);
              part[1] = __fadd2_rn(part[1], b);
            }
          };
          if (masked) weights(std::true_type{});
          else weights(std::false_type{});
        }
        tc_fence_before();
        mbar_arrive(s_empty + (u & 3));
      }
      float sum = ok ? (part[0].x + part[0].y) + (part[1].x + part[1].y) : NAN;
      if (h == 1) total[i & 1][lanes + lane] = sum;
      asm volatile("bar.sync 1, 256;" ::: "memory");       // the row warps; the place is written again behind the next tile's barrier
      if (h == 0 && key < len) score_put(C, at, old, sum + total[i & 1][lanes + lane]);
    }
    tc_fence_before();
  }
  __syncthreads();
  tc_fence_after();
  if (warp == 9) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512u) : "memory");
}

template <int D>
cudaError_t launch_stream(const AttnRows& A, const ScoreArgs& S, int box_rows, const CUtensorMap& mq, const CUtensorMap& mk, cudaStream_t st) {
  static std::atomic<unsigned long long> devices{0};
  const cudaError_t e = kernel_limits(score_stream_kernel<D>, StreamShape<D>::kSmem, devices);
  if (e != cudaSuccess) return e;
  const int heads = A.n_rows / A.n_queries, pack = kTcRows / box_rows, q_tiles = (heads + pack - 1) / pack;
  const int cols = (std::min(heads, pack) * box_rows + 31) / 32 * 32;
  // a CTA an SM, or two waves of them where the streams alone are more, with four tiles each while that leaves none idle
  const int64_t tiles = (A.cap + kTcKeys - 1) / kTcKeys;
  const int64_t parts = std::max<int64_t>(1, std::min<int64_t>((A.n_streams > kAttnSms ? 4 : 1) * kAttnSms / A.n_streams, tiles));
  const PdlConfig pc(dim3((unsigned)A.n_streams, (unsigned)parts), kStreamThreads, StreamShape<D>::kSmem, st);
  return cudaLaunchKernelEx(&pc.cfg, score_stream_kernel<D>, A, S, box_rows, q_tiles, cols, mq, mk);
}

template <int D>
cudaError_t launch(const AttnRows& A, const ScoreArgs& S, cudaStream_t st) {
  CUtensorMap mq, mk;
  const int box_rows = S.n_scored > 64 ? kTcRows : (S.n_scored + 7) / 8 * 8;      // (1024 bytes and more: boxes keep the swizzle's phase)
  cudaError_t e = cache_map(&mq, A.q, true, D, A.n_queries, A.total_rows / A.n_queries, box_rows);
  if (e == cudaSuccess) e = cache_map(&mk, A.K, true, D, A.cap, A.n_streams, kTcKeys);
  if (e != cudaSuccess) return e;
  // Up to two tiles of queries stay where they are, and the cached rows go by.
  const int heads = A.n_rows / A.n_queries;
  if (S.n_scored <= kTcRows && (heads + kTcRows / box_rows - 1) / (kTcRows / box_rows) <= 2) return launch_stream<D>(A, S, box_rows, mq, mk, st);
  static std::atomic<unsigned long long> devices{0};
  e = kernel_limits(score_tc_kernel<D>, Shape<D>::kSmem, devices);
  if (e != cudaSuccess) return e;
  // CTAs of a cluster: more while there are fewer than two waves and four tiles of queries are left for each.  (512 CTAs of a prompt of 8192:
  // 829 us with its attention by one CTA each, which take the SMs as they come free, 873 by pairs, which start and end together.)
  const int64_t blocks = (int64_t)((A.cap + kTcKeys - 1) / kTcKeys) * A.n_streams;
  const int tiles = box_rows < kTcRows ? 1 : A.n_rows / A.n_queries * ((S.n_scored + kTcRows - 1) / kTcRows);
  int P = 1;
  while (P < 8 && blocks * P < 2 * kAttnSms && tiles >= 8 * P) P *= 2;
  PdlConfig pc(dim3((unsigned)blocks, P), kThreads, Shape<D>::kSmem, st);
  cudaLaunchAttribute attrs[2] = {pc.attr, {}};
  attrs[1].id = cudaLaunchAttributeClusterDimension;
  attrs[1].val.clusterDim.x = attrs[1].val.clusterDim.z = 1;
  attrs[1].val.clusterDim.y = P;
  pc.cfg.attrs = attrs;
  pc.cfg.numAttrs = 2;
  return cudaLaunchKernelEx(&pc.cfg, score_tc_kernel<D>, A, S, box_rows, mq, mk);
}

}  // namespace

cudaError_t launch_score_tc(const AttnRows& A, const ScoreArgs& S, int d, cudaStream_t st) {
  return d == 128 ? launch<128>(A, S, st) : launch<64>(A, S, st);
}

}  // namespace bkv
