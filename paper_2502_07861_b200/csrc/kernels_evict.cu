// Eviction by accumulated weight: which rows of a cache stay, and the copies that make it so.
//
// evict_select_kernel, a cluster of CTAs per stream: rows become 32-bit keys that order like their scores (rows that are to stay
// whatever their score above all others), a radix select of 11 + 11 + 10 bits over the cluster's histograms finds the keep-th
// largest key, and of the rows that hold exactly that key the first ones stay.  Rows that stay below row `keep` are not moved; the
// n-th of those that stay behind it fills the n-th hole, so that an eviction in place moves as few rows as any can, and no source
// of a copy is another's destination.
#include <cooperative_groups.h>

#include <algorithm>
#include <utility>

#include "attn_rows.cuh"

namespace bkv {

namespace {

namespace cg = cooperative_groups;

constexpr int kThreads = 512, kWarps = kThreads / 32;
constexpr int kPasses = 3, kBins = 2048;
constexpr int kMaxCluster = 8;
constexpr int kStageRows = 24576;              // rows whose keys and positions a CTA keeps in shared memory; those of longer slices are read again
constexpr int kAhead = 4;                      // rows that a thread asks for at once

constexpr uint32_t kSafe = 0xffffffffu;

// Orders like the score: NaN below everything, -0 as 0.
__device__ inline uint32_t score_key(float x) {
  if (x != x) return 0;
  const uint32_t b = __float_as_uint(x + 0.f);
  return b & 0x80000000u ? ~b : b | 0x80000000u;
}

struct SelectShared {
  __align__(16) uint32_t hist[kPasses][kBins];
  uint32_t coarse[kPasses][kMaxCluster][kBins / 64];          // every CTA's sums of 64 bins
  int warp_a[kWarps], warp_b[kWarps];
  int cta[3][2];                                 // what the cluster's CTAs tell one another, a place per exchange
  int before_a, before_b, all_a;                 // of the CTAs before this one; of all
  int digit, above, equal;
  unsigned long long warp_least[kWarps], cta_least;
};

// Sums of a and b over the warps (a value per warp, by lane 0) and the cluster's CTAs: what lies before the warp, and all.  For all threads.
__device__ inline void sums_before(cg::cluster_group& cluster, SelectShared& sh, int place, int C, int c, int& a, int& b, int& all) {
  const int tid = threadIdx.x, warp = tid / 32, lane = tid % 32;
  if (lane == 0) { sh.warp_a[warp] = a; sh.warp_b[warp] = b; }
  __syncthreads();
  if (warp == 0) {
    const int x = __reduce_add_sync(0xffffffffu, lane < kWarps ? sh.warp_a[lane] : 0), y = __reduce_add_sync(0xffffffffu, lane < kWarps ? sh.warp_b[lane] : 0);
    if (lane == 0) { sh.cta[place][0] = x; sh.cta[place][1] = y; }
  }
  cluster.sync();
  if (warp == 0) {
    const int* far = lane < C ? cluster.map_shared_rank(&sh.cta[place][0], lane) : nullptr;
    const int x = far ? far[0] : 0, y = far ? far[1] : 0;
    const int bx = __reduce_add_sync(0xffffffffu, lane < c ? x : 0), by = __reduce_add_sync(0xffffffffu, lane < c ? y : 0), ax = __reduce_add_sync(0xffffffffu, x);
    if (lane == 0) { sh.before_a = bx; sh.before_b = by; sh.all_a = ax; }
  }
  __syncthreads();
  a = sh.before_a;
  b = sh.before_b;
  all = sh.all_a;
  for (int w = 0; w < warp; ++w) { a += sh.warp_a[w]; b += sh.warp_b[w]; }
  __syncthreads();                               // the next sums may go there
}

// The lane whose share of the values n, the first lane's first, holds the need-th, and the sum before it.
__device__ inline int lane_of(int n, int need, int& before) {
  int incl = n;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int x = __shfl_up_sync(0xffffffffu, incl, o);
    if ((threadIdx.x & 31) >= o) incl += x;
  }
  const uint32_t reached = __ballot_sync(0xffffffffu, incl >= need);
  const int at = __ffs(reached) - 1;
  before = __shfl_sync(0xffffffffu, incl - n, at);
  return at;
}

// `rows` of a stream, the i-th from row from(i) to row to(i), by the threads that count from `at` in steps of `step`: K, V, score, position.
template <class From, class To>
__device__ inline void copy_rows(const EvictArgs& E, int s, int rows, int at, int step, From from, To to) {
  constexpr int kBatch = 4;                      // rows in flight per thread
  const int vecs = E.row_bytes / 16, lane = at % vecs, groups = step / vecs;
  for (int i0 = at / vecs; i0 < rows; i0 += kBatch * groups) {
    int64_t src[kBatch], dst[kBatch];
    uint4 k[kBatch], v[kBatch];
#pragma unroll
    for (int j = 0; j < kBatch; ++j) {
      const int i = min(i0 + j * groups, rows - 1);
      src[j] = (int64_t)s * E.cap + from(i);
      dst[j] = i0 + j * groups < rows ? (int64_t)s * E.cap_out + to(i) : -1;
    }
#pragma unroll
    for (int j = 0; j < kBatch; ++j) {
      k[j] = __ldcs(static_cast<const uint4*>(E.K) + src[j] * vecs + lane);
      v[j] = __ldcs(static_cast<const uint4*>(E.V) + src[j] * vecs + lane);
    }
#pragma unroll
    for (int j = 0; j < kBatch; ++j)
      if (dst[j] >= 0) {
        __stcs(static_cast<uint4*>(E.K_out) + dst[j] * vecs + lane, k[j]);
        __stcs(static_cast<uint4*>(E.V_out) + dst[j] * vecs + lane, v[j]);
        if (lane == 0) {
          E.score_out[dst[j]] = E.score[src[j]];
          if (E.pos_out) E.pos_out[dst[j]] = E.pos ? E.pos[src[j]] : (int)(src[j] - (int64_t)s * E.cap);
        }
      }
  }
}

// kFused: the clusters copy their streams' rows themselves.  kCtas of them are to share an SM (0: with the registers that they would like, two),
// which serves launches of more CTAs than two an SM (256 streams of up to 4096 rows, 512 CTAs: 57 us by three, 62 by two; 2 streams of 4000: 15.4 by three, 13.4 by two).
template <bool kFused, int kCtas>
__global__ void __launch_bounds__(kThreads, kCtas) evict_select_kernel(const EvictArgs E, int per, int staged) {
  extern __shared__ uint32_t keys[];             // [per], behind them the positions (E.pos) [per]
  __shared__ SelectShared sh;
  cg::cluster_group cluster = cg::this_cluster();
  const int C = (int)cluster.num_blocks(), c = (int)cluster.block_rank();
  const int s = blockIdx.x / C, tid = threadIdx.x, warp = tid / 32, lane = tid % 32;
  for (int i = tid; i < kPasses * kBins / 4; i += kThreads) reinterpret_cast<uint4*>(&sh.hist[0][0])[i] = make_uint4(0, 0, 0, 0);
  // Nobody counts rows before the histograms are empty, and nobody writes into another CTA's shared memory before that CTA has begun.
  auto begun = cluster.barrier_arrive();
  grid_wait_and_release();
  const int len = E.lens ? max(0, min(E.lens[s], E.cap)) : E.cap, k = min(len, E.keep);
  cluster.barrier_wait(std::move(begun));
  const int64_t first = (int64_t)s * E.cap;
  int* holes = E.moves + (int64_t)s * (2 * (int64_t)E.list + (E.in_place ? 0 : E.keep));
  int* movers = holes + E.list;
  int* source = movers + E.list;
  if (len <= E.keep) {                           // nothing to evict (the same for the whole cluster, which has read lens by its barrier)
    cluster.sync();
    auto same = [](int i) { return i; };
    if (kFused && !E.in_place) copy_rows(E, s, len, c * kThreads + tid, C * kThreads, same, same);
    if (!kFused && !E.in_place)
      for (int i = c * kThreads + tid; i < len; i += C * kThreads) source[i] = i;
    if (c == 0 && tid == 0) {
      E.n_moves[s] = 0;
      if (E.lens_out) E.lens_out[s] = len;
    }
    return;
  }
  const int begin = min(len, c * per), end = min(len, begin + per);
  int* const places = reinterpret_cast<int*>(keys) + per;
  const bool aged = E.pos && E.n_recent > 0;     // the newest position has to be found
  int newest = E.pos ? INT32_MIN : len - 1;
  if (staged || aged)
    for (int i0 = begin + tid; i0 < end; i0 += kAhead * kThreads) {
      int pos[kAhead];
      float score[kAhead];
#pragma unroll
      for (int j = 0; j < kAhead; ++j) {
        const int64_t at = first + min(i0 + j * kThreads, end - 1);
        pos[j] = E.pos ? E.pos[at] : 0;
        score[j] = staged ? E.score[at] : 0.f;
      }
#pragma unroll
      for (int j = 0; j < kAhead; ++j) {
        const int i = i0 + j * kThreads;
        newest = E.pos ? max(newest, pos[j]) : newest;
        if (staged && i < end) {
          keys[i - begin] = score_key(score[j]);
          if (E.pos) places[i - begin] = pos[j];
        }
      }
    }
  if (aged) {
    newest = __reduce_max_sync(0xffffffffu, newest);
    if (lane == 0) sh.warp_a[warp] = newest;
    __syncthreads();
    if (warp == 0) {
      newest = __reduce_max_sync(0xffffffffu, lane < kWarps ? sh.warp_a[lane] : INT32_MIN);
      if (lane == 0) sh.cta[0][0] = newest;
    }
    cluster.sync();
    if (warp == 0) {
      newest = __reduce_max_sync(0xffffffffu, lane < C ? *cluster.map_shared_rank(&sh.cta[0][0], lane) : INT32_MIN);
      if (lane == 0) sh.all_a = newest;
    }
    __syncthreads();
    newest = sh.all_a;
  }
  const int64_t recent = E.n_recent > 0 ? (int64_t)newest - E.n_recent : INT32_MAX;      // positions above are safe
  auto safe = [&](int pos) { return pos < E.n_first || pos > recent; };
  auto form = [&](int i) { return safe(E.pos ? E.pos[first + i] : i) ? kSafe : score_key(E.score[first + i]); };
  auto key = [&](int i) { return staged ? keys[i - begin] : form(i); };

  if (len == k + 1) {
    // One row goes, every token's case: the last of those of the smallest key.  (The select below: 1025 rows 14 us, 9 here.)
    unsigned long long least = ~0ull;            // the key, then from the last row on
    for (int i = begin + tid; i < end; i += kThreads) {
      const uint32_t u = staged ? safe(E.pos ? places[i - begin] : i) ? kSafe : keys[i - begin] : form(i);
      least = min(least, (unsigned long long)u << 32 | (0xffffffffu - (uint32_t)i));
    }
    auto of_warp = [&](unsigned long long x) {
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) x = min(x, __shfl_xor_sync(0xffffffffu, x, o));
      return x;
    };
    least = of_warp(least);
    if (lane == 0) sh.warp_least[warp] = least;
    __syncthreads();
    if (warp == 0) {
      least = of_warp(lane < kWarps ? sh.warp_least[lane] : ~0ull);
      if (lane == 0) sh.cta_least = least;
    }
    cluster.sync();
    if (warp == 0) {
      least = of_warp(lane < C ? *cluster.map_shared_rank(&sh.cta_least, lane) : ~0ull);
      if (lane == 0) sh.digit = (int)(0xffffffffu - (uint32_t)least);
    }
    __syncthreads();
    const int gone = sh.digit;
    cluster.sync();                              // nobody reads this CTA's memory any more, nor what is copied over
    if (c == 0 && tid == 0) {
      E.n_moves[s] = gone < k;
      if (E.lens_out) E.lens_out[s] = k;
    }
    if (!E.in_place) {
      auto from = [&](int i) { return i == gone ? k : i; };
      if (kFused) copy_rows(E, s, k, c * kThreads + tid, C * kThreads, from, [](int i) { return i; });
      else
        for (int i = c * kThreads + tid; i < k; i += C * kThreads) source[i] = from(i);
    } else if (gone < k) {
      if (kFused) {
        if (c == 0) copy_rows(E, s, 1, tid, kThreads, [&](int) { return k; }, [&](int) { return gone; });
      } else if (c == 0 && tid == 0) {
        holes[0] = gone;
        movers[0] = k;
      }
    }
    return;
  }

  uint32_t prefix = 0;
  int need = k;
#pragma unroll 1
  for (int pass = 0; pass < kPasses; ++pass) {
    const int shift = pass == 0 ? 21 : pass == 1 ? 10 : 0;
    const uint32_t mask = pass == 2 ? 1023u : 2047u;
    for (int i = begin + tid; i < end; i += kThreads) {
      uint32_t u;
      if (pass == 0 && staged) {                 // (this thread's rows)
        u = safe(E.pos ? places[i - begin] : i) ? kSafe : keys[i - begin];
        keys[i - begin] = u;
      } else {
        u = key(i);
      }
      if (pass == 0 || u >> (pass == 1 ? 21 : 10) == prefix) atomicAdd(&sh.hist[pass][u >> shift & mask], 1u);
    }
    __syncthreads();
    {                                            // 64 bins to a sum: 16 threads with four bins each
      const uint4 h = reinterpret_cast<const uint4*>(sh.hist[pass])[tid];
      uint32_t n = h.x + h.y + h.z + h.w;
#pragma unroll
      for (int o = 8; o > 0; o >>= 1) n += __shfl_xor_sync(0xffffffffu, n, o);
      // to every CTA of the cluster (a store does not wait, a load from there does)
      if (tid % 16 < C) cluster.map_shared_rank(&sh.coarse[pass][c][0], tid % 16)[tid / 16] = n;
    }
    cluster.sync();
    // One warp finds the digit, from the largest down: which 64 bins, then which of them.  (Every thread adding the cluster's bins up
    // took 6000 cycles a pass: shared memory of other SMs is slow.)
    if (warp == 0) {
      int n = 0, before, rest;
#pragma unroll
      for (int b = 0; b < kMaxCluster; ++b)
        if (b < C) n += (int)sh.coarse[pass][b][31 - lane];
      const int group = 31 - lane_of(n, need, before);
      int hi = 0, lo = 0;                        // the bins 63 - 2 lane, 62 - 2 lane of the 64; all CTAs' asked for at once
      uint2 h[kMaxCluster];
#pragma unroll
      for (int b = 0; b < kMaxCluster; ++b) h[b] = *reinterpret_cast<const uint2*>(cluster.map_shared_rank(&sh.hist[pass][0], min(b, C - 1)) + 64 * group + 62 - 2 * lane);
#pragma unroll
      for (int b = 0; b < kMaxCluster; ++b) {
        hi += b < C ? (int)h[b].y : 0;
        lo += b < C ? (int)h[b].x : 0;
      }
      const int at = lane_of(hi + lo, need - before, rest);
      const int first_hi = __shfl_sync(0xffffffffu, hi, at), first_lo = __shfl_sync(0xffffffffu, lo, at);
      const bool low = need - before - rest > first_hi;
      if (lane == 0) {
        sh.digit = 64 * group + 63 - 2 * at - (low ? 1 : 0);
        sh.above = before + rest + (low ? first_hi : 0);
        sh.equal = low ? first_lo : first_hi;
      }
    }
    __syncthreads();
    prefix = prefix << (pass == 2 ? 10 : 11) | (uint32_t)sh.digit;
    need -= sh.above;
  }

  // A warp takes neighbouring rows, so that ranks follow from ballots; four times 32 at once.
  constexpr int kUnroll = 4;
  const int seg = ((per + kWarps - 1) / kWarps + 31) / 32 * 32, w0 = min(end, begin + warp * seg), w1 = min(end, w0 + seg);
  const uint32_t lower = (1u << lane) - 1u;
  int eq_before = 0, none = 0, all = 0;
  const bool some_equal = need < sh.equal;       // not all rows of the last key that stays do: the first ones
  if (some_equal) {
    for (int i = w0; i < w1; i += 32 * kUnroll) {
      uint32_t u[kUnroll];
#pragma unroll
      for (int j = 0; j < kUnroll; ++j) u[j] = i + 32 * j + lane < w1 ? key(i + 32 * j + lane) : ~prefix;
#pragma unroll
      for (int j = 0; j < kUnroll; ++j) eq_before += __popc(__ballot_sync(0xffffffffu, u[j] == prefix));
    }
    sums_before(cluster, sh, 1, C, c, eq_before, none, all);
  }
  // every row of the warp's, 32 at a time: which are holes, which move
  auto walk = [&](auto&& each) {
    int equal = eq_before;
    for (int i = w0; i < w1; i += 32 * kUnroll) {
      uint32_t u[kUnroll], hole[kUnroll], mover[kUnroll];
#pragma unroll
      for (int j = 0; j < kUnroll; ++j) u[j] = i + 32 * j + lane < w1 ? key(i + 32 * j + lane) : 0u;
#pragma unroll
      for (int j = 0; j < kUnroll; ++j) {
        const int row = i + 32 * j + lane;
        const bool held = row < w1;
        bool kept = held && u[j] >= prefix;
        if (some_equal) {
          const uint32_t same = __ballot_sync(0xffffffffu, held && u[j] == prefix);
          kept = held && (u[j] > prefix || (u[j] == prefix && equal + __popc(same & lower) < need));
          equal += __popc(same);
        }
        hole[j] = __ballot_sync(0xffffffffu, held && !kept && row < k);
        mover[j] = __ballot_sync(0xffffffffu, kept && row >= k);
      }
#pragma unroll
      for (int j = 0; j < kUnroll; ++j) each(i + 32 * j, hole[j], mover[j]);
    }
  };
  // What the first walk finds is kept for the second, in the place of the first histogram, which nobody reads any more.
  uint32_t *const hole_bits = sh.hist[0] + warp * (seg / 32), *const mover_bits = hole_bits + kBins / 2;
  const bool noted = kWarps * (seg / 32) <= kBins / 2;
  int at_hole = 0, at_mover = 0;
  walk([&](int row, uint32_t hole, uint32_t mover) {
    at_hole += __popc(hole);
    at_mover += __popc(mover);
    if (noted && lane == 0 && row < w1) {
      hole_bits[(row - w0) / 32] = hole;
      mover_bits[(row - w0) / 32] = mover;
    }
  });
  sums_before(cluster, sh, 2, C, c, at_hole, at_mover, all);
  auto put = [&](int first_row, uint32_t hole, uint32_t mover) {
    const int row = first_row + lane;
    if (hole >> lane & 1) holes[at_hole + __popc(hole & lower)] = row;
    else if (!E.in_place && row < min(w1, k)) source[row] = row;
    if (mover >> lane & 1) movers[at_mover + __popc(mover & lower)] = row;
    at_hole += __popc(hole);
    at_mover += __popc(mover);
  };
  if (noted) {
    for (int i = w0; i < w1; i += 32) put(i, hole_bits[(i - w0) / 32], mover_bits[(i - w0) / 32]);
  } else {
    walk(put);
  }
  if (c == 0 && tid == 0) {
    E.n_moves[s] = all;
    if (E.lens_out) E.lens_out[s] = k;
  }
  cluster.sync();                                // the lists are written; nobody reads this CTA's memory any more
  if (!E.in_place)
    for (int i = c * kThreads + tid; i < all; i += C * kThreads) source[__ldcg(holes + i)] = __ldcg(movers + i);
  if (!kFused) return;
  if (E.in_place) {
    copy_rows(E, s, all, c * kThreads + tid, C * kThreads, [&](int i) { return __ldcg(movers + i); }, [&](int i) { return __ldcg(holes + i); });
    return;
  }
  cluster.sync();                                // the list of sources is whole
  copy_rows(E, s, k, c * kThreads + tid, C * kThreads, [&](int i) { return __ldcg(source + i); }, [](int i) { return i; });
}

// A group of kVecs lanes per row: K, V, and by its first lane the score and the position.
constexpr int kMoveThreads = 256, kMoveRows = 2;
template <int kVecs>
__global__ void __launch_bounds__(kMoveThreads) evict_move_kernel(const EvictArgs E, int blocks) {
  constexpr int kGroups = kMoveThreads / kVecs;
  const int s = blockIdx.x / blocks, lane = threadIdx.x % kVecs;
  const int i0 = blockIdx.x % blocks * kGroups * kMoveRows + threadIdx.x / kVecs;
  grid_wait_and_release();
  const int* holes = E.moves + (int64_t)s * (2 * (int64_t)E.list + (E.in_place ? 0 : E.keep));
  const int* source = holes + (E.in_place ? E.list : 2 * E.list);
  const int n = E.in_place ? E.n_moves[s] : E.lens_out ? E.lens_out[s] : min(E.lens ? max(0, min(E.lens[s], E.cap)) : E.cap, E.keep);
  int64_t from[kMoveRows], to[kMoveRows];
  uint4 k[kMoveRows], v[kMoveRows];
#pragma unroll
  for (int j = 0; j < kMoveRows; ++j) {
    const int i = i0 + j * kGroups;
    from[j] = -1;
    if (i >= n) continue;
    from[j] = (int64_t)s * E.cap + source[i];
    to[j] = (int64_t)s * E.cap_out + (E.in_place ? holes[i] : i);
  }
#pragma unroll
  for (int j = 0; j < kMoveRows; ++j)
    if (from[j] >= 0) {
      k[j] = __ldcs(static_cast<const uint4*>(E.K) + from[j] * kVecs + lane);
      v[j] = __ldcs(static_cast<const uint4*>(E.V) + from[j] * kVecs + lane);
    }
#pragma unroll
  for (int j = 0; j < kMoveRows; ++j)
    if (from[j] >= 0) {
      __stcs(static_cast<uint4*>(E.K_out) + to[j] * kVecs + lane, k[j]);
      __stcs(static_cast<uint4*>(E.V_out) + to[j] * kVecs + lane, v[j]);
      if (lane == 0) {
        E.score_out[to[j]] = E.score[from[j]];
        if (E.pos_out) E.pos_out[to[j]] = E.pos ? E.pos[from[j]] : (int)(from[j] - (int64_t)s * E.cap);
      }
    }
}

template <int kVecs>
cudaError_t launch_move(const EvictArgs& E, cudaStream_t st) {
  const int most = E.in_place ? E.list : min(E.keep, E.cap);
  const int rows = kMoveThreads / kVecs * kMoveRows, blocks = (most + rows - 1) / rows;
  const PdlConfig pc(dim3((unsigned)blocks * E.n_streams), kMoveThreads, 0, st);
  return cudaLaunchKernelEx(&pc.cfg, evict_move_kernel<kVecs>, E, blocks);
}

}  // namespace

cudaError_t launch_evict(const EvictArgs& E, cudaStream_t st) {
  // CTAs of a stream: one for each 2048 rows, while a launch has not more of them than serve it.  An SM starts clusters slowly, and what a
  // CTA does beside reading its rows is the same for few and many.  One row over the budget, in place: a CTA an SM (256 streams of 4097 rows: 9.8 us by
  // 256 CTAs, 17.6 by 1024; 64 of 8193: 7.3 by 128, 13.0 by 512).  Others in place: two (256 full streams of 8192: 45 us by 256, 65 by
  // 1024; 64 of 16384: 30 by 256, 43 by 512).  Out of place, where a stream's list of sources is written too: three and a half (256 streams
  // of up to 8192: 102 us by 512, 110 by 1024; 256 of up to 4096: 57 by 512, 60 by 256).  A CTA always keeps its rows' keys on the chip
  // where eight can.
  const int64_t most = E.in_place ? (E.cap - E.keep <= 1 ? kAttnSms : 2 * kAttnSms) : 7 * kAttnSms / 2;
  int C = 1;
  while (C < kMaxCluster && E.cap > 2048 * C && ((int64_t)2 * C * E.n_streams <= most || E.cap > kStageRows * C)) C *= 2;
  // One launch where every CTA has an SM to itself and little to copy; larger clusters share the copying.  The second launch costs the
  // host 2.5 us and the device 4; a CTA moves about 100 KB a microsecond, half of that where sources come from a list (1 stream, 4000 of 16000
  // rows by 8 CTAs with 512 KB each: 26 us against 17 by two launches; 64 streams, 1024 of 1025: 15.6 us a call against 18.2).  With more
  // CTAs than SMs the copying waits in each CTA's turn, however little it is (1000 streams, one row of 1025 moved in place: 31.4 us
  // by one launch, 17.0 by two, a copy of lens included).
  const int64_t bytes = 4 * (int64_t)E.row_bytes * (E.in_place ? E.list : std::min(E.keep, E.cap));
  int F = C;
  while (F < kMaxCluster && 2 * F * E.n_streams <= kAttnSms && bytes > F * ((int64_t)128 << 10)) F *= 2;
  const bool fused = (int64_t)F * E.n_streams <= kAttnSms && bytes <= F * ((int64_t)(E.cap - E.keep <= 1 ? 512 : 128) << 10);
  if (fused) C = F;
  const int per = (E.cap + C - 1) / C, staged = per <= kStageRows;
  PdlConfig pc(dim3((unsigned)C * E.n_streams), kThreads, staged ? (size_t)per * (E.pos ? 8 : 4) : 0, st);
  cudaLaunchAttribute attrs[2] = {pc.attr, {}};
  attrs[1].id = cudaLaunchAttributeClusterDimension;
  attrs[1].val.clusterDim.x = C;
  attrs[1].val.clusterDim.y = attrs[1].val.clusterDim.z = 1;
  pc.cfg.attrs = attrs;
  pc.cfg.numAttrs = 2;
  static std::atomic<unsigned long long> devices[3];
  const bool crowded = !fused && (int64_t)C * E.n_streams > 2 * kAttnSms;
  auto kern = fused ? evict_select_kernel<true, 0> : crowded ? evict_select_kernel<false, 3> : evict_select_kernel<false, 0>;
  cudaError_t e = kernel_limits(kern, kStageRows * 8, devices[fused ? 0 : crowded ? 1 : 2]);
  if (e == cudaSuccess) e = cudaLaunchKernelEx(&pc.cfg, kern, E, per, staged);
  if (e != cudaSuccess || fused || (E.in_place && E.list == 0)) return e;
  switch (E.row_bytes / 16) {
    case 8: return launch_move<8>(E, st);
    case 16: return launch_move<16>(E, st);
    default: return launch_move<32>(E, st);
  }
}

}  // namespace bkv
