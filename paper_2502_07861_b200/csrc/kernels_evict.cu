// Eviction by accumulated weight: which rows of a cache stay, and the copies that make it so.
//
// evict_select_kernel, a cluster of CTAs per stream: rows become 32-bit keys that order like their scores (rows that are to stay
// whatever their score above all others), a radix select of 11 + 11 + 10 bits over the cluster's histograms finds the keep-th
// largest key, and of the rows that hold exactly that key the first ones stay.  Rows that stay below row `keep` are not moved; the
// n-th of those that stay behind it fills the n-th hole, so that an eviction in place moves as few rows as any can, and no source
// of a copy is another's destination.
#include <cooperative_groups.h>

#include "attn_rows.cuh"

namespace bkv {

namespace {

namespace cg = cooperative_groups;

constexpr int kThreads = 512, kWarps = kThreads / 32;
constexpr int kPasses = 3, kBins = 2048;
constexpr int kMaxCluster = 8;
constexpr int kStageRows = 49152;              // keys that a CTA keeps in shared memory; of longer slices they are formed anew

constexpr uint32_t kSafe = 0xffffffffu;

// Orders like the score: NaN below everything, -0 as 0.
__device__ inline uint32_t score_key(float x) {
  if (x != x) return 0;
  const uint32_t b = __float_as_uint(x + 0.f);
  return b & 0x80000000u ? ~b : b | 0x80000000u;
}

__global__ void __launch_bounds__(kThreads) evict_select_kernel(const EvictArgs E, int per, int staged) {
  extern __shared__ uint32_t keys[];
  __shared__ __align__(16) uint32_t hist[kPasses][kBins];
  __shared__ int warp_n[kWarps], warp_m[kWarps], scan[kWarps];
  __shared__ int cta_newest, cta_eq, cta_holes, cta_movers, found, above;
  cg::cluster_group cluster = cg::this_cluster();
  const int C = (int)cluster.num_blocks(), c = (int)cluster.block_rank();
  const int s = blockIdx.x / C, tid = threadIdx.x, warp = tid / 32, lane = tid % 32;
  for (int i = tid; i < kPasses * kBins; i += kThreads) (&hist[0][0])[i] = 0;
  grid_wait_and_release();
  const int len = E.lens ? max(0, min(E.lens[s], E.cap)) : E.cap, k = min(len, E.keep);
  const int64_t first = (int64_t)s * E.cap;
  int* holes = E.moves + (int64_t)s * (2 * E.list + (E.in_place ? 0 : E.keep));
  int* movers = holes + E.list;
  int* source = movers + E.list;
  if (len <= E.keep) {                           // nothing to evict (the same for the whole cluster, which has read lens by its barrier)
    cluster.sync();
    if (!E.in_place)
      for (int i = c * kThreads + tid; i < len; i += C * kThreads) source[i] = i;
    if (c == 0 && tid == 0) {
      E.n_moves[s] = 0;
      if (E.lens_out) E.lens_out[s] = len;
    }
    return;
  }
  const int begin = min(len, c * per), end = min(len, begin + per);
  int newest = len - 1;
  if (E.pos && E.n_recent > 0) {
    newest = INT32_MIN;
    for (int i = begin + tid; i < end; i += kThreads) newest = max(newest, E.pos[first + i]);
    newest = __reduce_max_sync(0xffffffffu, newest);
    if (lane == 0) warp_n[warp] = newest;
    __syncthreads();
    if (tid == 0) {
      for (int w = 1; w < kWarps; ++w) newest = max(newest, warp_n[w]);
      cta_newest = newest;
    }
    cluster.sync();
    for (int b = 0; b < C; ++b) newest = max(newest, *cluster.map_shared_rank(&cta_newest, b));
  }
  const int64_t recent = E.n_recent > 0 ? (int64_t)newest - E.n_recent : INT32_MAX;      // positions above are safe
  auto form = [&](int i) {
    const int pos = E.pos ? E.pos[first + i] : i;
    return pos < E.n_first || pos > recent ? kSafe : score_key(E.score[first + i]);
  };
  auto key = [&](int i) { return staged ? keys[i - begin] : form(i); };

  uint32_t prefix = 0;
  int need = k;
#pragma unroll 1
  for (int pass = 0; pass < kPasses; ++pass) {
    const int shift = pass == 0 ? 21 : pass == 1 ? 10 : 0;
    const uint32_t mask = pass == 2 ? 1023u : 2047u;
    for (int i = begin + tid; i < end; i += kThreads) {
      uint32_t u;
      if (pass == 0) {
        u = form(i);
        if (staged) keys[i - begin] = u;
      } else {
        u = key(i);
      }
      if (pass == 0 || u >> (pass == 1 ? 21 : 10) == prefix) atomicAdd(&hist[pass][u >> shift & mask], 1u);
    }
    cluster.sync();
    // each thread four neighbouring bins, from the largest down
    constexpr int kPer = kBins / kThreads;
    int n[kPer], sum = 0;
    const int top = kBins - 1 - kPer * tid;
    static_assert(kPer == 4, "a 16-byte load of the other CTAs' bins");
#pragma unroll
    for (int j = 0; j < kPer; ++j) n[j] = 0;
#pragma unroll
    for (int b = 0; b < kMaxCluster; ++b) {
      if (b >= C) break;
      const uint4 h = *reinterpret_cast<const uint4*>(cluster.map_shared_rank(&hist[pass][0], b) + top - 3);
      n[0] += (int)h.w;
      n[1] += (int)h.z;
      n[2] += (int)h.y;
      n[3] += (int)h.x;
    }
#pragma unroll
    for (int j = 0; j < kPer; ++j) sum += n[j];
    int incl = sum;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int x = __shfl_up_sync(0xffffffffu, incl, o);
      if (lane >= o) incl += x;
    }
    if (lane == 31) scan[warp] = incl;
    __syncthreads();
    int before = incl - sum;
    for (int w = 0; w < warp; ++w) before += scan[w];
#pragma unroll
    for (int j = 0; j < kPer; ++j) {
      if (before < need && need <= before + n[j]) {
        found = top - j;
        above = before;
      }
      before += n[j];
    }
    __syncthreads();
    prefix = prefix << (pass == 2 ? 10 : 11) | (uint32_t)found;
    need -= above;
  }

  // A warp takes neighbouring rows, so that ranks follow from ballots.
  const int seg = (per + kWarps - 1) / kWarps, w0 = min(end, begin + warp * seg), w1 = min(end, w0 + seg);
  const uint32_t lower = (1u << lane) - 1u;
  int eq = 0;
  for (int i = w0; i < w1; i += 32) eq += __popc(__ballot_sync(0xffffffffu, i + lane < w1 && key(i + lane) == prefix));
  if (lane == 0) warp_n[warp] = eq;
  __syncthreads();
  if (tid == 0) {
    int all = 0;
    for (int w = 0; w < kWarps; ++w) all += warp_n[w];
    cta_eq = all;
  }
  cluster.sync();
  int eq_before = 0;
  for (int b = 0; b < c; ++b) eq_before += *cluster.map_shared_rank(&cta_eq, b);
  for (int w = 0; w < warp; ++w) eq_before += warp_n[w];
  __syncthreads();
  // every row of the warp's: whether it is a hole or moves
  auto walk = [&](auto&& each) {
    int equal = eq_before;
    for (int i = w0; i < w1; i += 32) {
      const int row = i + lane;
      const bool held = row < w1;
      const uint32_t u = held ? key(row) : 0u;
      const uint32_t same = __ballot_sync(0xffffffffu, held && u == prefix);
      const bool kept = held && (u > prefix || (u == prefix && equal + __popc(same & lower) < need));
      equal += __popc(same);
      each(row, __ballot_sync(0xffffffffu, held && !kept && row < k), __ballot_sync(0xffffffffu, kept && row >= k), kept);
    }
  };
  int n_holes = 0, n_movers = 0;
  walk([&](int, uint32_t hole, uint32_t mover, bool) { n_holes += __popc(hole); n_movers += __popc(mover); });
  if (lane == 0) { warp_n[warp] = n_holes; warp_m[warp] = n_movers; }
  __syncthreads();
  if (tid == 0) {
    int h = 0, m = 0;
    for (int w = 0; w < kWarps; ++w) { h += warp_n[w]; m += warp_m[w]; }
    cta_holes = h;
    cta_movers = m;
  }
  cluster.sync();
  int at_hole = 0, at_mover = 0, all = 0;
  for (int b = 0; b < C; ++b) {
    const int h = *cluster.map_shared_rank(&cta_holes, b), m = *cluster.map_shared_rank(&cta_movers, b);
    if (b < c) { at_hole += h; at_mover += m; }
    all += h;
  }
  for (int w = 0; w < warp; ++w) { at_hole += warp_n[w]; at_mover += warp_m[w]; }
  walk([&](int row, uint32_t hole, uint32_t mover, bool kept) {
    if (hole >> lane & 1) holes[at_hole + __popc(hole & lower)] = row;
    if (mover >> lane & 1) movers[at_mover + __popc(mover & lower)] = row;
    if (!E.in_place && kept && row < k) source[row] = row;
    at_hole += __popc(hole);
    at_mover += __popc(mover);
  });
  if (c == 0 && tid == 0) {
    E.n_moves[s] = all;
    if (E.lens_out) E.lens_out[s] = k;
  }
  cluster.sync();                                // the lists are written; nobody reads this CTA's memory any more
  if (!E.in_place)
    for (int i = c * kThreads + tid; i < all; i += C * kThreads) source[__ldcg(holes + i)] = __ldcg(movers + i);
}

// A group of kVecs lanes per row: K, V, and by its first lane the score and the position.
constexpr int kMoveThreads = 256, kMoveRows = 4;
template <int kVecs>
__global__ void __launch_bounds__(kMoveThreads) evict_move_kernel(const EvictArgs E, int blocks) {
  constexpr int kGroups = kMoveThreads / kVecs;
  const int s = blockIdx.x / blocks, lane = threadIdx.x % kVecs;
  const int i0 = blockIdx.x % blocks * kGroups * kMoveRows + threadIdx.x / kVecs;
  grid_wait_and_release();
  const int* holes = E.moves + (int64_t)s * (2 * E.list + (E.in_place ? 0 : E.keep));
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
      k[j] = static_cast<const uint4*>(E.K)[from[j] * kVecs + lane];
      v[j] = static_cast<const uint4*>(E.V)[from[j] * kVecs + lane];
    }
#pragma unroll
  for (int j = 0; j < kMoveRows; ++j)
    if (from[j] >= 0) {
      static_cast<uint4*>(E.K_out)[to[j] * kVecs + lane] = k[j];
      static_cast<uint4*>(E.V_out)[to[j] * kVecs + lane] = v[j];
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
  int C = 1;
  while (C < kMaxCluster && E.cap > 4096 * C) C *= 2;
  const int per = (E.cap + C - 1) / C, staged = per <= kStageRows;
  PdlConfig pc(dim3((unsigned)C * E.n_streams), kThreads, staged ? (size_t)per * 4 : 0, st);
  cudaLaunchAttribute attrs[2] = {pc.attr, {}};
  attrs[1].id = cudaLaunchAttributeClusterDimension;
  attrs[1].val.clusterDim.x = C;
  attrs[1].val.clusterDim.y = attrs[1].val.clusterDim.z = 1;
  pc.cfg.attrs = attrs;
  pc.cfg.numAttrs = 2;
  cudaError_t e = cudaFuncSetAttribute(evict_select_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kStageRows * 4);
  if (e == cudaSuccess) e = cudaLaunchKernelEx(&pc.cfg, evict_select_kernel, E, per, staged);
  if (e != cudaSuccess || (E.in_place && E.list == 0)) return e;
  switch (E.row_bytes / 16) {
    case 8: return launch_move<8>(E, st);
    case 16: return launch_move<16>(E, st);
    default: return launch_move<32>(E, st);
  }
}

}  // namespace bkv
