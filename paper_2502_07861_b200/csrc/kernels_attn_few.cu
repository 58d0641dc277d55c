// Attention of few query rows per stream over a caller-held cache: one pass at memory speed, split over the cached rows.
//
//   x_{r,i} = <q_r, k_i> log2(e) / sqrt d + log2 w_i,   out_r = sum_i 2^(x_{r,i} - m_r) v_i / sum_i 2^(x_{r,i} - m_r)
//
// and where the rows are scored, the weights of every cached row: they need the finished sums of all splits, so the logits leave as
// fp32 (4 bytes per row and query against 2 d elements read) and a second launch turns them into weights while it joins the splits.
//
// A CTA takes up to eight query rows and is four warps (or two, few_warps), each with a ring of its own of tiles of 32 rows that TMA fills (K and V tiles in turn, boxes of 128 bytes x
// 32 rows, 128-byte swizzle): a warp waits for nothing but its own copies, and the lane that asks for the next tile does so as soon as
// its warp has read the last.  bf16 tiles go through mma.sync with the cached rows as the M dimension and the queries as the eight
// columns; fp32 tiles through packed FFMA.
// A bounded wait that gives up makes the results NaN.
#include <cooperative_groups.h>

#include <algorithm>
#include <climits>
#include <type_traits>
#include <utility>

#include "attn_rows.cuh"
#include "tma_mma.cuh"

namespace bkv {

namespace {

using namespace mma;

constexpr int kWarps = 4, kThreads = 32 * kWarps;      // of the clusters' CTAs; attn_few_kernel's: few_warps
constexpr int kTile = 32;                        // rows
constexpr float kGrow = 8.f;                     // a maximum follows when it would grow by more: weights stay below 2^8
constexpr uint32_t kBox = kTile * 128;           // bytes

// Query rows of a CTA: eight, of fp32 rows with 128 dims four, whose sums and queries fit the registers (eight query rows over 8 x 16384 such
// rows: 63.8 us by eight, 46.4 by four, which read the rows twice, the second time from L2).
__host__ __device__ constexpr int group_rows(bool bf16, int d) { return !bf16 && d == 128 ? 4 : kFewRows; }

template <bool kBf16, int D>
struct Few {
  static constexpr int kEsz = kBf16 ? 2 : 4, kBoxDims = 128 / kEsz, kBoxes = D / kBoxDims;
  static constexpr uint32_t kTileBytes = kBoxes * kBox;
  static constexpr int kRing = kTileBytes == 4096 ? 6 : 3;                   // tiles of a warp in flight
  static constexpr int kCtas = kTileBytes == 16384 ? 1 : 2;                  // of four warps that share an SM
  static constexpr int kPitch = D + 4;                                       // of a row in the merge buffer: sums, maximum, sum of weights
  static constexpr size_t kSmem = 1024 + (size_t)kWarps * kRing * kTileBytes;
  static_assert(kFewRows * kPitch * 4 <= (int)(kRing * kTileBytes), "the merge buffer takes the rings' place");
};
// Warps of a CTA of attn_few_kernel, so that two share an SM and one starts or ends while the other reads (fp32 rows of 128 dims, 1024 streams of up
// to 512 rows: 85 us by four warps, 77 by two; 2048 of 64, five query rows: 188 and 124).
__host__ __device__ constexpr int few_warps(bool bf16, int d) { return !bf16 && d == 128 ? 2 : kWarps; }
// Launches of more than two waves take less from a ring that stays full than from another CTA that is in the middle of its tiles while others start or
// end: three CTAs an SM with rings of two tiles, of 64 dims four with three.  bf16 rows, five query rows, two CTAs an SM and so: 256 streams of
// up to 8192 rows of 128 dims 96.3 and 94.5 us, 2048 of 128 rows 41.4 and 37.3, 296 of 512 (one wave) 10.5 and 13.9; of 64 dims 57.2 and
// 50.4, 29.7 and 21.5.
__host__ __device__ constexpr bool few_crowded(bool bf16, int64_t ctas) { return bf16 && ctas > 4 * kAttnSms; }
__host__ __device__ constexpr int crowd_ctas(int d) { return d == 128 ? 3 : 4; }
__host__ __device__ constexpr int crowd_ring(int d) { return d == 128 ? 2 : 3; }

struct FewArgs {
  AttnRows A;
  float* x;               // [n_streams, n_rows, pitch] logits; null: not wanted
  int64_t pitch;
};
// What a launch does: one set of streams, or two (a shared prefix and the sequences' own rows).
struct FewJobs {
  FewArgs job[2];
  int32_t groups[2];      // of query rows
  int32_t least[2];       // tiles of a CTA, where the stream has them: of shorter streams the last splits are left empty
  int32_t ctas0;          // CTAs of the first set
  int32_t leaving[2];     // the set's tiles leave L2 first
  int32_t order;          // FewOrder
};
struct FewMaps {
  CUtensorMap k[2], v[2];
};
// The query rows r0 .. r0 + g - 1 of a stream.
struct Group {
  int32_t r0, g;
};
// Where their logits go: that of row r0 + r and cached row i to x[r pitch + i]; null: nowhere.
struct Logits {
  float* x;
  int64_t pitch;
};

// This warp's tiles of the CTA's share: every W-th (a warp of the CTA each) of [t0, t1) from t0 + warp on.  Tile number n of the warp has the ring's
// entries 2 n (K) and 2 n + 1 (V).
template <bool kBf16, int D, int W, int N>
struct Ring {
  using F = Few<kBf16, D>;
  const CUtensorMap *mk, *mv;
  unsigned char* tiles;
  uint64_t* full;
  int stream, first_tile, entries;
  uint64_t policy;                               // L2's for the tiles

  __device__ void issue(int e) const {           // one lane
    const CUtensorMap* map = e & 1 ? mv : mk;
    const int s = e % N, row = (first_tile + (e >> 1) * W) * kTile;
    tc::mbar_expect_tx(full + s, F::kTileBytes);
#pragma unroll
    for (int b = 0; b < F::kBoxes; ++b) tma_load_3d(tiles + s * F::kTileBytes + b * kBox, map, b * F::kBoxDims, row, stream, full + s, policy);
  }
  __device__ void start(int lane) const {
    if (lane == 0)
      for (int e = 0; e < min(N, entries); ++e) issue(e);
  }
  __device__ bool wait(int e, int lane, int* abort_flag) const {
    bool ok = true;
    if (lane == 0) ok = tc::wait_bar(full + e % N, (uint32_t)(e / N) & 1u, abort_flag);
    ok = __shfl_sync(0xffffffffu, ok, 0);
    __syncwarp();
    return ok;
  }
  __device__ void next(int e, int lane) const {  // entry e has been read by the whole warp
    __syncwarp();
    if (lane == 0 && e + N < entries) issue(e + N);
  }
  // A wait gave up: the copies behind entry e that have been asked for are waited for, within limits, before the ring is left.
  __device__ void drain(int e, int lane) const {
    if (lane != 0) return;
    const long long t0 = clock64();
    for (int i = e; i < min(e + N, entries); ++i)
      while (!tc::mbar_try_wait(full + i % N, (uint32_t)(i / N) & 1u) && clock64() - t0 < tc::kWaitCycles) {}
  }
  __device__ const unsigned char* at(int e) const { return tiles + e % N * F::kTileBytes; }
};

// Byte offset of 16-byte piece p of a row.
__device__ inline uint32_t tile_off(int row, int piece) {
  return (uint32_t)(piece >> 3) * kBox + (uint32_t)row * 128u + (uint32_t)(((piece & 7) ^ (row & 7)) << 4);
}

// Of a warp's tile: the lane's row's log weight, and which rows count (none behind the last, none of weight zero), by bit.  The weight
// of the next tile is asked for a tile ahead.
struct TileWeights {
  const float* w;                                // of the stream; null: ones
  float next = 1.f;
  __device__ void ask(int row, int len) {
    if (w) next = row < len ? w[row] : 0.f;
  }
  __device__ uint32_t take(int rows, float& log_w) const {
    log_w = w ? log2f(next) : 0.f;
    const uint32_t held = rows >= kTile ? 0xffffffffu : (1u << rows) - 1u;
    return w ? held & __ballot_sync(0xffffffffu, !(next == 0.f)) : held;
  }
};

// The warp's sums of its tiles, to mrg[row][kPitch].
template <int D, int W, int N>
__device__ inline void few_warp_bf16(const AttnRows& A, const Group& G, const Logits& X, const Ring<true, D, W, N>& R, int s, int len, int n_tiles, int lane, int* abort_flag,
                                     float* mrg, bool& failed) {
  const int g = G.g;
  // With up to four rows the columns 4-7 repeat the rows 0-3, and in the second product they carry the low parts of the weights:
  // one MMA then does what takes two with more rows.
  const bool packed = g <= 4;
  const int hq = lane >> 2, tq = lane & 3;       // C fragment: cached rows hq, hq + 8; query rows 2 tq, 2 tq + 1
  uint32_t qb[D / 16][2];
  {
    const int hr = packed ? hq & 3 : hq;
    const __nv_bfloat16* qp = static_cast<const __nv_bfloat16*>(A.q) + (hr < g ? attn_row(A, s, G.r0 + hr) : 0) * D;
#pragma unroll
    for (int ks = 0; ks < D / 16; ++ks) {
      qb[ks][0] = hr < g ? __ldcg(reinterpret_cast<const uint32_t*>(qp + ks * 16 + 2 * tq)) : 0u;
      qb[ks][1] = hr < g ? __ldcg(reinterpret_cast<const uint32_t*>(qp + ks * 16 + 8 + 2 * tq)) : 0u;
    }
  }
  int limit[2];
  float* xs[2];
#pragma unroll
  for (int e = 0; e < 2; ++e) {
    const int h = packed ? (2 * tq + e) & 3 : 2 * tq + e;
    limit[e] = h < g ? attn_limit(A, len, G.r0 + h) : 0;
    xs[e] = X.x && 2 * tq + e < g ? X.x + h * X.pitch : nullptr;
  }
  constexpr int kMB = D / 16;
  float o[kMB][4];                               // dim 16 mb + hq + 8 (j >> 1), query row 2 tq + (j & 1)
#pragma unroll
  for (int n = 0; n < kMB; ++n) { o[n][0] = o[n][1] = o[n][2] = o[n][3] = 0.f; }
  float m[2] = {-INFINITY, -INFINITY}, l[2] = {0.f, 0.f};
  const int mi = lane >> 3, mr = lane & 7;
  const int k_row = (mi & 1) * 8 + mr, k_piece = mi >> 1;
  const int v_row = (mi >> 1) * 8 + mr, v_piece = mi & 1;
  TileWeights weights{A.w ? A.w + (int64_t)s * A.cap : nullptr};
  weights.ask(R.first_tile * kTile + lane, len);
  for (int n = 0; n < n_tiles; ++n) {
    const int row0 = (R.first_tile + n * W) * kTile, rows = min(kTile, len - row0);
    float log_w;
    const uint32_t alive = weights.take(rows, log_w);
    weights.ask(row0 + W * kTile + lane, len);
    if (!R.wait(2 * n, lane, abort_flag)) { R.drain(2 * n, lane); failed = true; break; }
    const uint32_t Kt = tc::smem_u32(R.at(2 * n));
    float sa[2][4][4];
#pragma unroll
    for (int tb = 0; tb < 2; ++tb)
#pragma unroll
      for (int c = 0; c < 4; ++c) { sa[tb][c][0] = sa[tb][c][1] = sa[tb][c][2] = sa[tb][c][3] = 0.f; }
#pragma unroll
    for (int kh = 0; kh < D / 64; ++kh) {
      uint32_t ka[4][2][4];
#pragma unroll
      for (int k4 = 0; k4 < 4; ++k4)
#pragma unroll
        for (int tb = 0; tb < 2; ++tb) ldsm_x4(Kt + tile_off(k_row + 16 * tb, (kh * 4 + k4) * 2 + k_piece), ka[k4][tb]);
#pragma unroll
      for (int k4 = 0; k4 < 4; ++k4)
#pragma unroll
        for (int tb = 0; tb < 2; ++tb) mma_bf16(sa[tb][k4], ka[k4][tb], qb[kh * 4 + k4][0], qb[kh * 4 + k4][1]);
    }
    R.next(2 * n, lane);
    float x[2][4];
    bool more = false;
#pragma unroll
    for (int tb = 0; tb < 2; ++tb)
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int in_tile = 16 * tb + hq + 8 * (j >> 1), row = row0 + in_tile;
        const float lw = A.w ? __shfl_sync(0xffffffffu, log_w, in_tile) : 0.f;
        x[tb][j] = row < limit[j & 1] && (alive >> in_tile & 1u) ? fmaf((sa[tb][0][j] + sa[tb][1][j]) + (sa[tb][2][j] + sa[tb][3][j]), A.scale, lw) : -INFINITY;
        if (xs[j & 1] && row < len) xs[j & 1][row] = x[tb][j];
        more = more || x[tb][j] > m[j & 1] + kGrow;
      }
    if (__any_sync(0xffffffffu, more)) {
      float a[2];
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        float mn = fmaxf(m[e], fmaxf(fmaxf(x[0][e], x[0][2 + e]), fmaxf(x[1][e], x[1][2 + e])));
#pragma unroll
        for (int off = 4; off < 32; off <<= 1) mn = fmaxf(mn, __shfl_xor_sync(0xffffffffu, mn, off));
        a[e] = mn == -INFINITY ? 0.f : exp2f(m[e] - mn);
        l[e] *= a[e];
        m[e] = mn;
      }
#pragma unroll
      for (int i = 0; i < kMB; ++i) { o[i][0] *= a[0]; o[i][1] *= a[1]; o[i][2] *= a[0]; o[i][3] *= a[1]; }
    }
    const float base[2] = {m[0] == -INFINITY ? 0.f : m[0], m[1] == -INFINITY ? 0.f : m[1]};
    // The weights enter the second product as bf16, split into a high and a low part (16 bits), so that the error stays that of the
    // final rounding.
    uint32_t bh[2][2], bl[2][2];
#pragma unroll
    for (int tb = 0; tb < 2; ++tb) {
#pragma unroll
      for (int j = 0; j < 4; ++j) x[tb][j] = exp2f(x[tb][j] - base[j & 1]);
      l[0] += x[tb][0] + x[tb][2];
      l[1] += x[tb][1] + x[tb][3];
      const uint32_t ph0 = pack_bf16(x[tb][0], x[tb][1]), ph1 = pack_bf16(x[tb][2], x[tb][3]);
      const uint32_t pl0 = pack_bf16(x[tb][0] - bf16_lo(ph0), x[tb][1] - bf16_hi(ph0));
      const uint32_t pl1 = pack_bf16(x[tb][2] - bf16_lo(ph1), x[tb][3] - bf16_hi(ph1));
      bh[tb][0] = movm_trans(packed && tq >= 2 ? pl0 : ph0);
      bh[tb][1] = movm_trans(packed && tq >= 2 ? pl1 : ph1);
      bl[tb][0] = packed ? 0u : movm_trans(pl0);
      bl[tb][1] = packed ? 0u : movm_trans(pl1);
    }
    if (!R.wait(2 * n + 1, lane, abort_flag)) { R.drain(2 * n + 1, lane); failed = true; break; }
    const uint32_t Vt = tc::smem_u32(R.at(2 * n + 1));
#pragma unroll
    for (int tb = 0; tb < 2; ++tb) {
      // a row that does not count is replaced by one that does, times zero: what it holds may be anything
      const int row = alive >> (v_row + 16 * tb) & 1u ? v_row + 16 * tb : __ffs(alive) - 1;
      if (alive == 0) break;
      uint32_t va[kMB][4];
#pragma unroll
      for (int mb = 0; mb < kMB; ++mb) ldsm_x4_trans(Vt + tile_off(row, mb * 2 + v_piece), va[mb]);
#pragma unroll
      for (int mb = 0; mb < kMB; ++mb) mma_bf16(o[mb], va[mb], bh[tb][0], bh[tb][1]);
      if (!packed) {
#pragma unroll
        for (int mb = 0; mb < kMB; ++mb) mma_bf16(o[mb], va[mb], bl[tb][0], bl[tb][1]);
      }
    }
    R.next(2 * n + 1, lane);
  }
#pragma unroll
  for (int off = 4; off < 32; off <<= 1) {
    l[0] += __shfl_xor_sync(0xffffffffu, l[0], off);
    l[1] += __shfl_xor_sync(0xffffffffu, l[1], off);
  }
  if (packed) {
#pragma unroll
    for (int n = 0; n < kMB; ++n)
#pragma unroll
      for (int j = 0; j < 4; ++j) o[n][j] += __shfl_xor_sync(0xffffffffu, o[n][j], 2);
  }
  __syncthreads();                               // every warp is done with its ring
#pragma unroll
  for (int e = 0; e < 2; ++e) {
    const int h = 2 * tq + e;
    if (h >= g) continue;
    float* to = mrg + h * Few<true, D>::kPitch;
#pragma unroll
    for (int n = 0; n < kMB; ++n) { to[16 * n + hq] = o[n][e]; to[16 * n + 8 + hq] = o[n][2 + e]; }
    if (hq == 0) { to[D] = m[e]; to[D + 1] = l[e]; }
  }
}

// The same with FFMA; kR >= g rows.  What bounds it is shared memory, whose loads return 128 bytes a cycle whether lanes read the same or not, so
// nothing is read that registers can hold.  Logits: kG neighbouring lanes share kG rows of the tile, every lane with a part of the
// channels of all of them and that part of the queries in registers; a lane ends up with the logit of row `lane`.  Sums: the lanes are kT
// sets that take every kT-th row, each lane a part of the columns.  (A lane per row with the queries read from shared memory, and all
// lanes on every row of V: 4300 cycles a tile of d = 64 and four queries.)
// qs: [kR][D]; ps: [kR][32] of this warp.
template <int D, int kR, int W, int N>
__device__ inline void few_warp_fp32(const AttnRows& A, const Group& G, const Logits& X, const Ring<false, D, W, N>& R, int s, int len, int n_tiles, int lane, int* abort_flag,
                                     const float* qs, float* ps, float* mrg, bool& failed) {
  const int g = G.g;
  constexpr int kAtOnce = kR < 4 ? kR : 4;       // queries whose logits are formed together; of more, they come from shared memory for each tile
  constexpr int kG = kAtOnce * D / 4 <= 64 ? 4 : 8, kPieces = D / 4 / kG;      // 16-byte pieces of a row that a lane takes: its number + kG c
  constexpr int kT = kR * D / 8 <= 64 ? 4 : 2, kLanes = 32 / kT, kC = D / 4 / kLanes;
  float2 q[kAtOnce][kPieces][2];
  auto ask = [&](int r0) {                       // the queries r0 .. r0 + kAtOnce - 1
#pragma unroll
    for (int r = 0; r < kAtOnce; ++r)
#pragma unroll
      for (int c = 0; c < kPieces; ++c) {
        const float4 w = *reinterpret_cast<const float4*>(qs + (r0 + r) * D + 4 * (lane % kG + kG * c));
        q[r][c][0] = make_float2(w.x, w.y);
        q[r][c][1] = make_float2(w.z, w.w);
      }
  };
  if (kR <= kAtOnce) ask(0);
  float2 o[kR][kC][2];
  float m[kR], l[kR];
  int limit[kR];
#pragma unroll
  for (int r = 0; r < kR; ++r) {
    m[r] = -INFINITY;
    l[r] = 0.f;
    limit[r] = r < g ? attn_limit(A, len, G.r0 + r) : 0;
#pragma unroll
    for (int c = 0; c < kC; ++c) o[r][c][0] = o[r][c][1] = make_float2(0.f, 0.f);
  }
  // piece c of this lane's columns: box and place of it
  const int set = lane / kLanes, in_set = lane % kLanes;
  auto piece = [&](int c) { return (in_set & 7) + 8 * ((in_set >> 3) + c * (kLanes / 8)); };
  TileWeights weights{A.w ? A.w + (int64_t)s * A.cap : nullptr};
  weights.ask(R.first_tile * kTile + lane, len);
  for (int n = 0; n < n_tiles; ++n) {
    const int row0 = (R.first_tile + n * W) * kTile, row = row0 + lane;
    float log_w;
    const uint32_t alive = weights.take(len - row0, log_w);
    weights.ask(row + W * kTile, len);
    if (!R.wait(2 * n, lane, abort_flag)) { R.drain(2 * n, lane); failed = true; break; }
    const unsigned char* Kt = R.at(2 * n);
    float x[kR];
    bool more = false;
#pragma unroll
    for (int r0 = 0; r0 < kR; r0 += kAtOnce) {
      if (kR > kAtOnce) ask(r0);
      float part[kAtOnce][kG];
#pragma unroll
      for (int i = 0; i < kG; ++i) {
        float2 acc[kAtOnce];
#pragma unroll
        for (int r = 0; r < kAtOnce; ++r) acc[r] = make_float2(0.f, 0.f);
#pragma unroll
        for (int c = 0; c < kPieces; ++c) {
          const float4 k = *reinterpret_cast<const float4*>(Kt + tile_off((lane & ~(kG - 1)) + i, lane % kG + kG * c));
#pragma unroll
          for (int r = 0; r < kAtOnce; ++r) {
            acc[r] = __ffma2_rn(make_float2(k.x, k.y), q[r][c][0], acc[r]);
            acc[r] = __ffma2_rn(make_float2(k.z, k.w), q[r][c][1], acc[r]);
          }
        }
#pragma unroll
        for (int r = 0; r < kAtOnce; ++r) part[r][i] = acc[r].x + acc[r].y;
      }
#pragma unroll
      for (int r = r0; r < r0 + kAtOnce; ++r) {
        const float dot = sum_scatter<kG>(part[r - r0], lane);
        x[r] = row < limit[r] && (alive >> lane & 1u) ? fmaf(dot, A.scale, log_w) : -INFINITY;
        if (X.x && r < g && row < len) X.x[r * X.pitch + row] = x[r];
        more = more || x[r] > m[r] + kGrow;
      }
    }
    R.next(2 * n, lane);
    if (__any_sync(0xffffffffu, more)) {
#pragma unroll
      for (int r = 0; r < kR; ++r) {
        const float mn = fmaxf(m[r], warp_max(x[r])), a = mn == -INFINITY ? 0.f : exp2f(m[r] - mn);
        m[r] = mn;
        l[r] *= a;
#pragma unroll
        for (int c = 0; c < kC; ++c) {
          o[r][c][0] = __fmul2_rn(o[r][c][0], make_float2(a, a));
          o[r][c][1] = __fmul2_rn(o[r][c][1], make_float2(a, a));
        }
      }
    }
#pragma unroll
    for (int r = 0; r < kR; ++r) {
      const float p = exp2f(x[r] - (m[r] == -INFINITY ? 0.f : m[r]));
      l[r] += p;
      ps[r * 32 + lane % kT * kLanes + lane / kT] = p;     // a set's rows next to one another
    }
    if (!R.wait(2 * n + 1, lane, abort_flag)) { R.drain(2 * n + 1, lane); failed = true; break; }        // (a warp barrier too: the weights are there)
    const unsigned char* Vt = R.at(2 * n + 1);
#pragma unroll
    for (int t0 = 0; t0 < kLanes; t0 += 4) {               // the set's rows t0 .. t0 + 3
      float4 v[4][kC];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int t = (t0 + i) * kT + set;
#pragma unroll
        for (int c = 0; c < kC; ++c) v[i][c] = *reinterpret_cast<const float4*>(Vt + tile_off(t, piece(c)));
        if (alive != 0xffffffffu && !(alive >> t & 1u)) {  // does not count: what it holds may be anything
#pragma unroll
          for (int c = 0; c < kC; ++c) v[i][c] = make_float4(0.f, 0.f, 0.f, 0.f);
        }
      }
#pragma unroll
      for (int r = 0; r < kR; ++r) {
        const float4 p4 = *reinterpret_cast<const float4*>(ps + r * 32 + set * kLanes + t0);
        const float p[4] = {p4.x, p4.y, p4.z, p4.w};
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
          for (int c = 0; c < kC; ++c) {
            o[r][c][0] = __ffma2_rn(make_float2(v[i][c].x, v[i][c].y), make_float2(p[i], p[i]), o[r][c][0]);
            o[r][c][1] = __ffma2_rn(make_float2(v[i][c].z, v[i][c].w), make_float2(p[i], p[i]), o[r][c][1]);
          }
      }
    }
    R.next(2 * n + 1, lane);
  }
  __syncthreads();
#pragma unroll
  for (int r = 0; r < kR; ++r) {
    const float sum = warp_sum(l[r]);
    float* to = mrg + r * Few<false, D>::kPitch;
#pragma unroll
    for (int c = 0; c < kC; ++c) {
      float w[4] = {o[r][c][0].x, o[r][c][0].y, o[r][c][1].x, o[r][c][1].y};
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int off = kLanes; off < 32; off <<= 1) w[i] += __shfl_xor_sync(0xffffffffu, w[i], off);
      if (r < g && set == 0) *reinterpret_cast<float4*>(to + 4 * piece(c)) = make_float4(w[0], w[1], w[2], w[3]);
    }
    if (r < g && lane == 0) { to[D] = m[r]; to[D + 1] = sum; }
  }
}

// What a CTA needs in shared memory besides the rings.
template <bool kBf16, int D, int kR, int W, int N>
struct FewShared {
  uint64_t full[W][N];
  int abort_flag;
  __align__(16) float qs[kBf16 ? 4 : kR * D];
  __align__(16) float ps[kBf16 ? 4 : W * kR * 32];
};

// The CTA's share [t0, t1) of the tiles: every warp's sums, to mrg[warp][row][kPitch] in the rings' place.
template <bool kBf16, int D, int kR, int W, int N>
__device__ inline void few_tiles(const AttnRows& A, const Group& G, const Logits& X, const CUtensorMap& mk, const CUtensorMap& mv, FewShared<kBf16, D, kR, W, N>& sh, unsigned char* tiles,
                                 int s, int len, int t0, int t1, bool leaving) {
  using F = Few<kBf16, D>;
  const int tid = threadIdx.x, warp = tid / 32, lane = tid % 32;
  const int n_tiles = max(0, (t1 - t0 - warp + W - 1) / W);
  const Ring<kBf16, D, W, N> R{&mk, &mv, tiles + warp * N * F::kTileBytes, sh.full[warp], s, t0 + warp, 2 * n_tiles, l2_policy(leaving)};
  R.start(lane);
  if constexpr (!kBf16) {
    for (int i = tid; i < kR * D; i += 32 * W)
      sh.qs[i] = i / D < G.g ? __ldcg(static_cast<const float*>(A.q) + attn_row(A, s, G.r0 + i / D) * D + i % D) : 0.f;
    __syncthreads();
  }
  float* mrg = reinterpret_cast<float*>(tiles) + warp * kFewRows * F::kPitch;
  bool failed = false;
  if constexpr (kBf16) few_warp_bf16<D, W, N>(A, G, X, R, s, len, n_tiles, lane, &sh.abort_flag, mrg, failed);
  else few_warp_fp32<D, kR, W, N>(A, G, X, R, s, len, n_tiles, lane, &sh.abort_flag, sh.qs, sh.ps + warp * kR * 32, mrg, failed);
  if (failed && lane == 0) tc::st_release(&sh.abort_flag, 1);
  __syncthreads();
}

template <bool kBf16, int D, int kR, int W, int N>
__device__ inline void few_init(FewShared<kBf16, D, kR, W, N>& sh, const CUtensorMap& mk, const CUtensorMap& mv) {
  if (threadIdx.x != 0) return;
  asm volatile("prefetch.tensormap [%0];" ::"l"(&mk) : "memory");
  asm volatile("prefetch.tensormap [%0];" ::"l"(&mv) : "memory");
  for (int i = 0; i < W * N; ++i) tc::mbar_init(&sh.full[0][0] + i, 1);
  sh.abort_flag = 0;
  asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
}

// `n` sets of sums, the i-th at from(i)[kPitch], brought to one maximum and added by a warp: its lane's D / 32 columns.
template <int D, int kMost, class From>
__device__ inline void few_join(int n, int lane, From from, float (&acc)[D / 32], float& top, float& sum) {
  constexpr int kC = D / 32;
  float m[kMost], l[kMost], v[kMost][kC];
  top = -INFINITY;
#pragma unroll
  for (int i = 0; i < kMost; ++i) {
    m[i] = -INFINITY;
    l[i] = 0.f;
    if (i < n) {
      const float* at = from(i);
      m[i] = at[D];
      l[i] = at[D + 1];
#pragma unroll
      for (int c = 0; c < kC; ++c) v[i][c] = at[lane * kC + c];
    }
    top = fmaxf(top, m[i]);
  }
  const float base = top == -INFINITY ? 0.f : top;
  sum = 0.f;
#pragma unroll
  for (int c = 0; c < kC; ++c) acc[c] = 0.f;
#pragma unroll
  for (int i = 0; i < kMost; ++i) {
    if (i >= n) break;
    const float f = exp2f(m[i] - base);
    sum = fmaf(l[i], f, sum);
#pragma unroll
    for (int c = 0; c < kC; ++c) acc[c] = fmaf(v[i][c], f, acc[c]);
  }
}

template <bool kBf16, int D>
__device__ inline void few_put(const AttnRows& A, int64_t row, int lane, const float (&acc)[D / 32], float sum) {
  constexpr int kC = D / 32;
  const float inv = sum == 0.f ? 0.f : 1.f / sum;
#pragma unroll
  for (int c = 0; c < kC; c += 2) {
    if constexpr (kBf16)
      *reinterpret_cast<__nv_bfloat162*>(static_cast<__nv_bfloat16*>(A.out) + row * D + lane * kC + c) = __floats2bfloat162_rn(acc[c] * inv, acc[c + 1] * inv);
    else
      *reinterpret_cast<float2*>(static_cast<float*>(A.out) + row * D + lane * kC + c) = make_float2(acc[c] * inv, acc[c + 1] * inv);
  }
}

// A row's sums and those of the slots before its own, by a warp.
template <int D>
__device__ inline void join_before(const AttnRows& A, int64_t row, int lane, float (&acc)[D / 32], float top, float& sum) {
  constexpr int kC = D / 32, kChunks = kAttnMaxSplits / 32, kAhead = 6;
  float2 ml[kChunks];
  float most = top, f[kChunks];
#pragma unroll
  for (int k = 0; k < kChunks; ++k) {
    ml[k] = lane + 32 * k < A.slot0 ? A.part_ml[(int64_t)(lane + 32 * k) * A.total_rows + row] : make_float2(-INFINITY, 0.f);
    most = fmaxf(most, ml[k].x);
  }
  most = warp_max(most);
  const float base = most == -INFINITY ? 0.f : most, own = exp2f(top - base);
  float rest = 0.f;
#pragma unroll
  for (int k = 0; k < kChunks; ++k) {
    f[k] = exp2f(ml[k].x - base);
    rest = fmaf(ml[k].y, f[k], rest);
  }
  sum = fmaf(sum, own, warp_sum(rest));
#pragma unroll
  for (int c = 0; c < kC; ++c) acc[c] *= own;
#pragma unroll
  for (int k = 0; k < kChunks; ++k)
    for (int i0 = 32 * k; i0 < min(32 * k + 32, A.slot0); i0 += kAhead) {
      float v[kAhead][kC];
#pragma unroll
      for (int j = 0; j < kAhead; ++j) {
        const float* from = A.part + ((int64_t)(i0 + j) * A.total_rows + row) * D + lane * kC;
        const bool in = i0 + j < min(32 * k + 32, A.slot0);
#pragma unroll
        for (int c = 0; c < kC; c += 2) {
          const float2 x = in ? *reinterpret_cast<const float2*>(from + c) : make_float2(0.f, 0.f);
          v[j][c] = x.x;
          v[j][c + 1] = x.y;
        }
      }
#pragma unroll
      for (int j = 0; j < kAhead; ++j) {
        if (i0 + j >= min(32 * k + 32, A.slot0)) break;
        const float w = __shfl_sync(0xffffffffu, f[k], i0 + j & 31);
#pragma unroll
        for (int c = 0; c < kC; ++c) acc[c] = fmaf(v[j][c], w, acc[c]);
      }
    }
}

// kR: rows that the fp32 form takes (bf16: 8).  kCtas share an SM (more than two: few_crowded).
template <bool kBf16, int D, int kR, int kCtas>
__global__ void __launch_bounds__(32 * few_warps(kBf16, D), kCtas) attn_few_kernel(const __grid_constant__ FewJobs J, const __grid_constant__ FewMaps maps) {
  using F = Few<kBf16, D>;
  constexpr int W = few_warps(kBf16, D), N = kCtas == 2 ? F::kRing : crowd_ring(D);
  extern __shared__ unsigned char smem_raw[];
  __shared__ FewShared<kBf16, D, kR, W, N> sh;
  unsigned char* tiles = smem_raw + (-tc::smem_u32(smem_raw) & 1023u);
  const int which = (int)blockIdx.x >= J.ctas0, cta = blockIdx.x - (which ? J.ctas0 : 0);
  const AttnRows& A = J.job[which].A;
  const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
  // the groups of a stream's query rows next to one another: they read the same rows
  const int group = cta % J.groups[which], split = cta / J.groups[which] % A.splits, s = cta / J.groups[which] / A.splits;
  constexpr int kGroup = group_rows(kBf16, D);
  const Group G{group * kGroup, min(kGroup, A.n_rows - group * kGroup)};
  few_init(sh, maps.k[which], maps.v[which]);
  // A launch beside or behind the prefix's reads nothing that that writes, until it joins its slots, and nothing that came before is still to
  // be written: the prefix's launch releases its dependents behind its own wait.
  const bool early = J.order != kFewAlone;
  if (!early) grid_wait_and_release();
  __syncthreads();
  const int len = attn_len(A, s), n_all = (len + kTile - 1) / kTile;
  const int used = max(1, min(A.splits, (n_all + J.least[which] - 1) / J.least[which]));      // splits
  if (split >= used) {
    if (warp == 0 && lane < G.g) A.part_ml[(int64_t)(A.slot0 + split) * A.total_rows + attn_row(A, s, G.r0 + lane)] = make_float2(-INFINITY, 0.f);
    if (early && blockIdx.x == gridDim.x - 1) grid_wait_and_release();
    return;
  }
  const int64_t pitch = J.job[which].pitch;
  const Logits X{J.job[which].x ? J.job[which].x + ((int64_t)s * A.n_rows + G.r0) * pitch : nullptr, pitch};
  few_tiles(A, G, X, maps.k[which], maps.v[which], sh, tiles, s, len, (int)((int64_t)n_all * split / used), (int)((int64_t)n_all * (split + 1) / used), J.leaving[which]);
  const float* mrg = reinterpret_cast<const float*>(tiles);
  if (J.order == kFewFinish) grid_wait_and_release();
  for (int r = warp; r < G.g; r += W) {
    float acc[D / 32], top, sum;
    few_join<D, W>(W, lane, [&](int w) { return mrg + (w * kFewRows + r) * F::kPitch; }, acc, top, sum);
    if (sh.abort_flag) sum = NAN;
    const int64_t row = attn_row(A, s, G.r0 + r);
    if (J.order == kFewFinish) {
      join_before<D>(A, row, lane, acc, top, sum);
      few_put<kBf16, D>(A, row, lane, acc, sum);
      continue;
    }
    if (A.n_slots > 1) {
      const int64_t at = (int64_t)(A.slot0 + split) * A.total_rows + row;
      if (lane == 0) A.part_ml[at] = make_float2(top, sum);
#pragma unroll
      for (int c = 0; c < D / 32; c += 2) *reinterpret_cast<float2*>(A.part + at * D + lane * (D / 32) + c) = make_float2(acc[c], acc[c + 1]);
      continue;
    }
    if (A.lse && lane == 0) A.lse[row] = sum == 0.f ? INFINITY : (top == -INFINITY ? 0.f : top) + log2f(sum);
    few_put<kBf16, D>(A, row, lane, acc, sum);
  }
  // The launch ends behind the prefix's, so that what waits for the one has both: one CTA waits.
  if (J.order == kFewBeside && blockIdx.x == gridDim.x - 1) grid_wait_and_release();
}

// A row's weight from its logit; a row that the query does not see has none, whatever the query's sum is.
__device__ inline float logit_weight(float x, float lse) { return x == -INFINITY ? 0.f : exp2f(x - lse); }

// The splits of a stream as a cluster of CTAs, where its logits fit their shared memory: they join their sums through it, every
// CTA then turns its own logits into weights, and nothing but results leaves the chip.  More than eight query rows are groups with a
// cluster each; what a cached row receives from a group goes to `sums` [groups, n_streams, cap] (one group: to the scores).
constexpr int kMaxCluster = 8;
// CTAs of a launch, by clusters of C, that all run at once: of fp32 rows with 128 dims, which have an SM to themselves, as many as the device takes (120
// by clusters of 8, 132 by 4, 148; 64 streams of 250 such rows, 128 CTAs: 9.7 us in a graph against 11.6 by two launches, 80 of 200, 160 CTAs:
// 16.9 against 13.0), of others two an SM, less than the 264 to 296 that it takes.
constexpr int most_clustered(int C, bool alone) { return alone ? (C > 4 ? 120 : C > 2 ? 132 : 148) : C > 4 ? 192 : 256; }
constexpr int logit_bytes(bool bf16, int d) { return !bf16 && d == 64 ? 8 * 1024 : 15 * 1024; }       // of a CTA: two (fp32, d = 128: one) still fit an SM

template <bool kBf16, int D, int kR>
__global__ void __launch_bounds__(kThreads, (Few<kBf16, D>::kCtas))
attn_few_cluster_kernel(const __grid_constant__ AttnRows A, const ScoreArgs S, int pitch, float* sums, const __grid_constant__ CUtensorMap mk, const __grid_constant__ CUtensorMap mv) {
  namespace cg = cooperative_groups;
  using F = Few<kBf16, D>;
  extern __shared__ unsigned char smem_raw[];
  __shared__ FewShared<kBf16, D, kR, kWarps, F::kRing> sh;
  __shared__ float lse[kFewRows];
  unsigned char* tiles = smem_raw + (-tc::smem_u32(smem_raw) & 1023u);
  float* x = reinterpret_cast<float*>(tiles + kWarps * F::kRing * F::kTileBytes);      // [g][pitch]
  float* joined = reinterpret_cast<float*>(tiles) + kWarps * kFewRows * F::kPitch;     // [g][kPitch] of the CTA, behind its warps'
  cg::cluster_group cluster = cg::this_cluster();
  const int tid = threadIdx.x, warp = tid / 32, lane = tid % 32;
  const int C = (int)gridDim.y, c = blockIdx.y, s = blockIdx.x % A.n_streams, group = blockIdx.x / A.n_streams;
  const Group G{group * kFewRows, min(kFewRows, A.n_rows - group * kFewRows)};
  few_init(sh, mk, mv);
  grid_wait_and_release();
  __syncthreads();
  const int len = attn_len(A, s), n_all = (len + kTile - 1) / kTile;
  const int t0 = (int)((int64_t)n_all * c / C), t1 = (int)((int64_t)n_all * (c + 1) / C);
  const int row0 = t0 * kTile, row1 = min(len, t1 * kTile);
  few_tiles(A, G, Logits{x - row0, pitch}, mk, mv, sh, tiles, s, len, t0, t1, false);
  const float* mrg = reinterpret_cast<const float*>(tiles);
  for (int r = warp; r < G.g; r += kWarps) {
    float acc[D / 32], top, sum;
    few_join<D, kWarps>(kWarps, lane, [&](int w) { return mrg + (w * kFewRows + r) * F::kPitch; }, acc, top, sum);
    if (sh.abort_flag) sum = NAN;
    float* to = joined + r * F::kPitch;
#pragma unroll
    for (int i = 0; i < D / 32; ++i) to[lane * (D / 32) + i] = acc[i];
    if (lane == 0) { to[D] = top; to[D + 1] = sum; }
  }
  // The old scores of this CTA's rows, the first kOld per thread, on their way while the cluster meets.
  constexpr int kOld = 4;
  const int64_t first = (int64_t)s * A.cap;
  float old[kOld];
#pragma unroll
  for (int j = 0; j < kOld; ++j) old[j] = !sums && row0 + tid + j * kThreads < row1 ? score_old(S, first + row0 + tid + j * kThreads) : 0.f;
  cluster.sync();
  // The rows' sums over the cluster, a lane per CTA: two rows of every warp's, asked for together.
  static_assert(kFewRows <= 2 * kWarps, "two rows a warp");
  float2 ml[2];
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int r = warp + i * kWarps;
    const float* at = cluster.map_shared_rank(joined, lane < C ? lane : 0) + r * F::kPitch;
    ml[i] = lane < C && r < G.g ? make_float2(at[D], at[D + 1]) : make_float2(-INFINITY, 0.f);
  }
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int r = warp + i * kWarps;
    const float top = warp_max(ml[i].x), base = top == -INFINITY ? 0.f : top, sum = warp_sum(ml[i].y * exp2f(ml[i].x - base));
    const bool counted = (G.r0 + r) % A.n_queries >= A.n_queries - S.n_scored;
    if (lane == 0 && r < G.g) lse[r] = sum == 0.f || !counted ? INFINITY : base + log2f(sum);
  }
  // The outputs: a warp of the cluster's each, the last warps first.
  for (int r = c + C * (kWarps - 1 - warp); r < G.g; r += C * kWarps) {
    float acc[D / 32], top, sum;
    few_join<D, kMaxCluster>(C, lane, [&](int b) { return cluster.map_shared_rank(joined, b) + r * F::kPitch; }, acc, top, sum);
    few_put<kBf16, D>(A, attn_row(A, s, G.r0 + r), lane, acc, sum);
  }
  __syncthreads();
  auto left = cluster.barrier_arrive();          // this CTA reads nobody's sums any more
  auto put = [&](int i, float before) {
    float sum = 0.f;
    for (int r = 0; r < G.g; ++r) sum += logit_weight(x[r * pitch + i - row0], lse[r]);
    if (sums) sums[(int64_t)group * A.n_streams * A.cap + first + i] = sum;
    else score_put(S, first + i, before, sum);
  };
#pragma unroll
  for (int j = 0; j < kOld; ++j)
    if (row0 + tid + j * kThreads < row1) put(row0 + tid + j * kThreads, old[j]);
  for (int i = row0 + tid + kOld * kThreads; i < row1; i += kThreads) put(i, sums ? 0.f : score_old(S, first + i));
  cluster.barrier_wait(std::move(left));         // nobody reads this CTA's
}

// The scores from the groups' sums.
constexpr int kEndThreads = 256;
__global__ void __launch_bounds__(kEndThreads) few_sum_kernel(const __grid_constant__ AttnRows A, const ScoreArgs S, const float* __restrict__ sums, int groups, int chunks) {
  const int s = blockIdx.x / chunks, i = blockIdx.x % chunks * kEndThreads + threadIdx.x;
  grid_wait_and_release();
  if (i >= attn_len(A, s)) return;
  const int64_t at = (int64_t)s * A.cap + i, step = (int64_t)A.n_streams * A.cap;
  float sum = 0.f;
#pragma unroll 8
  for (int k = 0; k < groups; ++k) sum += sums[k * step + at];
  score_put(S, at, sum);
}

// Behind attn_few_kernel with one group of query rows: the first `joins` CTAs join the splits; the others turn 1024 logits per query
// row into weights and add those of the scored rows up.
constexpr int kEndKeys = 1024;
template <bool kBf16, int D>
__global__ void __launch_bounds__(kEndThreads, 4) few_end_kernel(const __grid_constant__ FewArgs P, const ScoreArgs S, int joins, int chunks) {
  __shared__ float lse[kFewRows];
  __shared__ JoinShared<D> join;
  const AttnRows& A = P.A;
  const int tid = threadIdx.x, warp = tid / 32, lane = tid % 32;
  if ((int)blockIdx.x < joins) {
    grid_wait_and_release();
    join_splits<kBf16, D, 2>(A, blockIdx.x, join);
    return;
  }
  // What attn_few_kernel does not write is asked for before it has ended, and what does not depend on the sums ahead of them.
  const int s = ((int)blockIdx.x - joins) / chunks, k0 = ((int)blockIdx.x - joins) % chunks * kEndKeys;
  const int len = attn_len(A, s);
  constexpr int kPer = kEndKeys / kEndThreads;
  const float* x = P.x + (int64_t)s * A.n_rows * P.pitch + k0 + tid;
  float logit[kFewRows][kPer], old[kPer];
#pragma unroll
  for (int j = 0; j < kPer; ++j) old[j] = k0 + tid + j * kEndThreads < len ? score_old(S, (int64_t)s * A.cap + k0 + tid + j * kEndThreads) : 0.f;
  grid_wait_and_release();
  if (k0 >= len) return;
#pragma unroll
  for (int r = 0; r < kFewRows; ++r)
#pragma unroll
    for (int j = 0; j < kPer; ++j) logit[r][j] = r < A.n_rows && k0 + tid + j * kEndThreads < len ? x[r * P.pitch + j * kEndThreads] : -INFINITY;
  if (warp < A.n_rows) {                         // (eight warps, at most eight rows)
    const int64_t row = attn_row(A, s, warp);
    float v = 0.f;
    if (A.n_slots > 1) {
      float2 ml[kAttnMaxSplits / 32];
      float top = -INFINITY, l = 0.f;
#pragma unroll
      for (int i = 0; i < kAttnMaxSplits / 32; ++i) {
        ml[i] = lane + 32 * i < A.n_slots ? A.part_ml[(int64_t)(lane + 32 * i) * A.total_rows + row] : make_float2(-INFINITY, 0.f);
        top = fmaxf(top, ml[i].x);
      }
      top = warp_max(top);
      const float base = top == -INFINITY ? 0.f : top;
#pragma unroll
      for (int i = 0; i < kAttnMaxSplits / 32; ++i) l = fmaf(ml[i].y, exp2f(ml[i].x - base), l);
      l = warp_sum(l);
      v = l == 0.f ? INFINITY : base + log2f(l);
    } else {
      v = A.lse[row];
    }
    if (warp % A.n_queries < A.n_queries - S.n_scored) v = INFINITY;      // not counted
    if (lane == 0) lse[warp] = v;
  }
  __syncthreads();
  float sum[kPer] = {};
#pragma unroll
  for (int r = 0; r < kFewRows; ++r) {
    if (r >= A.n_rows) break;
    const float off = lse[r];
#pragma unroll
    for (int j = 0; j < kPer; ++j) sum[j] += exp2f(logit[r][j] - off);
  }
#pragma unroll
  for (int j = 0; j < kPer; ++j) {
    const int key = k0 + tid + j * kEndThreads;
    if (key >= len) continue;
    if (sum[j] != sum[j]) {                      // some query's sum is not a number: whether this row is seen by it, from the logits again
      sum[j] = 0.f;
      for (int r = 0; r < A.n_rows; ++r) sum[j] += logit_weight(x[r * P.pitch + j * kEndThreads], lse[r]);
    }
    score_put(S, (int64_t)s * A.cap + key, old[j], sum[j]);
  }
}

// kR for n_rows query rows, of which a CTA takes kMost at most.
template <bool kBf16, int kMost, class Run>
cudaError_t for_rows(int n_rows, Run run) {
  if constexpr (kBf16) return run(std::integral_constant<int, 8>{});
  else if constexpr (kMost == 4) return n_rows <= 2 ? run(std::integral_constant<int, 2>{}) : run(std::integral_constant<int, 4>{});
  else return n_rows <= 2 ? run(std::integral_constant<int, 2>{}) : n_rows <= 4 ? run(std::integral_constant<int, 4>{}) : run(std::integral_constant<int, 8>{});
}

template <bool kBf16, int D>
cudaError_t launch_few(const FewArgs& P, const FewArgs* also, FewOrder order, cudaStream_t st) {
  using F = Few<kBf16, D>;
  FewJobs J{};
  J.order = order;
  FewMaps maps;
  int64_t ctas = 0;
  int most = 0;
  for (int i = 0; i < (also ? 2 : 1); ++i) {
    const AttnRows& A = (J.job[i] = i ? *also : P).A;
    cudaError_t e = cache_map(&maps.k[i], A.K, kBf16, D, A.cap, A.n_streams, kTile);
    if (e == cudaSuccess) e = cache_map(&maps.v[i], A.V, kBf16, D, A.cap, A.n_streams, kTile);
    if (e != cudaSuccess) return e;
    J.groups[i] = (A.n_rows + group_rows(kBf16, D) - 1) / group_rows(kBf16, D);
    const int64_t mine = (int64_t)J.groups[i] * A.splits * A.n_streams;
    // Of caches beyond L2's size (126 MB) that are read once, the tiles leave first, so that logits and partial results stay (256 streams of up to
    // 8192 rows, five scored query rows: 102.0 us without, 95.7 so; 1024 of up to 1024: 55.5 and 52.2).  (Beside a prefix, which others read from L2, it gains nothing.)
    J.leaving[i] = order == kFewAlone && J.groups[i] == 1 && (int64_t)A.n_streams * A.cap * 2 * D * F::kEsz > ((int64_t)126 << 20);
    J.least[i] = few_warps(kBf16, D) * (mine > 4 * kAttnSms ? 8 : 1);
    ctas += mine;
    if (i == 0) J.ctas0 = (int)ctas;
    most = std::max(most, A.n_rows);
  }
  if (!also) {
    maps.k[1] = maps.k[0];
    maps.v[1] = maps.v[0];
  }
  if (ctas > INT32_MAX) return cudaErrorInvalidValue;
  return for_rows<kBf16, group_rows(kBf16, D)>(most, [&](auto rows) {
    auto run = [&](auto kern, int ring, std::atomic<unsigned long long>& devices) {
      constexpr int W = few_warps(kBf16, D);
      const size_t smem = 1024 + (size_t)W * ring * F::kTileBytes;
      const cudaError_t e = kernel_limits(kern, smem, devices);
      if (e != cudaSuccess) return e;
      const PdlConfig pc(dim3((unsigned)ctas), 32 * W, smem, st);
      return cudaLaunchKernelEx(&pc.cfg, kern, J, maps);
    };
    constexpr int kR = decltype(rows)::value;
    static std::atomic<unsigned long long> devices[2];
    if constexpr (kBf16)
      if (few_crowded(kBf16, ctas)) return run(attn_few_kernel<kBf16, D, kR, crowd_ctas(D)>, crowd_ring(D), devices[1]);
    return run(attn_few_kernel<kBf16, D, kR, 2>, F::kRing, devices[0]);
  });
}

int logit_pitch(int cap, int C) { return ((cap + kTile - 1) / kTile + C - 1) / C * kTile; }

template <bool kBf16, int D>
cudaError_t launch_cluster(const AttnRows& A, const ScoreArgs& S, int C, float* sums, cudaStream_t st) {
  using F = Few<kBf16, D>;
  CUtensorMap mk, mv;
  cudaError_t e = cache_map(&mk, A.K, kBf16, D, A.cap, A.n_streams, kTile);
  if (e == cudaSuccess) e = cache_map(&mv, A.V, kBf16, D, A.cap, A.n_streams, kTile);
  if (e != cudaSuccess) return e;
  const int groups = (A.n_rows + kFewRows - 1) / kFewRows;
  e = for_rows<kBf16, kFewRows>(A.n_rows, [&](auto rows) {
    auto kern = attn_few_cluster_kernel<kBf16, D, decltype(rows)::value>;
    static std::atomic<unsigned long long> devices{0};
    const cudaError_t e = kernel_limits(kern, F::kSmem + logit_bytes(kBf16, D), devices);
    if (e != cudaSuccess) return e;
    const int pitch = logit_pitch(A.cap, C);
    PdlConfig pc(dim3(A.n_streams * groups, C), kThreads, F::kSmem + (size_t)std::min(A.n_rows, kFewRows) * pitch * 4, st);
    cudaLaunchAttribute attrs[2] = {pc.attr, {}};
    attrs[1].id = cudaLaunchAttributeClusterDimension;
    attrs[1].val.clusterDim.x = attrs[1].val.clusterDim.z = 1;
    attrs[1].val.clusterDim.y = C;
    pc.cfg.attrs = attrs;
    pc.cfg.numAttrs = 2;
    return cudaLaunchKernelEx(&pc.cfg, kern, A, S, pitch, groups > 1 ? sums : nullptr, mk, mv);
  });
  if (e != cudaSuccess || groups == 1) return e;
  const int chunks = (A.cap + kEndThreads - 1) / kEndThreads;
  const PdlConfig pc(dim3((unsigned)chunks * A.n_streams), kEndThreads, 0, st);
  return cudaLaunchKernelEx(&pc.cfg, few_sum_kernel, A, S, (const float*)sums, groups, chunks);
}
template <bool kBf16, int D>
cudaError_t launch_end(const FewArgs& P, const ScoreArgs& S, cudaStream_t st) {
  const int joins = P.A.n_slots > 1 ? join_ctas(P.A) : 0;
  const int chunks = (P.A.cap + kEndKeys - 1) / kEndKeys;
  const PdlConfig pc(dim3((unsigned)(joins + chunks * P.A.n_streams)), kEndThreads, 0, st);
  return cudaLaunchKernelEx(&pc.cfg, few_end_kernel<kBf16, D>, P, S, joins, chunks);
}

}  // namespace

// Split factor of the kernels above: as many CTAs as fit the SMs at once, with a tile for each warp; and of long caches, in parts of 1024
// rows, up to six times as many, so that streams of different lengths even out (256 streams of up to 8192 rows: 96.6 us by 5 splits, 93.8 by 7).
int few_splits(int64_t streams, int cap, int n_rows, int d, int is_bf16) {
  const int64_t sets = streams * ((n_rows + group_rows(is_bf16, d) - 1) / group_rows(is_bf16, d));
  const int share = few_warps(is_bf16, d) * kTile;
  const int64_t fill = std::min<int64_t>(2 * kAttnSms / sets, (cap + share - 1) / share);
  const int64_t even = std::min<int64_t>((12 * kAttnSms + sets - 1) / sets, cap / 1024);
  return (int)std::max<int64_t>(1, std::min<int64_t>(std::max(fill, even), kAttnMaxSplits));
}

// CTAs of a stream's cluster, 0 where clusters do not serve the call: as many as leave a tile for every warp.  What they save is the second
// launch and the workspace, 4.4 us of the host's time (8 x 1024 rows: 11.1 us a call against 15.5; in a graph 7.1 against 7.3), and what they
// cost are their meetings, so that they serve small calls: the logits fit shared memory, a CTA reads 256 KB at most (4 x 5000 fp32 rows of 128
// dims, 640 KB each: 26.7 us against 20.7), and all clusters run at once, since they start and end as a whole (256 streams of up to 8192
// rows in clusters of 16: 228 us against 108; 32 x 1024 rows by clusters of 8 12.4 us, of 4 8.7).
int few_cluster(int64_t streams, int cap, int n_rows, int d, int is_bf16) {
  const int64_t sets = streams * ((n_rows + kFewRows - 1) / kFewRows);
  const bool alone = !is_bf16 && d == 128;
  static_assert(Few<false, 128>::kCtas == 1 && Few<false, 64>::kCtas == 2 && Few<true, 128>::kCtas == 2 && Few<true, 64>::kCtas == 2, "CTAs of a cluster that share an SM");
  int C = 1;
  while (C < kMaxCluster && 2 * sets * C <= most_clustered(2 * C, alone) && cap > C * kWarps * kTile) C *= 2;
  const int64_t rows = logit_pitch(cap, C);
  return sets * C <= most_clustered(C, alone) && std::min(n_rows, kFewRows) * rows * 4 <= logit_bytes(is_bf16, d) && rows * 2 * d * (is_bf16 ? 2 : 4) <= 256 << 10 ? C : 0;
}
// Floats of the workspace that they need.
int64_t few_cluster_sums(const AttnRows& A) { return A.n_rows > kFewRows ? (int64_t)(A.n_rows + kFewRows - 1) / kFewRows * A.n_streams * A.cap : 0; }

int64_t few_pitch(int cap) { return ((int64_t)cap + 31) / 32 * 32; }

// x: [n_streams, n_rows, few_pitch(cap)] where launch_few_end is to follow, else null.  `also`: a second set of streams of the same call.
cudaError_t launch_attn_few(const AttnRows& A, float* x, const AttnRows* also, FewOrder order, int d, int is_bf16, cudaStream_t st) {
  const FewArgs P{A, x, few_pitch(A.cap)}, Q{also ? *also : A, nullptr, 0}, *second = also ? &Q : nullptr;
  if (is_bf16) return d == 128 ? launch_few<true, 128>(P, second, order, st) : launch_few<true, 64>(P, second, order, st);
  return d == 128 ? launch_few<false, 128>(P, second, order, st) : launch_few<false, 64>(P, second, order, st);
}

// Outputs and scores by clusters of C CTAs.
cudaError_t launch_attn_few_cluster(const AttnRows& A, const ScoreArgs& S, int C, float* sums, int d, int is_bf16, cudaStream_t st) {
  if (is_bf16) return d == 128 ? launch_cluster<true, 128>(A, S, C, sums, st) : launch_cluster<true, 64>(A, S, C, sums, st);
  return d == 128 ? launch_cluster<false, 128>(A, S, C, sums, st) : launch_cluster<false, 64>(A, S, C, sums, st);
}

// The scores, and the outputs where there are several splits.
cudaError_t launch_few_end(const AttnRows& A, float* x, const ScoreArgs& S, int d, int is_bf16, cudaStream_t st) {
  const FewArgs P{A, x, few_pitch(A.cap)};
  if (is_bf16) return d == 128 ? launch_end<true, 128>(P, S, st) : launch_end<true, 64>(P, S, st);
  return d == 128 ? launch_end<false, 128>(P, S, st) : launch_end<false, 64>(P, S, st);
}

}  // namespace bkv
