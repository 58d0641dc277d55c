// Attention of many query rows over a caller-held cache in bf16 on the 5th-generation tensor cores.
//
//   x_{r,i} = <q_r, k_i> log2(e) / sqrt d + log2 w_i,   out_r = sum_i 2^(x_{r,i} - m_r) v_i / sum_i 2^(x_{r,i} - m_r)
//
// A CTA takes two tiles of up to 128 query rows of a stream and walks its share of the keys in tiles of 128.  Per tile of logits:
// S = Q K^T (tcgen05.mma, both operands in shared memory) into TMEM; a warpgroup, a thread per query row, turns S into weights and
// writes them over S as bf16; O += P V (P from TMEM), half of the keys as soon as their weights are there.  The two tiles take turns, so
// that the tensor core multiplies for one while the other's weights are formed: per pair of tiles the products take 2048 cycles
// (d = 128), and so would 32768 exponentials of the special-function unit; a share of them is therefore formed by FMAs.
// A stream with one tile of query rows has it twice, and the two take the even and the odd tiles of keys and add their sums up (by_keys).
// The maximum m_r is the one seen when it last grew by more than 8: weights then stay below 2^8, and O is brought to a new maximum
// only that often (usually in the first tiles).  Sums and maxima are fp32; the weights are rounded to bf16 for the second product, whose operands are
// of one type, their sum is not: 2^-8 of sum p |v| at most, 0.0022 of an output's norm in all against 0.0017 of the result's rounding alone.  (A low
// part, as the one-pass kernels have it, would be half as many products again.)
//
// What bounds it is a tile's chain: the products of S (590 cycles to issue), their way to the rows' warps (200), logits and maximum (400),
// weights (1100) and the product with V (490) follow one another, and TMEM has room for two chains only.
// Measured and dropped: two warpgroups per tile, half of the keys each (prompt of 8192: 521 us against 466; the weights of one tile
// were formed while the other's waited).
//
// Warps: 0-3 and 4-7 the rows of the two tiles, 8 asks for Q, K and V tiles (TMA, 128-byte swizzle, a ring), 9 issues the MMAs.
// Rows of V (weighted: of K too) that no query may see -- behind the last row in use, of weight zero -- are cleared in shared memory
// by warp 9 before it multiplies with them, since zero times what they hold need not be zero.
// Every wait is bounded; one that gives up makes the results NaN.
#include <algorithm>
#include <type_traits>

#include "attn_tc.cuh"

namespace bkv {

namespace {

using namespace tc;
using namespace mma;

constexpr int kThreads = 384;
// Registers of a thread at launch, and what the warps go on with: 8 x 208 + 4 x 80 <= 12 x 168.
constexpr int kRegs = 168, kRegsRows = 208, kRegsOther = 80;
static_assert(8 * kRegsRows + 4 * kRegsOther <= 12 * kRegs && kThreads * kRegs <= 65536, "a register split beyond the launch's waits forever");
constexpr float kGrow = 8.f;                     // the maximum follows when it would grow by more

template <int D, bool kWeighted>
struct Shape {
  static constexpr uint32_t kBox = 128 * 128;                          // bytes: 64 dims x 128 rows
  static constexpr uint32_t kTile = (D / 64) * kBox;
  static constexpr int kRing = D == 64 ? 8 : kWeighted ? 4 : 5;        // K and V tiles, in the order of their use
  // Tiles of log weights.  One takes the place of the eighth before it, whose readers are done: a K tile is asked for when the entry kRing
  // before it in the ring has been multiplied, at most four K tiles back, and a tile is multiplied only when its predecessor's weights are formed.
  static constexpr int kBias = 8;
  static constexpr size_t kSmem = 1024 + (2 + kRing) * (size_t)kTile;
};

struct TcArgs {
  AttnRows A;
  int32_t rows_per_tile;       // query rows of a tile: 128, or the largest multiple of the group that fits
  int32_t q_outer_rows;        // rows of the query box's outer dimension per tile (0: the query rows are contiguous)
  int32_t blocks;              // of two tiles of query rows (by_keys: of one), per stream
  int32_t by_keys;             // the tiles have the same query rows, and every other tile of keys each
};

// kWeighted: every query sees every row in use, with weights.
template <int D, bool kWeighted>
__global__ void __maxnreg__(kRegs)
attn_tc_kernel(const __grid_constant__ TcArgs P, const __grid_constant__ CUtensorMap mq, const __grid_constant__ CUtensorMap mk, const __grid_constant__ CUtensorMap mv) {
  using Sh = Shape<D, kWeighted>;
  constexpr int kRing = Sh::kRing;
  extern __shared__ unsigned char smem_raw[];
  __shared__ uint64_t q_full, kv_full[kRing], kv_empty[kRing], s_full[2], p_full[2][2], o_done[2], bias_full[Sh::kBias], drained;
  __shared__ uint32_t tmem_s;
  __shared__ int abort_flag;
  __shared__ __align__(16) float bias[kWeighted ? Sh::kBias : 1][kWeighted ? kTcKeys : 4];
  const AttnRows& A = P.A;
  unsigned char* sm = smem_raw + (-smem_u32(smem_raw) & 1023u);
  unsigned char* ring = sm + 2 * Sh::kTile;
  const int tid = threadIdx.x, warp = __shfl_sync(0xffffffffu, tid / 32, 0), lane = tid % 32;
  if (tid == 0) {
    mbar_init(&q_full, 1);
    mbar_init(&drained, 1);
    for (int i = 0; i < kRing; ++i) { mbar_init(kv_full + i, 1); mbar_init(kv_empty + i, 1); }
    for (int t = 0; t < 2; ++t) {
      mbar_init(s_full + t, 1);
      mbar_init(o_done + t, 1);
      mbar_init(&p_full[t][0], 128);
      mbar_init(&p_full[t][1], 128);
    }
    for (int i = 0; i < Sh::kBias; ++i) mbar_init(bias_full + i, 32);
    abort_flag = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
  }
  if (warp == 9) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&tmem_s)), "r"(512u) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  grid_wait_and_release();
  // the last query rows, which see the most, first
  const int s = blockIdx.x % A.n_streams, block = P.blocks - 1 - blockIdx.x / A.n_streams, split = blockIdx.y;
  const int len = attn_len(A, s);
  const bool by_keys = P.by_keys != 0;
  const int row0 = (by_keys ? block : 2 * block) * P.rows_per_tile, row1 = by_keys ? row0 : row0 + P.rows_per_tile;      // of the tiles
  // Tiles of keys that some row of a tile sees, and the first of them that not every row sees whole.
  auto seen = [&](int r0) {
    const int r1 = min(r0 + P.rows_per_tile, A.n_rows) - 1;
    return r0 >= A.n_rows ? 0 : ((r0 / A.n_queries != r1 / A.n_queries ? len : attn_limit(A, len, r1)) + kTcKeys - 1) / kTcKeys;
  };
  auto whole = [&](int r0) {
    const int r1 = min(r0 + P.rows_per_tile, A.n_rows) - 1;
    return attn_limit(A, len, r0 / A.n_queries != r1 / A.n_queries ? 0 : r0) / kTcKeys;
  };
  const int seen0 = seen(row0), seen1 = seen(row1), all = max(seen0, seen1);
  const int j0 = (int)((int64_t)all * split / A.splits), j1 = (int)((int64_t)all * (split + 1) / A.splits);
  // Tile t of the query rows takes the tiles of keys j0 + step j + off t, j < n_t.
  const int step = by_keys ? 2 : 1, off = by_keys ? 1 : 0;
  const int n0 = by_keys ? (j1 - j0 + 1) / 2 : max(0, min(seen0, j1) - j0), n1 = by_keys ? (j1 - j0) / 2 : max(0, min(seen1, j1) - j0), n = max(n0, n1);
  // Entries of the ring are loaded and used in this order: for j = -1, 0, ..: for t = 0, 1: V of (t, j), K of (t, j + 1) -- once for both t
  // where they share it, when the first of them needs it.
  auto uses = [&](int t, int j) { return j < (t ? n1 : n0); };
  auto loads = [&](int t, int j) { return uses(t, j) && (by_keys || t == 0 || !uses(0, j)); };
  auto frees = [&](int t, int j) { return by_keys || t == 1 || !uses(1, j); };
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = __shfl_sync(0xffffffffu, tmem_s, 0);

  if (warp >= 8) {
    regs_down<kRegsOther>();
    if (warp == 8 && n > 0) {
      bool ok = true;
      if (lane == 0) {
        mbar_expect_tx(&q_full, ((uint32_t)(n0 > 0) + (uint32_t)(n1 > 0)) * P.rows_per_tile * 2 * D);
        for (int t = 0; t < 2; ++t) {
          if (!uses(t, 0)) continue;
          const int r0 = t ? row1 : row0;
          for (int b = 0; b < D / 64; ++b) {
            if (P.q_outer_rows) tma_load_3d(sm + t * Sh::kTile + b * Sh::kBox, &mq, 64 * b, s * A.q_stream, r0 / A.q_inner, &q_full);
            else tma_load_3d(sm + t * Sh::kTile + b * Sh::kBox, &mq, 64 * b, s * A.q_stream + r0, 0, &q_full);
          }
        }
      }
      int e = 0, slot = 0, n_bias = 0;
      uint32_t lap = 0;
      auto load = [&](const CUtensorMap* map, int tile) {
        if (lap > 0) ok = ok && __all_sync(0xffffffffu, wait_bar(kv_empty + slot, (lap - 1) & 1u, &abort_flag));
        if (!ok) return;
        if (lane == 0) {
          mbar_expect_tx(kv_full + slot, Sh::kTile);
          for (int b = 0; b < D / 64; ++b) tma_load_3d(ring + slot * Sh::kTile + b * Sh::kBox, map, 64 * b, tile * kTcKeys, s, kv_full + slot);
        }
        __syncwarp();
        ++e;
        if (++slot == kRing) { slot = 0; ++lap; }
      };
      // Log weights, read a K tile ahead: waiting for them between two loads kept the ring from filling (a prefix of 32768 rows: 59 us).
      float ahead[kTcKeys / 32];
      auto read_ahead = [&](int tile) {
#pragma unroll
        for (int i = 0; i < kTcKeys / 32; ++i) {
          const int key = tile * kTcKeys + lane + 32 * i;
          ahead[i] = key < len ? (A.w ? A.w[(int64_t)s * A.cap + key] : 1.f) : 0.f;
        }
      };
      if (kWeighted) read_ahead(j0);
      for (int j = -1; j < n && ok; ++j)
        for (int t = 0; t < 2 && ok; ++t) {
          if (j >= 0 && loads(t, j)) load(&mv, j0 + step * j + off * t);
          if (!ok || !loads(t, j + 1)) continue;
          load(&mk, j0 + step * (j + 1) + off * t);
          if (kWeighted && ok) {
#pragma unroll
            for (int i = 0; i < kTcKeys / 32; ++i) bias[n_bias % Sh::kBias][lane + 32 * i] = log2f(ahead[i]);
            mbar_arrive(bias_full + n_bias % Sh::kBias);
            ++n_bias;
            read_ahead(j0 + n_bias);             // (K tiles are loaded in their order)
          }
        }
      if (lane == 0) {
        copy_landed(&q_full);
        copies_landed(kv_full, e);
      }
    } else if (warp == 9 && n > 0) {
      constexpr uint32_t kInstrPv = kInstrBf16<D> | kOuterB;
      bool ok = true;
      auto wait = [&](uint64_t* bar, uint32_t parity) { ok = ok && __all_sync(0xffffffffu, wait_bar(bar, parity, &abort_flag)); };
      int slot = 0, n_k = 0;                     // the next entry, K tiles so far
      uint32_t lap = 0;
      // The next entry, the tile of keys `tile` of K or V; b: its K tile's number.  Rows that nobody may see become zeros.
      auto take = [&](bool value, int tile, int b) {
        const int at = slot;
        wait(kv_full + at, lap & 1u);
        if (++slot == kRing) { slot = 0; ++lap; }
        const int key0 = tile * kTcKeys;
        bool any = value && key0 + kTcKeys > len;
        if constexpr (kWeighted) {
          wait(bias_full + b % Sh::kBias, (uint32_t)(b / Sh::kBias) & 1u);
          const float4 w = *reinterpret_cast<const float4*>(bias[b % Sh::kBias] + 4 * lane);
          any = __any_sync(0xffffffffu, w.x == -INFINITY || w.y == -INFINITY || w.z == -INFINITY || w.w == -INFINITY);
        }
        if (any && ok) {
          unsigned char* rows = ring + at * Sh::kTile;
          for (int r = 0; r < kTcKeys; ++r) {
            bool gone = key0 + r >= len;
            if constexpr (kWeighted) gone = bias[b % Sh::kBias][r] == -INFINITY;
            if (gone && lane < D / 8) *reinterpret_cast<uint4*>(rows + (lane / 8) * Sh::kBox + r * 128 + (lane % 8) * 16) = make_uint4(0, 0, 0, 0);
          }
          asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
          __syncwarp();
        }
        return at;
      };
      int k_at = 0, v_at = 0;                    // entries in use
      wait(&q_full, 0);
      for (int j = -1; j < n && ok; ++j) {
#pragma unroll
        for (int t = 0; t < 2; ++t) {
          if (!ok) break;
          if (j >= 0 && uses(t, j)) {
            if (loads(t, j)) v_at = take(true, j0 + step * j + off * t, by_keys ? 2 * j + t : j);
#pragma unroll
            for (int h = 0; h < 2; ++h) {
              wait(&p_full[t][h], (uint32_t)j & 1u);
              tc_fence_after();
              if (ok && elect_one()) {
                const uint32_t v = umma_desc_lo_outer(smem_u32(ring + v_at * Sh::kTile), Sh::kBox);
#pragma unroll
                for (int k = 4 * h; k < 4 * h + 4; ++k)
                  umma_ts<kInstrPv>(tmem + 256 + D * t, tmem + 128 * t + 8 * k, v + 128 * k, j > 0 || k > 0);
                if (h == 1) {
                  umma_commit(o_done + t);
                  if (frees(t, j)) umma_commit(kv_empty + v_at);
                }
              }
              __syncwarp();
            }
          }
          if (ok && uses(t, j + 1)) {
            if (loads(t, j + 1)) k_at = take(false, j0 + step * (j + 1) + off * t, n_k++);
            tc_fence_after();
            if (ok && elect_one()) {
              const uint32_t a = umma_desc_lo(smem_u32(sm + t * Sh::kTile)), b = umma_desc_lo(smem_u32(ring + k_at * Sh::kTile));
#pragma unroll
              for (int k = 0; k < D / 16; ++k) {
                const uint32_t at = (uint32_t)(k / 4) * (Sh::kBox >> 4) + 2 * (k % 4);
                if (k == 0) umma_bf16<0>(tmem + 128 * t, a + at, b + at);
                else umma_bf16<1>(tmem + 128 * t, a + at, b + at);
              }
              umma_commit(s_full + t);
              if (frees(t, j + 1)) umma_commit(kv_empty + k_at);
            }
            __syncwarp();
          }
        }
      }
      if (!ok) st_release(&abort_flag, 1);
      products_done(&drained);
    }
  } else {
    regs_up<kRegsRows>();
    const int t = warp / 4, in_tile = 32 * (warp % 4) + lane;
    const int r = (t ? row1 : row0) + in_tile;
    const bool valid = in_tile < P.rows_per_tile && r < A.n_rows;
    const int limit = valid ? attn_limit(A, len, r) : 0;
    const uint32_t lanes = (uint32_t)(32 * (warp % 4)) << 16;
    const uint32_t S = tmem + lanes + 128 * t, O = tmem + lanes + 256 + D * t;
    const int mine = t ? n1 : n0, first_masked = whole(t ? row1 : row0);
    const float2 scale2 = make_float2(A.scale, A.scale);
    float m = -INFINITY;
    float2 l2[4] = {};                           // the sum of weights, in eight parts
    bool ok = true;
    for (int j = 0; j < mine; ++j) {
      const int b = by_keys ? 2 * j + t : j, tile = j0 + step * j + off * t;
      ok = wait_bar(s_full + t, (uint32_t)j & 1u, &abort_flag);
      if (kWeighted) ok = ok && wait_bar(bias_full + b % Sh::kBias, (uint32_t)(b / Sh::kBias) & 1u, &abort_flag);
      ok = __all_sync(0xffffffffu, ok);
      if (!ok) break;
      tc_fence_after();
      float x[4][32];
#pragma unroll
      for (int c = 0; c < 4; ++c) tmem_ld32(S + 32 * c, x[c]);
      tmem_ld_wait();
      const bool masked = !kWeighted && tile >= first_masked;
      if constexpr (kWeighted) {
        const float4* b4 = reinterpret_cast<const float4*>(bias[b % Sh::kBias]);
#pragma unroll
        for (int c = 0; c < 4; ++c)
#pragma unroll
          for (int i = 0; i < 32; i += 4) {
            const float4 w = b4[(32 * c + i) / 4];
            const float2 lo = __ffma2_rn(make_float2(x[c][i], x[c][i + 1]), scale2, make_float2(w.x, w.y));
            const float2 hi = __ffma2_rn(make_float2(x[c][i + 2], x[c][i + 3]), scale2, make_float2(w.z, w.w));
            x[c][i] = lo.x; x[c][i + 1] = lo.y; x[c][i + 2] = hi.x; x[c][i + 3] = hi.y;
          }
      }
      if (masked) {
        const int sees = limit - tile * kTcKeys;
#pragma unroll
        for (int c = 0; c < 4; ++c)
#pragma unroll
          for (int i = 0; i < 32; ++i) x[c][i] = 32 * c + i < sees ? x[c][i] : -INFINITY;
      }
      float mx = fmaxf(fmaxf(max_of(x[0]), max_of(x[1])), fmaxf(max_of(x[2]), max_of(x[3])));
      if (!kWeighted) mx *= A.scale;
      const bool grow = mx > m + kGrow;
      if (__any_sync(0xffffffffu, grow)) {
        const float f = grow ? ex2(m - mx) : 1.f;
        if (grow) m = mx;
#pragma unroll
        for (int i = 0; i < 4; ++i) l2[i] = __fmul2_rn(l2[i], make_float2(f, f));
        if (j > 0) {                             // O at the new maximum, once the products before are in it
          ok = __all_sync(0xffffffffu, wait_bar(o_done + t, (uint32_t)(j - 1) & 1u, &abort_flag));
          if (!ok) break;
          tc_fence_after();
#pragma unroll 1
          for (int c = 0; c < D; c += 16) {
            float o[16];
            tmem_ld16(O + c, o);
            tmem_ld_wait();
            uint32_t w[16];
#pragma unroll
            for (int i = 0; i < 16; ++i) w[i] = __float_as_uint(o[i] * f);
            tmem_st16(O + c, w);
          }
        }
      }
      const float base = m == -INFINITY ? 0.f : -m;
      const float2 base2 = make_float2(base, base);
      const float2 one2 = kWeighted ? make_float2(1.f, 1.f) : scale2;
      auto weights = [&](auto all_mufu) {
#pragma unroll
        for (int c = 0; c < 4; ++c) {
          uint32_t w[16];
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            const float2 y = __ffma2_rn(make_float2(x[c][2 * i], x[c][2 * i + 1]), one2, base2);
            float2 p;
            if (!decltype(all_mufu)::value && i % 8 == 3) p = exp2_fma(y);      // an eighth of the pairs
            else p = make_float2(ex2(y.x), ex2(y.y));
            l2[i % 4] = __fadd2_rn(l2[i % 4], p);
            w[i] = pack_bf16(p.x, p.y);
          }
          tmem_st16(S + 16 * c, w);              // (the columns of S under them have been read)
          if (c & 1) {
            tmem_st_wait();
            tc_fence_before();
            mbar_arrive(&p_full[t][c / 2]);
          }
        }
      };
      if (masked) weights(std::true_type{});     // (what is masked has weight zero, which exp2_fma does not give)
      else weights(std::false_type{});
    }
    float l = ((l2[0].x + l2[0].y) + (l2[1].x + l2[1].y)) + ((l2[2].x + l2[2].y) + (l2[3].x + l2[3].y));
    if (mine > 0 && ok) {
      ok = __all_sync(0xffffffffu, wait_bar(o_done + t, (uint32_t)(mine - 1) & 1u, &abort_flag));
      tc_fence_after();
    }
    if (!ok) {
      l = NAN;
      copy_landed(&q_full);                      // (what follows takes the Q tiles' place)
    }
    // The results leave by way of shared memory, 32 columns of a warp's rows at a time, so that neighbouring lanes write neighbouring bytes
    // (a row per lane, 16 bytes at a time, took 8200 cycles for two tiles of sums).  Its Q tile is there for it: every S is formed.
    uint4* const stage = reinterpret_cast<uint4*>(sm + t * Sh::kTile) + (warp % 4) * (Sh::kTile / 64);
    const bool parts = A.n_slots > 1;
    const int row = valid ? (int)attn_row(A, s, r) : -1;
    float top = m, sum = l, f = 1.f;             // f: of this thread's O
    auto pair_sync = [&]() { asm volatile("bar.sync %0, 64;" ::"r"(1 + warp % 4) : "memory"); };      // the warps of the same query rows
    const uint4* const theirs = reinterpret_cast<const uint4*>(sm + (1 - t) * Sh::kTile) + (warp % 4) * (Sh::kTile / 64);
    if (by_keys) {                               // two sums of the same rows become one
      reinterpret_cast<float2*>(stage)[lane] = make_float2(m, l);
      pair_sync();
      const float2 other = reinterpret_cast<const float2*>(theirs)[lane];
      pair_sync();
      top = fmaxf(m, other.x);
      const float at = top == -INFINITY ? 0.f : top;
      f = ex2(m - at);
      // (added in the same order by both)
      const float mine_l = l * f, other_l = other.y * ex2(other.x - at);
      sum = t ? other_l + mine_l : mine_l + other_l;
    }
    if (valid && !(by_keys && t)) {
      if (parts) A.part_ml[(int64_t)(A.slot0 + split) * A.total_rows + row] = make_float2(top, sum);
      else if (A.lse) A.lse[row] = sum == 0.f ? INFINITY : top + log2f(sum);
    }
    if (!parts) f = sum == 0.f ? 0.f : f / sum;
    const bool any = mine > 0;
    auto take = [&](int c, float (&o)[32]) {
      if (any) {
        tmem_ld32(O + c, o);
        tmem_ld_wait();
      }
#pragma unroll
      for (int i = 0; i < 32; ++i) o[i] = any && l != 0.f ? o[i] * f : 0.f;
    };
    auto put = [&](int c, const float (&o)[32]) {
      __syncwarp();
      if (parts) {
#pragma unroll
        for (int i = 0; i < 8; ++i)
          stage[8 * lane + (i ^ (lane & 7))] = make_uint4(__float_as_uint(o[4 * i]), __float_as_uint(o[4 * i + 1]), __float_as_uint(o[4 * i + 2]), __float_as_uint(o[4 * i + 3]));
        __syncwarp();
        const int piece = lane % 8;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const int from = 4 * i + lane / 8, to = __shfl_sync(0xffffffffu, row, from);
          if (to >= 0) *reinterpret_cast<uint4*>(A.part + ((int64_t)(A.slot0 + split) * A.total_rows + to) * D + c + 4 * piece) = stage[8 * from + (piece ^ (from & 7))];
        }
      } else {
#pragma unroll
        for (int i = 0; i < 4; ++i)
          stage[4 * lane + (i ^ (lane >> 1 & 3))] =
              make_uint4(pack_bf16(o[8 * i], o[8 * i + 1]), pack_bf16(o[8 * i + 2], o[8 * i + 3]), pack_bf16(o[8 * i + 4], o[8 * i + 5]), pack_bf16(o[8 * i + 6], o[8 * i + 7]));
        __syncwarp();
        const int piece = lane % 4;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int from = 8 * i + lane / 4, to = __shfl_sync(0xffffffffu, row, from);
          if (to >= 0) *reinterpret_cast<uint4*>(static_cast<__nv_bfloat16*>(A.out) + (int64_t)to * D + c + 8 * piece) = stage[4 * from + (piece ^ (from >> 1 & 3))];
        }
      }
    };
    if (by_keys) {                               // a half of the columns each: the other half's sums to the other warp
      constexpr int kHalf = D / 2;
#pragma unroll
      for (int c = 0; c < kHalf; c += 32) {
        float o[32];
        take(kHalf * (1 - t) + c, o);
#pragma unroll
        for (int i = 0; i < 32; ++i) reinterpret_cast<float*>(stage)[32 * (c + i) + lane] = o[i];
      }
      float o[kHalf / 32][32];
#pragma unroll
      for (int c = 0; c < kHalf; c += 32) take(kHalf * t + c, o[c / 32]);
      pair_sync();
#pragma unroll
      for (int c = 0; c < kHalf; ++c) o[c / 32][c % 32] += reinterpret_cast<const float*>(theirs)[32 * c + lane];
      pair_sync();
#pragma unroll
      for (int c = 0; c < kHalf; c += 32) put(kHalf * t + c, o[c / 32]);
    } else {
#pragma unroll 1
      for (int c = 0; c < D; c += 32) {
        float o[32];
        take(c, o);
        put(c, o);
      }
    }
    tc_fence_before();
  }
  __syncthreads();
  tc_fence_after();
  if (warp == 9) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512u) : "memory");
}

// Query rows of a stream: contiguous (box 64 dims x 128 rows), or `inner` of each of an outer dimension's.
cudaError_t query_map(CUtensorMap* map, const AttnRows& A, int d, int outer_rows) {
  EncodeTiledFn encode = nullptr;
  const cudaError_t e = tensor_map_encoder(&encode);
  if (e != cudaSuccess) return e;
  const cuuint64_t inner = outer_rows ? (cuuint64_t)A.q_outer : (cuuint64_t)A.total_rows;
  const cuuint64_t dims[3] = {(cuuint64_t)d, inner, (cuuint64_t)A.total_rows / inner};
  const cuuint64_t strides[2] = {(cuuint64_t)d * 2, (cuuint64_t)d * 2 * inner};
  const cuuint32_t box[3] = {64, outer_rows ? (cuuint32_t)A.q_inner : 128u, outer_rows ? (cuuint32_t)outer_rows : 1u};
  const cuuint32_t estr[3] = {1, 1, 1};
  const CUresult r = encode(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, const_cast<void*>(A.q), dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
                            CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
  return r == CUDA_SUCCESS ? cudaSuccess : cudaErrorInvalidValue;
}

template <int D, bool kWeighted>
cudaError_t launch(const TcArgs& P, cudaStream_t st) {
  const AttnRows& A = P.A;
  CUtensorMap mq, mk, mv;
  cudaError_t e = query_map(&mq, A, D, P.q_outer_rows);
  if (e == cudaSuccess) e = cache_map(&mk, A.K, true, D, A.cap, A.n_streams, kTcKeys);
  if (e == cudaSuccess) e = cache_map(&mv, A.V, true, D, A.cap, A.n_streams, kTcKeys);
  static std::atomic<unsigned long long> devices{0};
  if (e == cudaSuccess) e = kernel_limits(attn_tc_kernel<D, kWeighted>, Shape<D, kWeighted>::kSmem, devices);
  if (e != cudaSuccess) return e;
  const PdlConfig pc(dim3((unsigned)P.blocks * A.n_streams, A.splits), kThreads, Shape<D, kWeighted>::kSmem, st);
  return cudaLaunchKernelEx(&pc.cfg, attn_tc_kernel<D, kWeighted>, P, mq, mk, mv);
}

// Rows of a tile: with an outer dimension whole groups of it.
int rows_per_tile(const AttnRows& A) { return A.q_outer ? 128 / A.q_inner * A.q_inner : 128; }
bool by_keys(const AttnRows& A) { return A.n_rows <= rows_per_tile(A); }
int blocks_of(const AttnRows& A) { return by_keys(A) ? 1 : (A.n_rows + 2 * rows_per_tile(A) - 1) / (2 * rows_per_tile(A)); }

}  // namespace

int attn_tc_blocks(const AttnRows& A) { return blocks_of(A) * A.n_streams; }
bool attn_tc_by_keys(const AttnRows& A) { return by_keys(A); }

// CTAs that share the keys of a block of query rows, each an SM: the factor of the shortest time, in tiles of keys: those of a wave's CTA
// and three for its start and end, and those that writing and joining the splits takes (fp32 rows there and back; a pair of query tiles and
// four splits about one); two tiles of keys each at least.  Where the blocks alone fill the SMs, splits have to save a quarter by that count: an
// idle SM leaves the others its power, and joining costs (8 x 1024 queries x 5 heads behind 32768 rows, 160 blocks: 880 us by one split, 683
// by eight; 40 x 512 x 4 behind 8192, 320 blocks: 368 against 425; 16 x 2048 x 3 behind 30000, 384 blocks: 1435 against 1521).  Blocks of a
// prompt differ in what they see, and even out by themselves.
int attn_tc_splits(const AttnRows& A) {
  const int64_t blocks = attn_tc_blocks(A), tiles = ((int64_t)A.cap + kTcKeys - 1) / kTcKeys;
  int best = 1;
  int64_t least = INT64_MAX;
  if (blocks >= kAttnSms && 2 * (int64_t)A.n_queries > A.cap) return 1;
  int64_t whole = 0;
  for (int splits = 1; splits <= kAttnMaxSplits && (splits == 1 || 2 * splits <= tiles); ++splits) {
    const int64_t time = 4 * ((blocks * splits + kAttnSms - 1) / kAttnSms * ((tiles + splits - 1) / splits + 3)) +
                         (splits > 1 ? 4 + (splits * blocks + kAttnSms - 1) / kAttnSms : 0);
    if (splits == 1) whole = time;
    if (time < least) { least = time; best = splits; }
  }
  return blocks >= kAttnSms && 4 * least > 3 * whole ? 1 : best;
}

cudaError_t launch_attn_tc(const AttnRows& A, int d, cudaStream_t st) {
  const TcArgs P{A, rows_per_tile(A), A.q_outer ? 128 / A.q_inner : 0, blocks_of(A), by_keys(A)};
  if (A.w) return d == 128 ? launch<128, true>(P, st) : launch<64, true>(P, st);
  return d == 128 ? launch<128, false>(P, st) : launch<64, false>(P, st);
}

}  // namespace bkv
