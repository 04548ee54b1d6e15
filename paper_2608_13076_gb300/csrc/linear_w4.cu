// linear_w4.cu -- y = x W^T (+ residual) with W in 4 bits: the verifier's linear
// layers (f_l in x_{l+1} = x_l + f_l(x_l), Sec. III-A) for the rows of a verify block
// or single tokens.
#include <cfloat>

#include "int4.cuh"
#include "internal.h"
#include "ptx.cuh"

namespace spade {
namespace w4 {

struct Params {
  const __nv_bfloat16 *x, *residual;
  const uint32_t *codes, *pairs;
  __nv_bfloat16 *out;
  int32_t *status;
  int R, N, K;
  int tile_rows, split;  // (more than eight rows) rows of a tile; CTAs that share a tile's units
};

// ---- up to eight rows: the weights streamed past mma.sync -----------------------------------
// y^T = W x^T on mma.sync (m16n8k16): 16 outputs on M, the rows of x on N.  Bound by the
// weights' bytes: 4 1/4 to 5 bits each, read once.  The order of K inside an MMA is free
// as long as both operands share it, so a thread's fragment of a group is simply its own
// contiguous part of the weight row (two bf16 pairs per MMA and row come out of one word
// with masks), and the same part of the row of x.  Codes minus zero are whole numbers,
// exact in bf16, and a group's products are summed apart and then scaled in fp32: nothing
// of W is rounded.
// The eight warps of a CTA take units of 128 k in turn, each with a ring of its own that
// its first lane fills (TMA, 64 bytes of each output's row; the copy's swizzle makes the
// fragments' reads free of bank conflicts for every group size), and add their sums in
// shared memory in a fixed order.  Fragments straight from global memory kept the L1 busy
// with 4-byte reads at group 32: 12288 x 4096 x 6 rows took 19.8 us.
constexpr int kThreads = 256;
constexpr int kWarps = kThreads / 32;
constexpr int kUnit = 128;   // k per unit
constexpr int kRing = 2;     // units in flight per warp
constexpr int kRows = 8;

SPADE_DEVICE void mma_bf16(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
      : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

// The words of thread t of a row's unit: W = G / 32 of each group, from the swizzled copy.
template <int W>
SPADE_DEVICE void read_words(const uint8_t *rows, int r, int t, uint32_t (&w)[4]) {
  const uint8_t *row = rows + r * 64;
  const int turn = (r >> 1) & 3;
  if constexpr (W == 4) {
    const uint4 v = *reinterpret_cast<const uint4 *>(row + ((t ^ turn) << 4));
    w[0] = v.x; w[1] = v.y; w[2] = v.z; w[3] = v.w;
  } else if constexpr (W == 2) {
#pragma unroll
    for (int q = 0; q < 2; ++q) {
      const uint2 v = *reinterpret_cast<const uint2 *>(row + (((2 * q + (t >> 1)) ^ turn) << 4) + (t & 1) * 8);
      w[2 * q] = v.x; w[2 * q + 1] = v.y;
    }
  } else {
#pragma unroll
    for (int q = 0; q < 4; ++q) w[q] = *reinterpret_cast<const uint32_t *>(row + ((q ^ turn) << 4) + t * 4);
  }
}

// The pairs of unit u's groups of one output (zeros past the last group).
template <int U>
SPADE_DEVICE void load_unit_pairs(const uint32_t *pairs, int u, int groups, bool whole, uint32_t (&p)[U]) {
  const uint32_t *at = pairs + static_cast<int64_t>(u) * U;
  if constexpr (U == 4) {
    if (whole) {
      const uint4 v = __ldg(reinterpret_cast<const uint4 *>(at));
      p[0] = v.x; p[1] = v.y; p[2] = v.z; p[3] = v.w;
      return;
    }
  } else if constexpr (U == 2) {
    if (whole) {
      const uint2 v = __ldg(reinterpret_cast<const uint2 *>(at));
      p[0] = v.x; p[1] = v.y;
      return;
    }
  }
#pragma unroll
  for (int q = 0; q < U; ++q) p[q] = u * U + q < groups ? __ldg(at + q) : 0u;
}

template <int G, int MT>
__global__ void __launch_bounds__(kThreads) few_rows_kernel(const __grid_constant__ Params p,
                                                            const __grid_constant__ CUtensorMap tm) {
  constexpr int W = G / 32, U = kUnit / G;  // words of a thread's part of a group; groups of a unit
  constexpr int kStage = MT * 16 * 64;
  extern __shared__ uint8_t smem_raw[];
  uint8_t *smem = smem_raw + ((1024u - (smem_u32(smem_raw) & 1023u)) & 1023u);
  __shared__ float s_sum[kWarps][MT * 16][kRows];
  __shared__ uint64_t s_full[kWarps][kRing];
  __shared__ int s_abort;
  const int warp = uniform_warp(), lane = threadIdx.x & 31;
  const int r = lane >> 2, t = lane & 3;
  const int groups = p.K / G, units = (groups + U - 1) / U;
  const int o0 = blockIdx.x * MT * 16;
  uint8_t *ring = smem + warp * kRing * kStage;
  uint64_t *full = s_full[warp];
  if (threadIdx.x == 0) {
    s_abort = 0;
    tma_prefetch_desc(&tm);
  }
  if (lane == 0) {
    for (int s = 0; s < kRing; ++s) mbar_init(&full[s], 1);
    fence_mbar_init();
  }
  __syncthreads();
  griddep_wait();
  griddep_launch_dependents();
  const int mine = warp < units ? (units - warp + kWarps - 1) / kWarps : 0;  // units of this warp
  auto fill = [&](int i) {
    uint64_t *bar = &full[i % kRing];
    mbar_arrive_expect_tx(bar, kStage);
    tma_load_2d(ring + (i % kRing) * kStage, &tm, (warp + i * kWarps) * (kUnit / 2), o0, bar, l2_policy_evict_first());
  };
  if (lane == 0)
    for (int i = 0; i < min(kRing, mine); ++i) fill(i);
  // Outputs past the end repeat the last one's pairs; what they give is not stored.
  const uint32_t *pair[MT][2];
#pragma unroll
  for (int m = 0; m < MT; ++m)
#pragma unroll
    for (int h = 0; h < 2; ++h) pair[m][h] = p.pairs + static_cast<int64_t>(min(o0 + m * 16 + h * 8 + r, p.N - 1)) * groups;
  const bool whole = groups % U == 0;
  const uint4 *x = reinterpret_cast<const uint4 *>(p.x + static_cast<int64_t>(min(r, p.R - 1)) * p.K) + W * t;
  // Pairs and x of a unit, loaded while the one before it is worked on.
  struct Rest {
    uint32_t pr[MT][2][U];
    uint4 xv[4];
  };
  Rest rest[2];
  auto load_rest = [&](int u, Rest &a) {
#pragma unroll
    for (int m = 0; m < MT; ++m)
#pragma unroll
      for (int h = 0; h < 2; ++h) load_unit_pairs<U>(pair[m][h], u, groups, whole, a.pr[m][h]);
#pragma unroll
    for (int q = 0; q < U; ++q)
#pragma unroll
      for (int e = 0; e < W; ++e)
        a.xv[q * W + e] = u * U + q < groups ? __ldg(x + (u * U + q) * (G / 8) + e) : make_uint4(0, 0, 0, 0);
  };
  if (mine) load_rest(warp, rest[0]);
  float acc[MT][4] = {};
  bool ok = true;
  int issued = min(kRing, mine);
  auto unit = [&](int i, const Rest &now, Rest &next) {
    if (i + 1 < mine) load_rest(warp + (i + 1) * kWarps, next);
    ok = __all_sync(0xffffffffu, mbar_wait_lean(&full[i % kRing], (i / kRing) & 1, &s_abort));
    if (!ok) return;
    uint32_t w[MT][2][4];
#pragma unroll
    for (int m = 0; m < MT; ++m)
#pragma unroll
      for (int h = 0; h < 2; ++h) read_words<W>(ring + (i % kRing) * kStage + m * 1024, h * 8 + r, t, w[m][h]);
    __syncwarp();
    if (i + kRing < mine) {
      if (lane == 0) fill(i + kRing);
      ++issued;
    }
#pragma unroll
    for (int q = 0; q < U; ++q) {
#pragma unroll
      for (int m = 0; m < MT; ++m) {
        const float2 lo = int4::pair_of(now.pr[m][0][q]), hi = int4::pair_of(now.pr[m][1][q]);
        const __nv_bfloat162 z0 = __float2bfloat162_rn(-128.f - lo.y), z1 = __float2bfloat162_rn(-128.f - hi.y);
        float c[4] = {};
#pragma unroll
        for (int e = 0; e < W; ++e) {
          uint32_t a[4], b[4];
          int4::unpack_bf16(w[m][0][q * W + e], z0, a);
          int4::unpack_bf16(w[m][1][q * W + e], z1, b);
          const uint4 v = now.xv[q * W + e];
          mma_bf16(c, a[0], b[0], a[1], b[1], v.x, v.y);
          mma_bf16(c, a[2], b[2], a[3], b[3], v.z, v.w);
        }
        acc[m][0] = fmaf(lo.x, c[0], acc[m][0]);
        acc[m][1] = fmaf(lo.x, c[1], acc[m][1]);
        acc[m][2] = fmaf(hi.x, c[2], acc[m][2]);
        acc[m][3] = fmaf(hi.x, c[3], acc[m][3]);
      }
    }
  };
  for (int i = 0; ok && i < mine; i += 2) {
    unit(i, rest[0], rest[1]);
    if (ok && i + 1 < mine) unit(i + 1, rest[1], rest[0]);
  }
  if (!ok && lane == 0) {
    atomicOr(p.status, SPADE_DEV_TIMEOUT);
    // Every copy issued must land before the CTA's shared memory goes away.
    for (int j = max(0, issued - kRing); j < issued; ++j) mbar_wait_unabortable(&full[j % kRing], (j / kRing) & 1);
  }
#pragma unroll
  for (int m = 0; m < MT; ++m)
#pragma unroll
    for (int e = 0; e < 4; ++e) s_sum[warp][m * 16 + (e >> 1) * 8 + r][2 * t + (e & 1)] = acc[m][e];
  __syncthreads();
  for (int e = threadIdx.x; e < MT * 16 * kRows; e += kThreads) {
    const int n = e / (MT * 16), o = e % (MT * 16);
    if (n >= p.R || o0 + o >= p.N) continue;
    float y = 0.f;
#pragma unroll
    for (int k = 0; k < kWarps; ++k) y += s_sum[k][o][n];
    const int64_t at = static_cast<int64_t>(n) * p.N + o0 + o;
    p.out[at] = __float2bfloat16_rn(y + (p.residual ? __bfloat162float(p.residual[at]) : 0.f));
  }
}

// ---- more rows: tcgen05 with the weights in tensor memory ----------------------------------
// y^T = W x^T again: 128 outputs on M, up to 64 rows of x on N, units of 128 k.  A thread
// unpacks one output's unit (64 bytes of codes) to whole numbers in bf16 and stores them
// to its lane of tensor memory, from where the MMA takes A (no shared-memory traffic for
// W beyond its codes, and no loss of MMA rate at small N); x comes by TMA as B.  Each
// group of k is accumulated apart, exact but for the fp32 sums, in one of two blocks of
// columns, and four warps drain the other under the outputs' scales into registers.
// Bound by the weights' bytes up to ~50 rows, by the unpacking's and draining's
// instructions and the MMAs (which share a unit about evenly at 64 rows) beyond.
// Two CTAs share an SM, so one's waits are the other's work.  Where the tiles do not fill
// the GPU, a cluster of 2, 4 or 8 CTAs takes a tile's units in equal parts and adds the
// sums through distributed shared memory in a fixed order.
namespace tc {

constexpr int kOut = 128;                       // outputs of a tile
constexpr int kStages = 4;                      // copy ring (units)
constexpr int kThreads = 320;                   // copies, MMA, four draining and four unpacking warps
constexpr int kWarpDrain = 2, kWarpUnpack = 6;
constexpr int kCodes = kOut * 64;               // a unit's codes: 8 KB
constexpr uint32_t kTmemCols = 256;             // sums: two blocks of 64 columns; weights: two of 64
constexpr uint32_t kColD = 0, kColA = 128;
constexpr int kMaxSplit = 8;

template <int NR>
struct Smem {
  static constexpr int kX = NR * 256;           // a unit of x: two slabs of [NR][64 k]
  static constexpr int kStage = kCodes + kX;
  static constexpr int kSums = kOut * NR * 4;   // the split's sums reuse the ring
  static constexpr int RING = 0;
  static constexpr int BYTES = (kStages * kStage > kSums ? kStages * kStage : kSums) + 1024;
};

template <int G, int NR>
__global__ void __launch_bounds__(kThreads, 2) rows_kernel(const __grid_constant__ Params p,
                                                           const __grid_constant__ CUtensorMap tm_w,
                                                           const __grid_constant__ CUtensorMap tm_x) {
  constexpr int U = kUnit / G;
  using S = Smem<NR>;
  extern __shared__ uint8_t smem_raw[];
  uint8_t *smem = smem_raw + ((1024u - (smem_u32(smem_raw) & 1023u)) & 1023u);
  __shared__ uint64_t s_full[kStages], s_empty[kStages], s_afull[2], s_afree[2], s_dfull[2], s_dfree[2], s_drain;
  __shared__ int s_abort;
  __shared__ uint32_t s_tmem;
  const int warp = uniform_warp(), lane = threadIdx.x & 31;
  if (threadIdx.x == 0) {
    s_abort = 0;
    tma_prefetch_desc(&tm_w);
    tma_prefetch_desc(&tm_x);
    for (int s = 0; s < kStages; ++s) {
      mbar_init(&s_full[s], 1);
      mbar_init(&s_empty[s], 5);  // four unpacking warps and the MMAs
    }
    for (int s = 0; s < 2; ++s) {
      mbar_init(&s_afull[s], 4);
      mbar_init(&s_afree[s], 1);
      mbar_init(&s_dfull[s], 1);
      mbar_init(&s_dfree[s], 4);
    }
    mbar_init(&s_drain, 1);
    fence_mbar_init();
  }
  if (warp == 1) {
    tmem_alloc(&s_tmem, kTmemCols);
    tmem_relinquish();
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = s_tmem;
  const int groups = p.K / G, units = (groups + U - 1) / U;
  const int split = p.split, rank = split > 1 ? static_cast<int>(cluster_ctarank()) : 0;
  const int o0 = static_cast<int>(blockIdx.x / split) * kOut, n0 = blockIdx.y * p.tile_rows;
  const int u0 = static_cast<int>(static_cast<int64_t>(units) * rank / split);
  const int u1 = static_cast<int>(static_cast<int64_t>(units) * (rank + 1) / split);
  griddep_wait();
  griddep_launch_dependents();
  float acc[NR];  // (draining warps: one output's sums)
  bool ok = true;
  if (warp == 0) {
    // ---- copies ----
    const bool leader = elect_one();
    const uint64_t once = l2_policy_evict_first(), again = l2_policy_evict_last();
    uint32_t issued = 0;
    for (int u = u0; u < u1; ++u, ++issued) {
      const int st = issued % kStages;
      ok = __all_sync(0xffffffffu, mbar_wait_lean(&s_empty[st], ((issued / kStages) & 1) ^ 1, &s_abort));
      if (!ok) break;
      uint8_t *stage = smem + st * S::kStage;
      if (leader) {
        mbar_arrive_expect_tx(&s_full[st], S::kStage);
        tma_load_2d(stage, &tm_w, u * (kUnit / 2), o0, &s_full[st], once);
        tma_load_2d(stage + kCodes, &tm_x, u * kUnit, n0, &s_full[st], again);
        tma_load_2d(stage + kCodes + S::kX / 2, &tm_x, u * kUnit + 64, n0, &s_full[st], again);
      }
    }
    if (!ok && leader)  // every copy issued must land before the CTA's shared memory goes away
      for (uint32_t j = issued > kStages ? issued - kStages : 0; j < issued; ++j)
        mbar_wait_unabortable(&s_full[j % kStages], (j / kStages) & 1);
  } else if (warp == 1) {
    // ---- MMAs ----
    constexpr uint32_t idesc = idesc_bf16_f32(kOut, NR);
    const bool leader = elect_one();
    const uint32_t base = smem_u32(smem);
    uint32_t it = 0, gi = 0;
    auto wait = [&](uint64_t *bar, uint32_t parity) {
      ok = __all_sync(0xffffffffu, mbar_wait_lean(bar, parity, &s_abort)) && ok;
    };
    for (int u = u0; ok && u < u1; ++u, ++it) {
      const int st = it % kStages, as = it & 1;
      wait(&s_full[st], (it / kStages) & 1);
      wait(&s_afull[as], (it / 2) & 1);
      if (!ok) break;
      const uint64_t dx = smem_desc_sw128(base + st * S::kStage + kCodes);
      const int ng = min(U, groups - u * U);
#pragma unroll
      for (int q = 0; q < U; ++q) {
        if (q >= ng) break;
        const int db = gi & 1;
        wait(&s_dfree[db], ((gi / 2) & 1) ^ 1);
        tc_fence_after();
#pragma unroll
        for (int k = 0; k < G / 16; ++k) {
          constexpr int kSlabSteps = 4;  // MMAs per 64-k slab
          const int kk = q * (G / 16) + k;
          const uint32_t off = ((kk / kSlabSteps) * (S::kX / 2) + (kk % kSlabSteps) * 32) >> 4;
          if (leader) tc_mma_f16_ta(tmem + kColD + db * 64, tmem + kColA + as * 64 + kk * 8, dx + off, idesc, k > 0);
        }
        if (leader) tc_commit(&s_dfull[db]);
        ++gi;
      }
      if (leader) {
        tc_commit(&s_afree[as]);
        tc_commit(&s_empty[st]);
      }
    }
    if (leader && (!ok || *const_cast<volatile int *>(&s_abort))) {
      // Every MMA issued must be done before its operands and the tensor memory go away.
      tc_commit(&s_drain);
      mbar_wait_unabortable(&s_drain, 0);
    }
  } else if (warp >= kWarpUnpack) {
    // ---- unpacking: a thread per output ----
    const int t = (warp & 3) * 32 + lane;
    const uint32_t taddr = tmem + (static_cast<uint32_t>((warp & 3) * 32) << 16) + kColA;
    const uint32_t *pair = p.pairs + static_cast<int64_t>(min(o0 + t, p.N - 1)) * groups;
    const bool whole = groups % U == 0;
    uint32_t now[U], next[U];
    if (u0 < u1) load_unit_pairs<U>(pair, u0, groups, whole, next);
    uint32_t it = 0;
    for (int u = u0; u < u1; ++u, ++it) {
#pragma unroll
      for (int q = 0; q < U; ++q) now[q] = next[q];
      if (u + 1 < u1) load_unit_pairs<U>(pair, u + 1, groups, whole, next);
      const int st = it % kStages, as = it & 1;
      ok = mbar_wait_lean(&s_full[st], (it / kStages) & 1, &s_abort) &&
           mbar_wait_lean(&s_afree[as], ((it / 2) & 1) ^ 1, &s_abort);
      ok = __all_sync(0xffffffffu, ok);
      if (!ok) break;
      tc_fence_after();
      const uint8_t *row = smem + st * S::kStage + t * 64;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const uint4 v = *reinterpret_cast<const uint4 *>(row + ((j ^ ((t >> 1) & 3)) << 4));
        const __nv_bfloat162 nz = __float2bfloat162_rn(-128.f - int4::pair_of(now[j * 32 / G]).y);
        uint32_t a[16];
        int4::unpack_bf16(v.x, nz, a);
        int4::unpack_bf16(v.y, nz, a + 4);
        int4::unpack_bf16(v.z, nz, a + 8);
        int4::unpack_bf16(v.w, nz, a + 12);
        tmem_st16(taddr + as * 64 + j * 16, a);
      }
      tmem_wait_st();
      tc_fence_before();
      __syncwarp();
      if (lane == 0) {
        mbar_arrive(&s_afull[as]);
        mbar_arrive(&s_empty[st]);
      }
    }
  } else {
    // ---- draining: a group's sums under the outputs' scales ----
    const int t = (warp & 3) * 32 + lane;
    const uint32_t taddr = tmem + (static_cast<uint32_t>((warp & 3) * 32) << 16) + kColD;
    const uint32_t *pair = p.pairs + static_cast<int64_t>(min(o0 + t, p.N - 1)) * groups;
    const bool whole = groups % U == 0;
    uint32_t now[U], next[U];
    if (u0 < u1) load_unit_pairs<U>(pair, u0, groups, whole, next);
    F2 sum[NR / 2];
#pragma unroll
    for (int r = 0; r < NR / 2; ++r) sum[r] = f2(0.f, 0.f);
    uint32_t gi = 0;
    for (int u = u0; ok && u < u1; ++u) {
#pragma unroll
      for (int q = 0; q < U; ++q) now[q] = next[q];
      if (u + 1 < u1) load_unit_pairs<U>(pair, u + 1, groups, whole, next);
      const int ng = min(U, groups - u * U);
#pragma unroll
      for (int q = 0; q < U; ++q) {
        if (q >= ng) break;
        const int db = gi & 1;
        ok = __all_sync(0xffffffffu, mbar_wait_lean(&s_dfull[db], (gi / 2) & 1, &s_abort));
        if (!ok) break;
        tc_fence_after();
        const float s = int4::pair_of(now[q]).x;
        const F2 ss = f2(s, s);
#pragma unroll
        for (int r = 0; r < NR; r += 16) {
          uint32_t y[16];
          tmem_ld8(taddr + db * 64 + r, y);
          tmem_ld8(taddr + db * 64 + r + 8, y + 8);
          tmem_wait_ld();
#pragma unroll
          for (int e = 0; e < 16; e += 2)
            sum[(r + e) / 2] = f2_fma(f2(__uint_as_float(y[e]), __uint_as_float(y[e + 1])), ss, sum[(r + e) / 2]);
        }
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(&s_dfree[db]);
        ++gi;
      }
    }
#pragma unroll
    for (int r = 0; r < NR; r += 2) f2_split(sum[r / 2], acc[r], acc[r + 1]);
  }
  if (!ok && lane == 0) atomicOr(p.status, SPADE_DEV_TIMEOUT);

  const int rows = min(p.tile_rows, p.R - n0);
  const bool drains = warp >= kWarpDrain && warp < kWarpUnpack;
  const int t = (warp & 3) * 32 + lane;
  if (split == 1) {
    if (drains && o0 + t < p.N) {
#pragma unroll
      for (int r = 0; r < NR; ++r) {
        if (r >= rows) break;
        const int64_t at = static_cast<int64_t>(n0 + r) * p.N + o0 + t;
        p.out[at] = __float2bfloat16_rn(acc[r] + (p.residual ? __bfloat162float(p.residual[at]) : 0.f));
      }
    }
  } else {
    // Every CTA's sums into its own ring (all copies and MMAs of it are done: the draining
    // warps have seen the last one's), then rows dealt to the CTAs.
    float *sums = reinterpret_cast<float *>(smem);
    __syncthreads();
    if (drains) {
#pragma unroll
      for (int r = 0; r < NR; ++r) sums[r * kOut + t] = acc[r];
    }
    __syncwarp();
    cluster_sync();
    const int r0 = rows * rank / split, r1 = rows * (rank + 1) / split;
    for (int e = threadIdx.x; e < (r1 - r0) * kOut; e += kThreads) {
      const int r = r0 + e / kOut, o = e % kOut;
      float y = 0.f;
      for (int c = 0; c < split; ++c) {
        float v;
        asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v) : "r"(cluster_map(sums + r * kOut + o, c)));
        y += v;
      }
      if (o0 + o < p.N) {
        const int64_t at = static_cast<int64_t>(n0 + r) * p.N + o0 + o;
        p.out[at] = __float2bfloat16_rn(y + (p.residual ? __bfloat162float(p.residual[at]) : 0.f));
      }
    }
    __syncwarp();
    cluster_sync();  // no CTA leaves while another reads its sums
  }
  tc_fence_before();
  __syncthreads();
  if (warp == 1) {
    tc_fence_after();
    tmem_dealloc(tmem, kTmemCols);
  }
}

}  // namespace tc

// `grid` CTAs of `kern` in clusters of `cluster`, programmatic dependent launch.
template <class... A>
static cudaError_t launch(void (*kern)(A...), dim3 grid, unsigned cluster, unsigned threads, size_t smem, cudaStream_t s,
                          A... a) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = grid;
  cfg.blockDim = dim3(threads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = s;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = cluster;
  attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = cluster > 1 ? 2 : 1;
  return cudaLaunchKernelEx(&cfg, kern, a...);
}

template <int G, int MT>
static cudaError_t few_rows_mt(const Params &p, const CUtensorMap &tm, cudaStream_t s) {
  constexpr int kBytes = kWarps * kRing * MT * 1024 + 1024;
  static OncePerDevice once;
  const cudaError_t e = set_max_smem(once, kBytes, few_rows_kernel<G, MT>);
  if (e != cudaSuccess) return e;
  return launch(few_rows_kernel<G, MT>, dim3((static_cast<unsigned>(p.N) + MT * 16 - 1) / (MT * 16)), 1, kThreads, kBytes, s,
                p, tm);
}
// 32 outputs a CTA halve the reads of x; 16 fill the SMs sooner.
static bool wide_tiles(int N, int sms) { return (static_cast<unsigned>(N) + 31) / 32 >= 2u * sms; }
template <int G>
static cudaError_t few_rows(const Params &p, const CUtensorMap &tm, bool wide, cudaStream_t s) {
  return wide ? few_rows_mt<G, 2>(p, tm, s) : few_rows_mt<G, 1>(p, tm, s);
}

template <int G, int NR>
static cudaError_t rows_nr(const Params &p, const CUtensorMap &w, const CUtensorMap &x, cudaStream_t s) {
  static OncePerDevice once;
  const cudaError_t e = set_max_smem(once, tc::Smem<NR>::BYTES, tc::rows_kernel<G, NR>);
  if (e != cudaSuccess) return e;
  const unsigned tiles = (static_cast<unsigned>(p.N) + tc::kOut - 1) / tc::kOut;
  const dim3 grid(tiles * p.split, (p.R + p.tile_rows - 1) / p.tile_rows);
  return launch(tc::rows_kernel<G, NR>, grid, p.split, tc::kThreads, tc::Smem<NR>::BYTES, s, p, w, x);
}
template <int G>
static cudaError_t rows_g(const Params &p, int nr, const CUtensorMap &w, const CUtensorMap &x, cudaStream_t s) {
  switch (nr) {
    case 16: return rows_nr<G, 16>(p, w, x, s);
    case 32: return rows_nr<G, 32>(p, w, x, s);
    case 48: return rows_nr<G, 48>(p, w, x, s);
    default: return rows_nr<G, 64>(p, w, x, s);
  }
}

// CTAs that share a tile's units: those that fill the GPU's slots (two per SM) in the
// fewest rounds per part, of at least four units each; the fewer the better.
static int split_of(int64_t tiles, int units, int sms) {
  int best = 1;
  double cost = 1e30;
  for (int s = 1; s <= tc::kMaxSplit && (s == 1 || units >= 4 * s); s *= 2) {
    const double c = static_cast<double>((tiles * s + 2 * sms - 1) / (2 * sms)) / s;
    if (c < cost) {
      cost = c;
      best = s;
    }
  }
  return best;
}

}  // namespace w4
}  // namespace spade

using namespace spade;

extern "C" spade_status spade_linear_w4(const void *x, const void *codes, const void *params, const void *residual,
                                        void *out, int32_t R, int32_t N, int32_t K, int32_t group, int32_t *status,
                                        spade_stream_t stream) {
  if (!x || !codes || !params || !out || !status)
    return fail(SPADE_ERR_INVALID_ARG, "spade_linear_w4: null pointer argument");
  if (R <= 0 || N <= 0 || K <= 0) return fail(SPADE_ERR_INVALID_ARG, "spade_linear_w4: non-positive size");
  if (group != 32 && group != 64 && group != 128)
    return fail(SPADE_ERR_SHAPE, "spade_linear_w4: group %d not supported (32, 64 or 128)", group);
  if (K % group) return fail(SPADE_ERR_SHAPE, "spade_linear_w4: K = %d must be a multiple of the group (%d)", K, group);
  if (!aligned(x, 16) || !aligned(codes, 16) || !aligned(params, 16) || !aligned(residual, 16) || !aligned(out, 16))
    return fail(SPADE_ERR_INVALID_ARG, "spade_linear_w4: pointers must be 16-byte aligned");
  int sms = 0;
  spade_status st = device_info(&sms, nullptr);
  if (st != SPADE_OK) return st;
  w4::Params p;
  p.x = static_cast<const __nv_bfloat16 *>(x);
  p.residual = static_cast<const __nv_bfloat16 *>(residual);
  p.codes = static_cast<const uint32_t *>(codes);
  p.pairs = static_cast<const uint32_t *>(params);
  p.out = static_cast<__nv_bfloat16 *>(out);
  p.status = status;
  p.R = R; p.N = N; p.K = K; p.tile_rows = R; p.split = 1;
  cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
  CUtensorMap w;
  cudaError_t e;
  if (R <= w4::kRows) {
    const bool wide = w4::wide_tiles(N, sms);
    if (!encode_tmap_bytes(&w, codes, K / 2, N, wide ? 32 : 16, 64)) return SPADE_ERR_CUDA;
    e = group == 128 ? w4::few_rows<128>(p, w, wide, s)
        : group == 64 ? w4::few_rows<64>(p, w, wide, s)
                      : w4::few_rows<32>(p, w, wide, s);
  } else {
    const int64_t row_tiles = (static_cast<int64_t>(R) + 63) / 64;
    if (row_tiles > 65535) return fail(SPADE_ERR_SHAPE, "spade_linear_w4: R = %d exceeds %d rows per call", R, 65535 * 64);
    p.tile_rows = static_cast<int>((R + row_tiles - 1) / row_tiles);
    const int nr = (p.tile_rows + 15) / 16 * 16;
    const int64_t tiles = (static_cast<int64_t>(N) + w4::tc::kOut - 1) / w4::tc::kOut * row_tiles;
    p.split = w4::split_of(tiles, (K + w4::kUnit - 1) / w4::kUnit, sms);
    CUtensorMap xm;
    if (!encode_tmap_bytes(&w, codes, K / 2, N, w4::tc::kOut, 64) ||
        !encode_tmap_bf16_sw128(&xm, x, K, R, static_cast<uint64_t>(K) * 2, 64, nr))
      return SPADE_ERR_CUDA;
    e = group == 128 ? w4::rows_g<128>(p, nr, w, xm, s)
        : group == 64 ? w4::rows_g<64>(p, nr, w, xm, s)
                      : w4::rows_g<32>(p, nr, w, xm, s);
  }
  return e == cudaSuccess ? SPADE_OK : cuda_fail(e, "linear_w4 launch");
}
