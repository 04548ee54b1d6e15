// linear_w4.cu -- y = x W^T (+ residual) with W in 4 bits: the verifier's linear
// layers (f_l in x_{l+1} = x_l + f_l(x_l), Sec. III-A) for the rows of a verify block
// or single tokens.
#include <cfloat>

#include "int4.cuh"
#include "internal.h"
#include "launch.h"
#include "ptx.cuh"

namespace spade {
namespace w4 {

struct Params {
  const __nv_bfloat16 *x, *residual;
  const uint32_t *codes, *pairs;
  __nv_bfloat16 *out;
  int32_t *status;
  int R, N, K;
  // (More than eight rows) rows of a tile, rounded up to 16, and the CTAs that share its units.
  int tile_rows, tile_n, split;
};

// ---- up to eight rows: the weights streamed past mma.sync -----------------------------------
// y^T = W x^T on mma.sync (m16n8k16): 16 outputs on M, the rows of x on N.  Bound by the
// weights' bytes: 4 1/4 to 5 bits each, read once.  The order of K inside an MMA is free
// as long as both operands share it, so a thread's fragment of a group is simply its own
// contiguous part of the weight row (two bf16 pairs per MMA and row come out of one word
// with masks), and the same part of the row of x.  Codes minus zero are whole numbers,
// exact in bf16, and a group's products are summed apart and then scaled in fp32: nothing
// of W is rounded.
// One CTA per SM takes a range of 16-output tiles; its warps share K, each with a span of
// 256 k whose part of x stays in registers while the range's weights pass by (with eight
// rows, fragments of x read again for every 32 outputs were as many bytes as the weights).
// A warp has a ring of its own, filled by its lanes with 16-byte copies; the copies' places
// make the fragments' reads free of bank conflicts for every group size.  Sums of a tile
// wait in shared memory and are added over the warps in a fixed order.
// 6 rows of 12288 x 4096, group 32: 10.7 us, 3.0 TB/s (9.9 where three such weights stay in L2);
// 1 row of 57344 x 8192, group 128: 54 us, 4.6 TB/s, where the copies alone take 43 us and the
// unpacking alone 43 us: both fill the SM.
constexpr int kWarps = 16, kThreads = 32 * kWarps;
constexpr int kUnit = 128;   // k per unit
constexpr int kSpan = 256;   // k of a warp: two units
constexpr int kTile = 16;    // outputs of a tile
constexpr int kRing = 2;     // spans in flight per warp (3 or 4: 1 to 5 % slower)
constexpr int kHold = 8;     // tiles per warp whose sums wait in shared memory
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

// Shared memory of a CTA: the rings (codes, then pairs of a span), the sums that wait.
template <int G>
struct Few {
  static constexpr int kPairs = kSpan / G;                     // pairs of an output in a span
  static constexpr int kStage = kTile * (kSpan / 2 + kPairs * 4);
  static constexpr int kRings = kWarps * kRing * kStage;
  static constexpr int kSums = kWarps * 512;                   // one tile per warp
};

template <int G>
__global__ void __launch_bounds__(kThreads, 1) few_rows_kernel(const __grid_constant__ Params p) {
  using F = Few<G>;
  constexpr int W = G / 32, U = kUnit / G;  // words of a thread's part of a group; groups of a unit
  constexpr int kCodes = kTile * kSpan / 2;
  extern __shared__ __align__(16) uint8_t smem[];
  const int warp = uniform_warp(), lane = threadIdx.x & 31;
  const int r = lane >> 2, t = lane & 3;
  const int groups = p.K / G, spans = (p.K - 1) / kSpan + 1, row_bytes = p.K / 2;
  uint8_t *ring = smem + warp * kRing * F::kStage;
  float4 *sums = reinterpret_cast<float4 *>(smem + F::kRings);
  // Warps along K (a power of two) and along the tiles.
  const int kw = p.split, tw = kWarps / kw;
  const int ki = warp & (kw - 1), ti = warp / kw;
  const int tiles = (p.N - 1) / kTile + 1;
  const int tile0 = static_cast<int>(static_cast<int64_t>(tiles) * blockIdx.x / gridDim.x);
  const int tile1 = static_cast<int>(static_cast<int64_t>(tiles) * (blockIdx.x + 1) / gridDim.x);
  const int slabs = ki < spans ? (spans - ki + kw - 1) / kw : 0;  // spans of this warp
  // Tiles of this warp among the kHold * tw from `base` on.
  auto tiles_from = [&](int base) { return min(kHold, (tile1 - base - ti + tw - 1) / tw); };
  griddep_wait();
  griddep_launch_dependents();

  // ---- copies: steps in the order of the loops below, kRing ahead ----
  // A lane copies pieces lane % 8 of rows lane / 8 + 0, 4, 8, 12: unit h = piece / 4 has a
  // block of 64-byte rows, piece t of row r at place t ^ (r / 2 mod 4) of row r ^ h.
  const bool whole = groups % F::kPairs == 0;
  struct {
    int base, slab, i;
  } at = {slabs ? tile0 : tile1, 0, 0};
  auto fetch = [&](int slot) {  // also counts a group where no step is left
    if (at.base + ti < tile1) {
      const int o0 = (at.base + ti + at.i * tw) * kTile, span = at.slab * kw + ki;
      uint8_t *stage = ring + slot * F::kStage;
      const int piece = lane & 7;
      const bool in = span * (kSpan / 2) + piece * 16 < row_bytes;
      const uint8_t *codes = reinterpret_cast<const uint8_t *>(p.codes) + (in ? span * (kSpan / 2) + piece * 16 : 0);
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const int row = q * 4 + (lane >> 3), h = piece >> 2;
        cp_async16(smem_u32(stage) + h * 1024 + (row ^ h) * 64 + (((piece & 3) ^ ((row >> 1) & 3)) << 4),
                   codes + static_cast<int64_t>(min(o0 + row, p.N - 1)) * row_bytes, in ? 16 : 0);
      }
      // Pairs: two lanes per row, a unit's each.
      const int row = lane >> 1, g0 = span * F::kPairs + (lane & 1) * U;
      const uint32_t *from = p.pairs + static_cast<int64_t>(min(o0 + row, p.N - 1)) * groups;
      const uint32_t to = smem_u32(stage) + kCodes + (row * F::kPairs + (lane & 1) * U) * 4;
      if (whole) {
        asm volatile("cp.async.ca.shared.global [%0], [%1], %2;" ::"r"(to), "l"(from + g0), "n"(U * 4) : "memory");
      } else {
#pragma unroll
        for (int q = 0; q < U; ++q) {
          const bool have = g0 + q < groups;
          asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(to + q * 4), "l"(have ? from + g0 + q : from),
                       "r"(have ? 4 : 0)
                       : "memory");
        }
      }
      if (++at.i == tiles_from(at.base)) {
        at.i = 0;
        if (++at.slab == slabs) {
          at.slab = 0;
          at.base += kHold * tw;
        }
      }
    }
    cp_async_commit();
  };
#pragma unroll
  for (int s = 0; s < kRing; ++s) fetch(s);

  const uint4 *x = reinterpret_cast<const uint4 *>(p.x + static_cast<int64_t>(min(r, p.R - 1)) * p.K) + W * t;
  int slot = 0;
  for (int base = tile0; base < tile1; base += kHold * tw) {
    const int mine = tiles_from(base);
    for (int slab = 0; slab < slabs; ++slab) {
      const int g0 = (slab * kw + ki) * F::kPairs;
      uint4 xv[8];
      if (mine > 0) {
#pragma unroll
        for (int q = 0; q < F::kPairs; ++q)
#pragma unroll
          for (int e = 0; e < W; ++e)
            xv[q * W + e] = g0 + q < groups ? x[static_cast<int64_t>(g0 + q) * (G / 8) + e] : make_uint4(0, 0, 0, 0);
      }
      for (int i = 0; i < mine; ++i) {
        cp_async_wait<kRing - 1>();
        __syncwarp();
        const uint8_t *stage = ring + slot * F::kStage;
        uint32_t w[2][2][4], pairs[2][F::kPairs];
#pragma unroll
        for (int m = 0; m < 2; ++m) {
#pragma unroll
          for (int h = 0; h < 2; ++h) read_words<W>(stage + h * 1024, (m * 8 + r) ^ h, t, w[h][m]);
          const uint32_t *pr = reinterpret_cast<const uint32_t *>(stage + kCodes) + (m * 8 + r) * F::kPairs;
#pragma unroll
          for (int q = 0; q < F::kPairs; q += 2) {
            const uint2 v = *reinterpret_cast<const uint2 *>(pr + q);
            pairs[m][q] = v.x;
            pairs[m][q + 1] = v.y;
          }
        }
        __syncwarp();
        fetch(slot);
        slot = slot + 1 == kRing ? 0 : slot + 1;
        float acc[4] = {};
#pragma unroll
        for (int q = 0; q < F::kPairs; ++q) {
          const float2 lo = int4::pair_of(pairs[0][q]), hi = int4::pair_of(pairs[1][q]);
          const __nv_bfloat162 z0 = __float2bfloat162_rn(-128.f - lo.y), z1 = __float2bfloat162_rn(-128.f - hi.y);
          float c[4] = {};
#pragma unroll
          for (int e = 0; e < W; ++e) {
            uint32_t a[4], b[4];
            int4::unpack_bf16(w[q / U][0][q % U * W + e], z0, a);
            int4::unpack_bf16(w[q / U][1][q % U * W + e], z1, b);
            const uint4 v = xv[q * W + e];
            mma_bf16(c, a[0], b[0], a[1], b[1], v.x, v.y);
            mma_bf16(c, a[2], b[2], a[3], b[3], v.z, v.w);
          }
          acc[0] = fmaf(lo.x, c[0], acc[0]);
          acc[1] = fmaf(lo.x, c[1], acc[1]);
          acc[2] = fmaf(hi.x, c[2], acc[2]);
          acc[3] = fmaf(hi.x, c[3], acc[3]);
        }
        float4 &sum = sums[(i * kWarps + warp) * 32 + lane];
        if (slab) {
          const float4 s = sum;
          acc[0] += s.x; acc[1] += s.y; acc[2] += s.z; acc[3] += s.w;
        }
        sum = make_float4(acc[0], acc[1], acc[2], acc[3]);
      }
    }
    __syncthreads();
    const int here = min(kHold * tw, tile1 - base);
    for (int e = threadIdx.x; e < here * 128; e += kThreads) {
      const int tile = e >> 7, l = (e >> 2) & 31, c = e & 3;
      const int n = 2 * (l & 3) + (c & 1);
      const int64_t o = static_cast<int64_t>(base + tile) * kTile + (c >> 1) * 8 + (l >> 2);
      if (n >= p.R || o >= p.N) continue;
      // Tile `tile` is number tile / tw of the warps (tile mod tw) * kw + 0 .. kw - 1.
      const float *from = reinterpret_cast<const float *>(sums) + ((tile / tw) * kWarps + (tile % tw) * kw) * 128 + (e & 127);
      float y = 0.f;
      for (int k = 0; k < min(kw, spans); ++k) y += from[k * 128];
      const int64_t to = n * static_cast<int64_t>(p.N) + o;
      p.out[to] = __float2bfloat16_rn(y + (p.residual ? __bfloat162float(p.residual[to]) : 0.f));
    }
    if (base + kHold * tw < tile1) __syncthreads();
  }
}

// ---- more rows: tcgen05 with the weights in tensor memory ----------------------------------
// y^T = W x^T again: 128 outputs on M, up to 128 rows of x on N, units of 128 k.  A
// thread unpacks one output's unit (64 bytes of codes) to whole numbers in bf16 and stores
// them to its lane of tensor memory, from where the MMA takes A (no shared-memory traffic
// for W beyond its codes, and no loss of MMA rate at small N); x comes by TMA as B.  Each
// group of k is accumulated apart, exact but for the fp32 sums, in one of two blocks of
// columns, and the draining warps take the other under the outputs' scales into registers.
// Bound by the weights' bytes at few rows, then by the instructions that unpack (each row
// tile unpacks W again) and drain (each group of k once), with the MMAs close behind: a unit
// of 128 x 128 sums takes 950 cycles at group 128, its MMAs 512.  Up to 32 rows a tile two
// CTAs share an SM, so that one's waits are the other's work; wider tiles take an SM each,
// since halving the unpacking is worth more (389 rows of 7168 x 5120 in tiles of 56 rows, two
// CTAs: 99 us).  At group 128 a CTA can take two tiles of outputs: they share the copies of x
// and a CTA's start and end, with three blocks of sums and two of unpacked weights in turn.
// 20 rows of 8192 x 8192, group 64: 16.1 us; 389 rows of 7168 x 5120, group 128: 39.6 us, and
// 1024 rows of 12288 x 4096: 110 us (720 and 935 TFLOP/s).
// Where the tiles do not fill the GPU, a cluster of 2, 4 or 8 CTAs takes a tile's units
// in equal parts and adds the sums through distributed shared memory in a fixed order.
namespace tc {

constexpr int kOut = 128;                       // outputs of a tile
constexpr int kCodes = kOut * 64;               // a unit's codes: 8 KB
constexpr int kMaxSplit = 8;
constexpr int kNarrow = 32, kMost = 128;        // rows of a narrow and of a wide tile, at most
constexpr int kMaxStages = 6, kMaxA = 4;

template <int G, bool kWide, int kTiles>
struct Shape {
  static constexpr int kRows = kWide ? kMost : kNarrow;  // most rows of a tile
  static constexpr int kM = kTiles;                    // tiles of outputs that share a tile of x
  static constexpr int kHalves = kWide ? 2 : 1;        // draining warps per lane quadrant and tile of outputs
  static constexpr int kHalfRows = kRows / kHalves;    // sums of a draining thread
  static constexpr int kWarpDrain = 2, kWarpUnpack = 2 + 4 * kHalves * kM;
  static constexpr int kThreads = 32 * (kWarpUnpack + 4);  // four unpacking warps
  static constexpr int kPerSm = kWide ? 1 : 2;
  static constexpr int kStages = kM == 2 ? 4 : 5;        // copy ring (units)
  static constexpr int kChunk = kM == 2 ? 16 : 32;       // sums that a draining thread reads at a time
  static constexpr int kBlock = !kWide && G <= 64 ? 2 : 1;  // groups accumulated side by side and drained together
  static constexpr int kD = kM == 2 ? 3 : 2;           // blocks of columns that sums go to
  static constexpr int kA = kM == 2 ? 2 : kWide ? 4 : kBlock == 2 ? 2 : 3;  // unpacked units
  static constexpr uint32_t kTmemCols = kWide ? 512 : 256;
  static constexpr uint32_t kColD = 0, kColA = kD * kBlock * kRows;
  static constexpr int kX = kRows * 256;               // a unit of x: two slabs of [rows][64 k]
  static constexpr int kPairs = kM * kOut * (kUnit / G) * 4;  // a unit's (scale, zero) pairs
  static constexpr int kAtX = kM * kCodes, kAtPairs = kAtX + kX;
  static constexpr int kStage = (kAtPairs + kPairs + 1023) / 1024 * 1024;
  static constexpr int kBytes = kStages * kStage + 1024;
  static_assert(kColA + kA * 64 <= kTmemCols, "tensor memory");
  static_assert(kM * kOut * kRows * 4 <= kStages * kStage, "a split's sums reuse the ring");
  static_assert(kStages <= kMaxStages && kA <= kMaxA, "barriers");
};

// Output t's pairs of a unit.
template <int U>
SPADE_DEVICE void read_pairs(const uint8_t *pairs, int t, uint32_t (&p)[U]) {
  if constexpr (U == 4) {
    const uint4 v = reinterpret_cast<const uint4 *>(pairs)[t];
    p[0] = v.x; p[1] = v.y; p[2] = v.z; p[3] = v.w;
  } else if constexpr (U == 2) {
    const uint2 v = reinterpret_cast<const uint2 *>(pairs)[t];
    p[0] = v.x; p[1] = v.y;
  } else {
    p[0] = reinterpret_cast<const uint32_t *>(pairs)[t];
  }
}

template <int G, bool kWide, int kTiles>
__global__ void __launch_bounds__(Shape<G, kWide, kTiles>::kThreads, Shape<G, kWide, kTiles>::kPerSm)
    rows_kernel(const __grid_constant__ Params p, const __grid_constant__ CUtensorMap tm_w,
                const __grid_constant__ CUtensorMap tm_x) {
  using S = Shape<G, kWide, kTiles>;
  constexpr int U = kUnit / G;
  extern __shared__ uint8_t smem_raw[];
  uint8_t *smem = smem_raw + ((1024u - (smem_u32(smem_raw) & 1023u)) & 1023u);
  __shared__ uint64_t s_full[kMaxStages], s_empty[kMaxStages], s_afull[kMaxA], s_afree[kMaxA], s_dfull[3], s_dfree[3],
      s_drain;
  __shared__ int s_abort;
  __shared__ uint32_t s_tmem;
  const int warp = uniform_warp(), lane = threadIdx.x & 31;
  if (threadIdx.x == 0) {
    s_abort = 0;
    tma_prefetch_desc(&tm_w);
    tma_prefetch_desc(&tm_x);
    for (int s = 0; s < S::kStages; ++s) {
      mbar_init(&s_full[s], 33);                   // the leader's copies, every lane's pairs
      mbar_init(&s_empty[s], 4 + 4 * S::kHalves * S::kM + 1);  // the unpacking and draining warps, and the MMAs
    }
    for (int s = 0; s < S::kA; ++s) {
      mbar_init(&s_afull[s], 4);
      mbar_init(&s_afree[s], 1);
    }
    for (int s = 0; s < S::kD; ++s) {
      mbar_init(&s_dfull[s], 1);
      mbar_init(&s_dfree[s], 4 * S::kHalves);
    }
    mbar_init(&s_drain, 1);
    fence_mbar_init();
  }
  if (warp == 1) {
    tmem_alloc(&s_tmem, S::kTmemCols);
    tmem_relinquish();
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = s_tmem;
  const int groups = p.K / G, units = (groups + U - 1) / U;
  const int split = p.split, rank = split > 1 ? static_cast<int>(cluster_ctarank()) : 0;
  const int o0 = static_cast<int>(blockIdx.x / split) * (S::kM * kOut), n0 = blockIdx.y * p.tile_rows;
  const int n = p.tile_n;  // rows of x in the MMA: the tile's, rounded up to 16
  const int u0 = static_cast<int>(static_cast<int64_t>(units) * rank / split);
  const int u1 = static_cast<int>(static_cast<int64_t>(units) * (rank + 1) / split);
  const int t = (warp & 3) * 32 + lane;                       // output of the unpacking and draining threads
  const uint32_t tlane = tmem + (static_cast<uint32_t>((warp & 3) * 32) << 16);
  const int half_rows = kWide ? (n / 16 + 1) / 2 * 16 : n;    // rows of the first draining half
  const int dm = (warp - S::kWarpDrain) / (4 * S::kHalves);   // (draining) the warp's tile of outputs
  const int r_lo = kWide && ((warp - S::kWarpDrain) & 4) ? half_rows : 0;  // and its thread's first row
  const int my_rows = min(half_rows, n - r_lo);
  griddep_wait();
  griddep_launch_dependents();
  F2 sum[S::kHalfRows / 2];  // (draining warps: one output's sums)
  bool ok = true;
  if (warp == 0) {
    // ---- copies ----
    const bool leader = elect_one();
    // x is read by every tile of outputs, W again by every tile of rows.
    const uint64_t pol = l2_policy_evict_last(), pol_w = gridDim.y > 1 ? pol : l2_policy_evict_first();
    uint32_t issued = 0;
    for (int u = u0; u < u1; ++u, ++issued) {
      const int st = issued % S::kStages;
      ok = __all_sync(0xffffffffu, mbar_wait_lean(&s_empty[st], ((issued / S::kStages) & 1) ^ 1, &s_abort));
      if (!ok) break;
      uint8_t *stage = smem + st * S::kStage;
      // Pairs: four outputs per lane, by asynchronous copies that arrive on the stage's barrier
      // themselves.
#pragma unroll
      for (int r = lane; r < S::kM * kOut; r += 32) {
        const uint32_t *from = p.pairs + static_cast<int64_t>(min(o0 + r, p.N - 1)) * groups + u * U;
        const uint32_t to = smem_u32(stage + S::kAtPairs) + r * (U * 4);
        if (groups % U == 0) {
          asm volatile("cp.async.ca.shared.global [%0], [%1], %2;" ::"r"(to), "l"(from), "n"(U * 4) : "memory");
        } else {
#pragma unroll
          for (int q = 0; q < U; ++q) {
            const bool in = u * U + q < groups;  // (zeros past the last group)
            asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(to + q * 4), "l"(in ? from + q : p.pairs),
                         "r"(in ? 4u : 0u) : "memory");
          }
        }
      }
      asm volatile("cp.async.mbarrier.arrive.noinc.shared::cta.b64 [%0];" ::"r"(smem_u32(&s_full[st])) : "memory");
      if (leader) {
        mbar_arrive_expect_tx(&s_full[st], S::kM * kCodes + n * 256);
#pragma unroll
        for (int m = 0; m < S::kM; ++m)
          tma_load_2d(stage + m * kCodes, &tm_w, u * (kUnit / 2), o0 + m * kOut, &s_full[st], pol_w);
        tma_load_2d(stage + S::kAtX, &tm_x, u * kUnit, n0, &s_full[st], pol);
        tma_load_2d(stage + S::kAtX + S::kX / 2, &tm_x, u * kUnit + 64, n0, &s_full[st], pol);
      }
    }
    asm volatile("cp.async.wait_all;" ::: "memory");
    // Every copy issued must land before the CTA's shared memory goes away, also where another
    // warp's wait expires once this one is done (else all have: the consumers waited for them).
    if (leader)
      for (uint32_t j = issued > S::kStages ? issued - S::kStages : 0; j < issued; ++j)
        mbar_wait_unabortable(&s_full[j % S::kStages], (j / S::kStages) & 1);
  } else if (warp == 1) {
    // ---- MMAs ----
    const uint32_t idesc = idesc_bf16_f32(kOut, n);
    const bool leader = elect_one();
    const uint32_t base = smem_u32(smem);
    uint32_t it = 0, bi = 0;
    auto wait = [&](uint64_t *bar, uint32_t parity) {
      ok = __all_sync(0xffffffffu, mbar_wait_lean(bar, parity, &s_abort)) && ok;
    };
    for (int u = u0; ok && u < u1; ++u, ++it) {
      const int st = it % S::kStages;
      wait(&s_full[st], (it / S::kStages) & 1);
      if constexpr (S::kM == 1) {
        wait(&s_afull[it % S::kA], (it / S::kA) & 1);
        if (!ok) break;
      }
      const uint64_t dx = smem_desc_sw128(base + st * S::kStage + S::kAtX);
      const int ng = min(U, groups - u * U);
#pragma unroll
      for (int q0 = 0; q0 < U; q0 += S::kBlock) {
        if (q0 >= ng) break;
#pragma unroll
        for (int m = 0; m < S::kM; ++m) {
          const uint32_t ai = it * S::kM + m;
          const int as = ai % S::kA;
          if (S::kM > 1 && q0 == 0) wait(&s_afull[as], (ai / S::kA) & 1);
          const int db = bi % S::kD;
          wait(&s_dfree[db], ((bi / S::kD) & 1) ^ 1);
          tc_fence_after();
#pragma unroll
          for (int q = q0; q < q0 + S::kBlock; ++q) {  // (a group past the last: zeros)
            const uint32_t d = tmem + S::kColD + (db * S::kBlock + q - q0) * S::kRows;
#pragma unroll
            for (int k = 0; k < G / 16; ++k) {
              const int kk = q * (G / 16) + k;  // four per 64-k slab
              const uint32_t off = ((kk / 4) * (S::kX / 2) + (kk % 4) * 32) >> 4;
              if (leader) tc_mma_f16_ta(d, tmem + S::kColA + as * 64 + kk * 8, dx + off, idesc, k > 0);
            }
          }
          if (leader) {
            tc_commit(&s_dfull[db]);
            if (S::kM > 1 && q0 + S::kBlock >= ng) tc_commit(&s_afree[as]);
          }
          ++bi;
        }
      }
      if (leader && ok) {
        if constexpr (S::kM == 1) tc_commit(&s_afree[it % S::kA]);
        tc_commit(&s_empty[st]);
      }
    }
    // Every MMA issued must be done before its operands and the tensor memory go away (see the copies).
    if (leader) {
      tc_commit(&s_drain);
      mbar_wait_unabortable(&s_drain, 0);
    }
  } else if (warp >= S::kWarpUnpack) {
    // ---- unpacking: a thread per output ----
    for (int u = u0; u < u1; ++u) {
      const int it = u - u0, st = it % S::kStages;
#pragma unroll
      for (int m = 0; m < S::kM; ++m) {
        const int ai = it * S::kM + m, as = ai % S::kA;
        ok = (m || mbar_wait_lean(&s_full[st], (it / S::kStages) & 1, &s_abort)) && mbar_wait_lean(&s_afree[as], ((ai / S::kA) & 1) ^ 1, &s_abort);
        ok = __all_sync(0xffffffffu, ok);
        if (!ok) break;
        tc_fence_after();
        uint32_t now[U];
        read_pairs<U>(smem + st * S::kStage + S::kAtPairs, m * kOut + t, now);
        const uint8_t *row = smem + st * S::kStage + m * kCodes + t * 64;
#pragma unroll
        for (int j = 0; j < 4; ++j) {  // 32 k each
          const uint4 v = *reinterpret_cast<const uint4 *>(row + ((j ^ ((t >> 1) & 3)) << 4));
          const __nv_bfloat162 nz = __float2bfloat162_rn(-128.f - int4::pair_of(now[j * 32 / G]).y);
          uint32_t a[16];
          int4::unpack_bf16(v.x, nz, a);
          int4::unpack_bf16(v.y, nz, a + 4);
          int4::unpack_bf16(v.z, nz, a + 8);
          int4::unpack_bf16(v.w, nz, a + 12);
          tmem_st16(tlane + S::kColA + as * 64 + j * 16, a);
        }
        tmem_wait_st();
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(&s_afull[as]);
      }
      if (!ok) break;
      if (lane == 0) mbar_arrive(&s_empty[st]);
    }
  } else {
    // ---- draining: a group's sums under the outputs' scales ----
#pragma unroll
    for (int r = 0; r < S::kHalfRows / 2; ++r) sum[r] = f2(0.f, 0.f);
    uint32_t it = 0, bi = 0;
    for (int u = u0; ok && u < u1; ++u, ++it) {
      const int ng = min(U, groups - u * U), st = it % S::kStages;
      uint32_t now[U];
#pragma unroll
      for (int q0 = 0; q0 < U; q0 += S::kBlock) {
        if (q0 >= ng) break;
        const uint32_t bm = S::kM == 1 ? bi : bi * S::kM + dm;
        const int db = bm % S::kD;
        // (The sums come after their unit's copies; the first wait is for the reads of those.)
        if (q0 == 0) ok = mbar_wait_lean(&s_full[st], (it / S::kStages) & 1, &s_abort);
        ok = __all_sync(0xffffffffu, ok && mbar_wait_lean(&s_dfull[db], (bm / S::kD) & 1, &s_abort));
        if (!ok) break;
        tc_fence_after();
        if (q0 == 0) read_pairs<U>(smem + st * S::kStage + S::kAtPairs, (S::kM == 1 ? 0 : dm * kOut) + t, now);
#pragma unroll
        for (int q = q0; q < q0 + S::kBlock; ++q) {
          if (q >= ng) break;
          const float s = int4::pair_of(now[q]).x;
          const F2 ss = f2(s, s);
          const uint32_t from = tlane + S::kColD + (db * S::kBlock + q - q0) * S::kRows + r_lo;
#pragma unroll
          for (int k = 0; k < S::kHalfRows; k += S::kChunk) {
            if (k >= my_rows) break;
            uint32_t y[S::kChunk];
#pragma unroll
            for (int j = 0; j < S::kChunk; j += 8) tmem_ld8(from + k + j, y + j);  // (columns past the tile's rows: unused)
            tmem_wait_ld();
#pragma unroll
            for (int e = 0; e < S::kChunk; e += 2)
              sum[(k + e) / 2] = f2_fma(f2(__uint_as_float(y[e]), __uint_as_float(y[e + 1])), ss, sum[(k + e) / 2]);
          }
        }
        tc_fence_before();
        __syncwarp();
        if (lane == 0) {
          mbar_arrive(&s_dfree[db]);
          if (q0 == 0) mbar_arrive(&s_empty[st]);
        }
        ++bi;
      }
    }
  }
  if (!ok && lane == 0) atomicOr(p.status, SPADE_DEV_TIMEOUT);

  const int rows = min(p.tile_rows, p.R - n0);
  const bool drains = warp >= S::kWarpDrain && warp < S::kWarpUnpack;
  if (S::kM == 2 || split == 1) {
    const int o = o0 + dm * kOut + t;
    if (drains && o < p.N) {
#pragma unroll
      for (int r = 0; r < S::kHalfRows; ++r) {
        if (r >= my_rows || r_lo + r >= rows) break;
        float y[2];
        f2_split(sum[r / 2], y[0], y[1]);
        const int64_t at = static_cast<int64_t>(n0 + r_lo + r) * p.N + o;
        p.out[at] = __float2bfloat16_rn(y[r & 1] + (p.residual ? __bfloat162float(p.residual[at]) : 0.f));
      }
    }
  } else {
    // Every CTA's sums into its own ring (all copies and MMAs of it are done: the draining
    // warps have seen the last one's), then rows dealt to the CTAs.
    float *sums = reinterpret_cast<float *>(smem);
    __syncthreads();
    if (drains) {
#pragma unroll
      for (int r = 0; r < S::kHalfRows; r += 2) {
        if (r >= my_rows) break;
        float y[2];
        f2_split(sum[r / 2], y[0], y[1]);
        sums[(r_lo + r) * kOut + t] = y[0];
        sums[(r_lo + r + 1) * kOut + t] = y[1];
      }
    }
    __syncwarp();
    cluster_sync();
    const int r0 = rows * rank / split, r1 = rows * (rank + 1) / split;
    for (int e = threadIdx.x; e < (r1 - r0) * (kOut / 4); e += S::kThreads) {
      const int r = r0 + e / (kOut / 4), o = e % (kOut / 4) * 4;
      float y[4] = {};
      for (int c = 0; c < split; ++c) {
        float v[4];
        asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];"
                     : "=f"(v[0]), "=f"(v[1]), "=f"(v[2]), "=f"(v[3])
                     : "r"(cluster_map(sums + r * kOut + o, c)));
#pragma unroll
        for (int k = 0; k < 4; ++k) y[k] += v[k];
      }
      const int64_t at = static_cast<int64_t>(n0 + r) * p.N + o0 + o;
#pragma unroll
      for (int k = 0; k < 4; ++k)
        if (o0 + o + k < p.N)
          p.out[at + k] = __float2bfloat16_rn(y[k] + (p.residual ? __bfloat162float(p.residual[at + k]) : 0.f));
    }
    __syncwarp();
    cluster_sync();  // no CTA leaves while another reads its sums
  }
  tc_fence_before();
  __syncthreads();
  if (warp == 1) {
    tc_fence_after();
    tmem_dealloc(tmem, S::kTmemCols);
  }
}

}  // namespace tc

template <int G>
static cudaError_t few_rows(Params p, int sms, cudaStream_t s) {
  using F = Few<G>;
  static OncePerDevice once;
  const cudaError_t e = set_max_smem(once, F::kRings + kHold * F::kSums, few_rows_kernel<G>);
  if (e != cudaSuccess) return e;
  const int tiles = (p.N - 1) / kTile + 1, spans = (p.K - 1) / kSpan + 1;
  const int grid = tiles < sms ? tiles : sms, most = (tiles - 1) / grid + 1;  // tiles of a CTA
  // Warps along K: as many as have a span; with a single tile all of them share it anyway.
  p.split = kWarps;
  while (p.split / 2 >= spans) p.split /= 2;
  const int each = (most - 1) / (kWarps / p.split) + 1;  // tiles of a warp
  return launch(few_rows_kernel<G>, dim3(grid), 1, kThreads, F::kRings + (each < kHold ? each : kHold) * F::kSums, s, p);
}

template <int G, bool kWide, int kTiles>
static cudaError_t rows(const Params &p, const CUtensorMap &w, const CUtensorMap &x, cudaStream_t s) {
  using S = tc::Shape<G, kWide, kTiles>;
  static OncePerDevice once;
  const cudaError_t e = set_max_smem(once, S::kBytes, tc::rows_kernel<G, kWide, kTiles>);
  if (e != cudaSuccess) return e;
  const unsigned tiles = (static_cast<unsigned>(p.N) - 1) / (S::kM * tc::kOut) + 1;
  const dim3 grid(tiles * p.split, (p.R + p.tile_rows - 1) / p.tile_rows);
  return launch(tc::rows_kernel<G, kWide, kTiles>, grid, p.split, S::kThreads, S::kBytes, s, p, w, x);
}

// How the work is dealt out: CTAs that share a tile's units, and what the slowest of
// `slots` CTAs at a time then takes, in units of one: its units and eight more (its start, its
// first copies, its sums).
struct Deal {
  int split;
  int64_t cost;
};
static Deal deal(int64_t tiles, int units, int slots) {
  constexpr int kFixed = 8;
  Deal best = {1, INT64_MAX};
  for (int s = 1; s <= tc::kMaxSplit && (s == 1 || units >= 4 * s); s *= 2) {  // (four units each at least)
    const int64_t c = ((tiles * s - 1) / slots + 1) * ((units - 1) / s + 1 + kFixed);
    if (c < best.cost) best = {s, c};
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
  p.R = R; p.N = N; p.K = K; p.tile_rows = p.tile_n = R; p.split = 1;
  cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
  CUtensorMap w;
  cudaError_t e;
  if (R <= w4::kRows) {
    e = group == 128 ? w4::few_rows<128>(p, sms, s)
        : group == 64 ? w4::few_rows<64>(p, sms, s)
                      : w4::few_rows<32>(p, sms, s);
  } else {
    const bool wide = R > w4::tc::kNarrow;
    const int most = wide ? w4::tc::kMost : w4::tc::kNarrow;
    int row_tiles = (R - 1) / most + 1;
    if (row_tiles > 65535) return fail(SPADE_ERR_SHAPE, "spade_linear_w4: R = %d exceeds %d rows per call", R, 65535 * most);
    const int units = (K - 1) / w4::kUnit + 1, slots = wide ? sms : 2 * sms;
    const int64_t outs = (N - 1) / w4::tc::kOut + 1, pairs = (N - 1) / (2 * w4::tc::kOut) + 1;
    // Two tiles of outputs to a CTA where the work fills the GPU without a split and few sums
    // are drained: 389 rows of 7168 x 5120 (in four tiles of rows) take 43.9 us against 48.5, 1024 rows of 12288 x 4096
    // 112 against 129; with a split 64 rows of 4096 x 4096 take 21.0 against 9.7; at group 32
    // (389 rows) 101 against 76.
    const bool pair = wide && group == 128 && w4::deal(pairs * row_tiles, units, sms).split == 1;
    if (wide) {
      // More row tiles than the fewest where SMs would idle: a unit takes as long as 300
      // rows' worth of its own and its rows (rounded up to 16).  The 389 rows in five
      // tiles of 80: 39.6 us against 43.5.
      const int fewest = row_tiles;
      int64_t cost = INT64_MAX;
      for (int t = fewest; t <= fewest + 2 && t <= 65535; ++t) {
        const w4::Deal d = w4::deal((pair ? pairs : outs) * t, units, slots);
        const int64_t c = d.cost * (300 + ((R - 1) / t + 16) / 16 * 16);
        if (c < cost && (!pair || d.split == 1)) {
          cost = c;
          row_tiles = t;
        }
      }
    }
    p.tile_rows = (R - 1) / row_tiles + 1;
    p.tile_n = (p.tile_rows + 15) / 16 * 16;
    p.split = pair ? 1 : w4::deal(outs * row_tiles, units, slots).split;
    CUtensorMap xm;
    if (!encode_tmap_bytes(&w, codes, K / 2, N, w4::tc::kOut, 64) ||
        !encode_tmap_bf16_sw128(&xm, x, K, R, static_cast<uint64_t>(K) * 2, 64, p.tile_n))
      return SPADE_ERR_CUDA;
    if (pair)
      e = w4::rows<128, true, 2>(p, w, xm, s);
    else if (wide)
      e = group == 128 ? w4::rows<128, true, 1>(p, w, xm, s)
          : group == 64 ? w4::rows<64, true, 1>(p, w, xm, s)
                        : w4::rows<32, true, 1>(p, w, xm, s);
    else
      e = group == 128 ? w4::rows<128, false, 1>(p, w, xm, s)
          : group == 64 ? w4::rows<64, false, 1>(p, w, xm, s)
                        : w4::rows<32, false, 1>(p, w, xm, s);
  }
  return e == cudaSuccess ? SPADE_OK : cuda_fail(e, "linear_w4 launch");
}
