// kv4_attention_tc.cu -- the verify attention over the paged 4-bit cache on the
// fifth-generation tensor cores: softmax(q K^T / sqrt D) V of the k_b+1 verify
// positions, causal inside the draft block (Sec. III-B "Verification Stage",
// Algorithm 1 cloud step), for head dims 64 and 128.
//
// The work is laid out as in verify_attention_tc.cu: units of (sequence, KV head,
// <= 64 query rows), a stream-K split over 64-key slices, keys on the MMA's M side
// (S^T[key][row] = K q^T and O^T[d][row] += V^T P^T), lazy rescaling, fp32 partials
// merged by log-sum-exp.  What the 4-bit cache changes:
//  * A key's codes minus its zero are whole numbers in -15 .. 15, exact in bf16, so
//    the scores' products are exact: S^T is accumulated once per group of 64 dims and
//    the softmax warps, whose lane is the key, apply the groups' scales in fp32.
//    No rounding of q or k enters.
//  * Those numbers are the MMA's A operand and go straight into tensor memory: a
//    thread unpacks one key (64 bytes of codes -> 64 columns of its lane), which
//    spares the write and the MMA's read of 32 KB of shared memory per 128 keys.
//  * V^T needs its rows across lanes, so values are unpacked to float16 (scale times
//    a whole number: one rounding, 2^-11) in shared memory, where the MMA reads them
//    MN-major.  P is float16 too: P = 2^(s - m + 7) with the lazy maximum keeps it
//    below 2^15, and what is 2^-32 of the largest weight or less is lost.
//  * Warp roles: warp 0 copies codes and pairs (TMA; 18 KB per 128 keys, four
//    stages, so that 18 KB stages cover the latency that 64 KB ones did), warp 1
//    issues the MMAs, warps 2-9 run the softmax and the epilogue, warps 10-13 unpack
//    keys, warps 14-17 values (96 registers a thread; the merge takes two rows at a
//    time to stay within them).
//  * Bound, at few rows, by a chunk's chain of latencies (copy, unpack, MMA, softmax, MMA
//    over two-stage buffers: 1800 cycles per 128 keys), at many by the softmax warps'
//    instructions (2500): 64 sequences of 0 to 8192 keys, 40 heads over 8, one row each,
//    102 us; four of 32768, 64 heads over 8, five rows each, 64 us.
//  * Slots that no row may see get P = 0 by their index and zero values, whatever
//    their scales hold.  A scale that is not finite in a slot that is seen (of the
//    key or the value) turns the slot's score into NaN and its values into zeros, so
//    the rows that see it, and no others, are NaN.
#include <cuda_fp16.h>

#include "attn_common.cuh"
#include "int4.cuh"
#include "kv4_attention.h"

namespace spade {
namespace attn {
namespace kv4 {

constexpr int kKeys = 128;                       // keys per MMA chunk (two slices)
constexpr int kRing = 4;                         // copy stages (chunks)
constexpr int kStages = 2;                       // unpacked keys, scores, values and weights
constexpr int kSoftWarps = 8;
constexpr int kSoftThreads = 32 * kSoftWarps;
constexpr int kWarpSoft = 2;                     // first softmax warp (after the copying and the MMA warp)
constexpr int kWarpK = kWarpSoft + kSoftWarps;   // four warps that unpack keys
constexpr int kWarpV = kWarpK + 4;               // four warps that unpack values
constexpr int kThreads = 32 * (kWarpV + 4);
constexpr int kCodes = kKeys * 64;               // codes of a chunk's keys (or values): 8 KB
constexpr int kPairs = kKeys * 8;                // their (scale, zero) pairs: 1 KB
constexpr int kStage = 2 * kCodes + 2 * kPairs;  // K codes, V codes, K pairs, V pairs
constexpr int kSlab = kKeys * 128;               // 64 dims of the chunk's values in fp16: 16 KB
constexpr int kTile = 2 * kSlab;
constexpr int kQSlab = kRowBlock * 128;          // 64 dims of Q in bf16: 8 KB
constexpr int kPBytes = kKeys * 128;             // P^T: [128 keys][64 rows] fp16
constexpr int kScaleSlots = 4;                   // chunks whose key scales are kept
constexpr float kPBias = 7.f;                    // log2 of the weight of a row's maximum ...
constexpr float kRescaleLog2 = 15.f;             // ... and of the largest weight before the maxima move

// What the copying warp says of a chunk: the first or the last of its segment; or
// that the CTA's range is done.
constexpr int kFirst = 1, kLast = 2, kEnd = 4;

// Tensor memory: S^T (two stages of a 64-column block per group), O^T, unpacked keys.
constexpr uint32_t kTmemCols = 512;
constexpr uint32_t kColS = 0, kColO = 256, kColK = 320;

// mbarriers.  The MMA warp issues S(j), PV(j-1), S(j+1), ... and a commit completes when
// every MMA before it has, so two commits per chunk say everything: SDone (S(j)) that
// the keys' columns of chunk j and, through PV(j-2) before it, the weights' buffer of
// chunk j-2 are free; PVDone (PV(j)) that the values' buffer is, and O^T complete.  The
// scores' buffer is free once the weights are written, which PV(j-2) waited for.  No
// phase can run two ahead of a waiter: each next one needs the waiter's own next arrival.
constexpr int kBarFull = 0, kBarEmpty = 4, kBarKFull = 8, kBarSDone = 10, kBarVFull = 12, kBarPVDone = 14,
              kBarPFull = 16, kBarScale = 18, kBarQ = 22, kBarDrain = 23, kNumBars = 24;

struct Smem {
  static constexpr int RING = 0;
  static constexpr int V = RING + kRing * kStage;           // [stage][2 slabs][128 keys][128 B]
  static constexpr int Q = V + kStages * kTile;             // [2 bufs][2 slabs][64 rows][128 B]
  static constexpr int P = Q + 4 * kQSlab;                  // [2 bufs][128 keys][128 B]
  static constexpr int SCALE = P + kStages * kPBytes;       // float2 [slot][128 keys]: the key's scales
  static constexpr int RMETA = SCALE + kScaleSlots * kKeys * 8;  // int2 [stage]: live keys of the chunk, its flags
  static constexpr int CMETA = RMETA + kRing * 8;           // int [slot]: flags
  static constexpr int PREF = round_up_c(CMETA + kScaleSlots * 4, 16);
  static constexpr int CTX = PREF + (kMaxB + 1) * 8;
  static constexpr int KD = CTX + kMaxB * 4;
  static constexpr int WRED = round_up_c(KD + kMaxB * 4, 128);
  static constexpr int ROWV = WRED + 4 * kRowBlock * 4;
  static constexpr int RMAX = ROWV + kRowBlock * 4;         // float [64 rows]: kPBias - running maximum
  static constexpr int ALPHA = RMAX + kRowBlock * 4;
  static constexpr int BAR = ALPHA + kRowBlock * 4;
  static constexpr int MISC = BAR + kNumBars * 8;           // abort, last, tmem base
  static constexpr int SEG0 = round_up_c(MISC + 16, 64);
  static constexpr int RANGE = SEG0 + 64;
  static constexpr int BYTES = RANGE + 64 + 1024;           // + slack for 1024-byte alignment
};
static_assert(Smem::V % 1024 == 0 && Smem::Q % 1024 == 0 && Smem::P % 1024 == 0 && kStage % 1024 == 0 && kCodes % 1024 == 0,
              "swizzled tiles need 1024-byte alignment");
static_assert(Smem::BAR % 8 == 0 && Smem::RMAX % 16 == 0 && Smem::SCALE % 16 == 0, "alignment");
static_assert(Smem::BYTES <= 227 * 1024, "shared memory budget");

SPADE_DEVICE bool finite_scale(uint32_t pair) { return (pair & 0x7c00u) != 0x7c00u; }

// The (scale, zero) pairs of key t: one per group of 64 dims.
template <int NG>
SPADE_DEVICE void load_pairs(const uint8_t *pairs, int t, uint32_t (&p)[NG]) {
  if constexpr (NG == 2) {
    const uint2 v = reinterpret_cast<const uint2 *>(pairs)[t];
    p[0] = v.x;
    p[1] = v.y;
  } else {
    p[0] = reinterpret_cast<const uint32_t *>(pairs)[t];
  }
}

// Piece j (16 bytes: 32 dims) of key t's codes, as the swizzled copy left it.
template <int D>
SPADE_DEVICE uint4 load_codes(const uint8_t *codes, int t, int j) {
  const int at = D == 128 ? j ^ ((t >> 1) & 3) : j ^ ((t >> 2) & 1);
  return *reinterpret_cast<const uint4 *>(codes + t * (D / 2) + at * 16);
}

template <int NR, int D>
__global__ void __launch_bounds__(kThreads, 1)
    verify_attention_kv4_kernel(const __grid_constant__ Params p, const __grid_constant__ CUtensorMap tm_kc,
                                const __grid_constant__ CUtensorMap tm_vc, const __grid_constant__ CUtensorMap tm_kp,
                                const __grid_constant__ CUtensorMap tm_vp) {
  static_assert(NR % 16 == 0 && NR >= 16 && NR <= kRowBlock, "MMA N must be 16..64, step 16");
  static_assert(D == 64 || D == 128, "head dim 64 or 128");
  constexpr int NG = D / 64;  // groups of a head
  extern __shared__ uint8_t smem_raw[];
  uint8_t *smem = smem_raw + ((1024u - (smem_u32(smem_raw) & 1023u)) & 1023u);
  int64_t *s_pref = reinterpret_cast<int64_t *>(smem + Smem::PREF);
  int32_t *s_ctx = reinterpret_cast<int32_t *>(smem + Smem::CTX);
  int32_t *s_kd = reinterpret_cast<int32_t *>(smem + Smem::KD);
  float *s_wred = reinterpret_cast<float *>(smem + Smem::WRED);
  float *s_rowv = reinterpret_cast<float *>(smem + Smem::ROWV);
  float *s_rmax = reinterpret_cast<float *>(smem + Smem::RMAX);
  float *s_alpha = reinterpret_cast<float *>(smem + Smem::ALPHA);
  float2 *s_scale = reinterpret_cast<float2 *>(smem + Smem::SCALE);
  int2 *s_rmeta = reinterpret_cast<int2 *>(smem + Smem::RMETA);
  int *s_cmeta = reinterpret_cast<int *>(smem + Smem::CMETA);
  uint64_t *bars = reinterpret_cast<uint64_t *>(smem + Smem::BAR);
  volatile int *s_abort = reinterpret_cast<volatile int *>(smem + Smem::MISC);
  volatile int *s_last = s_abort + 1;
  uint32_t *s_tmem = reinterpret_cast<uint32_t *>(smem + Smem::MISC + 8);

  const int tid = threadIdx.x;
  const int warp = uniform_warp();
  const int lane = tid & 31;

  if (tid == 0) { *s_abort = 0; *s_last = 0; }
  // Set-up that reads no input overlaps the previous kernel in the stream.
  if (warp == 0 && lane < 2) {
    tma_prefetch_desc(lane ? &tm_vc : &tm_kc);
    tma_prefetch_desc(lane ? &tm_vp : &tm_kp);
  } else if (warp == 1) {
    if (lane == 0) {
      for (int s = 0; s < kRing; ++s) {
        mbar_init(&bars[kBarFull + s], 1);
        mbar_init(&bars[kBarEmpty + s], 8);   // the unpacking warps
      }
      for (int s = 0; s < kStages; ++s) {
        mbar_init(&bars[kBarKFull + s], 4);
        mbar_init(&bars[kBarSDone + s], 1);
        mbar_init(&bars[kBarVFull + s], 4);
        mbar_init(&bars[kBarPVDone + s], 1);
        mbar_init(&bars[kBarPFull + s], kSoftWarps);
      }
      for (int s = 0; s < kScaleSlots; ++s) mbar_init(&bars[kBarScale + s], 4);
      mbar_init(&bars[kBarQ], kSoftWarps);
      mbar_init(&bars[kBarDrain], 1);
      fence_mbar_init();
    }
    __syncwarp();
    tmem_alloc(s_tmem, kTmemCols);
    tmem_relinquish();
  }
  if constexpr (D == 64) {
    // The value tiles' second 64-dim slab: zeros for the whole launch (O^T keeps M = 128).
    for (int e = tid; e < kStages * (kSlab / 16); e += kThreads) {
      const int st = e / (kSlab / 16), o = e % (kSlab / 16);
      *reinterpret_cast<uint4 *>(smem + Smem::V + st * kTile + kSlab + o * 16) = make_uint4(0, 0, 0, 0);
    }
    fence_proxy_async_smem();
  }
  griddep_wait();
  griddep_launch_dependents();
  sched_validate(p, s_ctx, s_kd, tid, kThreads);
  tc_fence_before();
  block_sync();
  tc_fence_after();
  Sched sc;
  sc.pref = s_pref; sc.ctx = s_ctx; sc.kd = s_kd;
  sc.B = p.B; sc.Hkv = p.Hkv; sc.G = p.G; sc.RB = p.RB; sc.E = p.unit_cost; sc.num_ctas = p.num_ctas;
  SegInfo *s_seg0 = reinterpret_cast<SegInfo *>(smem + Smem::SEG0);
  CtaRange *s_range = reinterpret_cast<CtaRange *>(smem + Smem::RANGE);
  if (warp == 0) {
    sched_scan(p, sc, s_pref, lane);
    __syncwarp();
    Sched s0 = sc;
    s0.total = s_pref[p.B];
    s0.num_ctas = static_cast<int>(s0.total < p.num_ctas ? s0.total : p.num_ctas);
    CtaRange r;
    r.total = s0.total;
    r.num_ctas = s0.num_ctas;
    r.active = s0.total > 0 && static_cast<int>(blockIdx.x) < s0.num_ctas;
    r.x_begin = r.x_end = 0;
    SegInfo seg0{};
    if (r.active) {
      r.x_begin = div_nn(static_cast<int64_t>(blockIdx.x) * s0.total, s0.num_ctas);
      r.x_end = div_nn(static_cast<int64_t>(blockIdx.x + 1) * s0.total, s0.num_ctas);
      seg0 = next_seg_warp(s0, r.x_begin, r.x_end, lane);
    }
    if (lane == 0) {
      *s_range = r;
      *s_seg0 = seg0;
    }
  }
  block_sync();
  if (!s_range->active) {
    if (warp == 1) tmem_dealloc(*s_tmem, kTmemCols);
    return;
  }
  const uint32_t tmem = *s_tmem;
  const uint32_t smem_base = smem_u32(smem);

  if (warp == 0) {
    // ============================ producer: TMA ============================
    const bool leader = elect_one();
    const uint64_t pol = l2_policy_evict_first();
    sc.total = s_range->total;
    sc.num_ctas = s_range->num_ctas;
    const int64_t x_begin = s_range->x_begin, x_end = s_range->x_end;
    constexpr uint32_t kSliceBytes = 2 * kChunk * (D / 2) + 2 * kChunk * NG * 4;
    uint32_t st = 0, ph = 1, issued = 0;
    bool ok = true;
    for (int64_t x = x_begin; ok && x < x_end;) {
      const SegInfo si = x == x_begin ? *s_seg0 : next_seg_warp(sc, x, x_end, lane);
      const int n_here = uniform(si.n_here), nchunk = uniform(si.nchunk), ci = uniform(si.g.ci);
      if (n_here == 0) break;
      const int b = uniform(si.g.b), kvh = uniform(si.g.kvh);
      const int live = s_ctx[b] + s_kd[b] + 1;  // live slots of the sequence
      // Each slice lies in one page; the lanes look up 32 slices at once, one batch ahead (a
      // lookup per chunk held this warp for 600 cycles of its 1900).
      auto rows_of = [&](int slice) {
        return slice + lane < n_here ? paged_row(p, b, kvh, (ci + slice + lane) * kChunk) : 0;
      };
      int rows = rows_of(0), rows_next = 0;
      for (int c = 0; c < nchunk; ++c) {
        const int nsl = min(2, n_here - 2 * c);
        const int key0 = (ci + 2 * c) * kChunk;
        if (c % 16 == 0) {
          if (c) rows = rows_next;
          rows_next = rows_of(2 * c + 32);
        }
        const int row_a = __shfl_sync(0xffffffffu, rows, 2 * c % 32), row_b = __shfl_sync(0xffffffffu, rows, (2 * c + 1) % 32);
        uint8_t *stage = smem + Smem::RING + st * kStage;
        ok = warp_wait(&bars[kBarEmpty + st], ph, s_abort);
        if (!ok) break;
        if (leader) {
          s_rmeta[st] = make_int2(min(nsl * kChunk, live - key0), (c == 0 ? kFirst : 0) | (c == nchunk - 1 ? kLast : 0));
          mbar_arrive_expect_tx(&bars[kBarFull + st], nsl * kSliceBytes);
        }
        for (int i = 0; i < nsl; ++i) {
          const int row = i ? row_b : row_a;
          uint8_t *codes = stage + i * kChunk * (D / 2);
          uint8_t *pairs = stage + 2 * kCodes + i * kChunk * NG * 4;
          if (leader) {
            tma_load_2d(codes, &tm_kc, 0, row, &bars[kBarFull + st], pol);
            tma_load_2d(pairs, &tm_kp, 0, row / kChunk, &bars[kBarFull + st], pol);
            tma_load_2d(codes + kCodes, &tm_vc, 0, row, &bars[kBarFull + st], pol);
            tma_load_2d(pairs + kPairs, &tm_vp, 0, row / kChunk, &bars[kBarFull + st], pol);
          }
        }
        ++issued;
        if (++st == kRing) { st = 0; ph ^= 1u; }
      }
      x = si.seg_end;
    }
    if (ok) ok = warp_wait(&bars[kBarEmpty + st], ph, s_abort);
    if (ok && leader) {
      s_rmeta[st] = make_int2(0, kEnd);
      mbar_arrive(&bars[kBarFull + st]);
    }
    if (leader) {
      if (!ok) atomicOr(p.status, SPADE_DEV_TIMEOUT);
      // Every copy issued must land before the CTA's shared memory goes away, also where
      // another warp's wait expires once this one is done (else all have: the unpacking warps
      // waited for them).  The stage of kEnd was waited for above.
      const uint32_t left = ok ? kRing - 1 : kRing;
      for (uint32_t j = issued > left ? issued - left : 0; j < issued; ++j)
        mbar_wait_unabortable(&bars[kBarFull + j % kRing], (j / kRing) & 1);
    }
  } else if (warp == 1) {
    // ============================ MMA issuer ===============================
    constexpr uint32_t idesc_s = idesc_bf16_f32(128, NR);                          // A in tensor memory, K-major B
    constexpr uint32_t idesc_pv = idesc_f16_f32(128, NR) | (1u << 15) | (1u << 16);  // MN-major A, B
    const bool leader = elect_one();
    bool ok = true;
    uint32_t it = 0, seg = 0;
    auto wait = [&](int bar, uint32_t parity) {
      ok = __all_sync(0xffffffffu, mbar_wait_lean(&bars[bar], parity, s_abort)) && ok;
    };
    auto issue_pv = [&](uint32_t j, bool first) {
      const int st = j % kStages;
      const uint32_t ph = (j / kStages) & 1;
      // (A segment's first weights come after the epilogue of the one before has read O^T.)
      ok = __all_sync(0xffffffffu, mbar_wait_lean(&bars[kBarVFull + st], ph, s_abort) &&
                                       mbar_wait_lean(&bars[kBarPFull + st], ph, s_abort)) && ok;
      tc_fence_after();
      const uint64_t dv = desc_sw128(smem_base + Smem::V + st * kTile, kSlab, 1024);
      const uint64_t dp = desc_sw128(smem_base + Smem::P + st * kPBytes, kSlab, 1024);
#pragma unroll
      for (int kk = 0; kk < kKeys / 16; ++kk)
        if (leader) tc_mma_f16(tmem + kColO, dv + 128u * kk, dp + 128u * kk, idesc_pv, (first && kk == 0) ? 0u : 1u);
      if (leader) tc_commit(&bars[kBarPVDone + st]);
    };
    bool before_first = false;  // whether the chunk before was the first of its segment
    for (;;) {
      const int st = it % kStages;
      const uint32_t ph = (it / kStages) & 1;
      wait(kBarKFull + st, ph);
      if (!ok) break;
      const int flags = s_cmeta[it % kScaleSlots];
      if (flags & kEnd) break;
      const bool first = flags & kFirst;
      // The segment's Q is staged: its S products may start while the previous
      // segment's epilogue still reads O^T.
      if (first) wait(kBarQ, seg & 1);
      tc_fence_after();
      const uint64_t dq = desc_sw128(smem_base + Smem::Q + (seg & 1) * 2 * kQSlab, 16, 1024);
#pragma unroll
      for (int g = 0; g < NG; ++g) {
        const uint32_t d = tmem + kColS + static_cast<uint32_t>((st * NG + g) * 64);
#pragma unroll
        for (int kk = 0; kk < 4; ++kk) {
          const uint32_t a = tmem + kColK + static_cast<uint32_t>(st * (D / 2) + g * 32 + kk * 8);
          const uint32_t qo = (g * kQSlab + kk * 32) >> 4;  // in the descriptor's address field
          if (leader) tc_mma_f16_ta(d, a, dq + qo, idesc_s, kk > 0 ? 1u : 0u);
        }
      }
      if (leader) tc_commit(&bars[kBarSDone + st]);
      if (!first) issue_pv(it - 1, before_first);
      if (!ok) break;
      if (flags & kLast) {
        issue_pv(it, first);
        if (!ok) break;
        ++seg;
      }
      before_first = first;
      ++it;
    }
    if (leader) {
      if (!ok || *s_abort) atomicOr(p.status, SPADE_DEV_TIMEOUT);
      // Every MMA issued must be done before its operands and the tensor memory go away.
      tc_commit(&bars[kBarDrain]);
      mbar_wait_unabortable(&bars[kBarDrain], 0);
    }
  } else if (warp >= kWarpK) {
    // ==================== unpacking: a thread per key ======================
    const bool is_v = warp >= kWarpV;
    const int q4 = warp & 3;              // tensor-memory lane quadrant of this warp
    const int t = q4 * 32 + lane;         // key of the chunk
    uint32_t it = 0;
    bool ok = true;
    for (;; ++it) {
      const int rs = it % kRing, st = it % kStages;
      const uint32_t ph = (it / kStages) & 1;
      const uint8_t *stage = smem + Smem::RING + rs * kStage;
      ok = mbar_wait_lean(&bars[kBarFull + rs], (it / kRing) & 1, s_abort) &&
           mbar_wait_lean(&bars[(is_v ? kBarPVDone : kBarSDone) + st], ph ^ 1, s_abort);
      if (!__all_sync(0xffffffffu, ok)) {
        ok = false;
        break;
      }
      const int2 meta = s_rmeta[rs];
      if (!is_v && warp == kWarpK && lane == 0) s_cmeta[it % kScaleSlots] = meta.y;
      if (meta.y & kEnd) {
        __syncwarp();
        if (!is_v && lane == 0) mbar_arrive(&bars[kBarKFull + st]);  // the MMA warp reads the flags
        break;
      }
      uint32_t kp[NG], vp[NG];
      load_pairs<NG>(stage + 2 * kCodes + kPairs, t, vp);
      bool finite = true;
#pragma unroll
      for (int g = 0; g < NG; ++g) finite = finite && finite_scale(vp[g]);
      if (!is_v) {
        load_pairs<NG>(stage + 2 * kCodes, t, kp);
        tc_fence_after();  // S of the chunk two before has read these columns
#pragma unroll
        for (int j = 0; j < D / 32; ++j) {
          const uint4 v = load_codes<D>(stage, t, j);
          const __nv_bfloat162 nz = __float2bfloat162_rn(-128.f - int4::pair_of(kp[j / 2]).y);
          uint32_t a[16];
          int4::unpack_bf16(v.x, nz, a);
          int4::unpack_bf16(v.y, nz, a + 4);
          int4::unpack_bf16(v.z, nz, a + 8);
          int4::unpack_bf16(v.w, nz, a + 12);
          tmem_st16(tmem + (static_cast<uint32_t>(q4 * 32) << 16) + kColK + st * (D / 2) + j * 16, a);
        }
        // The scales that the scores take, in log2 units: NaN where the key's or the value's is not finite.
        // (One group: the second stays 0, see the scores.)
        float2 s = make_float2(0.f, 0.f);
        const float poison = finite ? p.scale_log2 : NAN;
        s.x = (finite_scale(kp[0]) ? int4::pair_of(kp[0]).x : NAN) * poison;
        if constexpr (NG == 2) s.y = (finite_scale(kp[1]) ? int4::pair_of(kp[1]).x : NAN) * poison;
        s_scale[(it % kScaleSlots) * kKeys + t] = s;
        tmem_wait_st();
        tc_fence_before();
        __syncwarp();
        if (lane == 0) {
          mbar_arrive(&bars[kBarKFull + st]);
          mbar_arrive(&bars[kBarScale + it % kScaleSlots]);
          mbar_arrive(&bars[kBarEmpty + rs]);
        }
      } else {
        // Slots that were not loaded or lie past the live ones are zeros.
        const bool real = finite && t < meta.x;
        uint8_t *row = smem + Smem::V + st * kTile + t * 128;
#pragma unroll
        for (int j = 0; j < D / 32; ++j) {
          const uint4 v = load_codes<D>(stage + kCodes, t, j);
          const float2 pair = real ? int4::pair_of(vp[j / 2]) : make_float2(0.f, 0.f);
          const __half2 s = __float2half2_rn(pair.x), nz = __float2half2_rn(-1024.f - pair.y);
          const __half2 nz16 = __float2half2_rn(-64.f - pair.y);
          const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            uint32_t h[4];
            int4::unpack_fp16(w[i], s, nz, nz16, h);
            *reinterpret_cast<uint4 *>(row + (j / 2) * kSlab + ((((j % 2) * 4 + i) ^ (t & 7)) << 4)) =
                make_uint4(h[0], h[1], h[2], h[3]);
          }
        }
        fence_proxy_async_smem();
        __syncwarp();
        if (lane == 0) {
          mbar_arrive(&bars[kBarVFull + st]);
          mbar_arrive(&bars[kBarEmpty + rs]);
        }
      }
    }
    if (!ok && lane == 0) atomicOr(p.status, SPADE_DEV_TIMEOUT);
  } else {
    // ===================== softmax and epilogue =============================
    constexpr int NH = NR / 2;             // rows (S^T / O^T columns) per softmax warp
    constexpr int NP = NH <= 8 ? 8 : (NH <= 16 ? 16 : 32);  // NH padded to a power of two
    const int q4 = warp & 3;
    const int half = (warp - kWarpSoft) >> 2;      // which half of the rows
    const int t = q4 * 32 + lane;          // key lane (softmax) / head-dim lane (epilogue)
    const int stid = tid - 32 * kWarpSoft; // 0..255
    const uint32_t tlane = tmem + (static_cast<uint32_t>(q4 * 32) << 16);
    const int c0 = half * NH;              // first row (column) of this warp
    bool expired = false;
    uint32_t it = 0, seg = 0;

    // Q of a segment into buffer qb: rows >= nrow zero-filled, 128-byte swizzle.
    auto prefetch_q = [&](const SegInfo &sq, int qb) {
      const int kdq = s_kd[sq.g.b];
      const int nrq = min(kRowBlock, p.G * (kdq + 1) - kRowBlock * sq.g.rb);
      const int qr0 = p.cu_q[sq.g.b];
      const uint32_t base = smem_base + Smem::Q + qb * 2 * kQSlab;
      for (int e = stid; e < NR * (D / 8); e += kSoftThreads) {
        const int r = e / (D / 8), c = e % (D / 8);
        const bool real = r < nrq;
        const __nv_bfloat16 *src = real ? p.q + out_row(p, qr0, sq.g.kvh, sq.g.rb, r) * D + c * 8 : p.q;
        cp_async16(base + (c >> 3) * kQSlab + r * 128 + (((c & 7) ^ (r & 7)) << 4), src, real ? 16u : 0u);
      }
    };

    sc.total = s_range->total;
    sc.num_ctas = s_range->num_ctas;
    const int64_t x_end = s_range->x_end;
    SegInfo si = *s_seg0;
    if (si.n_here > 0) prefetch_q(si, 0);
    cp_async_commit();
    for (int64_t x = s_range->x_begin; x < x_end && si.n_here > 0;) {
      const Seg g = si.g;
      const int ctx = s_ctx[g.b];
      const int kd = s_kd[g.b];
      const int nrow = min(kRowBlock, p.G * (kd + 1) - kRowBlock * g.rb);
      const int q_row0 = p.cu_q[g.b];
      const int hi = nrow - c0;            // rows r < hi of this warp are real
      // Rows past nrow (zeros in Q, never stored) keep a maximum of 0, so that only keys
      // need masks.
      if (stid < kRowBlock) s_rmax[stid] = stid < nrow ? INFINITY : 0.f;
      cp_async_wait<0>();  // this segment's Q has landed
      fence_proxy_async_smem();
      named_bar(1, kSoftThreads);
      __syncwarp();
      if (lane == 0 && seg == 0) mbar_arrive(&bars[kBarQ]);
      SegInfo si_next = si;
      si_next.n_here = 0;
      if (si.seg_end < x_end) {
        si_next = next_seg(sc, si.seg_end, x_end);
        if (si_next.n_here > 0) prefetch_q(si_next, (seg + 1) & 1);
      }
      cp_async_commit();

      float x_[NP];
      F2 l2[NH / 2];  // row sums of this key lane, rows in pairs
#pragma unroll
      for (int r = 0; r < NH / 2; ++r) l2[r] = f2(0.f, 0.f);
      for (int c = 0; c < si.nchunk; ++c, ++it) {
        const int st = it % kStages;
        const uint32_t ph = (it / kStages) & 1;
        const int key0 = (g.ci + 2 * c) * kChunk;
        const int nk = min(2, si.n_here - 2 * c) * kChunk;
        const int kg = key0 + t;
        // Row R = 64 rb + rr (position R / G) sees key kg iff R >= (kg - ctx) G (every row where
        // kg <= ctx: far behind it the product would pass 32 bits).
        const int lo = (t < nk) ? max(kg - ctx, 0) * p.G - kRowBlock * g.rb - c0 : NH;
        const bool masked = __any_sync(0xffffffffu, lo > 0);  // (the last keys of a sequence or segment)
        const uint32_t taddr = tlane + kColS + st * NG * 64 + c0;

        // Scores of this key lane relative to `off` (one per row), in log2 units: the groups'
        // sums under their scales.
        expired = expired || !mbar_wait_lean(&bars[kBarScale + it % kScaleSlots], (it / kScaleSlots) & 1, s_abort);
        const float2 sk = s_scale[(it % kScaleSlots) * kKeys + t];
        auto load_scores = [&](const float *off) {
#pragma unroll
          for (int r0 = 0; r0 < NH; r0 += 16) {  // 16 rows at a time: registers
            constexpr int kMost = NH < 16 ? NH : 16;
            uint32_t y[NG][kMost];
#pragma unroll
            for (int g2 = 0; g2 < NG; ++g2)
#pragma unroll
              for (int j = 0; j < kMost && r0 + j < NH; j += 8) tmem_ld8(taddr + g2 * 64 + r0 + j, y[g2] + j);
            tmem_wait_ld();
#pragma unroll
            for (int j = 0; j < kMost && r0 + j < NH; j += 4) {
              const float4 mv = off ? *reinterpret_cast<const float4 *>(off + r0 + j)
                                    : make_float4(-kPBias, -kPBias, -kPBias, -kPBias);
#pragma unroll
              for (int e = 0; e < 4; e += 2) {
                // -m = inf (no visible key yet) gives inf for a visible score: a vote.
                // (The score is rounded before the maximum is taken off, as where it was found:
                // the largest one's weight is 2^kPBias whatever the scores' size.  With one group
                // the product is taken as a sum with 0, sk.y, which keeps it apart from the sum
                // that follows: fused, scores past 2^28 gave weights past float16.)
                const F2 s0 = f2(__uint_as_float(y[0][j + e]), __uint_as_float(y[0][j + e + 1])), k0 = f2(sk.x, sk.x);
                F2 s;
                if constexpr (NG == 2)
                  s = f2_fma(f2(__uint_as_float(y[NG - 1][j + e]), __uint_as_float(y[NG - 1][j + e + 1])),
                             f2(sk.y, sk.y), f2_mul(s0, k0));
                else
                  s = f2_fma(s0, k0, f2(sk.y, sk.y));
                s = f2_add(s, e ? f2(mv.z, mv.w) : f2(mv.x, mv.y));
                f2_split(s, x_[r0 + j + e], x_[r0 + j + e + 1]);
              }
            }
          }
          if (masked) {
#pragma unroll
            for (int r = 0; r < NH; ++r) x_[r] = r < lo ? -INFINITY : x_[r];
          }
        };
        expired = expired || !mbar_wait_lean(&bars[kBarSDone + st], ph, s_abort);
        __syncwarp();
        tc_fence_after();
        load_scores(s_rmax + c0);
        float high = fmaxf(x_[0], x_[1]);
#pragma unroll
        for (int r = 2; r < NH; r += 2) high = max3(high, x_[r], x_[r + 1]);
        // The two halves own disjoint rows: each votes and rescales on its own barriers.
        if (bar_any(2 + half, kSoftThreads / 2, high > kRescaleLog2)) {
          // Some weight would pass 2^15 (always so in a unit's first chunk): take this
          // chunk's exact row maxima.  (S^T is reused only after this chunk's P is signalled.)
          load_scores(nullptr);
#pragma unroll
          for (int r = NH; r < NP; ++r) x_[r] = -INFINITY;
          {
            const float wm = warp_reduce_scatter<NP, true>(x_, lane);
            if (lane < NH) s_wred[q4 * kRowBlock + c0 + lane] = wm;
          }
          named_bar(4 + half, kSoftThreads / 2);
          const int hs = stid - half * (kSoftThreads / 2);
          if (hs < NH) {
            const int row = c0 + hs;
            const float mo = -s_rmax[row];
            const float mn = fmaxf(fmaxf(mo, fmaxf(s_wred[row], s_wred[kRowBlock + row])),
                                   fmaxf(s_wred[2 * kRowBlock + row], s_wred[3 * kRowBlock + row]));
            s_alpha[row] = mn > mo ? ex2(mo - mn) : 1.f;  // mo = -inf gives 0: nothing to keep
            s_rmax[row] = -mn;
          }
          named_bar(4 + half, kSoftThreads / 2);
#pragma unroll
          for (int r = 0; r < NH / 2; ++r) l2[r] = f2_mul(l2[r], f2(s_alpha[c0 + 2 * r], s_alpha[c0 + 2 * r + 1]));
          if (c > 0) {
            // O^T's columns are rescaled once the last PV has landed.
            if (!mbar_wait(&bars[kBarPVDone + (it - 1) % kStages], ((it - 1) / kStages) & 1, s_abort)) expired = true;
            tc_fence_after();
#pragma unroll
            for (int j = 0; j < NH / 8; ++j) {
              uint32_t o8[8];
              tmem_ld8(tlane + kColO + c0 + j * 8, o8);
              tmem_wait_ld();
#pragma unroll
              for (int e = 0; e < 8; ++e)
                o8[e] = __float_as_uint(__uint_as_float(o8[e]) * s_alpha[c0 + j * 8 + e]);
              tmem_st8(tlane + kColO + c0 + j * 8, o8);
            }
            tmem_wait_st();
          }
          load_scores(s_rmax + c0);
        }

        // ---- P^T row of this key (this warp's rows): fp16, 128-byte swizzle ----
        uint8_t *prow = smem + Smem::P + st * kPBytes + t * 128;
#pragma unroll
        for (int j = 0; j < NH / 8; ++j) {
          uint32_t w[4];
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const int r0 = j * 8 + 2 * e;
            const float p0 = ex2(x_[r0]), p1 = ex2(x_[r0 + 1]);
            l2[r0 / 2] = f2_add(l2[r0 / 2], f2(p0, p1));
            const __half2 h = __floats2half2_rn(p0, p1);
            w[e] = *reinterpret_cast<const uint32_t *>(&h);
          }
          *reinterpret_cast<uint4 *>(prow + (((c0 / 8 + j) ^ (t & 7)) << 4)) = make_uint4(w[0], w[1], w[2], w[3]);
        }
        fence_proxy_async_smem();
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(&bars[kBarPFull + st]);
      }
      // The next segment's Q lets the MMA warp start its S products during this epilogue.
      if (si_next.n_here > 0) {
        cp_async_wait<0>();
        fence_proxy_async_smem();
        named_bar(1, kSoftThreads);
        __syncwarp();
        if (lane == 0) mbar_arrive(&bars[kBarQ]);
      }

      // ---- epilogue: row sums, O^T from tensor memory, output or partial ----
      const bool row_writer = q4 == 0 && lane < NH && lane < hi;
      const float m_own = row_writer ? -s_rmax[c0 + lane] : 0.f;
      float l[NH];
      {
        float v[NP];
#pragma unroll
        for (int r = 0; r < NP; r += 2) {
          v[r] = v[r + 1] = 0.f;
          if (r < NH) f2_split(l2[r / 2], v[r], v[r + 1]);
        }
        const float ws = warp_reduce_scatter<NP, false>(v, lane);
        if (lane < NH) s_wred[q4 * kRowBlock + c0 + lane] = ws;
      }
      named_bar(1, kSoftThreads);
      if (stid < NR)
        s_rowv[stid] = (s_wred[stid] + s_wred[kRowBlock + stid]) +
                       (s_wred[2 * kRowBlock + stid] + s_wred[3 * kRowBlock + stid]);
      named_bar(1, kSoftThreads);
#pragma unroll
      for (int r = 0; r < NH; ++r) l[r] = s_rowv[c0 + r];
      const float l_own = row_writer ? s_rowv[c0 + lane] : 1.f;
      const int unit = (g.b * p.Hkv + g.kvh) * p.RB + g.rb;
      const int64_t c_first = sc.owner(g.ust + sc.E);
      const int64_t c_last = sc.owner(g.ust + sc.E + g.nch - 1);
      const int nparts = static_cast<int>(c_last - c_first + 1);
      if (!mbar_wait(&bars[kBarPVDone + (it - 1) % kStages], ((it - 1) / kStages) & 1, s_abort)) expired = true;
      tc_fence_after();
      if (nparts == 1) {
        const int row0 = kRowBlock * g.rb + c0;
        int gh = row0 % p.G;
        size_t orow = static_cast<size_t>(q_row0 + row0 / p.G) * p.Hq + g.kvh * p.G + gh;
#pragma unroll
        for (int j = 0; j < NH / 8; ++j) {
          uint32_t o8[8];
          tmem_ld8(tlane + kColO + c0 + j * 8, o8);
          tmem_wait_ld();
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            // l >= 2^7 (the row maximum's own term, but for rounding) and far from 2^126:
            // the fast divide is good to a few fp32 ulps.
            if (j * 8 + e < hi && t < D)
              p.out[orow * D + t] = __float2bfloat16_rn(__fdividef(__uint_as_float(o8[e]), l[j * 8 + e]));
            if (++gh == p.G) {
              gh = 0;
              orow += p.Hq - p.G + 1;
            } else {
              ++orow;
            }
          }
        }
        tc_fence_before();
        if (p.lse && row_writer)
          p.lse[out_row(p, q_row0, g.kvh, g.rb, c0 + lane)] = (m_own + log2f(l_own)) * 0.69314718055994531f;
      } else {
        const int64_t slot = blockIdx.x + unit;
        float *part = p.partials + slot * slot_floats(D);
#pragma unroll
        for (int j = 0; j < NH / 8; ++j) {
          uint32_t o8[8];
          tmem_ld8(tlane + kColO + c0 + j * 8, o8);
          tmem_wait_ld();
#pragma unroll
          for (int e = 0; e < 8; ++e)
            if (j * 8 + e < hi && t < D) __stcg(part + (c0 + j * 8 + e) * D + t, __uint_as_float(o8[e]));
        }
        tc_fence_before();
        if (row_writer) {
          __stcg(part + kRowBlock * D + c0 + lane, m_own);
          __stcg(part + kRowBlock * D + kRowBlock + c0 + lane, l_own);
        }
        named_bar(1, kSoftThreads);
        // (Of the units whose slices begin in a CTA's range only the last goes on in another's.)
        if (stid == 0) *s_last = arrive_part(&p.counters[c_first], nparts);
        named_bar(1, kSoftThreads);
        if (*s_last) {
          static_assert(kSoftWarps == kMergeWarps, "the softmax warps merge");
          merge_partials<D, 2>(p, c_first + unit, nparts, nrow, g.rb, g.kvh, q_row0, s_wred, stid, warp - kWarpSoft, lane);
          if (stid == 0) p.counters[c_first] = 0;  // every part has arrived: reset for the next call
        }
      }
      ++seg;
      x = si.seg_end;
      si = si_next;
    }
    cp_async_wait<0>();
    if (expired) atomicOr(p.status, SPADE_DEV_TIMEOUT);
  }

  tc_fence_before();
  block_sync();
  if (warp == 1) {
    tc_fence_after();
    tmem_dealloc(tmem, kTmemCols);
  }
}

template <int NR, int D>
static cudaError_t launch_nr(const Params &p, const CUtensorMap &kc, const CUtensorMap &vc, const CUtensorMap &kp,
                             const CUtensorMap &vp, cudaStream_t stream) {
  auto kern = verify_attention_kv4_kernel<NR, D>;
  static OncePerDevice once;
  const cudaError_t e = set_max_smem(once, Smem::BYTES, kern);
  if (e != cudaSuccess) return e;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(p.num_ctas);
  cfg.blockDim = dim3(kThreads);
  cfg.dynamicSmemBytes = Smem::BYTES;
  cfg.stream = stream;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, kern, p, kc, vc, kp, vp);
}

}  // namespace kv4

cudaError_t launch_kv4(const Params &p, const CUtensorMap &kc, const CUtensorMap &vc, const CUtensorMap &kp,
                       const CUtensorMap &vp, int nr, int d, cudaStream_t stream) {
  if (d == 64) {
    switch (nr) {
      case 16: return kv4::launch_nr<16, 64>(p, kc, vc, kp, vp, stream);
      case 32: return kv4::launch_nr<32, 64>(p, kc, vc, kp, vp, stream);
      case 48: return kv4::launch_nr<48, 64>(p, kc, vc, kp, vp, stream);
      default: return kv4::launch_nr<64, 64>(p, kc, vc, kp, vp, stream);
    }
  }
  switch (nr) {
    case 16: return kv4::launch_nr<16, 128>(p, kc, vc, kp, vp, stream);
    case 32: return kv4::launch_nr<32, 128>(p, kc, vc, kp, vp, stream);
    case 48: return kv4::launch_nr<48, 128>(p, kc, vc, kp, vp, stream);
    default: return kv4::launch_nr<64, 128>(p, kc, vc, kp, vp, stream);
  }
}

}  // namespace attn
}  // namespace spade
