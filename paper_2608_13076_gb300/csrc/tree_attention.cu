// tree_attention.cu -- verify attention whose blocks are trees of drafts: every node of a sequence's block
// against the committed context and the nodes that its mask names (Sec. III-B "Verification Stage",
// Algorithm 1 cloud step, with a draft block that branches).
//
// Trees have many rows to a KV head (64 nodes x 4 query heads: 256), so rows are on the MMA M side here:
//   S = Q K^T, M = 128 rows, N = 128 keys; softmax by two threads a row; O += P V with P from tensor memory.
//  * A unit is (sequence, KV head, up to 256 rows): two tiles of whole nodes x the head group's rows.
//    Two streams of softmax warps (eight each: a thread has a row's scores for half of a chunk's keys) alternate
//    with the tensor core: a unit of two tiles gives each stream a tile and every key, a unit of one tile gives both
//    the same rows and every other chunk of 128 keys (their sums are joined in the epilogue).  So a step j of
//    a segment belongs to stream j % 2, and the issue order is PV(j), S(j + 2).
//  * Tensor memory: S of each stream (128 columns; P, packed to bf16, takes the first 64 of them over) and O of
//    each stream (D columns).  S(j + 2) follows PV(j), which reads P, in the same in-order pipe.
//  * K and V tiles by TMA, two stages each.  A warp goes over every V tile that reaches into the block before
//    its product: rows past the live cache (or not loaded) become zeros, and rows of the block with a value that
//    is not finite too (those that see them are made NaN in the epilogue, noted a step later: the scores do not wait
//    for the values), as 0 times NaN would reach rows that do not see them.
//  * Lazy rescaling: a row's maximum moves only when a score exceeds it by more than 2^8 (a vote of the row's two
//    warps); those then rescale their own lanes of O (their stream's last PV is done when S is).
//  * The chunks of all units lie end to end and are cut into one equal range per SM (every unit also carries
//    kUnitCost virtual chunks, its start and end); parts of a unit are merged by log-sum-exp, in the order of the
//    parts, by the CTA that finishes last, straight from its tensor memory.  (A part that is finished draws a
//    number; the last one waits for those before it to be written.  What those still wait for is their own CTA's
//    products at most, which wait for no other CTA, so the wait ends.)
//    More than kMany parts are written, added up in groups by as many CTAs, and then the groups (nothing waits there).
// Measured (bf16, back to back; D = 128): 8 x 64 nodes x 4 heads over 4096 slots 45 us (its keys and values once: 21),
// 64 ragged ones over 0 .. 8192 slots 214 (163), 2 x 512 nodes x 8 heads over 16384 410-417 (386 in runs of a few
// milliseconds, where the clock is higher; products at the tensor rate: 292).
// Long contexts of few nodes are bound by HBM; many rows by a stream's chain: scores from tensor memory, maximum, 64
// powers and their packing a thread, about 1650 cycles for a tile step, against 1070 of the products; few chunks by
// the start and the end of a unit, whose code is fetched anew each time.
#include "attn_common.cuh"
#include "launch.h"

namespace spade {
namespace attn_tree {

using attn::block_sync;
using attn::desc_sw128;
using attn::named_bar;
using attn::paged_row;

constexpr int kKeys = 128;                    // keys per chunk
constexpr int kRows = 128;                    // rows per tile
constexpr int kStages = 2;                    // K and V ring depth
constexpr int kBadRing = 4;                   // chunks whose words of values that are not finite are held
constexpr int kThreads = 640;                 // K, MMA, cleaning, V warps; two streams of eight softmax warps
constexpr int kSlab = 128 * 128;              // 64 dims of 128 keys or rows
constexpr int kTile = 2 * kSlab;
constexpr uint32_t kTmemCols = 512;
constexpr uint32_t kColS = 0, kColO = 256;    // + 128 per stream
constexpr float kRescaleLog2 = 8.f;
constexpr int kUnitCost = 4;                  // virtual chunks at a unit's start
constexpr int kMinRange = 5;                  // least range of a CTA, where units are split
constexpr int kMany = 8;                      // parts of a unit that one CTA merges; of more, groups are merged first
constexpr int kMaxB = attn::kMaxB;

struct Params {
  __nv_bfloat16 *out;
  float *lse;
  const int32_t *ctx_lens, *n_draft, *cu_q, *mask;
  int32_t *counters;  // [num_ctas][2 tiles]{parts finished, parts written} of the split unit that begins in a CTA's range
  int32_t *groups;    // [num_ctas][2 segments][2 tiles]: the parts that a group has.  Zero between calls, as the counters are
  float *partials;    // [num_ctas][2 segments][2 tiles][part_floats(D)]
  int32_t *status;
  const int32_t *block_table;  // null: dense
  int B, Hq, Hkv, G, cap, max_k, R, words;
  int tile_nodes;     // nodes of a tile: 128 / G
  int num_ctas;
  int page_size, max_pages, num_pages;
  float scale_log2;
};

// A tile's part: O [D / 4][128 rows] float4, then m and l.
__host__ __device__ constexpr int part_floats(int D) { return kRows * D + 2 * kRows; }

constexpr int kBarKFull = 0, kBarKEmpty = 2, kBarVFull = 4, kBarVReady = 6, kBarVEmpty = 8, kBarSFull = 10, kBarPFull = 12,
              kBarOFinal = 14, kBarOFree = 16, kBarQFull = 18, kBarQFree = 20, kBarPHalf = 21, kBarDrain = 23, kBarBad = 24, kBarStart = kBarBad + kBadRing,
              kNumBars = kBarStart + 1;

// A CTA's range of the cost space: of `num_ctas` ranges the first `longer` are one longer than `size`.
struct Range {
  int x_begin, x_end, total, num_ctas, size, longer, active;
};
// Part of a unit's chunks in a CTA's range.
struct Seg {
  int b, kvh, group;   // group: which 2 * tile_nodes of the sequence's nodes
  int c0, n;           // chunks
  int nch;             // of the unit
  int ust, end;        // cost positions: the unit's start, the segment's end
};

struct Smem {
  static constexpr int K = 0;
  static constexpr int V = K + kStages * kTile;
  static constexpr int Q = V + kStages * kTile;             // two tiles
  static constexpr int X = Q + 2 * kTile;                   // [8 warps][16 columns][32 lanes] floats: stream 1's O to stream 0
  static constexpr int ML = X + 8 * 2048;                   // [2 streams][2 halves][128 rows] floats: maxima, sums
  static constexpr int M1 = ML + 4 * kRows * 4;             // stream 1's m and l: [2][128] floats
  static constexpr int PREF = M1 + 2 * kRows * 4;           // int32 [kMaxB + 2]
  static constexpr int CTX = PREF + (kMaxB + 2) * 4;
  static constexpr int KD = CTX + kMaxB * 4;
  static constexpr int Q0 = KD + kMaxB * 4;                 // int32 [kMaxB]: first rows
  static constexpr int BAR = (Q0 + kMaxB * 4 + 7) / 8 * 8;
  static constexpr int BAD = BAR + kNumBars * 8;            // uint32 [kBadRing][4]: rows of V that are not finite
  static constexpr int MISC = BAD + kBadRing * 16;          // abort, last (2), tensor-memory base
  static constexpr int RANGE = MISC + 16;
  static constexpr int BYTES = RANGE + 64 + 1024;           // + slack for 1024-byte alignment
};
static_assert(Smem::RANGE % 8 == 0 && Smem::BAR % 8 == 0, "alignment");
static_assert(Smem::BYTES <= 227 * 1024, "shared memory");

SPADE_DEVICE void tmem_ld32(uint32_t taddr, uint32_t *r) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
      "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]),
        "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]),
        "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]),
        "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
      : "r"(taddr));
}

// tmem_wait_ld for 32 loaded registers, which nothing uses before it.
SPADE_DEVICE void tmem_wait_ld32(uint32_t *r) {
  asm volatile("tcgen05.wait::ld.sync.aligned;"
               : "+r"(r[0]), "+r"(r[1]), "+r"(r[2]), "+r"(r[3]), "+r"(r[4]), "+r"(r[5]), "+r"(r[6]), "+r"(r[7]),
                 "+r"(r[8]), "+r"(r[9]), "+r"(r[10]), "+r"(r[11]), "+r"(r[12]), "+r"(r[13]), "+r"(r[14]), "+r"(r[15]),
                 "+r"(r[16]), "+r"(r[17]), "+r"(r[18]), "+r"(r[19]), "+r"(r[20]), "+r"(r[21]), "+r"(r[22]), "+r"(r[23]),
                 "+r"(r[24]), "+r"(r[25]), "+r"(r[26]), "+r"(r[27]), "+r"(r[28]), "+r"(r[29]), "+r"(r[30]), "+r"(r[31])
               :
               : "memory");
}

// A finished part's number (0: the first); then, for all but the last, that it is written.
SPADE_DEVICE int take_number(int32_t *counter) { return atomicAdd(counter, 1); }
SPADE_DEVICE void publish_part(int32_t *counter) {
  asm volatile("red.release.gpu.global.add.s32 [%0], 1;" ::"l"(counter) : "memory");
}
// For parts that are written first: how many were.
SPADE_DEVICE int publish_counted(int32_t *counter) {
  int n;
  asm volatile("atom.acq_rel.gpu.global.add.s32 %0, [%1], 1;" : "=r"(n) : "l"(counter) : "memory");
  return n;
}
// Waits (bounded) until `n` parts are written.  Their CTAs have finished their products and wait for nothing.
SPADE_DEVICE bool await_parts(const int32_t *counter, int n) {
  const uint64_t t0 = globaltimer();
  int v;
  do {
    asm volatile("ld.acquire.gpu.global.s32 %0, [%1];" : "=r"(v) : "l"(counter) : "memory");
    if (v >= n) return true;
  } while (globaltimer() - t0 <= kWaitLimitNs);
  return false;
}

// warp_wait with its long part out of line: the loops that wait a few times a step stay short (2 x 512 nodes over 16384 slots, in
// short runs, 372 us; 381 with all of it in its place; with the first try out of line as well 374).
__device__ __noinline__ bool wait_long(uint64_t *bar, uint32_t parity, volatile int *abort) { return warp_wait(bar, parity, abort); }
SPADE_DEVICE bool wait_short(uint64_t *bar, uint32_t parity, volatile int *abort) {
  return __all_sync(0xffffffffu, mbar_test_wait(bar, parity)) || __all_sync(0xffffffffu, mbar_try_wait(bar, parity)) ||
         wait_long(bar, parity, abort);
}

// Of numbers that are not negative (a division of signed ones takes longer by some tens of cycles).
SPADE_DEVICE int over(int a, int b) { return static_cast<int>(static_cast<unsigned>(a) / static_cast<unsigned>(b)); }

struct Sched {
  const int32_t *pref, *ctx, *kd;
  int B, Hkv, nodes2;  // nodes2: nodes of a unit
  int size, longer;    // see Range

  // (Where they can be left out divisions are: one short sequence 8.4 us, 8.9 with all of them and signed.)
  __device__ int groups(int b) const { return kd[b] < 0 ? 0 : kd[b] < nodes2 ? 1 : over(kd[b], nodes2) + 1; }
  __device__ int chunks(int b) const { return (ctx[b] + kd[b] + kKeys) / kKeys; }  // of ctx + kd + 1 slots
  __device__ int begin_of(int cta) const { return cta * size + min(cta, longer); }
  __device__ int owner(int x) const {
    const int head = longer * (size + 1);
    return x < head ? x / (size + 1) : longer + (x - head) / size;
  }

  // The part at cost position x, by a whole warp.
  __device__ Seg at(int x, int x_end, int lane) const {
    int b = 0;
#pragma unroll 1
    for (int b0 = 0; b0 < B; b0 += 32) {
      const int bb = b0 + lane;
      const unsigned hit = __ballot_sync(0xffffffffu, bb < B && pref[bb] <= x && x < pref[bb + 1]);
      if (hit) {
        b = b0 + __ffs(hit) - 1;
        break;
      }
    }
    Seg s;
    s.b = b;
    s.nch = chunks(b);
    const int span = s.nch + kUnitCost, ng = groups(b);
    const int off = x - pref[b], u = off < span ? 0 : over(off, span);
    s.kvh = ng == 1 ? u : over(u, ng);
    s.group = u - s.kvh * ng;
    s.ust = pref[b] + u * span;
    s.end = min(x_end, s.ust + span);
    s.c0 = max(0, x - s.ust - kUnitCost);
    s.n = max(0, s.end - s.ust - kUnitCost) - s.c0;
    return s;
  }
  // The first at or after x that holds chunks (n = 0: none left).
  __device__ Seg next(int x, int x_end, int lane) const {
    Seg s;
    s.end = x;
#pragma unroll 1
    do s = at(s.end, x_end, lane);
    while (s.n == 0 && s.end < x_end);
    return s;
  }
};

// Not 0 if one of the eight bf16 numbers is not finite.
SPADE_DEVICE uint32_t times_zero(const uint4 &v) {
  uint32_t a, b;
  asm("fma.rn.bf16x2 %0, %1, %2, %2;" : "=r"(a) : "r"(v.x), "r"(0u));
  asm("fma.rn.bf16x2 %0, %1, %2, %2;" : "=r"(b) : "r"(v.y), "r"(0u));
  asm("fma.rn.bf16x2 %0, %1, %2, %0;" : "+r"(a) : "r"(v.z), "r"(0u));
  asm("fma.rn.bf16x2 %0, %1, %2, %0;" : "+r"(b) : "r"(v.w), "r"(0u));
  return a | b;
}

// Word i of a row's mask, w as it is stored (of any word where there is none): context before it, nothing behind node kd.
SPADE_DEVICE uint32_t seen_word(uint32_t w, int i, int kd) {
  const int left = kd - 32 * i;  // bits 0 .. left are nodes
  return i < 0 ? 0xffffffffu : left < 0 ? 0u : left < 31 ? w & ((2u << left) - 1) : w;
}

// A warp's half of the columns of O: NaN in the lanes of `odd` rows.  (Out of line: hardly ever needed.)
template <int D>
__device__ __noinline__ void make_nan(uint32_t t_o, bool odd) {
#pragma unroll 1
  for (int w = 0; w < D / 32; ++w) {
    uint32_t o[16];
    tmem_ld8(t_o + 16 * w, o);
    tmem_ld8(t_o + 16 * w + 8, o + 8);
    tmem_wait_ld();
#pragma unroll
    for (int e = 0; e < 16; ++e) o[e] = odd ? 0x7fffffffu : o[e];
    tmem_st16(t_o + 16 * w, o);
  }
  tmem_wait_st();
}

// Many parts: a part's O has been written; here its m and l.  The CTA whose part completes a group adds the group up, its sum
// taking the first part's place, and the one whose group completes the unit adds those up, in their order, for the row
// `orow` (-1: none).  A part is 64 KB, which a CTA reads in about a microsecond: 1 sequence, 1 KV head of 32000 slots
// 31 us, merged by one CTA 52.  By a stream's 256 threads; out of line, between loops that everything waits for.
template <int D>
__device__ __noinline__ void merge_groups(const Params &p, float m, float l, int first_slot, int my_part, int nparts, int32_t *unit,
                                          volatile int *s_last, int team, int row, int half, int64_t orow) {
  int gs = 3;
  while (gs * gs < nparts) ++gs;
  const int ngroups = (nparts + gs - 1) / gs, group = my_part / gs;
  auto slot_of = [&](int i) {  // only the first part may be its CTA's second segment
    return i == 0 ? first_slot : ((first_slot >> 2) + i) << 2 | (first_slot & 1);
  };
  auto at = [&](int i) { return p.partials + static_cast<int64_t>(slot_of(i)) * part_floats(D); };
  auto there = [&](int32_t *counter, int n) {
    named_bar(team, 256);
    if (row == 0 && half == 0) {
      const bool all = publish_counted(counter) == n - 1;
      if (all) *counter = 0;  // ready for the next call
      *s_last = all;
    }
    named_bar(team, 256);
    return *s_last != 0;
  };
  float *mine = at(my_part);
  int from = group * gs, stride = 1, n = min(gs, nparts - from);
#pragma unroll 1
  for (int level = 0;; ++level) {
    if (orow >= 0 && half == 0) {
      __stcg(mine + kRows * D + row, m);
      __stcg(mine + kRows * D + kRows + row, l);
    }
    if (!there(level ? unit : p.groups + slot_of(from), n)) return;
    const bool result = level > 0;
    mine = at(from);
    if (orow >= 0) {
      // 16 columns of up to kBatch parts at once; the next are asked for as soon as those have been added.
      constexpr int kBatch = 3;
      float4 q[kBatch][4];
      float f[kBatch];
      auto load = [&](int w, int i0) {
#pragma unroll
        for (int i = 0; i < kBatch; ++i) {
          const float *x = at(from + min(i0 + i, n - 1) * stride);
          f[i] = __ldcg(x + kRows * D + row);
#pragma unroll
          for (int e = 0; e < 4; ++e)
            q[i][e] = __ldcg(reinterpret_cast<const float4 *>(x) + (half * (D / 8) + 4 * w + e) * kRows + row);
        }
      };
      load(0, 0);
      m = -INFINITY;
      l = 0.f;
#pragma unroll 1
      for (int i0 = 0; i0 < n; i0 += 4) {
        float mp[4], lp[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float *ml = at(from + min(i0 + i, n - 1) * stride) + kRows * D + row;
          mp[i] = i0 + i < n ? __ldcg(ml) : -INFINITY;
          lp[i] = i0 + i < n ? __ldcg(ml + kRows) : 0.f;
        }
        const float mn = fmaxf(m, fmaxf(fmaxf(mp[0], mp[1]), fmaxf(mp[2], mp[3]))), base = mn == -INFINITY ? 0.f : mn;
        l *= ex2(m - base);
#pragma unroll
        for (int i = 0; i < 4; ++i) l += ex2(mp[i] - base) * lp[i];
        m = mn;
      }
      const float base = m == -INFINITY ? 0.f : m;
      const float inv = l == 0.f ? 0.f : 1.f / l;
      if (result && p.lse && half == 0) p.lse[orow] = l == 0.f ? -INFINITY : (m + log2f(l)) * 0.69314718055994531f;
      float4 acc[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) acc[e] = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 1
      for (int w = 0, i0 = 0; w < D / 32;) {
#pragma unroll
        for (int i = 0; i < kBatch; ++i) {
          if (i0 + i >= n) break;
          const float a = ex2(f[i] - base);
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            acc[e].x = fmaf(a, q[i][e].x, acc[e].x);
            acc[e].y = fmaf(a, q[i][e].y, acc[e].y);
            acc[e].z = fmaf(a, q[i][e].z, acc[e].z);
            acc[e].w = fmaf(a, q[i][e].w, acc[e].w);
          }
        }
        const int done = w;
        i0 += kBatch;
        if (i0 >= n) {
          i0 = 0;
          ++w;
        }
        if (w < D / 32) load(w, i0);
        if (w == done) continue;
        const int col = half * (D / 2) + 16 * done;
        if (result) {
          uint4 *dst = reinterpret_cast<uint4 *>(p.out + orow * D + col);
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            const float4 x = acc[2 * e], y = acc[2 * e + 1];
            auto two = [&](float a, float b) { return pack_bf16(fmaf(a, inv, 0.f), fmaf(b, inv, 0.f)); };
            dst[e] = make_uint4(two(x.x, x.y), two(x.z, x.w), two(y.x, y.y), two(y.z, y.w));
          }
        } else {
#pragma unroll
          for (int e = 0; e < 4; ++e) __stcg(reinterpret_cast<float4 *>(mine) + (col / 4 + e) * kRows + row, acc[e]);
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[e] = make_float4(0.f, 0.f, 0.f, 0.f);
      }
    }
    if (result) return;
    named_bar(team, 256);  // (the first part's m and l have been read by all)
    from = 0;
    stride = gs;
    n = ngroups;
  }
}

template <int D>
__global__ void __launch_bounds__(kThreads, 1)
    tree_attention_kernel(const __grid_constant__ Params p, const __grid_constant__ CUtensorMap tm_q,
                          const __grid_constant__ CUtensorMap tm_k2, const __grid_constant__ CUtensorMap tm_v2,
                          const __grid_constant__ CUtensorMap tm_k1, const __grid_constant__ CUtensorMap tm_v1) {
  constexpr int kSlabs = D / 64;
  extern __shared__ uint8_t smem_raw[];
  uint8_t *smem = smem_raw + ((1024u - (smem_u32(smem_raw) & 1023u)) & 1023u);
  int32_t *s_pref = reinterpret_cast<int32_t *>(smem + Smem::PREF);
  int32_t *s_ctx = reinterpret_cast<int32_t *>(smem + Smem::CTX);
  int32_t *s_kd = reinterpret_cast<int32_t *>(smem + Smem::KD);
  int32_t *s_q0 = reinterpret_cast<int32_t *>(smem + Smem::Q0);
  uint64_t *bars = reinterpret_cast<uint64_t *>(smem + Smem::BAR);
  uint32_t *s_bad = reinterpret_cast<uint32_t *>(smem + Smem::BAD);
  volatile int *s_abort = reinterpret_cast<volatile int *>(smem + Smem::MISC);
  volatile int *s_last = s_abort + 1;
  uint32_t *s_tmem = reinterpret_cast<uint32_t *>(smem + Smem::MISC + 12);
  Range *s_range = reinterpret_cast<Range *>(smem + Smem::RANGE);
  const int tid = threadIdx.x;
  const int warp = uniform_warp();
  const int lane = tid & 31;

  if (tid == 0) *s_abort = 0;
  if (warp == 0 && lane < 5) {
    const CUtensorMap *maps[5] = {&tm_q, &tm_k2, &tm_v2, &tm_k1, &tm_v1};
    tma_prefetch_desc(maps[lane]);
  } else if (warp == 1) {
    if (lane == 0) {
      for (int i = 0; i < 2; ++i) {
        mbar_init(&bars[kBarKFull + i], 1);
        mbar_init(&bars[kBarKEmpty + i], 1);
        mbar_init(&bars[kBarVFull + i], 1);
        mbar_init(&bars[kBarVReady + i], 1);
        mbar_init(&bars[kBarVEmpty + i], 1);
        mbar_init(&bars[kBarSFull + i], 1);
        mbar_init(&bars[kBarPFull + i], 4);
        mbar_init(&bars[kBarPHalf + i], 4);
        mbar_init(&bars[kBarQFull + i], 1);
        mbar_init(&bars[kBarOFinal + i], 1);
        mbar_init(&bars[kBarOFree + i], 8);
      }
      for (int i = 0; i < kBadRing; ++i) mbar_init(&bars[kBarBad + i], 1);
      mbar_init(&bars[kBarQFree], 1);
      mbar_init(&bars[kBarDrain], 1);
      mbar_init(&bars[kBarStart], 1);
      fence_mbar_init();
    }
    __syncwarp();
    tmem_alloc(s_tmem, kTmemCols);
    tmem_relinquish();
  }
  griddep_wait();
  griddep_launch_dependents();
  for (int b = tid; b < p.B; b += kThreads) {
    const int c = p.ctx_lens[b], k = p.n_draft[b], q0 = p.cu_q[b], q1 = p.cu_q[b + 1];
    int bad = 0;
    if (c < 0 || k < 0 || k > p.max_k || q0 < 0 || q1 > p.R || static_cast<int64_t>(q1) - q0 != static_cast<int64_t>(k) + 1)
      bad = SPADE_DEV_BAD_INDEX;
    else if (static_cast<int64_t>(c) + k + 1 > p.cap) bad = SPADE_DEV_CAPACITY;
    if (bad && blockIdx.x == 0) atomicOr(p.status, bad);
    s_ctx[b] = c;
    s_kd[b] = bad ? -1 : k;
    s_q0[b] = q0;
  }
  tc_fence_before();
  block_sync();
  tc_fence_after();
  Sched sc;
  sc.pref = s_pref; sc.ctx = s_ctx; sc.kd = s_kd; sc.B = p.B; sc.Hkv = p.Hkv; sc.nodes2 = 2 * p.tile_nodes;
  if (warp == 0) {
    int carry = 0;
    for (int b0 = 0; b0 < p.B; b0 += 32) {
      const int b = b0 + lane;
      const int w = b < p.B && s_kd[b] >= 0 ? p.Hkv * sc.groups(b) * (sc.chunks(b) + kUnitCost) : 0;
      int incl = w;
      for (int o = 1; o < 32; o <<= 1) {
        const int v = __shfl_up_sync(0xffffffffu, incl, o);
        if (lane >= o) incl += v;
      }
      if (b < p.B) s_pref[b] = carry + incl - w;
      carry += __shfl_sync(0xffffffffu, incl, 31);
    }
    int units = 0;
    for (int b = lane; b < p.B; b += 32) units += p.Hkv * sc.groups(b);
    units = __reduce_add_sync(0xffffffffu, units);
    if (lane == 0) {
      s_pref[p.B] = carry;
      Range r;
      r.total = carry;
      // More ranges than units only if there are twice as many, of kMinRange at least (a split costs its merge: 4 units of
      // 97 chunks 37 us, with ranges of 8 45).
      const int ranges = carry / kMinRange;
      r.num_ctas = max(1, min(p.num_ctas, ranges >= 2 * units ? ranges : units));
      r.size = carry / r.num_ctas;
      r.longer = carry - r.size * r.num_ctas;
      r.active = carry > 0 && static_cast<int>(blockIdx.x) < r.num_ctas;
      const int c = blockIdx.x;
      r.x_begin = r.active ? c * r.size + min(c, r.longer) : 0;
      r.x_end = r.active ? (c + 1) * r.size + min(c + 1, r.longer) : 0;
      *s_range = r;
    }
  }
  block_sync();
  const Range rng = *s_range;
  sc.size = rng.size;
  sc.longer = rng.longer;
  const uint32_t tmem = *s_tmem;
  const uint32_t smem_base = smem_u32(smem);
  const int x_end = rng.x_end;

  // The softmax threads hold half a row of scores: the launch's 96 registers a thread are dealt 64 to 104 (128 x 64 + 512 x 104
  // of 640 x 96).
  if (warp < 4) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 64;");
    if (!rng.active) {
      // nothing
    } else if (warp == 0 || warp == 3) {
    // ============================ producers: TMA ===========================
    const bool is_v = warp == 3;
    const bool leader = elect_one();
    const CUtensorMap *tm2 = is_v ? &tm_v2 : &tm_k2;
    const CUtensorMap *tm1 = is_v ? &tm_v1 : &tm_k1;
    uint64_t *const empty = bars + (is_v ? kBarVEmpty : kBarKEmpty);
    uint64_t *const full = bars + (is_v ? kBarVFull : kBarKFull);
    uint8_t *const ring = smem + (is_v ? Smem::V : Smem::K);
    const uint64_t pol = l2_policy_evict_first(), keep = l2_policy_evict_last();
    uint32_t it = 0, seg = 0, seg1 = 0;
    bool ok = true;
    for (int x = rng.x_begin; ok && x < x_end;) {
      const Seg g = sc.next(x, x_end, lane);
      const int n = uniform(g.n), b = uniform(g.b), kvh = uniform(g.kvh), c0 = uniform(g.c0);
      if (n == 0) break;
      const int live = uniform(s_ctx[b] + s_kd[b] + 1), node0 = uniform(g.group) * 2 * p.tile_nodes;
      const int nodes = uniform(s_kd[b]) + 1 - node0;
      const bool dual = nodes > p.tile_nodes;
      const int ngroups = uniform(sc.groups(b));
      const int row0 = (b * p.Hkv + kvh) * p.cap;
      for (int c = 0; c < n; ++c, ++it) {
        const int st = it % kStages;
        const int key0 = (c0 + c) * kKeys;
        const int slices = live - key0 > 64 ? 2 : 1;
        int row_a = row0 + key0, row_b = row_a + 64;
        if (p.block_table) {
          row_a = uniform(paged_row(p, b, kvh, key0));
          row_b = slices == 2 ? uniform(paged_row(p, b, kvh, key0 + 64)) : 0;
        }
        uint8_t *tile = ring + st * kTile;
        // (The first values wait until the first queries have come: scores need those and one tile of keys.  The barrier of
        // the queries themselves may have gone on to the next ones before this warp looks at it; this one completes once.)
        if (is_v && it == 0) ok = wait_short(&bars[kBarStart], 0, s_abort);
        ok = ok && wait_short(&empty[st], ((it / kStages) & 1) ^ 1, s_abort);
        if (!ok) break;
        if (leader) {
          mbar_arrive_expect_tx(&full[st], slices * 64 * D * 2);
          // (Read again by the KV head's other row groups: kept in L2.)
          const uint64_t how = ngroups > 1 ? keep : pol;
          if (slices == 2 && row_b == row_a + 64) {
            tma_load_3d(tile, tm2, 0, row_a, 0, &full[st], how);
          } else {
            for (int i = 0; i < slices; ++i)
              for (int sl = 0; sl < kSlabs; ++sl)
                tma_load_3d(tile + sl * kSlab + i * 64 * 128, tm1, 0, i ? row_b : row_a, sl, &full[st], how);
          }
        }
        __syncwarp();
        if (!is_v && c == 0) {
          // Q after the first K tile: its buffers free with the last segment's last S.
          ok = wait_short(&bars[kBarQFree], (seg & 1) ^ 1, s_abort);
          if (!ok) {
            ++it;
            break;
          }
          if (leader) {
            const int tiles = dual ? 2 : 1;
            for (int t = 0; t < tiles; ++t) {
              mbar_arrive_expect_tx(&bars[kBarQFull + t], kSlabs * p.tile_nodes * p.G * 128);
              for (int sl = 0; sl < kSlabs; ++sl)
                tma_load_4d(smem + Smem::Q + t * kTile + sl * kSlab, &tm_q, 0, kvh * p.G,
                            s_q0[b] + node0 + t * p.tile_nodes, sl, &bars[kBarQFull + t], keep);
            }
          }
          __syncwarp();
          ++seg;
          if (dual) ++seg1;
        }
      }
      x = g.end;
    }
    if (!ok && leader) {
      atomicOr(p.status, SPADE_DEV_TIMEOUT);
      // Every copy issued must land before the CTA's shared memory goes away.
      for (uint32_t j = it > kStages ? it - kStages : 0; j < it; ++j)
        mbar_wait_unabortable(&full[j % kStages], (j / kStages) & 1);
      if (seg > 0) mbar_wait_unabortable(&bars[kBarQFull], (seg - 1) & 1);
      if (seg1 > 0) mbar_wait_unabortable(&bars[kBarQFull + 1], (seg1 - 1) & 1);
    }
  } else if (warp == 1) {
    // ============================ MMA issuer ===============================
    constexpr uint32_t idesc_s = idesc_bf16_f32(128, kKeys);
    constexpr uint32_t idesc_pv = idesc_bf16_f32(128, D) | (1u << 16);  // B (V) MN-major
    const bool leader = elect_one();
    bool ok = true;
    // (Streams are compile-time constants, so that the MMAs' operands sit in uniform registers.)
    const uint32_t t_mem = static_cast<uint32_t>(uniform(static_cast<int>(tmem)));
    const uint32_t s_base = static_cast<uint32_t>(uniform(static_cast<int>(smem_base)));
    uint32_t it0 = 0, seg = 0, step0 = 0, step1 = 0, seg1 = 0, duals = 0;
    for (int x = rng.x_begin; ok && x < x_end;) {
      const Seg g = sc.next(x, x_end, lane);
      const int n = uniform(g.n), b = uniform(g.b);
      if (n == 0) break;
      const bool dual = uniform(s_kd[b]) + 1 - uniform(g.group) * 2 * p.tile_nodes > p.tile_nodes;
      const int nsteps = dual ? 2 * n : n;
      ok = wait_short(&bars[kBarQFull], seg & 1, s_abort);
      if (seg == 0 && lane == 0) mbar_arrive(&bars[kBarStart]);
      auto wait_k = [&](int j) {
        const uint32_t it = it0 + (dual ? j >> 1 : j);
        ok &= wait_short(&bars[kBarKFull + it % kStages], (it / kStages) & 1, s_abort);
      };
      auto issue_s = [&](auto stream, int j) {
        constexpr int s = decltype(stream)::value;
        const uint32_t it = it0 + (dual ? j >> 1 : j);
        const int st = it % kStages;
        const uint64_t dq = desc_sw128(s_base + Smem::Q + (dual ? s : 0) * kTile, 16, 1024);
        const uint64_t dk = desc_sw128(s_base + Smem::K + st * kTile, 16, 1024);
        if (leader) {
#pragma unroll
        for (int kk = 0; kk < D / 16; ++kk) {
          const uint32_t o = ((kk >> 2) * kSlab + (kk & 3) * 32) >> 4;
          tc_mma_f16(t_mem + kColS + s * 128, dq + o, dk + o, idesc_s, kk > 0 ? 1u : 0u);
        }
          tc_commit(&bars[kBarSFull + s]);
          if (!dual || s == 1) tc_commit(&bars[kBarKEmpty + st]);
          if (j == nsteps - 1) tc_commit(&bars[kBarQFree]);
        }
        __syncwarp();
      };
      auto issue_pv = [&](auto stream, int j) {
        constexpr int s = decltype(stream)::value;
        const uint32_t it = it0 + (dual ? j >> 1 : j);
        const int st = it % kStages;
        if (!dual || s == 0) ok &= wait_short(&bars[kBarVReady + st], (it / kStages) & 1, s_abort);
        ok &= wait_short(&bars[kBarPHalf + s], (s ? step1 : step0) & 1, s_abort);
        // The first product overwrites O: the epilogue of the stream's last segment has read it.
        if (j < 2) ok &= wait_short(&bars[kBarOFree + s], ((s ? seg1 : seg) & 1) ^ 1, s_abort);
        // (A segment of one step is stream 0's alone: the other has left the last of its own, whose words of kBarBad it read.)
        if (nsteps == 1) ok &= wait_short(&bars[kBarOFree + 1], (seg1 & 1) ^ 1, s_abort);
        tc_fence_after();
        const uint64_t dv = desc_sw128(s_base + Smem::V + st * kTile, kSlab, 1024);
        const uint32_t old = j < 2 ? 0u : 1u;
        if (leader) {
#pragma unroll
          for (int kk = 0; kk < kKeys / 32; ++kk)
            tc_mma_f16_ta(t_mem + kColO + s * 128, t_mem + kColS + s * 128 + 8 * kk, dv + 128u * kk, idesc_pv, kk > 0 ? 1u : old);
        }
        __syncwarp();
        ok &= wait_short(&bars[kBarPFull + s], (s ? step1 : step0) & 1, s_abort);
        tc_fence_after();
        if (leader) {
#pragma unroll
          for (int kk = kKeys / 32; kk < kKeys / 16; ++kk)
            tc_mma_f16_ta(t_mem + kColO + s * 128, t_mem + kColS + s * 128 + 8 * kk, dv + 128u * kk, idesc_pv, 1u);
          if (!dual || s == 1) tc_commit(&bars[kBarVEmpty + st]);
          if (j >= nsteps - 2) tc_commit(&bars[kBarOFinal + s]);
        }
        __syncwarp();
        if (s) ++step1; else ++step0;
      };
      const std::integral_constant<int, 0> s0{};
      const std::integral_constant<int, 1> s1{};
      wait_k(0);
      tc_fence_after();
      issue_s(s0, 0);
      if (dual) ok = ok && wait_short(&bars[kBarQFull + 1], duals++ & 1, s_abort);
      if (!dual && nsteps > 1) wait_k(1);
      tc_fence_after();
      if (nsteps > 1) issue_s(s1, 1);
      // (The next keys are waited for before P: they are there first, and a wait takes 100 cycles.)
      for (int j = 0; ok && j < nsteps; j += 2) {
        if (j + 2 < nsteps) wait_k(j + 2);
        issue_pv(s0, j);
        if (ok && j + 2 < nsteps) issue_s(s0, j + 2);
        if (!ok || j + 1 >= nsteps) break;
        if (!dual && j + 3 < nsteps) wait_k(j + 3);
        issue_pv(s1, j + 1);
        if (ok && j + 3 < nsteps) issue_s(s1, j + 3);
      }
      if (nsteps > 1) ++seg1;
      ++seg;
      it0 += n;
      x = g.end;
    }
    if (!ok && leader) {
      atomicOr(p.status, SPADE_DEV_TIMEOUT);
      tc_commit(&bars[kBarDrain]);
      mbar_wait_unabortable(&bars[kBarDrain], 0);
    }
  } else if (warp == 2) {
    // ============================ V rows of the block =======================
    constexpr int kLanes = D / 8, kRowsAtOnce = 32 / kLanes;
    const int l = lane % kLanes;
    uint32_t it = 0;
    bool ok = true;
    for (int x = rng.x_begin; ok && x < x_end;) {
      const Seg g = sc.next(x, x_end, lane);
      const int n = uniform(g.n), b = uniform(g.b), c0 = uniform(g.c0);
      if (n == 0) break;
      const int ctx = uniform(s_ctx[b]), live = ctx + uniform(s_kd[b]) + 1;
      for (int c = 0; c < n; ++c, ++it) {
        const int st = it % kStages;
        const int key0 = (c0 + c) * kKeys;
        ok = wait_short(&bars[kBarVFull + st], (it / kStages) & 1, s_abort);
        if (!ok) break;
        if (key0 + kKeys > ctx) {
          uint32_t *bad = s_bad + 4 * (it % kBadRing);
          if (lane < 4) bad[lane] = 0;
          __syncwarp();
          auto spot = [&](int r) {
            return reinterpret_cast<uint4 *>(smem + Smem::V + st * kTile + (l >> 3) * kSlab + r * 128 + (l & 7) * 16);
          };
          const int sub = lane / kLanes;
          const int r_live = min(max(live - key0, 0), kKeys);
          constexpr int kBatch = 8;
          for (int r0 = max(0, ctx - key0); r0 < r_live; r0 += kBatch * kRowsAtOnce) {
            uint4 x[kBatch];
#pragma unroll
            for (int i = 0; i < kBatch; ++i) {
              const int r = r0 + i * kRowsAtOnce + sub;
              x[i] = r < r_live ? *spot(r) : make_uint4(0, 0, 0, 0);
            }
            // (0 times a number that is not finite is NaN.)
            uint32_t odd[kBatch], any = 0;
#pragma unroll
            for (int i = 0; i < kBatch; ++i) {
              odd[i] = times_zero(x[i]);
              any |= odd[i];
            }
            if (!__any_sync(0xffffffffu, any)) continue;
#pragma unroll
            for (int i = 0; i < kBatch; ++i) {
              const int r = r0 + i * kRowsAtOnce + sub;
              const unsigned vote = __ballot_sync(0xffffffffu, odd[i]) >> (lane & ~(kLanes - 1)) & ((1u << kLanes) - 1);
              if (vote) {
                *spot(r) = make_uint4(0, 0, 0, 0);
                if (l == 0) atomicOr(&bad[r >> 5], 1u << (r & 31));
              }
            }
          }
          for (int r = r_live + sub; r < kKeys; r += kRowsAtOnce) *spot(r) = make_uint4(0, 0, 0, 0);
          fence_proxy_async_smem();
        }
        __syncwarp();
        if (lane == 0) {
          mbar_arrive(&bars[kBarVReady + st]);
          mbar_arrive(&bars[kBarBad + it % kBadRing]);
        }
      }
      x = g.end;
    }
    if (!ok && lane == 0) atomicOr(p.status, SPADE_DEV_TIMEOUT);
    }
  } else {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 104;");
    if (rng.active) {
    // ===================== softmax and epilogue (warps 4-19) ================
    // Two threads to a row, one for the first 64 keys of a chunk and one for the others, in warps that meet once a step.
    const int s = (warp - 4) >> 3;         // stream
    const int half = (warp >> 2) - 1 & 1;  // of the chunk's keys, and of O's columns
    const int q4 = warp & 3;               // tensor-memory lane quadrant
    const int row = q4 * 32 + lane;        // row of the tile
    const int pair = 1 + 4 * s + q4, quad = 9 + q4, team = 13 + s;  // named barriers: of the row's two warps, of both streams', of the stream
    const uint32_t tlane = tmem + (static_cast<uint32_t>(q4 * 32) << 16);
    const uint32_t t_s = tlane + kColS + s * 128, t_o = tlane + kColO + s * 128 + half * (D / 2);
    const int my_node = row / p.G, my_head = row - my_node * p.G;
    float *s_x = reinterpret_cast<float *>(smem + Smem::X) + (4 * half + q4) * 512 + lane;
    float *s_half = reinterpret_cast<float *>(smem + Smem::ML) + s * 2 * kRows + row;
    float *s_ml = reinterpret_cast<float *>(smem + Smem::M1);
    bool expired = false;
    uint32_t it0 = 0, step = 0, seg = 0;
    Seg next = sc.next(rng.x_begin, x_end, lane);
    while (next.n > 0) {
      const Seg g = next;
      const int ctx = s_ctx[g.b], kd = s_kd[g.b];
      const int node0 = g.group * 2 * p.tile_nodes;
      const bool dual = kd + 1 - node0 > p.tile_nodes;
      const int mysteps = dual ? g.n : (g.n - s + 1) / 2;
      const int node = node0 + (dual ? s * p.tile_nodes : 0) + my_node;
      const bool real = my_node < p.tile_nodes && node <= kd;
      const bool busy = __any_sync(0xffffffffu, real);  // the warp has rows
      const int q_row = s_q0[g.b] + node;
      const int32_t *mask = p.mask + static_cast<int64_t>(real ? q_row : s_q0[g.b]) * p.words;
      float m = -INFINITY, l = 0.f;
      bool odd = false;  // the row sees a value of the block that is not finite: its O becomes NaN, its l is the scores' alone
      // From the step j_tail on, chunks reach into the block.  The words of the row's mask are asked for a step ahead, and
      // what they name of values that are not finite is looked at a step later (the values are there later than the
      // scores): such a row becomes NaN.
      const int to_tail = ctx / kKeys - g.c0;
      const int j_tail = max(0, dual ? to_tail : (to_tail - s + 1) >> 1);
      uint32_t word[3] = {0, 0, 0}, was[2] = {0, 0};
      auto rel_of = [&](int j) { return (g.c0 + (dual ? j : 2 * j + s)) * kKeys + 64 * half - ctx; };
      auto look = [&](int j) {
        const int i = rel_of(j) >> 5;
#pragma unroll
        for (int t = 0; t < 3; ++t) word[t] = static_cast<uint32_t>(mask[min(max(i + t, 0), p.words - 1)]);
      };
      auto look_back = [&](int j) {
        const uint32_t it = it0 + (dual ? j : 2 * j + s);
        if (!mbar_wait(&bars[kBarBad + it % kBadRing], (it / kBadRing) & 1, s_abort)) expired = true;
        const uint32_t *bad = s_bad + 4 * (it % kBadRing) + 2 * half;
        if ((was[0] & bad[0]) | (was[1] & bad[1])) odd = true;
      };
      if (j_tail == 0 && mysteps > 0) look(0);
      for (int j = 0; j < mysteps; ++j, ++step) {
        if (!mbar_wait(&bars[kBarSFull + s], step & 1, s_abort)) expired = true;
        tc_fence_after();
        if (busy) {
          uint32_t v[64];
          tmem_ld32(t_s + 64 * half, v);
          tmem_ld32(t_s + 64 * half + 32, v + 32);
          tmem_wait_ld32(v);
          tmem_wait_ld32(v + 32);
          if (j >= j_tail) {
            if (j > j_tail) look_back(j - 1);
            // What the row does not see at -infinity.
            const int rel = rel_of(j);
            uint32_t w[3];
#pragma unroll
            for (int t = 0; t < 3; ++t) w[t] = real ? seen_word(word[t], (rel >> 5) + t, kd) : 0u;
#pragma unroll
            for (int t = 0; t < 2; ++t) {
              was[t] = __funnelshift_r(w[t], w[t + 1], rel & 31);
#pragma unroll
              for (int e = 0; e < 32; ++e) v[32 * t + e] = was[t] >> e & 1 ? v[32 * t + e] : 0xff800000u;
            }
          }
          if (j + 1 >= j_tail && j + 1 < mysteps) look(j + 1);
          float top[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
          for (int e = 0; e < 64; e += 8)
#pragma unroll
            for (int t = 0; t < 4; ++t) top[t] = max3(top[t], __uint_as_float(v[e + 2 * t]), __uint_as_float(v[e + 2 * t + 1]));
          const float mx = fmaxf(fmaxf(top[0], top[1]), fmaxf(top[2], top[3])) * p.scale_log2;
          // m = -infinity (nothing seen yet) moves with any score.  (The row's two warps meet here in any case: P takes
          // over columns of S that both have read.)
          if (attn::bar_any(pair, 64, mx > m + kRescaleLog2)) {
            s_half[half * kRows] = mx;
            named_bar(pair, 64);
            const float mn = fmaxf(fmaxf(m, mx), s_half[(half ^ 1) * kRows]);
            const float a = mn == m ? 1.f : ex2(m - mn);
            m = mn;
            l *= a;
            if (j > 0) {
              // The row's own lane of O follows, each warp half of its columns.
#pragma unroll 1
              for (int w = 0; w < D / 32; ++w) {
                uint32_t o[16];
                tmem_ld8(t_o + 16 * w, o);
                tmem_ld8(t_o + 16 * w + 8, o + 8);
                tmem_wait_ld();
#pragma unroll
                for (int e = 0; e < 16; ++e) o[e] = __float_as_uint(__uint_as_float(o[e]) * a);
                tmem_st16(t_o + 16 * w, o);
              }
            }
            named_bar(pair, 64);  // (the maxima have been read)
          }
          // P = 2^(s - m); the product with the first half of the keys may start before the second is done.
          const float base = m == -INFINITY ? 0.f : m;
          const F2 sc2 = f2(p.scale_log2, p.scale_log2), mb = f2(-base, -base);
          F2 sum[2] = {f2(0.f, 0.f), f2(0.f, 0.f)};
#pragma unroll
          for (int w = 0; w < 2; ++w) {
            uint32_t pk[16];
#pragma unroll
            for (int e = 0; e < 16; ++e) {
              float a, b;
              f2_split(f2_fma(f2(__uint_as_float(v[32 * w + 2 * e]), __uint_as_float(v[32 * w + 2 * e + 1])), sc2, mb), a, b);
              a = ex2(a);
              b = ex2(b);
              sum[e & 1] = f2_add(sum[e & 1], f2(a, b));
              pk[e] = pack_bf16(a, b);
            }
            tmem_st16(t_s + 32 * half + 16 * w, pk);
          }
          float a, b, c2, d;
          f2_split(sum[0], a, b);
          f2_split(sum[1], c2, d);
          l += (a + b) + (c2 + d);
          tmem_wait_st();
        }
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(&bars[(half ? kBarPFull : kBarPHalf) + s]);
      }
      // ---- epilogue: O of the streams to the output or a part ----
      next.n = 0;
      if (g.end < x_end) next = sc.next(g.end, x_end, lane);  // (under the last product)
      int c_first = blockIdx.x, nparts = 1;
      if (g.ust + kUnitCost < rng.x_begin || g.ust + kUnitCost + g.nch > x_end) {
        c_first = sc.owner(g.ust + kUnitCost);
        nparts = sc.owner(g.ust + kUnitCost + g.nch - 1) - c_first + 1;
      }
      const int tile = dual ? s : 0;
      const bool joined = !dual && g.n > 1;  // stream 1 has every other chunk of the same rows
      if (mysteps > 0) {
        if (!mbar_wait(&bars[kBarOFinal + s], seg & 1, s_abort)) expired = true;
        tc_fence_after();
        if (busy) {
          // The row's sum over both halves of the keys.
          if (mysteps > j_tail) look_back(mysteps - 1);
          // (A sum is not negative: its sign says that the half is odd.)
          s_half[half * kRows] = odd ? -l : l;
          named_bar(pair, 64);
          const float rest = s_half[(half ^ 1) * kRows];
          l += fabsf(rest);
          odd |= static_cast<int32_t>(__float_as_uint(rest)) < 0 && rest == rest;
          if (__any_sync(0xffffffffu, odd)) make_nan<D>(t_o, odd);
        }
      }
      float mine = 1.f, other = 0.f;  // factors of this stream's O and of the other's
      if (joined) {
        if (s == 1 && half == 0) {
          s_ml[row] = m;
          s_ml[kRows + row] = l;
        }
        named_bar(quad, 128);
        if (s == 0) {
          const float m1 = s_ml[row], l1 = s_ml[kRows + row];
          const float mn = fmaxf(m, m1), base = mn == -INFINITY ? 0.f : mn;
          mine = ex2(m - base);
          other = ex2(m1 - base);
          m = mn;
          l = l * mine + l1 * other;
        }
      }
      const bool writes = dual || s == 0;
      const size_t orow = static_cast<size_t>(q_row) * p.Hq + g.kvh * p.G + my_head;
      // A range has at most two split units: the one that it begins in and the one that it ends in.
      const int which = g.ust > rng.x_begin ? 1 : 0;
      float *part = p.partials + ((static_cast<int64_t>(blockIdx.x) * 2 + which) * 2 + tile) * part_floats(D);
      // The parts in order; the first is its CTA's second split unit, unless it begins that CTA's range.
      const int my_part = static_cast<int>(blockIdx.x) - c_first;
      const int second = g.ust > sc.begin_of(c_first) ? 1 : 0;
      auto part_at = [&](int i) {  // float4 of this row, columns 0 .. 3
        return reinterpret_cast<const float4 *>(
                   p.partials + ((static_cast<int64_t>(c_first + i) * 2 + (i == 0 ? second : 0)) * 2 + tile) * part_floats(D)) + row;
      };
      auto ml_at = [&](int i) {  // its m; kRows behind that, its l
        return reinterpret_cast<const float *>(part_at(i) - row) + kRows * D + row;
      };
      // (Of the units that begin in a CTA's range only the last goes on in another's.)
      int32_t *counter = p.counters + 4 * c_first + 2 * tile;
      const bool many = nparts > kMany;
      bool last = !many;
      if (writes && nparts > 1 && !many) {
        if (row == 0 && half == 0) s_last[s] = take_number(counter) == nparts - 1;
        named_bar(team, 256);
        last = s_last[s];
        if (last) {
          if (row == 0 && half == 0) {
            if (!await_parts(counter + 1, nparts - 1)) expired = true;
            counter[0] = counter[1] = 0;  // ready for the next call
          }
          named_bar(team, 256);
        }
      }
      // The row's maximum and sum over all parts.  (What follows runs once or twice in a CTA: short code, as it comes
      // from the L2 cache each time; unrolled it took 13 us to merge three parts.)
      float M = m, L = l;
      const bool merges = writes && last && nparts > 1;
      if (merges && real) {
        M = -INFINITY;
        L = 0.f;
#pragma unroll 1
        for (int i0 = 0; i0 < nparts; i0 += 4) {
          float mp[4], lp[4];
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const bool in = i0 + i < nparts && i0 + i != my_part;
            mp[i] = in ? __ldcg(ml_at(i0 + i)) : i0 + i == my_part ? m : -INFINITY;
            lp[i] = in ? __ldcg(ml_at(i0 + i) + kRows) : i0 + i == my_part ? l : 0.f;
          }
          float mn = M;
#pragma unroll
          for (int i = 0; i < 4; ++i) mn = fmaxf(mn, mp[i]);
          const float base = mn == -INFINITY ? 0.f : mn;
          L *= ex2(M - base);
#pragma unroll
          for (int i = 0; i < 4; ++i) L += ex2(mp[i] - base) * lp[i];
          M = mn;
        }
      }
      const float U = M == -INFINITY ? 0.f : M;
      const float inv = L == 0.f ? 0.f : 1.f / L;
      if (mysteps > 0 && busy) {
#pragma unroll 1
        for (int w = 0; w < D / 32; ++w) {
          const int col = half * (D / 2) + 16 * w;
          uint32_t o[16];
          tmem_ld8(t_o + 16 * w, o);
          tmem_ld8(t_o + 16 * w + 8, o + 8);
          tmem_wait_ld();
          if (joined) {
            if (s == 1) {
#pragma unroll
              for (int e = 0; e < 16; ++e) s_x[32 * e] = __uint_as_float(o[e]);
            }
            named_bar(quad, 128);
            if (s == 0) {
#pragma unroll
              for (int e = 0; e < 16; ++e) o[e] = __float_as_uint(__uint_as_float(o[e]) * mine + s_x[32 * e] * other);
            }
            named_bar(quad, 128);
          }
          if (!writes || !real) continue;
          if (!last) {
#pragma unroll
            for (int e = 0; e < 4; ++e)
              __stcg(reinterpret_cast<uint4 *>(part) + (col / 4 + e) * kRows + row,
                     make_uint4(o[4 * e], o[4 * e + 1], o[4 * e + 2], o[4 * e + 3]));
            continue;
          }
          if (merges) {
            float acc[16];
#pragma unroll
            for (int e = 0; e < 16; ++e) acc[e] = 0.f;
#pragma unroll 1
            for (int i0 = 0; i0 < nparts; i0 += 2) {
              float4 q[2][4];
              float a[2];
#pragma unroll
              for (int i = 0; i < 2; ++i) {
                const bool in = i0 + i < nparts && i0 + i != my_part;
                const float4 *src = part_at(i0 + i) + col / 4 * kRows;
                a[i] = in ? __ldcg(ml_at(i0 + i)) : i0 + i == my_part ? m : -INFINITY;
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                  q[i][e] = make_float4(__uint_as_float(o[4 * e]), __uint_as_float(o[4 * e + 1]), __uint_as_float(o[4 * e + 2]),
                                        __uint_as_float(o[4 * e + 3]));
                  if (in) q[i][e] = __ldcg(src + e * kRows);
                }
              }
#pragma unroll
              for (int i = 0; i < 2; ++i) {
                if (i0 + i >= nparts) break;
                const float f = ex2(a[i] - U);
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                  acc[4 * e] = fmaf(f, q[i][e].x, acc[4 * e]);
                  acc[4 * e + 1] = fmaf(f, q[i][e].y, acc[4 * e + 1]);
                  acc[4 * e + 2] = fmaf(f, q[i][e].z, acc[4 * e + 2]);
                  acc[4 * e + 3] = fmaf(f, q[i][e].w, acc[4 * e + 3]);
                }
              }
            }
#pragma unroll
            for (int e = 0; e < 16; ++e) o[e] = __float_as_uint(acc[e]);
          }
          uint4 *dst = reinterpret_cast<uint4 *>(p.out + orow * D + col);
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            uint32_t r[4];
#pragma unroll
            for (int t = 0; t < 4; ++t)
              r[t] = pack_bf16(fmaf(__uint_as_float(o[8 * e + 2 * t]), inv, 0.f), fmaf(__uint_as_float(o[8 * e + 2 * t + 1]), inv, 0.f));
            dst[e] = make_uint4(r[0], r[1], r[2], r[3]);
          }
        }
      }
      tc_fence_before();
      __syncwarp();
      if (mysteps > 0 && lane == 0) mbar_arrive(&bars[kBarOFree + s]);
      if (writes && last && p.lse && real && half == 0) p.lse[orow] = L == 0.f ? -INFINITY : (M + log2f(L)) * 0.69314718055994531f;
      if (writes && many) {
        merge_groups<D>(p, m, l, (c_first * 2 + second) * 2 + tile, my_part, nparts, counter, s_last + s, team, row, half,
                        real ? static_cast<int64_t>(orow) : -1);
      } else if (writes && !last) {
        if (real && half == 0) {
          __stcg(part + kRows * D + row, m);
          __stcg(part + kRows * D + kRows + row, l);
        }
        named_bar(team, 256);
        if (row == 0 && half == 0) publish_part(counter + 1);
      }
      if (mysteps > 0) ++seg;
      it0 += g.n;
    }
    if (expired) atomicOr(p.status, SPADE_DEV_TIMEOUT);
    }
  }

  tc_fence_before();
  block_sync();
  if (warp == 1) {
    tc_fence_after();
    tmem_dealloc(tmem, kTmemCols);
  }
}

// The sizes that the kernel's 32-bit numbers and the schedule hold.
static spade_status check_sizes(const char *name, int B, int Hq, int Hkv, int D, int cap, int max_k) {
  if (B <= 0 || Hq <= 0 || Hkv <= 0 || cap <= 0 || max_k < 0) return fail(SPADE_ERR_INVALID_ARG, "%s: non-positive size", name);
  if (Hq % Hkv) return fail(SPADE_ERR_SHAPE, "%s: Hq (%d) must be a multiple of Hkv (%d)", name, Hq, Hkv);
  if (D != 64 && D != 128) return fail(SPADE_ERR_SHAPE, "%s: head dim %d not supported (64 or 128)", name, D);
  if (B > kMaxB) return fail(SPADE_ERR_SHAPE, "%s: B = %d exceeds %d sequences per call", name, B, kMaxB);
  const int G = Hq / Hkv;
  if (G > kRows) return fail(SPADE_ERR_SHAPE, "%s: %d query heads per KV head exceed %d", name, G, kRows);
  // Slots and nodes up to a chunk past the last, and units, are 32-bit numbers; a node's slot is below the capacity.
  const int64_t nodes2 = 2 * (kRows / G), most = max_k < cap ? max_k : cap - 1;
  const int64_t groups = most / nodes2 + 1, units = static_cast<int64_t>(B) * Hkv * groups;
  // (The chunks of all units, with the virtual ones, too.)
  const int64_t chunks = (static_cast<int64_t>(cap) + kKeys - 1) / kKeys + kUnitCost;
  if (cap > INT32_MAX - 2 * kKeys || units > INT32_MAX / 4 || units * chunks > INT32_MAX - 2 * kThreads)
    return fail(SPADE_ERR_CAPACITY, "%s: %d x %d KV heads, %d slots and max_k = %d leave 32-bit numbers", name, B, Hkv, cap, max_k);
  return SPADE_OK;
}

// The workspace: counters of split units, those of groups of parts, the parts.  Where the counters lie depends on the device
// alone, so that calls of all sizes find them as the last call left them, whatever it was.  (SPADE_TREE_ATTN_ZEROED has
// room for those of 2048 SMs.)
static size_t counter_bytes(int sms) { return round_up(static_cast<size_t>(sms) * 16, 256); }
static size_t workspace_bytes_of(int sms, int D) {
  return 2 * counter_bytes(sms) + static_cast<size_t>(sms) * 4 * part_floats(D) * sizeof(float);
}

static spade_status attend(const char *name, Params p, const void *q, const void *k, const void *v, int D, int64_t cache_rows,
                           void *workspace, size_t workspace_bytes, cudaStream_t stream) {
  if (!q || !k || !v || !p.ctx_lens || !p.n_draft || !p.cu_q || !p.mask || !p.out || !p.status)
    return fail(SPADE_ERR_INVALID_ARG, "%s: null pointer argument", name);
  spade_status st = check_sizes(name, p.B, p.Hq, p.Hkv, D, p.cap, p.max_k);
  if (st != SPADE_OK) return st;
  if (p.R <= 0 || p.R < p.B) return fail(SPADE_ERR_INVALID_ARG, "%s: R = %d < B = %d", name, p.R, p.B);
  if (p.words < p.max_k / 32 + 1)
    return fail(SPADE_ERR_SHAPE, "%s: %d mask words for blocks of %lld nodes", name, p.words, static_cast<long long>(p.max_k) + 1);
  if (cache_rows >= (int64_t(1) << 31))
    return fail(SPADE_ERR_CAPACITY, "%s: KV cache rows (B or pages) * Hkv * slots exceed 2^31", name);
  if (!aligned(q, 16) || !aligned(k, 16) || !aligned(v, 16) || !aligned(p.out, 16))
    return fail(SPADE_ERR_INVALID_ARG, "%s: q, caches and out must be 16-byte aligned", name);
  int sms = 0;
  st = device_info(&sms, nullptr);
  if (st != SPADE_OK) return st;
  const size_t need = workspace_bytes_of(sms, D);
  if (!workspace || workspace_bytes < need || !aligned(workspace, 256))
    return fail(SPADE_ERR_WORKSPACE, "%s: workspace needs %zu bytes, 256-byte aligned (got %zu)", name, need, workspace_bytes);
  p.counters = static_cast<int32_t *>(workspace);
  p.groups = p.counters + counter_bytes(sms) / 4;
  p.partials = reinterpret_cast<float *>(p.groups + counter_bytes(sms) / 4);
  p.G = p.Hq / p.Hkv;
  p.tile_nodes = kRows / p.G;
  p.scale_log2 = 1.4426950408889634f / sqrtf(static_cast<float>(D));
  p.num_ctas = sms;  // the schedule leaves those out that have no work: results do not depend on bounds
  const uint64_t q_dims[4] = {64, static_cast<uint64_t>(p.Hq), static_cast<uint64_t>(p.R), static_cast<uint64_t>(D / 64)};
  const uint64_t q_strides[3] = {static_cast<uint64_t>(D) * 2, static_cast<uint64_t>(p.Hq) * D * 2, 128};
  const uint32_t q_box[4] = {64, static_cast<uint32_t>(p.G), static_cast<uint32_t>(p.tile_nodes), 1};
  const uint64_t rows = static_cast<uint64_t>(cache_rows);
  CUtensorMap mq, k2, v2, k1, v1;
  if (!encode_tmap_bf16_sw128_nd(&mq, q, 4, q_dims, q_strides, q_box) || !encode_tmap_rows_by_slab(&k2, k, rows, D, kKeys) ||
      !encode_tmap_rows_by_slab(&v2, v, rows, D, kKeys) || !encode_tmap_rows_by_slab(&k1, k, rows, D, 64, 1) ||
      !encode_tmap_rows_by_slab(&v1, v, rows, D, 64, 1))
    return SPADE_ERR_CUDA;
  cudaError_t e;
  if (D == 128) {
    static OncePerDevice once;
    e = set_max_smem(once, Smem::BYTES, tree_attention_kernel<128>);
    if (e == cudaSuccess)
      e = launch(tree_attention_kernel<128>, dim3(p.num_ctas), 1, kThreads, Smem::BYTES, stream, p, mq, k2, v2, k1, v1);
  } else {
    static OncePerDevice once;
    e = set_max_smem(once, Smem::BYTES, tree_attention_kernel<64>);
    if (e == cudaSuccess)
      e = launch(tree_attention_kernel<64>, dim3(p.num_ctas), 1, kThreads, Smem::BYTES, stream, p, mq, k2, v2, k1, v1);
  }
  return e == cudaSuccess ? SPADE_OK : cuda_fail(e, name);
}

}  // namespace attn_tree
}  // namespace spade

using namespace spade;

extern "C" size_t spade_tree_attn_workspace_size(int32_t B, int32_t Hq, int32_t Hkv, int32_t D, int32_t cap, int32_t max_k) {
  int sms = 0;
  if (attn_tree::check_sizes("spade_tree_attn_workspace_size", B, Hq, Hkv, D, cap, max_k) != SPADE_OK) return 0;
  if (device_info(&sms, nullptr) != SPADE_OK) return 0;
  return attn_tree::workspace_bytes_of(sms, D);
}

extern "C" spade_status spade_verify_attention_tree(const void *q, const void *k_cache, const void *v_cache,
                                                    const int32_t *ctx_lens, const int32_t *n_draft, const int32_t *cu_q,
                                                    const int32_t *tree_mask, void *out, float *lse, int32_t B, int32_t Hq,
                                                    int32_t Hkv, int32_t D, int32_t cap, int32_t mask_words, int32_t max_k,
                                                    int32_t R, void *workspace, size_t workspace_bytes, int32_t *status,
                                                    spade_stream_t stream) {
  attn_tree::Params p = {};
  p.out = static_cast<__nv_bfloat16 *>(out); p.lse = lse; p.ctx_lens = ctx_lens; p.n_draft = n_draft; p.cu_q = cu_q;
  p.mask = tree_mask; p.status = status; p.B = B; p.Hq = Hq; p.Hkv = Hkv; p.cap = cap; p.max_k = max_k; p.R = R;
  p.words = mask_words;
  return attn_tree::attend("spade_verify_attention_tree", p, q, k_cache, v_cache, D, static_cast<int64_t>(B) * Hkv * cap,
                           workspace, workspace_bytes, reinterpret_cast<cudaStream_t>(stream));
}

extern "C" spade_status spade_verify_attention_tree_paged(
    const void *q, const void *k_pool, const void *v_pool, const int32_t *block_table, const int32_t *ctx_lens,
    const int32_t *n_draft, const int32_t *cu_q, const int32_t *tree_mask, void *out, float *lse, int32_t B, int32_t Hq,
    int32_t Hkv, int32_t D, int32_t page_size, int32_t num_pages, int32_t max_pages, int32_t mask_words, int32_t max_k,
    int32_t R, void *workspace, size_t workspace_bytes, int32_t *status, spade_stream_t stream) {
  static const char *name = "spade_verify_attention_tree_paged";
  if (!block_table) return fail(SPADE_ERR_INVALID_ARG, "%s: null block_table", name);
  if (page_size <= 0 || num_pages <= 0 || max_pages <= 0)
    return fail(SPADE_ERR_INVALID_ARG, "%s: non-positive page geometry", name);
  if (page_size % 64) return fail(SPADE_ERR_SHAPE, "%s: page size %d must be a multiple of 64", name, page_size);
  if (static_cast<int64_t>(max_pages) * page_size >= (int64_t(1) << 31))
    return fail(SPADE_ERR_CAPACITY, "%s: max_pages * page_size exceeds 2^31", name);
  attn_tree::Params p = {};
  p.out = static_cast<__nv_bfloat16 *>(out); p.lse = lse; p.ctx_lens = ctx_lens; p.n_draft = n_draft; p.cu_q = cu_q;
  p.mask = tree_mask; p.status = status; p.block_table = block_table; p.B = B; p.Hq = Hq; p.Hkv = Hkv;
  p.cap = max_pages * page_size; p.max_k = max_k; p.R = R; p.words = mask_words; p.page_size = page_size;
  p.max_pages = max_pages; p.num_pages = num_pages;
  return attn_tree::attend(name, p, q, k_pool, v_pool, D, static_cast<int64_t>(num_pages) * Hkv * page_size, workspace,
                           workspace_bytes, reinterpret_cast<cudaStream_t>(stream));
}
