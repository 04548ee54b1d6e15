// sample.cu -- a token drawn from each row of logits by a given uniform (the verifier's or the
// drafter's sampling, "for diversity", Sec. III-A), under temperature, top-k, top-p and min-p.
//
// The tokens are those of the definition in 64 bits (but for uniforms within about 2^-36 of an
// edge), not of fp32 sums: a weight 2^((l - m) log2(e) / T) is computed to 2^-39 of itself and
// summed as a whole number, in units of 2^-60 of the largest, so sums are exact, whatever their order, and a
// tail of a million tokens below the unit is off by 2^-40 at most.  (Sums are 128 bits wide; 64 leave a million
// tokens a unit of 2^-42 and an error of 2^-22.)  Where few tokens are summed the unit is 2^-50.
//
// A cluster of CTAs takes a row: each copies its part once into shared memory, and what follows (the
// largest logit, counts, sums) meets through distributed shared memory.  The kept set is always
// {x : l_x >= tau}, ties with the last token included, so that one number describes it:
//   min_p:  tau = m + T ln(min_p);
//   top-k, top-p: every thread's largest logit is known; a bound that enough of those reach (the k
//   asked for, or some hundred) is found from a histogram of them, and the tokens that reach the bound
//   are listed.  If they are few (kList) and hold what is asked for, one CTA decides on them and draws,
//   by comparing each with each or by bisection.  The nucleus needs the mass of the tokens behind the list
//   only to the precision that settles where it ends: that mass is summed in fp32 with a bound of its
//   error, and summed exactly by the deciding CTA where the bound does not settle it;
//   else tau is found by rounds of histograms with exact counts or masses: 256 bins of values, then of the order
//   of the type's numbers within the bin of the boundary, down to one number.
// Where more tokens are kept than one CTA lists, the draw sums weights known to 2^-20 first, and exact ones only where
// those do not settle the token.
//
// Measured, back to back (in brackets the time in which the logits, and probabilities, pass HBM once): 8 rows of 128256 fp32
// with top-k, top-p and probabilities 14.4 us (1.2), 512 rows in bf16 with top-p and min-p 81 (19), with top-p alone
// 139, with top-k 72, greedy 38, with nothing to leave out 97; nuclei of tens of thousands of tokens 820.  Few rows are bound by the meetings of the cluster and
// of the deciding CTA's threads (about a microsecond each, 14 of them), many by the same on 456 CTAs at a time: a
// part's 51 KB are there after 1 of its 15 us.  384 threads, three CTAs to an SM: 256 and four take 77 us for the 512
// rows with top-p and min-p, but 46 instead of 41 for 72 rows with top-p; 512 and two 82 and 55.
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include <cfloat>

#include "internal.h"
#include "launch.h"
#include "ptx.cuh"

namespace spade {
namespace sample {

constexpr int kThreads = 384;
constexpr int kWarps = kThreads / 32;
constexpr int kBins = 256;
constexpr int kLocal = 1024;               // tokens that a CTA lists
constexpr int kList = 2048;                // tokens that one CTA decides on
// Of up to so many, by comparing each with each; of more, by bisection (70 tokens: 2 us instead of 12; from 64 to 256 no
// case differs).
constexpr int kPairs = 128;
constexpr int kSteps = 4;                  // of that between looks at the range
// Tokens listed for a nucleus of unknown size (of a CTA's at most 0.7 kLocal): 512 x 128256 bf16 rows with top_p = 0.95 136
// us, with 1000 140, with 1400 146.
constexpr int kAim = 800;
constexpr int kMaxCluster = 16;
constexpr int kSliceBytes = 56 * 1024;     // of a row in a CTA: three CTAs to an SM
constexpr int kMinBytes = 8 * (kList + kPairs);  // a part's room holds the list, and masses, later
constexpr int kMaxSliceBytes = 192 * 1024; // of rows that no cluster holds in that
constexpr int kCopyBytes = 8192;           // of one bulk copy

struct Params {
  const void *logits;
  const float *uniforms, *temperature, *top_p, *min_p;
  const int32_t *top_k;
  int32_t *tokens, *status;
  float *probs, *chosen;
  int64_t stride;  // of the logits' rows, in elements
  int V, slice;    // slice: 16-byte vectors of a CTA
  int shift;       // unit of the rough draw's sums: 2^-shift of the largest weight
};

// 2^(j / 256) in units of 2^-40, by the exponential series at compile time.
struct Powers {
  uint64_t v[256];
};
constexpr Powers make_powers() {
  Powers t{};
  for (int j = 0; j < 256; ++j) {
    const double x = 0.69314718055994530942 * j / 256;
    double sum = 1, term = 1;
    for (int i = 1; i < 24; ++i) {
      term *= x / i;
      sum += term;
    }
    t.v[j] = static_cast<uint64_t>(sum * 1099511627776.0 + 0.5);
  }
  return t;
}
__device__ constexpr Powers kPowers = make_powers();

// Where T is 2^64 and more, logits and T are 2^64 times smaller here: their differences stay finite, log2(e) / T stays
// a normal number, and what a logit loses below 2^-126 is nothing beside T.
struct Row {
  float m;       // largest logit, times scale
  float scale;   // 1 or 2^-64
  float ch, cl;  // log2(e) / (T scale), high and low part
};
constexpr float kHuge = 18446744073709551616.f;  // 2^64

// Sums of weights in units of 2^-kMassShift of the largest: 2^21 weights of up to 2^60, and a product with a number of 24
// bits, stay below 2^106.  A vector's sum is below 2^64.
using Mass = unsigned __int128;
constexpr int kMassShift = 60;
// The unit of a list of up to kList tokens: its sums stay below 2^62, and what is below it makes 2^-39.
constexpr int kListShift = 50;

// Weight of a logit relative to the largest, as 2^40 .. 2^41 times 2^(-40 - e) (e < 0: it is 0).
// With x = (l - m) log2(e) / T = n / 256 + r, |r| <= 1/512, the weight is 2^(n/256) (1 + y),
// y = e^(r ln 2) - 1 by four terms of its series, r and y held as pairs of fp32 numbers.
SPADE_DEVICE uint64_t weight40(const Row &w, const uint64_t *powers, float l, int *e) {
  const float s = fmaf(l, w.scale, -w.m);
  *e = 0;
  if (s == 0.f) return uint64_t(1) << 40;
  const float x = l * w.scale, back = s - x;
  const float rest = (x - (s - back)) + (-w.m - back);  // x - m = s + rest
  const float ph = s * w.ch;
  if (!(ph > -1075.f)) {  // less than the smallest number of 64 bits: 0
    *e = -1;
    return 0;
  }
  const float pl = fmaf(s, w.ch, -ph) + fmaf(s, w.cl, rest * w.ch);
  constexpr float kMagic = 12582912.f;  // 1.5 2^23: adding it rounds to a whole number
  const float t = fmaf(ph, 256.f, kMagic);
  const int n = __float_as_int(t) - __float_as_int(kMagic);
  const float rh = fmaf(t - kMagic, -1.f / 256.f, ph);
  constexpr float kLn2 = 0.693147182464599609375f, kLn2Low = -1.904654299957767e-9f;
  const float zh = rh * kLn2;
  const float zl = fmaf(rh, kLn2, -zh) + fmaf(rh, kLn2Low, pl * kLn2);
  const float yl = zl + fmaf(zh, zl, zh * zh * fmaf(zh, 1.f / 6.f, 0.5f));
  const int y = __float2int_rn(zh * 1099511627776.f) + __float2int_rn(yl * 1099511627776.f);
  const uint64_t p = powers[n & 255];
  *e = -(n >> 8);
  return p + ((static_cast<int64_t>(static_cast<int>(p >> 10)) * y) >> 30);
}
// The weight to 2^-21 of itself (the power on the SFU 2^-22, its argument as a pair of numbers), of finite l.
template <bool kInexact>
SPADE_DEVICE float weight_about(const Row &w, float l) {
  const float s = fmaf(l, w.scale, -w.m);
  const float ph = s * w.ch;
  float pl = fmaf(s, w.ch, -ph) + s * w.cl;
  if constexpr (kInexact) {  // (the difference of two 16-bit numbers is off only where its weight is nothing)
    const float x = l * w.scale, back = s - x;
    pl = fmaf((x - (s - back)) + (-w.m - back), w.ch, pl);
  }
  const float q = ex2(ph);
  return s == 0.f ? 1.f : ph > -120.f ? fmaf(q * pl, 0.693147181f, q) : 0.f;
}
// The weight in units of 2^-kMassShift, or of a list; at least one unit if it is not 0.
template <int kShift = kMassShift>
SPADE_DEVICE uint64_t weight(const Row &w, const uint64_t *powers, float l) {
  int e;
  const uint64_t v = weight40(w, powers, l, &e);
  if (e < 0) return 0;
  const uint64_t u = e > 63 ? 0 : v << (kShift - 40) >> e;
  return u ? u : 1;
}

// fp32 numbers as whole numbers of the same order (-0 taken as 0).
SPADE_DEVICE uint32_t order_of(float x) {
  const uint32_t u = __float_as_uint(x + 0.f);
  return u ^ (static_cast<int32_t>(u) < 0 ? 0xffffffffu : 0x80000000u);
}
SPADE_DEVICE float number_of(uint32_t o) { return __uint_as_float(o ^ (o & 0x80000000u ? 0x80000000u : 0xffffffffu)); }

// The larger of each of a vector's numbers and of those before (NaN if there is one), two 16-bit numbers at a time.
struct Tops32 {
  float v = -INFINITY;
  static constexpr int kSize = 4, kSpare = 0;
  SPADE_DEVICE static float number(const uint4 &x, int e) { return __uint_as_float((&x.x)[e]); }
  SPADE_DEVICE static uint32_t out() { return 0xff800000u; }
  SPADE_DEVICE static float nan_max(float a, float b) {
    float r;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
    return r;
  }
  SPADE_DEVICE void take(const uint4 &x) {
    v = nan_max(v, nan_max(nan_max(number(x, 0), number(x, 1)), nan_max(number(x, 2), number(x, 3))));
  }
  SPADE_DEVICE float top() const { return v; }
  SPADE_DEVICE static float largest(const uint4 &x) { return fmaxf(fmaxf(number(x, 0), number(x, 1)), fmaxf(number(x, 2), number(x, 3))); }
};
template <bool kBf16>
struct Tops16 {
  uint32_t v = kBf16 ? 0xff80ff80u : 0xfc00fc00u;
  static constexpr int kSize = 2;
  static constexpr int kSpare = kBf16 ? 16 : 13;  // low bits of the order that all of the type's numbers share
  SPADE_DEVICE static float number(const uint4 &x, int e) {
    const uint32_t w = (&x.x)[e >> 1];
    if constexpr (kBf16) {
      return __uint_as_float(e & 1 ? w & 0xffff0000u : w << 16);
    } else {
      return __half2float(__ushort_as_half(static_cast<uint16_t>(e & 1 ? w >> 16 : w & 0xffffu)));
    }
  }
  SPADE_DEVICE static uint32_t out() { return kBf16 ? 0xff80u : 0xfc00u; }
  SPADE_DEVICE static uint32_t nan_max(uint32_t a, uint32_t b) {
    uint32_t r;
    if constexpr (kBf16) asm("max.NaN.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    else asm("max.NaN.f16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    return r;
  }
  SPADE_DEVICE void take(const uint4 &x) { v = nan_max(v, nan_max(nan_max(x.x, x.y), nan_max(x.z, x.w))); }
  SPADE_DEVICE static float larger(uint32_t pair) {
    const uint4 x = make_uint4(pair, 0, 0, 0);
    return Tops32::nan_max(number(x, 0), number(x, 1));
  }
  SPADE_DEVICE float top() const { return larger(v); }
  SPADE_DEVICE static float largest(const uint4 &x) { return larger(nan_max(nan_max(x.x, x.y), nan_max(x.z, x.w))); }
};

// ---- distributed shared memory ----
SPADE_DEVICE void st_cluster(uint32_t addr, uint64_t v) {
  asm volatile("st.shared::cluster.b64 [%0], %1;" ::"r"(addr), "l"(v) : "memory");
}
SPADE_DEVICE uint64_t ld_cluster64(uint32_t addr) {
  uint64_t v;
  asm volatile("ld.shared::cluster.b64 %0, [%1];" : "=l"(v) : "r"(addr) : "memory");
  return v;
}
SPADE_DEVICE uint32_t ld_cluster32(uint32_t addr) {
  uint32_t v;
  asm volatile("ld.shared::cluster.b32 %0, [%1];" : "=r"(v) : "r"(addr) : "memory");
  return v;
}

template <class V, class F>
SPADE_DEVICE V warp_reduce(V v, F f) {
#pragma unroll
  for (int o = 16; o; o /= 2) v = f(v, __shfl_xor_sync(0xffffffffu, v, o));
  return v;
}
SPADE_DEVICE uint64_t add64(uint64_t a, uint64_t b) { return a + b; }
SPADE_DEVICE uint64_t low_of(Mass v) { return static_cast<uint64_t>(v); }
SPADE_DEVICE uint64_t high_of(Mass v) { return static_cast<uint64_t>(v >> 64); }
SPADE_DEVICE Mass mass_of(uint64_t low, uint64_t high) { return static_cast<Mass>(high) << 64 | low; }
SPADE_DEVICE uint64_t shuffled_up(uint64_t v, int o) { return __shfl_up_sync(0xffffffffu, v, o); }
SPADE_DEVICE Mass shuffled_up(Mass v, int o) { return mass_of(shuffled_up(low_of(v), o), shuffled_up(high_of(v), o)); }
SPADE_DEVICE uint64_t last_lane(uint64_t v) { return __shfl_sync(0xffffffffu, v, 31); }
SPADE_DEVICE Mass last_lane(Mass v) { return mass_of(last_lane(low_of(v)), last_lane(high_of(v))); }
template <class V>
SPADE_DEVICE V warp_scan(V v, int lane) {  // inclusive
#pragma unroll
  for (int o = 1; o < 32; o *= 2) {
    const V x = shuffled_up(v, o);
    if (lane >= o) v += x;
  }
  return v;
}
SPADE_DEVICE uint64_t warp_add(uint64_t v) { return warp_reduce(v, add64); }
SPADE_DEVICE Mass warp_add(Mass v) {
#pragma unroll
  for (int o = 16; o; o /= 2)
    v += mass_of(__shfl_xor_sync(0xffffffffu, low_of(v), o), __shfl_xor_sync(0xffffffffu, high_of(v), o));
  return v;
}

struct Shared {
  uint64_t powers[256];
  uint64_t list[kLocal];     // the part's listed tokens: order (descending) and index; read by the leader
  uint32_t hist[kBins], mid[kBins], high[kBins];  // counts, or the three words of masses
  uint64_t warp[kWarps];     // results of the warps
  Mass wide[kWarps];
  uint64_t sums[2][kWarps];
  float masses[2][kWarps];
  uint64_t meet[2][3][kMaxCluster];  // results of the cluster's CTAs, by turns
  uint64_t bar;              // the part's copies
  double reach;              // T ln(min_p)
  uint32_t count, settled;
  int cut;
  int cuts[2];               // a round of histograms' boundary bin, and what is above it: by turns, as a thread late in
  Mass above[2];             // reading one round's must not find the next round's
  float ch, cl, scale, tau;  // see Row
  float u, top_p, temp;      // options, for the code after the loops that need the registers
};

// What a block's threads need for the meetings of its cluster.
struct Team {
  Shared *s;
  int tid, lane, warp, rank, size, turn;

  // Sum or maximum over the CTA's threads, on every thread.
  template <class F>
  SPADE_DEVICE uint64_t block(uint64_t v, F f) {
    v = warp_reduce(v, f);
    if (lane == 0) s->warp[warp] = v;
    __syncthreads();
    uint64_t r = s->warp[0];
    for (int i = 1; i < kWarps; ++i) r = f(r, s->warp[i]);
    __syncthreads();
    return r;
  }
  // n numbers of every CTA (of v in its first threads: tid < n), as all[i][rank] on every thread after the call.
  // (A CTA may already write the next meeting's while another reads this one's: two arrays by turns.)
  SPADE_DEVICE const uint64_t (*exchange(int n, uint64_t v0, uint64_t v1, uint64_t v2))[kMaxCluster] {
    const int t = turn;
    turn ^= 1;
    if (tid < size) {
      st_cluster(cluster_map(&s->meet[t][0][rank], tid), v0);
      if (n > 1) st_cluster(cluster_map(&s->meet[t][1][rank], tid), v1);
      if (n > 2) st_cluster(cluster_map(&s->meet[t][2][rank], tid), v2);
    }
    cluster_sync();
    return s->meet[t];
  }
  // The CTA's result on every thread of warp 0 (others: of no meaning).
  template <class F>
  SPADE_DEVICE uint64_t gather(uint64_t v, F f) {
    v = warp_reduce(v, f);
    if (lane == 0) s->warp[warp] = v;
    __syncthreads();
    if (warp == 0) {
      v = s->warp[0];
      for (int j = 1; j < kWarps; ++j) v = f(v, s->warp[j]);
    }
    return v;
  }
  // (The warps' results are read before the cluster meets, so its barrier frees them.)
  template <class F>
  SPADE_DEVICE uint64_t cluster(uint64_t x, F f) {
    const uint64_t(*all)[kMaxCluster] = exchange(1, gather(x, f), 0, 0);
    uint64_t r = all[0][0];
    for (int i = 1; i < size; ++i) r = f(r, all[0][i]);
    return r;
  }
  // Sums of masses over the CTA's threads and over the cluster, on every thread.
  SPADE_DEVICE Mass block_sum(Mass v) {
    v = warp_add(v);
    if (lane == 0) s->wide[warp] = v;
    __syncthreads();
    Mass r = s->wide[0];
    for (int i = 1; i < kWarps; ++i) r += s->wide[i];
    __syncthreads();
    return r;
  }
  SPADE_DEVICE Mass cluster_sum(Mass v) {
    v = block_sum(v);
    const uint64_t(*all)[kMaxCluster] = exchange(2, low_of(v), high_of(v), 0);
    Mass r = 0;
    for (int i = 0; i < size; ++i) r += mass_of(all[0][i], all[1][i]);
    return r;
  }
};

// f = digits 2^-q, q >= 24, of f in [0, 1).
SPADE_DEVICE uint32_t digits_of(float f, int *q) {
  const uint32_t bits = __float_as_uint(f);
  const int exponent = static_cast<int>(bits >> 23);
  *q = 150 - (exponent ? exponent : 1);
  return (bits & 0x7fffffu) | (exponent ? 0x800000u : 0u);
}
// f * total for f in [0, 1], rounded down (up: up).
SPADE_DEVICE uint64_t part_of(float f, uint64_t total, bool up) {
  if (f >= 1.f) return total;
  int q;
  const uint64_t digits = digits_of(f, &q), hi = __umul64hi(total, digits), lo = total * digits;
  uint64_t t = 0;
  bool rest;
  if (q < 64) {
    t = hi << (64 - q) | lo >> q;
    rest = (lo & ((uint64_t(1) << q) - 1)) != 0;
  } else {
    if (q < 128) t = hi >> (q - 64);
    rest = lo != 0 || (q < 128 ? (hi & ((uint64_t(1) << (q - 64)) - 1)) : hi) != 0;
  }
  return t + (up && rest);
}
SPADE_DEVICE Mass part_of(float f, Mass total, bool up) {
  if (f >= 1.f) return total;
  int q;
  const Mass t = total * digits_of(f, &q), whole = q < 128 ? t >> q : 0;
  return whole + (up && (q < 128 ? whole << q : 0) != t);
}
// x 2^kBits of a list, where all that matters of a bound past its sums is that it is.
template <int kBits>
SPADE_DEVICE uint64_t widened(uint64_t x) { return x >> (64 - kBits) ? ~0ull : x << kBits; }
// Cumulative mass > u Z is cumulative mass > this.
template <class V>
SPADE_DEVICE V target_of(float u, V total) {
  const V t = part_of(u, total, false);
  return t < total ? t : total - 1;
}
SPADE_DEVICE float unit_of(uint64_t total, int shift) { return __fdiv_rn(static_cast<float>(uint64_t(1) << shift), static_cast<float>(total)); }
// A weight of weight40() times `unit` (2^shift over the sum).
SPADE_DEVICE float share(const Row &w, const uint64_t *powers, float l, float unit) {
  int e;
  const uint64_t v = weight40(w, powers, l, &e);
  return e < 0 ? 0.f : ldexpf(static_cast<float>(v) * unit, -40 - e);
}
// The same for one token, with a rounding less.
SPADE_DEVICE float share_of(const Row &w, const uint64_t *powers, float l, uint64_t total, int shift) {
  int e;
  const uint64_t v = weight40(w, powers, l, &e);
  return e < 0 ? 0.f : ldexpf(__fdiv_rn(static_cast<float>(v), static_cast<float>(total)), shift - 40 - e);
}

// The sum over a warp's lanes on every lane, by the 32-bit reductions of 20, 20 and 24 bits.
SPADE_DEVICE uint64_t warp_sum(uint64_t v) {
  const uint32_t a = __reduce_add_sync(0xffffffffu, static_cast<uint32_t>(v) & 0xfffffu);
  const uint32_t b = __reduce_add_sync(0xffffffffu, static_cast<uint32_t>(v >> 20) & 0xfffffu);
  const uint32_t c = __reduce_add_sync(0xffffffffu, static_cast<uint32_t>(v >> 40));
  return a + (static_cast<uint64_t>(b) << 20) + (static_cast<uint64_t>(c) << 40);
}
// The rank at which tokens in order reach `goal` together (more than any rank if they do not; more than 0 is asked for),
// which lies in [lo, hi] then, by bisection: a thread holds kPer ranks with what each counts.  Every kSteps-th step
// shrinks the range to the ranks that it holds (4 x 32000 fp32 with top-p: 16.7 us, 24.3 without; 18.5 with every sixth).
template <int kPer, class R, class M>
SPADE_DEVICE uint32_t reach(const Team &team, R rank, M mass, uint64_t goal, uint32_t lo, uint32_t hi) {
  int turn = 0;
  for (int step = 0; lo < hi; ++step) {
    uint64_t v;
    if (step % kSteps == kSteps - 1) {
      uint32_t first = ~0u, last = 0;
#pragma unroll
      for (int e = 0; e < kPer; ++e)
        if (mass(e) && rank(e) >= lo && rank(e) <= hi) {
          first = min(first, rank(e));
          last = max(last, rank(e));
        }
      v = static_cast<uint64_t>(__reduce_min_sync(0xffffffffu, first)) << 32 | __reduce_max_sync(0xffffffffu, last);
    } else {
      const uint32_t g = lo + (hi - lo) / 2 + ((hi - lo) & 1);
      v = 0;
#pragma unroll
      for (int e = 0; e < kPer; ++e) v += rank(e) < g ? mass(e) : 0;
      v = warp_sum(v);
    }
    // (Two arrays by turns: one meeting a step.)
    if (team.lane == 0) team.s->sums[turn][team.warp] = v;
    __syncthreads();
    v = team.lane < kWarps ? team.s->sums[turn][team.lane] : 0;
    turn ^= 1;
    if (step % kSteps == kSteps - 1) {
      lo = __reduce_min_sync(0xffffffffu, team.lane < kWarps ? static_cast<uint32_t>(v >> 32) : ~0u);
      hi = __reduce_max_sync(0xffffffffu, static_cast<uint32_t>(v));
    } else {
      const uint32_t g = lo + (hi - lo) / 2 + ((hi - lo) & 1);
      if (warp_sum(v) < goal) lo = g;
      else hi = g - 1;
    }
  }
  __syncthreads();
  return lo;
}

// The leader's part: which of the n listed tokens are kept, and the draw.  keys: order (descending) and index of each.
// A token is kept if fewer than k tokens, and less than top_p of the mass, have a larger logit (ties are kept or
// dropped together), and it reaches tau.  So what is kept are the orders up to one, which is the smallest that any
// bound leaves; each is found by comparing each token with each (n^2: 100 tokens 1 us) or by bisection (n log: 1000
// tokens about 4 us, where a sort took 20).
template <class T>
SPADE_DEVICE void decide(const Params &p, Shared &s, Team &team, const Row &w, float peak, uint64_t *keys, uint64_t *mass, int n,
                         uint64_t out_mass, float bound, const uint8_t *row, int r, int k, float top_p, float u, float tau,
                         bool has_k, bool has_p, bool has_m, float *probs) {
  const int tid = team.tid;
  const uint64_t *powers = s.powers;
  constexpr int kPer = (kList + kThreads - 1) / kThreads;
  const bool pairs = n <= kPairs;
  uint32_t order[kPer], index[kPer];  // of the thread's tokens
  uint64_t own[kPer];                 // and their weights, 0 when dropped
#pragma unroll
  for (int e = 0; e < kPer; ++e) {
    const int i = tid + e * kThreads;
    const uint64_t key = i < n ? keys[i] : ~0ull;
    order[e] = static_cast<uint32_t>(key >> 32);
    index[e] = static_cast<uint32_t>(key);
    own[e] = i < n ? weight<kListShift>(w, powers, number_of(~order[e])) : 0;
  }
  // Orders of listed tokens, without the bits that the type's numbers share.
  const uint32_t least = ~order_of(peak) >> T::kSpare, most_order = ~order_of(bound) >> T::kSpare;
  auto rank = [&](int e) { return order[e] >> T::kSpare; };
  auto weight_of = [&](int e) { return own[e]; };
  uint64_t larger = 0;  // with few tokens, one to a thread: the mass of those with a larger logit, and their number
  int count = 0;
  if (pairs) {
    if (tid < n) mass[tid] = own[0];
    __syncthreads();
    if (tid < n) {
#pragma unroll 4
      for (int j = 0; j < n; ++j)
        if (static_cast<uint32_t>(keys[j] >> 32) < order[0]) {
          larger += mass[j];
          ++count;
        }
    }
    __syncthreads();  // (the masses are written again)
  }
  // Keeps ranks up to `last`.
  auto keep = [&](uint32_t last) {
#pragma unroll
    for (int e = 0; e < kPer; ++e)
      if (rank(e) > last) own[e] = 0;
  };
  auto total_of = [&] {
    uint64_t v = 0;
#pragma unroll
    for (int e = 0; e < kPer; ++e) v += own[e];
    return team.block(v, add64);
  };
  if (has_k) {
    if (pairs) {
      if (count >= k) own[0] = 0;
    } else {
      keep(reach<kPer>(team, rank, [&](int e) -> uint64_t { return tid + e * kThreads < n; }, static_cast<uint64_t>(k), least, most_order));
    }
  }
  if (has_p) {
    uint64_t all = total_of();
    uint64_t goal = part_of(top_p, all, true), most = goal;
    if (!has_k) {
      // The row's mass, in units of 2^-40 and known to 2^-16 of what is not listed: where that does not settle every
      // token, exactly.
      constexpr int kBits = kListShift - 40;
      const uint64_t slack = out_mass >> 16;
      most = widened<kBits>(part_of(top_p, (all >> kBits) + 1 + out_mass + slack + (p.V >> kBits) + 1 + kThreads * kMaxCluster, true));
      goal = widened<kBits>(part_of(top_p, (all >> kBits) + out_mass - slack, false));
    }
    for (int exact = 0; exact < 2; ++exact) {
      bool open = false;
      uint32_t last = 0;
      if (pairs) {
        open = own[0] > 0 && (larger < goal) != (larger < most);
      } else {
        // Tokens up to `last` have what is asked for; there are others, and it may be too little.
        last = reach<kPer>(team, rank, weight_of, goal, least, most_order);
        uint64_t v = 0;
#pragma unroll
        for (int e = 0; e < kPer; ++e) v += rank(e) <= last ? own[e] : 0;
        v = team.block(v, add64);
        open = v < most && v < all;
      }
      if (!__syncthreads_or(open)) {
        if (!pairs) keep(last);
        else if (larger >= goal) own[0] = 0;
        break;
      }
      Mass v = 0;
      for (int i = tid; i < p.V; i += kThreads) {
        uint4 x = make_uint4(0, 0, 0, 0);
        if constexpr (T::kSize == 4) x.x = reinterpret_cast<const uint32_t *>(row)[i];
        else x.x = reinterpret_cast<const uint16_t *>(row)[i];
        v += weight(w, powers, T::number(x, 0));
      }
      // (In the list's units, rounded up: whole numbers reach it where they reach that.)
      constexpr int kBits = kMassShift - kListShift;
      const Mass units = (part_of(top_p, team.block_sum(v), true) + ((1 << kBits) - 1)) >> kBits;
      goal = most = high_of(units) ? ~0ull : low_of(units);
    }
  }
  if (has_m) {
    const uint32_t last = ~order_of(tau);  // (of any fp32 number)
#pragma unroll
    for (int e = 0; e < kPer; ++e)
      if (order[e] > last) own[e] = 0;
  }
  const uint64_t total = total_of();
  const float unit = unit_of(total, kListShift);
  const uint64_t target = target_of(u, total);
  if (probs) {
#pragma unroll
    for (int e = 0; e < kPer; ++e)
      if (tid + e * kThreads < n) probs[index[e]] = own[e] ? share(w, powers, number_of(~order[e]), unit) : 0.f;
  }
  // The draw: cumulative masses in the tokens' own order, up to the one that passes the target.
  uint32_t drawn = 0;
  if (pairs) {
    if (tid < n) mass[tid] = own[0];
    __syncthreads();
    uint64_t before = 0;
    if (tid < n) {
#pragma unroll 4
      for (int j = 0; j < n; ++j) before += static_cast<uint32_t>(keys[j]) < index[0] ? mass[j] : 0;
    }
    drawn = before <= target && target - before < own[0] ? index[0] : ~0u;
  } else {
    drawn = reach<kPer>(team, [&](int e) { return index[e]; }, weight_of, target + 1, 0, static_cast<uint32_t>(p.V) - 1);
  }
#pragma unroll
  for (int e = 0; e < kPer; ++e)
    if (tid + e * kThreads < n && index[e] == drawn) {
      p.tokens[r] = static_cast<int32_t>(drawn);
      if (p.chosen) p.chosen[r] = share_of(w, powers, number_of(~order[e]), total, kListShift);
    }
}

template <class T>
__global__ void __launch_bounds__(kThreads, 3) sample_kernel(const __grid_constant__ Params p) {
  constexpr int E = 16 / T::kSize;
  extern __shared__ __align__(16) uint8_t smem[];
  __shared__ Shared s;
  uint4 *s_vec = reinterpret_cast<uint4 *>(smem);
  Team team;
  team.s = &s;
  team.tid = threadIdx.x;
  team.lane = threadIdx.x & 31;
  team.warp = threadIdx.x >> 5;
  team.rank = blockIdx.x;
  team.size = gridDim.x;
  team.turn = 0;
  const int tid = team.tid, lane = team.lane, warp = team.warp;
  const int r = blockIdx.y;
  // (Nothing is written to another CTA's shared memory before it has started.)
  cluster_arrive();
  if (tid == 0) {
    s.count = 0;
    mbar_init(&s.bar, 1);
    fence_mbar_init();
  }
  if (tid < kBins) s.hist[tid] = 0;
  __syncthreads();
  griddep_wait();
  griddep_launch_dependents();

  // ---- the CTA's part of the row into shared memory ----
  // Whole vectors by bulk copies; the row's first and last, where they hold tokens of others, by elements.
  const uint8_t *row = static_cast<const uint8_t *>(p.logits) + r * p.stride * T::kSize;
  const int lead = static_cast<int>(reinterpret_cast<uintptr_t>(row) & 15) / T::kSize;  // elements before the row in its first vector
  const int nv = (lead + p.V + E - 1) / E;
  const int v0 = min(team.rank * p.slice, nv), v1 = min(v0 + p.slice, nv), n_vec = v1 - v0;
  const int first = v0 * E - lead;  // token of the part's first element
  const int lo_x = max(first, 0), hi_x = min(first + n_vec * E, p.V);  // tokens of this part
  const int a = first < 0 ? 1 : 0, b = first + n_vec * E > p.V ? n_vec - 1 : n_vec;  // whole vectors
  if (warp == 0) {
    const int bytes = max(b - a, 0) * 16;
    if (lane == 0) mbar_arrive_expect_tx(&s.bar, bytes);
    __syncwarp();
    for (int o = lane * kCopyBytes; o < bytes; o += 32 * kCopyBytes)
      bulk_load(smem + a * 16 + o, row + (static_cast<int64_t>(first) + a * E) * T::kSize + o, min(kCopyBytes, bytes - o), &s.bar);
  } else if (warp == 1) {
    // (A part of one vector may be the first and the last.)
    for (int j = 0; j < 2; ++j) {
      const int i = j ? n_vec - 1 : 0;
      if (n_vec == 0 || (j ? b == n_vec || (a && n_vec == 1) : !a)) continue;
      if (lane < E) {
        const int x = first + i * E + lane;
        if constexpr (T::kSize == 4)
          reinterpret_cast<uint32_t *>(s_vec + i)[lane] = x >= 0 && x < p.V ? reinterpret_cast<const uint32_t *>(row)[x] : T::out();
        else
          reinterpret_cast<uint16_t *>(s_vec + i)[lane] = x >= 0 && x < p.V ? reinterpret_cast<const uint16_t *>(row)[x] : T::out();
      }
    }
  }
  // ---- options of the row (under the copies) ----
  int bad = 0;
  float temp = p.temperature ? p.temperature[r] : 1.f;
  if (!(temp >= 0.f && temp <= FLT_MAX)) {
    temp = 1.f;
    bad = SPADE_DEV_BAD_INDEX;
  }
  int k = p.top_k ? p.top_k[r] : 0;
  if (k < 0) bad = SPADE_DEV_BAD_INDEX;
  if (k <= 0 || k > p.V) k = p.V;
  float top_p = p.top_p ? p.top_p[r] : 1.f;
  if (!(top_p > 0.f && top_p <= 1.f)) {
    top_p = 1.f;
    bad = SPADE_DEV_BAD_INDEX;
  }
  float min_p = p.min_p ? p.min_p[r] : 0.f;
  if (!(min_p >= 0.f && min_p <= 1.f)) {
    min_p = 0.f;
    bad = SPADE_DEV_BAD_INDEX;
  }
  float u = p.uniforms[r];
  if (!(u >= 0.f && u < 1.f)) {
    u = u >= 1.f ? 0.99999994f : 0.f;  // the largest below 1
    bad = SPADE_DEV_BAD_INDEX;
  }
  const bool greedy = temp == 0.f;
  const bool has_k = k < p.V, has_p = top_p < 1.f, has_m = min_p > 0.f;
  if (tid < 256) s.powers[tid] = kPowers.v[tid];
  if (tid == 0) {
    s.u = u;
    s.top_p = top_p;
    s.temp = temp;
  }
  if (tid == kThreads - 1 && !greedy) {
    // log2(e) / T as a pair of numbers, the quotient and what it leaves; how far min_p reaches.
    constexpr float kLog2e = 1.44269502162933349609f, kLog2eLow = 1.92596299112661746887e-8f;
    s.scale = temp >= kHuge ? 1.f / kHuge : 1.f;
    const float t = temp * s.scale, q = __fdiv_rn(kLog2e, t);
    s.ch = q;
    s.cl = q <= FLT_MAX ? __fdiv_rn(__fmaf_rn(-q, t, kLog2e) + kLog2eLow, t) : 0.f;
    if (has_m) s.reach = static_cast<double>(temp) * log(static_cast<double>(min_p));
  }
  if (!mbar_wait_unabortable(&s.bar, 0)) atomicOr(p.status, SPADE_DEV_TIMEOUT);
  __syncthreads();

  // ---- the largest logit, and the least of the threads' largest ----
  T tops;
  for (int i = tid; i < n_vec; i += kThreads) tops.take(s_vec[i]);
  const float top = tops.top();
  const bool odd = !(top < INFINITY);  // a NaN or +infinity: gets the largest order
  cluster_wait();
  const uint32_t high = __reduce_max_sync(0xffffffffu, odd ? 0xffffffffu : order_of(top));
  const uint32_t low = __reduce_max_sync(0xffffffffu, top > -INFINITY && !odd ? ~order_of(top) : 0u);
  const uint64_t ends = team.cluster(static_cast<uint64_t>(high) << 32 | low, [](uint64_t x, uint64_t y) {
    const uint32_t hi = max(static_cast<uint32_t>(x >> 32), static_cast<uint32_t>(y >> 32));
    return static_cast<uint64_t>(hi) << 32 | max(static_cast<uint32_t>(x), static_cast<uint32_t>(y));
  });
  const float peak = number_of(static_cast<uint32_t>(ends >> 32));
  float *probs = p.probs ? p.probs + static_cast<int64_t>(r) * p.V : nullptr;
  auto number = [&](int x) {  // token x of this part
    const int i = x - first;
    return T::number(s_vec[i / E], i % E);
  };
  if (ends >> 32 == 0xffffffffull || peak == -INFINITY) {
    // Nothing to draw from.
    if (team.rank == 0 && tid == 0) {
      p.tokens[r] = -1;
      if (p.chosen) p.chosen[r] = 0.f;
      atomicOr(p.status, SPADE_DEV_BAD_INDEX);
    }
    if (probs)
      for (int x = lo_x + tid; x < hi_x; x += kThreads) probs[x] = 0.f;
    return;
  }
  if (bad && team.rank == 0 && tid == 0) atomicOr(p.status, bad);

  if (greedy) {
    uint64_t at = 0xffffffffull;
    if (top == peak)
      for (int i = tid; i < n_vec && at == 0xffffffffull; i += kThreads) {
        const uint4 x = s_vec[i];
#pragma unroll
        for (int e = E - 1; e >= 0; --e)
          if (T::number(x, e) == peak) at = first + i * E + e;
      }
    at = team.cluster(at, [](uint64_t x, uint64_t y) { return x < y ? x : y; });
    if (team.rank == 0 && tid == 0) {
      p.tokens[r] = static_cast<int32_t>(at);
      if (p.chosen) p.chosen[r] = 1.f;
    }
    if (probs)
      for (int x = lo_x + tid; x < hi_x; x += kThreads) probs[x] = x == static_cast<int>(at) ? 1.f : 0.f;
    return;
  }
  Row w;
  w.scale = s.scale;
  w.m = peak * w.scale;
  w.ch = s.ch;
  w.cl = s.cl;
  const uint64_t *powers = s.powers;
  // The least logit that min_p keeps: ln(min_p) T above the largest, rounded up to fp32.
  float tau = -FLT_MAX;
  if (has_m) {
    if (tid == 0) s.tau = __double2float_ru(static_cast<double>(peak) + s.reach);
    __syncthreads();
    tau = fmaxf(tau, s.tau);
  }

  if (has_k || has_p || has_m) {
    // What min_p drops matters to the mass of top-k's tokens only: its bound is tried first.
    const bool by_min_p = has_m && !(has_k && has_p);
    const bool masses = has_p && !has_k;
    for (int attempt = by_min_p ? 0 : 1; attempt < 2; ++attempt) {
      // ---- a bound that enough tokens reach ----
      float bound = by_min_p ? tau : -FLT_MAX;
      bool whole_set = true;  // every token that can be kept is listed
      if (attempt && p.V > kLocal && (has_k || has_p)) {
        const float range = peak - number_of(~static_cast<uint32_t>(ends));
        const float scale = static_cast<float>(kBins) / range;
        if (top > -INFINITY) atomicAdd(&s.hist[static_cast<int>(fminf((peak - top) * scale, static_cast<float>(kBins - 1)))], 1u);
        if (tid == 0) s.cut = kBins;
        cluster_sync();
        // Every CTA adds up all parts' bins and finds the same cut.  A nucleus: as many threads as have kAim tokens
        // when tokens are spread at random, N (1 - e^(-kAim / N)) of N threads.
        const float threads = static_cast<float>(kThreads * team.size);
        const uint32_t wanted = has_k ? static_cast<uint32_t>(k)
                                      : static_cast<uint32_t>(threads * (1.f - __expf(-fminf(kAim, 0.7f * kLocal * team.size) / threads)));
        uint32_t n = 0;
        if (tid < kBins) {
          uint32_t part[kMaxCluster];
#pragma unroll
          for (int c = 0; c < kMaxCluster; ++c) part[c] = c < team.size ? ld_cluster32(cluster_map(&s.hist[tid], c)) : 0;
#pragma unroll
          for (int c = 0; c < kMaxCluster; ++c) n += part[c];
        }
        const uint64_t counted = warp_scan(static_cast<uint64_t>(n), lane);
        if (lane == 31) s.warp[warp] = counted;
        __syncthreads();
        uint64_t count = counted;
        for (int i = 0; i < warp; ++i) count += s.warp[i];
        if (tid < kBins && count >= wanted) atomicMin(&s.cut, tid);
        __syncthreads();
        // (A little lower than the bin's edge, whose tokens it has to let in.)
        const float edge = peak - (static_cast<float>(s.cut) + 1.0005f) * (range * (1.f / kBins));
        if (s.cut < kBins && edge > bound) {
          bound = edge;
          whole_set = false;
        }
      }
      // (The bound that has just listed too many: it would do so again.)
      if (attempt && by_min_p && whole_set) break;
      // ---- the tokens that reach it; roughly, the mass of those and of the others ----
      // (A vector's largest number first: few vectors hold a token of the list.)
      float in = 0.f;
      F2 outs[2] = {f2(0.f, 0.f), f2(0.f, 0.f)};
      const F2 scale = f2(w.scale, w.scale), minus_m = f2(-w.m, -w.m), ch = f2(w.ch, w.ch);
#pragma unroll 2
      for (int i = tid; i < n_vec; i += kThreads) {
        const uint4 x = s_vec[i];
        const bool has = T::largest(x) >= bound;
        float q[E];
        if (masses) {
#pragma unroll
          for (int e = 0; e < E; e += 2) {
            f2_split(f2_mul(f2_fma(f2(T::number(x, e), T::number(x, e + 1)), scale, minus_m), ch), q[e], q[e + 1]);
            q[e] = ex2(q[e]);
            q[e + 1] = ex2(q[e + 1]);
          }
        }
        if (has) {
#pragma unroll
          for (int e = 0; e < E; ++e) {
            const float l = T::number(x, e);
            if (l >= bound) {
              const uint32_t at = atomicAdd(&s.count, 1u);
              if (at < kLocal) s.list[at] = static_cast<uint64_t>(~order_of(l)) << 32 | static_cast<uint32_t>(first + i * E + e);
              if (masses) {
                in += q[e];
                q[e] = 0.f;
              }
            }
          }
        }
        if (masses) {
#pragma unroll
          for (int e = 0; e < E; e += 2) outs[e / 2 & 1] = f2_add(outs[e / 2 & 1], f2(q[e], q[e + 1]));
        }
      }
      // Masses in units of 2^-40 of the largest weight, counts (a part too many counts as too many of all).
      const auto plus = [](float a, float b) { return a + b; };
      if (masses) {
        float a, b, c, d;
        f2_split(outs[0], a, b);
        f2_split(outs[1], c, d);
        in = warp_reduce(in, plus);
        a = warp_reduce((a + b) + (c + d), plus);
        if (lane == 0) {
          s.masses[0][warp] = in;
          s.masses[1][warp] = a;
        }
      }
      __syncthreads();
      const uint32_t mine = s.count;
      uint64_t part[2] = {0, 0};
      if (masses && warp == 0)
        for (int i = 0; i < kWarps; ++i)
          for (int j = 0; j < 2; ++j) part[j] += static_cast<uint64_t>(s.masses[j][i] * 1099511627776.f);
      const uint64_t(*all)[kMaxCluster] = team.exchange(masses ? 3 : 1, mine > kLocal ? kList + 1 : mine, part[0], part[1]);
      uint64_t counts = 0, in_mass = 0, out_mass = 0, ahead = 0;
      for (int c = 0; c < team.size; ++c) {
        if (c < team.rank) ahead += all[0][c];
        counts += all[0][c];
        if (masses) {
          in_mass += all[1][c];
          out_mass += all[2][c];
        }
      }
      // Errors of these sums: an argument of up to 64 rounded three times (64 ln 2 3 2^-24), the power (2^-22), sums of
      // some forty terms (40 2^-24): below 2^-16 in all; and V weights below 2^-64, and what a warp's sum loses as a
      // whole number.
      const bool enough = whole_set || (has_k ? counts >= static_cast<uint64_t>(k)
                                              : in_mass - (in_mass >> 15) >= part_of(s.top_p, in_mass + out_mass + (out_mass >> 15), true));
      if (counts > kList || !enough) {
        if (tid == 0) s.count = 0;  // (read by all before the cluster met)
        __syncthreads();
        continue;
      }
      // ---- one CTA decides: it gets the list; every other token's probability is 0 ----
      uint64_t *keys = reinterpret_cast<uint64_t *>(smem), *mass = keys + kList;
      auto zeros = [&] {
        if (probs)
          for (int x = lo_x + tid; x < hi_x; x += kThreads)
            if (!(number(x) >= bound)) probs[x] = 0.f;
      };
      // (The leader's part makes room for the list: its own zeros come first.)
      if (probs) {
        if (team.rank == 0) zeros();
        cluster_sync();
      }
      for (int i = tid; i < static_cast<int>(mine); i += kThreads) st_cluster(cluster_map(&keys[ahead + i], 0), s.list[i]);
      cluster_sync();
      if (team.rank != 0) {
        zeros();
        return;
      }
      decide<T>(p, s, team, w, peak, keys, mass, static_cast<int>(counts), out_mass, bound, row, r, k, s.top_p, s.u, tau, has_k, has_p, has_m, probs);
      return;
    }
  }
  if (has_k || has_p) {
    // ---- many tokens: rounds of histograms ----
    // The largest `g` (an order without the spare bits) such that tokens from it on reach `goal`, in counts or masses;
    // tokens are those from `lo` on, which reach it unless there are too few (then lo).
    auto boundary = [&](uint32_t lo, Mass goal, bool masses) {
      uint32_t hi = (order_of(peak) >> T::kSpare) + 1;
      Mass above = 0;  // of tokens from hi on
      // First round: bins of equal width, to 24 T below the largest logit (or as far as the threads' largest reach).
      const float width = fmaxf(fminf(24.f * s.temp, FLT_MAX), peak - number_of(~static_cast<uint32_t>(ends))) * (1.f / kBins);
      const float scale = __fdiv_rn(1.f, width);
      bool by_value = scale > 0.f && scale <= FLT_MAX;
      for (int turn = 0; hi - lo > 1; turn ^= 1) {
        if (tid < kBins) s.hist[tid] = s.mid[tid] = s.high[tid] = 0;
        if (tid == 0) s.cuts[turn] = kBins;
        __syncthreads();
        int shift = 0;
        while ((hi - 1 - lo) >> shift >= kBins) ++shift;
        // Bin b begins at the order top_of(b), the first below the bin before.
        auto top_of = [&](int b) { return by_value ? order_of(fmaf(static_cast<float>(-b), width, peak)) >> T::kSpare : hi - 1 - (static_cast<uint32_t>(b) << shift); };
        for (int i = tid; i < n_vec; i += kThreads) {
          const uint4 x = s_vec[i];
#pragma unroll
          for (int e = 0; e < E; ++e) {
            const float l = T::number(x, e);
            const uint32_t g = order_of(l) >> T::kSpare;
            if (g < lo || g >= hi) continue;
            int b;
            if (by_value) {
              b = static_cast<int>(fminf((peak - l) * scale, static_cast<float>(kBins - 1)));
              while (b > 0 && g > top_of(b)) --b;
              while (b < kBins - 1 && g <= top_of(b + 1)) ++b;
            } else {
              b = (hi - 1 - g) >> shift;
            }
            if (masses) {
              // (The third word takes what a bin of sixteen largest weights carries over.)
              const uint64_t q = weight(w, powers, l);
              const uint32_t low = static_cast<uint32_t>(q), old = atomicAdd(&s.hist[b], low);
              const uint32_t mid = static_cast<uint32_t>(q >> 32) + (old + low < old);
              if (mid) {
                const uint32_t was = atomicAdd(&s.mid[b], mid);
                if (was + mid < was) atomicAdd(&s.high[b], 1u);
              }
            } else {
              atomicAdd(&s.hist[b], 1u);
            }
          }
        }
        cluster_sync();
        Mass n = 0;
        if (tid < kBins)
          for (int c = 0; c < team.size; ++c) {
            const uint32_t low = ld_cluster32(cluster_map(&s.hist[tid], c));
            const uint64_t mid = ld_cluster32(cluster_map(&s.mid[tid], c));
            n += mass_of(mid << 32 | low, ld_cluster32(cluster_map(&s.high[tid], c)));
          }
        const Mass incl = warp_scan(n, lane);
        if (lane == 31) s.wide[warp] = incl;
        __syncthreads();
        Mass upto = above + incl;
        for (int i = 0; i < warp; ++i) upto += s.wide[i];
        if (tid < kBins && upto >= goal && upto - n < goal) {
          s.cuts[turn] = tid;
          s.above[turn] = upto - n;
        }
        cluster_sync();  // (the bins have been read by all)
        const int cut = s.cuts[turn];
        if (cut == kBins) return lo;
        above = s.above[turn];
        const uint32_t top = cut ? top_of(cut) + 1 : hi;
        if (by_value ? cut < kBins - 1 : static_cast<uint64_t>(cut + 1) << shift <= hi - 1 - lo) lo = max(lo, top_of(cut + 1) + 1);
        hi = min(hi, top);
        by_value = false;
      }
      return lo;
    };
    uint32_t edge = order_of(-FLT_MAX) >> T::kSpare;
    if (has_k) edge = boundary(edge, static_cast<Mass>(k), false);
    if (has_p) {
      Mass whole = 0;
      for (int i = tid; i < n_vec; i += kThreads) {
        const uint4 x = s_vec[i];
#pragma unroll
        for (int e = 0; e < E; ++e) {
          const float l = T::number(x, e);
          if (order_of(l) >> T::kSpare >= edge) whole += weight(w, powers, l);
        }
      }
      whole = team.cluster_sum(whole);
      edge = boundary(edge, part_of(s.top_p, whole, true), true);
    }
    tau = fmaxf(tau, number_of(edge << T::kSpare));
  }

  // ---- draw in ascending order: sums of warps' stretches, of CTAs, then the stretch again ----
  const int per = (p.slice + kWarps - 1) / kWarps;
  const int w0 = min(warp * per, n_vec), w1 = min(w0 + per, n_vec);
  uint64_t total = 0;  // in units of 2^-40 where it is exact
  // With sums of type M: exact ones, or 64 bits of weights known to 2^-20.  False: those do not settle the token.
  auto draw = [&](auto sums) -> bool {
    using M = decltype(sums);
    constexpr bool exact = sizeof(M) > 8;
    const float units = static_cast<float>(uint64_t(1) << p.shift);
    auto token_mass = [&](float l) -> uint64_t {
      if (!(l >= tau)) return 0;
      if constexpr (exact) return weight(w, powers, l);
      else return __float2ull_rn(weight_about<T::kSize == 4>(w, l) * units);
    };
    auto lane_mass = [&](int i) {  // of vector i's kept tokens
      uint64_t m = 0;
      if (i < w1) {
        const uint4 x = s_vec[i];
        if constexpr (exact) {
#pragma unroll
          for (int e = 0; e < E; ++e) m += token_mass(T::number(x, e));
        } else {
          float q = 0.f;
#pragma unroll
          for (int e = 0; e < E; ++e) {
            const float l = T::number(x, e);
            const float a = weight_about<T::kSize == 4>(w, l);
            q += l >= tau ? a : 0.f;
          }
          m = __float2ull_rn(q * units);
        }
      }
      return m;
    };
    M mine = 0;
    for (int i = w0 + lane; i < w1; i += 32) mine += lane_mass(i);
    mine = warp_add(mine);
    if (lane == 0) s.wide[warp] = mine;
    if (tid == 0) s.settled = 0;
    __syncthreads();
    M before = 0, part = 0;
    for (int i = 0; i < kWarps; ++i) {
      const M m = static_cast<M>(s.wide[i]);
      if (i < warp) before += m;
      part += m;
    }
    const uint64_t(*parts)[kMaxCluster] = team.exchange(exact ? 2 : 1, low_of(part), exact ? high_of(part) : 0, 0);
    M all = 0;
    for (int c = 0; c < team.size; ++c) {
      const M m = exact ? static_cast<M>(mass_of(parts[0][c], parts[1][c])) : static_cast<M>(parts[0][c]);
      if (c < team.rank) before += m;
      all += m;
    }
    total = exact ? low_of(all >> (kMassShift - 40)) : low_of(all);
    // A token's end and the target differ by the weights before it times 1 - u less those behind times u: that is off by
    // 2 u (1 - u) <= 1/2 of the weights' errors, 2^-20 and little more of the whole (roundings to units: one a token).
    const M target = target_of(s.u, all), margin = exact ? 0 : static_cast<M>((low_of(all) >> 20) + p.V);
    if (target >= before && target < before + mine) {
      for (int i0 = w0; i0 < w1; i0 += 32) {
        const M m = lane_mass(i0 + lane), upto = before + warp_scan(m, lane);
        const unsigned hit = __ballot_sync(0xffffffffu, upto > target);
        if (hit) {
          if (lane == __ffs(hit) - 1) {
            M at = upto - m;
            for (int e = 0; e < E; ++e) {
              const int x = first + (i0 + lane) * E + e;
              if (x < lo_x || x >= hi_x) continue;
              const M q = token_mass(number(x));
              if (at + q > target) {
                if (exact || (target >= at + margin && at + q >= target + margin)) {
                  s.settled = 1;
                  p.tokens[r] = x;
                  if (p.chosen) p.chosen[r] = share_of(w, powers, number(x), total, exact ? 40 : p.shift);
                }
                break;
              }
              at += q;
            }
          }
          break;
        }
        before = last_lane(upto);
      }
    }
    if constexpr (exact) {
      return true;
    } else {
      __syncthreads();
      const uint64_t *done = team.exchange(1, s.settled, 0, 0)[0];
      uint64_t settled = 0;
      for (int c = 0; c < team.size; ++c) settled += done[c];
      return settled != 0;
    }
  };
  // Weights to 2^-20 first (sums of eight 2^-21): they settle the token where the target is further than their errors
  // from its ends.  (With probabilities asked for, exact ones at once.)
  if (!probs && draw(uint64_t())) return;
  draw(Mass());
  if (probs) {
    const float unit = unit_of(total, 40);
    for (int x = lo_x + tid; x < hi_x; x += kThreads) {
      const float l = number(x);
      probs[x] = l >= tau ? share(w, powers, l, unit) : 0.f;
    }
  }
}

// Sizes of a launch: the fewest CTAs whose parts leave room for three on an SM; more while few rows leave
// SMs idle and a part is longer than a few vectors a thread.
static bool plan(int V, int size, int R, int sms, int *ctas, int *slice) {
  const int per = 16 / size;
  const int64_t nv = (static_cast<int64_t>(V) + per - 1 + per - 1) / per;
  auto part = [&](int n) { return static_cast<int>((nv + n - 1) / n); };
  int c = 1;
  while (c < kMaxCluster && part(c) * int64_t(16) > kSliceBytes) ++c;
  while (c < kMaxCluster && static_cast<int64_t>(R) * (c + 1) <= sms && part(c) > 2 * kThreads) ++c;
  *ctas = c;
  *slice = part(c);
  return part(c) * int64_t(16) <= kMaxSliceBytes;
}

template <class T>
static cudaError_t run(const Params &p, int R, int ctas, cudaStream_t stream) {
  auto kern = sample_kernel<T>;
  static OncePerDevice once, wide;
  cudaError_t e = set_max_smem(once, kMaxSliceBytes, kern);
  if (e != cudaSuccess) return e;
  int dev = 0;
  e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  e = wide(dev, [&] { return cudaFuncSetAttribute(kern, cudaFuncAttributeNonPortableClusterSizeAllowed, 1); });
  if (e != cudaSuccess) return e;
  const size_t bytes = static_cast<size_t>(p.slice) * 16;
  return launch(kern, dim3(ctas, R), ctas, kThreads, bytes < kMinBytes ? kMinBytes : bytes, stream, p);
}

}  // namespace sample
}  // namespace spade

using namespace spade;

extern "C" spade_status spade_sample(const void *logits, int32_t dtype, int64_t row_stride, const float *uniforms,
                                     const float *temperature, const int32_t *top_k, const float *top_p,
                                     const float *min_p, int32_t *tokens, float *probs, float *chosen, int32_t R, int32_t V,
                                     int32_t *status, spade_stream_t stream) {
  static const char *name = "spade_sample";
  if (!logits || !uniforms || !tokens || !status) return fail(SPADE_ERR_INVALID_ARG, "%s: null pointer argument", name);
  if (R <= 0 || V <= 0) return fail(SPADE_ERR_INVALID_ARG, "%s: non-positive size", name);
  if (dtype < SPADE_F32 || dtype > SPADE_F16) return fail(SPADE_ERR_INVALID_ARG, "%s: unknown dtype %d", name, dtype);
  if (row_stride < V) return fail(SPADE_ERR_INVALID_ARG, "%s: row stride %lld < V = %d", name, static_cast<long long>(row_stride), V);
  if (R > 65535) return fail(SPADE_ERR_SHAPE, "%s: R = %d exceeds 65535 rows per call", name, R);
  const int size = dtype == SPADE_F32 ? 4 : 2;
  if (!aligned(logits, size)) return fail(SPADE_ERR_INVALID_ARG, "%s: logits must be aligned to their type", name);
  sample::Params p;
  int ctas = 0;
  // (The limit on V does not depend on the device.)
  if (!sample::plan(V, size, R, 0, &ctas, &p.slice))
    return fail(SPADE_ERR_SHAPE, "%s: rows of %d entries do not fit the shared memory of %d CTAs", name, V, sample::kMaxCluster);
  int sms = 0;
  const spade_status st = device_info(&sms, nullptr);
  if (st != SPADE_OK) return st;
  sample::plan(V, size, R, sms, &ctas, &p.slice);
  p.logits = logits; p.stride = row_stride; p.uniforms = uniforms; p.temperature = temperature; p.top_k = top_k;
  p.top_p = top_p; p.min_p = min_p; p.tokens = tokens; p.probs = probs; p.chosen = chosen; p.status = status; p.V = V;
  // (The rough draw's sum of V weights of up to 2^shift stays below 2^62.)
  int bits = 0;
  while ((int64_t(1) << bits) < V) ++bits;
  p.shift = 62 - bits < 44 ? 62 - bits : 44;
  cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
  const cudaError_t e = dtype == SPADE_F32    ? sample::run<sample::Tops32>(p, R, ctas, s)
                        : dtype == SPADE_BF16 ? sample::run<sample::Tops16<true>>(p, R, ctas, s)
                                              : sample::run<sample::Tops16<false>>(p, R, ctas, s);
  return e == cudaSuccess ? SPADE_OK : cuda_fail(e, name);
}
