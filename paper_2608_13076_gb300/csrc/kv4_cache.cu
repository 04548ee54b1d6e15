// kv4_cache.cu -- the paged 4-bit KV cache of the verify step: the verify block's
// heads normed, rotated and stored into it (the input side of the attention in
// x_{l+1} = x_l + f_l(x_l), Sec. III-A), the commit of accepted positions
// (Algorithm 1's context update), and reading slots back.
//
// A head's D dims lie on D / 8 lanes, eight neighbours each: a lane's 16-byte load
// is its part of the head, its codes are one 32-bit word, a quantisation group is
// eight lanes, and the rotation's partner (dim j + D/2) is D / 16 lanes away.
#include <cfloat>

#include "int4.cuh"
#include "internal.h"
#include "launch.h"
#include "ptx.cuh"

namespace spade {
namespace kv4 {

using int4::Cache;

constexpr int kThreads = 256;
constexpr int kWarps = kThreads / 32;

struct NormRope {
  Cache cache;
  const __nv_bfloat16 *qkv, *q_norm, *k_norm;
  const float4 *rope;  // two (cos, sin) pairs each
  __nv_bfloat16 *q_out;
  const int32_t *ctx_lens, *n_draft, *cu_q;
  int32_t *status;
  int R, Hq, max_pos, max_k;
  int parts;           // warps that share a row
  float eps;
};

// Eight bf16 of a 16-byte vector.
SPADE_DEVICE void unpack8(const uint4 &v, float (&x)[8]) {
  const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    x[2 * e] = __uint_as_float(w[e] << 16);
    x[2 * e + 1] = __uint_as_float(w[e] & 0xffff0000u);
  }
}
SPADE_DEVICE uint4 pack8(const float (&x)[8]) {
  return make_uint4(pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3]), pack_bf16(x[4], x[5]), pack_bf16(x[6], x[7]));
}

// Why sequence b's block cannot be stored (0: it can).
SPADE_DEVICE int block_error(const NormRope &p, int ctx, int k, int q0, int q1) {
  if (ctx < 0 || k < 0 || k > p.max_k || q0 < 0 || q1 > p.R || q1 - q0 != k + 1) return SPADE_DEV_BAD_INDEX;
  const int64_t end = static_cast<int64_t>(ctx) + k + 1;
  if (end > p.cache.capacity()) return SPADE_DEV_CAPACITY;
  return end > p.max_pos ? SPADE_DEV_BAD_INDEX : 0;
}

// x / s for a scale s, correctly rounded: with y = 1 / s correctly rounded and q = x y,
// q + (x - q s) y is (Markstein, IBM J. Res. Dev. 34, 1990; the significand of s, a
// float16, is not all ones).  Three operations for a division's dozen.
SPADE_DEVICE float divided(float x, float s, float y) {
  const float q = __fmul_rn(x, y);
  return __fmaf_rn(__fmaf_rn(-q, s, x), y, q);
}

// Group of 64 dims (eight lanes): the lane's code word and the group's pair.
SPADE_DEVICE void quantise(const float (&x)[8], uint32_t &codes, uint32_t &pair) {
  float lo = 0.f, hi = 0.f, none = 0.f;
#pragma unroll
  for (int e = 0; e < 8; e += 2) {
    lo = min3(lo, x[e], x[e + 1]);
    hi = max3(hi, x[e], x[e + 1]);
    none = __fmaf_rn(x[e], 0.f, __fmaf_rn(x[e + 1], 0.f, none));  // NaN for an infinity or a NaN
  }
  const bool finite = none == 0.f;
#pragma unroll
  for (int o = 1; o < 8; o *= 2) {
    lo = fminf(lo, __shfl_xor_sync(0xffffffffu, lo, o));
    hi = fmaxf(hi, __shfl_xor_sync(0xffffffffu, hi, o));
  }
  const unsigned vote = __ballot_sync(0xffffffffu, finite) >> (threadIdx.x & 24) & 0xffu;
  // (hi - lo overflows for spans past fp32's range: infinity, cut like any other.)
  const __half hs = __float2half_rn(fminf(__fmul_rn(__fsub_rn(hi, lo), 1.f / 15.f), int4::kMaxScale));
  const float s = __half2float(hs);
  const bool real = vote == 0xffu && s > 0.f;
  const float y = __frcp_rn(real ? s : 1.f);
  constexpr float kWhole = 12582912.f;  // 1.5 2^23: adding it rounds to a whole number, ties to even
  const float z = real ? fminf(divided(-lo, s, y) + kWhole - kWhole, 15.f) : 0.f;
  // A quotient within -z .. 15 - z rounds to within them (they are whole), and the fields'
  // sum needs no mask: kWhole's bits and z go in and out of all eight at once.
  uint32_t w = static_cast<uint32_t>(static_cast<int>(z)) * 0x11111111u - 0x11111111u * __float_as_uint(kWhole);
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const float q = fminf(fmaxf(divided(x[e], s, y), -z), 15.f - z);
    w += __float_as_uint(q + kWhole) << (4 * ((e >> 1) + 4 * (e & 1)));
  }
  codes = real ? w : 0u;
  const __half2 h = __halves2half2(vote == 0xffu ? hs : __ushort_as_half(0x7fff), __float2half_rn(z));
  pair = *reinterpret_cast<const uint32_t *>(&h);
}

// A warp takes kHeads x 32 / (D / 8) heads of one row, all their loads in flight at once;
// the rotation's angles, the same for every head, stay in registers.  Bound by the bytes:
// a row's heads once in, the queries out in bf16 and the rest in 4 bits.  (One group of
// heads per warp, a quantisation of every head, queries too, and a division per number:
// 12288 rows of 32 + 8 + 8 heads took 204 us; they take 77, issue slots 68 % and DRAM 36 % busy.)
template <int D, int kHeads>
__global__ void __launch_bounds__(kThreads) norm_rope_kernel(const __grid_constant__ NormRope p) {
  constexpr int kLanes = D / 8;          // lanes of a head
  constexpr int kSlots = 32 / kLanes;    // heads side by side in a warp
  const int b = blockIdx.y;
  const int lane = threadIdx.x & 31;
  const int item = blockIdx.x * kWarps + (threadIdx.x >> 5);
  const int i = item / p.parts, part = item - i * p.parts;
  griddep_wait();
  griddep_launch_dependents();
  const int ctx = p.ctx_lens[b], k = p.n_draft[b], q0 = p.cu_q[b], q1 = p.cu_q[b + 1];
  const int err = block_error(p, ctx, k, q0, q1);
  if (err) {
    if (item == 0 && lane == 0) atomicOr(p.status, err);
    return;
  }
  if (i > k) return;
  const int pos = ctx + i;
  const int row = q0 + i;
  const int sub = lane / kLanes, l = lane % kLanes;
  const int Hkv = p.cache.Hkv, heads = p.Hq + 2 * Hkv;
  const int h0 = part * kSlots * kHeads + sub;
  const uint4 *src = reinterpret_cast<const uint4 *>(p.qkv) + static_cast<int64_t>(row) * heads * kLanes + l;
  uint4 in[kHeads];
#pragma unroll
  for (int j = 0; j < kHeads; ++j) {
    const int h = h0 + j * kSlots;
    in[j] = h < heads ? src[h * kLanes] : make_uint4(0, 0, 0, 0);
  }
  // cos and sin of the lane's eight dims (the second half of the dims repeats the first's): a
  // dim of the first half becomes own cos - other sin, one of the second own cos + other sin,
  // so the sine carries the sign.
  const bool second = l >= kLanes / 2;
  float cs[8], sn[8];
  const float4 *turn = p.rope + (static_cast<int64_t>(pos) * (D / 2) + (l % (kLanes / 2)) * 8) / 2;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const float4 t = turn[e];
    cs[2 * e] = t.x;
    sn[2 * e] = second ? t.y : -t.y;
    cs[2 * e + 1] = t.z;
    sn[2 * e + 1] = second ? t.w : -t.w;
  }
  const bool stores = (part + 1) * kSlots * kHeads > p.Hq;  // the warp has key or value heads
  const int64_t slot = stores ? p.cache.row(b, pos) : 0;
  if (slot < 0 && lane == 0) atomicOr(p.status, SPADE_DEV_BAD_INDEX);
#pragma unroll
  for (int j = 0; j < kHeads; ++j) {
    const int h = h0 + j * kSlots;
    if (h - sub >= heads) break;
    float x[8];
    unpack8(in[j], x);
    const bool is_q = h < p.Hq, is_v = h >= p.Hq + Hkv;
    // (The shuffles are the whole warp's, whatever its heads are.)
    if (!__all_sync(0xffffffffu, is_v)) {
      const __nv_bfloat16 *weight = is_q ? p.q_norm : p.k_norm;
      float sum = 0.f;
#pragma unroll
      for (int e = 0; e < 8; ++e) sum = fmaf(x[e], x[e], sum);
#pragma unroll
      for (int o = 1; o < kLanes; o *= 2) sum += __shfl_xor_sync(0xffffffffu, sum, o);
      if (!is_v && weight) {
        const float r = rsqrtf(__fadd_rn(sum * (1.f / D), p.eps));
        float w[8];
        unpack8(reinterpret_cast<const uint4 *>(weight)[l], w);
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = __fmul_rn(__fmul_rn(x[e], r), w[e]);
      }
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float other = __shfl_xor_sync(0xffffffffu, x[e], kLanes / 2);
        if (!is_v) x[e] = __fadd_rn(__fmul_rn(x[e], cs[e]), __fmul_rn(other, sn[e]));
      }
    }
    if (is_q) reinterpret_cast<uint4 *>(p.q_out)[(static_cast<int64_t>(row) * p.Hq + h) * kLanes + l] = pack8(x);
    if (__all_sync(0xffffffffu, is_q)) continue;
    uint32_t code, pair;
    quantise(x, code, pair);
    if (h < heads && !is_q && slot >= 0) {
      const int64_t r = slot + static_cast<int64_t>(h - p.Hq - (is_v ? Hkv : 0)) * p.cache.page_size;
      reinterpret_cast<uint32_t *>(is_v ? p.cache.v_codes : p.cache.k_codes)[r * kLanes + l] = code;
      if (l % 8 == 0) (is_v ? p.cache.v_params : p.cache.k_params)[r * (D / int4::kKvGroup) + l / 8] = pair;
    }
  }
}

// ---- commit --------------------------------------------------------------------------------
// One CTA per sequence: every thread reads ctx_lens[b] before one writes new_ctx_lens[b],
// which may be the same word.
__global__ void __launch_bounds__(kThreads) commit_kernel(const __grid_constant__ Cache c, const int32_t *ctx_lens,
                                                         const int32_t *accepted, const int32_t *n_draft,
                                                         int32_t *new_ctx_lens, int32_t *status) {
  const int b = blockIdx.x;
  griddep_wait();
  griddep_launch_dependents();
  const int ctx = ctx_lens[b], a = accepted[b], k = n_draft[b];
  int bad = 0;
  if (ctx < 0 || k < 0 || a < 0 || a > k) bad = SPADE_DEV_BAD_INDEX;
  else if (static_cast<int64_t>(ctx) + k + 1 > c.capacity()) bad = SPADE_DEV_CAPACITY;
  const int lo = bad ? 0 : ctx + a + 1, n = bad ? 0 : k - a;
  // Every page of the rejected slots must exist before anything is cleared.
  int missing = 0;
  for (int s = threadIdx.x; s < n; s += kThreads) missing |= c.row(b, lo + s) < 0;
  if (__syncthreads_or(missing)) bad = SPADE_DEV_BAD_INDEX;
  if (threadIdx.x == 0) {
    new_ctx_lens[b] = bad ? ctx : lo;
    if (bad) atomicOr(status, bad);
  }
  if (bad) return;
  // A warp per slot: its heads' code words and pairs.
  const int words = c.D / 8, pairs = c.D / int4::kKvGroup, per = words + pairs;
  const int lane = threadIdx.x & 31;
  for (int s = threadIdx.x >> 5; s < n; s += kWarps) {
    const int64_t slot = c.row(b, lo + s);
    for (int e = lane; e < c.Hkv * per; e += 32) {
      const int h = e / per, j = e - h * per;
      const int64_t at = slot + static_cast<int64_t>(h) * c.page_size;
      if (j < words) {
        reinterpret_cast<uint32_t *>(c.k_codes)[at * words + j] = 0;
        reinterpret_cast<uint32_t *>(c.v_codes)[at * words + j] = 0;
      } else {
        c.k_params[at * pairs + j - words] = 0;
        c.v_params[at * pairs + j - words] = 0;
      }
    }
  }
}

// ---- read ----------------------------------------------------------------------------------
// Warps stride the slots: warp w takes part w % parts (32 / (D / 8) heads of keys and
// values) of slots w / parts, + step, ...  (12288 rows of 8 heads: 17 us, 3.8 TB/s.)
template <int D>
__global__ void __launch_bounds__(kThreads) read_kernel(const __grid_constant__ Cache c, const int32_t *starts,
                                                       const int32_t *cu_rows, uint4 *k_out, uint4 *v_out, int R,
                                                       int parts, int32_t *status) {
  constexpr int kLanes = D / 8;
  const int b = blockIdx.y;
  griddep_wait();
  griddep_launch_dependents();
  const int s0 = starts[b], r0 = cu_rows[b], r1 = cu_rows[b + 1];
  int bad = 0;
  if (s0 < 0 || r0 < 0 || r1 < r0 || r1 > R) bad = SPADE_DEV_BAD_INDEX;
  else if (static_cast<int64_t>(s0) + (r1 - r0) > c.capacity()) bad = SPADE_DEV_CAPACITY;
  if (bad) {
    if (blockIdx.x == 0 && threadIdx.x == 0) atomicOr(status, bad);
    return;
  }
  const int lane = threadIdx.x & 31, w = blockIdx.x * kWarps + (threadIdx.x >> 5);
  const int part = w % parts, step = gridDim.x * kWarps / parts;
  const int h = part * (32 / kLanes) + lane / kLanes, l = lane % kLanes;
  for (int64_t i = w / parts; i < r1 - r0; i += step) {
    const int64_t slot = c.row(b, s0 + static_cast<int>(i));
    if (slot < 0 && part == 0 && lane == 0) atomicOr(status, SPADE_DEV_BAD_INDEX);
    if (h >= c.Hkv) continue;
    const int64_t at = slot + static_cast<int64_t>(h) * c.page_size;
    uint32_t word[2] = {}, pair[2] = {};
    if (slot >= 0) {
      word[0] = reinterpret_cast<const uint32_t *>(c.k_codes)[at * kLanes + l];
      word[1] = reinterpret_cast<const uint32_t *>(c.v_codes)[at * kLanes + l];
      pair[0] = c.k_params[at * (D / int4::kKvGroup) + l / 8];
      pair[1] = c.v_params[at * (D / int4::kKvGroup) + l / 8];
    }
#pragma unroll
    for (int kv = 0; kv < 2; ++kv) {
      const float2 p = int4::pair_of(pair[kv]);
      float x[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) x[e] = p.x * (static_cast<float>(int4::code_of(word[kv], e)) - p.y);
      (kv ? v_out : k_out)[((r0 + i) * c.Hkv + h) * kLanes + l] = pack8(x);
    }
  }
}

// The checks that every call on the cache makes.
static spade_status check_cache(const char *name, const Cache &c, int B) {
  if (!c.k_codes || !c.k_params || !c.v_codes || !c.v_params || !c.block_table)
    return fail(SPADE_ERR_INVALID_ARG, "%s: null pointer argument", name);
  if (B <= 0 || c.Hkv <= 0 || c.page_size <= 0 || c.num_pages <= 0 || c.max_pages <= 0)
    return fail(SPADE_ERR_INVALID_ARG, "%s: non-positive size", name);
  if (c.D != 64 && c.D != 128) return fail(SPADE_ERR_SHAPE, "%s: head dim %d not supported (64 or 128)", name, c.D);
  if (c.page_size % 64) return fail(SPADE_ERR_SHAPE, "%s: page size %d must be a multiple of 64", name, c.page_size);
  if (B > 65535) return fail(SPADE_ERR_SHAPE, "%s: B = %d exceeds 65535 sequences per call", name, B);
  if (static_cast<int64_t>(c.max_pages) * c.page_size >= (int64_t(1) << 31))
    return fail(SPADE_ERR_CAPACITY, "%s: max_pages * page_size exceeds 2^31", name);
  if (!aligned(c.k_codes, 16) || !aligned(c.k_params, 16) || !aligned(c.v_codes, 16) || !aligned(c.v_params, 16))
    return fail(SPADE_ERR_INVALID_ARG, "%s: pools must be 16-byte aligned", name);
  return SPADE_OK;
}

static Cache cache_of(const void *k_codes, const void *k_params, const void *v_codes, const void *v_params,
                      const int32_t *block_table, int Hkv, int D, int page_size, int num_pages, int max_pages) {
  Cache c;
  c.k_codes = static_cast<uint8_t *>(const_cast<void *>(k_codes));
  c.v_codes = static_cast<uint8_t *>(const_cast<void *>(v_codes));
  c.k_params = static_cast<uint32_t *>(const_cast<void *>(k_params));
  c.v_params = static_cast<uint32_t *>(const_cast<void *>(v_params));
  c.block_table = block_table;
  c.Hkv = Hkv; c.D = D; c.page_size = page_size; c.num_pages = num_pages; c.max_pages = max_pages;
  return c;
}

}  // namespace kv4
}  // namespace spade

using namespace spade;

extern "C" spade_status spade_verify_qk_norm_rope_kv4(
    const void *qkv, const void *q_norm, const void *k_norm, const float *rope, void *q_out, void *k_codes,
    void *k_params, void *v_codes, void *v_params, const int32_t *block_table, const int32_t *ctx_lens,
    const int32_t *n_draft, const int32_t *cu_q, int32_t B, int32_t R, int32_t Hq, int32_t Hkv, int32_t D,
    int32_t page_size, int32_t num_pages, int32_t max_pages, int32_t max_pos, int32_t max_k, float eps,
    int32_t *status, spade_stream_t stream) {
  static const char *name = "spade_verify_qk_norm_rope_kv4";
  if (!qkv || !rope || !q_out || !ctx_lens || !n_draft || !cu_q || !status)
    return fail(SPADE_ERR_INVALID_ARG, "%s: null pointer argument", name);
  kv4::NormRope p;
  p.cache = kv4::cache_of(k_codes, k_params, v_codes, v_params, block_table, Hkv, D, page_size, num_pages, max_pages);
  spade_status st = kv4::check_cache(name, p.cache, B);
  if (st != SPADE_OK) return st;
  if (R <= 0 || Hq <= 0 || max_pos <= 0 || max_k < 0)
    return fail(SPADE_ERR_INVALID_ARG, "%s: non-positive size", name);
  if (Hq % Hkv) return fail(SPADE_ERR_SHAPE, "%s: Hq (%d) must be a multiple of Hkv (%d)", name, Hq, Hkv);
  if (R < B) return fail(SPADE_ERR_INVALID_ARG, "%s: R = %d < B = %d", name, R, B);
  if (!(eps >= 0.f && eps <= FLT_MAX)) return fail(SPADE_ERR_INVALID_ARG, "%s: eps must be finite and >= 0", name);
  if (!aligned(qkv, 16) || !aligned(q_out, 16) || !aligned(q_norm, 16) || !aligned(k_norm, 16) || !aligned(rope, 16))
    return fail(SPADE_ERR_INVALID_ARG, "%s: pointers must be 16-byte aligned", name);
  int sms = 0;
  st = device_info(&sms, nullptr);
  if (st != SPADE_OK) return st;
  p.qkv = static_cast<const __nv_bfloat16 *>(qkv);
  p.q_norm = static_cast<const __nv_bfloat16 *>(q_norm);
  p.k_norm = static_cast<const __nv_bfloat16 *>(k_norm);
  p.rope = reinterpret_cast<const float4 *>(rope);
  p.q_out = static_cast<__nv_bfloat16 *>(q_out);
  p.ctx_lens = ctx_lens; p.n_draft = n_draft; p.cu_q = cu_q; p.status = status;
  p.R = R; p.Hq = Hq; p.max_pos = max_pos; p.max_k = max_k; p.eps = eps;
  // Heads of a warp: one group of them while the rows are few (latency), four when the
  // warps fill the GPU either way.
  const int slots = 256 / D, heads = Hq + 2 * Hkv;
  const bool many = static_cast<int64_t>(R) * heads / (4 * slots) >= 16 * static_cast<int64_t>(sms);
  p.parts = (heads + slots * (many ? 4 : 1) - 1) / (slots * (many ? 4 : 1));
  // A block longer than the rows given cannot be valid.
  const int64_t longest = (max_k < R ? max_k : R - 1) + int64_t(1);
  const int64_t items = longest * p.parts;
  if (items > (int64_t(1) << 31) - kv4::kWarps) return fail(SPADE_ERR_CAPACITY, "%s: too many rows per sequence", name);
  const dim3 grid(static_cast<unsigned>((items + kv4::kWarps - 1) / kv4::kWarps), B);
  auto kern = D == 64 ? (many ? kv4::norm_rope_kernel<64, 4> : kv4::norm_rope_kernel<64, 1>)
                      : (many ? kv4::norm_rope_kernel<128, 4> : kv4::norm_rope_kernel<128, 1>);
  const cudaError_t e = launch(kern, grid, 1, kv4::kThreads, 0, reinterpret_cast<cudaStream_t>(stream), p);
  return e == cudaSuccess ? SPADE_OK : cuda_fail(e, "verify_qk_norm_rope_kv4 launch");
}

extern "C" spade_status spade_kv_commit_kv4(void *k_codes, void *k_params, void *v_codes, void *v_params,
                                            const int32_t *block_table, const int32_t *ctx_lens,
                                            const int32_t *accepted_len, const int32_t *n_draft,
                                            int32_t *new_ctx_lens, int32_t B, int32_t Hkv, int32_t D,
                                            int32_t page_size, int32_t num_pages, int32_t max_pages, int32_t *status,
                                            spade_stream_t stream) {
  static const char *name = "spade_kv_commit_kv4";
  if (!ctx_lens || !accepted_len || !n_draft || !new_ctx_lens || !status)
    return fail(SPADE_ERR_INVALID_ARG, "%s: null pointer argument", name);
  const kv4::Cache c =
      kv4::cache_of(k_codes, k_params, v_codes, v_params, block_table, Hkv, D, page_size, num_pages, max_pages);
  spade_status st = kv4::check_cache(name, c, B);
  if (st != SPADE_OK) return st;
  st = device_info(nullptr, nullptr);
  if (st != SPADE_OK) return st;
  const cudaError_t e = launch(kv4::commit_kernel, dim3(B), 1, kv4::kThreads, 0, reinterpret_cast<cudaStream_t>(stream), c,
                               ctx_lens, accepted_len, n_draft, new_ctx_lens, status);
  return e == cudaSuccess ? SPADE_OK : cuda_fail(e, "kv_commit_kv4 launch");
}

extern "C" spade_status spade_kv_read_kv4(const void *k_codes, const void *k_params, const void *v_codes,
                                          const void *v_params, const int32_t *block_table, const int32_t *starts,
                                          const int32_t *cu_rows, void *k_out, void *v_out, int32_t B, int32_t R,
                                          int32_t Hkv, int32_t D, int32_t page_size, int32_t num_pages,
                                          int32_t max_pages, int32_t *status, spade_stream_t stream) {
  static const char *name = "spade_kv_read_kv4";
  if (!starts || !cu_rows || !k_out || !v_out || !status)
    return fail(SPADE_ERR_INVALID_ARG, "%s: null pointer argument", name);
  const kv4::Cache c =
      kv4::cache_of(k_codes, k_params, v_codes, v_params, block_table, Hkv, D, page_size, num_pages, max_pages);
  spade_status st = kv4::check_cache(name, c, B);
  if (st != SPADE_OK) return st;
  if (R <= 0) return fail(SPADE_ERR_INVALID_ARG, "%s: non-positive size", name);
  if (!aligned(k_out, 16) || !aligned(v_out, 16))
    return fail(SPADE_ERR_INVALID_ARG, "%s: outputs must be 16-byte aligned", name);
  int sms = 0;
  st = device_info(&sms, nullptr);
  if (st != SPADE_OK) return st;
  // Enough warps for the rows if one sequence has them all, but no more than fill the GPU
  // a few times over: the rest is the loop's.  (Whole rounds of `parts`, so that a warp
  // keeps its part.)
  const int parts = (Hkv * (D / 8) + 31) / 32;
  const int64_t most = (16 * static_cast<int64_t>(sms) + B - 1) / B;       // CTAs per sequence
  const int64_t rows = most * kv4::kWarps / parts + 1;                     // rows that those take at once
  const int64_t warps = (R < rows ? R : rows) * parts;
  const unsigned round = parts % kv4::kWarps ? parts : parts / kv4::kWarps;  // CTAs of whole rounds
  const unsigned ctas = static_cast<unsigned>((warps + kv4::kWarps - 1) / kv4::kWarps + round - 1) / round * round;
  const cudaError_t e = launch(D == 64 ? kv4::read_kernel<64> : kv4::read_kernel<128>, dim3(ctas, B), 1, kv4::kThreads, 0,
                               reinterpret_cast<cudaStream_t>(stream), c, starts, cu_rows, static_cast<uint4 *>(k_out),
                               static_cast<uint4 *>(v_out), R, parts, status);
  return e == cudaSuccess ? SPADE_OK : cuda_fail(e, "kv_read_kv4 launch");
}
