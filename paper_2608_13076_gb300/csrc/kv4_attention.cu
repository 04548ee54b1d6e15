// kv4_attention.cu -- attention of the k+1 verify positions over the paged 4-bit KV
// cache (the verifier's single forward pass over the draft block: Sec. III-B
// "Verification Stage", Algorithm 1 cloud step).
#include <cfloat>

#include "attn_common.cuh"
#include "int4.cuh"
#include "internal.h"

namespace spade {
namespace kv4_attn {

struct Params {
  int4::Cache cache;
  const __nv_bfloat16 *q;
  __nv_bfloat16 *out;
  float *lse;
  const int32_t *ctx_lens, *n_draft, *cu_q;
  int32_t *status;
  int R, Hq, max_k;
  float scale_log2;  // log2(e) / sqrt(D)
};

// One warp per (query head, position); its lanes stride the keys, each with a running
// maximum, sum and output of its own, which are joined at the end.
template <int D>
__global__ void __launch_bounds__(32) row_kernel(const __grid_constant__ Params p) {
  const int h = blockIdx.x, b = blockIdx.y, i = blockIdx.z, lane = threadIdx.x;
  const int ctx = p.ctx_lens[b], k = p.n_draft[b], q0 = p.cu_q[b], q1 = p.cu_q[b + 1];
  int bad = 0;
  if (ctx < 0 || k < 0 || k > p.max_k || q0 < 0 || q1 > p.R || q1 - q0 != k + 1) bad = SPADE_DEV_BAD_INDEX;
  else if (static_cast<int64_t>(ctx) + k + 1 > p.cache.capacity()) bad = SPADE_DEV_CAPACITY;
  if (bad) {
    if (h == 0 && i == 0 && lane == 0) atomicOr(p.status, bad);
    return;
  }
  if (i > k) return;
  __shared__ float q[D];
  const int64_t row = static_cast<int64_t>(q0 + i) * p.Hq + h;
  for (int d = lane; d < D; d += 32) q[d] = __bfloat162float(p.q[row * D + d]);
  __syncwarp();
  const int g = h / (p.Hq / p.cache.Hkv);
  float m = -INFINITY, l = 0.f, o[D];
#pragma unroll
  for (int d = 0; d < D; ++d) o[d] = 0.f;
  for (int s = lane; s <= ctx + i; s += 32) {
    const int64_t slot = p.cache.row(b, s);
    float t = 0.f;
    const int64_t at = slot + static_cast<int64_t>(g) * p.cache.page_size;
    if (slot < 0) {
      atomicOr(p.status, SPADE_DEV_BAD_INDEX);  // read as zeros
    } else {
#pragma unroll
      for (int j = 0; j < D / 8; ++j) {
        const uint32_t w = reinterpret_cast<const uint32_t *>(p.cache.k_codes)[at * (D / 8) + j];
        const float2 pair = int4::pair_of(p.cache.k_params[at * (D / 64) + j / 8]);
#pragma unroll
        for (int e = 0; e < 8; ++e)
          t = fmaf(q[8 * j + e], pair.x * (static_cast<float>(int4::code_of(w, e)) - pair.y), t);
      }
    }
    t *= p.scale_log2;
    // A scale that is not finite, of the key or the value, makes the rows that see the slot NaN.
    for (int j = 0; slot >= 0 && j < D / 64; ++j)
      if (!(fabsf(int4::pair_of(p.cache.k_params[at * (D / 64) + j]).x) <= FLT_MAX) ||
          !(fabsf(int4::pair_of(p.cache.v_params[at * (D / 64) + j]).x) <= FLT_MAX))
        t = NAN;
    const float mn = fmaxf(m, t), keep = m == -INFINITY ? 0.f : exp2f(m - mn);
    const float w_ = exp2f(t - mn);
    l = l * keep + w_;
    m = mn;
#pragma unroll
    for (int j = 0; j < D / 8; ++j) {
      uint32_t w = 0;
      float2 pair = make_float2(0.f, 0.f);
      if (slot >= 0) {
        w = reinterpret_cast<const uint32_t *>(p.cache.v_codes)[at * (D / 8) + j];
        pair = int4::pair_of(p.cache.v_params[at * (D / 64) + j / 8]);
      }
#pragma unroll
      for (int e = 0; e < 8; ++e)
        o[8 * j + e] = fmaf(w_, pair.x * (static_cast<float>(int4::code_of(w, e)) - pair.y), o[8 * j + e] * keep);
    }
  }
  float M = m;
#pragma unroll
  for (int x = 16; x; x /= 2) M = fmaxf(M, __shfl_xor_sync(0xffffffffu, M, x));
  const float keep = m == -INFINITY ? 0.f : exp2f(m - M);
  l *= keep;
#pragma unroll
  for (int x = 16; x; x /= 2) l += __shfl_xor_sync(0xffffffffu, l, x);
#pragma unroll
  for (int d = 0; d < D; ++d) {
    float v = o[d] * keep;
#pragma unroll
    for (int x = 16; x; x /= 2) v += __shfl_xor_sync(0xffffffffu, v, x);
    if (lane == d % 32) p.out[row * D + d] = __float2bfloat16_rn(v / l);
  }
  if (p.lse && lane == 0) p.lse[row] = (M + log2f(l)) * 0.69314718055994531f;
}

}  // namespace kv4_attn
}  // namespace spade

using namespace spade;

extern "C" spade_status spade_verify_attention_kv4(
    const void *q, const void *k_codes, const void *k_params, const void *v_codes, const void *v_params,
    const int32_t *block_table, const int32_t *ctx_lens, const int32_t *n_draft, const int32_t *cu_q, void *out,
    float *lse, int32_t B, int32_t Hq, int32_t Hkv, int32_t D, int32_t page_size, int32_t num_pages,
    int32_t max_pages, int32_t max_k, int32_t R, void *workspace, size_t workspace_bytes, int32_t *status,
    spade_stream_t stream) {
  static const char *name = "spade_verify_attention_kv4";
  if (!q || !k_codes || !k_params || !v_codes || !v_params || !block_table || !ctx_lens || !n_draft || !cu_q || !out ||
      !status)
    return fail(SPADE_ERR_INVALID_ARG, "%s: null pointer argument", name);
  if (B <= 0 || Hq <= 0 || Hkv <= 0 || page_size <= 0 || num_pages <= 0 || max_pages <= 0 || max_k < 0 || R <= 0)
    return fail(SPADE_ERR_INVALID_ARG, "%s: non-positive size", name);
  if (Hq % Hkv) return fail(SPADE_ERR_SHAPE, "%s: Hq (%d) must be a multiple of Hkv (%d)", name, Hq, Hkv);
  if (D != 64 && D != 128) return fail(SPADE_ERR_SHAPE, "%s: head dim %d not supported (64 or 128)", name, D);
  if (page_size % attn::kChunk)
    return fail(SPADE_ERR_SHAPE, "%s: page size %d must be a multiple of %d", name, page_size, attn::kChunk);
  if (B > attn::kMaxB) return fail(SPADE_ERR_SHAPE, "%s: B = %d exceeds %d sequences per call", name, B, attn::kMaxB);
  if (R < B) return fail(SPADE_ERR_INVALID_ARG, "%s: R = %d < B = %d", name, R, B);
  if (static_cast<int64_t>(max_pages) * page_size >= (int64_t(1) << 31))
    return fail(SPADE_ERR_CAPACITY, "%s: max_pages * page_size exceeds 2^31", name);
  if (static_cast<int64_t>(num_pages) * Hkv * page_size >= (int64_t(1) << 31))
    return fail(SPADE_ERR_CAPACITY, "%s: pool rows (pages * Hkv * page_size) exceed 2^31", name);
  if (!aligned(q, 16) || !aligned(out, 16) || !aligned(k_codes, 16) || !aligned(k_params, 16) || !aligned(v_codes, 16) ||
      !aligned(v_params, 16))
    return fail(SPADE_ERR_INVALID_ARG, "%s: q, pools and out must be 16-byte aligned", name);
  spade_status st = device_info(nullptr, nullptr);
  if (st != SPADE_OK) return st;
  const size_t need = spade_attn_workspace_size(B, Hq, Hkv, D, max_pages * page_size, max_k);
  if (!workspace || workspace_bytes < need || !aligned(workspace, 256))
    return fail(SPADE_ERR_WORKSPACE, "%s: workspace needs %zu bytes, 256-byte aligned (got %zu)", name, need,
                workspace_bytes);
  kv4_attn::Params p;
  p.cache.k_codes = static_cast<uint8_t *>(const_cast<void *>(k_codes));
  p.cache.v_codes = static_cast<uint8_t *>(const_cast<void *>(v_codes));
  p.cache.k_params = static_cast<uint32_t *>(const_cast<void *>(k_params));
  p.cache.v_params = static_cast<uint32_t *>(const_cast<void *>(v_params));
  p.cache.block_table = block_table;
  p.cache.Hkv = Hkv; p.cache.D = D; p.cache.page_size = page_size; p.cache.num_pages = num_pages;
  p.cache.max_pages = max_pages;
  p.q = static_cast<const __nv_bfloat16 *>(q);
  p.out = static_cast<__nv_bfloat16 *>(out);
  p.lse = lse;
  p.ctx_lens = ctx_lens; p.n_draft = n_draft; p.cu_q = cu_q; p.status = status;
  p.R = R; p.Hq = Hq; p.max_k = max_k;
  p.scale_log2 = 1.4426950408889634f / sqrtf(static_cast<float>(D));
  const int longest = max_k < R ? max_k + 1 : R;  // a block longer than the rows given cannot be valid
  if (longest > 65535) return fail(SPADE_ERR_SHAPE, "%s: max_k = %d exceeds 65534", name, max_k);
  const dim3 grid(Hq, B, longest);
  cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
  if (D == 64) kv4_attn::row_kernel<64><<<grid, 32, 0, s>>>(p);
  else kv4_attn::row_kernel<128><<<grid, 32, 0, s>>>(p);
  const cudaError_t e = cudaGetLastError();
  return e == cudaSuccess ? SPADE_OK : cuda_fail(e, "verify_attention_kv4 launch");
}
