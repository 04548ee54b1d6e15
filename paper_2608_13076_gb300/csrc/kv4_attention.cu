// kv4_attention.cu -- attention of the k+1 verify positions over the paged 4-bit KV
// cache (the verifier's single forward pass over the draft block: Sec. III-B
// "Verification Stage", Algorithm 1 cloud step).
// This file holds the C-ABI entry point: argument checks, tensor maps and the launch of
// the kernel in kv4_attention_tc.cu.  Workspace, schedule and merge are those of the
// attention over bf16 caches (attn_common.cuh).
#include "internal.h"
#include "kv4_attention.h"

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
  const int G = Hq / Hkv;
  spade_status st = attn::check_rows(name, B, Hkv, G, max_k, max_pages * page_size);
  if (st != SPADE_OK) return st;
  if (!aligned(q, 16) || !aligned(out, 16) || !aligned(k_codes, 16) || !aligned(k_params, 16) || !aligned(v_codes, 16) ||
      !aligned(v_params, 16))
    return fail(SPADE_ERR_INVALID_ARG, "%s: q, pools and out must be 16-byte aligned", name);
  int sms = 0;
  st = device_info(&sms, nullptr);
  if (st != SPADE_OK) return st;
  const int cap = max_pages * page_size;
  const size_t need = spade_attn_workspace_size(B, Hq, Hkv, D, cap, max_k);
  if (!workspace || workspace_bytes < need || !aligned(workspace, 256))
    return fail(SPADE_ERR_WORKSPACE, "%s: workspace needs %zu bytes, 256-byte aligned (got %zu)", name, need,
                workspace_bytes);
  const int RB = (G * (max_k + 1) + attn::kRowBlock - 1) / attn::kRowBlock;
  const int units = B * Hkv * RB;

  attn::Params p;
  p.q = static_cast<const __nv_bfloat16 *>(q);
  p.out = static_cast<__nv_bfloat16 *>(out);
  p.lse = lse;
  p.ctx_lens = ctx_lens;
  p.n_draft = n_draft;
  p.cu_q = cu_q;
  p.counters = static_cast<int32_t *>(workspace);
  p.partials = reinterpret_cast<float *>(static_cast<uint8_t *>(workspace) +
                                         round_up(static_cast<size_t>(units) * 4, 256));
  p.status = status;
  p.B = B; p.Hq = Hq; p.Hkv = Hkv; p.G = G; p.cap = cap; p.max_k = max_k; p.R = R; p.RB = RB;
  p.scale_log2 = 1.4426950408889634f / sqrtf(static_cast<float>(D));
  p.block_table = block_table;
  p.page_size = page_size;
  p.max_pages = max_pages;
  p.num_pages = num_pages;
  p.unit_cost = D == 128 ? attn::kUnitCostKv4 : 2 * attn::kUnitCostKv4;
  const int64_t max_chunks = static_cast<int64_t>(units) * ((cap + attn::kChunk - 1) / attn::kChunk);
  p.num_ctas = static_cast<int>(max_chunks < sms ? max_chunks : sms);

  const uint64_t rows = static_cast<uint64_t>(num_pages) * Hkv * page_size;
  CUtensorMap kc, vc, kp, vp;
  if (!encode_tmap_bytes(&kc, k_codes, D / 2, rows, attn::kChunk, D / 2) ||
      !encode_tmap_bytes(&vc, v_codes, D / 2, rows, attn::kChunk, D / 2) ||
      !encode_tmap_words(&kp, k_params, attn::kChunk * (D / 64), rows / attn::kChunk) ||
      !encode_tmap_words(&vp, v_params, attn::kChunk * (D / 64), rows / attn::kChunk))
    return SPADE_ERR_CUDA;
  const int rows_max = G * (max_k + 1) < attn::kRowBlock ? G * (max_k + 1) : attn::kRowBlock;
  const cudaError_t e = attn::launch_kv4(p, kc, vc, kp, vp, (rows_max + 15) / 16 * 16, D,
                                         reinterpret_cast<cudaStream_t>(stream));
  return e == cudaSuccess ? SPADE_OK : cuda_fail(e, "verify_attention_kv4 launch");
}
