// kv4_attention.h -- launch of the attention over the 4-bit cache (kv4_attention_tc.cu).
#pragma once
#include "attn_common.cuh"

namespace spade {
namespace attn {

// The cache's pools, as bytes; `rows` slots of a head (num_pages * Hkv * page_size) in all.
struct Kv4Pool {
  const uint8_t *k_codes, *k_pairs, *v_codes, *v_pairs;
  int rows;
};

// nr: rows of a unit, rounded up to 16.
cudaError_t launch_kv4(const Params &p, const Kv4Pool &pool, int nr, int d, cudaStream_t stream);

}  // namespace attn
}  // namespace spade
