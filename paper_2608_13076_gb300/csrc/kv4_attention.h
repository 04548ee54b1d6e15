// kv4_attention.h -- launch of the attention over the 4-bit cache (kv4_attention_tc.cu).
#pragma once
#include "attn_common.cuh"

namespace spade {
namespace attn {

// Tensor maps: `kc`/`vc` fetch the codes of 64 slots of a head (encode_tmap_bytes),
// `kp`/`vp` their (scale, zero) pairs (encode_tmap_words).  nr: rows of a unit, rounded
// up to 16.
cudaError_t launch_kv4(const Params &p, const CUtensorMap &kc, const CUtensorMap &vc, const CUtensorMap &kp,
                       const CUtensorMap &vp, int nr, int d, cudaStream_t stream);

}  // namespace attn
}  // namespace spade
