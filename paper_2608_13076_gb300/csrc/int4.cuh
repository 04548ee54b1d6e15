// int4.cuh -- numbers in 4 bits as include/spade.h lays them out: value = scale *
// (code - zero), eight codes to a 32-bit word whose fields 4p .. 4p + 3 hold numbers
// 0, 2, 4, 6, 1, 3, 5, 7, and (scale, zero) pairs of float16 per group.  (Codes placed so
// that a mask picks neighbours, and turned into numbers by the low bits of a larger one, is a
// published technique: Kim et al., "Who Says Elephants Can't Run", arXiv:2211.10017, 2022.)
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include <cstdint>

#include "ptx.cuh"

namespace spade {
namespace int4 {

constexpr int kKvGroup = 64;          // dims of a head per (scale, zero) pair of the cache
constexpr float kMaxScale = 4364.f;   // 15 steps of it stay within float16

// Number i (compile-time after unrolling) of a word.
SPADE_DEVICE uint32_t code_of(uint32_t w, int i) { return (w >> (4 * ((i >> 1) + 4 * (i & 1)))) & 15u; }

// A 4-byte (scale, zero) pair as floats.
SPADE_DEVICE float2 pair_of(uint32_t bits) {
  const __half2 h = *reinterpret_cast<const __half2 *>(&bits);
  return __half22float2(h);
}

// A word's eight codes minus the zero, as four pairs of bf16 (exact): a code in the
// low bits of the bf16 of 128 is 128 + code, and nz = -(128 + zero).
SPADE_DEVICE void unpack_bf16(uint32_t w, __nv_bfloat162 nz, uint32_t *out) {
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const uint32_t u = and_or(w >> (4 * e), 0x000f000fu, 0x43004300u);
    const __nv_bfloat162 v = __hadd2(*reinterpret_cast<const __nv_bfloat162 *>(&u), nz);
    out[e] = *reinterpret_cast<const uint32_t *>(&v);
  }
}
// The values in fp16: scale * (code - zero).  The float16 of 1024 holds a code in its
// low bits, or 16 times one in the next: nz = -(1024 + zero), nz16 = -(64 + zero).
SPADE_DEVICE void unpack_fp16(uint32_t w, __half2 s, __half2 nz, __half2 nz16, uint32_t *out) {
  const __half2 sixteenth = __float2half2_rn(0.0625f);
#pragma unroll
  for (int e = 0; e < 2; ++e) {
    const uint32_t lo = and_or(w, 0x000f000fu, 0x64006400u), hi = and_or(w, 0x00f000f0u, 0x64006400u);
    const __half2 a = __hmul2(__hadd2(*reinterpret_cast<const __half2 *>(&lo), nz), s);
    const __half2 b = __hmul2(__hfma2(*reinterpret_cast<const __half2 *>(&hi), sixteenth, nz16), s);
    out[2 * e] = *reinterpret_cast<const uint32_t *>(&a);
    out[2 * e + 1] = *reinterpret_cast<const uint32_t *>(&b);
    w >>= 8;
  }
}

// The cache's pages (see include/spade.h).
struct Cache {
  uint8_t *k_codes, *v_codes;
  uint32_t *k_params, *v_params;  // one (scale, zero) pair per entry
  const int32_t *block_table;
  int Hkv, D, page_size, num_pages, max_pages;
  __device__ int64_t capacity() const { return static_cast<int64_t>(max_pages) * page_size; }
  // Pool row of head 0 of sequence b's slot, in rows of D / 2 code bytes (head h is
  // h * page_size rows on); negative where the page is not in the pool.
  __device__ int64_t row(int b, int slot) const {
    const int page = block_table[static_cast<int64_t>(b) * max_pages + slot / page_size];
    if (page < 0 || page >= num_pages) return -1;
    return static_cast<int64_t>(page) * Hkv * page_size + slot % page_size;
  }
};

}  // namespace int4
}  // namespace spade
