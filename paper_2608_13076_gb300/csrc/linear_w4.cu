// linear_w4.cu -- y = x W^T (+ residual) with W in 4 bits: the verifier's linear
// layers (f_l in x_{l+1} = x_l + f_l(x_l), Sec. III-A) for the rows of a verify block
// or single tokens.
#include <cfloat>

#include "int4.cuh"
#include "internal.h"
#include "ptx.cuh"

namespace spade {
namespace w4 {

struct Params {
  const __nv_bfloat16 *x, *residual;
  const uint32_t *codes, *pairs;
  __nv_bfloat16 *out;
  int32_t *status;
  int R, N, K, group;
};

constexpr int kThreads = 256;
constexpr int kRows = 4;

// One warp per output entry of up to four rows; its lanes stride the words of the
// weight row, and the sums are joined by shuffles.
__global__ void __launch_bounds__(kThreads) rows_kernel(const __grid_constant__ Params p) {
  const int lane = threadIdx.x & 31;
  const int n = blockIdx.x * (kThreads / 32) + (threadIdx.x >> 5);
  const int r0 = blockIdx.y * kRows;
  if (n >= p.N) return;
  const int words = p.K / 8, groups = p.K / p.group;
  float acc[kRows] = {};
  for (int j = lane; j < words; j += 32) {
    const uint32_t w = __ldg(p.codes + static_cast<int64_t>(n) * words + j);
    const float2 pair = int4::pair_of(__ldg(p.pairs + static_cast<int64_t>(n) * groups + j * 8 / p.group));
#pragma unroll
    for (int r = 0; r < kRows; ++r) {
      if (r0 + r >= p.R) break;
      const uint4 v = __ldg(reinterpret_cast<const uint4 *>(p.x + static_cast<int64_t>(r0 + r) * p.K) + j);
      const uint32_t xw[4] = {v.x, v.y, v.z, v.w};
      float sum = 0.f;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float x = __uint_as_float(e & 1 ? xw[e / 2] & 0xffff0000u : xw[e / 2] << 16);
        sum = fmaf(x, static_cast<float>(int4::code_of(w, e)) - pair.y, sum);
      }
      acc[r] = fmaf(pair.x, sum, acc[r]);
    }
  }
#pragma unroll
  for (int r = 0; r < kRows; ++r)
#pragma unroll
    for (int o = 16; o; o /= 2) acc[r] += __shfl_xor_sync(0xffffffffu, acc[r], o);
  if (lane == 0) {
#pragma unroll
    for (int r = 0; r < kRows; ++r) {
      if (r0 + r >= p.R) break;
      const int64_t at = static_cast<int64_t>(r0 + r) * p.N + n;
      p.out[at] = __float2bfloat16_rn(acc[r] + (p.residual ? __bfloat162float(p.residual[at]) : 0.f));
    }
  }
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
  spade_status st = device_info(nullptr, nullptr);
  if (st != SPADE_OK) return st;
  w4::Params p;
  p.x = static_cast<const __nv_bfloat16 *>(x);
  p.residual = static_cast<const __nv_bfloat16 *>(residual);
  p.codes = static_cast<const uint32_t *>(codes);
  p.pairs = static_cast<const uint32_t *>(params);
  p.out = static_cast<__nv_bfloat16 *>(out);
  p.status = status;
  p.R = R; p.N = N; p.K = K; p.group = group;
  const int64_t gy = (static_cast<int64_t>(R) + w4::kRows - 1) / w4::kRows;
  if (gy > 65535) return fail(SPADE_ERR_SHAPE, "spade_linear_w4: R = %d exceeds %d rows per call", R, 65535 * w4::kRows);
  const int warps = w4::kThreads / 32;
  w4::rows_kernel<<<dim3((static_cast<unsigned>(N) + warps - 1) / warps, static_cast<unsigned>(gy)), w4::kThreads, 0,
                    reinterpret_cast<cudaStream_t>(stream)>>>(p);
  const cudaError_t e = cudaGetLastError();
  return e == cudaSuccess ? SPADE_OK : cuda_fail(e, "linear_w4 launch");
}
