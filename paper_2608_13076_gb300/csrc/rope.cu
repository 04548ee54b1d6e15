// rope.cu -- the verify block's query, key and value heads on their way into the attention, for
// projections made elsewhere: rotary embedding at given positions (the nodes of a tree of drafts
// have other positions than slots), keys and values stored into the bf16 cache (the input side of
// the attention in x_{l+1} = x_l + f_l(x_l), Sec. III-A).
#include <cuda_bf16.h>

#include <cfloat>

#include "kv_cache.cuh"
#include "launch.h"
#include "ptx.cuh"

namespace spade {
namespace rope {

struct Params {
  KvCache cache;
  const __nv_bfloat16 *qkv;
  const double *inv_freq;
  const int32_t *positions;  // null: ctx + i
  const int32_t *ctx_lens, *n_draft, *cu_q;
  __nv_bfloat16 *q_out;
  int32_t *status;
  int64_t row_stride;  // of qkv, in 16-byte vectors
  int B, R, Hq, rot, max_k;
  float mscale;
};

// Sequence whose valid block holds row `row` (-1: none), by a whole warp.
SPADE_DEVICE int sequence_of(const Params &p, int row, int lane, int *ctx, int *node) {
  constexpr int kSets = 2;  // of 32 sequences at once
  for (int b0 = 0; b0 < p.B; b0 += 32 * kSets) {
    int c[kSets], k[kSets], q0[kSets], q1[kSets];
#pragma unroll
    for (int i = 0; i < kSets; ++i) {
      const int b = min(b0 + 32 * i + lane, p.B - 1);
      q0[i] = p.cu_q[b];
      q1[i] = p.cu_q[b + 1];
      k[i] = p.n_draft[b];
      c[i] = p.ctx_lens[b];
    }
#pragma unroll
    for (int i = 0; i < kSets; ++i) {
      const bool mine = b0 + 32 * i + lane < p.B && row >= q0[i] && row < q1[i] &&
                        !tree_block_error(c[i], k[i], q0[i], q1[i], p.max_k, p.R, p.cache.cap);
      const unsigned vote = __ballot_sync(0xffffffffu, mine);
      if (vote) {
        const int src = __ffs(vote) - 1;
        *ctx = __shfl_sync(0xffffffffu, c[i], src);
        *node = row - __shfl_sync(0xffffffffu, q0[i], src);
        return b0 + 32 * i + src;
      }
    }
  }
  return -1;
}

// One CTA per row.  Its angles (rot / 2 of them) are made once and shared by all heads: the position
// times frequency / 2 pi in 64 bits, so that the turns that are dropped cost next to nothing at far
// positions (2^-24 of a turn at 2^31), then sincospif of the rest in fp32 (2^-25 of a turn).  A head's D dims lie on D / 8
// lanes, eight neighbours each; in the half layout the rotation's partner is rot / 16 lanes away.
// The heads' loads are issued before all else, and the last threads make the angles while the first
// look for the row's sequence.  A lane's angles lie a lane's width apart in shared memory, where the
// lanes of a warp read neighbours (eight next to each other per lane met the same banks: 1376 rows of
// 56 heads 14.2 us instead of 9.1).
// Bound by the bytes where rows are many: a row's heads once in, once out (12288 rows of 48 heads of
// 128: 47 us, 6.4 TB/s; 1376 of 56 9.1 us, 4.3 TB/s, in a step of several layers and 10 alone; 4096 rows of 512
// sequences 22, 4.6 TB/s), by latency where they are few (512 rows of 48 heads 3.7 us; 3.9 with one product at a time instead of two).  Five CTAs of 256 threads to an SM: with six,
// 1376 rows 9.5 us, with seven 11.2; two or eight vectors a thread were slower as well, and angles in registers.
constexpr int kVecs = 4;  // 16-byte vectors of a thread in flight
constexpr int kMaxThreads = 256;
template <int D, bool kInterleaved>
__global__ void __launch_bounds__(kMaxThreads, 5) rope_kernel(const __grid_constant__ Params p) {
  constexpr int kLanes = D / 8;
  __shared__ float4 s_turn[kInterleaved ? D / 4 : D / 2];  // (half layout: twice, for a pair's first and second dims)
  __shared__ int s_ctx, s_b, s_node;
  const int row = blockIdx.x, lane = threadIdx.x & 31;
  // (The next kernel comes when this one ends: its CTAs, let in early, take room from this one's rows.  512 rows: 3.9
  // us, 4.9 with an early start.)
  griddep_wait();
  if (threadIdx.x < 32) {
    int ctx = 0, node = 0;
    const int b = sequence_of(p, row, lane, &ctx, &node);
    if (lane == 0) {
      s_b = b;
      s_ctx = ctx;
      s_node = node;
    }
  } else if (row == 0) {
    // Blocks that cannot be used are reported once.
    for (int b = threadIdx.x - 32; b < p.B; b += blockDim.x - 32) {
      const int bad = tree_block_error(p.ctx_lens[b], p.n_draft[b], p.cu_q[b], p.cu_q[b + 1], p.max_k, p.R, p.cache.cap);
      if (bad) atomicOr(p.status, bad);
    }
  }
  // (What does not depend on the sequence is asked for at once.  The last threads make the angles, as the first look for
  // the sequence.)
  const int given = p.positions ? p.positions[row] : 0;
  const int pair = static_cast<int>(blockDim.x - 1 - threadIdx.x);
  const bool turning = pair < p.rot / 2;  // (of up to 64)
  const double freq = turning ? p.inv_freq[pair] : 0.0;
  const int Hkv = p.cache.Hkv, heads = p.Hq + 2 * Hkv, vecs = heads * kLanes;
  const uint4 *src = reinterpret_cast<const uint4 *>(p.qkv) + row * p.row_stride;
  uint4 in[kVecs];
#pragma unroll
  for (int j = 0; j < kVecs; ++j) {
    const int v = threadIdx.x + j * blockDim.x;
    in[j] = v < vecs ? src[v] : make_uint4(0, 0, 0, 0);
  }
  // A lane's e-th pair, where neighbouring lanes find theirs next to each other.
  constexpr int kPairs = kInterleaved ? 4 : 8;  // of a lane
  const int turning_lanes = p.rot / 2 / kPairs;
  auto turn_by = [&](int pos) {
    const double turns = pos * (freq * 0.15915494309189533577);  // 1 / (2 pi)
    float s, c;
    sincospif(2.f * static_cast<float>(turns - rint(turns)), &s, &c);
    c *= p.mscale;
    s *= p.mscale;
    const int at_lane = pair / kPairs, e = pair % kPairs;
    if constexpr (kInterleaved) {
      reinterpret_cast<float2 *>(s_turn)[e * turning_lanes + at_lane] = make_float2(c, s);
    } else {
      // Two neighbours' cosines, then their sines, to be used two at a time.
      float *to = reinterpret_cast<float *>(s_turn + e / 2 * turning_lanes + at_lane) + e % 2;
      to[0] = c;
      to[2] = -s;
      to += 4 * (4 * turning_lanes);
      to[0] = c;
      to[2] = s;
    }
  };
  if (p.positions && turning) turn_by(given);
  __syncthreads();
  const int b = s_b;
  if (b < 0) return;
  const int slot = s_ctx + s_node;
  const int64_t at = p.cache.row(b, slot);
  if (!p.positions) {
    if (turning) turn_by(slot);
    __syncthreads();
  }
  if (at < 0 && threadIdx.x == 0) atomicOr(p.status, SPADE_DEV_BAD_INDEX);
  const int half = p.rot / 16;  // lanes of half the turning dims
  for (int v0 = 0; v0 < vecs; v0 += kVecs * blockDim.x) {
    if (v0 > 0) {
#pragma unroll
      for (int j = 0; j < kVecs; ++j) {
        const int v = v0 + threadIdx.x + j * blockDim.x;
        in[j] = v < vecs ? src[v] : make_uint4(0, 0, 0, 0);
      }
    }
#pragma unroll
    for (int j = 0; j < kVecs; ++j) {
      const int v = v0 + threadIdx.x + j * blockDim.x;
      if (v - lane >= vecs) break;
      const int h = v / kLanes, l = v % kLanes;
      const bool turns = l < 2 * half && h < p.Hq + Hkv;
      uint32_t w[4] = {in[j].x, in[j].y, in[j].z, in[j].w};
      auto low = [](uint32_t x) { return __uint_as_float(x << 16); };
      auto high = [](uint32_t x) { return __uint_as_float(x & 0xffff0000u); };
      if constexpr (kInterleaved) {
        if (turns) {
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const float2 t = reinterpret_cast<const float2 *>(s_turn)[e * turning_lanes + l];
            const float a = low(w[e]), b = high(w[e]);
            w[e] = pack_bf16(a * t.x - b * t.y, b * t.x + a * t.y);
          }
        }
      } else {
        // A dim of the first half becomes own cos - other sin, one of the second own cos + other sin.
        const bool second = l >= half;
        const int partner = lane + (turns ? (second ? -half : half) : 0);
        uint32_t o[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) o[e] = __shfl_sync(0xffffffffu, w[e], partner);
        if (turns) {
          const float4 *t = s_turn + (second ? 4 * turning_lanes + l - half : l);
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const float4 cs = t[e * turning_lanes];
            float a, b;
            f2_split(f2_fma(f2(low(o[e]), high(o[e])), f2(cs.z, cs.w), f2_mul(f2(low(w[e]), high(w[e])), f2(cs.x, cs.y))), a, b);
            w[e] = pack_bf16(a, b);
          }
        }
      }
      if (v >= vecs) continue;
      const uint4 out = make_uint4(w[0], w[1], w[2], w[3]);
      if (h < p.Hq) {
        reinterpret_cast<uint4 *>(p.q_out)[(static_cast<int64_t>(row) * p.Hq + h) * kLanes + l] = out;
      } else if (at >= 0) {
        const bool is_v = h >= p.Hq + Hkv;
        const int64_t r = at + static_cast<int64_t>(h - p.Hq - (is_v ? Hkv : 0)) * p.cache.span;
        reinterpret_cast<uint4 *>(is_v ? p.cache.v : p.cache.k)[r * kLanes + l] = out;
      }
    }
  }
}

static spade_status run(const char *name, Params p, int64_t qkv_stride, bool interleaved, cudaStream_t stream) {
  if (!p.qkv || !p.inv_freq || !p.q_out || !p.ctx_lens || !p.n_draft || !p.cu_q || !p.status)
    return fail(SPADE_ERR_INVALID_ARG, "%s: null pointer argument", name);
  const int Hkv = p.cache.Hkv, D = p.cache.D;
  if (p.R <= 0 || p.Hq <= 0 || p.max_k < 0) return fail(SPADE_ERR_INVALID_ARG, "%s: non-positive size", name);
  if (p.Hq % Hkv) return fail(SPADE_ERR_SHAPE, "%s: Hq (%d) must be a multiple of Hkv (%d)", name, p.Hq, Hkv);
  if (p.R < p.B) return fail(SPADE_ERR_INVALID_ARG, "%s: R = %d < B = %d", name, p.R, p.B);
  if (p.rot < 16 || p.rot > D || p.rot % 16)
    return fail(SPADE_ERR_SHAPE, "%s: %d turning dims: must be a multiple of 16 up to the head dim %d", name, p.rot, D);
  const int64_t vecs = (p.Hq + int64_t(2) * Hkv) * (D / 8);
  if (vecs > (int64_t(1) << 30)) return fail(SPADE_ERR_CAPACITY, "%s: too many heads", name);
  if (qkv_stride % 8 || qkv_stride < 8 * vecs)
    return fail(SPADE_ERR_SHAPE, "%s: qkv row stride %lld must be a multiple of 8 and hold the row's heads", name,
                static_cast<long long>(qkv_stride));
  if (!(p.mscale >= -FLT_MAX && p.mscale <= FLT_MAX)) return fail(SPADE_ERR_INVALID_ARG, "%s: mscale must be finite", name);
  if (!aligned(p.qkv, 16) || !aligned(p.q_out, 16) || !aligned(p.inv_freq, 8))
    return fail(SPADE_ERR_INVALID_ARG, "%s: qkv and q_out must be 16-byte aligned", name);
  const spade_status st = device_info(nullptr, nullptr);
  if (st != SPADE_OK) return st;
  p.row_stride = qkv_stride / 8;
  // Threads: a quarter of the row's vectors each takes (whole warps, the second one reports).
  int64_t threads = ((vecs + kVecs - 1) / kVecs + 31) / 32 * 32;
  threads = threads < 64 ? 64 : threads > kMaxThreads ? kMaxThreads : threads;
  auto kern = D == 64 ? (interleaved ? rope_kernel<64, true> : rope_kernel<64, false>)
                      : (interleaved ? rope_kernel<128, true> : rope_kernel<128, false>);
  const cudaError_t e = launch(kern, dim3(p.R), 1, static_cast<unsigned>(threads), 0, stream, p);
  return e == cudaSuccess ? SPADE_OK : cuda_fail(e, name);
}

}  // namespace rope
}  // namespace spade

using namespace spade;

extern "C" spade_status spade_verify_rope(const void *qkv, int64_t qkv_stride, const double *inv_freq,
                                          const int32_t *positions, const int32_t *ctx_lens, const int32_t *n_draft,
                                          const int32_t *cu_q, void *q_out, void *k_cache, void *v_cache, int32_t B,
                                          int32_t R, int32_t Hq, int32_t Hkv, int32_t D, int32_t cap, int32_t rot_dims,
                                          int32_t interleaved, int32_t max_k, float mscale, int32_t *status,
                                          spade_stream_t stream) {
  static const char *name = "spade_verify_rope";
  rope::Params p;
  const spade_status st = kv_cache_of(name, &p.cache, k_cache, v_cache, false, nullptr, B, Hkv, D, cap, B, 1);
  if (st != SPADE_OK) return st;
  p.qkv = static_cast<const __nv_bfloat16 *>(qkv);
  p.q_out = static_cast<__nv_bfloat16 *>(q_out);
  p.inv_freq = inv_freq; p.positions = positions; p.ctx_lens = ctx_lens; p.n_draft = n_draft; p.cu_q = cu_q;
  p.status = status; p.B = B; p.R = R; p.Hq = Hq; p.rot = rot_dims; p.max_k = max_k; p.mscale = mscale;
  return rope::run(name, p, qkv_stride, interleaved != 0, reinterpret_cast<cudaStream_t>(stream));
}

extern "C" spade_status spade_verify_rope_paged(const void *qkv, int64_t qkv_stride, const double *inv_freq,
                                                const int32_t *positions, const int32_t *block_table,
                                                const int32_t *ctx_lens, const int32_t *n_draft, const int32_t *cu_q,
                                                void *q_out, void *k_pool, void *v_pool, int32_t B, int32_t R,
                                                int32_t Hq, int32_t Hkv, int32_t D, int32_t page_size,
                                                int32_t num_pages, int32_t max_pages, int32_t rot_dims,
                                                int32_t interleaved, int32_t max_k, float mscale, int32_t *status,
                                                spade_stream_t stream) {
  static const char *name = "spade_verify_rope_paged";
  rope::Params p;
  const spade_status st =
      kv_cache_of(name, &p.cache, k_pool, v_pool, true, block_table, B, Hkv, D, page_size, num_pages, max_pages);
  if (st != SPADE_OK) return st;
  p.qkv = static_cast<const __nv_bfloat16 *>(qkv);
  p.q_out = static_cast<__nv_bfloat16 *>(q_out);
  p.inv_freq = inv_freq; p.positions = positions; p.ctx_lens = ctx_lens; p.n_draft = n_draft; p.cu_q = cu_q;
  p.status = status; p.B = B; p.R = R; p.Hq = Hq; p.rot = rot_dims; p.max_k = max_k; p.mscale = mscale;
  return rope::run(name, p, qkv_stride, interleaved != 0, reinterpret_cast<cudaStream_t>(stream));
}
