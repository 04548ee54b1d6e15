// tree.cu -- the bookkeeping of a verify step over trees of drafts (the block of Sec. III-B with
// several continuations): positions and masks of the nodes before the layers run, and afterwards
// Algorithm 1's context update along the accepted path.
//
// A sequence's block has n_draft + 1 nodes; node 0 is its last accepted token and node i >= 1,
// draft i - 1, hangs from node parents[i] < i.
#include <cuda_bf16.h>

#include "kv_cache.cuh"
#include "launch.h"
#include "ptx.cuh"

namespace spade {
namespace tree {

constexpr int kThreads = 256;
constexpr int kMaxNodes = 16384;  // of a sequence: the commit's lists of 12 bytes a node fit shared memory

// ---- layout --------------------------------------------------------------------------------
struct Layout {
  const int32_t *parents, *ctx_lens, *n_draft, *cu_q;
  int32_t *positions, *mask, *status;
  int R, words, max_k;
};

// One CTA per sequence.  Nodes are taken in blocks of 32, a warp's lanes: within its block a
// node's ancestors are found by five doublings of the path (bits |= bits[up], up = up[up]) in
// registers; what is left is the first ancestor in an earlier block, so the walk to the root
// takes one step per block that the path meets, not one per node.  Latency is all there is, in a
// graph 1.6 us for 8 trees of 64 nodes (8 KB) and 3.8 for 64 of up to 512 (1.4 MB, 0.2 us of HBM);
// calls from the host take 3.1 and 4.0.
__global__ void __launch_bounds__(kThreads) layout_kernel(const __grid_constant__ Layout p, int nodes) {
  extern __shared__ int32_t smem[];
  uint32_t *s_bits = reinterpret_cast<uint32_t *>(smem);  // [nodes] ancestors within the node's block
  int32_t *s_up = smem + nodes;                           // [nodes] first ancestor in an earlier block, -1: none
  const int b = blockIdx.x;
  const int lane = threadIdx.x & 31;
  griddep_wait();
  griddep_launch_dependents();
  const int ctx = p.ctx_lens[b], k = p.n_draft[b], q0 = p.cu_q[b], q1 = p.cu_q[b + 1];
  int bad = tree_block_error(ctx, k, q0, q1, p.max_k, p.R, INT32_MAX);
  const int n = bad ? 0 : k + 1;
  int wrong = 0;
  for (int i0 = threadIdx.x & ~31; i0 < n; i0 += kThreads) {
    const int i = i0 + lane;
    int up = i < n ? p.parents[q0 + i] : -1;
    if (i < n && (i == 0 ? up != -1 : up < 0 || up >= i)) {
      wrong = 1;
      up = -1;
    }
    uint32_t bits = 1u << lane;
#pragma unroll
    for (int o = 0; o < 5; ++o) {
      const bool inside = up >= i0;
      const uint32_t more = __shfl_sync(0xffffffffu, bits, up & 31);
      const int next = __shfl_sync(0xffffffffu, up, up & 31);
      if (inside) {
        bits |= more;
        up = next;
      }
    }
    if (i < n) {
      s_bits[i] = bits;
      s_up[i] = up;
    }
  }
  if (__syncthreads_or(wrong)) bad = SPADE_DEV_BAD_INDEX;
  if (bad) {
    if (threadIdx.x == 0) atomicOr(p.status, bad);
    return;
  }
  const bool wide = p.words % 4 == 0 && (reinterpret_cast<uintptr_t>(p.mask) & 15) == 0;
  for (int i = threadIdx.x; i < n; i += kThreads) {
    int32_t *row = p.mask + static_cast<int64_t>(q0 + i) * p.words;
    int at = i, depth = -1;
    if (wide) {
      for (int g = p.words / 4 - 1; g >= 0; --g) {
        uint32_t w[4] = {};
#pragma unroll
        for (int e = 3; e >= 0; --e)
          if (at >= 0 && at >> 5 == 4 * g + e) {
            w[e] = s_bits[at];
            at = s_up[at];
            depth += __popc(w[e]);
          }
        reinterpret_cast<uint4 *>(row)[g] = make_uint4(w[0], w[1], w[2], w[3]);
      }
    } else {
      for (int g = p.words - 1; g >= 0; --g) {
        uint32_t w = 0;
        if (at >= 0 && at >> 5 == g) {
          w = s_bits[at];
          at = s_up[at];
          depth += __popc(w);
        }
        row[g] = static_cast<int32_t>(w);
      }
    }
    p.positions[q0 + i] = ctx + depth;
  }
}

// ---- commit --------------------------------------------------------------------------------
struct Commit {
  KvCache cache;
  int64_t layer_rows;  // cache rows of a layer
  const int32_t *ctx_lens, *parents, *drafts, *tokens, *n_draft, *cu_q;
  int32_t *accepted, *next_token, *path, *new_ctx, *status;
  int layers, R, max_k;
  int planes;          // (layer, K or V, head) of one CTA
};

// CTA (b, part) walks sequence b's tree (the lowest child of every node whose draft is the node's
// token, by atomicMin, then a chain of steps through shared memory) and then moves and clears the
// block's rows in its planes.  Rows of the path move to lower slots in order, a thread per 16-byte
// column, so that no row is overwritten before it has been read; the barrier between moving and
// clearing is the CTA's own, as planes are not shared.  (Walking again in every CTA takes no
// longer than a second launch would.)  8 x 64 nodes, one layer 3.8 us, of which the bytes 0.5; 8
// layers of 64 x 21 nodes (42 MB, mostly zeros) 14.1, of which 6.3 (three sets of caches in turn).
__global__ void __launch_bounds__(kThreads) commit_kernel(const __grid_constant__ Commit p, int nodes) {
  extern __shared__ int32_t smem[];
  int32_t *s_next = smem;               // [nodes] accepted child
  int32_t *s_path = smem + nodes;       // [nodes] the path
  int32_t *s_row = smem + 2 * nodes;    // [nodes] cache row of the slot, head 0
  __shared__ int s_len;
  const int b = blockIdx.x, part = blockIdx.y;
  griddep_wait();
  griddep_launch_dependents();
  const int ctx = p.ctx_lens[b], k = p.n_draft[b], q0 = p.cu_q[b], q1 = p.cu_q[b + 1];
  const KvCache &c = p.cache;
  int bad = tree_block_error(ctx, k, q0, q1, p.max_k, p.R, c.cap);
  // The drafts of earlier sequences and of this one lie within the array.
  if (!bad && (q0 < b || q1 - b - 1 > p.R - static_cast<int>(gridDim.x))) bad = SPADE_DEV_BAD_INDEX;
  const int n = bad ? 0 : k + 1;
  for (int i = threadIdx.x; i < n; i += kThreads) s_next[i] = INT32_MAX;
  __syncthreads();
  int wrong = 0;
  for (int i = threadIdx.x; i < n; i += kThreads) {
    const int up = p.parents[q0 + i];
    // Every page that the block uses must exist before anything is moved.
    const int64_t row = c.row(b, ctx + i);
    s_row[i] = static_cast<int32_t>(row);
    if (row < 0 || (i == 0 ? up != -1 : up < 0 || up >= i)) {
      wrong = 1;
    } else if (i > 0) {
      const int draft = p.drafts[q0 - b + i - 1];
      if (draft >= 0 && draft == p.tokens[q0 + up]) atomicMin(&s_next[up], i);
    }
  }
  if (__syncthreads_or(wrong)) bad = SPADE_DEV_BAD_INDEX;
  if (threadIdx.x == 0 && !bad) {
    int len = 0;
    for (int at = 0; at != INT32_MAX; at = s_next[at]) s_path[len++] = at;
    s_len = len;
  }
  __syncthreads();
  const int len = bad ? 0 : s_len;
  if (part == 0) {
    if (threadIdx.x == 0) {
      p.accepted[b] = len - 1;
      p.next_token[b] = bad ? -1 : p.tokens[q0 + s_path[len - 1]];
      if (p.new_ctx != p.ctx_lens) p.new_ctx[b] = ctx + len;
      if (bad) atomicOr(p.status, bad);
    }
    for (int i = threadIdx.x; i < n && !bad; i += kThreads) p.path[q0 + i] = i < len ? s_path[i] : -1;
  }
  if (bad) return;
  const int vec = c.D / 8, shift = c.D == 128 ? 4 : 3;  // 16-byte vectors of a row
  const int plane0 = part * p.planes, planes = min(p.planes, 2 * p.layers * c.Hkv - plane0);
  // A plane: layer, keys or values, head (planes of a layer's keys come before its values').
  auto plane_base = [&](int plane) {
    const int layer = plane / (2 * c.Hkv), r = plane - layer * 2 * c.Hkv;
    const int is_v = r >= c.Hkv;
    return reinterpret_cast<uint4 *>(is_v ? c.v : c.k) +
           (static_cast<int64_t>(layer) * p.layer_rows + static_cast<int64_t>(r - is_v * c.Hkv) * c.span) * vec;
  };
  // The nodes before the first that moves stay where they are.
  int first = 1;
  while (first < len && s_path[first] == first) ++first;
  if (first < len) {
    for (int e = threadIdx.x; e < planes << shift; e += kThreads) {
      uint4 *base = plane_base(plane0 + (e >> shift)) + (e & (vec - 1));
      constexpr int kBatch = 4;
      for (int j = first; j < len; j += kBatch) {
        uint4 x[kBatch];
#pragma unroll
        for (int u = 0; u < kBatch; ++u)
          if (j + u < len) x[u] = base[static_cast<int64_t>(s_row[s_path[j + u]]) * vec];
#pragma unroll
        for (int u = 0; u < kBatch; ++u)
          if (j + u < len) base[static_cast<int64_t>(s_row[j + u]) * vec] = x[u];
      }
    }
    __syncthreads();
  }
  const uint4 zero = make_uint4(0, 0, 0, 0);
  for (int pl = 0; pl < planes; ++pl) {
    uint4 *base = plane_base(plane0 + pl) + (threadIdx.x & (vec - 1));
    for (int slot = len + (threadIdx.x >> shift); slot < n; slot += kThreads >> shift)
      base[static_cast<int64_t>(s_row[slot]) * vec] = zero;
  }
}

// ctx += a + 1 in place, after every CTA of the commit has read it.
__global__ void __launch_bounds__(kThreads) advance_kernel(int32_t *ctx_lens, const int32_t *accepted, int B) {
  griddep_wait();
  griddep_launch_dependents();
  const int b = blockIdx.x * kThreads + threadIdx.x;
  if (b < B) ctx_lens[b] += accepted[b] + 1;
}

static spade_status check_tree(const char *name, int B, int R, int max_k, int *nodes) {
  if (B <= 0 || R <= 0 || max_k < 0) return fail(SPADE_ERR_INVALID_ARG, "%s: non-positive size", name);
  if (R < B) return fail(SPADE_ERR_INVALID_ARG, "%s: R = %d < B = %d", name, R, B);
  // A block longer than the rows given cannot be valid.
  *nodes = max_k < R ? max_k + 1 : R;
  if (*nodes > kMaxNodes) return fail(SPADE_ERR_SHAPE, "%s: trees of up to %d nodes (got %d)", name, kMaxNodes, *nodes);
  return SPADE_OK;
}

static spade_status commit(const char *name, Commit p, int B, cudaStream_t stream) {
  if (!p.ctx_lens || !p.parents || !p.tokens || !p.n_draft || !p.cu_q || !p.accepted || !p.next_token || !p.path ||
      !p.new_ctx || !p.status || (!p.drafts && p.R > B))
    return fail(SPADE_ERR_INVALID_ARG, "%s: null pointer argument", name);
  int nodes = 0, sms = 0;
  spade_status st = check_tree(name, B, p.R, p.max_k, &nodes);
  if (st != SPADE_OK) return st;
  if (p.layers <= 0) return fail(SPADE_ERR_INVALID_ARG, "%s: non-positive size", name);
  const int64_t planes = int64_t(2) * p.layers * p.cache.Hkv;
  if (planes >= (int64_t(1) << 20)) return fail(SPADE_ERR_CAPACITY, "%s: too many layers or heads", name);
  st = device_info(&sms, nullptr);
  if (st != SPADE_OK) return st;
  static OncePerDevice once;
  cudaError_t e = set_max_smem(once, 12 * kMaxNodes, commit_kernel);
  if (e != cudaSuccess) return cuda_fail(e, name);
  // CTAs of a sequence: enough to fill the GPU four times with the batch (8 layers of 64 sequences: 11.7 us, with two
  // times 14.3, with 16 13.9), each with a plane at least and with at most as many as make 512 vectors (one layer of
  // 8 x 64 nodes: 3.6 us, with 2048 3.9).
  const int64_t plane_vecs = static_cast<int64_t>(nodes) * (p.cache.D / 8);
  int64_t parts = (4 * static_cast<int64_t>(sms) + B - 1) / B;
  const int64_t worth = (planes * plane_vecs + 511) / 512;
  parts = parts < worth ? parts : worth;
  parts = parts < planes ? parts : planes;
  p.planes = static_cast<int>((planes + parts - 1) / parts);
  parts = (planes + p.planes - 1) / p.planes;
  e = launch(commit_kernel, dim3(B, static_cast<unsigned>(parts)), 1, kThreads, 12 * static_cast<size_t>(nodes), stream, p,
             nodes);
  if (e == cudaSuccess && p.new_ctx == p.ctx_lens)
    e = launch(advance_kernel, dim3((B + kThreads - 1) / kThreads), 1, kThreads, 0, stream, p.new_ctx,
               static_cast<const int32_t *>(p.accepted), B);
  return e == cudaSuccess ? SPADE_OK : cuda_fail(e, name);
}

}  // namespace tree
}  // namespace spade

using namespace spade;

extern "C" spade_status spade_tree_layout(const int32_t *parents, const int32_t *ctx_lens, const int32_t *n_draft,
                                          const int32_t *cu_q, int32_t *positions, int32_t *tree_mask, int32_t B,
                                          int32_t R, int32_t mask_words, int32_t max_k, int32_t *status,
                                          spade_stream_t stream) {
  static const char *name = "spade_tree_layout";
  if (!parents || !ctx_lens || !n_draft || !cu_q || !positions || !tree_mask || !status)
    return fail(SPADE_ERR_INVALID_ARG, "%s: null pointer argument", name);
  int nodes = 0;
  spade_status st = tree::check_tree(name, B, R, max_k, &nodes);
  if (st != SPADE_OK) return st;
  if (mask_words < max_k / 32 + 1)
    return fail(SPADE_ERR_SHAPE, "%s: %d mask words for blocks of %d nodes", name, mask_words, max_k + 1);
  st = device_info(nullptr, nullptr);
  if (st != SPADE_OK) return st;
  static OncePerDevice once;
  cudaError_t e = set_max_smem(once, 8 * tree::kMaxNodes, tree::layout_kernel);
  if (e != cudaSuccess) return cuda_fail(e, name);
  const tree::Layout p{parents, ctx_lens, n_draft, cu_q, positions, tree_mask, status, R, mask_words, max_k};
  e = launch(tree::layout_kernel, dim3(B), 1, tree::kThreads, 8 * static_cast<size_t>(nodes),
             reinterpret_cast<cudaStream_t>(stream), p, nodes);
  return e == cudaSuccess ? SPADE_OK : cuda_fail(e, name);
}

extern "C" spade_status spade_tree_commit(void *k_cache, void *v_cache, const int32_t *ctx_lens, const int32_t *parents,
                                          const int32_t *draft_tokens, const int32_t *target_tokens,
                                          const int32_t *n_draft, const int32_t *cu_q, int32_t *accepted_len,
                                          int32_t *next_token, int32_t *path, int32_t *new_ctx_lens, int32_t layers,
                                          int32_t B, int32_t R, int32_t Hkv, int32_t D, int32_t cap, int32_t max_k,
                                          int32_t *status, spade_stream_t stream) {
  static const char *name = "spade_tree_commit";
  tree::Commit p;
  const spade_status st = kv_cache_of(name, &p.cache, k_cache, v_cache, false, nullptr, B, Hkv, D, cap, B, 1);
  if (st != SPADE_OK) return st;
  p.layer_rows = static_cast<int64_t>(B) * Hkv * cap;
  p.ctx_lens = ctx_lens; p.parents = parents; p.drafts = draft_tokens; p.tokens = target_tokens;
  p.n_draft = n_draft; p.cu_q = cu_q; p.accepted = accepted_len; p.next_token = next_token; p.path = path;
  p.new_ctx = new_ctx_lens; p.status = status; p.layers = layers; p.R = R; p.max_k = max_k; p.planes = 0;
  return tree::commit(name, p, B, reinterpret_cast<cudaStream_t>(stream));
}

extern "C" spade_status spade_tree_commit_paged(
    void *k_pool, void *v_pool, const int32_t *block_table, const int32_t *ctx_lens, const int32_t *parents,
    const int32_t *draft_tokens, const int32_t *target_tokens, const int32_t *n_draft, const int32_t *cu_q,
    int32_t *accepted_len, int32_t *next_token, int32_t *path, int32_t *new_ctx_lens, int32_t layers, int32_t B, int32_t R,
    int32_t Hkv, int32_t D, int32_t page_size, int32_t num_pages, int32_t max_pages, int32_t max_k, int32_t *status,
    spade_stream_t stream) {
  static const char *name = "spade_tree_commit_paged";
  tree::Commit p;
  const spade_status st =
      kv_cache_of(name, &p.cache, k_pool, v_pool, true, block_table, B, Hkv, D, page_size, num_pages, max_pages);
  if (st != SPADE_OK) return st;
  p.layer_rows = static_cast<int64_t>(num_pages) * Hkv * page_size;
  p.ctx_lens = ctx_lens; p.parents = parents; p.drafts = draft_tokens; p.tokens = target_tokens;
  p.n_draft = n_draft; p.cu_q = cu_q; p.accepted = accepted_len; p.next_token = next_token; p.path = path;
  p.new_ctx = new_ctx_lens; p.status = status; p.layers = layers; p.R = R; p.max_k = max_k; p.planes = 0;
  return tree::commit(name, p, B, reinterpret_cast<cudaStream_t>(stream));
}
