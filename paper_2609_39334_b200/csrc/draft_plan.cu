// ss_draft_attention: host side, the planner, the plain kernel and the merge.
//
//   plan (a block per path: chain length, checks, and for every draft the set of drafts it sees, as 128 bits)
//     -> tensor-core kernel (draft_umma.cu)  -> merge of the units that several blocks shared
//     or the plain kernel: a warp per query row, key by key, in fp32.
//
// Planner and merge are bound by latency: the planner by the walk up a chain (a trip to memory a node) and the parents, the merge by
// reading at most 2 partials a block of the tensor-core kernel (148 blocks: at most 39 MB, mostly in the L2).  Cold, alone, they take 6.5
// and 15 us; behind each other in a stream some 5 each.
#include <math.h>
#include <string.h>

#include "draft_attn.cuh"

namespace ss {
namespace draft {

int32_t launch_tiles(const Params& P, cudaStream_t st, int blocks);

constexpr int kPlanThreads = SS_MAX_DRAFT;
constexpr int kPlainWarps = 4, kPlainBlocks = 16;              // warps of a block, blocks of a path
constexpr int kMergeWarps = 8, kMergeBlocks = 8;               // (of a shared unit)

__global__ void __launch_bounds__(kPlanThreads) draft_plan_kernel(const __grid_constant__ Params P) {
  ss::grid_dependency_enter();
  __shared__ int parent[SS_MAX_DRAFT];
  __shared__ PathInfo info;
  const int tid = threadIdx.x;
  const int live = P.num_paths_dev ? min(max(*P.num_paths_dev, 0), P.num_paths) : P.num_paths;
  if (blockIdx.x == 0 && tid == 0) P.hdr->status = SS_OK;
  for (int p = blockIdx.x; p < P.num_paths; p += gridDim.x) {
    __syncthreads();
    if (tid == 0) {
      PathInfo I = {};
      I.tiles = I.blocks = 1;
      int bad = SS_OK;
      if (p < live) {
        I.leaf = P.path_leaf_node[p];
        I.T = P.path_q_len[p];
        I.dst = P.q_offsets[p];
        I.src = P.q_src_offsets ? P.q_src_offsets[p] : I.dst;
        int64_t tokens = 0, pages = 0;
        int depth = 0, a = I.leaf;
        for (; a >= 0 && a < P.num_nodes && depth < SS_MAX_DEPTH; ++depth) {
          const int len = P.node_kv_len[a], up = P.node_parent[a];
          const int64_t e0 = P.node_page_offsets[a], e1 = P.node_page_offsets[a + 1];
          if (len < 0 || e0 < 0 || e1 > P.total_node_pages || (len + kPage - 1) / kPage > e1 - e0) bad = SS_ERR_BAD_INPUT;
          if (depth > 0 && len % kPage) I.holes = 1;
          tokens += len;
          pages += (len + kPage - 1) / kPage;
          a = up;
        }
        if (a >= 0) bad = a < P.num_nodes ? SS_ERR_UNSUPPORTED : SS_ERR_BAD_INPUT;       // deeper than SS_MAX_DEPTH
        if (I.leaf < 0 || I.leaf >= P.num_nodes || I.T < 0) bad = SS_ERR_BAD_INPUT;
        if (pages > 0 && P.num_pages < 1) bad = SS_ERR_BAD_INPUT;
        if (I.T > SS_MAX_DRAFT || tokens > 0x3fffffff) bad = SS_ERR_UNSUPPORTED;
        if (bad == SS_OK && (I.src < 0 || I.src + I.T > P.q_rows || I.dst < 0 || I.dst + I.T > P.total_q)) bad = SS_ERR_BAD_INPUT;
        I.L = static_cast<int>(tokens);
        I.tiles = pages > kTilePages ? static_cast<int>((pages + kTilePages - 1) / kTilePages) : 1;
        if (bad != SS_OK) I.T = 0;
        else chain_of(P.chains[p], P, I.leaf);
        I.status = bad;
        I.blocks = (I.T + 2 * P.tok_per_tile - 1) / (2 * P.tok_per_tile);
        if (I.blocks < 1) I.blocks = 1;
        I.per_block = (I.T + I.blocks - 1) / I.blocks;
      }
      info = I;
    }
    __syncthreads();
    const int T = info.T;
    if (tid < T) {
      int up = P.draft_parent ? P.draft_parent[info.src + tid] : tid - 1;
      if (up < -1 || up >= tid) {
        info.status = SS_ERR_BAD_INPUT;
        up = -1;
      }
      parent[tid] = up;
    }
    __syncthreads();
    if (tid == 0) P.paths[p] = info;
    if (tid < T) {
      uint32_t m[4] = {0u, 0u, 0u, 0u};
      for (int t = tid; t >= 0; t = parent[t]) {               // (a parent is smaller: it ends)
        const uint32_t b = 1u << (t & 31);
#pragma unroll
        for (int w = 0; w < 4; ++w) m[w] |= (t >> 5) == w ? b : 0u;
      }
      P.seen[info.dst + tid] = make_uint4(m[0], m[1], m[2], m[3]);
    }
  }
}

__global__ void __launch_bounds__(kPlainWarps * 32) draft_plain_kernel(const __grid_constant__ Params P) {
  ss::grid_dependency_enter();
  const int lane = threadIdx.x & 31;
  const int part = blockIdx.x % kPlainBlocks;
  for (int p = blockIdx.x / kPlainBlocks; p < P.num_paths; p += gridDim.x / kPlainBlocks) {
    const PathInfo I = P.paths[p];
    if (I.status != SS_OK && threadIdx.x == 0) set_status(&P.hdr->status, I.status);
    if (I.T == 0) continue;
    const Chain& C = P.chains[p];
    for (int x = part * kPlainWarps + (threadIdx.x >> 5); x < I.T * P.Hq; x += kPlainBlocks * kPlainWarps) {
      const int t = x / P.Hq, h = x - t * P.Hq;
      Row r;
      row_start(r, P.q + ((I.src + t) * P.Hq + h) * kDim, lane);
      row_visit(r, C, P, h / P.G, 0, C.first[C.n], I.L - I.T, P.seen[I.dst + t], lane);
      const float inv = r.l == 0.f ? 0.f : 1.f / r.l;
      const float o[4] = {r.acc[0] * inv, r.acc[1] * inv, r.acc[2] * inv, r.acc[3] * inv};
      store_out(P, I.dst + t, h, lane, r.l == 0.f ? *reinterpret_cast<const float(*)[4]>(&r.acc) : o, row_lse(r.m, r.l));
    }
  }
}

// A warp per row of a unit that was shared: out = sum_i e^(lse_i - LSE) o_i over its partials, LSE = ln sum_i e^lse_i.
__global__ void __launch_bounds__(kMergeWarps * 32) draft_merge_kernel(const __grid_constant__ Params P) {
  ss::grid_dependency_enter();
  const int lane = threadIdx.x & 31, block = blockIdx.x / kMergeBlocks, part = blockIdx.x % kMergeBlocks;
  const CutUnit u = P.cuts[block];
  if (u.n == 0) return;
  for (int r = part * kMergeWarps + (threadIdx.x >> 5); r < u.n_tok * P.G; r += kMergeBlocks * kMergeWarps) {
    const int t = r / P.G, h = u.g * P.G + r - t * P.G;
    // (tokens of the second tile of a block start at row kRows)
    const int at = t < P.tok_per_tile ? r : kRows + r - P.tok_per_tile * P.G;
    auto slot = [&](int i) { return static_cast<int64_t>(i ? 2 * (block + i) : u.first) * (2 * kRows) + at; };
    float top = -INFINITY;
    for (int i = lane; i < u.n; i += 32) top = fmaxf(top, P.part_lse[slot(i)]);
    top = warp_max(top);
    float acc[4] = {0.f, 0.f, 0.f, 0.f}, sum = 0.f;
    for (int i0 = 0; i0 < u.n; i0 += 32) {
      const float mine = i0 + lane < u.n ? P.part_lse[slot(i0 + lane)] : -INFINITY;
      const float w_mine = mine == -INFINITY ? 0.f : __expf(mine - top);
      const int n = min(32, u.n - i0);
#pragma unroll 4
      for (int i = 0; i < n; ++i) {
        const float w = __shfl_sync(0xffffffffu, w_mine, i);
        const float4 o = *reinterpret_cast<const float4*>(P.part_o + slot(i0 + i) * kDim + 4 * lane);
        sum += w;
        if (w != 0.f) {                                        // (a NaN stays one)
          acc[0] = fmaf(w, o.x, acc[0]); acc[1] = fmaf(w, o.y, acc[1]); acc[2] = fmaf(w, o.z, acc[2]); acc[3] = fmaf(w, o.w, acc[3]);
        }
      }
    }
    const float inv = sum == 0.f ? 0.f : 1.f / sum;
    const float o[4] = {acc[0] * inv, acc[1] * inv, acc[2] * inv, acc[3] * inv};
    store_out(P, u.dst + t, h, lane, o, row_lse(top, sum));
  }
}

static int32_t check_desc(const ss_attn_desc_t* d) {
  if (!d || d->struct_size != sizeof(ss_attn_desc_t)) return SS_ERR_INVALID_ARG;
  if (d->flags & ~(SS_FLAG_VALIDATE | SS_FLAG_FORCE_GENERIC | SS_FLAG_NO_TCGEN05 | SS_FLAG_TILES_2CTA)) return SS_ERR_INVALID_ARG;
  if (d->num_q_heads < 1 || d->num_kv_heads < 1 || d->num_nodes < 0 || d->num_paths < 0 || d->total_q < 0 || d->total_node_pages < 0 ||
      d->num_pages < 0 || d->max_sms < 0 || (d->q_src_offsets && d->q_src_rows < 0))
    return SS_ERR_INVALID_ARG;
  if (d->head_dim != kDim || d->page_size != kPage || d->num_q_heads % d->num_kv_heads || d->num_q_heads / d->num_kv_heads > kRows)
    return SS_ERR_UNSUPPORTED;
  if (d->kv_token_stride != kDim || d->kv_page_stride % 128 || d->kv_head_stride % 128 || d->kv_page_stride <= 0 || d->kv_head_stride <= 0)
    return SS_ERR_UNSUPPORTED;
  if (!(d->sm_scale >= 0.f) || isinf(d->sm_scale)) return SS_ERR_INVALID_ARG;
  const int64_t most = 0x7fffffffLL / d->num_q_heads;
  if (d->total_q > most || (d->q_src_offsets && d->q_src_rows > most) || d->total_node_pages > 0x7fffffffLL) return SS_ERR_UNSUPPORTED;
  return SS_OK;
}

static size_t carve(const ss_attn_desc_t* d, void* base, Params* P) {
  Carver c(base);
  const size_t blocks = static_cast<size_t>(sm_count_of_current_device());
  P->hdr = c.take<Header>(1);
  P->paths = c.take<PathInfo>(static_cast<size_t>(d->num_paths) + 1);
  P->chains = c.take<Chain>(static_cast<size_t>(d->num_paths) + 1);
  P->seen = c.take<uint4>(static_cast<size_t>(d->total_q) + 1);
  P->cuts = c.take<CutUnit>(blocks);
  P->part_lse = c.take<float>(blocks * 2 * 2 * kRows);
  P->part_o = c.take<float>(blocks * 2 * 2 * kRows * kDim);
  return c.off;
}

}  // namespace draft
}  // namespace ss

extern "C" int32_t ss_draft_attention_workspace_bytes(const ss_attn_desc_t* desc, size_t* out_bytes) {
  using namespace ss::draft;
  if (!out_bytes) return SS_ERR_INVALID_ARG;
  const int32_t rc = check_desc(desc);
  if (rc != SS_OK) return rc;
  Params P;
  *out_bytes = carve(desc, nullptr, &P);
  return SS_OK;
}

extern "C" int32_t ss_draft_attention(const ss_attn_desc_t* d, const int32_t* draft_parent, void* workspace, size_t workspace_bytes,
                                      void* stream) {
  using namespace ss::draft;
  const int32_t rc = check_desc(d);
  if (rc != SS_OK) return rc;
  if (!workspace || reinterpret_cast<uintptr_t>(workspace) % ss::kAlign) return SS_ERR_INVALID_ARG;
  if (!d->k_pool || !d->v_pool || !d->node_parent || !d->node_kv_len || !d->node_page_offsets || !d->node_pages || !d->path_leaf_node ||
      !d->path_q_len || !d->q_offsets)
    return SS_ERR_INVALID_ARG;
  if (d->total_q > 0 && (!d->q || !d->out)) return SS_ERR_INVALID_ARG;
  if (reinterpret_cast<uintptr_t>(d->k_pool) % 256 || reinterpret_cast<uintptr_t>(d->v_pool) % 256 || reinterpret_cast<uintptr_t>(d->q) % 16 ||
      reinterpret_cast<uintptr_t>(d->out) % 32)
    return SS_ERR_UNSUPPORTED;
  Params P;
  memset(&P, 0, sizeof P);
  if (workspace_bytes < carve(d, workspace, &P)) return SS_ERR_WORKSPACE_TOO_SMALL;
  P.Hq = d->num_q_heads;
  P.Hkv = d->num_kv_heads;
  P.G = P.Hq / P.Hkv;
  P.tok_per_tile = kRows / P.G;
  P.scale = d->sm_scale > 0.f ? d->sm_scale : 1.0f / sqrtf(static_cast<float>(kDim));
  P.scale_log2 = P.scale * 1.4426950408889634f;
  P.k_pool = static_cast<const __nv_bfloat16*>(d->k_pool);
  P.v_pool = static_cast<const __nv_bfloat16*>(d->v_pool);
  P.num_pages = d->num_pages;
  P.page_stride = d->kv_page_stride;
  P.head_stride = d->kv_head_stride;
  P.num_nodes = d->num_nodes;
  P.node_parent = d->node_parent;
  P.node_kv_len = d->node_kv_len;
  P.node_page_offsets = d->node_page_offsets;
  P.node_pages = d->node_pages;
  P.total_node_pages = d->total_node_pages;
  P.num_paths = d->num_paths;
  P.num_paths_dev = d->num_paths_dev;
  P.path_leaf_node = d->path_leaf_node;
  P.path_q_len = d->path_q_len;
  P.draft_parent = draft_parent;
  P.q_offsets = d->q_offsets;
  P.q_src_offsets = d->q_src_offsets;
  P.total_q = d->total_q;
  P.q_rows = d->q_src_offsets ? d->q_src_rows : d->total_q;
  P.q = static_cast<const __nv_bfloat16*>(d->q);
  P.out = static_cast<__nv_bfloat16*>(d->out);
  P.lse = d->lse;
  cudaStream_t st = ss::as_stream(stream);
  int sms = ss::sm_count_of_current_device();
  if (d->max_sms > 0 && d->max_sms < sms) sms = d->max_sms;
  SS_LAUNCH(draft_plan_kernel, d->num_paths < 1 ? 1 : d->num_paths < 65535 ? d->num_paths : 65535, kPlanThreads, 0, st, P);
  if (d->num_paths == 0) return SS_OK;
  // (without rows as well: it has none to work on then, and hands on what the planner found wrong)
  if (d->total_q == 0 || (d->flags & (SS_FLAG_FORCE_GENERIC | SS_FLAG_NO_TCGEN05))) {
    SS_LAUNCH(draft_plain_kernel, static_cast<unsigned>(d->num_paths < 65535 ? d->num_paths : 65535) * kPlainBlocks, kPlainWarps * 32, 0, st, P);
    return SS_OK;
  }
  const int32_t tiles = launch_tiles(P, st, sms);
  if (tiles != SS_OK) return tiles;
  SS_LAUNCH(draft_merge_kernel, sms * kMergeBlocks, kMergeWarps * 32, 0, st, P);
  return SS_OK;
}
