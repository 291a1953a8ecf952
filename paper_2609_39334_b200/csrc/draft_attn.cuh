// Structures of ss_draft_attention shared by its planner, its tensor-core kernel and its plain kernel.
#pragma once
#include "common.cuh"

namespace ss {
namespace draft {

constexpr int kDim = 128, kPage = 16;
constexpr int kTile = 128;                   // keys per step of the tensor-core kernel: 8 pages
constexpr int kTilePages = kTile / kPage;
constexpr int kRows = 128;                   // query rows (tokens x heads of a group) of one tile; a block of rows has one or two

struct Header {
  int32_t status;                            // first: read by ss_last_device_status
  int32_t pad[63];
};
// What the planner finds out about a path.
struct alignas(16) PathInfo {
  int32_t leaf, T, L;                        // T = 0: nothing to do
  int32_t tiles;                             // steps of kTile keys, at least 1 (a path without keys writes zeros)
  int32_t blocks;                            // blocks of rows of one kv head: up to two tiles of tokens each
  int32_t per_block;                         // tokens of a block (the last may have fewer)
  int32_t holes;                             // an inner node of the chain ends inside a page
  int32_t status;                            // what is wrong with it (the next kernel hands it on: this one clears the header's)
  int64_t src, dst;                          // first row of q and of out
};
// A unit that several blocks of the grid share: its partial results, merged by draft_merge_kernel.
struct alignas(16) CutUnit {
  int32_t n;                                 // partials: slot `first`, then 2 * (block + 1), 2 * (block + 2), ...; 0: no such unit
  int32_t first, g, n_tok;
  int64_t dst;
};

// The chain of a path as segments of whole pages, in key order.
struct Chain {
  int n;
  int first[SS_MAX_DEPTH + 1];               // first page of a segment in the chain's pages
  int len[SS_MAX_DEPTH];                     // its tokens
  int start[SS_MAX_DEPTH];                   // index of its first token in the path's sequence
  int page0[SS_MAX_DEPTH];                   // its first entry in node_pages
};

struct Params {
  int Hq, Hkv, G;
  int tok_per_tile;
  float scale, scale_log2;
  const __nv_bfloat16 *k_pool, *v_pool;
  int64_t num_pages, page_stride, head_stride;
  int num_nodes;
  const int32_t *node_parent, *node_kv_len, *node_pages;
  const int64_t* node_page_offsets;
  int64_t total_node_pages;
  int num_paths;
  const int32_t *num_paths_dev, *path_leaf_node, *path_q_len, *draft_parent;
  const int64_t *q_offsets, *q_src_offsets;
  int64_t total_q, q_rows;
  const __nv_bfloat16* q;
  __nv_bfloat16* out;
  float* lse;
  // workspace
  Header* hdr;
  PathInfo* paths;
  Chain* chains;
  uint4* seen;                               // by row of out: the drafts that its token sees, one bit each
  CutUnit* cuts;                             // one per block of the grid
  float *part_o, *part_lse;                  // 2 slots per block of the grid: [slot][2 * kRows][kDim], [slot][2 * kRows]
};

#ifdef __CUDACC__
__device__ __forceinline__ void chain_of(Chain& C, const Params& P, int leaf) {
  int node[SS_MAX_DEPTH], d = 0;
  for (int a = leaf; a >= 0 && a < P.num_nodes && d < SS_MAX_DEPTH; a = P.node_parent[a]) node[d++] = a;
  int pages = 0, tokens = 0, n = 0;
  for (int c = d - 1; c >= 0; --c) {
    const int len = P.node_kv_len[node[c]];
    if (len <= 0) continue;
    C.first[n] = pages;
    C.len[n] = len;
    C.start[n] = tokens;
    C.page0[n] = static_cast<int>(P.node_page_offsets[node[c]]);
    pages += (len + kPage - 1) / kPage;
    tokens += len;
    ++n;
  }
  C.first[n] = pages;
  C.n = n;
}
// Segment of the chain's page vp (vp < first[n]).
__device__ __forceinline__ int segment_of(const Chain& C, int vp) {
  int s = 0;
  while (s + 1 < C.n && vp >= C.first[s + 1]) ++s;
  return s;
}
__device__ __forceinline__ int64_t physical_page(const Chain& C, const Params& P, int s, int vp) {
  const int64_t entry = static_cast<int64_t>(C.page0[s]) + (vp - C.first[s]);
  int64_t page = entry >= 0 && entry < P.total_node_pages ? static_cast<int64_t>(P.node_pages[entry]) : -1;
  if (page < 0 || page >= P.num_pages) {
    set_status(&P.hdr->status, SS_ERR_BAD_INPUT);
    page = 0;
  }
  return page;
}
// The tokens of page vp that a row sees, bit o = token o; `drafts0`: index of the first draft in the path's sequence, `seen`: its
// drafts.
__device__ __forceinline__ uint32_t page_mask(const Chain& C, int s, int vp, int drafts0, const uint4& seen) {
  const int in = (vp - C.first[s]) * kPage;
  const int valid = min(kPage, C.len[s] - in);
  const int d0 = C.start[s] + in - drafts0;                    // draft index of token 0 (negative: cached)
  uint32_t m;
  if (d0 <= -kPage) {
    m = 0xffffu;
  } else {
    const uint64_t lo = (static_cast<uint64_t>(seen.y) << 32) | seen.x, hi = (static_cast<uint64_t>(seen.w) << 32) | seen.z;
    if (d0 < 0) m = static_cast<uint32_t>(lo << -d0) | ((1u << -d0) - 1u);
    else if (d0 == 0) m = static_cast<uint32_t>(lo);
    else if (d0 < 64) m = static_cast<uint32_t>((lo >> d0) | (hi << (64 - d0)));
    else if (d0 < 128) m = static_cast<uint32_t>(hi >> (d0 - 64));
    else m = 0u;
  }
  return m & 0xffffu & ((1u << valid) - 1u);
}

struct Row {                                 // one query row of a warp: lane l has values 4 l .. 4 l + 3
  float q[4], acc[4], m, l;
};
__device__ __forceinline__ void load4(const __nv_bfloat16* p, float (&v)[4]) {
  const uint2 u = *reinterpret_cast<const uint2*>(p);
  v[0] = __uint_as_float(u.x << 16); v[1] = __uint_as_float(u.x & 0xffff0000u);
  v[2] = __uint_as_float(u.y << 16); v[3] = __uint_as_float(u.y & 0xffff0000u);
}
// The keys of pages [vp0, vp1) that the row sees, one after the other (all in fp32).
__device__ __forceinline__ void row_visit(Row& r, const Chain& C, const Params& P, int g, int vp0, int vp1, int drafts0, const uint4& seen,
                                          int lane) {
  vp1 = min(vp1, C.first[C.n]);
  for (int vp = vp0; vp < vp1; ++vp) {
    const int s = segment_of(C, vp);
    const int64_t base = physical_page(C, P, s, vp) * P.page_stride + static_cast<int64_t>(g) * P.head_stride + 4 * lane;
    for (uint32_t m = page_mask(C, s, vp, drafts0, seen); m; m &= m - 1) {
      const int64_t off = base + static_cast<int64_t>(__ffs(m) - 1) * kDim;
      float k[4], v[4];
      load4(P.k_pool + off, k);
      load4(P.v_pool + off, v);
      const float x = warp_sum(r.q[0] * k[0] + r.q[1] * k[1] + r.q[2] * k[2] + r.q[3] * k[3]) * P.scale;
      const float top = fmaxf(r.m, x);
      const float a = top == -INFINITY ? 1.f : __expf(r.m - top), p = top == -INFINITY ? 0.f : __expf(x - top);
      r.l = r.l * a + p;
#pragma unroll
      for (int i = 0; i < 4; ++i) r.acc[i] = r.acc[i] * a + p * v[i];
      r.m = top;
    }
  }
}
__device__ __forceinline__ void row_start(Row& r, const __nv_bfloat16* q, int lane) {
  load4(q + 4 * lane, r.q);
  r.acc[0] = r.acc[1] = r.acc[2] = r.acc[3] = 0.f;
  r.m = -INFINITY;
  r.l = 0.f;
}
__device__ __forceinline__ float row_lse(float m, float l) { return l == 0.f ? -INFINITY : m + __logf(l); }
__device__ __forceinline__ void store_out(const Params& P, int64_t row, int h, int lane, const float (&o)[4], float lse) {
  const __nv_bfloat162 a = __floats2bfloat162_rn(o[0], o[1]), b = __floats2bfloat162_rn(o[2], o[3]);
  uint2 u;
  u.x = *reinterpret_cast<const uint32_t*>(&a);
  u.y = *reinterpret_cast<const uint32_t*>(&b);
  *reinterpret_cast<uint2*>(P.out + (row * P.Hq + h) * kDim + 4 * lane) = u;
  if (P.lse && lane == 0) P.lse[row * P.Hq + h] = lse;
}
#endif

}  // namespace draft
}  // namespace ss
