// Structures of ss_key_weights shared by its planner, its tensor-core kernel and its plain kernel.
#pragma once
#include "common.cuh"

namespace ss {
namespace keyw {

constexpr int kDim = 128, kPage = 16;
constexpr int kTile = 128;                   // keys of a unit: 8 pages
constexpr int kTilePages = kTile / kPage;
constexpr int kCols = 128;                   // query rows (tokens x heads of a group) of a step, at most
constexpr int kTileCost = 8;                 // (of keys and what a unit takes besides, in 16 query rows)
constexpr int kLeastQuota = 2 * (kTileCost + kCols / 16);     // a block's share: at least a step of two tiles, wherever it starts

struct Header {
  int32_t status;                            // first: read by ss_last_device_status
  int32_t n_recs;
  int64_t total;                             // cost of all units
  int32_t pad[60];
};
// A node with something to do.  Its units are (pair of tiles of keys, kv head), head by head; each has `steps` steps of kCols / G tokens.
struct alignas(16) Rec {
  int64_t off;                               // cost of what is in front of it
  int64_t page0;                             // its first entry in node_pages
  int len;                                   // keys
  int row0, rows;                            // tokens that add to them, in the table of rows
  int steps;
  int known;                                 // keys in front of the step's own
  int hides;                                 // token x of the rows sees keys < len - hides + x + 1 only (0: all are seen)
  int order0;                                // sequence number of key `known`
  int cost;                                  // of a tile: kTileCost, and 1 for 16 query rows
};

struct Params {
  int Hq, Hkv, G;
  float scale, scale_log2, decay;
  int last_tokens;
  const __nv_bfloat16* k_pool;
  int64_t num_pages, page_stride, head_stride;
  int num_nodes;
  const int32_t *node_parent, *node_kv_len, *node_pages;
  const int64_t* node_page_offsets;
  int64_t total_node_pages;
  int num_paths;
  const int32_t *num_paths_dev, *path_leaf_node, *path_q_len, *path_order;
  const int64_t *q_offsets, *q_src_offsets;
  int64_t total_q, q_rows;
  const __nv_bfloat16* q;
  const float* lse;
  const float* weights_in;
  float* weights_out;
  int32_t* order;
  // workspace
  Header* hdr;
  Rec* recs;
  int2* rows;                                // of a token: row of q, row of lse
  int *first, *last, *below, *fresh, *leaf_path;     // by node: paths below it, their number, longest step that it is the leaf of, whose
  int *path_row, *path_start;                // by path: its first token in the table, sequence number of its step's first token
  float* part;                               // [2 per block of the grid][2 tiles][kTile]: a block's sums of a unit that it shares
  int* arrived;                              // [block of the grid][tile]: how many have left theirs of the unit that starts there and goes on
};

#ifdef __CUDACC__
__device__ __forceinline__ int64_t page_of(const Params& P, const Rec& R, int i) {
  const int64_t page = __ldg(P.node_pages + R.page0 + i / kPage);
  if (page >= 0 && page < P.num_pages) return page;
  set_status(&P.hdr->status, SS_ERR_BAD_INPUT);
  return -1;
}
// What a key's sum becomes, on its page.
__device__ __forceinline__ void store_key(const Params& P, const Rec& R, int64_t page, int g, int i, float sum, float before) {
  const int64_t at = (page * P.Hkv + g) * kPage + i % kPage;
  P.weights_out[at] = fmaf(P.decay, before, sum);
  if (P.order && i >= R.known) P.order[at] = R.order0 + (i - R.known);
}
__device__ __forceinline__ float load_before(const Params& P, const Rec& R, int64_t page, int g, int i) {
  return P.weights_in && i < R.known ? P.weights_in[(page * P.Hkv + g) * kPage + i % kPage] : 0.f;
}
#endif

}  // namespace keyw
}  // namespace ss
