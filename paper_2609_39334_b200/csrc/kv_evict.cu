// ss_kv_evict: the keys of least weight leave the nodes of the cache, what stays is brought together in a node's first slots.
//
// Per node of n keys and kv head: k = min(keep, n) keys stay, chosen by (must stay, weight, slot).  Kept keys in slots < k remain where
// they are; the i-th kept key behind them goes into the i-th free slot < k.  So no slot is read that another move writes, at most
// min(k, n - k) keys move, and a call may be repeated.
//
//   evict_nodes_kernel   checks the nodes, copies what the others need of them, writes the new lengths (which may be the tree's own)
//   evict_select_kernel  a cluster of blocks per node and kv head, each with a stretch of slots: the border between what stays and what goes
//                        by at most three histograms of 2048 bins over a range that shrinks (the first from the smallest to the largest
//                        weight; done when a bin stays as a whole), then ranks by counts, and lists of free slots and of late keys
//   evict_move_kernel    blocks for every node and head: the moves
// Bound: the moves by HBM, 256 bytes here and there (256 nodes of 2048 to 4096 keys cut to half, 4 heads: 268 us a call, some 4.5 TB/s while they move); the
// selection by latency (131072 keys of 8 heads: 51 us of 112).  One kernel that selects and moves took 353 and 263 us.
#include <string.h>

#include "common.cuh"

namespace ss {
namespace evict {

constexpr int kDim = 128, kPage = 16;
constexpr int kNodesThreads = 1024;
constexpr int kThreads = 512, kWarps = kThreads / 32;
constexpr int kBins = 2048, kBinBits = 11;
constexpr int kPasses = 3;                     // 33 bits
constexpr int kMostCluster = 8;
static_assert(kBins == 4 * kThreads && kBins % kMostCluster == 0, "bins of a thread, and of a block");
constexpr int kStaged = 16384;                 // ranks of a block's slots that are kept in shared memory, at most; behind them they are made again
constexpr int kAhead = 4;                      // quads of slots that a thread has on their way
constexpr int64_t kMostPages = (0x80000000LL - 2 * 4 * kThreads * kAhead) / kPage;       // (slots and what is looked at behind them, in 32 bits)
constexpr int kMoveThreads = 256, kMoveWarps = kMoveThreads / 32, kBatch = 4;
constexpr uint32_t kMust = 0xffffffffu;
constexpr uint32_t kAllTies = 0xffffffffu;

struct Header {
  int32_t status;                              // first: read by ss_last_device_status
  int32_t pad[63];
};
struct alignas(16) Node {
  int64_t page0;                               // its first entry in node_pages
  int n, k;                                    // keys, keys that stay; k < 0: not a node to work on
};
struct Params {
  int Hkv;
  __nv_bfloat16 *k_pool, *v_pool;
  int64_t num_pages, page_stride, head_stride, total_node_pages;
  int num_nodes;
  const int32_t *node_kv_len, *node_pages;
  const int64_t* node_page_offsets;
  int n, sinks, recent;
  int staged;                                  // room for so many ranks in a block's shared memory
  int move_blocks;                             // of a node and head
  const int32_t *nodes, *keep;
  const float* weights;
  float* weights_out;
  const int32_t* order;
  int32_t *order_out, *source_out, *kv_len_out;
  // workspace
  Header* hdr;
  Node* info;
  int32_t* claim;                              // per node of the tree: the smallest index at which it is listed
  int32_t* moves;                              // per node and head: how many
  int32_t* lists;                              // per slot of node_pages and head: free slots and late keys
};

__global__ void __launch_bounds__(kNodesThreads) evict_nodes_kernel(const __grid_constant__ Params P) {
  ss::grid_dependency_enter();
  __shared__ int bad;
  if (threadIdx.x == 0) bad = 0;
  // (a node that is listed twice is taken once: its blocks would write the same lists)
  const int mine = static_cast<int>(threadIdx.x) < P.n ? P.nodes[threadIdx.x] : -1;
  auto for_each = [&](auto f) {
    for (int i = threadIdx.x; i < P.n; i += kNodesThreads) {
      const int node = i < kNodesThreads ? mine : P.nodes[i];
      f(i, node, node >= 0 && node < P.num_nodes);
    }
    __syncthreads();
  };
  for_each([&](int, int node, bool there) { if (there) P.claim[node] = INT32_MAX; });
  for_each([&](int i, int node, bool there) { if (there) atomicMin(P.claim + node, i); });
  for_each([&](int i, int node, bool there) {
    Node I = {0, 0, -1};
    if (there && P.claim[node] == i) {
      const int n = P.node_kv_len[node];
      const int64_t e0 = P.node_page_offsets[node], e1 = P.node_page_offsets[node + 1];
      if (n >= 0 && e0 >= 0 && e1 <= P.total_node_pages && (static_cast<int64_t>(n) + kPage - 1) / kPage <= e1 - e0)
        I = {e0, n, min(max(P.keep[i], 0), n)};
    }
    if (I.k < 0) bad = 1;
    P.info[i] = I;
  });
  for_each([&](int i, int node, bool) {        // (behind all reads of the lengths, which these may be)
    if (P.kv_len_out && P.info[i].k >= 0) P.kv_len_out[node] = P.info[i].k;
  });
  if (threadIdx.x == 0) P.hdr->status = bad ? SS_ERR_BAD_INPUT : SS_OK;
}

__device__ __forceinline__ uint32_t cluster_rank() { uint32_t r; asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r)); return r; }
__device__ __forceinline__ uint32_t cluster_size() { uint32_t r; asm volatile("mov.u32 %0, %%cluster_nctarank;" : "=r"(r)); return r; }
__device__ __forceinline__ void cluster_sync() {
  asm volatile("barrier.cluster.arrive.release;" ::: "memory");
  asm volatile("barrier.cluster.wait.acquire;" ::: "memory");
}
__device__ __forceinline__ void blocks_sync(uint32_t blocks) {
  if (blocks == 1) __syncthreads(); else cluster_sync();
}
// Address of the same variable in block `rank` of the cluster.
__device__ __forceinline__ uint32_t remote(const void* p, uint32_t rank) {
  uint32_t r;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(static_cast<uint32_t>(__cvta_generic_to_shared(p))), "r"(rank));
  return r;
}
__device__ __forceinline__ uint32_t load_remote(uint32_t at) {
  uint32_t v;
  asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(v) : "r"(at) : "memory");
  return v;
}

// What a block tells the others of its cluster.
struct Told {
  uint32_t lowest, highest, must;              // ranks that go by weight, number of keys that must stay
  int last;                                    // largest order
  uint32_t holes, late, share;
};
struct Shared {
  uint32_t own[2][kBins];                      // this block's keys by bin, in passes in turn
  Told told;
  uint32_t warp_sum[2][kWarps + 1];
  uint32_t warp_lo[kWarps], warp_hi[kWarps];
  int warp_last[kWarps];
  uint32_t pick_bin, pick_left, pick_whole;
  uint32_t kept[kStaged / 32];
};

struct Work {                                  // a node and head
  const Params* P;
  int64_t page0;
  int n, g;
  __device__ __forceinline__ int64_t page(int slot) const {
    const int64_t p = __ldg(P->node_pages + page0 + slot / kPage);
    return p >= 0 && p < P->num_pages ? p : -1;
  }
  __device__ __forceinline__ int64_t beside(int64_t page, int slot) const { return (page * P->Hkv + g) * kPage + slot % kPage; }
  // (signed values in an order of unsigned ones; -0 is 0, NaN ranks last)
  __device__ __forceinline__ uint32_t rank_of(float weight, int o, int last) const {
    if (o < P->sinks || static_cast<int64_t>(o) > static_cast<int64_t>(last) - P->recent) return kMust;
    const float w = weight + 0.f;
    if (w != w) return 0u;
    const uint32_t u = __float_as_uint(w);
    return u >> 31 ? ~u : u | 0x80000000u;
  }
  __device__ __forceinline__ uint32_t rank(int slot, int last) const {
    const int64_t pg = page(slot);
    if (pg < 0) return 0u;
    const int64_t at = beside(pg, slot);
    return rank_of(P->weights[at], P->order ? P->order[at] : slot, last);
  }
};

// f(first slot of the first of kAhead quads, 4 * kThreads apart and so at the same place of their pages; their pages, -1: bad, -2: behind the end)
// for all quads of [s0, s1) (whole block; s0 a multiple of 32).
template <typename F>
__device__ __forceinline__ void for_quads(const Work& W, int s0, int s1, F f) {
  for (int i0 = s0 + 4 * static_cast<int>(threadIdx.x); i0 < s1; i0 += 4 * kThreads * kAhead) {
    int64_t page[kAhead];
#pragma unroll
    for (int x = 0; x < kAhead; ++x) page[x] = i0 + x * 4 * kThreads < s1 ? W.page(i0 + x * 4 * kThreads) : -2;
    f(i0, page);
  }
}

// Sum over the block's warps in front of this one; *total: over all.  (One of two buffers: the other may still be read.)
__device__ __forceinline__ uint32_t block_before(uint32_t warp_count, Shared& S, int buffer, uint32_t* total) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  if (lane == 0) S.warp_sum[buffer][warp] = warp_count;
  __syncthreads();
  uint32_t before = 0, all = 0;
#pragma unroll
  for (int w = 0; w < kWarps; ++w) {
    const uint32_t c = S.warp_sum[buffer][w];
    before += w < warp ? c : 0u;
    all += c;
  }
  *total = all;
  return before;
}

__global__ void __launch_bounds__(kThreads) evict_select_kernel(const __grid_constant__ Params P) {
  ss::grid_dependency_enter();
  extern __shared__ uint32_t staged[];         // ranks of the block's first slots
  __shared__ Shared S;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const uint32_t r = cluster_rank(), C = cluster_size();
  const int64_t pair = blockIdx.x / C;
  const Node I = P.info[pair / P.Hkv];
  Work W;
  W.P = &P;
  W.page0 = I.page0;
  W.n = I.n;
  W.g = static_cast<int>(pair % P.Hkv);
  const int n = I.n, k = I.k;
  const int stretch = (static_cast<int>((static_cast<int64_t>(n) + C - 1) / C) + 31) / 32 * 32;    // slots of a block
  const int s0 = static_cast<int>(min(static_cast<int64_t>(stretch) * r, static_cast<int64_t>(n))), s1 = min(s0 + stretch, n);
  if (k <= 0 || k == n) {                      // (the whole cluster) nothing moves
    if (r == 0 && tid == 0) P.moves[pair] = 0;
    for (int i = s0 + tid; i < s1; i += kThreads) {
      const int64_t pg = W.page(i);
      if (pg < 0) set_status(&P.hdr->status, SS_ERR_BAD_INPUT);
      if (pg < 0 || k == 0) continue;
      const int64_t at = W.beside(pg, i);
      if (P.weights_out != P.weights) P.weights_out[at] = P.weights[at];
      if (P.order_out && P.order_out != P.order) P.order_out[at] = P.order ? P.order[at] : i;
      if (P.source_out) P.source_out[at] = i;
    }
    return;
  }

  // ---- the largest order of the node
  int last = n - 1;
  if (P.order && P.recent > 0) {
    int mine = INT32_MIN;
    for_quads(W, s0, s1, [&](int i0, const int64_t (&page)[kAhead]) {
      int4 o[kAhead];
#pragma unroll
      for (int x = 0; x < kAhead; ++x)
        if (page[x] >= 0) o[x] = *reinterpret_cast<const int4*>(P.order + W.beside(page[x], i0));
#pragma unroll
      for (int x = 0; x < kAhead; ++x) {
        const int i = i0 + x * 4 * kThreads;
        if (page[x] < 0) continue;
        mine = max(mine, o[x].x);
        if (i + 1 < s1) mine = max(mine, o[x].y);
        if (i + 2 < s1) mine = max(mine, o[x].z);
        if (i + 3 < s1) mine = max(mine, o[x].w);
      }
    });
    mine = __reduce_max_sync(0xffffffffu, mine);
    if (lane == 0) S.warp_last[warp] = mine;
    __syncthreads();
    if (tid == 0) {
      for (int w = 1; w < kWarps; ++w) mine = max(mine, S.warp_last[w]);
      S.told.last = mine;
    }
    blocks_sync(C);
    last = INT32_MIN;
    for (uint32_t c = 0; c < C; ++c) last = max(last, static_cast<int>(load_remote(remote(&S.told.last, c))));
  } else if (P.order) {
    last = INT32_MAX;                          // (recent = 0: no order is larger)
  }

  // ---- ranks, their range, how many must stay
  uint32_t lo = 0xffffffffu, hi = 0, must = 0;
  for_quads(W, s0, s1, [&](int i0, const int64_t (&page)[kAhead]) {
    float4 w[kAhead];
    int4 o[kAhead];
#pragma unroll
    for (int x = 0; x < kAhead; ++x) {
      const int i = i0 + x * 4 * kThreads;
      w[x] = make_float4(0.f, 0.f, 0.f, 0.f);
      o[x] = make_int4(i, i + 1, i + 2, i + 3);
      if (page[x] >= 0) {
        const int64_t at = W.beside(page[x], i0);
        w[x] = *reinterpret_cast<const float4*>(P.weights + at);
        if (P.order) o[x] = *reinterpret_cast<const int4*>(P.order + at);
      } else if (page[x] == -1) {
        set_status(&P.hdr->status, SS_ERR_BAD_INPUT);
      }
    }
#pragma unroll
    for (int x = 0; x < kAhead; ++x) {
      const int i = i0 + x * 4 * kThreads;
      const float wx[4] = {w[x].x, w[x].y, w[x].z, w[x].w};
      const int ox[4] = {o[x].x, o[x].y, o[x].z, o[x].w};
#pragma unroll
      for (int y = 0; y < 4; ++y) {
        if (i + y >= s1) continue;
        const uint32_t u = page[x] >= 0 ? W.rank_of(wx[y], ox[y], last) : 0u;
        if (i + y - s0 < P.staged) staged[i + y - s0] = u;
        if (u == kMust) ++must;
        else { lo = min(lo, u); hi = max(hi, u); }
      }
    }
  });
  lo = __reduce_min_sync(0xffffffffu, lo);
  hi = __reduce_max_sync(0xffffffffu, hi);
  must = __reduce_add_sync(0xffffffffu, must);
  if (lane == 0) { S.warp_lo[warp] = lo; S.warp_hi[warp] = hi; }
  uint32_t must_here;
  (void)block_before(must, S, 0, &must_here);
  if (tid == 0) {
    for (int w = 0; w < kWarps; ++w) { lo = min(lo, S.warp_lo[w]); hi = max(hi, S.warp_hi[w]); }
    S.told.lowest = lo;
    S.told.highest = hi;
    S.told.must = must_here;
    S.pick_bin = S.pick_left = S.pick_whole = 0;
  }
  blocks_sync(C);
  uint32_t must_all = 0;
  lo = 0xffffffffu;
  hi = 0;
  for (uint32_t c = 0; c < C; ++c) {
    lo = min(lo, load_remote(remote(&S.told.lowest, c)));
    hi = max(hi, load_remote(remote(&S.told.highest, c)));
    must_all += load_remote(remote(&S.told.must, c));
  }
  auto rank_of = [&](int i) { return i - s0 < P.staged ? staged[i - s0] : W.rank(i, last); };

  // ---- the border: `border` the smallest rank that stays, `ties` how many keys of that rank do, by slot
  uint32_t border = kMust, ties = static_cast<uint32_t>(k), ties_before = 0;
  if (must_all >= static_cast<uint32_t>(k)) {  // among those that must stay
    for (uint32_t c = 0; c < r; ++c) ties_before += load_remote(remote(&S.told.must, c));
  } else {
    uint32_t left = static_cast<uint32_t>(k) - must_all;       // of those that go by weight, in [lo, hi]
    for (int pass = 0; pass < kPasses; ++pass) {
      uint32_t (&own)[kBins] = S.own[pass & 1];                // (the other one may still be read)
      const uint32_t range = hi - lo;
      const int shift = range >= kBins ? 32 - __clz(range) - kBinBits : 0;       // (range >> shift) < kBins
      for (int i = tid; i < kBins; i += kThreads) own[i] = 0;
      __syncthreads();
      for (int i = s0 + tid; i < s1; i += kThreads) {
        const uint32_t u = rank_of(i);
        if (u != kMust && u >= lo && u <= hi) atomicAdd(&own[(u - lo) >> shift], 1u);
      }
      blocks_sync(C);
      // The bin in which the border lies.  Bins from the top; a block adds up its share of them over the cluster, then all look at the shares' sums, and
      // the block that has the border in its share tells.  (All bins of all blocks read by every block: a cluster of 8 took 76 us for 131072 keys
      // a head, one of 16 172.)
      const int share = kBins / static_cast<int>(C), mine_n = max(1, share / kThreads), bin0 = static_cast<int>(r) * share + mine_n * tid;
      uint32_t c[4] = {0u, 0u, 0u, 0u}, sum = 0;
#pragma unroll
      for (int x = 0; x < 4; ++x) {
        if (x >= mine_n || mine_n * tid >= share) continue;
        for (uint32_t b = 0; b < C; ++b) c[x] += load_remote(remote(&own[kBins - 1 - (bin0 + x)], b));
        sum += c[x];
      }
      uint32_t incl = sum;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const uint32_t up = __shfl_up_sync(0xffffffffu, incl, o);
        if (lane >= o) incl += up;
      }
      uint32_t share_sum;
      uint32_t above = block_before(__shfl_sync(0xffffffffu, incl, 31), S, pass & 1, &share_sum) + incl - sum;
      if (tid == 0) S.told.share = share_sum;
      blocks_sync(C);
      uint32_t before = 0, owner = 0;
      for (uint32_t b = 0; b < C; ++b) {
        const uint32_t t = load_remote(remote(&S.told.share, b));
        if (before + t < left) { before += t; owner = b + 1; } else break;
      }
      if (owner == r) {
        above += before;
#pragma unroll
        for (int x = 0; x < 4; ++x) {
          if (c[x] && above < left && left <= above + c[x]) {
            S.pick_bin = static_cast<uint32_t>(kBins - 1 - (bin0 + x));
            S.pick_left = left - above;
            S.pick_whole = left == above + c[x];
          }
          above += c[x];
        }
      }
      owner = min(owner, C - 1);
      blocks_sync(C);
      const uint32_t bin = load_remote(remote(&S.pick_bin, owner));
      const bool whole = load_remote(remote(&S.pick_whole, owner)) != 0;
      left = load_remote(remote(&S.pick_left, owner));
      lo += bin << shift;
      hi = shift ? min(hi, lo + ((1u << shift) - 1u)) : lo;
      if (whole) {                             // (all blocks at once) all of the bin stay, and none of it is tied with what goes
        left = kAllTies;
        break;
      }
      if (lo == hi) {                          // this block's keys of the border's rank are in own[bin]
        if (tid == 0) S.told.must = own[bin];
        blocks_sync(C);
        for (uint32_t c2 = 0; c2 < r; ++c2) ties_before += load_remote(remote(&S.told.must, c2));
        break;
      }
      __syncthreads();
    }
    border = lo;
    ties = left;
  }

  // ---- who stays.  A warp has a stretch of rows of 32 slots; ties by slot.
  const int rows = (s1 - s0 + 31) / 32, per = (rows + kWarps - 1) / kWarps;
  const int row0 = min(warp * per, rows), row1 = min(row0 + per, rows);
  uint32_t mine = 0;
  if (ties != kAllTies) {
    for (int w = row0; w < row1; ++w) {
      const int i = s0 + 32 * w + lane;
      mine += __popc(__ballot_sync(0xffffffffu, i < s1 && rank_of(i) == border));
    }
  }
  uint32_t unused;
  __syncthreads();
  uint32_t tie = ties_before + block_before(mine, S, 0, &unused);
  // Bits of the row's kept keys (whole warp, rows in order).
  auto kept_row = [&](int w) {
    const int i = s0 + 32 * w + lane;
    const uint32_t u = i < s1 ? rank_of(i) : 0u;
    const uint32_t even = __ballot_sync(0xffffffffu, i < s1 && u == border);
    const uint32_t number = tie + __popc(even & ((1u << lane) - 1u));
    tie += __popc(even);
    return __ballot_sync(0xffffffffu, i < s1 && (u > border || (u == border && number < ties)));
  };
  const uint32_t tie0 = tie;
  uint32_t holes = 0, late = 0;
  auto below = [&](int w) -> uint32_t {        // bits of the row's slots < k
    const int d = k - (s0 + 32 * w);
    return d >= 32 ? 0xffffffffu : d <= 0 ? 0u : (1u << d) - 1u;
  };
  for (int w = row0; w < row1; ++w) {
    const uint32_t bits = kept_row(w), front = below(w);
    if (w < kStaged / 32 && lane == 0) S.kept[w] = bits;
    holes += __popc(~bits & front);
    late += __popc(bits & ~front);
  }
  __syncwarp();
  uint32_t holes_here, late_here;
  uint32_t hole_at = block_before(holes, S, 1, &holes_here);
  __syncthreads();
  uint32_t late_at = block_before(late, S, 0, &late_here);
  if (tid == 0) { S.told.holes = holes_here; S.told.late = late_here; }
  blocks_sync(C);
  uint32_t moves = 0;
  for (uint32_t c = 0; c < C; ++c) {
    const uint32_t h = load_remote(remote(&S.told.holes, c));
    if (c < r) { hole_at += h; late_at += load_remote(remote(&S.told.late, c)); }
    moves += h;
  }
  if (r == 0 && tid == 0) P.moves[pair] = static_cast<int>(moves);
  const int pages = (n + kPage - 1) / kPage;
  int32_t* free_list = P.lists + (W.page0 * P.Hkv + static_cast<int64_t>(W.g) * pages) * kPage;
  int32_t* late_list = free_list + pages * (kPage / 2);
  const bool noted = row1 <= kStaged / 32;     // (a row's ties go by all the rows in front of it)
  const bool copies = P.weights_out != P.weights || (P.order_out && P.order_out != P.order) || P.source_out;
  tie = tie0;
#pragma unroll 4
  for (int w = row0; w < row1; ++w) {
    const uint32_t bits = noted ? S.kept[w] : kept_row(w), front = below(w), me = 1u << lane;
    const uint32_t hole = ~bits & front, behind = bits & ~front;
    const int i = s0 + 32 * w + lane;
    if (hole & me) free_list[hole_at + __popc(hole & (me - 1u))] = i;
    if (behind & me) late_list[late_at + __popc(behind & (me - 1u))] = i;
    hole_at += __popc(hole);
    late_at += __popc(behind);
    if (copies && (bits & front & me)) {       // remains
      const int64_t pg = W.page(i);
      if (pg >= 0) {
        const int64_t at = W.beside(pg, i);
        if (P.weights_out != P.weights) P.weights_out[at] = P.weights[at];
        if (P.order_out && P.order_out != P.order) P.order_out[at] = P.order ? P.order[at] : i;
        if (P.source_out) P.source_out[at] = i;
      }
    }
  }
  blocks_sync(C);                              // (no block leaves while another may read what it tells)
}

// The moves of a node and head, P.move_blocks blocks for them: kBatch at a time a warp, whose places are looked up, and whose weights and orders
// moved, by a lane each, a batch ahead; their rows by the warp together, K in the lower lanes, V in the upper.
// (Batches of 16, 8, 4 with 2, 4, 6 blocks an SM: 339, 313, 279 us a call for 256 nodes of 2048 to 4096 keys cut to half, 4 heads.)
__global__ void __launch_bounds__(kMoveThreads, 6) evict_move_kernel(const __grid_constant__ Params P) {
  ss::grid_dependency_enter();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int64_t pair = blockIdx.x / P.move_blocks;
  const int part = static_cast<int>(blockIdx.x - pair * P.move_blocks);
  const int moves = P.moves[pair];
  const Node I = P.info[pair / P.Hkv];
  Work W;
  W.P = &P;
  W.page0 = I.page0;
  W.n = I.n;
  W.g = static_cast<int>(pair % P.Hkv);
  const int pages = (I.n + kPage - 1) / kPage, stride = P.move_blocks * kMoveWarps * kBatch;
  const int32_t* free_list = P.lists + (W.page0 * P.Hkv + static_cast<int64_t>(W.g) * pages) * kPage;
  const int32_t* late_list = free_list + pages * (kPage / 2);
  __nv_bfloat16* pool = (lane < 16 ? P.k_pool : P.v_pool) + static_cast<int64_t>(W.g) * P.head_stride + (lane & 15) * 8;
  int to = -1, from = -1;                      // of the lane's move: page * 16 + slot; -1: none
  auto look = [&](int j0) {
    to = from = -1;
    if (lane < kBatch && j0 + lane < moves) {
      const int dst = free_list[j0 + lane], src = late_list[j0 + lane];
      const int64_t dp = W.page(dst), sp = W.page(src);
      if (dp >= 0 && sp >= 0) {
        to = static_cast<int>(dp) * kPage + dst % kPage;
        from = static_cast<int>(sp) * kPage + src % kPage;
        const int64_t a = W.beside(dp, dst), b = W.beside(sp, src);
        P.weights_out[a] = P.weights[b];
        if (P.order_out) P.order_out[a] = P.order ? P.order[b] : src;
        if (P.source_out) P.source_out[a] = src;
      }
    }
  };
  int j0 = (part * kMoveWarps + warp) * kBatch;
  if (j0 < moves) look(j0);
  for (; j0 < moves; j0 += stride) {
    uint4 data[kBatch];
    int t[kBatch];
#pragma unroll
    for (int x = 0; x < kBatch; ++x) {
      t[x] = __shfl_sync(0xffffffffu, to, x);
      const int f = __shfl_sync(0xffffffffu, from, x);
      if (t[x] >= 0) data[x] = *reinterpret_cast<const uint4*>(pool + (f / kPage) * P.page_stride + (f % kPage) * kDim);
    }
    look(j0 + stride);
#pragma unroll
    for (int x = 0; x < kBatch; ++x)
      if (t[x] >= 0) *reinterpret_cast<uint4*>(pool + (t[x] / kPage) * P.page_stride + (t[x] % kPage) * kDim) = data[x];
  }
}

static int32_t check(const ss_attn_desc_t* d, const ss_evict_t* e) {
  if (!d || d->struct_size != sizeof(ss_attn_desc_t) || !e || e->struct_size != sizeof(ss_evict_t) || e->flags) return SS_ERR_INVALID_ARG;
  if (d->num_kv_heads < 1 || d->num_nodes < 0 || d->total_node_pages < 0 || d->num_pages < 0) return SS_ERR_INVALID_ARG;
  if (e->n_nodes < 0 || e->max_keys < 0 || e->sinks < 0 || e->recent < 0) return SS_ERR_INVALID_ARG;
  if (d->head_dim != kDim || d->page_size != kPage || d->kv_token_stride != kDim || d->kv_page_stride % 128 || d->kv_head_stride % 128 ||
      d->kv_page_stride <= 0 || d->kv_head_stride <= 0)
    return SS_ERR_UNSUPPORTED;
  if (d->num_kv_heads > 65536 || d->total_node_pages > kMostPages || d->num_pages > 0x7ffffff || static_cast<int64_t>(e->n_nodes) * d->num_kv_heads > 0x7fffffffLL / kMostCluster)
    return SS_ERR_UNSUPPORTED;
  return SS_OK;
}

static size_t carve(const ss_attn_desc_t* d, const ss_evict_t* e, void* base, Params* P) {
  Carver c(base);
  P->hdr = c.take<Header>(1);
  P->info = c.take<Node>(static_cast<size_t>(e->n_nodes) + 1);
  P->claim = c.take<int32_t>(static_cast<size_t>(d->num_nodes) + 1);
  P->moves = c.take<int32_t>(static_cast<size_t>(e->n_nodes) * d->num_kv_heads + 1);
  P->lists = c.take<int32_t>(static_cast<size_t>(d->total_node_pages) * d->num_kv_heads * kPage + 1);
  return c.off;
}

// Blocks of a cluster: as many as it takes for two blocks an SM, as long as each has a thousand slots.
static int cluster_of(const ss_attn_desc_t* d, const ss_evict_t* e) {
  const int64_t pairs = static_cast<int64_t>(e->n_nodes) * d->num_kv_heads, all = d->total_node_pages * kPage;
  const int64_t keys = e->max_keys > 0 && e->max_keys < all ? e->max_keys : all;
  int c = 1;
  while (c < kMostCluster && pairs * c < 2 * sm_count_of_current_device() && keys >= 2048 * c) c *= 2;
  return c;
}

static int32_t launch_evict(Params P, const ss_attn_desc_t* d, const ss_evict_t* e, cudaStream_t st) {
  static bool done[kDeviceSlots] = {false};
  const int slot = current_device_slot();
  if (slot < 0 || !done[slot]) {
    if (cudaFuncSetAttribute(evict_select_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kStaged * 4) != cudaSuccess) {
      (void)cudaGetLastError();
      return SS_ERR_CUDA;
    }
    if (slot >= 0) done[slot] = true;
  }
  const int c = cluster_of(d, e);
  const int64_t pairs = static_cast<int64_t>(e->n_nodes) * d->num_kv_heads, all = d->total_node_pages * kPage;
  const int64_t keys = e->max_keys > 0 && e->max_keys < all ? e->max_keys : all, each = ceil_div64(ceil_div64(keys, c), 32) * 32;
  P.staged = static_cast<int>(each < kStaged ? each : kStaged);
  // eight blocks of moves an SM, as long as each has a batch for its warps; half of the keys move at most
  const int64_t wanted = ceil_div64(8LL * sm_count_of_current_device(), pairs), most = ceil_div64(keys, 2 * kBatch * kMoveWarps);
  P.move_blocks = static_cast<int>(wanted < most ? wanted : most < 1 ? 1 : most);
  if (pairs * P.move_blocks > 0x7fffffffLL) return SS_ERR_UNSUPPORTED;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(static_cast<unsigned>(pairs * c));
  cfg.blockDim = dim3(kThreads);
  cfg.dynamicSmemBytes = static_cast<size_t>(P.staged) * 4;
  cfg.stream = st;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = static_cast<unsigned>(c);
  attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
  attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[1].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = ss::pdl_enabled() ? 2 : 1;
  const cudaError_t err = cudaLaunchKernelEx(&cfg, evict_select_kernel, P);
  ss::g_launch_count.fetch_add(1, std::memory_order_relaxed);
  if (err != cudaSuccess || cudaPeekAtLastError() != cudaSuccess) {
    (void)cudaGetLastError();
    return SS_ERR_CUDA;
  }
  SS_LAUNCH(evict_move_kernel, static_cast<unsigned>(pairs * P.move_blocks), kMoveThreads, 0, st, P);
  return SS_OK;
}

}  // namespace evict
}  // namespace ss

extern "C" int32_t ss_kv_evict_workspace_bytes(const ss_attn_desc_t* desc, const ss_evict_t* ev, size_t* out_bytes) {
  using namespace ss::evict;
  if (!out_bytes) return SS_ERR_INVALID_ARG;
  const int32_t rc = check(desc, ev);
  if (rc != SS_OK) return rc;
  Params P;
  *out_bytes = carve(desc, ev, nullptr, &P);
  return SS_OK;
}

extern "C" int32_t ss_kv_evict(const ss_attn_desc_t* d, const ss_evict_t* e, void* workspace, size_t workspace_bytes, void* stream) {
  using namespace ss::evict;
  const int32_t rc = check(d, e);
  if (rc != SS_OK) return rc;
  if (!workspace || reinterpret_cast<uintptr_t>(workspace) % ss::kAlign) return SS_ERR_INVALID_ARG;
  Params P;
  memset(&P, 0, sizeof P);
  if (workspace_bytes < carve(d, e, workspace, &P)) return SS_ERR_WORKSPACE_TOO_SMALL;
  if (e->n_nodes > 0 && (!e->nodes || !e->keep || !e->weights || !d->k_pool || !d->v_pool || !d->node_kv_len || !d->node_page_offsets ||
                         !d->node_pages))
    return SS_ERR_INVALID_ARG;
  if (reinterpret_cast<uintptr_t>(d->k_pool) % 256 || reinterpret_cast<uintptr_t>(d->v_pool) % 256 || reinterpret_cast<uintptr_t>(e->weights) % 64 ||
      reinterpret_cast<uintptr_t>(e->weights_out) % 64 || reinterpret_cast<uintptr_t>(e->order) % 64 || reinterpret_cast<uintptr_t>(e->order_out) % 64 ||
      reinterpret_cast<uintptr_t>(e->source_out) % 64)
    return SS_ERR_UNSUPPORTED;
  P.Hkv = d->num_kv_heads;
  P.k_pool = static_cast<__nv_bfloat16*>(const_cast<void*>(d->k_pool));
  P.v_pool = static_cast<__nv_bfloat16*>(const_cast<void*>(d->v_pool));
  P.num_pages = d->num_pages;
  P.page_stride = d->kv_page_stride;
  P.head_stride = d->kv_head_stride;
  P.total_node_pages = d->total_node_pages;
  P.num_nodes = d->num_nodes;
  P.node_kv_len = d->node_kv_len;
  P.node_pages = d->node_pages;
  P.node_page_offsets = d->node_page_offsets;
  P.n = e->n_nodes;
  P.sinks = e->sinks;
  P.recent = e->recent;
  P.nodes = e->nodes;
  P.keep = e->keep;
  P.weights = e->weights;
  P.weights_out = e->weights_out ? e->weights_out : e->weights;
  P.order = e->order;
  P.order_out = e->order_out ? e->order_out : e->order;
  P.source_out = e->source_out;
  P.kv_len_out = e->kv_len_out;
  cudaStream_t st = ss::as_stream(stream);
  SS_LAUNCH(evict_nodes_kernel, 1, kNodesThreads, 0, st, P);
  if (e->n_nodes == 0) return SS_OK;
  return launch_evict(P, d, e, st);
}
