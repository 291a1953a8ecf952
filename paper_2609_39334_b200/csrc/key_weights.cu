// ss_key_weights: host side, the planner and the plain kernel.
//
//   plan (one cluster: which paths are below a node, the table of query rows, the nodes with something to do and their steps)
//     -> tensor-core kernel (key_weights_umma.cu), or the plain kernel: a warp per key, in fp32
// The planner is bound by latency, five barriers of its cluster and some ten trips to memory: 14 us alone for 8 paths, 19 for 1024.
#include <math.h>
#include <string.h>

#include "key_weights.cuh"

namespace ss {
namespace keyw {

int32_t launch_tiles(const Params& P, cudaStream_t st, int blocks);

constexpr int kPlanThreads = 1024, kPlanWarps = kPlanThreads / 32, kPlanBlocks = 8;
constexpr int kPlainThreads = 256;
// (Loops over keys look two tiles ahead, those over nodes and paths step by the planner's threads, in 32 bits.)
constexpr int64_t kMostPages = (0x80000000LL - 2 * kTile) / kPage;
constexpr int kMostListed = 1 << 30;

__device__ __forceinline__ uint32_t cluster_rank() { uint32_t r; asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r)); return r; }
__device__ __forceinline__ uint32_t cluster_size() { uint32_t r; asm volatile("mov.u32 %0, %%cluster_nctarank;" : "=r"(r)); return r; }
__device__ __forceinline__ void cluster_sync() {
  asm volatile("barrier.cluster.arrive.release;" ::: "memory");
  asm volatile("barrier.cluster.wait.acquire;" ::: "memory");
}
__device__ __forceinline__ long long load_remote(const long long* p, uint32_t rank) {
  uint32_t at;
  long long v;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(at) : "r"(static_cast<uint32_t>(__cvta_generic_to_shared(p))), "r"(rank));
  asm volatile("ld.shared::cluster.s64 %0, [%1];" : "=l"(v) : "r"(at) : "memory");
  return v;
}
// Sums over the cluster's threads in front of this one (and of all in *total_a, *total_b).  A barrier over the cluster.
struct Scan { long long warp_a[kPlanWarps], warp_b[kPlanWarps], block_a, block_b; };
__device__ __forceinline__ long long scanned(long long v, int lane) {
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const long long up = __shfl_up_sync(0xffffffffu, v, o);
    if (lane >= o) v += up;
  }
  return v;
}
__device__ __forceinline__ void cluster_before(long long& a, long long& b, Scan& S, long long* total_a, long long* total_b) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const long long ia = scanned(a, lane), ib = scanned(b, lane);
  if (lane == 31) { S.warp_a[warp] = ia; S.warp_b[warp] = ib; }
  __syncthreads();
  if (warp == 0) {
    const long long wa = S.warp_a[lane], wb = S.warp_b[lane], ja = scanned(wa, lane), jb = scanned(wb, lane);
    S.warp_a[lane] = ja - wa;
    S.warp_b[lane] = jb - wb;
    if (lane == 31) { S.block_a = ja; S.block_b = jb; }
  }
  cluster_sync();
  const uint32_t r = cluster_rank(), C = cluster_size();
  a = S.warp_a[warp] + ia - a;
  b = S.warp_b[warp] + ib - b;
  *total_a = *total_b = 0;
  for (uint32_t c = 0; c < C; ++c) {
    const long long sa = load_remote(&S.block_a, c), sb = load_remote(&S.block_b, c);
    if (c < r) { a += sa; b += sb; }
    *total_a += sa;
    *total_b += sb;
  }
}

__global__ void __launch_bounds__(kPlanThreads, 1) key_plan_kernel(const __grid_constant__ Params P, int grid_blocks) {
  ss::grid_dependency_enter_then_release();
  __shared__ Scan scan[2];
  const uint32_t C = cluster_size();
  const int tid = static_cast<int>(cluster_rank()) * kPlanThreads + threadIdx.x, threads = static_cast<int>(C) * kPlanThreads;
  const int lane = threadIdx.x & 31;
  for (int i = tid; i < P.num_nodes; i += threads) {
    P.first[i] = P.leaf_path[i] = INT32_MAX;
    P.last[i] = -1;
    P.below[i] = P.fresh[i] = 0;
  }
  for (int i = tid; i < 2 * grid_blocks; i += threads) P.arrived[i] = 0;
  if (tid == 0) P.hdr->status = SS_OK;
  cluster_sync();

  // ---- paths, a stretch a thread: their tokens that count, and a mark on every node of their chains
  const int live = P.num_paths_dev ? min(max(*P.num_paths_dev, 0), P.num_paths) : P.num_paths;
  const int each = (live + threads - 1) / threads;
  const int p0 = min(static_cast<int64_t>(tid) * each, static_cast<int64_t>(live)), p1 = min(p0 + each, live);
  auto used_of = [&](int T) { return P.last_tokens > 0 ? min(T, P.last_tokens) : T; };
  long long used = 0;
  for (int p = p0; p < p1; ++p) {
    const int leaf = P.path_leaf_node[p];
    int T = P.path_q_len[p], bad = SS_OK;
    const int64_t dst = P.q_offsets[p], src = P.q_src_offsets ? P.q_src_offsets[p] : dst;
    if (leaf < 0 || leaf >= P.num_nodes || T < 0 || src < 0 || src + T > P.q_rows || dst < 0 || dst + T > P.total_q) bad = SS_ERR_BAD_INPUT;
    else if (T > P.node_kv_len[leaf]) bad = SS_ERR_UNSUPPORTED;
    if (bad != SS_OK) T = 0;
    int64_t tokens = 0;
    int depth = 0, a = leaf;
    for (; a >= 0 && a < P.num_nodes && depth < SS_MAX_DEPTH; ++depth) {
      atomicMin(P.first + a, p);
      atomicMax(P.last + a, p);
      atomicAdd(P.below + a, 1);
      tokens += P.node_kv_len[a];
      a = P.node_parent[a];
    }
    if (bad == SS_OK && a >= 0) bad = a < P.num_nodes ? SS_ERR_UNSUPPORTED : SS_ERR_BAD_INPUT;      // deeper than SS_MAX_DEPTH
    if (bad != SS_OK) { set_status(&P.hdr->status, bad); T = 0; }
    if (T > 0) {
      atomicMax(P.fresh + leaf, T);
      atomicMin(P.leaf_path + leaf, p);
    }
    P.path_start[p] = P.path_order ? P.path_order[p] : static_cast<int>(tokens) - T;
    P.path_row[p] = used_of(T);                                // (its place follows)
    used += used_of(T);
  }
  long long all, unused, none = 0, at = used;
  cluster_before(at, none, scan[0], &all, &unused);
  for (int p = p0; p < p1; ++p) {
    const int u = P.path_row[p];
    // (rows of different paths that overlap would not fit the table)
    if (at + u > P.total_q) set_status(&P.hdr->status, SS_ERR_BAD_INPUT);
    P.path_row[p] = static_cast<int>(min(at, static_cast<long long>(P.total_q)));
    at += u;
  }
  const int all_rows = static_cast<int>(min(all, static_cast<long long>(P.total_q)));
  if (tid == 0) P.path_row[live] = all_rows;
  cluster_sync();

  // ---- the table of rows, a warp per path
  for (int p = tid / 32; p < live; p += threads / 32) {
    const int r0 = P.path_row[p], u = P.path_row[p + 1] - r0;
    const int64_t dst = P.q_offsets[p], src = P.q_src_offsets ? P.q_src_offsets[p] : dst;
    const int skip = P.path_q_len[p] - u;
    for (int x = lane; x < u; x += 32) P.rows[r0 + x] = make_int2(static_cast<int>(src + skip + x), static_cast<int>(dst + skip + x));
  }

  // ---- nodes, a stretch a thread
  const int each_node = (P.num_nodes + threads - 1) / threads;
  const int n0 = min(static_cast<int64_t>(tid) * each_node, static_cast<int64_t>(P.num_nodes)), n1 = min(n0 + each_node, P.num_nodes);
  // Steps of a node's units; R.len = 0: nothing to do.
  auto rec_of = [&](int n, Rec& R, bool tell) -> long long {
    R.len = 0;
    const int first = P.first[n], last = P.last[n];
    if (last < 0) return 0;
    const int len = P.node_kv_len[n], fresh = P.fresh[n];
    const int64_t e0 = P.node_page_offsets[n], e1 = P.node_page_offsets[n + 1];
    int bad = SS_OK;
    if (len < 0 || (len > 0 && P.num_pages < 1) || e0 < 0 || e1 > P.total_node_pages || (static_cast<int64_t>(len) + kPage - 1) / kPage > e1 - e0 || P.below[n] != last - first + 1)
      bad = SS_ERR_BAD_INPUT;
    else if (fresh > 1 && first != last) bad = SS_ERR_UNSUPPORTED;
    if (bad != SS_OK) {
      if (tell) set_status(&P.hdr->status, bad);
      return 0;
    }
    if (len == 0) return 0;
    R.page0 = e0;
    R.len = len;
    R.row0 = P.path_row[first];
    R.rows = P.path_row[last + 1] - R.row0;
    R.steps = max(1, (R.rows + kCols / P.G - 1) / (kCols / P.G));
    R.known = len - fresh;
    R.hides = fresh > 0 && first == last ? R.rows : 0;
    R.order0 = fresh > 0 ? P.path_start[P.leaf_path[n]] : 0;
    const int per_step = kCols / P.G, last_rows = (R.rows - (R.steps - 1) * per_step) * P.G;
    R.cost = kTileCost + (R.steps - 1) * ((per_step * P.G + 15) / 16) + max(1, (last_rows + 15) / 16);
    return static_cast<long long>((len + kTile - 1) / kTile) * P.Hkv * R.cost;
  };
  Rec R;
  long long cost = 0, count = 0;
  for (int n = n0; n < n1; ++n) {
    cost += rec_of(n, R, true);
    count += R.len > 0;
  }
  long long total, n_recs, off = cost, rec = count;
  cluster_before(off, rec, scan[1], &total, &n_recs);
  for (int n = n0; n < n1; ++n) {
    // (the one node that a thread of a small tree has is still there)
    const long long c = n1 - n0 == 1 ? cost : rec_of(n, R, false);
    if (R.len == 0) continue;
    R.off = off;
    P.recs[rec++] = R;
    off += c;
  }
  if (tid == 0) {
    P.hdr->n_recs = static_cast<int>(n_recs);
    P.hdr->total = total;
  }
  cluster_sync();                              // (no block leaves while another may read its sums)
}

__global__ void __launch_bounds__(kPlainThreads) key_plain_kernel(const __grid_constant__ Params P) {
  ss::grid_dependency_enter();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  auto load4 = [](const __nv_bfloat16* p, float (&v)[4]) {
    const uint2 u = *reinterpret_cast<const uint2*>(p);
    v[0] = __uint_as_float(u.x << 16); v[1] = __uint_as_float(u.x & 0xffff0000u);
    v[2] = __uint_as_float(u.y << 16); v[3] = __uint_as_float(u.y & 0xffff0000u);
  };
  for (int x = 0; x < P.hdr->n_recs; ++x) {
    const Rec R = P.recs[x];
    const int64_t units = static_cast<int64_t>((R.len + kTile - 1) / kTile) * P.Hkv;
    // (a stretch of the line of all units: every block looks at every node)
    for (int64_t u = blockIdx.x; u < units; u += gridDim.x) {
      const int tile = static_cast<int>(u / P.Hkv), g = static_cast<int>(u % P.Hkv);
      for (int i = tile * kTile + warp; i < min(R.len, (tile + 1) * kTile); i += kPlainThreads / 32) {
        const int64_t page = page_of(P, R, i);
        if (page < 0) continue;
        float k[4];
        double sum = 0.;                       // (of as many tokens as there are, one by one)
        load4(P.k_pool + page * P.page_stride + static_cast<int64_t>(g) * P.head_stride + (i % kPage) * kDim + 4 * lane, k);
        for (int t = max(0, i - R.len + R.hides); t < R.rows; ++t) {
          const int2 row = P.rows[R.row0 + t];
          float part = 0.f;
          for (int h = 0; h < P.G; ++h) {
            float q[4];
            load4(P.q + (static_cast<int64_t>(row.x) * P.Hq + g * P.G + h) * kDim + 4 * lane, q);
            const float s = warp_sum(q[0] * k[0] + q[1] * k[1] + q[2] * k[2] + q[3] * k[3]) * P.scale;
            const float lse = P.lse[static_cast<int64_t>(row.y) * P.Hq + g * P.G + h];
            part += lse == -INFINITY ? 0.f : expf(s - lse);
          }
          sum += part;
        }
        if (lane == 0) store_key(P, R, page, g, i, static_cast<float>(sum), load_before(P, R, page, g, i));
      }
    }
  }
}

static int32_t check_desc(const ss_attn_desc_t* d, const ss_key_weights_t* kw) {
  if (!d || d->struct_size != sizeof(ss_attn_desc_t) || !kw || kw->struct_size != sizeof(ss_key_weights_t) || kw->flags) return SS_ERR_INVALID_ARG;
  if (d->flags & ~(SS_FLAG_VALIDATE | SS_FLAG_FORCE_GENERIC | SS_FLAG_NO_TCGEN05 | SS_FLAG_TILES_2CTA)) return SS_ERR_INVALID_ARG;
  if (d->num_q_heads < 1 || d->num_kv_heads < 1 || d->num_nodes < 0 || d->num_paths < 0 || d->total_q < 0 || d->total_node_pages < 0 ||
      d->num_pages < 0 || d->max_sms < 0 || (d->q_src_offsets && d->q_src_rows < 0))
    return SS_ERR_INVALID_ARG;
  if (!(kw->decay >= 0.f) || isinf(kw->decay) || kw->last_tokens < 0) return SS_ERR_INVALID_ARG;
  if (d->head_dim != kDim || d->page_size != kPage || d->num_q_heads % d->num_kv_heads || d->num_q_heads / d->num_kv_heads > kCols)
    return SS_ERR_UNSUPPORTED;
  if (d->kv_token_stride != kDim || d->kv_page_stride % 128 || d->kv_head_stride % 128 || d->kv_page_stride <= 0 || d->kv_head_stride <= 0)
    return SS_ERR_UNSUPPORTED;
  if (!(d->sm_scale >= 0.f) || isinf(d->sm_scale)) return SS_ERR_INVALID_ARG;
  const int64_t most = 0x7fffffffLL / d->num_q_heads;
  if (d->total_q > most || (d->q_src_offsets && d->q_src_rows > most) || d->total_node_pages > kMostPages) return SS_ERR_UNSUPPORTED;
  if (d->num_nodes > kMostListed || d->num_paths > kMostListed) return SS_ERR_UNSUPPORTED;
  return SS_OK;
}

static size_t carve(const ss_attn_desc_t* d, void* base, Params* P) {
  Carver c(base);
  const size_t blocks = static_cast<size_t>(sm_count_of_current_device()), nodes = static_cast<size_t>(d->num_nodes) + 1,
               paths = static_cast<size_t>(d->num_paths) + 1;
  P->hdr = c.take<Header>(1);
  P->recs = c.take<Rec>(nodes);
  P->rows = c.take<int2>(static_cast<size_t>(d->total_q) + 1);
  P->first = c.take<int>(nodes);
  P->last = c.take<int>(nodes);
  P->below = c.take<int>(nodes);
  P->fresh = c.take<int>(nodes);
  P->leaf_path = c.take<int>(nodes);
  P->path_row = c.take<int>(paths);
  P->path_start = c.take<int>(paths);
  P->part = c.take<float>(blocks * 2 * 2 * kTile);
  P->arrived = c.take<int>(blocks * 2);
  return c.off;
}

static int32_t launch_plan(const Params& P, cudaStream_t st, int blocks) {
  // (small trees: one block, whose barriers are the cheapest)
  const int64_t size = static_cast<int64_t>(P.num_nodes) + P.num_paths + P.total_q / 32;
  const int c = size <= 2 * kPlanThreads ? 1 : blocks < kPlanBlocks ? blocks : kPlanBlocks;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(c);
  cfg.blockDim = dim3(kPlanThreads);
  cfg.stream = st;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = static_cast<unsigned>(c);
  attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
  attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[1].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = ss::pdl_enabled() ? 2 : 1;
  const cudaError_t err = cudaLaunchKernelEx(&cfg, key_plan_kernel, P, blocks);
  ss::g_launch_count.fetch_add(1, std::memory_order_relaxed);
  if (err != cudaSuccess || cudaPeekAtLastError() != cudaSuccess) {
    (void)cudaGetLastError();
    return SS_ERR_CUDA;
  }
  return SS_OK;
}

}  // namespace keyw
}  // namespace ss

extern "C" int32_t ss_key_weights_workspace_bytes(const ss_attn_desc_t* desc, const ss_key_weights_t* kw, size_t* out_bytes) {
  using namespace ss::keyw;
  if (!out_bytes) return SS_ERR_INVALID_ARG;
  const int32_t rc = check_desc(desc, kw);
  if (rc != SS_OK) return rc;
  Params P;
  *out_bytes = carve(desc, nullptr, &P);
  return SS_OK;
}

extern "C" int32_t ss_key_weights(const ss_attn_desc_t* d, const ss_key_weights_t* kw, void* workspace, size_t workspace_bytes, void* stream) {
  using namespace ss::keyw;
  const int32_t rc = check_desc(d, kw);
  if (rc != SS_OK) return rc;
  if (!workspace || reinterpret_cast<uintptr_t>(workspace) % ss::kAlign) return SS_ERR_INVALID_ARG;
  if (!d->k_pool || !d->node_parent || !d->node_kv_len || !d->node_page_offsets || !d->node_pages || !d->path_leaf_node || !d->path_q_len ||
      !d->q_offsets || !kw->weights_out)
    return SS_ERR_INVALID_ARG;
  if (d->total_q > 0 && (!d->q || !d->lse)) return SS_ERR_INVALID_ARG;
  if (reinterpret_cast<uintptr_t>(d->k_pool) % 256 || reinterpret_cast<uintptr_t>(d->q) % 16 || reinterpret_cast<uintptr_t>(kw->weights_in) % 64 ||
      reinterpret_cast<uintptr_t>(kw->weights_out) % 64 || reinterpret_cast<uintptr_t>(kw->order) % 64)
    return SS_ERR_UNSUPPORTED;
  Params P;
  memset(&P, 0, sizeof P);
  if (workspace_bytes < carve(d, workspace, &P)) return SS_ERR_WORKSPACE_TOO_SMALL;
  P.Hq = d->num_q_heads;
  P.Hkv = d->num_kv_heads;
  P.G = P.Hq / P.Hkv;
  P.scale = d->sm_scale > 0.f ? d->sm_scale : 1.0f / sqrtf(static_cast<float>(kDim));
  P.scale_log2 = P.scale * 1.4426950408889634f;
  P.decay = kw->decay;
  P.last_tokens = kw->last_tokens;
  P.k_pool = static_cast<const __nv_bfloat16*>(d->k_pool);
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
  P.path_order = kw->path_order;
  P.q_offsets = d->q_offsets;
  P.q_src_offsets = d->q_src_offsets;
  P.total_q = d->total_q;
  P.q_rows = d->q_src_offsets ? d->q_src_rows : d->total_q;
  P.q = static_cast<const __nv_bfloat16*>(d->q);
  P.lse = d->lse;
  P.weights_in = kw->decay > 0.f ? kw->weights_in : nullptr;
  P.weights_out = kw->weights_out;
  P.order = kw->order;
  cudaStream_t st = ss::as_stream(stream);
  int sms = ss::sm_count_of_current_device();
  if (d->max_sms > 0 && d->max_sms < sms) sms = d->max_sms;
  const int32_t planned = launch_plan(P, st, sms);
  if (planned != SS_OK || d->num_paths == 0 || d->num_nodes == 0) return planned;
  if (d->flags & (SS_FLAG_FORCE_GENERIC | SS_FLAG_NO_TCGEN05)) {
    // (blocks go to all SMs before any gets a second one)
    SS_LAUNCH(key_plain_kernel, sms < ss::sm_count_of_current_device() ? sms : 8 * sms, kPlainThreads, 0, st, P);
    return SS_OK;
  }
  return launch_tiles(P, st, sms);
}
