// ss_qk_norm_rope and ss_kv_append: head rows of 128 values on their way from a projection into the attention - normalised
// (keys and queries of models that do), rotated to their positions, rounded once, and written to where the attention reads
// them: the caller's tensors or, keys and values of a step, the slots of the paged pool.
//
//   y = x * w / sqrt(mean(x^2) + eps)                        (w absent: y = x)
//   (y_a, y_b) -> (y_a cos f - y_b sin f, y_b cos f + y_a sin f)   f = position * inv_freq[i], pairs (i, i + R/2) or (2i, 2i + 1)
//
// Eight lanes share a head row: each has two chunks of 8 values (16 bytes) that hold both members of its 8 pairs, so that a
// rotation needs no exchange, and a row's sum of squares takes three shuffles.  A warp has four rows at a time and goes through
// the heads of ONE token (or, with few tokens, through a part of them), so the eight angles of a lane are made once a token: the
// product in fp64 (a position of a million times a frequency of one has no bits behind the point left in fp32), the whole turns
// off, the rest through sincospif.  Sums, norm and rotation are fp32.
// Bound: HBM, every row read and written once.  The loads of kAhead head rows are issued before the first is used; the weights are
// in shared memory, which leaves room for kBlocks blocks an SM.
#include "common.cuh"

namespace ss {
namespace rows {

constexpr int kDim = 128, kPage = 16;
constexpr int kWarps = 8;                    // of a block
constexpr int kBlocks = 3;                   // per SM
constexpr int kAhead = 2;                    // head rows of a lane group in flight

struct Tensor { const __nv_bfloat16* p; int64_t row, head; };
struct TensorOut { __nv_bfloat16* p; int64_t row, head; };
struct Args {
  Tensor q, k, v;
  TensorOut q_out, k_out;
  const float* inv_freq;
  const __nv_bfloat16 *q_weight, *k_weight;
  const int32_t* positions;
  int64_t n_rows;
  float eps;
  int rot, hq, hk, hv;                       // heads to go through (0: tensor absent)
  int split;                                 // warps that share a token's heads
};
struct Place {                               // where the rows of a step go
  const int32_t *node_parent, *node_kv_len, *node_pages, *path_leaf_node, *path_q_len, *num_paths_dev;
  const int64_t *node_page_offsets, *q_offsets, *q_src_offsets;
  __nv_bfloat16 *k_pool, *v_pool;
  int64_t num_pages, page_stride, head_stride, total_node_pages, total_q;
  int num_nodes, num_paths;
  int run;                                   // tokens in a row that a warp takes
};

struct Lane {
  int c0, c1;                                // this lane's chunks of 8 values
  bool turn0, turn1;                         // which of them are rotated
  float cs[8], sn[8];                        // INTER: four pairs of chunk c0, then of c1; else pair j = value j of both
};

__device__ __forceinline__ void unpack8(const uint4& u, float (&f)[8]) {
  const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    f[2 * i] = __uint_as_float(w[i] << 16);
    f[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
  }
}
__device__ __forceinline__ uint4 pack8(const float (&f)[8]) {
  uint32_t w[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const __nv_bfloat162 b = __floats2bfloat162_rn(f[2 * i], f[2 * i + 1]);
    w[i] = *reinterpret_cast<const uint32_t*>(&b);
  }
  return make_uint4(w[0], w[1], w[2], w[3]);
}

template <bool INTER>
__device__ __forceinline__ void lane_setup(Lane& L, const Args& A, int sub) {
  if (INTER) {
    L.c0 = sub; L.c1 = sub + 8;
    L.turn0 = L.c0 < A.rot / 8; L.turn1 = L.c1 < A.rot / 8;
  } else {
    const int half = A.rot / 16;             // chunks from one member of a pair to the other
    L.turn0 = L.turn1 = sub < half;
    L.c0 = sub < half ? sub : 2 * sub;       // (behind the 2 * half rotated chunks the others follow two by two)
    L.c1 = sub < half ? sub + half : 2 * sub + 1;
  }
}
// The weights of queries and keys, [2][16] chunks (whole block).
__device__ __forceinline__ void load_weights(uint4 (&w)[32], const Args& A) {
  const int t = threadIdx.x;
  if (t < 32) {
    const __nv_bfloat16* p = t < 16 ? A.q_weight : A.k_weight;
    if (p) w[t] = __ldg(reinterpret_cast<const uint4*>(p) + (t & 15));
  }
  __syncthreads();
}

template <bool INTER>
__device__ __forceinline__ void lane_angles(Lane& L, const Args& A, double position) {
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    const int chunk = INTER ? (j < 4 ? L.c0 : L.c1) : L.c0;
    const int i = INTER ? chunk * 4 + (j & 3) : chunk * 8 + j;
    const bool turn = INTER ? (j < 4 ? L.turn0 : L.turn1) : L.turn0;
    if (turn) {
      double turns = position * static_cast<double>(__ldg(A.inv_freq + i)) * 0.15915494309189533577;   // / (2 pi)
      turns -= rint(turns);
      sincospif(static_cast<float>(2.0 * turns), &L.sn[j], &L.cs[j]);
    } else {
      L.cs[j] = 1.f;
      L.sn[j] = 0.f;
    }
  }
}

// One head row (its two chunks in a, b): norm (with the weights at w, if any) and rotation.
template <bool INTER>
__device__ __forceinline__ void turn_row(const Lane& L, const uint4* w, float eps, uint4& a, uint4& b) {
  float x0[8], x1[8];
  unpack8(a, x0);
  unpack8(b, x1);
  float sum = 0.f;
#pragma unroll
  for (int j = 0; j < 8; ++j) sum = fmaf(x0[j], x0[j], fmaf(x1[j], x1[j], sum));
#pragma unroll
  for (int o = 4; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
  if (w) {
    const float r = rsqrtf(sum * (1.f / kDim) + eps);
    float f[8];
    unpack8(w[L.c0], f);
#pragma unroll
    for (int j = 0; j < 8; ++j) x0[j] = x0[j] * r * f[j];
    unpack8(w[L.c1], f);
#pragma unroll
    for (int j = 0; j < 8; ++j) x1[j] = x1[j] * r * f[j];
  }
  // (values that are not rotated stay as they are: a product with a sine of 0 would carry an infinity over)
  if (INTER) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float a0 = x0[2 * i], b0 = x0[2 * i + 1], a1 = x1[2 * i], b1 = x1[2 * i + 1];
      if (L.turn0) { x0[2 * i] = a0 * L.cs[i] - b0 * L.sn[i]; x0[2 * i + 1] = b0 * L.cs[i] + a0 * L.sn[i]; }
      if (L.turn1) { x1[2 * i] = a1 * L.cs[4 + i] - b1 * L.sn[4 + i]; x1[2 * i + 1] = b1 * L.cs[4 + i] + a1 * L.sn[4 + i]; }
    }
  } else if (L.turn0) {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const float p = x0[j], q = x1[j];
      x0[j] = p * L.cs[j] - q * L.sn[j];
      x1[j] = q * L.cs[j] + p * L.sn[j];
    }
  }
  a = pack8(x0);
  b = pack8(x1);
}

// The heads part, part + split, ... (in units of four: one per lane group) of row `row`: queries, then keys, then values.
// `kd` / `vd`: where the row's keys and values go (head h at + h * d_head); null: nowhere.
template <bool INTER>
__device__ __forceinline__ void token_heads(const Lane& L, const Args& A, const uint4* weights, int64_t row, int part, int lane,
                                            __nv_bfloat16* kd, __nv_bfloat16* vd, int64_t d_head) {
  const int n_heads = A.hq + A.hk + A.hv;
  const int step = 4 * A.split;
#pragma unroll 1
  for (int h0 = 4 * part; h0 < n_heads; h0 += step * kAhead) {                    // (warp-uniform)
    uint4 a[kAhead], b[kAhead];
    __nv_bfloat16* dst[kAhead];
#pragma unroll
    for (int x = 0; x < kAhead; ++x) {
      const int h = h0 + x * step + (lane >> 3);
      const __nv_bfloat16* src = nullptr;
      dst[x] = nullptr;
      if (h < A.hq) {
        src = A.q.p + row * A.q.row + h * A.q.head;
        dst[x] = A.q_out.p + row * A.q_out.row + h * A.q_out.head;
      } else if (h < A.hq + A.hk) {
        src = A.k.p + row * A.k.row + (h - A.hq) * A.k.head;
        if (kd) dst[x] = kd + (h - A.hq) * d_head;
      } else if (h < n_heads) {
        src = A.v.p + row * A.v.row + (h - A.hq - A.hk) * A.v.head;
        if (vd) dst[x] = vd + (h - A.hq - A.hk) * d_head;
      }
      a[x] = b[x] = make_uint4(0, 0, 0, 0);
      if (dst[x]) {
        a[x] = *(reinterpret_cast<const uint4*>(src) + L.c0);                     // (not __ldg: q_out may be q)
        b[x] = *(reinterpret_cast<const uint4*>(src) + L.c1);
      }
    }
#pragma unroll
    for (int x = 0; x < kAhead; ++x) {
      const int h1 = h0 + x * step, h = h1 + (lane >> 3);
      if (h1 >= n_heads) break;                                                   // (warp-uniform, as the next)
      if (h1 < A.hq + A.hk) {
        const bool is_q = h < A.hq;
        const uint4* w = is_q ? (A.q_weight ? weights : nullptr) : (A.k_weight ? weights + 16 : nullptr);
        uint4 y0 = a[x], y1 = b[x];
        turn_row<INTER>(L, w, A.eps, y0, y1);
        if (h < A.hq + A.hk) { a[x] = y0; b[x] = y1; }
      }
      if (dst[x]) {
        *(reinterpret_cast<uint4*>(dst[x]) + L.c0) = a[x];
        *(reinterpret_cast<uint4*>(dst[x]) + L.c1) = b[x];
      }
    }
  }
}

template <bool INTER>
__global__ void __launch_bounds__(kWarps * 32, kBlocks) norm_rope_kernel(const __grid_constant__ Args A) {
  ss::grid_dependency_enter();
  __shared__ uint4 weights[32];
  load_weights(weights, A);
  const int lane = threadIdx.x & 31;
  const int64_t warps = static_cast<int64_t>(gridDim.x) * kWarps;
  Lane L;
  lane_setup<INTER>(L, A, lane & 7);
  for (int64_t w = static_cast<int64_t>(blockIdx.x) * kWarps + (threadIdx.x >> 5); w < A.n_rows * A.split; w += warps) {
    const int64_t row = w / A.split;
    lane_angles<INTER>(L, A, A.positions ? static_cast<double>(__ldg(A.positions + row)) : 0.0);
    token_heads<INTER>(L, A, weights, row, static_cast<int>(w - row * A.split), lane,
                       A.k_out.p ? A.k_out.p + row * A.k_out.row : nullptr, nullptr, A.k_out.head);
  }
}

// Number of offsets[0 .. n] that are <= r, less one: the path of row r (whole warp; 32 probes a round).
__device__ __forceinline__ int path_of(const int64_t* offsets, int n, int64_t r, int lane) {
  int lo = 0, hi = n;                                          // offsets[lo] <= r < offsets[hi]
  while (hi - lo > 1) {
    const int step = (hi - lo + 31) / 32, at = min(lo + (lane + 1) * step, hi);
    const unsigned over = __ballot_sync(0xffffffffu, at >= hi || __ldg(offsets + at) > r);
    const int first = __ffs(over) - 1;                         // (the last lane's probe is hi)
    hi = min(lo + (first + 1) * step, hi);
    lo = lo + first * step;
  }
  return lo;
}

// A warp takes `run` tokens in a row (of a part of their heads): it looks for the first one's path, the others follow it.
template <bool INTER>
__global__ void __launch_bounds__(kWarps * 32, kBlocks) append_kernel(const __grid_constant__ Args A, const __grid_constant__ Place P) {
  ss::grid_dependency_enter();
  __shared__ uint4 weights[32];
  load_weights(weights, A);
  const int lane = threadIdx.x & 31;
  const int live = P.num_paths_dev ? min(max(__ldg(P.num_paths_dev), 0), P.num_paths) : P.num_paths;
  if (live == 0) return;
  const int64_t w = static_cast<int64_t>(blockIdx.x) * kWarps + (threadIdx.x >> 5);
  const int64_t first_row = __ldg(P.q_offsets), rows = min(__ldg(P.q_offsets + live) - first_row, P.total_q);
  int64_t r = first_row + w / A.split * P.run;
  const int part = static_cast<int>(w % A.split);
  const int64_t r_end = min(r + P.run, first_row + rows);
  if (r >= r_end) return;
  Lane L;
  lane_setup<INTER>(L, A, lane & 7);
  int p = path_of(P.q_offsets, live, r, lane);
  while (r < r_end) {
    const int64_t q0 = __ldg(P.q_offsets + p), q1 = __ldg(P.q_offsets + p + 1);
    const int leaf = __ldg(P.path_leaf_node + p), T = __ldg(P.path_q_len + p);
    const int64_t src0 = P.q_src_offsets ? __ldg(P.q_src_offsets + p) : q0;
    ++p;
    if (r >= q1) {
      if (p == live) break;
      continue;
    }
    const int64_t stop = min(r_end, q1);
    if (leaf < 0 || leaf >= P.num_nodes) { r = stop; if (p == live) break; continue; }
    const int len = __ldg(P.node_kv_len + leaf);
    const int64_t page0 = __ldg(P.node_page_offsets + leaf), page1 = __ldg(P.node_page_offsets + leaf + 1);
    int64_t before = 0;                                        // tokens in front of the leaf
    if (!A.positions && A.rot) {
      int a = __ldg(P.node_parent + leaf);
      for (int d = 1; d < SS_MAX_DEPTH && a >= 0 && a < P.num_nodes; ++d) {
        before += __ldg(P.node_kv_len + a);
        a = __ldg(P.node_parent + a);
      }
    }
    for (; r < stop; ++r) {
      const int64_t t = r - q0, row = src0 + t;
      if (t >= T || row < 0 || row >= A.n_rows) continue;
      const int at = len - T + static_cast<int>(t);            // token of the leaf
      __nv_bfloat16 *kd = nullptr, *vd = nullptr;
      if (at >= 0) {
        const int64_t entry = page0 + at / kPage;
        if (entry >= 0 && entry < page1 && entry < P.total_node_pages) {
          const int64_t page = __ldg(P.node_pages + entry);
          if (page >= 0 && page < P.num_pages) {
            const int64_t off = page * P.page_stride + static_cast<int64_t>(at % kPage) * kDim;
            kd = P.k_pool + off;
            vd = P.v_pool + off;
          }
        }
      }
      lane_angles<INTER>(L, A, A.positions ? static_cast<double>(__ldg(A.positions + row)) : static_cast<double>(before + at));
      token_heads<INTER>(L, A, weights, row, part, lane, kd, vd, P.head_stride);
    }
    if (p == live) break;
  }
}

// Checks what both calls share and fills the kernel's arguments.
static int32_t rows_args(const ss_rows_t* r, Args* A) {
  if (!r || r->struct_size != sizeof(ss_rows_t)) return SS_ERR_INVALID_ARG;
  if (r->flags & ~SS_ROWS_INTERLEAVED) return SS_ERR_INVALID_ARG;
  if (r->num_q_heads < 0 || r->num_kv_heads < 0 || r->n_rows < 0 || r->rot_dim < 0 || !(r->eps >= 0.f)) return SS_ERR_INVALID_ARG;
  if (r->head_dim != kDim || r->rot_dim > kDim || r->rot_dim % 16) return SS_ERR_UNSUPPORTED;
  if (r->num_q_heads > 65536 || r->num_kv_heads > 65536) return SS_ERR_UNSUPPORTED;
  if (r->n_rows == 0) return SS_OK;                            // (an empty tensor has no address)
  if (r->rot_dim && !r->inv_freq) return SS_ERR_INVALID_ARG;
  if ((r->q != nullptr) != (r->q_out != nullptr) || (r->q && r->num_q_heads < 1) || (r->k && r->num_kv_heads < 1)) return SS_ERR_INVALID_ARG;
  const int64_t strides = r->q_row_stride | r->q_head_stride | r->k_row_stride | r->k_head_stride | r->v_row_stride | r->v_head_stride |
                          r->q_out_row_stride | r->q_out_head_stride | r->k_out_row_stride | r->k_out_head_stride;
  const uintptr_t addresses = reinterpret_cast<uintptr_t>(r->q) | reinterpret_cast<uintptr_t>(r->k) | reinterpret_cast<uintptr_t>(r->v) |
                              reinterpret_cast<uintptr_t>(r->q_out) | reinterpret_cast<uintptr_t>(r->k_out) |
                              reinterpret_cast<uintptr_t>(r->q_weight) | reinterpret_cast<uintptr_t>(r->k_weight);
  if (strides % 8 || addresses % 16) return SS_ERR_UNSUPPORTED;
  const auto bf16 = [](const void* p) { return static_cast<const __nv_bfloat16*>(p); };
  A->q = {bf16(r->q), r->q_row_stride, r->q_head_stride};
  A->k = {bf16(r->k), r->k_row_stride, r->k_head_stride};
  A->v = {bf16(r->v), r->v_row_stride, r->v_head_stride};
  A->q_out = {static_cast<__nv_bfloat16*>(r->q_out), r->q_out_row_stride, r->q_out_head_stride};
  A->k_out = {static_cast<__nv_bfloat16*>(r->k_out), r->k_out_row_stride, r->k_out_head_stride};
  A->inv_freq = r->inv_freq;
  A->q_weight = bf16(r->q_weight);
  A->k_weight = bf16(r->k_weight);
  A->positions = r->positions;
  A->n_rows = r->n_rows;
  A->eps = r->eps;
  A->rot = r->rot_dim;
  A->hq = r->q ? r->num_q_heads : 0;
  A->hk = r->k ? r->num_kv_heads : 0;
  A->hv = 0;
  return SS_OK;
}

// Warps that share a token: as many as it takes to occupy the machine, at most one for four heads.  A token on one warp makes its
// angles once.
static int heads_split(int64_t tokens, int heads) {
  const int64_t want = static_cast<int64_t>(sm_count_of_current_device()) * 16;
  const int most = ceil_div(heads, 4);
  const int64_t split = tokens > 0 ? ceil_div64(want, tokens) : 1;
  return static_cast<int>(split < 1 ? 1 : split > most ? most : split);
}
static unsigned grid_of(int64_t warps) {
  const int64_t blocks = ceil_div64(warps, kWarps), most = static_cast<int64_t>(sm_count_of_current_device()) * 64;
  return static_cast<unsigned>(blocks < 1 ? 1 : blocks > most ? most : blocks);
}

}  // namespace rows
}  // namespace ss

extern "C" int32_t ss_qk_norm_rope(const ss_rows_t* rows, void* stream) {
  using namespace ss::rows;
  Args A = {};
  const int32_t rc = rows_args(rows, &A);
  if (rc != SS_OK || rows->n_rows == 0) return rc;
  if ((!rows->q && !rows->k) || (rows->k != nullptr) != (rows->k_out != nullptr) || (rows->rot_dim && !rows->positions)) return SS_ERR_INVALID_ARG;
  A.split = heads_split(rows->n_rows, A.hq + A.hk);
  const unsigned grid = grid_of(rows->n_rows * A.split);
  if (rows->flags & SS_ROWS_INTERLEAVED) {
    SS_LAUNCH(norm_rope_kernel<true>, grid, kWarps * 32, 0, ss::as_stream(stream), A);
  } else {
    SS_LAUNCH(norm_rope_kernel<false>, grid, kWarps * 32, 0, ss::as_stream(stream), A);
  }
  return SS_OK;
}

extern "C" int32_t ss_kv_append(const ss_attn_desc_t* d, const ss_rows_t* rows, void* stream) {
  using namespace ss::rows;
  Args A = {};
  const int32_t rc = rows_args(rows, &A);
  if (rc != SS_OK) return rc;
  if (!d || d->struct_size != sizeof(ss_attn_desc_t)) return SS_ERR_INVALID_ARG;
  if (d->num_nodes < 0 || d->num_paths < 0 || d->total_q < 0 || d->total_node_pages < 0 || d->num_pages < 0) return SS_ERR_INVALID_ARG;
  if (d->head_dim != kDim || d->page_size != kPage || d->kv_token_stride != kDim || d->kv_page_stride % 128 || d->kv_head_stride % 128 ||
      d->kv_page_stride <= 0 || d->kv_head_stride <= 0)
    return SS_ERR_UNSUPPORTED;
  if (rows->n_rows == 0) return SS_OK;
  if (!rows->k || !rows->v || rows->k_out || rows->num_kv_heads != d->num_kv_heads || (rows->q && rows->num_q_heads != d->num_q_heads))
    return SS_ERR_INVALID_ARG;
  if (!d->k_pool || !d->v_pool || !d->node_parent || !d->node_kv_len || !d->node_page_offsets || !d->node_pages || !d->path_leaf_node ||
      !d->path_q_len || !d->q_offsets)
    return SS_ERR_INVALID_ARG;
  if (reinterpret_cast<uintptr_t>(d->k_pool) % 256 || reinterpret_cast<uintptr_t>(d->v_pool) % 256) return SS_ERR_UNSUPPORTED;
  if (d->num_paths == 0 || d->total_q == 0) return SS_OK;
  A.hv = rows->num_kv_heads;
  Place P = {};
  P.node_parent = d->node_parent;
  P.node_kv_len = d->node_kv_len;
  P.node_pages = d->node_pages;
  P.path_leaf_node = d->path_leaf_node;
  P.path_q_len = d->path_q_len;
  P.num_paths_dev = d->num_paths_dev;
  P.node_page_offsets = d->node_page_offsets;
  P.q_offsets = d->q_offsets;
  P.q_src_offsets = d->q_src_offsets;
  P.k_pool = static_cast<__nv_bfloat16*>(const_cast<void*>(d->k_pool));
  P.v_pool = static_cast<__nv_bfloat16*>(const_cast<void*>(d->v_pool));
  P.num_pages = d->num_pages;
  P.page_stride = d->kv_page_stride;
  P.head_stride = d->kv_head_stride;
  P.total_node_pages = d->total_node_pages;
  P.num_nodes = d->num_nodes;
  P.num_paths = d->num_paths;
  P.total_q = d->total_q;
  A.split = heads_split(d->total_q, A.hq + A.hk + A.hv);
  // Tokens of a step lie side by side in their pages: a warp takes up to four in a row once there are enough of them for all warps
  // four times over.
  const int64_t resident = static_cast<int64_t>(ss::sm_count_of_current_device()) * kBlocks * kWarps;
  const int64_t run = d->total_q * A.split / (resident * 4);
  P.run = static_cast<int>(run < 1 ? 1 : run > 4 ? 4 : run);
  const int64_t blocks = ss::ceil_div64(ss::ceil_div64(d->total_q, P.run) * A.split, kWarps);
  if (blocks > 0x7fffffffLL) return SS_ERR_UNSUPPORTED;
  const unsigned grid = static_cast<unsigned>(blocks);
  if (rows->flags & SS_ROWS_INTERLEAVED) {
    SS_LAUNCH(append_kernel<true>, grid, kWarps * 32, 0, ss::as_stream(stream), A, P);
  } else {
    SS_LAUNCH(append_kernel<false>, grid, kWarps * 32, 0, ss::as_stream(stream), A, P);
  }
  return SS_OK;
}
