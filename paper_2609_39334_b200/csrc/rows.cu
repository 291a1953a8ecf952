// ss_qk_norm_rope and ss_kv_append: head rows of 128 values on their way from a projection into the attention - normalised
// (keys and queries of models that do), rotated to their positions, rounded once, and written to where the attention reads
// them: the caller's tensors or, keys and values of a step, the slots of the paged pool.
//
//   y = x * w / sqrt(mean(x^2) + eps)                        (w absent: y = x)
//   (y_a, y_b) -> (y_a cos f - y_b sin f, y_b cos f + y_a sin f)   f = position * inv_freq[i], pairs (i, i + R/2) or (2i, 2i + 1)
//
// Eight lanes share a head row: each has two chunks of 8 values (16 bytes) that hold both members of its 8 pairs, so that a
// rotation needs no exchange, and a row's sum of squares takes three shuffles.  A warp has four rows at a time and goes through
// the heads of ONE token after the other (or, with few tokens, through a part of them): queries, keys, values.  The angles are made
// once a token, two a lane: the product in fp64 (a position of a million times a frequency of one has no bits behind the point left
// in fp32), the whole turns off, the rest through sincospif.  Sums, norm and rotation are fp32, two values an instruction, with
// weight and angle in one factor per lane: y = r (x A + x' B), r the norm's.
// Bound: HBM, every row read and written once, and issue slots not far behind (a row takes 22 clocks of an SM's share of the
// bandwidth, and about 30 warp instructions).  65536 tokens of 32 + 8 heads take 230 us, 5.8 TB/s; the steps of 64 of 1024 paths into the
// pool, 32 + 16 heads, 286 us, 5.6 TB/s; eight tokens 4.5 us, the launch and three trips to memory.  What a token needs - row, place,
// position - is looked up by one lane each, for a warp's whole run of tokens at once.
#include "common.cuh"

namespace ss {
namespace rows {

constexpr int kDim = 128, kPage = 16;
constexpr int kWarps = 8;                    // of a block
constexpr int kBlocks = 2;                   // per SM
constexpr int kStages = 8;                   // head rows of a lane group in shared memory or on their way there
constexpr int kSmem = kWarps * kStages * 1024;
// Tokens in a row that a warp takes: longer runs look up and start less, shorter ones end together.  1, 2, 4, 8: 18437 x 32 head rows
// 53.2, 50.8, 52.3, 57.7 us; 65536 x 40 246, 234, 229, 229; appending 18.7 k x 36 80.4, 69.6, 66.9, 71.9; 65.5 k x 48 304, 281, 285, 284.
constexpr int kMostRun = 4;

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
  int run;                                   // tokens in a row that a warp takes
};
struct Place {                               // where the rows of a step go
  const int32_t *node_parent, *node_kv_len, *node_pages, *path_leaf_node, *path_q_len, *num_paths_dev;
  const int64_t *node_page_offsets, *q_offsets, *q_src_offsets;
  __nv_bfloat16 *k_pool, *v_pool;
  int64_t num_pages, page_stride, head_stride, total_node_pages, total_q;
  int num_nodes, num_paths;
};
// What is to be known of a token; lane t of a warp has that of the run's token t.
struct Token {
  int64_t row;                               // of the inputs (and q_out); -1: skipped
  int64_t kv;                                // where its keys and values go, relative to kd / vd (elements); -1: nowhere
  double position;
};

// Fused factors of a lane's 16 values: y = x A + x' B, x' the other member of the pair.  Not INTER: pairs (value j of chunk c0, of
// chunk c1), A and B hold c0's four pairs of values, then c1's; INTER: pairs within a chunk.
typedef unsigned long long f32x2;
struct Lane {
  int c0, c1;                                // this lane's chunks of 8 values
  bool turn0, turn1;                         // which of them are rotated
  f32x2 a[8], b[8];
};
struct Yes { static constexpr bool value = true; };
struct No { static constexpr bool value = false; };
struct alignas(16) WarpShared {                // (sines and cosines are read two at a time: 8 bytes)
  float cs[64], sn[64];
};
static_assert(alignof(WarpShared) % alignof(float2) == 0 && sizeof(WarpShared) % alignof(float2) == 0, "pairs of angles");

__device__ __forceinline__ f32x2 pack2(float a, float b) { f32x2 r; asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b)); return r; }
__device__ __forceinline__ void unpack2(f32x2 v, float& a, float& b) { asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(v)); }
__device__ __forceinline__ f32x2 fma2(f32x2 a, f32x2 b, f32x2 c) { f32x2 r; asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c)); return r; }
__device__ __forceinline__ f32x2 mul2(f32x2 a, f32x2 b) { f32x2 r; asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b)); return r; }
__device__ __forceinline__ f32x2 swap2(f32x2 v) { float a, b; unpack2(v, a, b); return pack2(b, a); }

__device__ __forceinline__ void unpack8(const uint4& u, f32x2 (&f)[4]) {
  const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) f[i] = pack2(__uint_as_float(w[i] << 16), __uint_as_float(w[i] & 0xffff0000u));
}
__device__ __forceinline__ uint4 pack8(const f32x2 (&f)[4]) {
  uint32_t w[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    float x, y;
    unpack2(f[i], x, y);
    const __nv_bfloat162 b = __floats2bfloat162_rn(x, y);
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
// The weights of queries and keys, [2][16] chunks, ones where there are none (whole block).
__device__ __forceinline__ void load_weights(uint4 (&w)[32], const Args& A) {
  const int t = threadIdx.x;
  if (t < 32) {
    const __nv_bfloat16* p = t < 16 ? A.q_weight : A.k_weight;
    w[t] = p ? __ldg(reinterpret_cast<const uint4*>(p) + (t & 15)) : make_uint4(0x3f803f80u, 0x3f803f80u, 0x3f803f80u, 0x3f803f80u);
  }
  __syncthreads();
}

// Sines and cosines of a token's angles (whole warp).
__device__ __forceinline__ void token_angles(WarpShared& W, const Args& A, double position, int lane) {
  __syncwarp();
#pragma unroll
  for (int x = 0; x < 2; ++x) {
    const int i = lane + 32 * x;
    if (i < A.rot / 2) {
      double turns = position * static_cast<double>(__ldg(A.inv_freq + i)) * 0.15915494309189533577;   // / (2 pi)
      turns -= rint(turns);
      sincospif(static_cast<float>(2.0 * turns), &W.sn[i], &W.cs[i]);
    }
  }
  __syncwarp();
}
// A lane's factors for rows with the weights at w.
template <bool INTER>
__device__ __forceinline__ void lane_factors(Lane& L, const WarpShared& W, const uint4* w) {
  f32x2 w0[4], w1[4];
  unpack8(w[L.c0], w0);
  unpack8(w[L.c1], w1);
  if (INTER) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float c0 = L.turn0 ? W.cs[4 * L.c0 + i] : 1.f, s0 = L.turn0 ? W.sn[4 * L.c0 + i] : 0.f;
      const float c1 = L.turn1 ? W.cs[4 * L.c1 + i] : 1.f, s1 = L.turn1 ? W.sn[4 * L.c1 + i] : 0.f;
      L.a[i] = mul2(w0[i], pack2(c0, c0));
      L.b[i] = mul2(swap2(w0[i]), pack2(-s0, s0));
      L.a[4 + i] = mul2(w1[i], pack2(c1, c1));
      L.b[4 + i] = mul2(swap2(w1[i]), pack2(-s1, s1));
    }
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float2 c = L.turn0 ? *reinterpret_cast<const float2*>(W.cs + 8 * L.c0 + 2 * i) : make_float2(1.f, 1.f);
      const float2 s = L.turn0 ? *reinterpret_cast<const float2*>(W.sn + 8 * L.c0 + 2 * i) : make_float2(0.f, 0.f);
      L.a[i] = mul2(w0[i], pack2(c.x, c.y));
      L.b[i] = mul2(w1[i], pack2(-s.x, -s.y));
      L.a[4 + i] = mul2(w1[i], pack2(c.x, c.y));
      L.b[4 + i] = mul2(w0[i], pack2(s.x, s.y));
    }
  }
}

// One head row (its two chunks in a, b).
template <bool INTER>
__device__ __forceinline__ void turn_row(const Lane& L, bool norm, float eps, uint4& a, uint4& b) {
  f32x2 x0[4], x1[4], y0[4], y1[4];
  unpack8(a, x0);
  unpack8(b, x1);
  f32x2 r = pack2(1.f, 1.f);
  if (norm) {
    f32x2 sq = mul2(x0[0], x0[0]);
#pragma unroll
    for (int i = 1; i < 4; ++i) sq = fma2(x0[i], x0[i], sq);
#pragma unroll
    for (int i = 0; i < 4; ++i) sq = fma2(x1[i], x1[i], sq);
    float s0, s1;
    unpack2(sq, s0, s1);
    float sum = s0 + s1;
#pragma unroll
    for (int o = 4; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
    const float f = rsqrtf(sum * (1.f / kDim) + eps);
    r = pack2(f, f);
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    y0[i] = mul2(x0[i], L.a[i]);
    y1[i] = mul2(x1[i], L.a[4 + i]);
  }
  // (values that are not rotated stay as they are: a product with a sine of 0 would carry an infinity over)
  if (L.turn0) {
#pragma unroll
    for (int i = 0; i < 4; ++i) y0[i] = fma2(INTER ? swap2(x0[i]) : x1[i], L.b[i], y0[i]);
  }
  if (L.turn1) {
#pragma unroll
    for (int i = 0; i < 4; ++i) y1[i] = fma2(INTER ? swap2(x1[i]) : x0[i], L.b[4 + i], y1[i]);
  }
  if (norm) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      y0[i] = mul2(y0[i], r);
      y1[i] = mul2(y1[i], r);
    }
  }
  a = pack8(y0);
  b = pack8(y1);
}

__device__ __forceinline__ void copy_16(uint32_t dst, const void* src) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
}

// The heads of the run's tokens that are this warp's: of every tensor those part, part + split, .. in units of four, a lane group
// each.  Keys of head h go to kd + kv + h * d_head, values to vd + kv + h * d_head.  Copies run kStages - 1 head rows ahead of
// their use, across tensors and tokens; a lane reads only what it copied itself, so no barrier is needed.
template <bool INTER>
__device__ __forceinline__ void run_heads(const Args& A, const uint4* weights, WarpShared& W, uint4* ring, const Token& mine, int n_tok,
                                          int part, int lane, __nv_bfloat16* kd, __nv_bfloat16* vd, int64_t d_head) {
  Lane L;
  lane_setup<INTER>(L, A, lane & 7);
  const int step = 4 * A.split, h0 = 4 * part + (lane >> 3);
  auto rounds = [&](int n) { return n > 4 * part ? (n - 4 * part + step - 1) / step : 0; };
  const int q_rounds = rounds(A.hq), k_rounds = rounds(A.hk), v_rounds = rounds(A.hv);
  ring += lane;
  const uint32_t ring_at = static_cast<uint32_t>(__cvta_generic_to_shared(ring));

  // the next copy
  int pt = -1, pwhich = 2, pleft = 0, ph = 0, pn = 0, ps = 0;
  const __nv_bfloat16* pp = nullptr;
  int64_t pstep = 0;
  auto ahead = [&]() {
    while (pleft == 0 && pt < n_tok) {                                            // (warp-uniform: the next tensor, the next token)
      if (++pwhich == 3) { pwhich = 0; ++pt; }
      if (pt == n_tok) break;
      const int64_t row = __shfl_sync(0xffffffffu, mine.row, pt), kv = __shfl_sync(0xffffffffu, mine.kv, pt);
      if (row < 0 || (pwhich && kv < 0)) continue;
      const Tensor& T = pwhich == 0 ? A.q : pwhich == 1 ? A.k : A.v;
      pn = pwhich == 0 ? A.hq : pwhich == 1 ? A.hk : A.hv;
      pleft = pwhich == 0 ? q_rounds : pwhich == 1 ? k_rounds : v_rounds;
      ph = h0;
      pp = T.p + row * T.row + h0 * T.head + 8 * L.c0;
      pstep = step * T.head;
    }
    if (pleft > 0) {
      if (ph < pn) {
        copy_16(ring_at + ps * 1024, pp);
        copy_16(ring_at + ps * 1024 + 512, pp + 8 * (L.c1 - L.c0));
      }
      ph += step;
      pp += pstep;
      --pleft;
      ps = ps + 1 == kStages ? 0 : ps + 1;
    }
    asm volatile("cp.async.commit_group;" ::: "memory");
  };
  int cs = 0;
  auto through = [&](auto turn, __nv_bfloat16* dst, int64_t dst_step, int n, int rounds_here, bool norm) {
    dst += 8 * L.c0;
    int h = h0;
#pragma unroll 1
    for (int g = 0; g < rounds_here; ++g) {
      ahead();
      asm volatile("cp.async.wait_group %0;" ::"n"(kStages - 1) : "memory");
      uint4 a = ring[cs * 64], b = ring[cs * 64 + 32];
      cs = cs + 1 == kStages ? 0 : cs + 1;
      if (decltype(turn)::value) turn_row<INTER>(L, norm, A.eps, a, b);
      if (h < n) {
        *reinterpret_cast<uint4*>(dst) = a;
        *reinterpret_cast<uint4*>(dst + 8 * (L.c1 - L.c0)) = b;
      }
      dst += dst_step;
      h += step;
    }
  };
#pragma unroll 1
  for (int x = 0; x < kStages - 1; ++x) ahead();
#pragma unroll 1
  for (int t = 0; t < n_tok; ++t) {
    const int64_t row = __shfl_sync(0xffffffffu, mine.row, t), kv = __shfl_sync(0xffffffffu, mine.kv, t);
    const double position = __shfl_sync(0xffffffffu, mine.position, t);
    if (row < 0) continue;                                                        // (warp-uniform)
    if (q_rounds | k_rounds) token_angles(W, A, position, lane);
    if (q_rounds) {
      lane_factors<INTER>(L, W, weights);
      through(Yes(), A.q_out.p + row * A.q_out.row + h0 * A.q_out.head, step * A.q_out.head, A.hq, q_rounds, A.q_weight != nullptr);
    }
    if (kv < 0) continue;
    if (k_rounds) {
      lane_factors<INTER>(L, W, weights + 16);
      through(Yes(), kd + kv + h0 * d_head, step * d_head, A.hk, k_rounds, A.k_weight != nullptr);
    }
    if (v_rounds) through(No(), vd + kv + h0 * d_head, step * d_head, A.hv, v_rounds, false);
  }
}

template <bool INTER>
__global__ void __launch_bounds__(kWarps * 32, kBlocks) norm_rope_kernel(const __grid_constant__ Args A) {
  ss::grid_dependency_enter();
  extern __shared__ uint4 ring[];
  __shared__ uint4 weights[32];
  __shared__ WarpShared W[kWarps];
  load_weights(weights, A);
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int64_t w = static_cast<int64_t>(blockIdx.x) * kWarps + warp, r0 = w / A.split * A.run;
  const int n_tok = static_cast<int>(min(static_cast<int64_t>(A.run), A.n_rows - r0));
  if (n_tok <= 0) return;
  Token mine{-1, 0, 0.0};
  if (lane < n_tok) {
    mine.row = r0 + lane;
    mine.kv = mine.row * A.k_out.row;
    if (A.positions) mine.position = static_cast<double>(__ldg(A.positions + mine.row));
  }
  run_heads<INTER>(A, weights, W[warp], ring + warp * (kStages * 64), mine, n_tok, static_cast<int>(w % A.split), lane, A.k_out.p, nullptr, A.k_out.head);
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

template <bool INTER>
__global__ void __launch_bounds__(kWarps * 32, kBlocks) append_kernel(const __grid_constant__ Args A, const __grid_constant__ Place P) {
  ss::grid_dependency_enter();
  extern __shared__ uint4 ring[];
  __shared__ uint4 weights[32];
  __shared__ WarpShared W[kWarps];
  load_weights(weights, A);
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int live = P.num_paths_dev ? min(max(__ldg(P.num_paths_dev), 0), P.num_paths) : P.num_paths;
  if (live == 0) return;
  const int64_t w = static_cast<int64_t>(blockIdx.x) * kWarps + warp;
  const int64_t first = __ldg(P.q_offsets), rows = min(__ldg(P.q_offsets + live) - first, P.total_q);
  const int64_t r0 = w / A.split * A.run;
  const int n_tok = static_cast<int>(min(static_cast<int64_t>(A.run), rows - r0));
  if (n_tok <= 0) return;
  // the first token's path by the whole warp, the others' from there on
  int p = path_of(P.q_offsets, live, first + r0, lane);
  Token mine{-1, -1, 0.0};
  if (lane < n_tok) {
    const int64_t r = first + r0 + lane;
    while (p + 1 < live && __ldg(P.q_offsets + p + 1) <= r) ++p;
    const int64_t q0 = __ldg(P.q_offsets + p), t = r - q0, row = (P.q_src_offsets ? __ldg(P.q_src_offsets + p) : q0) + t;
    const int leaf = __ldg(P.path_leaf_node + p), T = __ldg(P.path_q_len + p);
    if (leaf >= 0 && leaf < P.num_nodes && t < T && row >= 0 && row < A.n_rows) {
      const int at = __ldg(P.node_kv_len + leaf) - T + static_cast<int>(t);       // token of the leaf
      mine.row = row;
      if (at >= 0) {
        const int64_t entry = __ldg(P.node_page_offsets + leaf) + at / kPage;
        if (entry >= 0 && entry < __ldg(P.node_page_offsets + leaf + 1) && entry < P.total_node_pages) {
          const int64_t page = __ldg(P.node_pages + entry);
          if (page >= 0 && page < P.num_pages) mine.kv = page * P.page_stride + static_cast<int64_t>(at % kPage) * kDim;
        }
      }
      int64_t position = at;
      if (A.positions) {
        position = __ldg(A.positions + row);
      } else if (A.rot) {
        int a = __ldg(P.node_parent + leaf);
        for (int d = 1; d < SS_MAX_DEPTH && a >= 0 && a < P.num_nodes; ++d) {
          position += __ldg(P.node_kv_len + a);
          a = __ldg(P.node_parent + a);
        }
      }
      mine.position = static_cast<double>(position);
    }
  }
  __syncwarp();
  run_heads<INTER>(A, weights, W[warp], ring + warp * (kStages * 64), mine, n_tok, static_cast<int>(w % A.split), lane, P.k_pool, P.v_pool, P.head_stride);
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
  if (strides % 8 || strides < 0 || addresses % 16) return SS_ERR_UNSUPPORTED;   // (< 0: one of them is)
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

static int64_t resident_warps() { return static_cast<int64_t>(sm_count_of_current_device()) * kBlocks * kWarps; }
// Warps that share a token: as many as are resident at once, at most one for four heads.  A token on one warp makes its angles once.
static int heads_split(int64_t tokens, int heads) {
  const int most = ceil_div(heads, 4);
  const int64_t split = tokens > 0 ? resident_warps() / tokens : 1;
  return static_cast<int>(split < 1 ? 1 : split > most ? most : split);
}
// Tokens of a warp's run: all warps resident at once, as long as that takes no more than kMostRun.
static int run_of(int64_t tokens, int split) {
  const int64_t run = ceil_div64(tokens * split, resident_warps());
  return static_cast<int>(run < 1 ? 1 : run > kMostRun ? kMostRun : run);
}
template <typename Kernel>
static int32_t prepare(Kernel kernel, bool (&done)[kDeviceSlots]) {
  const int slot = current_device_slot();
  if (slot >= 0 && done[slot]) return SS_OK;
  if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmem) != cudaSuccess) {
    (void)cudaGetLastError();
    return SS_ERR_CUDA;
  }
  if (slot >= 0) done[slot] = true;
  return SS_OK;
}
template <bool INTER>
static int32_t launch_norm_rope(const Args& A, unsigned grid, cudaStream_t st) {
  static bool done[kDeviceSlots] = {false};
  const int32_t rc = prepare(norm_rope_kernel<INTER>, done);
  if (rc != SS_OK) return rc;
  SS_LAUNCH(norm_rope_kernel<INTER>, grid, kWarps * 32, kSmem, st, A);
  return SS_OK;
}
template <bool INTER>
static int32_t launch_append(const Args& A, const Place& P, unsigned grid, cudaStream_t st) {
  static bool done[kDeviceSlots] = {false};
  const int32_t rc = prepare(append_kernel<INTER>, done);
  if (rc != SS_OK) return rc;
  SS_LAUNCH(append_kernel<INTER>, grid, kWarps * 32, kSmem, st, A, P);
  return SS_OK;
}
static int32_t grid_of(int64_t tokens, const Args& A, unsigned* grid) {
  const int64_t blocks = ceil_div64(ceil_div64(tokens, A.run) * A.split, kWarps);
  if (blocks > 0x7fffffffLL) return SS_ERR_UNSUPPORTED;
  *grid = static_cast<unsigned>(blocks);
  return SS_OK;
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
  A.run = run_of(rows->n_rows, A.split);
  unsigned grid = 0;
  const int32_t gc = grid_of(rows->n_rows, A, &grid);
  if (gc != SS_OK) return gc;
  return rows->flags & SS_ROWS_INTERLEAVED ? launch_norm_rope<true>(A, grid, ss::as_stream(stream))
                                           : launch_norm_rope<false>(A, grid, ss::as_stream(stream));
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
  A.run = run_of(d->total_q, A.split);
  unsigned grid = 0;
  const int32_t gc = grid_of(d->total_q, A, &grid);
  if (gc != SS_OK) return gc;
  return rows->flags & SS_ROWS_INTERLEAVED ? launch_append<true>(A, P, grid, ss::as_stream(stream))
                                           : launch_append<false>(A, P, grid, ss::as_stream(stream));
}
