// Tensor-core kernel of ss_draft_attention (tcgen05 + TMEM + TMA): one block per SM, 128 keys a step.
//
// A UNIT is a block of rows of one path and kv head - up to two tiles of 128 rows, token-major, the G heads of the group side by
// side - against the path's whole chain.  The steps of all units in a line are dealt out evenly: block b of the grid has steps
// [b * quota, (b + 1) * quota), so every block has the same work whatever the lengths, and at most its first and its last unit are
// shared with its neighbours.  What a block has of a shared unit goes out as a partial result (normalised, with its log-sum),
// merged by the kernel behind this one; everything else is written once, final.
//
// Two softmax STREAMS of four warps, a thread per row, each with its own scores (2 x 64 TMEM columns) and accumulator (128), go
// over a step's keys in halves of 64:
//   a unit of two tiles: stream s has tile s and both halves (a key is read once for up to 256 rows);
//   a unit of one tile:  stream s has half s, and the two accumulators are joined at the end.
// A stream's products are issued by one lane: S(q) = Q K^T of half step q goes out before O += P(q-1) V, so that the next scores are
// there when the softmax is through with the last ones.  tcgen05 instructions of one thread run in order: S(q) may overwrite P(q-2),
// and when S(q) is there, the products up to P(q-2) V are in the accumulator.
// (With scores of 128 keys in one buffer, Q K^T then with N = 128, a stream waits for P V and Q K^T after every softmax: 64 paths of 64
// drafts over 5120 keys, 32q / 8kv heads, 364 us with the streams' products in turn from one warp, against 350 on the same box.)
// Softmax of a half step: exponentials relative to the reference there is, their fp32 sum, probabilities in bf16 over the scores they
// come from; nothing waits for a maximum.  Where the sum exceeds 2^16 (or is none), where the row has no reference yet, and in steps with
// masks, the scores are read (again) for their exact maximum, which becomes the reference if it exceeds that by 2^8; the accumulator is
// then rescaled.  So no exponential is ever larger than 2^16, and no row pays for another block's.
// What bounds it: a half step of both streams takes the tensor cores 1280 clocks (Q K^T with N = 64 reads more shared memory than it
// multiplies for: 48 clocks an instruction, 32 of them products) and the special-function units 1024 for its exponentials.  Every fourth pair of
// exponentials goes to the FMA pipe instead (exp2_pair): 378 -> 350 us in that case on that box, every eighth pair 352, three of eight 353.  Both
// streams together then take some 1700 clocks: their tails (load, vote, store: 400) hardly overlap.  Two threads a row and strict turns
// of the streams at their exponentials were slower.  How long the case takes goes by the clock that the power cap leaves: back to back over
// changing inputs 415 us at 1.46 GHz and 985 W, 374 us with pauses between the calls (another box than the figures above).
// Masks: from 128 bits per row (which drafts it sees) and the page's place in the chain, in steps that reach the drafts only.
// Keys that nobody may read (behind a node's end) have their V rows cleared in shared memory; a draft that holds NaN or an infinity
// and is hidden from some rows reaches them as 0 * NaN: a row that is not finite is computed again, key by key, without it.
// Roles: warps 0-3, 4-7 streams; 8 K and Q through TMA and the next unit's description; 9 V through TMA; 10, 11 issue the streams'
// products.  They go from unit to unit on their own (descriptions in two slots): while the streams write a unit's rows out, the
// next one's first keys and its queries are on their way and multiplied.  Every wait is bounded (see umma.cuh, wait_behind_rows).
#include "draft_attn.cuh"
#include "exp2.cuh"
#include "umma.cuh"

namespace ss {
namespace draft {

using namespace umma;

constexpr int kSoftmaxWarps = 8;
constexpr int kThreads = (kSoftmaxWarps + 4) * 32;
constexpr int kStageBytes = kTile * 256;       // one K or V step: [16 groups of 8 keys][2 halves of 64 dims][8 rows][128 B]
constexpr int kStagesK = 3, kStagesV = 2;
constexpr uint32_t kTmemCols = 512, kColS = 0, kColO = 256;
constexpr int kOffQ = 0, kOffK = 65536, kOffV = kOffK + kStagesK * kStageBytes;
constexpr int kSmem = kOffV + kStagesV * kStageBytes;
constexpr float kLazyLog2 = 8.0f;
constexpr float kMostSum = 65536.0f;           // of a half step's exponentials

struct Unit {
  int valid;                                   // 0: the block's work is done
  int g, n_tok, dual;
  int tile0, n_tiles;                          // this block's steps of it
  int slot;                                    // of its partial result; -1: the unit is this block's alone
  int drafts0;                                 // index of the first draft in the path's sequence
  int holes, clear_last;                       // a node that ends inside a page: anywhere, or in the last step
  int64_t src, dst;                            // rows of q and out of its first token
  Chain C;
};
struct Ctrl {
  uint64_t unit_ready[2], unit_free[2], q_free;
  uint64_t q_full, k_full[kStagesK], k_empty[kStagesK], v_full[kStagesV], v_empty[kStagesV], v_land, s_full[2][2], p_full[2][2], o_before[2], o_final[2];
  uint32_t tmem_slot;
  int abort_flag;
  int redo[2];                                 // by unit slot: some row is to be computed again
  int stop;                                    // a softmax thread has given up
  alignas(16) int coord[2][32];                // pool rows of the pages of four steps, by producer warp
  long long warp_total[kThreads / 32];
  long long pos, end, quota, off;              // this block's place in the line; off: in the steps of path `path`
  int path;
  float exchange[2][128];                      // between the streams of a row
  Unit unit[2];
};
static_assert(sizeof(Ctrl) + kSmem <= 232448, "shared memory of a block");

// mbar_wait of a role that the softmax warps keep waiting while they compute rows again (unit_rows_exact: 0.35 us a row and key of a warp, 0.2 s
// at 18000 keys of 256 rows, and no wait in it that could fail to end).  The limit counts from when they were last seen at that.
__device__ __forceinline__ bool wait_behind_rows(uint64_t* bar, uint32_t parity, Ctrl& C) {
  if (mbar_try_wait(bar, parity)) return true;
  const volatile int* redo = C.redo;
  volatile int* abort_flag = &C.abort_flag;
  long long t0 = 0;
  uint32_t spins = 0;
  while (!mbar_try_wait_suspend(bar, parity, 20000u)) {
    if ((++spins & 15u) != 0u) continue;
    if (*abort_flag) return false;
    if (t0 == 0 || (redo[0] | redo[1]) != 0) {
      t0 = clock64();
    } else if (clock64() - t0 > kWaitCycles) {
      *abort_flag = 1;
      return false;
    }
  }
  return true;
}
__device__ __forceinline__ float max3(float a, float b, float c) { float r; asm("max.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c)); return r; }
__device__ __forceinline__ uint32_t pack_bf16(float a, float b) {
  const __nv_bfloat162 pk = __floats2bfloat162_rn(a, b);
  return *reinterpret_cast<const uint32_t*>(&pk);
}
__device__ __forceinline__ void store_32B(void* p, const uint32_t (&w)[8]) {
  asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(p), "r"(w[0]), "r"(w[1]), "r"(w[2]), "r"(w[3]),
               "r"(w[4]), "r"(w[5]), "r"(w[6]), "r"(w[7]) : "memory");
}

// 128 bytes of every lane to its own line (null: nowhere): four lanes' quarters are exchanged, so that a store instruction writes eight
// whole lines and not a sector of 32.
__device__ __forceinline__ void store_lines(void* line, uint32_t (&w)[32], int lane) {
#pragma unroll
  for (int m = 1; m <= 2; m *= 2) {
    const bool upper = (lane & m) != 0;
#pragma unroll
    for (int p = 0; p < 4; ++p) {
      if (p & m) continue;
#pragma unroll
      for (int x = 0; x < 8; ++x) {
        uint32_t &a = w[8 * p + x], &b = w[8 * (p | m) + x];
        const uint32_t v = __shfl_xor_sync(0xffffffffu, upper ? a : b, m);
        if (upper) a = v; else b = v;
      }
    }
  }
  // quarter `lane & 3` of the lines of lanes 4 g .. 4 g + 3
  const unsigned long long mine = reinterpret_cast<unsigned long long>(line);
#pragma unroll
  for (int p = 0; p < 4; ++p) {
    const unsigned long long to = __shfl_sync(0xffffffffu, mine, (lane & ~3) | p);
    const uint32_t q[8] = {w[8 * p], w[8 * p + 1], w[8 * p + 2], w[8 * p + 3], w[8 * p + 4], w[8 * p + 5], w[8 * p + 6], w[8 * p + 7]};
    if (to) store_32B(reinterpret_cast<char*>(to) + 32 * (lane & 3), q);
  }
}

__device__ __forceinline__ long long path_cost(const PathInfo& I, int Hkv) {
  return I.T > 0 ? static_cast<long long>(I.tiles) * I.blocks * Hkv : 0;
}

// (A division of 64 bits takes some hundred clocks.)
__device__ __forceinline__ long long quotient(long long a, long long b) {
  return (a | b) >> 31 ? a / b : static_cast<int>(a) / static_cast<int>(b);
}

// The next unit of this block's line into slot `dst` (whole warp).
__device__ __noinline__ void fetch_unit(Ctrl& C, const Params& P, int dst, int lane) {
  Unit& U = C.unit[dst];
  const long long pos = C.pos, end = C.end, quota = C.quota;
  if (pos >= end || *const_cast<volatile int*>(&C.abort_flag)) {
    __syncwarp();
    if (lane == 0) U.valid = 0;
    return;
  }
  int path = C.path;
  long long off = C.off;
  // (the chain's words are on their way while the path is looked at: it is the right one for all but a path's last unit)
  constexpr int kWords = static_cast<int>(sizeof(Chain) / 4), kMine = (kWords + 31) / 32;
  uint32_t word[kMine];
  auto load_chain = [&]() {
    const uint32_t* from = reinterpret_cast<const uint32_t*>(P.chains + path);
#pragma unroll
    for (int x = 0; x < kMine; ++x) word[x] = x * 32 + lane < kWords ? from[x * 32 + lane] : 0u;
  };
  load_chain();
  PathInfo I = P.paths[path];
  if (off >= path_cost(I, P.Hkv)) {            // (ends: steps are left)
    do {
      off -= path_cost(I, P.Hkv);
      I = P.paths[++path];
    } while (off >= path_cost(I, P.Hkv));
    load_chain();
  }
  uint32_t* to = reinterpret_cast<uint32_t*>(&U.C);
#pragma unroll
  for (int x = 0; x < kMine; ++x)
    if (x * 32 + lane < kWords) to[x * 32 + lane] = word[x];
  const int u = static_cast<int>(quotient(off, I.tiles));
  const int tile0 = static_cast<int>(off - static_cast<long long>(u) * I.tiles);
  const int n_tiles = static_cast<int>(min(static_cast<long long>(I.tiles - tile0), end - pos));
  __syncwarp();
  if (lane == 0) {
    U.tile0 = tile0;
    U.n_tiles = n_tiles;
    U.g = u / I.blocks;
    const int tok0 = (u - U.g * I.blocks) * I.per_block;
    U.n_tok = min(I.per_block, I.T - tok0);
    U.dual = U.n_tok > P.tok_per_tile;
    U.drafts0 = I.L - I.T;
    U.holes = I.holes;
    U.clear_last = I.L % kTile != 0 || I.L == 0;
    U.src = I.src + tok0;
    U.dst = I.dst + tok0;
    const bool first = pos == quota * blockIdx.x, whole = n_tiles == I.tiles;
    U.slot = whole ? -1 : 2 * static_cast<int>(blockIdx.x) + (first ? 0 : 1);
    if (!whole && tile0 == 0) {                // it starts here and ends with block `last`: the merge begins at this block
      const int last = static_cast<int>(quotient(pos + I.tiles - 1, quota));
      P.cuts[blockIdx.x] = CutUnit{last - static_cast<int>(blockIdx.x) + 1, U.slot, U.g, U.n_tok, U.dst};
    }
    C.pos = pos + n_tiles;
    C.off = off + n_tiles;
    C.path = path;
    U.valid = 1;
  }
}

// The rows of a unit's part once more, a warp per row, key by key: what a row does not see is not touched.
__device__ __noinline__ void unit_rows_exact(const Params& P, const Unit& U, int warp, int lane) {
  const int rows = U.n_tok * P.G;
  for (int x = warp; x < rows; x += kSoftmaxWarps) {
    const int t = x / P.G, h = U.g * P.G + x - t * P.G;
    Row r;
    row_start(r, P.q + ((U.src + t) * P.Hq + h) * kDim, lane);
    row_visit(r, U.C, P, U.g, U.tile0 * kTilePages, (U.tile0 + U.n_tiles) * kTilePages, U.drafts0, P.seen[U.dst + t], lane);
    const float inv = r.l == 0.f ? 0.f : 1.f / r.l;
    float o[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) o[i] = r.l == 0.f ? 0.f : r.acc[i] * inv;
    if (U.slot < 0) {
      store_out(P, U.dst + t, h, lane, o, row_lse(r.m, r.l));
    } else {
      const int64_t at = static_cast<int64_t>(U.slot) * (2 * kRows) + (t < P.tok_per_tile ? x : kRows + x - P.tok_per_tile * P.G);
      *reinterpret_cast<float4*>(P.part_o + at * kDim + 4 * lane) = make_float4(o[0], o[1], o[2], o[3]);
      if (lane == 0) P.part_lse[at] = row_lse(r.m, r.l);
    }
  }
}

// BLOCKS: a page's rows of one head start on 8-row boundaries of the pool and come as one copy, else as four.
template <bool BLOCKS>
__global__ void __launch_bounds__(kThreads, 1)
draft_umma_kernel(const __grid_constant__ CUtensorMap tmap_k, const __grid_constant__ CUtensorMap tmap_v,
                  const __grid_constant__ CUtensorMap tmap_q, const __grid_constant__ Params P) {
  ss::grid_dependency_enter();
  extern __shared__ __align__(1024) uint8_t smem[];
  __shared__ Ctrl C;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  volatile int* abort_flag = &C.abort_flag;

  if (tid == kThreads - 32) {                  // (a warp that has few paths to look at)
    C.abort_flag = (smem_u32(smem) & 1023u) ? 1 : 0;
    C.redo[0] = C.redo[1] = C.stop = 0;
    for (int s = 0; s < 2; ++s) { mbar_init(&C.unit_ready[s], 1); mbar_init(&C.unit_free[s], kSoftmaxWarps + 3); }
    mbar_init(&C.q_full, 1);
    mbar_init(&C.q_free, 2);
    for (int s = 0; s < kStagesK; ++s) { mbar_init(&C.k_full[s], 1); mbar_init(&C.k_empty[s], 2); }
    for (int s = 0; s < kStagesV; ++s) { mbar_init(&C.v_full[s], 1); mbar_init(&C.v_empty[s], 2); }
    mbar_init(&C.v_land, 1);
    for (int s = 0; s < 2; ++s) {
      for (int b = 0; b < 2; ++b) { mbar_init(&C.s_full[s][b], 1); mbar_init(&C.p_full[s][b], 128); }
      mbar_init(&C.o_before[s], 1);
      mbar_init(&C.o_final[s], 1);
    }
    fence_barrier_init();
    prefetch_tensormap(&tmap_k);
    prefetch_tensormap(&tmap_v);
    prefetch_tensormap(&tmap_q);
    P.cuts[blockIdx.x].n = 0;
  }
  // (What shared memory holds in rows that no box of Q rows reaches comes out in rows that nobody reads.)
  if (warp == kSoftmaxWarps) tmem_alloc(&C.tmem_slot, kTmemCols);

  // ---- this block's place in the line: sums over the paths, a stretch of them per thread
  const int chunk = (P.num_paths + kThreads - 1) / kThreads;
  const int p0 = min(tid * chunk, P.num_paths), p1 = min(p0 + chunk, P.num_paths);
  long long mine = 0;
  for (int p = p0; p < p1; ++p) {
    const PathInfo I = P.paths[p];
    if (I.status != SS_OK && blockIdx.x == 0) set_status(&P.hdr->status, I.status);
    mine += path_cost(I, P.Hkv);
  }
  long long incl = mine;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const long long up = __shfl_up_sync(0xffffffffu, incl, o);
    if (lane >= o) incl += up;
  }
  if (lane == 31) C.warp_total[warp] = incl;
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  long long before = 0, total = 0;
#pragma unroll
  for (int w = 0; w < kThreads / 32; ++w) {
    if (w < warp) before += C.warp_total[w];
    total += C.warp_total[w];
  }
  incl += before;
  const long long quota = max(quotient(total + gridDim.x - 1, gridDim.x), 1LL), start = quota * blockIdx.x;
  if (tid == 0) { C.pos = start; C.end = min(start + quota, total); C.quota = quota; }
  if (start < total && incl - mine <= start && start < incl) {
    C.path = p0;
    C.off = start - (incl - mine);
  }
  __syncthreads();
  const uint32_t tmem = C.tmem_slot;
  const int G = P.G, tpt = P.tok_per_tile;
  uint32_t g_tile = 0;                         // steps behind this block (the same in every role)
  uint32_t n_half = 0;                         // half steps behind each stream
  uint32_t n_before = 0;                       // units with more than one half step behind
  uint32_t n_land = 0;                         // V producer: cleared steps so far
  uint32_t seq = 0;

  // The next unit, when its description is there; false: none, or a wait has run out.
  auto unit_there = [&]() -> bool { return wait_behind_rows(&C.unit_ready[seq & 1], (seq >> 1) & 1, C); };
  auto unit_done = [&]() {
    __syncwarp();
    if (lane == 0) mbar_arrive(&C.unit_free[seq & 1]);
  };
  if (warp == kSoftmaxWarps) {
    fetch_unit(C, P, 0, lane);
    __syncwarp();
    if (lane == 0) mbar_arrive(&C.unit_ready[0]);
  }

  for (;; ++seq) {
    const Unit& U = C.unit[seq & 1];
    bool there = unit_there();
    if (warp < kSoftmaxWarps) {                                  // (they meet at barriers: all of them go on, or none)
      if (!there) C.stop = 1;
      asm volatile("bar.sync 1, 256;" ::: "memory");
      there = *const_cast<volatile int*>(&C.stop) == 0;
    } else {
      there = __all_sync(0xffffffffu, there);
    }
    if (!there || !U.valid) break;
    const int n_tiles = U.n_tiles, dual = U.dual;
    const int halves = dual ? 2 * n_tiles : n_tiles;             // of each stream

    if (warp < kSoftmaxWarps) {
      // =================================================== softmax + epilogue ==================================
      const int s = warp >> 2, row = tid & 127;
      const int tok_base = dual && s ? tpt : 0, tok_here = dual ? (s ? U.n_tok - tpt : tpt) : U.n_tok;
      const int i = row / G, hl = row - i * G;
      const bool row_valid = i < tok_here;
      const bool any_row = __any_sync(0xffffffffu, row_valid);
      const uint4 seen = row_valid ? P.seen[U.dst + tok_base + i] : make_uint4(0, 0, 0, 0);
      const uint32_t lanes = static_cast<uint32_t>((warp & 3) * 32) << 16;
      const uint32_t t_o = tmem + lanes + kColO + s * 128;
      const float cl2 = P.scale_log2, lazy_raw = kLazyLog2 / cl2;
      float m = -INFINITY, l = 0.f;
      bool ok = true;
      for (int q = 0; q < halves; ++q) {
        const uint32_t gq = n_half + q;
        const int jt = U.tile0 + (dual ? q >> 1 : q), hf = dual ? q & 1 : s;      // step of the chain, half of it
        const uint32_t t_s = tmem + lanes + kColS + s * 128 + (gq & 1) * 64;
        if (!mbar_wait(&C.s_full[s][gq & 1], (gq >> 1) & 1, abort_flag)) ok = false;
        if (!any_row) {                        // (products of rows that nobody asked for come out in rows that nobody reads)
          mbar_arrive(&C.p_full[s][gq & 1]);
          continue;
        }
        tc_fence_after();
        uint32_t sr[64], pr[32];
        uint32_t (&sr0)[32] = *reinterpret_cast<uint32_t(*)[32]>(&sr[0]), (&sr1)[32] = *reinterpret_cast<uint32_t(*)[32]>(&sr[32]);
        const f32x2 cl2_2 = pack2(cl2, cl2);
        f32x2 sum2[2];
        // Exponentials of 32 scores; `fast`: some on the FMA pipe (where none is of a masked key).
        auto exps = [&](int c0, f32x2 nmc2, bool fast) {
#pragma unroll
          for (int c = c0; c < c0 + 32; c += 2) {
            const f32x2 x = fma2(pack2(__uint_as_float(sr[c]), __uint_as_float(sr[c + 1])), cl2_2, nmc2);
            float e0, e1;
            unpack2(x, e0, e1);
            if (fast && (c & 6) == 6) {
              exp2_pair(e0, e1, -126.f);
            } else {
              e0 = ex2(e0);
              e1 = ex2(e1);
            }
            sum2[(c >> 1) & 1] = add2(sum2[(c >> 1) & 1], pack2(e0, e1));
            pr[c >> 1] = pack_bf16(e0, e1);
          }
        };
        auto sum_of = [&]() {
          float a0, a1, a2, a3;
          unpack2(sum2[0], a0, a1);
          unpack2(sum2[1], a2, a3);
          return (a0 + a1) + (a2 + a3);
        };
        const bool masked = U.holes || jt * kTile + hf * 64 + 64 > U.drafts0;    // (block-uniform) not everything is seen
        bool fits = !masked && !__any_sync(0xffffffffu, row_valid && m == -INFINITY);
        float alpha = 1.f, sum = 0.f;
        bool move = false;
        tmem_ld32(t_s, sr0);
        if (fits) {                            // by the reference there is
          const f32x2 nmc2 = pack2(-m * cl2, -m * cl2);
          sum2[0] = sum2[1] = pack2(0.f, 0.f);
          tmem_wait_ld();
          tmem_pin32(sr0);
          tmem_ld32(t_s + 32, sr1);
          exps(0, nmc2, true);
          tmem_wait_ld();
          tmem_pin32(sr1);
          exps(32, nmc2, true);
          sum = sum_of();
          fits = !__any_sync(0xffffffffu, row_valid && !(sum <= kMostSum));      // (not for a NaN)
          if (!fits) tmem_ld32(t_s, sr0);
        }
        if (!fits) {                           // by the maximum
          tmem_ld32(t_s + 32, sr1);
          tmem_wait_ld();
          tmem_pin32(sr0);
          tmem_pin32(sr1);
          if (masked) {
            const int pages = U.C.first[U.C.n];
#pragma unroll
            for (int w = 0; w < 4; ++w) {
              const int vp = jt * kTilePages + hf * 4 + w;
              const uint32_t mask = vp < pages ? page_mask(U.C, segment_of(U.C, vp), vp, U.drafts0, seen) : 0u;
#pragma unroll
              for (int c = 0; c < 16; ++c)
                if (!((mask >> c) & 1u)) sr[16 * w + c] = 0xff800000u;           // -inf
            }
          }
          float e[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
          for (int c = 0; c < 64; c += 2) e[(c >> 1) & 3] = max3(e[(c >> 1) & 3], __uint_as_float(sr[c]), __uint_as_float(sr[c + 1]));
          const float mx = fmaxf(fmaxf(e[0], e[1]), fmaxf(e[2], e[3]));
          move = row_valid && (mx > m + lazy_raw || (m == -INFINITY && mx > -INFINITY));    // (the row's first visible key)
          if (move) {
            alpha = ex2((m - mx) * cl2);                                         // 0 for the first
            m = mx;
            l *= alpha;
          }
          const float mc = m == -INFINITY ? 0.f : m * cl2;
          sum2[0] = sum2[1] = pack2(0.f, 0.f);
          exps(0, pack2(-mc, -mc), false);
          exps(32, pack2(-mc, -mc), false);
          sum = sum_of();
        }
        tmem_st32(t_s, pr);                                                      // over the scores they come from
        l += sum;
        if (__any_sync(0xffffffffu, move && q > 0)) {                            // rescale O (warp-collective), once P(q-1) V is in it:
          // the scores of the half step after this one were asked for behind that product
          const uint32_t gn = gq + 1;
          ok = (q + 1 < halves ? mbar_wait(&C.s_full[s][gn & 1], (gn >> 1) & 1, abort_flag)
                               : mbar_wait(&C.o_before[s], n_before & 1, abort_flag)) && ok;
          tc_fence_after();
#pragma unroll 1
          for (int c0 = 0; c0 < kDim; c0 += 32) {
            uint32_t o[32];
            __syncwarp();
            tmem_ld32(t_o + c0, o);
            tmem_wait_ld();
#pragma unroll
            for (int x = 0; x < 32; ++x) o[x] = __float_as_uint(__uint_as_float(o[x]) * alpha);
            tmem_st32(t_o + c0, o);
          }
        }
        tmem_wait_st();
        tc_fence_before();
        mbar_arrive(&C.p_full[s][gq & 1]);
      }
      // ---- epilogue
#pragma unroll
      for (int x = 0; x < 2; ++x)
        if (x == s || !dual) ok = mbar_wait(&C.o_final[x], seq & 1, abort_flag) && ok;
      ok = __all_sync(0xffffffffu, ok);
      tc_fence_after();
      float w_own = 1.f, w_oth = 0.f;
      if (!dual) {                                                               // the two streams of a row become one
        auto other = [&](float mine) {
          C.exchange[s][row] = mine;
          asm volatile("bar.sync 1, 256;" ::: "memory");
          const float got = C.exchange[s ^ 1][row];
          asm volatile("bar.sync 1, 256;" ::: "memory");
          return got;
        };
        const float m2 = other(m), l2 = other(l);
        const float top = fmaxf(m, m2);
        w_own = m == -INFINITY ? 0.f : ex2((m - top) * cl2);
        w_oth = m2 == -INFINITY ? 0.f : ex2((m2 - top) * cl2);
        l = s == 0 ? l * w_own + l2 * w_oth : l2 * w_oth + l * w_own;
        m = top;
      }
      const float inv = l == 0.f ? 0.f : 1.f / l;
      const float lse = l == 0.f ? -INFINITY : m * P.scale + __logf(l);
      w_own *= inv;
      w_oth *= inv;
      const uint32_t t_oth = tmem + lanes + kColO + (s ^ 1) * 128;
      bool finite = lse < INFINITY;                                              // (not for a NaN)
      // 32 columns of the row's result from c0 on
      auto result32 = [&](int c0, uint32_t (&o)[32]) {
        __syncwarp();
        tmem_ld32(t_o + c0, o);
        tmem_wait_ld();
#pragma unroll
        for (int x = 0; x < 32; ++x) o[x] = __float_as_uint(__uint_as_float(o[x]) * w_own);
        if (!dual) {
          uint32_t o2[32];
          tmem_ld32(t_oth + c0, o2);
          tmem_wait_ld();
#pragma unroll
          for (int x = 0; x < 32; ++x) o[x] = __float_as_uint(fmaf(__uint_as_float(o2[x]), w_oth, __uint_as_float(o[x])));
        }
#pragma unroll
        for (int x = 0; x < 32; ++x) finite = finite && fabsf(__uint_as_float(o[x])) < INFINITY;
      };
      if (ok) {
        const int c_begin = dual ? 0 : s * 64, c_end = dual ? kDim : s * 64 + 64;
        if (U.slot < 0) {
          __nv_bfloat16* dst = P.out + ((U.dst + tok_base + i) * P.Hq + U.g * G + hl) * kDim;
#pragma unroll 1
          for (int c0 = c_begin; c0 < c_end; c0 += 64) {
            uint32_t o[32], w[32];
#pragma unroll
            for (int y = 0; y < 2; ++y) {
              result32(c0 + 32 * y, o);
#pragma unroll
              for (int x = 0; x < 16; ++x) w[16 * y + x] = pack_bf16(__uint_as_float(o[2 * x]), __uint_as_float(o[2 * x + 1]));
            }
            store_lines(row_valid ? dst + c0 : nullptr, w, lane);
          }
        } else {
          float* dst = P.part_o + (static_cast<int64_t>(U.slot) * (2 * kRows) + (dual && s ? kRows : 0) + row) * kDim;
#pragma unroll 1
          for (int c0 = c_begin; c0 < c_end; c0 += 32) {
            uint32_t o[32];
            result32(c0, o);
            store_lines(row_valid ? dst + c0 : nullptr, o, lane);
          }
        }
        // (hidden keys are drafts: where none is near, what is not finite is the result)
        if (row_valid && !finite && (U.holes || (U.tile0 + n_tiles) * kTile > U.drafts0)) C.redo[seq & 1] = 1;
        if (row_valid && (dual || s == 0)) {
          if (U.slot >= 0) P.part_lse[static_cast<int64_t>(U.slot) * (2 * kRows) + (dual && s ? kRows : 0) + row] = lse;
          else if (P.lse) P.lse[(U.dst + tok_base + i) * P.Hq + U.g * G + hl] = lse;
        }
      }
      tc_fence_before();
      asm volatile("bar.sync 1, 256;" ::: "memory");             // (each stream has read the other's accumulator, too)
      if (C.redo[seq & 1]) {
        unit_rows_exact(P, U, warp, lane);
        asm volatile("bar.sync 1, 256;" ::: "memory");
        if (tid == 0) C.redo[seq & 1] = 0;                       // (set again two units on)
      }
      unit_done();
    } else if (warp < kSoftmaxWarps + 2) {
      // =================================================== producers ==============================================
      const int which = warp - kSoftmaxWarps;                    // 0: K (and Q), 1: V
      const int n_stages = which ? kStagesV : kStagesK;
      const CUtensorMap* tm = which ? &tmap_v : &tmap_k;
      uint64_t* full = which ? C.v_full : C.k_full;
      uint64_t* empty = which ? C.v_empty : C.k_empty;
      uint8_t* ring = smem + (which ? kOffV : kOffK);
      const int pages = U.C.first[U.C.n];
      bool ok = true;
      // Q rows, once the products of the unit before have read theirs (behind the first steps' keys, which need not wait for that)
      auto load_q = [&]() {
        if (seq > 0) ok = wait_behind_rows(&C.q_free, (seq - 1) & 1, C);
        ok = __all_sync(0xffffffffu, ok);
        if (ok && elect_one()) {
          mbar_arrive_expect_tx(&C.q_full, static_cast<uint32_t>((dual ? 2 : 1) * 2 * 128 * G * tpt));
          for (int x = 0; x < 1 + dual; ++x) {
            uint8_t* dst = smem + kOffQ + x * 32768;
            const int src = static_cast<int>(U.src) + x * tpt;
            tma_load_3d(dst, &tmap_q, 0, U.g * G, src, &C.q_full);
            tma_load_3d(dst + 16384, &tmap_q, 64, U.g * G, src, &C.q_full);
          }
        }
        __syncwarp();
      };
      // The pages of four steps at a time, one a lane, a block ahead of their use; one elected lane issues the copies.
      auto pool_row = [&](int j, int pg) -> int {
        const int vp = (U.tile0 + j) * kTilePages + pg;
        if (j >= n_tiles || vp >= pages) return 0;
        return static_cast<int>((physical_page(U.C, P, segment_of(U.C, vp), vp) * P.page_stride + static_cast<int64_t>(U.g) * P.head_stride) >> 7);
      };
      int* coord = C.coord[which];
      int cur = pool_row(lane >> 3, lane & 7);
      if (which == 0 && seq == 0) load_q();
      for (int j0 = 0; j0 < n_tiles && ok; j0 += 4) {
        const int nxt = pool_row(j0 + 4 + (lane >> 3), lane & 7);
        coord[lane] = cur;
        __syncwarp();
        for (int t = 0; t < 4 && j0 + t < n_tiles && ok; ++t) {
          const uint32_t gj = g_tile + j0 + t;
          const int st = gj % n_stages, jt = U.tile0 + j0 + t;
          const uint32_t u = gj / n_stages;
          const int n_pages = max(0, min(kTilePages, pages - jt * kTilePages));
          const bool last = (jt + 1) * kTilePages >= pages;
          const bool clear = which == 1 && (U.holes || (last && U.clear_last));
          if (u > 0) ok = wait_behind_rows(&empty[st], (u - 1) & 1, C);
          ok = __all_sync(0xffffffffu, ok);
          if (!ok) break;
          uint8_t* dst = ring + st * kStageBytes;
          if (elect_one()) {
            uint64_t* bar = clear ? &C.v_land : &full[st];
            mbar_arrive_expect_tx(bar, static_cast<uint32_t>(n_pages) * 4096u);
#pragma unroll
            for (int pg = 0; pg < kTilePages; ++pg) {
              if (pg < n_pages) {
                const int y = coord[t * 8 + pg];
                if (BLOCKS) {
                  tma_load_4d(dst + pg * 4096, tm, 0, 0, 0, y >> 3, bar);
                } else {
#pragma unroll
                  for (int x = 0; x < 4; ++x) tma_load_2d(dst + pg * 4096 + x * 1024, tm, (x & 1) * 64, y + (x >> 1) * 8, bar);
                }
              }
            }
          }
          __syncwarp();
          if (clear) {                                           // V rows of keys that are none
            ok = wait_behind_rows(&C.v_land, n_land & 1, C);
            ++n_land;
            ok = __all_sync(0xffffffffu, ok);
            if (!ok) break;
            for (int r = lane; r < kTile; r += 32) {
              const int vp = jt * kTilePages + (r >> 4);
              bool there = false;
              if (vp < pages) {
                const int sg = segment_of(U.C, vp);
                there = (vp - U.C.first[sg]) * kPage + (r & 15) < U.C.len[sg];
              }
              if (!there) {
#pragma unroll
                for (int x = 0; x < 16; ++x) *reinterpret_cast<uint4*>(dst + (r >> 3) * 2048 + (x >> 3) * 1024 + (r & 7) * 128 + (x & 7) * 16) = make_uint4(0, 0, 0, 0);
              }
            }
            fence_proxy_async_smem();
            __syncwarp();
            if (lane == 0) mbar_arrive(&full[st]);
          }
          if (which == 0 && seq > 0 && j0 + t == min(1, n_tiles - 1)) load_q();
        }
        __syncwarp();
        cur = nxt;
      }
      if (which == 0) {
        const int next = (seq & 1) ^ 1;
        if (seq > 0) ok = wait_behind_rows(&C.unit_free[next], ((seq - 1) >> 1) & 1, C) && ok;
        __syncwarp();
        fetch_unit(C, P, next, lane);
        __syncwarp();
        if (lane == 0) mbar_arrive(&C.unit_ready[next]);
      } else {
        unit_done();
      }
    } else {
      // =================================================== products of stream s =================================
      const int s = warp - (kSoftmaxWarps + 2);
      if (elect_one()) {
        constexpr uint32_t idesc_qk = instr_desc_bf16(128, 64, false), idesc_pv = instr_desc_bf16(128, kDim, true);
        const uint64_t q_desc = smem_desc_sw128(smem_u32(smem + kOffQ + (dual ? s : 0) * 32768), 0, 1024);
        const uint64_t k_desc0 = smem_desc_sw128(smem_u32(smem + kOffK), 0, 2048);
        const uint64_t v_desc0 = smem_desc_sw128(smem_u32(smem + kOffV), 1024, 2048);
        const uint32_t t_s = tmem + kColS + s * 128, t_o = tmem + kColO + s * 128;
        auto issue_qk = [&](int q) -> bool {
          const uint32_t gq = n_half + q, gj = g_tile + (dual ? q >> 1 : q);
          const int sk = gj % kStagesK, hf = dual ? q & 1 : s;
          if (!wait_behind_rows(&C.k_full[sk], (gj / kStagesK) & 1, C)) return false;
          tc_fence_after();
          const uint64_t k_desc = smem_desc_advance(k_desc0, static_cast<uint32_t>(sk) * kStageBytes + hf * 16384u);
#pragma unroll
          for (int kk = 0; kk < 8; ++kk)
            mma_bf16_ss(t_s + (gq & 1) * 64, smem_desc_advance(q_desc, (kk >> 2) * 16384 + (kk & 3) * 32),
                        smem_desc_advance(k_desc, (kk >> 2) * 1024 + (kk & 3) * 32), idesc_qk, kk > 0 ? 1u : 0u);
          mma_commit(&C.s_full[s][gq & 1]);
          if (!dual || hf) mma_commit(&C.k_empty[sk]);
          if (q + 1 == halves) mma_commit(&C.q_free);
          return true;
        };
        bool ok = wait_behind_rows(&C.q_full, seq & 1, C) && issue_qk(0);
        for (int q = 0; q < halves && ok; ++q) {
          if (q + 1 < halves) ok = issue_qk(q + 1);
          const uint32_t gq = n_half + q, gj = g_tile + (dual ? q >> 1 : q);
          const int sv = gj % kStagesV, hf = dual ? q & 1 : s;
          ok = ok && wait_behind_rows(&C.v_full[sv], (gj / kStagesV) & 1, C) && wait_behind_rows(&C.p_full[s][gq & 1], (gq >> 1) & 1, C);
          if (!ok) break;
          tc_fence_after();
          const uint64_t v_desc = smem_desc_advance(v_desc0, static_cast<uint32_t>(sv) * kStageBytes + hf * 16384u);
#pragma unroll
          for (int kk = 0; kk < 4; ++kk)
            mma_bf16_ts(t_o, t_s + (gq & 1) * 64 + kk * 8, smem_desc_advance(v_desc, kk * 4096), idesc_pv, (q > 0 || kk > 0) ? 1u : 0u);
          if (!dual || hf) mma_commit(&C.v_empty[sv]);
          if (q + 2 == halves) mma_commit(&C.o_before[s]);
          if (q + 1 == halves) mma_commit(&C.o_final[s]);
        }
      }
      unit_done();
    }
    g_tile += n_tiles;
    n_half += halves;
    n_before += halves > 1 ? 1 : 0;
  }

  __syncthreads();
  if (C.abort_flag) {
    if (tid == 0) set_status(&P.hdr->status, SS_ERR_TIMEOUT);
    const long long t0 = clock64();                              // let copies and products that are in flight land
    while (clock64() - t0 < 4000000LL) __nanosleep(1000);
    __syncthreads();
  }
  if (warp == kSoftmaxWarps) tmem_dealloc(tmem, kTmemCols);
}

template <bool BLOCKS>
static int32_t launch(const Params& P, cudaStream_t st, int blocks, const CUtensorMap& tk, const CUtensorMap& tv, const CUtensorMap& tq) {
  static bool configured[kDeviceSlots] = {false};
  const int dev_slot = current_device_slot();
  if (dev_slot < 0 || !configured[dev_slot]) {
    if (cudaFuncSetAttribute(draft_umma_kernel<BLOCKS>, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmem) != cudaSuccess) {
      (void)cudaGetLastError();
      return SS_ERR_CUDA;
    }
    if (dev_slot >= 0) configured[dev_slot] = true;
  }
  SS_LAUNCH(draft_umma_kernel<BLOCKS>, blocks, kThreads, kSmem, st, tk, tv, tq, P);
  return SS_OK;
}

int32_t launch_tiles(const Params& P, cudaStream_t st, int blocks) {
  const int64_t rows = ((P.num_pages > 0 ? P.num_pages - 1 : 0) * P.page_stride + (P.Hkv - 1) * P.head_stride) / 128 + kPage;
  if (rows >= 0x7fffffffLL) return SS_ERR_UNSUPPORTED;
  CUtensorMap tk, tv, tq;
  const bool whole = P.page_stride % 1024 == 0 && P.head_stride % 1024 == 0;
  auto encode = [&](CUtensorMap* map, const void* pool) {
    return whole ? tmap::encode_kv_block_bf16(map, pool, static_cast<uint64_t>(rows))
                 : tmap::encode_2d_bf16(map, pool, kDim, static_cast<uint64_t>(rows), kDim * 2, 8);
  };
  if (!encode(&tk, P.k_pool) || !encode(&tv, P.v_pool) ||
      !tmap::encode_q_bf16(&tq, P.q, static_cast<uint64_t>(P.Hq), static_cast<uint64_t>(P.q_rows > 0 ? P.q_rows : 1),
                           static_cast<uint32_t>(P.G), static_cast<uint32_t>(P.tok_per_tile)))
    return SS_ERR_CUDA;
  return whole ? launch<true>(P, st, blocks, tk, tv, tq) : launch<false>(P, st, blocks, tk, tv, tq);
}

}  // namespace draft
}  // namespace ss
