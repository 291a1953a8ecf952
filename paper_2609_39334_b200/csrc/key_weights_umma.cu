// Tensor-core kernel of ss_key_weights (tcgen05 + TMEM + TMA): one block per SM.
//
// A UNIT is a pair of tiles of 128 keys of a node (or its last, single tile) and a kv head, against all query rows that add to them (tokens
// of the paths below the node x heads of the group).  S^T = K Q^T: a key is a lane of TMEM, a query row a column, so that a key's sum of
// exponentials stays in one thread and nothing is exchanged.  A unit's rows go by in STEPS of as many whole tokens as 128 rows hold.  What all units cost,
// in a line, is dealt out evenly: block b of the grid has the steps that start in [b * quota, (b + 1) * quota), so that every block has the
// same work whatever the nodes' lengths and the numbers of their rows.  (Cost of a tile: its rows, and as much as 128 rows for its keys and
// what a unit takes besides.  By steps alone, 302 us instead of 227 for 8 x 8 paths of 64 tokens over 5120 keys; a step more a tile, 149
// instead of 141 for 1024 paths of one token over 1000.)  A unit that several blocks share leaves a sum of each in
// the workspace; the one that comes last adds them up in the order of the blocks, so the result does not depend on who that is.
// Sums: 32 terms at a time in four fp32 accumulators, then a step's, then the unit's, so that thousands of rows lose no more than
// the last bits.
// Roles: four groups of four warps add up exponentials, a group for each tile of a unit and even or odd steps; warp 16 describes units (a ring
// of kUnits); 17 multiplies; 18, 19 load the query rows (TMA, as one box where they lie behind each other, else token by token) and the
// log-sums of even and odd steps; 20, 21 load the keys of even and odd tiles (TMA).  (Rows by cp.async: 460 us where this took 281, 8 x 8 paths of 64 tokens over 5120
// keys: 64 instructions a step, and a fence that waits for them.)  Every wait is bounded (see umma.cuh).
#include "exp2.cuh"
#include "key_weights.cuh"
#include "umma.cuh"

namespace ss {
namespace keyw {

using namespace umma;

constexpr int kSumWarps = 16, kQWarps = 2, kKWarps = 2;
constexpr int kWarpUnits = kSumWarps, kWarpMma = kSumWarps + 1, kWarpQ = kSumWarps + 2, kWarpK = kWarpQ + kQWarps;
constexpr int kThreads = (kWarpK + kKWarps) * 32;
constexpr int kStageBytes = 128 * 256;         // keys or rows: [16 groups of 8][2 halves of 64 dims][8 rows][128 B]
constexpr int kStagesK = 4, kStagesQ = 2;
constexpr int kBuffers = 2;                    // of scores, for each tile: even and odd steps
constexpr int kFewTokens = 8;                  // up to here a step's tokens come one by one, not as a whole step's box
constexpr int kLse = 4;                        // steps whose log-sums there is room for
// (A barrier is waited for by the parity of its phase, so whoever waits must see every phase, and none may end before it has seen the one in
// front: each stage is filled by one warp alone, which waits for it each time.)
static_assert(kStagesQ % kQWarps == 0 && kLse % kQWarps == 0 && kStagesK % kKWarps == 0, "a stage belongs to one warp");
constexpr int kUnits = 8;
constexpr uint32_t kTmemCols = 2 * kBuffers * kCols;
constexpr int kOffQ = kStagesK * kStageBytes, kSmem = kOffQ + kStagesQ * kStageBytes;

struct alignas(16) Unit {
  int valid;                                   // 0: the block's work is done
  int key0, tiles, g;                          // first key, 1 or 2 tiles
  int step0, step1;                            // this block's
  int parts, owner;                            // parts > 1: shared by so many blocks, the first of which is `owner`
  int row0, rows, len, known, hides, order0;   // of the node's Rec
  int pad[2];
  int page[2 * kTilePages];                    // -1: none, or outside the pool (whoever writes a key tells, by whether the node has it)
};
struct Ctrl {
  uint64_t unit_ready[kUnits], unit_free[kUnits];
  uint64_t k_full[kStagesK], k_empty[kStagesK], q_full[kStagesQ], q_empty[kStagesQ];
  uint64_t s_full[2][kBuffers], s_empty[2][kBuffers], l_full[kLse], l_empty[kLse];
  uint64_t other_full[2][2], other_free[2][2];
  uint32_t tmem_slot;
  int abort_flag;
  int steps;                                   // that have been multiplied
  int last[4];
  alignas(16) float minus_lse[kLse][kCols];    // - lse * log2(e) of a step's rows; inf: the row adds nothing
  float other[2][2][kTile];                    // sums on their way from one group of a tile to the other
  Unit unit[kUnits];
};
static_assert(sizeof(Ctrl) + kSmem <= 232448, "shared memory of a block");

__device__ __forceinline__ void tmem_ld16(uint32_t taddr, uint32_t (&r)[16]) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]),
        "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
      : "r"(taddr)
      : "memory");
}
__device__ __forceinline__ void tmem_ld2(uint32_t taddr, uint32_t (&r)[2]) {
  asm volatile("tcgen05.ld.sync.aligned.32x32b.x2.b32 {%0, %1}, [%2];"
               : "=r"(r[0]), "=r"(r[1])
               : "r"(taddr)
               : "memory");
}
__device__ __forceinline__ long long quotient(long long a, long long b) {        // (a division of 64 bits takes some hundred clocks)
  return (a | b) >> 31 ? a / b : static_cast<int>(a) / static_cast<int>(b);
}
// Barrier `id` of 128 threads; whether any of them says so.
__device__ __forceinline__ bool group_any(int id, bool mine) {
  uint32_t any;
  asm volatile(
      "{\n\t.reg .pred p, q;\n\t"
      "setp.ne.u32 p, %1, 0;\n\t"
      "bar.red.or.pred q, %2, 128, p;\n\t"
      "selp.u32 %0, 1, 0, q;\n\t}"
      : "=r"(any)
      : "r"(mine ? 1u : 0u), "r"(id)
      : "memory");
  return any != 0;
}
// The first of a unit's steps that starts at or behind `at` of its cost (see Rec: kTileCost for a tile first, then `per_step` for a step).
__device__ __forceinline__ int step_at(long long at, int tiles, int steps, int per_step) {
  const long long v = (tiles == 1 ? at : (at + 1) >> 1) - kTileCost;
  if (v <= 0) return 0;
  return static_cast<int>(min(quotient(v + per_step - 1, per_step), static_cast<long long>(steps)));
}
// mbar_wait of a role that waits for whole units of others: their steps may take longer than the limit (2500 clocks a step, and as many steps as
// there are query rows), and no wait within a step is without one.  The limit counts from the last step that was seen to begin.
__device__ __forceinline__ bool wait_behind_steps(uint64_t* bar, uint32_t parity, Ctrl& C) {
  if (mbar_try_wait(bar, parity)) return true;
  const volatile int* steps = &C.steps;
  volatile int* abort_flag = &C.abort_flag;
  long long t0 = 0;
  uint32_t spins = 0;
  int seen = 0;
  while (!mbar_try_wait_suspend(bar, parity, 20000u)) {
    if ((++spins & 15u) != 0u) continue;
    if (*abort_flag) return false;
    const int now = *steps;
    if (t0 == 0 || now != seen) {
      t0 = clock64();
      seen = now;
    } else if (clock64() - t0 > kWaitCycles) {
      *abort_flag = 1;
      return false;
    }
  }
  return true;
}
__device__ __forceinline__ int columns_padded(int n) { return n <= 16 ? 16 : (n + 15) & ~15; }

// Exponentials of 32 scores of a key, added up.  A term that is not finite, and one of a row that adds nothing (which comes out as infinity, or
// NaN), makes the sum kLarge or more, or a NaN (see exp2_pair): the step's columns are then added up again by sum_exps_masked<true>.
constexpr float kLarge = 8.507059173e37f;      // 2^126
__device__ __forceinline__ float sum_exps(const uint32_t (&s)[32], const float* minus_lse, float scale) {
  const f32x2 scale2 = pack2(scale, scale);
  f32x2 sum[2] = {pack2(0.f, 0.f), pack2(0.f, 0.f)};
#pragma unroll
  for (int c = 0; c < 32; c += 4) {
    const float4 l = *reinterpret_cast<const float4*>(minus_lse + c);
#pragma unroll
    for (int y = 0; y < 2; ++y) {
      const f32x2 x = fma2(pack2(__uint_as_float(s[c + 2 * y]), __uint_as_float(s[c + 2 * y + 1])), scale2, y ? pack2(l.z, l.w) : pack2(l.x, l.y));
      float e0, e1;
      unpack2(x, e0, e1);
      if (y && c % 16 == 12) {
        exp2_pair(e0, e1, -127.f);
      } else {
        e0 = ex2(e0);
        e1 = ex2(e1);
      }
      sum[y] = add2(sum[y], pack2(e0, e1));
    }
  }
  float a, b, c, d;
  unpack2(sum[0], a, b);
  unpack2(sum[1], c, d);
  return (a + b) + (c + d);
}
// The same for columns [from, to) alone; EXACT: of rows that add nothing, nothing, whatever their scores are, and infinities and NaN as they are.
template <bool EXACT, int N>
__device__ __forceinline__ float sum_exps_masked(const uint32_t (&s)[N], const float* minus_lse, float scale, int from, int to) {
  float sum[2] = {0.f, 0.f};
#pragma unroll
  for (int c = 0; c < N; ++c) {
    const float l = minus_lse[c], e = ex2(fmaf(__uint_as_float(s[c]), scale, l));
    sum[c & 1] += c >= from && c < to && !(EXACT && l == INFINITY) ? e : 0.f;
  }
  return sum[0] + sum[1];
}

// BLOCKS: a page's rows of one head start on 8-row boundaries of the pool and come as one copy, else as four.
template <bool BLOCKS>
__global__ void __launch_bounds__(kThreads, 1)
key_umma_kernel(const __grid_constant__ CUtensorMap tmap_k, const __grid_constant__ CUtensorMap tmap_step,
                const __grid_constant__ CUtensorMap tmap_token, const __grid_constant__ Params P) {
  ss::grid_dependency_enter();
  extern __shared__ __align__(1024) uint8_t smem[];
  __shared__ Ctrl C;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  volatile int* abort_flag = &C.abort_flag;
  if (tid == 0) {
    C.abort_flag = (smem_u32(smem) & 1023u) ? 1 : 0;
    C.steps = 0;
    for (int x = 0; x < kUnits; ++x) { mbar_init(&C.unit_ready[x], 1); mbar_init(&C.unit_free[x], kSumWarps + 1 + kQWarps + kKWarps); }
    for (int x = 0; x < kStagesK; ++x) { mbar_init(&C.k_full[x], 1); mbar_init(&C.k_empty[x], 1); }
    for (int x = 0; x < kStagesQ; ++x) { mbar_init(&C.q_full[x], 1); mbar_init(&C.q_empty[x], 1); }
    for (int w = 0; w < 2; ++w)
      for (int x = 0; x < kBuffers; ++x) { mbar_init(&C.s_full[w][x], 1); mbar_init(&C.s_empty[w][x], 4); }
    for (int x = 0; x < kLse; ++x) { mbar_init(&C.l_full[x], 1); mbar_init(&C.l_empty[x], 8); }
    for (int w = 0; w < 2; ++w)
      for (int x = 0; x < 2; ++x) { mbar_init(&C.other_full[w][x], 4); mbar_init(&C.other_free[w][x], 4); }
    fence_barrier_init();
    prefetch_tensormap(&tmap_k);
    prefetch_tensormap(&tmap_step);
    prefetch_tensormap(&tmap_token);
  }
  if (warp == kWarpMma) tmem_alloc(&C.tmem_slot, kTmemCols);
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = C.tmem_slot;
  const int G = P.G, per_step = kCols / G;     // tokens
  auto tokens_of = [&](int rows, int step) { return min(per_step, rows - step * per_step); };
  uint32_t seq = 0, step = 0;                  // units and steps behind this block (the same in every role)

  if (warp == kWarpUnits) {
    // =================================================== units ===================================================
    const long long total = P.hdr->total, quota = max(quotient(total + gridDim.x - 1, gridDim.x), static_cast<long long>(kLeastQuota)), start = quota * blockIdx.x;
    const long long end = min(start + quota, total);
    const uint32_t pool_pages = static_cast<uint32_t>(min(P.num_pages, static_cast<int64_t>(0x7fffffff)));
    const int n_recs = P.hdr->n_recs, step_cost = (per_step * G + 15) / 16;
    bool ok = true;
    Rec R = {}, N = {}, M = {};                // the unit's node, the next one, the one behind that
    int x = 0, key0 = 0, g = 0;
    long long off = end;                       // of the unit, in tiles of steps
    if (start < end) {
      int lo = 0, hi = n_recs;                                 // recs[lo].off <= start < recs[hi].off
      while (hi - lo > 1) {
        const int stride = (hi - lo + 31) / 32, at = min(lo + (lane + 1) * stride, hi);
        const unsigned over = __ballot_sync(0xffffffffu, at >= hi || P.recs[at].off > start);
        const int first = __ffs(over) - 1;                     // (the last lane's probe is hi)
        hi = min(lo + (first + 1) * stride, hi);
        lo += first * stride;
      }
      x = lo;
      R = P.recs[x];
      if (x + 1 < n_recs) N = P.recs[x + 1];
      if (x + 2 < n_recs) M = P.recs[x + 2];
      const long long rel = start - R.off, row = 2LL * R.cost * P.Hkv;           // of a pair of tiles, all heads
      const int pair = static_cast<int>(quotient(rel, row)), cost = R.cost * min(2, (R.len - pair * 2 * kTile + kTile - 1) / kTile);
      g = static_cast<int>(quotient(rel - pair * row, cost));
      key0 = pair * 2 * kTile;
      off = R.off + pair * row + static_cast<long long>(g) * cost;
    }
    // Pages of a pair of tiles, one a lane
    auto pages_of = [&](const Rec& r, int key) -> int {
      const int at = key / kPage + lane;
      return lane < 2 * kTilePages && r.len > at * kPage ? __ldg(P.node_pages + r.page0 + at) : -1;
    };
    auto pages_behind = [&]() { return key0 + 2 * kTile < R.len ? pages_of(R, key0 + 2 * kTile) : pages_of(N, 0); };
    int page = pages_of(R, key0);
    int ahead = pages_behind();
    while (off < end) {
      const int tiles = min(2, (R.len - key0 + kTile - 1) / kTile);
      const long long cost = static_cast<long long>(R.cost) * tiles;
      const int step0 = step_at(start - off, tiles, R.steps, step_cost), step1 = step_at(end - off, tiles, R.steps, step_cost);
      if (step0 < step1) {
        Unit& U = C.unit[seq % kUnits];
        int parts = 1, owner = 0;
        if (step1 - step0 < R.steps) {
          // (the first and the last block that its cost reaches into may have none of its steps, those between have: see kLeastQuota)
          const long long b0 = quotient(off, quota), b1 = quotient(off + cost - 1, quota);
          owner = static_cast<int>(b0) + (step_at((b0 + 1) * quota - off, tiles, R.steps, step_cost) == 0 ? 1 : 0);
          parts = static_cast<int>(b1) + (step_at(b1 * quota - off, tiles, R.steps, step_cost) < R.steps ? 1 : 0) - owner;
        }
        if (seq >= kUnits) ok = wait_behind_steps(&C.unit_free[seq % kUnits], (seq / kUnits - 1) & 1, C);
        ok = __all_sync(0xffffffffu, ok);
        if (!ok) break;
        if (lane < 2 * kTilePages) U.page[lane] = static_cast<uint32_t>(page) < pool_pages ? page : -1;
        if (lane == 0) {
          int4* to = reinterpret_cast<int4*>(&U);
          to[0] = make_int4(1, key0, tiles, g);
          to[1] = make_int4(step0, step1, parts, owner);
          to[2] = make_int4(R.row0, R.rows, R.len, R.known);
          to[3] = make_int4(R.hides, R.order0, 0, 0);
        }
        __syncwarp();
        if (lane == 0) mbar_arrive(&C.unit_ready[seq % kUnits]);
        ++seq;
      }
      // the next unit
      off += cost;
      if (++g == P.Hkv) {
        g = 0;
        page = ahead;
        key0 += 2 * kTile;
        if (key0 >= R.len) {
          key0 = 0;
          R = N;
          N = M;
          ++x;
          if (x + 2 < n_recs) M = P.recs[x + 2]; else M.len = 0;
        }
        ahead = pages_behind();
      }
    }
    if (seq >= kUnits) ok = wait_behind_steps(&C.unit_free[seq % kUnits], (seq / kUnits - 1) & 1, C) && ok;
    __syncwarp();
    if (lane == 0) { C.unit[seq % kUnits].valid = 0; mbar_arrive(&C.unit_ready[seq % kUnits]); }
  } else if (warp >= kWarpK) {
    // =================================================== keys ====================================================
    const int w = warp - kWarpK;
    uint32_t n_tiles = 0;                      // tiles behind this block
    bool ok = true;
    for (;; ++seq) {
      ok = mbar_wait(&C.unit_ready[seq % kUnits], (seq / kUnits) & 1, abort_flag) && ok;
      ok = __all_sync(0xffffffffu, ok);
      const Unit& U = C.unit[seq % kUnits];
      if (!ok || !U.valid) break;
      const int tiles = U.tiles, keys = U.len - U.key0;
      // (a page outside the pool: any page's keys, which nobody's weights are made of)
      const int row = static_cast<int>((static_cast<int64_t>(max(U.page[lane % (2 * kTilePages)], 0)) * P.page_stride +
                                        static_cast<int64_t>(U.g) * P.head_stride) >> 7);
      __syncwarp();
      if (lane == 0) mbar_arrive(&C.unit_free[seq % kUnits]);
      for (int x = 0; x < tiles; ++x) {
        const uint32_t kt = n_tiles + x;
        if (static_cast<int>(kt % kKWarps) != w) continue;
        const int st = kt % kStagesK, n_pages = min(kTilePages, (keys - x * kTile + kPage - 1) / kPage);
        int rows[kTilePages];
#pragma unroll
        for (int p = 0; p < kTilePages; ++p) rows[p] = __shfl_sync(0xffffffffu, row, x * kTilePages + p);
        if (kt >= kStagesK) ok = wait_behind_steps(&C.k_empty[st], (kt / kStagesK - 1) & 1, C) && ok;
        ok = __all_sync(0xffffffffu, ok);
        if (!ok) break;
        if (elect_one()) {
          uint8_t* dst = smem + st * kStageBytes;
          mbar_arrive_expect_tx(&C.k_full[st], static_cast<uint32_t>(n_pages) * 4096u);
#pragma unroll
          for (int p = 0; p < kTilePages; ++p) {
            if (p < n_pages) {
              if (BLOCKS) {
                tma_load_4d(dst + p * 4096, &tmap_k, 0, 0, 0, rows[p] >> 3, &C.k_full[st]);
              } else {
#pragma unroll
                for (int y = 0; y < 4; ++y) tma_load_2d(dst + p * 4096 + y * 1024, &tmap_k, (y & 1) * 64, rows[p] + (y >> 1) * 8, &C.k_full[st]);
              }
            }
          }
        }
        __syncwarp();
      }
      n_tiles += tiles;
    }
  } else if (warp == kWarpMma) {
    // =================================================== products ================================================
    if (elect_one()) {
      const uint64_t k_desc0 = smem_desc_sw128(smem_u32(smem), 0, 2048), q_desc0 = smem_desc_sw128(smem_u32(smem + kOffQ), 0, 1024);
      uint32_t n_tiles = 0, used[2][kBuffers] = {};        // tiles behind this block; uses of a buffer of scores
      bool ok = true;
      for (; ok; ++seq) {
        ok = mbar_wait(&C.unit_ready[seq % kUnits], (seq / kUnits) & 1, abort_flag);
        const Unit& U = C.unit[seq % kUnits];
        if (!ok || !U.valid) break;
        const int step0 = U.step0, step1 = U.step1, tiles = U.tiles, rows = U.rows;
        mbar_arrive(&C.unit_free[seq % kUnits]);
        for (int j = step0; j < step1 && ok; ++j, ++step) {
          const int qs = step % kStagesQ;
          *const_cast<volatile int*>(&C.steps) = static_cast<int>(step);
          ok = mbar_wait(&C.q_full[qs], (step / kStagesQ) & 1, abort_flag);
          const uint32_t idesc = instr_desc_bf16(128, columns_padded(tokens_of(rows, j) * G), false);
          const uint64_t q_desc = smem_desc_advance(q_desc0, static_cast<uint32_t>(qs) * kStageBytes);
#pragma unroll
          for (int w = 0; w < 2; ++w) {
            if (w >= tiles || !ok) continue;
            const uint32_t kt = n_tiles + w;
            const int ks = kt % kStagesK, buf = step % kBuffers;
            const uint32_t u = buf ? used[w][1]++ : used[w][0]++;
            if (j == step0) ok = mbar_wait(&C.k_full[ks], (kt / kStagesK) & 1, abort_flag);
            if (ok && u > 0) ok = mbar_wait(&C.s_empty[w][buf], (u - 1) & 1, abort_flag);
            if (!ok) continue;
            tc_fence_after();
            const uint64_t k_desc = smem_desc_advance(k_desc0, static_cast<uint32_t>(ks) * kStageBytes);
#pragma unroll
            for (int kk = 0; kk < 8; ++kk)
              mma_bf16_ss(tmem + (w * kBuffers + buf) * kCols, smem_desc_advance(k_desc, (kk >> 2) * 1024 + (kk & 3) * 32),
                          smem_desc_advance(q_desc, (kk >> 2) * 16384 + (kk & 3) * 32), idesc, kk > 0 ? 1u : 0u);
            mma_commit(&C.s_full[w][buf]);
            if (j + 1 == step1) mma_commit(&C.k_empty[ks]);
          }
          if (ok) mma_commit(&C.q_empty[qs]);
        }
        n_tiles += tiles;
      }
    }
    __syncwarp();
  } else if (warp >= kWarpQ) {
    // =================================================== query rows ==============================================
    const int w = warp - kWarpQ;
    bool ok = true;
    for (;; ++seq) {
      ok = mbar_wait(&C.unit_ready[seq % kUnits], (seq / kUnits) & 1, abort_flag) && ok;
      ok = __all_sync(0xffffffffu, ok);
      const Unit& U = C.unit[seq % kUnits];
      if (!ok || !U.valid) break;
      const int step0 = U.step0, step1 = U.step1, g = U.g, row0 = U.row0, rows = U.rows;
      __syncwarp();
      if (lane == 0) mbar_arrive(&C.unit_free[seq % kUnits]);
      for (int j = step0; j < step1; ++j, ++step) {
        if (static_cast<int>(step % kQWarps) != w) continue;
        const int qs = step % kStagesQ, ls = step % kLse, token0 = j * per_step, tokens = tokens_of(rows, j);
        // rows of q by token, rows of lse by column; loads without branches, so that they go out together
        int src[4], dst[4];
#pragma unroll
        for (int x = 0; x < 4; ++x) {
          const int last = max(tokens - 1, 0);
          src[x] = P.rows[row0 + token0 + min(32 * x + lane, last)].x;
          dst[x] = P.rows[row0 + token0 + min((32 * x + lane) / G, last)].y;
        }
        const int src0 = __shfl_sync(0xffffffffu, src[0], 0);
        bool run = true;
        float l[4];
#pragma unroll
        for (int x = 0; x < 4; ++x) {
          const int c = 32 * x + lane;
          run = run && (c >= tokens || src[x] == src0 + c);
          l[x] = -INFINITY;
          if (c < tokens * G) l[x] = __ldg(P.lse + static_cast<int64_t>(dst[x]) * P.Hq + g * G + c % G);
        }
        run = __all_sync(0xffffffffu, run) && (tokens > kFewTokens || tokens == per_step);
        if (step >= kLse) ok = mbar_wait(&C.l_empty[ls], (step / kLse - 1) & 1, abort_flag) && ok;
        if (step >= kStagesQ) ok = mbar_wait(&C.q_empty[qs], (step / kStagesQ - 1) & 1, abort_flag) && ok;
        ok = __all_sync(0xffffffffu, ok);
        if (!ok) break;
        uint8_t* to = smem + kOffQ + qs * kStageBytes;
        if (lane == 0) mbar_arrive_expect_tx(&C.q_full[qs], static_cast<uint32_t>((run ? per_step : tokens) * G) * 256u);
        __syncwarp();
        if (run) {                             // (rows behind the step's last token: nobody adds them up)
          if (elect_one()) {
            tma_load_3d(to, &tmap_step, 0, g * G, src0, &C.q_full[qs]);
            tma_load_3d(to + kStageBytes / 2, &tmap_step, 64, g * G, src0, &C.q_full[qs]);
          }
        } else {
#pragma unroll
          for (int x = 0; x < 4; ++x) {
            const int t = 32 * x + lane;
            if (t < tokens) {
              tma_load_3d(to + t * G * 128, &tmap_token, 0, g * G, src[x], &C.q_full[qs]);
              tma_load_3d(to + kStageBytes / 2 + t * G * 128, &tmap_token, 64, g * G, src[x], &C.q_full[qs]);
            }
          }
        }
#pragma unroll
        for (int x = 0; x < 4; ++x) {
          const float m = -l[x] * 1.4426950408889634f;
          C.minus_lse[ls][32 * x + lane] = l[x] != -INFINITY && m == INFINITY ? 3.402823466e38f : m;
        }
        __syncwarp();
        if (lane == 0) mbar_arrive(&C.l_full[ls]);
      }
    }
  } else {
    // =================================================== sums ====================================================
    const int group = warp >> 2, w = group & 1, p = group >> 1, key = tid & 127;
    const uint32_t t_s = tmem + (static_cast<uint32_t>((warp & 3) * 32) << 16) + (w * kBuffers + p) * kCols;
    const float scale = P.scale_log2;
    uint32_t used = 0;                         // of this group's buffer of scores
    uint32_t n_joined = 0;                     // units whose sums two groups of this tile have joined
    bool ok = true;
    for (;; ++seq) {
      ok = mbar_wait(&C.unit_ready[seq % kUnits], (seq / kUnits) & 1, abort_flag) && ok;
      if (group_any(group + 1, !ok)) break;                      // (a group goes on as a whole, or not)
      const Unit& U = C.unit[seq % kUnits];
      if (!U.valid) break;
      const int step0 = U.step0, step1 = U.step1, g = U.g, len = U.len, i = U.key0 + w * kTile + key, rows = U.rows;
      const bool there = w < U.tiles, both = step1 - step0 > 1;
      const bool writes = ((step + (step1 - step0) - 1) & 1) == p;               // (the last step's group has the unit's sums in the end)
      const int page = there && i < len ? U.page[w * kTilePages + key / kPage] : -1;
      const int64_t to = (static_cast<int64_t>(page) * P.Hkv + g) * kPage + key % kPage;
      const float before = writes && P.weights_in && page >= 0 && i < U.known ? P.weights_in[to] : 0.f;
      const int hidden = max(i - len + U.hides, 0) * G;          // (no more than the rows there are: a product of all keys would not fit)
      float sum = 0.f;
      for (int j = step0; j < step1; ++j, ++step) {
        if (static_cast<int>(step & 1) != p) continue;
        const int ls = step % kLse, n = tokens_of(rows, j) * G;
        ok = mbar_wait(&C.l_full[ls], (step / kLse) & 1, abort_flag) && ok;
        if (there) {
          ok = mbar_wait(&C.s_full[w][p], used & 1, abort_flag) && ok;
          ++used;
          tc_fence_after();
          const float* minus_lse = C.minus_lse[ls];
          const int from = hidden - j * per_step * G;            // the first column that sees the key
          // (from grows with the key: columns in front of the warp's first key's see none of its keys, from its last key's on all)
          const int least = __shfl_sync(0xffffffffu, from, 0), most = __shfl_sync(0xffffffffu, from, 31);
          float part = 0.f;
          int c = max(least, 0) & ~15;
#pragma unroll 1
          for (;;) {
            __syncwarp();
            if (c >= most) {
#pragma unroll 1
              for (; c + 32 <= n; c += 32) {
                uint32_t a[32];
                tmem_ld32(t_s + c, a);
                tmem_wait_ld();
                part += sum_exps(a, minus_lse + c, scale);
              }
            }
            if (c >= n) break;
            uint32_t a[16];
            tmem_ld16(t_s + c, a);
            tmem_wait_ld();
            part += sum_exps_masked<false>(a, minus_lse + c, scale, from - c, n - c);
            c += 16;
          }
          // (Hardly ever; two columns at a time, for what stands here is paid for by all: with sixteen 1024 paths of one token took 142 us, not 138)
          if (__any_sync(0xffffffffu, page >= 0 && !(part < kLarge))) {         // (what lies behind a node's keys may be anything)
            part = 0.f;
#pragma unroll 1
            for (c = 0; c < n; c += 2) {
              uint32_t a[2];
              tmem_ld2(t_s + c, a);
              tmem_wait_ld();
              part += sum_exps_masked<true>(a, minus_lse + c, scale, from - c, n - c);
            }
          }
          tc_fence_before();
          sum += part;
        }
        __syncwarp();
        if (lane == 0) {
          if (there) mbar_arrive(&C.s_empty[w][p]);
          mbar_arrive(&C.l_empty[ls]);
        }
      }
      if (there && both) {                     // the other group's sums come to the last step's
        const int x = n_joined & 1;
        if (!writes) {
          if (n_joined >= 2) ok = mbar_wait(&C.other_free[w][x], (n_joined / 2 - 1) & 1, abort_flag) && ok;
          C.other[w][x][key] = sum;
          __syncwarp();
          if (lane == 0) mbar_arrive(&C.other_full[w][x]);
        } else {
          ok = mbar_wait(&C.other_full[w][x], (n_joined / 2) & 1, abort_flag) && ok;
          sum += C.other[w][x][key];
          __syncwarp();
          if (lane == 0) mbar_arrive(&C.other_free[w][x]);
        }
        ++n_joined;
      }
      if (there && writes) {
        bool write = page >= 0;
        if (!write && i < len) set_status(&P.hdr->status, SS_ERR_BAD_INPUT);
        if (U.parts > 1) {
          const int owner = U.owner, parts = U.parts;
          auto part_of = [&](int b) { return P.part + (static_cast<int64_t>(2 * b + (b == owner ? 1 : 0)) * 2 + w) * kTile + key; };
          *part_of(blockIdx.x) = sum;
          __threadfence();
          (void)group_any(group + 1, false);
          if (key == 0) C.last[group] = atomicAdd(P.arrived + 2 * owner + w, 1) == parts - 1;
          (void)group_any(group + 1, false);
          const bool last = C.last[group] != 0;                  // the others' parts are there
          write = write && last;
          if (last) {
            __threadfence();
            sum = __ldcg(part_of(owner));
            for (int b = owner + 1; b < owner + parts; ++b) sum += __ldcg(part_of(b));
          }
        }
        if (ok && write) {
          P.weights_out[to] = fmaf(P.decay, before, sum);
          if (P.order && i >= U.known) P.order[to] = U.order0 + (i - U.known);
        }
      }
      __syncwarp();
      if (lane == 0) mbar_arrive(&C.unit_free[seq % kUnits]);
    }
  }

  __syncthreads();
  if (C.abort_flag) {
    if (tid == 0) set_status(&P.hdr->status, SS_ERR_TIMEOUT);
    const long long t0 = clock64();                              // let copies and products that are in flight land
    while (clock64() - t0 < 4000000LL) __nanosleep(1000);
    __syncthreads();
  }
  if (warp == kWarpMma) tmem_dealloc(tmem, kTmemCols);
}

template <bool BLOCKS>
static int32_t launch(const Params& P, cudaStream_t st, int blocks, const CUtensorMap& tk, const CUtensorMap& ts, const CUtensorMap& tt) {
  static bool configured[kDeviceSlots] = {false};
  const int dev_slot = current_device_slot();
  if (dev_slot < 0 || !configured[dev_slot]) {
    if (cudaFuncSetAttribute(key_umma_kernel<BLOCKS>, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmem) != cudaSuccess) {
      (void)cudaGetLastError();
      return SS_ERR_CUDA;
    }
    if (dev_slot >= 0) configured[dev_slot] = true;
  }
  SS_LAUNCH(key_umma_kernel<BLOCKS>, blocks, kThreads, kSmem, st, tk, ts, tt, P);
  return SS_OK;
}

int32_t launch_tiles(const Params& P, cudaStream_t st, int blocks) {
  const int64_t rows = ((P.num_pages > 0 ? P.num_pages - 1 : 0) * P.page_stride + (P.Hkv - 1) * P.head_stride) / 128 + kPage;
  if (rows >= 0x7fffffffLL) return SS_ERR_UNSUPPORTED;
  CUtensorMap tk, ts, tt;
  const bool whole = P.page_stride % 1024 == 0 && P.head_stride % 1024 == 0;
  // (without tokens nothing is loaded through the queries' maps)
  const void* q = P.q ? static_cast<const void*>(P.q) : static_cast<const void*>(P.k_pool);
  const uint64_t tokens = static_cast<uint64_t>(P.q_rows > 0 ? P.q_rows : 1);
  if (!(whole ? tmap::encode_kv_block_bf16(&tk, P.k_pool, static_cast<uint64_t>(rows))
              : tmap::encode_2d_bf16(&tk, P.k_pool, kDim, static_cast<uint64_t>(rows), kDim * 2, 8)) ||
      !tmap::encode_q_bf16(&ts, q, static_cast<uint64_t>(P.Hq), tokens, static_cast<uint32_t>(P.G), static_cast<uint32_t>(kCols / P.G)) ||
      !tmap::encode_q_bf16(&tt, q, static_cast<uint64_t>(P.Hq), tokens, static_cast<uint32_t>(P.G), 1))
    return SS_ERR_CUDA;
  return whole ? launch<true>(P, st, blocks, tk, ts, tt) : launch<false>(P, st, blocks, tk, ts, tt);
}

}  // namespace keyw
}  // namespace ss
