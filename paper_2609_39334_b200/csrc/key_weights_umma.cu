// Tensor-core kernel of ss_key_weights (tcgen05 + TMEM + TMA): one block per SM.
//
// A UNIT is a tile of 128 keys of a node and a kv head, against all query rows that add to them (tokens of the paths below the node x
// heads of the group).  S^T = K Q^T: a key is a lane of TMEM, a query row a column, so that a key's sum of exponentials stays in one
// thread and nothing is exchanged.  A unit's rows go by in STEPS of up to 128; the steps of all units in a line are dealt out evenly, block
// b of the grid has steps [b * quota, (b + 1) * quota), so that every block has the same work whatever the nodes' lengths and the
// numbers of their rows.  A unit that several blocks share leaves a sum of each in the workspace; the one that comes last adds them up in
// the order of the blocks, so the result does not depend on who that is.
// Sums: 32 terms at a time in four fp32 accumulators, then a step's, then the unit's, so that thousands of rows lose no more than
// the last bits.
// Roles: warps 0-3, 4-7 add up exponentials, even and odd steps; 8 describes units (a ring of kUnits) and loads keys through TMA; 9
// multiplies; 10-13 gather query rows (cp.async: the rows of a step may lie anywhere) and their log-sums.  Every wait is bounded (see umma.cuh).
#include "exp2.cuh"
#include "key_weights.cuh"
#include "umma.cuh"

namespace ss {
namespace keyw {

using namespace umma;

constexpr int kSumWarps = 8, kQWarps = 4;
constexpr int kWarpK = kSumWarps, kWarpMma = kSumWarps + 1, kWarpQ = kSumWarps + 2;
constexpr int kThreads = (kSumWarps + 2 + kQWarps) * 32;
constexpr int kStageBytes = 128 * 256;         // keys or rows: [16 groups of 8][2 halves of 64 dims][8 rows][128 B]
constexpr int kStagesK = 3, kStagesQ = 3, kBuffers = 4;
constexpr int kUnits = 4;
constexpr uint32_t kTmemCols = kBuffers * kCols;
constexpr int kOffQ = kStagesK * kStageBytes, kSmem = kOffQ + kStagesQ * kStageBytes;

struct Unit {
  int valid;                                   // 0: the block's work is done
  int tile, g;
  int step0, step1;                            // this block's
  int parts, owner, slot;                      // parts > 1: shared by so many blocks, the first of which is `owner`; this one's sums go to `slot`
  int owner_slot;
  Rec R;
  int page[kTilePages];                        // -1: none, or outside the pool
};
struct Ctrl {
  uint64_t unit_ready[kUnits], unit_free[kUnits];
  uint64_t k_full[kStagesK], k_empty[kStagesK], q_full[kStagesQ], q_empty[kStagesQ];
  uint64_t s_full[kBuffers], s_empty[kBuffers], l_full[kBuffers];
  uint64_t other_full[2], other_free[2];
  uint32_t tmem_slot;
  int abort_flag;
  int last[2];
  alignas(16) float minus_lse[kBuffers][kCols];  // - lse * log2(e) of a step's rows; -inf: the row adds nothing
  float other[2][kTile];                       // sums of the odd steps
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
__device__ __forceinline__ void copy_16(uint32_t dst, const void* src, bool there) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(there ? 16 : 0) : "memory");
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
__device__ __forceinline__ int columns_of(const Rec& R, int G, int step) { return min(kCols, R.rows * G - step * kCols); }
__device__ __forceinline__ int columns_padded(int n) { return n <= 16 ? 16 : (n + 15) & ~15; }

// Exponentials of 32 (or 16) scores of a key, added up.
template <int N, bool FAST>
__device__ __forceinline__ float sum_exps(const uint32_t (&s)[N], const float* minus_lse, f32x2 scale2) {
  f32x2 sum[2] = {pack2(0.f, 0.f), pack2(0.f, 0.f)};
#pragma unroll
  for (int c = 0; c < N; c += 4) {
    const float4 l = *reinterpret_cast<const float4*>(minus_lse + c);
#pragma unroll
    for (int y = 0; y < 2; ++y) {
      const f32x2 x = fma2(pack2(__uint_as_float(s[c + 2 * y]), __uint_as_float(s[c + 2 * y + 1])), scale2, y ? pack2(l.z, l.w) : pack2(l.x, l.y));
      float e0, e1;
      unpack2(x, e0, e1);
      if (FAST && (c & 4) && y) {
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
// The same for columns [from, to) alone.
template <int N>
__device__ __forceinline__ float sum_exps_masked(const uint32_t (&s)[N], const float* minus_lse, float scale, int from, int to) {
  float sum[2] = {0.f, 0.f};
#pragma unroll
  for (int c = 0; c < N; ++c) {
    const float e = ex2(fmaf(__uint_as_float(s[c]), scale, minus_lse[c]));
    sum[c & 1] += c >= from && c < to ? e : 0.f;
  }
  return sum[0] + sum[1];
}

// BLOCKS: a page's rows of one head start on 8-row boundaries of the pool and come as one copy, else as four.
template <bool BLOCKS>
__global__ void __launch_bounds__(kThreads, 1)
key_umma_kernel(const __grid_constant__ CUtensorMap tmap_k, const __grid_constant__ Params P) {
  ss::grid_dependency_enter();
  extern __shared__ __align__(1024) uint8_t smem[];
  __shared__ Ctrl C;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  volatile int* abort_flag = &C.abort_flag;
  if (tid == 0) {
    C.abort_flag = (smem_u32(smem) & 1023u) ? 1 : 0;
    for (int x = 0; x < kUnits; ++x) { mbar_init(&C.unit_ready[x], 1); mbar_init(&C.unit_free[x], kSumWarps + 1 + kQWarps); }
    for (int x = 0; x < kStagesK; ++x) { mbar_init(&C.k_full[x], 1); mbar_init(&C.k_empty[x], 1); }
    for (int x = 0; x < kStagesQ; ++x) { mbar_init(&C.q_full[x], kQWarps); mbar_init(&C.q_empty[x], 1); }
    for (int x = 0; x < kBuffers; ++x) { mbar_init(&C.s_full[x], 1); mbar_init(&C.s_empty[x], 4); mbar_init(&C.l_full[x], kQWarps); }
    for (int x = 0; x < 2; ++x) { mbar_init(&C.other_full[x], 4); mbar_init(&C.other_free[x], 4); }
    fence_barrier_init();
    prefetch_tensormap(&tmap_k);
  }
  if (warp == kWarpMma) tmem_alloc(&C.tmem_slot, kTmemCols);
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = C.tmem_slot;
  const int G = P.G;
  uint32_t seq = 0, step = 0;                  // units and steps behind this block (the same in every role)

  if (warp == kWarpK) {
    // =================================================== units and keys ==========================================
    const long long total = P.hdr->total, quota = max(quotient(total + gridDim.x - 1, gridDim.x), 1LL), start = quota * blockIdx.x;
    const long long end = min(start + quota, total);
    const int n_recs = P.hdr->n_recs;
    long long pos = start;
    bool ok = true;
    Rec R = {}, N = {};
    int x = 0, tile = 0, g = 0, step0 = 0, tiles = 0;
    if (pos < end) {
      int lo = 0, hi = n_recs;                                 // recs[lo].off <= pos < recs[hi].off
      while (hi - lo > 1) {
        const int stride = (hi - lo + 31) / 32, at = min(lo + (lane + 1) * stride, hi);
        const unsigned over = __ballot_sync(0xffffffffu, at >= hi || P.recs[at].off > pos);
        const int first = __ffs(over) - 1;                     // (the last lane's probe is hi)
        hi = min(lo + (first + 1) * stride, hi);
        lo += first * stride;
      }
      x = lo;
      R = P.recs[x];
      if (x + 1 < n_recs) N = P.recs[x + 1];
      const long long u = quotient(pos - R.off, R.steps);
      step0 = static_cast<int>(pos - R.off - u * R.steps);
      tile = static_cast<int>(quotient(u, P.Hkv));
      g = static_cast<int>(u - static_cast<long long>(tile) * P.Hkv);
      tiles = (R.len + kTile - 1) / kTile;
    }
    // Pages of a tile, one a lane
    auto pages_of = [&](const Rec& r, int t) -> int {
      const int at = t * kTilePages + lane;
      return lane < kTilePages && r.len > at * kPage ? __ldg(P.node_pages + r.page0 + at) : -1;
    };
    int page = pages_of(R, tile);
    int ahead = tile + 1 < tiles ? pages_of(R, tile + 1) : pages_of(N, 0);
    for (;; ++seq) {
      Unit& U = C.unit[seq % kUnits];
      if (seq >= kUnits) ok = mbar_wait(&C.unit_free[seq % kUnits], (seq / kUnits - 1) & 1, abort_flag) && ok;
      ok = __all_sync(0xffffffffu, ok);
      const bool any = ok && pos < end;
      if (!any) {
        if (lane == 0) { U.valid = 0; mbar_arrive(&C.unit_ready[seq % kUnits]); }
        break;
      }
      const int step1 = static_cast<int>(min(static_cast<long long>(R.steps), step0 + (end - pos)));
      const bool bad = page != -1 && (page < 0 || page >= P.num_pages);
      if (bad) set_status(&P.hdr->status, SS_ERR_BAD_INPUT);
      const int good = bad ? -1 : page;
      if (lane < kTilePages) U.page[lane] = good;
      if (lane == 0) {
        U.valid = 1;
        U.tile = tile;
        U.g = g;
        U.step0 = step0;
        U.step1 = step1;
        U.R = R;
        U.parts = 1;
        U.owner = U.slot = U.owner_slot = 0;
        if (step1 - step0 < R.steps) {
          const long long first = pos - step0, b0 = quotient(first, quota), b1 = quotient(first + R.steps - 1, quota);
          U.parts = static_cast<int>(b1 - b0) + 1;
          U.owner = static_cast<int>(b0);
          U.owner_slot = static_cast<int>(2 * b0) + (first == b0 * quota ? 0 : 1);
          U.slot = b0 == blockIdx.x ? U.owner_slot : 2 * static_cast<int>(blockIdx.x);
        }
      }
      __syncwarp();
      if (lane == 0) mbar_arrive(&C.unit_ready[seq % kUnits]);
      const int st = seq % kStagesK;
      if (seq >= kStagesK) ok = mbar_wait(&C.k_empty[st], (seq / kStagesK - 1) & 1, abort_flag);
      ok = __all_sync(0xffffffffu, ok);
      if (!ok) continue;
      const int n_pages = min(kTilePages, (R.len - tile * kTile + kPage - 1) / kPage);
      // (a page outside the pool: any page's keys, which nobody's weights are made of)
      const int row = static_cast<int>((static_cast<int64_t>(max(good, 0)) * P.page_stride + static_cast<int64_t>(g) * P.head_stride) >> 7);
      int rows[kTilePages];
#pragma unroll
      for (int p = 0; p < kTilePages; ++p) rows[p] = __shfl_sync(0xffffffffu, row, p);
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
      // the next unit
      pos += step1 - step0;
      step0 = 0;
      if (++g == P.Hkv) {
        g = 0;
        page = ahead;
        if (++tile == tiles) {
          tile = 0;
          R = N;
          ++x;
          tiles = (R.len + kTile - 1) / kTile;
          N.len = 0;
          if (x + 1 < n_recs) N = P.recs[x + 1];
        }
        ahead = tile + 1 < tiles ? pages_of(R, tile + 1) : pages_of(N, 0);
      }
    }
  } else if (warp == kWarpMma) {
    // =================================================== products ================================================
    if (elect_one()) {
      const uint64_t k_desc0 = smem_desc_sw128(smem_u32(smem), 0, 2048), q_desc0 = smem_desc_sw128(smem_u32(smem + kOffQ), 0, 2048);
      bool ok = true;
      for (; ok; ++seq) {
        ok = mbar_wait(&C.unit_ready[seq % kUnits], (seq / kUnits) & 1, abort_flag);
        const Unit& U = C.unit[seq % kUnits];
        if (!ok || !U.valid) break;
        const int ks = seq % kStagesK, step0 = U.step0, step1 = U.step1;
        ok = mbar_wait(&C.k_full[ks], (seq / kStagesK) & 1, abort_flag);
        const uint64_t k_desc = smem_desc_advance(k_desc0, static_cast<uint32_t>(ks) * kStageBytes);
        for (int j = step0; j < step1 && ok; ++j, ++step) {
          const int qs = step % kStagesQ, buf = step % kBuffers;
          ok = mbar_wait(&C.q_full[qs], (step / kStagesQ) & 1, abort_flag);
          if (ok && step >= kBuffers) ok = mbar_wait(&C.s_empty[buf], (step / kBuffers - 1) & 1, abort_flag);
          if (!ok) break;
          tc_fence_after();
          const uint32_t idesc = instr_desc_bf16(128, columns_padded(columns_of(U.R, G, j)), false);
          const uint64_t q_desc = smem_desc_advance(q_desc0, static_cast<uint32_t>(qs) * kStageBytes);
#pragma unroll
          for (int kk = 0; kk < 8; ++kk)
            mma_bf16_ss(tmem + buf * kCols, smem_desc_advance(k_desc, (kk >> 2) * 1024 + (kk & 3) * 32),
                        smem_desc_advance(q_desc, (kk >> 2) * 1024 + (kk & 3) * 32), idesc, kk > 0 ? 1u : 0u);
          mma_commit(&C.s_full[buf]);
          mma_commit(&C.q_empty[qs]);
          if (j + 1 == step1) mma_commit(&C.k_empty[ks]);
        }
        mbar_arrive(&C.unit_free[seq % kUnits]);
      }
    }
    __syncwarp();
  } else if (warp >= kWarpQ) {
    // =================================================== query rows ==============================================
    const int w = warp - kWarpQ;
    bool ok = true;
    auto landed = [&](uint32_t s) {            // this warp's rows of step s are in shared memory
      fence_proxy_async_smem();
      __syncwarp();
      if (lane == 0) mbar_arrive(&C.q_full[s % kStagesQ]);
    };
    for (;; ++seq) {
      ok = mbar_wait(&C.unit_ready[seq % kUnits], (seq / kUnits) & 1, abort_flag) && ok;
      ok = __all_sync(0xffffffffu, ok);
      const Unit& U = C.unit[seq % kUnits];
      if (!ok || !U.valid) break;
      const int step0 = U.step0, step1 = U.step1, g = U.g, row0 = U.R.row0, all = U.R.rows * G;
      for (int j = step0; j < step1; ++j, ++step) {
        const int qs = step % kStagesQ, buf = step % kBuffers;
        const int n = min(kCols, all - j * kCols), padded = columns_padded(n);
        // this lane's row
        const int c = 32 * w + lane;
        int row = -1;
        int64_t lse_at = -1;
        if (c < n) {
          const int t = (j * kCols + c) / G, h = g * G + (j * kCols + c) - t * G;
          const int2 r = P.rows[row0 + t];
          row = r.x * P.Hq + h;
          lse_at = static_cast<int64_t>(r.y) * P.Hq + h;
        }
        if (step >= kStagesQ) ok = mbar_wait(&C.q_empty[qs], (step / kStagesQ - 1) & 1, abort_flag) && ok;
        ok = __all_sync(0xffffffffu, ok);
        if (!ok) break;
        const uint32_t base = smem_u32(smem + kOffQ + qs * kStageBytes);
        if (32 * w < padded) {
          const int ch = lane & 15;
#pragma unroll
          for (int y = 0; y < 16; ++y) {
            const int r = 2 * y + (lane >> 4), at = 32 * w + r;
            const int of = __shfl_sync(0xffffffffu, row, r);
            if (at < padded)
              copy_16(base + (at >> 3) * 2048 + (ch >> 3) * 1024 + (at & 7) * 128 + (((ch & 7) ^ (at & 7)) << 4),
                      P.q + static_cast<int64_t>(max(of, 0)) * kDim + ch * 8, of >= 0);
          }
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
        float l = -INFINITY;
        if (lse_at >= 0) {
          const float lse = __ldg(P.lse + lse_at);
          l = lse == -INFINITY ? -INFINITY : -lse * 1.4426950408889634f;
        }
        if (step >= kBuffers) ok = mbar_wait(&C.s_empty[buf], (step / kBuffers - 1) & 1, abort_flag) && ok;
        C.minus_lse[buf][c] = l;
        __syncwarp();
        if (lane == 0) mbar_arrive(&C.l_full[buf]);
        if (step > 0) {
          asm volatile("cp.async.wait_group 1;" ::: "memory");
          landed(step - 1);
        }
      }
      __syncwarp();
      if (lane == 0) mbar_arrive(&C.unit_free[seq % kUnits]);
    }
    asm volatile("cp.async.wait_group 0;" ::: "memory");
    if (ok && step > 0) landed(step - 1);
  } else {
    // =================================================== sums ====================================================
    const int s = warp >> 2, key = tid & 127;
    const uint32_t lanes = static_cast<uint32_t>((warp & 3) * 32) << 16;
    const float scale = P.scale_log2;
    const f32x2 scale2 = pack2(scale, scale);
    uint32_t n_shared = 0;                     // units with sums of both groups behind this one
    bool ok = true;
    for (;; ++seq) {
      ok = mbar_wait(&C.unit_ready[seq % kUnits], (seq / kUnits) & 1, abort_flag) && ok;
      if (group_any(s + 1, !ok)) break;                          // (a group goes on as a whole, or not)
      const Unit& U = C.unit[seq % kUnits];
      if (!U.valid) break;
      const int step0 = U.step0, step1 = U.step1, g = U.g, i = U.tile * kTile + key, len = U.R.len;
      const bool both = step1 - step0 > 1;
      const bool mine = both ? s == 0 : static_cast<int>(step & 1) == s;         // this group writes the unit's sums
      const int page = i < len ? U.page[key / kPage] : -1;
      const float before = mine && page >= 0 ? load_before(P, U.R, page, g, i) : 0.f;
      const int hidden = (i - len + U.R.hides) * G, most_hidden = (min(len, (U.tile + 1) * kTile) - 1 - len + U.R.hides) * G;
      float sum = 0.f;
      for (int j = step0; j < step1; ++j, ++step) {
        if (static_cast<int>(step & 1) != s) continue;
        const int buf = step % kBuffers, n = columns_of(U.R, G, j), padded = columns_padded(n);
        const int from = hidden - j * kCols;                     // the first column that sees the key
        const bool masked = n != padded || most_hidden > j * kCols;
        ok = mbar_wait(&C.l_full[buf], (step / kBuffers) & 1, abort_flag) && ok;
        ok = mbar_wait(&C.s_full[buf], (step / kBuffers) & 1, abort_flag) && ok;
        tc_fence_after();
        const uint32_t t_s = tmem + lanes + buf * kCols;
        const float* minus_lse = C.minus_lse[buf];
        float part = 0.f;
        __syncwarp();
        if (!masked && n == kCols) {
          uint32_t a[32], b[32];
          tmem_ld32(t_s, a);
          tmem_wait_ld();
          tmem_pin32(a);
          tmem_ld32(t_s + 32, b);
          part += sum_exps<32, true>(a, minus_lse, scale2);
          tmem_wait_ld();
          tmem_pin32(b);
          tmem_ld32(t_s + 64, a);
          part += sum_exps<32, true>(b, minus_lse + 32, scale2);
          tmem_wait_ld();
          tmem_pin32(a);
          tmem_ld32(t_s + 96, b);
          part += sum_exps<32, true>(a, minus_lse + 64, scale2);
          tmem_wait_ld();
          tmem_pin32(b);
          part += sum_exps<32, true>(b, minus_lse + 96, scale2);
        } else {
          for (int c = 0; c < padded; c += 16) {
            uint32_t a[16];
            __syncwarp();
            tmem_ld16(t_s + c, a);
            tmem_wait_ld();
            part += masked ? sum_exps_masked<16>(a, minus_lse + c, scale, from - c, n - c) : sum_exps<16, false>(a, minus_lse + c, scale2);
          }
        }
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(&C.s_empty[buf]);
        sum += part;
      }
      if (both) {                              // the odd group's (or the second step's) sums come to the even one's
        const int x = n_shared & 1;
        if (s == 1) {
          if (n_shared >= 2) ok = mbar_wait(&C.other_free[x], (n_shared / 2 - 1) & 1, abort_flag) && ok;
          C.other[x][key] = sum;
          __syncwarp();
          if (lane == 0) mbar_arrive(&C.other_full[x]);
        } else {
          ok = mbar_wait(&C.other_full[x], (n_shared / 2) & 1, abort_flag) && ok;
          sum += C.other[x][key];
          __syncwarp();
          if (lane == 0) mbar_arrive(&C.other_free[x]);
        }
        ++n_shared;
      }
      if (mine) {
        if (U.parts == 1) {
          if (ok && page >= 0) store_key(P, U.R, page, g, i, sum, before);
        } else {
          P.part[U.slot * kTile + key] = sum;
          __threadfence();
          asm volatile("bar.sync %0, 128;" ::"r"(s + 1) : "memory");
          if (key == 0) C.last[s] = atomicAdd(P.arrived + U.owner, 1) == U.parts - 1;
          asm volatile("bar.sync %0, 128;" ::"r"(s + 1) : "memory");
          if (C.last[s]) {                     // the others' parts are there
            __threadfence();
            float all = __ldcg(P.part + U.owner_slot * kTile + key);
            for (int b = 1; b < U.parts; ++b) all += __ldcg(P.part + 2 * (U.owner + b) * kTile + key);
            if (ok && page >= 0) store_key(P, U.R, page, g, i, all, before);
          }
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
static int32_t launch(const Params& P, cudaStream_t st, int blocks, const CUtensorMap& tk) {
  static bool configured[kDeviceSlots] = {false};
  const int dev_slot = current_device_slot();
  if (dev_slot < 0 || !configured[dev_slot]) {
    if (cudaFuncSetAttribute(key_umma_kernel<BLOCKS>, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmem) != cudaSuccess) {
      (void)cudaGetLastError();
      return SS_ERR_CUDA;
    }
    if (dev_slot >= 0) configured[dev_slot] = true;
  }
  SS_LAUNCH(key_umma_kernel<BLOCKS>, blocks, kThreads, kSmem, st, tk, P);
  return SS_OK;
}

int32_t launch_tiles(const Params& P, cudaStream_t st, int blocks) {
  const int64_t rows = ((P.num_pages > 0 ? P.num_pages - 1 : 0) * P.page_stride + (P.Hkv - 1) * P.head_stride) / 128 + kPage;
  if (rows >= 0x7fffffffLL) return SS_ERR_UNSUPPORTED;
  CUtensorMap tk;
  const bool whole = P.page_stride % 1024 == 0 && P.head_stride % 1024 == 0;
  if (!(whole ? tmap::encode_kv_block_bf16(&tk, P.k_pool, static_cast<uint64_t>(rows))
              : tmap::encode_2d_bf16(&tk, P.k_pool, kDim, static_cast<uint64_t>(rows), kDim * 2, 8)))
    return SS_ERR_CUDA;
  return whole ? launch<true>(P, st, blocks, tk) : launch<false>(P, st, blocks, tk);
}

}  // namespace keyw
}  // namespace ss
