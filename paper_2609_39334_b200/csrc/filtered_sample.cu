// ss_filtered_sample: draws behind temperature, top-k, top-p and min-p.
//
// The filters keep a prefix of the tokens in the order (logit descending, index ascending), so all of them together are one BORDER:
// a logit `key` and how many of the tokens that have exactly this logit are kept, the lowest indices first.  top-k gives one by
// counting, top-p one by adding up probabilities, min-p one by a bound on the logit; the least of the three holds.  A draw then
// goes by the running sum over the kept tokens in index order.  Logits are compared as order-preserving integers (bf16 ones are
// widened: exact); probabilities are fp64 relative to the row's maximum.
#include <math.h>

#include "common.cuh"

namespace ss {
namespace filtered {

constexpr int kMaxVocab = 2097152;
constexpr int kThreads = 512, kWarps = kThreads / 32;          // of a block that goes through whole rows
constexpr int kSeg = 512;                                      // tokens of a segment (a sum each, for the draws)
constexpr uint32_t kNegInf = 0x007fffffu;                      // key of -inf; those of NaN are below it or above kPosInf
constexpr uint32_t kPosInf = 0xff800000u;

struct Args {
  const void* logits;
  const int64_t* draw_offsets;
  const float *uniforms, *temperature, *top_p, *min_p;
  const int32_t* top_k;
  int32_t* tokens_out;
  int64_t* seq_out;
  int32_t* kept_out;
  int64_t row_stride;
  float temperature_all, top_p_all, min_p_all;
  int top_k_all;
  int n_seq, vocab;
  int32_t* marks;                              // [n_seq]: rows that the list is not enough for
  int whole_rows;                              // rows of one block each; the others are split into
  int parts;                                   // so many parts
  struct Part* part;                           // [blocks]
};
struct RowParams {
  float temperature, top_p, min_p;
  int top_k;
};
__device__ __forceinline__ RowParams row_params(const Args& A, int s) {
  RowParams r;
  r.temperature = A.temperature ? __ldg(A.temperature + s) : A.temperature_all;
  r.top_p = A.top_p ? __ldg(A.top_p + s) : A.top_p_all;
  r.min_p = A.min_p ? __ldg(A.min_p + s) : A.min_p_all;
  r.top_k = A.top_k ? __ldg(A.top_k + s) : A.top_k_all;
  return r;
}

// Order-preserving integer of a logit and back; -0 counts as +0.
__device__ __forceinline__ uint32_t key_of(float x) {
  const uint32_t u = __float_as_uint(x + 0.f);
  return u ^ (static_cast<uint32_t>(static_cast<int32_t>(u) >> 31) | 0x80000000u);
}
__device__ __forceinline__ float logit_of(uint32_t k) {
  return __uint_as_float(k & 0x80000000u ? k ^ 0x80000000u : ~k);
}
template <bool HALF>
__device__ __forceinline__ float load_logit(const void* row, int v) {
  if (HALF) return __uint_as_float(static_cast<uint32_t>(__ldg(static_cast<const unsigned short*>(row) + v)) << 16);
  return __ldg(static_cast<const float*>(row) + v);
}
template <bool HALF>
__device__ __forceinline__ const void* row_of(const Args& A, int s) {
  return static_cast<const char*>(A.logits) + static_cast<int64_t>(s) * A.row_stride * (HALF ? 2 : 4);
}

__device__ __forceinline__ unsigned long long entry_of(float x, int v) {
  return (static_cast<unsigned long long>(key_of(x)) << 32) | static_cast<uint32_t>(v);
}

struct Border {
  uint32_t key;                                // tokens above it are kept,
  int ties;                                    // and so many with exactly this key
};
__device__ __forceinline__ bool less(const Border& a, const Border& b) { return a.key > b.key || (a.key == b.key && a.ties < b.ties); }

// e_v of a row: K = the integer nearest to 128 x for x = (logit - max) log2(e) / T, r = 128 x - K, 2^(K / 128) from a table of 128
// entries and an integer addition to the exponent, 2^(r / 128) by a polynomial of degree 4 (as the branch sampler's; after Tang,
// "Table-driven implementation of the exponential function in IEEE floating-point arithmetic", ACM TOMS 15, 1989): 2e-16 of itself, in
// a sixth of the instructions of exp.  Terms below 2^-1000 count as that.
constexpr int kTable = 128;
struct Term {
  double max, c, lowest;                       // c: 128 log2(e) / T
  const double* table;                         // shared memory
  __device__ __forceinline__ double operator()(float x) const {
    constexpr double a1 = 0.005415212348124257, a2 = 1.466226238764014e-05, a3 = 2.6466431340771855e-08, a4 = 3.5830331985890313e-11;
    constexpr double kRound = 6755399441055744.0;              // 1.5 * 2^52
    const double d = fmax(static_cast<double>(x) - max, lowest);
    const double k = fma(d, c, kRound), r = fma(d, c, kRound - k);
    const int bits = __double2loint(k);
    const double t0 = table[bits & (kTable - 1)];
    const double t = __hiloint2double(__double2hiint(t0) + ((bits >> 7) << 20), __double2loint(t0));
    return fma(t * r, fma(fma(fma(a4, r, a3), r, a2), r, a1), t);
  }
};
__device__ __forceinline__ Term term_of(float max, float temperature, const double* table) {
  Term e;
  e.max = static_cast<double>(max);
  e.c = kTable * 1.4426950408889634 / static_cast<double>(temperature);
  e.lowest = -1000.0 * kTable / e.c;
  e.table = table;
  return e;
}
__device__ __forceinline__ void make_table(double* table) {    // (whole block; a barrier has to follow)
  if (threadIdx.x < kTable) table[threadIdx.x] = exp2(threadIdx.x * (1.0 / kTable));
}
// The smallest key whose token passes min-p (e does not fall with the logit): from the logarithm, then by the definition itself, in
// doubling steps and by halves - a step is enough but where a rounded e^x is the same for many logits.
__device__ __noinline__ uint32_t min_p_key(const Term& e, float temperature, float min_p, uint32_t max_key) {
  const double m = static_cast<double>(min_p);
  if (!(m > 0.0)) return kNegInf + 1;
  if (m > 1.0) return max_key;                 // (at least one token)
  const double x = e.max + static_cast<double>(temperature) * log(m);
  uint32_t k = x > -3.4e38 ? key_of(static_cast<float>(x)) : kNegInf + 1;
  k = min(max(k, kNegInf + 1), max_key);
  uint32_t lo = kNegInf, hi = max_key;         // lo does not pass, hi does
  if (k == hi || e(logit_of(k)) >= m) {
    hi = k;
    for (uint32_t step = 1; hi - lo > step; step *= 2) {
      if (!(e(logit_of(hi - step)) >= m)) { lo = hi - step; break; }
      hi -= step;
    }
  } else {
    lo = k;
    for (uint32_t step = 1; hi - lo > step; step *= 2) {
      if (e(logit_of(lo + step)) >= m) { hi = lo + step; break; }
      lo += step;
    }
  }
  while (hi - lo > 1) {
    const uint32_t mid = lo + (hi - lo) / 2;
    if (e(logit_of(mid)) >= m) hi = mid; else lo = mid;
  }
  return hi;
}

__device__ __forceinline__ double warp_sum_d(double v) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}
__device__ __forceinline__ double warp_scan_d(double v, int lane) {
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const double up = __shfl_up_sync(0xffffffffu, v, o);
    if (lane >= o) v += up;
  }
  return v;
}

// ---- most rows: one pass over the row, the rest on a short list --------------------------------------------------------------------
// What is kept is nearly always among the few largest logits, so one pass collects those above a THRESHOLD in shared memory (the
// list) and, where top-p is over the whole row, adds up all terms in fp32 (with a bound: quick_error).  The threshold comes from a
// sample spread over the row: of the maxima of 64 groups of n sampled tokens a share e^(-n f) lies below the value that a share f of
// the row exceeds.  Nothing rests on it: a border found on the list is the row's if it does not lie below the threshold, and where
// the list is too short or too long, or a sum comes too close to top-p's target to tell, the row is marked and made again by the
// kernel behind this one.  (Short rows are on the list as a whole.)
// On the list: one histogram to the at most 512 candidates for what is kept, those in order, a thread each, and every filter's end by
// a running sum (fp64).  Where more are kept: borders by find_on_list, the kept ones sorted by index.  A draw is a thread's.
// Two blocks an SM, so that one is in its pass while the other is on its list.  In the pass every lane has the next four vectors on
// their way to shared memory while it works on the last four: 16 warps then ask for as much as an SM's share of the bandwidth takes
// (straight into registers, with room for four vectors, a block got 11.8 bytes a clock, alone or beside the other one).  Rows that are
// left over behind whole rounds, one a block, are split over the blocks: each hands its part's list over in the workspace, the next
// kernel puts them together.
constexpr int kListThreads = 512, kListWarps = kListThreads / 32;
constexpr int kCap = 8192;                                     // entries of a list
constexpr int kBins = 512;
constexpr int kGroups = 64;                                    // of sampled tokens: 8 lanes each
constexpr double kFix = 1125899906842624.0;                    // 2^50: kCap terms of at most 1 stay below 2^63
constexpr double kFixError = 1e-11;                            // kCap * 2^-51 of the largest term, and the sums' own roundings
constexpr float kLowest = -3.4028235e38f;

struct RowBuffer {                                             // a row between the pass and its list
  unsigned long long list[kCap];                               // key, token; then token, key; then running sums
  unsigned n;                                                  // entries offered to the list
  float low, base;                                             // threshold; the quick sum is relative to 2^base
  bool skip;                                                   // nothing to do
  int64_t d0, d1;
  RowParams R;
  float max[kListWarps];
  double sum[kListWarps];
};
struct ListShared {
  double table[kTable];
  union {
    uint32_t token[kCap];
    uint4 ring[kListWarps][4][32];                             // in the pass
  };
  unsigned long long order[kListThreads];                      // candidates in order; running sums of stretches of kept ones
  unsigned count[kBins];
  unsigned part[3][kBins];                                     // a sum of terms in fixed point, see add_fixed
  double d[kListWarps];
  float group[kGroups];
  unsigned bin, moved;
  uint32_t min_key;                                            // of the list
  unsigned long long above, in_bin, all;
  unsigned long long u[kListWarps];
  double z;
};
constexpr int kPartCap = kCap / 2;                             // entries of a part's list: twice what begin_row wants of one of two parts
struct Part {                                                  // of a row, in the workspace
  unsigned n;
  float low, base, max;
  double sum;
  unsigned long long list[kPartCap];
};

// The kListThreads threads that work on a list.
__device__ __forceinline__ void list_sync() { asm volatile("bar.sync 1, %0;" ::"n"(kListThreads) : "memory"); }
__device__ __forceinline__ int list_count(bool p) {
  int n;
  asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %1, 0;\n\tbar.red.popc.u32 %0, 1, %2, p;\n\t}" : "=r"(n) : "r"(static_cast<int>(p)), "n"(kListThreads) : "memory");
  return n;
}

// Sum of the first `warp` of kListWarps values.
template <typename T>
__device__ __forceinline__ T warps_before(const T* per_warp, int warp, int lane) {
  T v = lane < warp ? per_warp[lane] : T(0);
#pragma unroll
  for (int o = 8; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return __shfl_sync(0xffffffffu, v, 0);
}
// Inclusive sum over the block's threads (a barrier inside; `per_warp` is free again behind the next one).
__device__ __forceinline__ double block_scan_d(double* per_warp, double v, int warp, int lane) {
  const double incl = warp_scan_d(v, lane);
  if (lane == 31) per_warp[warp] = incl;
  list_sync();
  return incl + warps_before(per_warp, warp, lane);
}

// Terms in fixed point (at most 2^50) by 17 bits of them at a time: kCap of those fit 32 bits, which shared memory adds up by itself
// (64 bits are a loop of compare-and-swaps: 0.27 ms a list where a bin has many).
__device__ __forceinline__ void add_fixed(ListShared& S, int bin, unsigned long long m) {
  atomicAdd(&S.part[0][bin], static_cast<unsigned>(m) & 0x1ffffu);
  atomicAdd(&S.part[1][bin], static_cast<unsigned>(m >> 17) & 0x1ffffu);
  atomicAdd(&S.part[2][bin], static_cast<unsigned>(m >> 34));
}
__device__ __forceinline__ unsigned long long take_fixed(ListShared& S, int bin) {   // and leaves 0
  const unsigned long long m = S.part[0][bin] + (static_cast<unsigned long long>(S.part[1][bin]) << 17) +
                               (static_cast<unsigned long long>(S.part[2][bin]) << 34);
  S.part[0][bin] = S.part[1][bin] = S.part[2][bin] = 0;
  return m;
}

struct Found {                                                 // where a running count or sum over falling keys reaches its target
  bool there;
  uint32_t key;
  unsigned long long above, at_key;                            // over the larger keys, over this one
};
// `entry(i, k)`: key of list entry i, and whether it counts; `weight(key)`: what it counts for.  Whole block; keys of [lo, hi].  The
// bins are zero before and after.
template <bool MASS, typename Entry, typename Weight>
__device__ __forceinline__ Found find_on_list(ListShared& S, int n, uint32_t lo, uint32_t hi, unsigned long long target, Entry entry, Weight weight) {
  static_assert(kBins == kListThreads, "a bin per thread");
  const int tid = threadIdx.x % kListThreads, lane = tid & 31, warp = tid >> 5;
  unsigned long long above = 0;
  for (;;) {
    const uint32_t range = hi - lo;
    const int shift = range < kBins ? 0 : 32 - __clz(range) - 9;
    for (int i = tid; i < n; i += kListThreads) {
      uint32_t k;
      if (entry(i, k) && k >= lo && k <= hi) {
        const uint32_t b = (k - lo) >> shift;
        if (MASS) add_fixed(S, b, weight(k));
        else atomicAdd(&S.count[b], 1u);
      }
    }
    list_sync();
    const int bin = kBins - 1 - tid;                           // from the top
    const unsigned long long here = MASS ? take_fixed(S, bin) : static_cast<unsigned long long>(S.count[bin]);
    if (!MASS) S.count[bin] = 0;
    unsigned long long incl = here;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const unsigned long long up = __shfl_up_sync(0xffffffffu, incl, o);
      if (lane >= o) incl += up;
    }
    if (lane == 31) S.u[warp] = incl;
    if (tid == 0) S.bin = kBins;
    list_sync();
    incl += warps_before(S.u, warp, lane) + above;
    if (incl >= target && incl - here < target) { S.bin = bin; S.above = incl - here; S.in_bin = here; }
    if (tid == kListThreads - 1) S.all = incl;
    list_sync();
    const uint32_t at = S.bin;
    if (at == kBins) return Found{false, lo, S.all, 0};
    above = S.above;
    lo += at << shift;
    if (shift == 0) return Found{true, lo, above, S.in_bin};
    hi = min(hi, lo + ((1u << shift) - 1u));
  }
}

typedef unsigned long long f32x2;
__device__ __forceinline__ f32x2 pack2(float a, float b) { f32x2 r; asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b)); return r; }
__device__ __forceinline__ void unpack2(f32x2 v, float& a, float& b) { asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(v)); }
__device__ __forceinline__ f32x2 fma2(f32x2 a, f32x2 b, f32x2 c) { f32x2 r; asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c)); return r; }
__device__ __forceinline__ f32x2 add2(f32x2 a, f32x2 b) { f32x2 r; asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b)); return r; }
__device__ __forceinline__ f32x2 both(float a) { return pack2(a, a); }
__device__ __forceinline__ float ex2(float x) { float y; asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x)); return y; }
__device__ __forceinline__ float max3_nan(float a, float b, float c) {
  float r;
  asm("max.NaN.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
  return r;
}
// x[i], i from 0 to 15
__device__ __forceinline__ float pick16(const float (&x)[16], int i) {
  float a[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) a[j] = i & 8 ? x[j + 8] : x[j];
#pragma unroll
  for (int j = 0; j < 4; ++j) a[j] = i & 4 ? a[j + 4] : a[j];
  a[0] = i & 2 ? a[2] : a[0];
  a[1] = i & 2 ? a[3] : a[1];
  return i & 1 ? a[1] : a[0];
}
__device__ __forceinline__ float max_nan(float a, float b) {
  float r;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
  return r;
}

// Logits of one 16-byte vector.
template <bool HALF>
__device__ __forceinline__ void unpack(const uint4& u, float* x) {
  const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if (HALF) {
      x[2 * i] = __uint_as_float(w[i] << 16);
      x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
    } else {
      x[i] = __uint_as_float(w[i]);
    }
  }
}

// Many candidates, or an end that is none of a few: borders by find_on_list, the kept ones in the order of their indices.  Returns how
// many are kept (S.token: their places on the list); 0: the list cannot tell.
__device__ __noinline__ int wide_list(ListShared& S, unsigned long long* list, const RowParams R, const Term e, int V, int m_list, uint32_t low_key, uint32_t max_key, bool limit,
                                      bool greedy, bool whole, bool add_up, double total_quick, double error_quick) {
  const int tid = threadIdx.x % kListThreads, lane = tid & 31, warp = tid >> 5;
  bool sure = true;
  list_sync();
  Border border{kNegInf, 0};
  bool known = false;
  auto take = [&](const Border& b) {
    if (!known || less(b, border)) border = b;
    known = true;
  };
  auto by_key = [&](int i, uint32_t& k) { k = static_cast<uint32_t>(list[i] >> 32); return true; };
  auto fixed = [&](uint32_t k) { return __double2ull_rn(e(logit_of(k)) * kFix); };
  auto one = [](uint32_t) { return 1ull; };
  if (greedy) {
    take(Border{max_key, 1});
  } else {
    bool k_known = !limit;
    Border by_count{low_key, 0x7fffffff};
    if (limit) {
      const Found f = find_on_list<false>(S, m_list, low_key, max_key, static_cast<unsigned long long>(R.top_k), by_key, one);
      if (f.there) {
        const unsigned long long ties = R.top_k - f.above;
        by_count = Border{f.key, ties < f.at_key ? static_cast<int>(ties) : 0x7fffffff};
        take(by_count);
        k_known = true;
      }
    }
    const uint32_t size_key = min_p_key(e, R.temperature, R.min_p, max_key);
    const bool by_m = R.min_p > 0.f;
    if (by_m && (whole || size_key >= low_key)) take(R.min_p > 1.f ? Border{max_key, 1} : Border{max(size_key, low_key), 0x7fffffff});
    if (R.top_p < 1.f) {
      if (!k_known || (!limit && !whole && !add_up)) {
        sure = false;                                          // (the sum that top-p is a share of is not known)
      } else {
        double total, error = kFixError;
        if (limit || whole) {
          // (a sum over the list: everything down to the border by count, or to the end)
          const Found f = find_on_list<true>(S, m_list, by_count.key, max_key, ~0ull, by_key, fixed);
          double sum = static_cast<double>(f.above);
          if (by_count.ties != 0x7fffffff) {
            const unsigned long long each = fixed(by_count.key);
            // (the list holds all that have the border's key: take those off that are not kept)
            unsigned long long same = 0;
            for (int i = tid; i < m_list; i += kListThreads) same += static_cast<uint32_t>(list[i] >> 32) == by_count.key ? 1 : 0;
#pragma unroll
            for (int o = 16; o > 0; o >>= 1) same += __shfl_xor_sync(0xffffffffu, same, o);
            list_sync();
            if (lane == 0) S.d[warp] = static_cast<double>(same);
            list_sync();
            double all = 0.0;
#pragma unroll
            for (int w = 0; w < kListWarps; ++w) all += S.d[w];
            sum -= (all - static_cast<double>(by_count.ties)) * static_cast<double>(each);
          }
          total = sum / kFix;
        } else {
          total = total_quick;
          error = error_quick;
        }
        const double target = static_cast<double>(R.top_p) * total;
        const double t_lo = target * (1.0 - error) * kFix, t_hi = target * (1.0 + error) * kFix;
        if (!(t_hi < 9.0e18)) {
          sure = false;
        } else {
          const unsigned long long need = t_lo > 1.0 ? __double2ull_ru(t_lo) : 1ull;
          const Found f = find_on_list<true>(S, m_list, by_count.key, max_key, need, by_key, fixed);
          if (!f.there) {
            sure = known && !limit && !whole && border.key >= low_key;    // below the list: another border is on it
          } else {
            const unsigned long long each = max(fixed(f.key), 1ull);
            const unsigned long long ties = (need - f.above + each - 1) / each;
            const Border by_sum{f.key, ties * each < f.at_key ? static_cast<int>(ties) : 0x7fffffff};
            const bool clear = static_cast<double>(f.above + ties * each) >= t_hi;
            if (clear) take(by_sum);
            else if (!known || !less(border, by_sum)) sure = false;
          }
        }
      }
    }
    if (!known) {
      if (whole) take(Border{low_key, 0x7fffffff});
      else sure = false;
    }
  }
  if (!sure) return 0;

  // ---- the lowest indices among those with the border's key
  uint32_t cut = 0xffffffffu;
  {
    const Found f = border.ties == 0x7fffffff
                        ? Found{false, 0, 0, 0}
                        : find_on_list<false>(S, m_list, 0, 0xffffffffu, static_cast<unsigned long long>(border.ties),
                                              [&](int i, uint32_t& k) {
                                                k = ~static_cast<uint32_t>(list[i]);
                                                return static_cast<uint32_t>(list[i] >> 32) == border.key;
                                              }, one);
    if (f.there) cut = ~f.key;
  }
  // ---- the kept ones by index: into 512 buckets by their leading bits, then by rank in their bucket; S.token: their places on the list
  auto keeps = [&](unsigned long long x) {
    const uint32_t k = static_cast<uint32_t>(x >> 32), v = static_cast<uint32_t>(x);
    return k > border.key || (k == border.key && v <= cut);
  };
  const int shift = max(0, 32 - __clz(V) - 9);
  auto bucket = [&](unsigned long long x) { return static_cast<uint32_t>(x) >> shift; };
  list_sync();
  for (int i = tid; i < m_list; i += kListThreads)
    if (keeps(list[i])) atomicAdd(&S.count[bucket(list[i])], 1u);
  list_sync();
  const unsigned in_bucket = S.count[tid];
  unsigned start = in_bucket;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const unsigned up = __shfl_up_sync(0xffffffffu, start, o);
    if (lane >= o) start += up;
  }
  if (lane == 31) S.u[warp] = start;
  list_sync();
  start += static_cast<unsigned>(warps_before(S.u, warp, lane)) - in_bucket;
  S.part[0][tid] = S.part[1][tid] = start;
  if (tid == kListThreads - 1) S.moved = start + in_bucket;
  list_sync();
  const int kept = static_cast<int>(S.moved);
  for (int i = tid; i < m_list; i += kListThreads)
    if (keeps(list[i])) S.token[atomicAdd(&S.part[0][bucket(list[i])], 1u)] = static_cast<uint32_t>(i);
  list_sync();
  uint32_t move[kCap / kListThreads];                          // place on the list, place in order
#pragma unroll
  for (int y = 0; y < kCap / kListThreads; ++y) {
    const int t = tid + y * kListThreads;
    move[y] = 0;
    if (t < kept) {
      const uint32_t i = S.token[t], v = static_cast<uint32_t>(list[i]), b = bucket(list[i]);
      const int b0 = S.part[1][b], b1 = b0 + S.count[b];
      int at = b0;
      for (int u = b0; u < b1; ++u) at += static_cast<uint32_t>(list[S.token[u]]) < v ? 1 : 0;
      move[y] = i << 16 | static_cast<uint32_t>(at);
    }
  }
  list_sync();
#pragma unroll
  for (int y = 0; y < kCap / kListThreads; ++y)
    if (tid + y * kListThreads < kept) S.token[move[y] & 0xffffu] = move[y] >> 16;
  S.count[tid] = S.part[0][tid] = S.part[1][tid] = 0;
  list_sync();
  return kept;
}

// A part of a row, from 16-byte boundary to 16-byte boundary but for the row's ends.
template <bool HALF>
struct Slice {
  static constexpr int kVec = HALF ? 8 : 4;                    // tokens of a vector
  const void* row;
  const uint4* vecs;
  int lead, n_vec, vec0, vec1;                                 // tokens in front of the first whole vector; vectors; the part's
};
template <bool HALF>
__device__ __forceinline__ Slice<HALF> slice_of(const Args& A, int s, int part, int parts) {
  using T = Slice<HALF>;
  T t;
  t.row = row_of<HALF>(A, s);
  const int skew = static_cast<int>(reinterpret_cast<uintptr_t>(t.row) % 16) / (HALF ? 2 : 4);
  t.lead = skew ? min(T::kVec - skew, A.vocab) : 0;
  t.n_vec = (A.vocab - t.lead) / T::kVec;
  const int per = (t.n_vec + parts - 1) / parts;
  t.vec0 = min(part * per, t.n_vec);
  t.vec1 = min(t.vec0 + per, t.n_vec);
  t.vecs = reinterpret_cast<const uint4*>(static_cast<const char*>(t.row) + t.lead * (HALF ? 2 : 4));
  return t;
}
// What a row's parameters make of it.
struct RowKind {
  bool fine, greedy, by_k, whole, add_up;
};
__device__ __forceinline__ RowKind kind_of(const RowParams& R, int V) {
  RowKind k;
  k.fine = R.temperature >= 0.f && R.temperature < INFINITY;
  k.greedy = R.temperature == 0.f || R.top_k == 1 || R.top_p <= 0.f;
  k.by_k = R.top_k > 0 && R.top_k < V;
  k.whole = V <= kCap;                                         // every finite logit goes on the list
  k.add_up = k.fine && !k.greedy && !k.whole && !k.by_k && R.top_p < 1.f;
  return k;
}
// Bound of a quick sum's relative error: terms 2^(fma(l, c', -base)) by the special-function unit (documented: 2^-22), c' = log2(e) / T in
// fp32, eight added pairwise (three roundings of 2^-24), from there in fp64.  The exponent x of a term is off by 2^-24 |x| (its rounding),
// and relative to the largest term by 2^-24 of their distance (the rounding of c').  On average over the terms, each with its weight,
// a distance from the largest is at most log2 V (the entropy of the row), |x| at most `far` more: the largest one's, or, of a row
// in parts, which have bases of their own, the mean over the parts by their sums.  About 2e-6 where the sample saw the largest terms: where a
// row's end by top-p lies closer to a token's than that, its sum is made again in fp64 (exact_total).
__device__ __forceinline__ double quick_error(double far, int V) {
  const double spread = 33 - __clz(V);
  return 0.6932 * 0x1p-24 * (2.0 * spread + far) + 0x1p-22 + 4 * 0x1p-24;
}
__device__ __forceinline__ float quick_c(const RowParams& R) { return static_cast<float>(1.4426950408889634 / static_cast<double>(R.temperature)); }
// The sum of all of a row's terms (the threads of a list).
template <bool HALF>
__device__ __noinline__ double exact_total(ListShared& S, const void* row, int V, const Term e) {
  const int tid = threadIdx.x % kListThreads;
  double sum = 0.0;
#pragma unroll 8
  for (int v = tid; v < V; v += kListThreads) sum += e(load_logit<HALF>(row, v));
  sum = warp_sum_d(sum);
  list_sync();
  if ((tid & 31) == 0) S.d[tid >> 5] = sum;
  list_sync();
  sum = 0.0;
#pragma unroll
  for (int w = 0; w < kListWarps; ++w) sum += S.d[w];
  list_sync();
  return sum;
}
struct Job {                                                   // of a block: a row or a part of one
  int s, part, parts;
};
// What a job begins with: parameters, and a vector a thread of the sample (a warp's 512 bytes in a row, the warps spread over the part).
struct RowHead {
  int64_t d0, d1;
  RowParams R;
  uint4 sample;
};
template <bool HALF>
__device__ __forceinline__ RowHead row_head(const Args& A, const Job& job) {
  const int tid = threadIdx.x % kListThreads;
  RowHead h;
  h.d0 = __ldg(A.draw_offsets + job.s);
  h.d1 = __ldg(A.draw_offsets + job.s + 1);
  h.R = row_params(A, job.s);
  h.sample = make_uint4(0, 0, 0, 0);
  if (A.vocab > kCap) {
    const Slice<HALF> t = slice_of<HALF>(A, job.s, job.part, job.parts);
    const int n = t.vec1 - t.vec0, at = (tid >> 5) * (n / kListWarps) + (tid & 31);
    if (n > 0) h.sample = __ldg(t.vecs + t.vec0 + min(at, n - 1));
  }
  return h;
}
// The buffer for a job's pass: its threshold (the threads of lists).
template <bool HALF>
__device__ __forceinline__ void begin_row(const Args& A, ListShared& S, RowBuffer& B, const Job& job, const RowHead& H) {
  constexpr int kVec = Slice<HALF>::kVec;
  const int tid = threadIdx.x % kListThreads, lane = tid & 31;
  const RowKind K = kind_of(H.R, A.vocab);
  list_sync();
  if (!K.whole) {
    float x[kVec], m = -INFINITY;
    unpack<HALF>(H.sample, x);
#pragma unroll
    for (int i = 0; i < kVec; ++i) m = fmaxf(m, x[i]);
#pragma unroll
    for (int o = 1; o < 8; o <<= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
    if ((lane & 7) == 0) S.group[tid >> 3] = m;
    list_sync();
  }
  if (tid >= 32) return;
  float low = kLowest, base = 0.f;
  if (!K.whole) {
    const Slice<HALF> t = slice_of<HALF>(A, job.s, job.part, job.parts);
    // Candidates wanted: top-k says how many it needs, min-p needs few, top-p of the whole row may need many.
    const float want = (K.by_k ? fminf(fmaxf(512.f, 2.f * static_cast<float>(H.R.top_k)), 4096.f) : H.R.min_p > 0.f ? 512.f : 4096.f) / job.parts;
    const float share = fminf(want / static_cast<float>(max((t.vec1 - t.vec0) * kVec, 1)), 1.f);
    const int at = min(static_cast<int>(kGroups * __expf(-8.f * kVec * share)), kGroups - 1);
    const float m0 = S.group[lane], m1 = S.group[lane + 32];
    int below0 = 0, below1 = 0;
    for (int i = 0; i < kGroups; ++i) {
      const float o = S.group[i];
      below0 += o < m0 || (o == m0 && i < lane) ? 1 : 0;
      below1 += o < m1 || (o == m1 && i < lane + 32) ? 1 : 0;
    }
    const float mine = below0 == at ? m0 : below1 == at ? m1 : -INFINITY;
    low = fmaxf(warp_max(mine), kLowest);                      // (one lane has it)
    if (K.add_up) {
      base = rintf(fminf(fmaxf(warp_max(fmaxf(m0, m1)) * quick_c(H.R), -1e6f), 1e6f));
    }
  }
  if (lane == 0) {
    B.n = 0;
    B.low = low;
    B.base = base;
    B.skip = H.d1 <= H.d0 && !A.kept_out;
    B.d0 = H.d0;
    B.d1 = H.d1;
    B.R = H.R;
  }
}

// One pass over a job's logits (the first kListThreads threads).
template <bool HALF>
__device__ __forceinline__ void pass_row(const Args& A, uint4 (&ring)[4][32], RowBuffer& B, const Job& job) {
  constexpr int kVec = Slice<HALF>::kVec;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, V = A.vocab;
  if (B.skip) return;
  const Slice<HALF> L = slice_of<HALF>(A, job.s, job.part, job.parts);
  const RowParams R = B.R;
  const float low = B.low, base = B.base;
  const bool add_up = kind_of(R, V).add_up;
  const float c = add_up ? quick_c(R) : 0.f;
  float mx = -INFINITY;
  double z = 0.0;
  auto single = [&](int v) {
    const float x = load_logit<HALF>(L.row, v);
    mx = max_nan(mx, x);
    if (x >= low) {                                            // (a NaN is not taken)
      const unsigned at = atomicAdd(&B.n, 1u);
      if (at < kCap) B.list[at] = entry_of(x, v);
    }
    if (add_up) z += static_cast<double>(ex2(fmaf(x, c, -base)));
  };
  if (job.part == 0 && tid < L.lead) single(tid);
  if (job.part == job.parts - 1 && tid < V - L.lead - L.n_vec * kVec) single(L.lead + L.n_vec * kVec + tid);
  const uint4 nothing = HALF ? make_uint4(0xff80ff80u, 0xff80ff80u, 0xff80ff80u, 0xff80ff80u)
                             : make_uint4(0xff800000u, 0xff800000u, 0xff800000u, 0xff800000u);   // -inf
  const uint32_t slot = static_cast<uint32_t>(__cvta_generic_to_shared(&ring[0][lane]));
  auto fetch = [&](int v0) {
    const uint4* from = L.vecs + v0 + lane;
    const bool full = v0 + 128 <= L.vec1;                      // (warp-uniform)
#pragma unroll
    for (int j = 0; j < 4; ++j)
      if (full || v0 + j * 32 + lane < L.vec1)
        asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(slot + j * 512), "l"(from + j * 32) : "memory");
    asm volatile("cp.async.commit_group;" ::: "memory");
  };
  constexpr int kStep = kListWarps * 128;
  int v0 = L.vec0 + warp * 128;
  if (v0 < L.vec1) fetch(v0);
  for (; v0 < L.vec1; v0 += kStep) {
    asm volatile("cp.async.wait_group 0;" ::: "memory");
    uint4 u[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) u[j] = ring[j][lane];
    if (v0 + 128 > L.vec1) {                                   // past the end: nothing
#pragma unroll
      for (int j = 0; j < 4; ++j)
        if (v0 + j * 32 + lane >= L.vec1) u[j] = nothing;
    }
    __syncwarp();
    if (v0 + kStep < L.vec1) fetch(v0 + kStep);
    // 16 tokens at a time
#pragma unroll
    for (int g = 0; g < (HALF ? 2 : 1); ++g) {
    constexpr int kVecs = HALF ? 2 : 4;                        // vectors of them
    float x[16];
#pragma unroll
    for (int j = 0; j < kVecs; ++j) unpack<HALF>(u[g * kVecs + j], x + j * kVec);
    float top = x[0];
#pragma unroll
    for (int i = 1; i < 15; i += 2) top = max3_nan(top, x[i], x[i + 1]);
    mx = max3_nan(mx, top, x[15]);
    unsigned hits = 0;
#pragma unroll
    for (int i = 0; i < 16; ++i) hits |= x[i] >= low ? 1u << i : 0u;
    if (hits) {
      unsigned at = atomicAdd(&B.n, static_cast<unsigned>(__popc(hits)));
      for (; hits; hits &= hits - 1, ++at) {
        const int i = __ffs(hits) - 1;
        if (at < kCap) B.list[at] = entry_of(pick16(x, i), L.lead + (v0 + (g * kVecs + i / kVec) * 32 + lane) * kVec + i % kVec);
      }
    }
    if (add_up) {
      const f32x2 c2 = both(c), shift = both(-base);
#pragma unroll
      for (int h = 0; h < 16; h += 8) {
        float e[8];
#pragma unroll
        for (int y = 0; y < 8; y += 2) {
          float x0, x1;
          unpack2(fma2(pack2(x[h + y], x[h + y + 1]), c2, shift), x0, x1);
          e[y] = ex2(x0);
          e[y + 1] = ex2(x1);
        }
        float a, b;
        unpack2(add2(add2(pack2(e[0], e[1]), pack2(e[2], e[3])), add2(pack2(e[4], e[5]), pack2(e[6], e[7]))), a, b);
        z += static_cast<double>(a + b);
      }
    }
    }
  }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) mx = max_nan(mx, __shfl_xor_sync(0xffffffffu, mx, o));
  z = warp_sum_d(z);
  // (terms out of range: the sample was far off)
  if (lane == 0) { B.max[warp] = mx; B.sum[warp] = !add_up || mx * c <= base + 100.f ? z : static_cast<double>(NAN); }
}
__device__ __forceinline__ void passed(const RowBuffer& B, float& mx, double& z) {
  mx = B.max[0];
  z = B.sum[0];
#pragma unroll
  for (int w = 1; w < kListWarps; ++w) { mx = max_nan(mx, B.max[w]); z += B.sum[w]; }
}

// Row s from its list (all of it): false, and nothing given, where the list cannot tell.  z, base, far: its quick sum, see quick_error.
template <bool HALF>
__device__ __forceinline__ bool list_row(const Args& A, ListShared& S, unsigned long long* list, int s, int64_t d0, int64_t d1, const RowParams& R,
                                         int m_list, bool fits, float low, float mx, double z, float base, double far) {
  const int tid = threadIdx.x % kListThreads, lane = tid & 31, warp = tid >> 5;
  const RowKind K = kind_of(R, A.vocab);
  const bool fine = K.fine, greedy = K.greedy, by_k = K.by_k, whole = K.whole, add_up = K.add_up;
  uint32_t low_key = whole ? kNegInf + 1 : key_of(low);
  // ---- the border
  auto give_all = [&](int token, int kept) {
    for (int64_t d = d0 + tid; d < d1; d += kListThreads) {
      A.tokens_out[d] = token;
      if (A.seq_out) A.seq_out[d] = s;
    }
    if (tid == 0 && A.kept_out) A.kept_out[s] = kept;
  };
  if (!fine || !(mx < INFINITY) || mx == -INFINITY) {          // (a NaN is not less)
    give_all(-1, 0);
    return true;
  }
  const uint32_t max_key = key_of(mx);
  const Term e = term_of(mx, greedy ? 1.f : R.temperature, S.table);
  auto fixed = [&](uint32_t k) { return __double2ull_rn(e(logit_of(k)) * kFix); };
  const bool limit = !greedy && by_k && !(whole && R.top_k >= m_list);            // top-k leaves something out
  const bool by_p = !greedy && R.top_p < 1.f, by_m = !greedy && R.min_p > 0.f;
  double total_quick = 0.0, error_quick = 0.0;
  if (add_up) {
    const double top = e.max * static_cast<double>(quick_c(R));
    total_quick = z * exp2(static_cast<double>(base) - top);
    error_quick = quick_error(far, A.vocab);
  }
  // (once it is needed)
  auto make_exact = [&]() {
    total_quick = exact_total<HALF>(S, row_of<HALF>(A, s), A.vocab, e);
    error_quick = kFixError;
  };
  double* sums = reinterpret_cast<double*>(list);            // (behind the borders: running sums of the kept ones, beside S.token)
  int kept = 0;

  // ---- few candidates (what no filter can keep left out): in order, a thread each
  bool sure = fits && (!by_p || limit || whole || add_up);
  if (sure) {
    uint32_t head = greedy ? max_key : low_key, m_key = 0;     // they have at least the key `head`
    double total = total_quick, error = error_quick;
    if (whole) {
      if (tid == 0) S.min_key = max_key;
      list_sync();
      uint32_t lowest = max_key;
      for (int i = tid; i < m_list; i += kListThreads) lowest = min(lowest, static_cast<uint32_t>(list[i] >> 32));
      lowest = __reduce_min_sync(0xffffffffu, lowest);
      if (lane == 0) atomicMin(&S.min_key, lowest);
      list_sync();
      low_key = S.min_key;
      if (!greedy) head = low_key;
    }
    if (by_m) {                                                // (a bound that is sure; the definition decides below)
      const double x = e.max + static_cast<double>(R.temperature) * log(fmin(static_cast<double>(R.min_p), 1.0));
      const double y = x - 1e-6 * (fabs(x) + fabs(e.max)) - 1e-30;
      if (y > -3.4e38) m_key = min(key_of(static_cast<float>(y)), max_key);
      head = max(head, m_key);
    }
    if ((limit || by_p) && m_list > (whole && !limit ? kListThreads : 128)) {   // one histogram: the bin that top-k or top-p ends in
      const uint32_t range = max_key - low_key;
      const int shift = range < kBins ? 0 : 32 - __clz(range) - 9;
      for (int i = tid; i < m_list; i += kListThreads) {
        const uint32_t k = static_cast<uint32_t>(list[i] >> 32);
        if (k < low_key) continue;
        const uint32_t b = (k - low_key) >> shift;
        if (limit) atomicAdd(&S.count[b], 1u);
        else add_fixed(S, b, fixed(k));
      }
      if (tid == 0) S.bin = 0;
      list_sync();
      const int bin = kBins - 1 - tid;
      const unsigned long long here = limit ? static_cast<unsigned long long>(S.count[bin]) : take_fixed(S, bin);
      S.count[bin] = 0;
      unsigned long long incl = here;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const unsigned long long up = __shfl_up_sync(0xffffffffu, incl, o);
        if (lane >= o) incl += up;
      }
      if (lane == 31) S.u[warp] = incl;
      list_sync();
      incl += warps_before(S.u, warp, lane);
      if (whole && !limit) {                                   // (the list is all there is)
        if (tid == kListThreads - 1) S.all = incl;
        list_sync();
        total = static_cast<double>(S.all) / kFix;
        error = kFixError;
      }
      const double most = static_cast<double>(R.top_p) * total * (1.0 + 2.0 * error) * kFix;
      const unsigned long long target = limit ? static_cast<unsigned long long>(R.top_k) : most < 1.8e19 ? __double2ull_ru(most) : ~0ull;
      if (incl >= target && incl - here < target) S.bin = bin;
      list_sync();
      // (top-p's share is of all that top-k keeps: min-p must not shorten those then)
      const uint32_t to = low_key + (S.bin << shift);
      head = limit && by_p ? to : max(head, to);
    } else if (by_p) {
      head = low_key;                                          // (all of a short list)
    }
    if (tid == 0) S.moved = 0;
    list_sync();
    for (int i = tid; i < m_list; i += kListThreads) {
      if (static_cast<uint32_t>(list[i] >> 32) >= head) {
        const unsigned at = atomicAdd(&S.moved, 1u);
        if (at < kListThreads) S.token[at] = static_cast<uint32_t>(i);
      }
    }
    list_sync();
    const int h = static_cast<int>(S.moved);
    if (h <= kListThreads) {
      // in order: largest logit first, equal ones by index
      unsigned long long y = tid < h ? list[S.token[tid]] ^ 0xffffffffull : 0;
      if (tid < h) S.order[tid] = y;
      list_sync();
      int at = 0;
      if (tid < h)
        for (int j = 0; j < h; ++j) at += S.order[j] > y ? 1 : 0;
      list_sync();
      if (tid < h) S.order[at] = y;
      list_sync();
      y = tid < h ? S.order[tid] : 0;
      const double mine = tid < h ? e(logit_of(static_cast<uint32_t>(y >> 32))) : 0.0;
      const double sum = block_scan_d(S.d, mine, warp, lane);
      // The least of the ends that lie among the candidates; an end that does not is not less.
      int end = greedy ? 1 : 0x7fffffff;
      if (limit && R.top_k <= h) end = min(end, R.top_k);
      if (!limit && whole && h == m_list) end = min(end, h);
      if (by_m) {
        const int passing = max(list_count(tid < h && mine >= static_cast<double>(R.min_p)), 1);
        if (passing < h || (head <= m_key && m_key >= low_key)) end = min(end, passing);
      }
      if (by_p) {
        const int n = limit ? R.top_k : h;                     // top-p's share is of these, or more
        if (n > h) {
          sure = false;
        } else {
          if (tid == n - 1) S.z = sum;
          list_sync();
          if (limit || (whole && h == m_list)) { total = S.z; error = 0.0; }
          int least, most;
          double target;
          // (a sum that is 0, infinite or none says nothing: terms out of range)
          auto known = [](double x) { return x > 0.0 && x < static_cast<double>(INFINITY); };
          for (int round = 0;; ++round) {
            target = static_cast<double>(R.top_p) * total;
            least = 1 + list_count(tid < n && sum < target * (1.0 - error));
            most = 1 + list_count(tid < n && sum < target * (1.0 + error));
            // (too close to tell, and nothing else ends before: by the exact sum, whose own error no longer counts)
            if (!add_up || round == 1 || !((least < most && least <= n && end > least) || !known(target))) break;
            make_exact();
            total = total_quick;
            error = 0.0;
          }
          if (!known(target)) sure = false;
          else if (least == most && least <= n) end = min(end, least);
          else if (least <= n) sure = end <= least;            // too close to tell, unless something else ends before
        }
      }
      if (sure && end <= h) {                                  // the kept ones by index, and their running sums
        kept = end;
        const uint32_t v = ~static_cast<uint32_t>(y);
        if (tid < kept) S.token[tid] = v;
        list_sync();
        int place = 0;
        if (tid < kept)
          for (int j = 0; j < kept; ++j) place += S.token[j] < v ? 1 : 0;
        list_sync();
        if (tid < kept) {
          S.token[place] = v;
          sums[place] = mine;
        }
        list_sync();
        const double running = block_scan_d(S.d, tid < kept ? sums[tid] : 0.0, warp, lane);
        if (tid < kept) sums[tid] = running;
        list_sync();
      }
    }
  }
  if (!sure) return false;
  if (kept == 0 && add_up && !(error_quick <= kFixError)) make_exact();
  const bool wide = kept == 0;
  if (wide) kept = wide_list(S, list, R, e, A.vocab, m_list, low_key, max_key, limit, greedy, whole, add_up, total_quick, error_quick);
  if (kept == 0) return false;
  if (tid == 0 && A.kept_out) A.kept_out[s] = kept;
  if (d1 <= d0) return true;
  // Draws.  Few kept ones: their running sums, S.token their tokens.  Many: a running sum for every stretch of them (a thread's), terms
  // made again within one.
  const int stretch = wide ? (kept + kListThreads - 1) / kListThreads : 1, n_sums = (kept + stretch - 1) / stretch;
  auto term_at = [&](int p) { return e(logit_of(static_cast<uint32_t>(list[S.token[p]] >> 32))); };
  if (wide) {
    sums = reinterpret_cast<double*>(S.order);
    double mine = 0.0;
    for (int p = tid * stretch; p < min((tid + 1) * stretch, kept); ++p) mine += term_at(p);
    const double running = block_scan_d(S.d, mine, warp, lane);
    sums[tid] = running;
    list_sync();
  }
  const double total = sums[n_sums - 1];
  for (int64_t d = d0 + tid; d < d1; d += kListThreads) {
    const float u = __ldg(A.uniforms + d);
    const double target = (u < 1.f ? fmaxf(u, 0.f) : 1.f) * total;
    int a = 0, b = n_sums;
    while (a < b) {
      const int mid = (a + b) >> 1;
      if (sums[mid] > target) b = mid; else a = mid + 1;
    }
    if (a == n_sums) {                                         // none: the last one that adds something
      --a;
      while (a > 0 && !(sums[a] > sums[a - 1])) --a;
    }
    uint32_t token;
    if (wide) {
      double run = a > 0 ? sums[a - 1] : 0.0;
      int at = a * stretch, last = at;
      for (int p = at; p < min((a + 1) * stretch, kept); ++p) {
        const double t = term_at(p);
        run += t;
        if (t > 0.0) last = p;
        at = p;
        if (run > target && t > 0.0) break;
      }
      token = static_cast<uint32_t>(list[S.token[run > target ? at : last]]);   // (the two sums of a stretch may differ in their last bits)
    } else {
      token = S.token[a];
    }
    A.tokens_out[d] = static_cast<int32_t>(token);
    if (A.seq_out) A.seq_out[d] = s;
  }
  return true;
}

struct RowsShared {
  RowBuffer B;
  ListShared S;
};
template <bool HALF>
__global__ void __launch_bounds__(kListThreads, 2) list_rows_kernel(const __grid_constant__ Args A) {
  ss::grid_dependency_enter();
  extern __shared__ __align__(16) unsigned char smem[];
  RowsShared& M = *reinterpret_cast<RowsShared*>(smem);
  RowBuffer& B = M.B;
  const int tid = threadIdx.x, block = blockIdx.x;
  const int mine = block < A.whole_rows ? (A.whole_rows - block + gridDim.x - 1) / gridDim.x : 0;
  const bool part = A.parts > 1 && block < (A.n_seq - A.whole_rows) * A.parts;
  const int jobs = mine + (part ? 1 : 0);
  if (jobs == 0) return;
  // The second half of the blocks (an SM's second, as blocks are dealt out) has its part first, the first half last: the two blocks
  // of an SM then are not on their lists at the same time.
  const int lead = part && 2 * block >= static_cast<int>(gridDim.x) ? 1 : 0;
  auto job_of = [&](int j) {
    const int row = j - lead;
    return row >= 0 && row < mine ? Job{block + row * static_cast<int>(gridDim.x), 0, 1}
                                  : Job{A.whole_rows + block / A.parts, block % A.parts, A.parts};
  };
  M.S.count[tid] = 0;
  for (int x = 0; x < 3; ++x) M.S.part[x][tid] = 0;
  make_table(M.S.table);
  RowHead H = row_head<HALF>(A, job_of(0));
  for (int j = 0; j < jobs; ++j) {
    const Job job = job_of(j);
    begin_row<HALF>(A, M.S, B, job, H);
    list_sync();
    pass_row<HALF>(A, M.S.ring[tid >> 5], B, job);
    list_sync();
    if (j + 1 < jobs) H = row_head<HALF>(A, job_of(j + 1));
    if (!B.skip) {
      float mx;
      double z;
      passed(B, mx, z);
      if (job.parts == 1) {
        const bool done = list_row<HALF>(A, M.S, B.list, job.s, B.d0, B.d1, B.R, static_cast<int>(min(B.n, static_cast<unsigned>(kCap))), B.n <= kCap,
                                   B.low, mx, z, B.base, fabs(static_cast<double>(mx) * quick_c(B.R) - B.base));
        if (tid == 0) A.marks[job.s] = done ? 0 : 1;
      } else {
        Part& P = A.part[block];
        for (unsigned i = tid; i < min(B.n, static_cast<unsigned>(kPartCap)); i += kListThreads) P.list[i] = B.list[i];
        if (tid == 0) { P.n = B.n; P.low = B.low; P.base = B.base; P.max = mx; P.sum = z; }
      }
    } else if (tid == 0 && job.parts == 1) {
      A.marks[job.s] = 0;
    }
  }
}

// The border of a row whose kept tokens are too many for a list, by top-k or by top-p (not both), on a list of its surroundings: a
// histogram over the logit (2048 bins, counts) says in which bin it lies - for top-p by the terms at the bins' middles, off by far less
// than a bin - and one more pass adds up, in fp64, what lies above that bin and its neighbours, and collects those.  The list then
// decides, and says whether the border is in it at all.  `kept`: how many are, `cut`: the last index of those with the border's key.
struct Bracketed {
  bool there;
  Border border;
  int kept, cut;
};
template <bool HALF>
__device__ __noinline__ Bracketed bracket_row(ListShared& S, unsigned long long* list, const void* row, int V, const RowParams R, const Term e, float top,
                                              unsigned long long finite) {
  constexpr int kFine = 2048, kPer = kFine / kListThreads;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const Bracketed none{false, Border{0, 0}, 0, 0};
  const bool limit = R.top_k > 0 && static_cast<unsigned long long>(R.top_k) < finite, by_p = R.top_p < 1.f;
  if (limit == by_p) return none;
  __syncthreads();
  float least = INFINITY;
  if (limit) {
    for (int v = tid; v < V; v += kListThreads) {
      const float x = load_logit<HALF>(row, v);
      if (x > -INFINITY) least = fminf(least, x);
    }
  } else {
    least = top - 40.f * R.temperature;                        // (what lies below adds up to less than 1e-11)
  }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) least = fminf(least, __shfl_xor_sync(0xffffffffu, least, o));
  if (lane == 0) S.group[warp] = least;
  for (int x = 0; x < kPer; ++x) S.token[tid + x * kListThreads] = 0;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < kListWarps; ++w) least = fminf(least, S.group[w]);
  const float width = (top - least) / (kFine - 1), per_width = 1.f / width;
  if (!(width > 0.f) || !(per_width < INFINITY)) return none;
  auto bin_of = [&](float x) { return static_cast<int>(fminf(fmaxf((x - least) * per_width, 0.f), static_cast<float>(kFine - 1))); };
  for (int v = tid; v < V; v += kListThreads) {
    const float x = load_logit<HALF>(row, v);
    if (x > -INFINITY) atomicAdd(&S.token[bin_of(x)], 1u);
  }
  if (tid == 0) { S.bin = 0; S.moved = 0; }
  __syncthreads();
  // counts and terms from the top, kPer bins a thread
  unsigned counts[kPer];
  double terms[kPer], terms_here = 0.0;
  unsigned long long here = 0;
#pragma unroll
  for (int x = 0; x < kPer; ++x) {
    const int b = kFine - 1 - (tid * kPer + x);
    counts[x] = S.token[b];
    here += counts[x];
    terms[x] = by_p && counts[x] ? counts[x] * e(fminf(least + (static_cast<float>(b) + 0.5f) * width, top)) : 0.0;
    terms_here += terms[x];
  }
  unsigned long long incl = here;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const unsigned long long up = __shfl_up_sync(0xffffffffu, incl, o);
    if (lane >= o) incl += up;
  }
  if (lane == 31) S.u[warp] = incl;
  const double terms_incl = block_scan_d(S.d, terms_here, warp, lane);          // (a barrier)
  incl += warps_before(S.u, warp, lane);
  if (tid == kListThreads - 1) S.z = terms_incl;
  __syncthreads();
  {
    const double target = static_cast<double>(R.top_p) * S.z;
    unsigned long long n = incl - here;
    double m = terms_incl - terms_here;
#pragma unroll
    for (int x = 0; x < kPer; ++x) {
      const bool in = limit ? n < static_cast<unsigned long long>(R.top_k) && n + counts[x] >= static_cast<unsigned long long>(R.top_k)
                            : m < target && m + terms[x] >= target;
      if (in) S.bin = kFine - 1 - (tid * kPer + x);
      n += counts[x];
      m += terms[x];
    }
  }
  __syncthreads();
  const int bin = static_cast<int>(S.bin), b0 = limit ? bin : bin - 1, b1 = limit ? bin : bin + 1;
  if (b0 < 1 && !limit) return none;                           // (the lowest bin holds all that is below)
  // what lies above, and the surroundings
  double above = 0.0, all = 0.0;
  unsigned n_above = 0;
  for (int v = tid; v < V; v += kListThreads) {
    const float x = load_logit<HALF>(row, v);
    if (!(x > -INFINITY)) continue;
    const int b = bin_of(x);
    if (by_p) {
      const double t = e(x);
      all += t;
      above += b > b1 ? t : 0.0;
    }
    n_above += b > b1 ? 1 : 0;
    if (b >= b0 && b <= b1) {
      const unsigned at = atomicAdd(&S.moved, 1u);
      if (at < kCap) list[at] = entry_of(x, v);
    }
  }
  above = warp_sum_d(above);
  all = warp_sum_d(all);
  n_above = __reduce_add_sync(0xffffffffu, n_above);
  __syncthreads();
  if (lane == 0) { S.d[warp] = above; S.order[warp] = static_cast<unsigned long long>(__double_as_longlong(all)); S.u[warp] = n_above; }
  __syncthreads();
  above = all = 0.0;
  unsigned long long larger = 0;
#pragma unroll
  for (int w = 0; w < kListWarps; ++w) {
    above += S.d[w];
    all += __longlong_as_double(static_cast<long long>(S.order[w]));
    larger += S.u[w];
  }
  const unsigned n = S.moved;
  if (n == 0 || n > kCap) return none;
  auto by_key = [&](int i, uint32_t& k) { k = static_cast<uint32_t>(list[i] >> 32); return true; };
  auto fixed = [&](uint32_t k) { return __double2ull_rn(e(logit_of(k)) * kFix); };
  auto one = [](uint32_t) { return 1ull; };
  Bracketed B = none;
  unsigned long long ties, same;
  if (limit) {
    if (larger >= static_cast<unsigned long long>(R.top_k)) return none;
    const Found f = find_on_list<false>(S, static_cast<int>(n), 0, 0xffffffffu, R.top_k - larger, by_key, one);
    if (!f.there) return none;
    ties = R.top_k - larger - f.above;
    same = f.at_key;
    B.border.key = f.key;
  } else {
    const double target = static_cast<double>(R.top_p) * all, slack = 4e-12 * all;    // (kCap 2^-51, and a share of it for the sums)
    if (!(target - above > slack)) return none;
    const unsigned long long need = __double2ull_ru((target - above - slack) * kFix);
    const Found f = find_on_list<true>(S, static_cast<int>(n), 0, 0xffffffffu, need, by_key, fixed);
    if (!f.there) return none;
    const unsigned long long each = max(fixed(f.key), 1ull);
    ties = (need - f.above + each - 1) / each;
    if (!(static_cast<double>(f.above + ties * each) >= (target - above + slack) * kFix)) return none;
    same = f.at_key / each;
    B.border.key = f.key;
  }
  B.border.ties = ties < same ? static_cast<int>(ties) : 0x7fffffff;
  B.cut = V;
  if (ties < same) {
    const Found f = find_on_list<false>(S, static_cast<int>(n), 0, 0xffffffffu, ties,
                                        [&](int i, uint32_t& k) {
                                          k = ~static_cast<uint32_t>(list[i]);
                                          return static_cast<uint32_t>(list[i] >> 32) == B.border.key;
                                        }, one);
    if (!f.there) return none;
    B.cut = static_cast<int>(~f.key);
  }
  int mine = 0;
  for (unsigned i = tid; i < n; i += kListThreads) {
    const uint32_t k = static_cast<uint32_t>(list[i] >> 32), v = static_cast<uint32_t>(list[i]);
    mine += k > B.border.key || (k == B.border.key && v <= static_cast<uint32_t>(B.cut)) ? 1 : 0;
  }
  mine = __reduce_add_sync(0xffffffffu, mine);
  __syncthreads();
  if (lane == 0) S.u[warp] = mine;
  __syncthreads();
  unsigned long long kept = larger;
#pragma unroll
  for (int w = 0; w < kListWarps; ++w) kept += S.u[w];
  B.kept = static_cast<int>(kept);
  B.there = true;
  __syncthreads();
  return B;
}

// ---- any row, one block, several passes ------------------------------------------------------------------------------------------
struct WholeShared {
  double d[kWarps];
  unsigned long long u[kWarps];
  unsigned count[256];
  unsigned long long mass[256];
  double seg[kMaxVocab / kSeg];                // running sum of the kept tokens at every segment's end
  Border border;
  unsigned pick;
  unsigned left;
  double above;
  int cut;
};

__device__ __forceinline__ double block_sum(WholeShared& S, double v) {
  v = warp_sum_d(v);
  __syncthreads();
  if ((threadIdx.x & 31) == 0) S.d[threadIdx.x >> 5] = v;
  __syncthreads();
  double t = 0.0;
#pragma unroll
  for (int w = 0; w < kWarps; ++w) t += S.d[w];
  return t;
}
__device__ __forceinline__ unsigned long long block_sum_u(WholeShared& S, unsigned long long v) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  __syncthreads();
  if ((threadIdx.x & 31) == 0) S.u[threadIdx.x >> 5] = v;
  __syncthreads();
  unsigned long long t = 0;
#pragma unroll
  for (int w = 0; w < kWarps; ++w) t += S.u[w];
  return t;
}
__device__ __forceinline__ unsigned long long block_max_u(WholeShared& S, unsigned long long v) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v = max(v, __shfl_xor_sync(0xffffffffu, v, o));
  __syncthreads();
  if ((threadIdx.x & 31) == 0) S.u[threadIdx.x >> 5] = v;
  __syncthreads();
  unsigned long long t = 0;
#pragma unroll
  for (int w = 0; w < kWarps; ++w) t = max(t, S.u[w]);
  return t;
}

template <bool HALF>
__device__ void whole_row(const Args& A, WholeShared& S, ListShared& L, unsigned long long* list, int s) {   // (list: S's memory)
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, V = A.vocab;
  const int64_t d0 = A.draw_offsets[s], d1 = A.draw_offsets[s + 1];
  if (d1 <= d0 && !A.kept_out) return;
  const void* row = row_of<HALF>(A, s);
  const RowParams R = row_params(A, s);
  auto give_all = [&](int token, int kept) {
    for (int64_t d = d0 + tid; d < d1; d += kThreads) {
      A.tokens_out[d] = token;
      if (A.seq_out) A.seq_out[d] = s;
    }
    if (tid == 0 && A.kept_out) A.kept_out[s] = kept;
  };
  // ---- the maximum (lowest index first), what is no number, how many tokens there are
  unsigned long long best = 0, finite = 0;
  for (int v = tid; v < V; v += kThreads) {
    const uint32_t k = key_of(load_logit<HALF>(row, v));
    best = max(best, (static_cast<unsigned long long>(k < kNegInf ? 0xffffffffu : k) << 32) | static_cast<uint32_t>(~v));
    finite += k > kNegInf ? 1 : 0;
  }
  best = block_max_u(S, best);
  finite = block_sum_u(S, finite);
  const uint32_t max_key = static_cast<uint32_t>(best >> 32);
  if (max_key >= kPosInf || finite == 0 || !(R.temperature >= 0.f) || R.temperature == INFINITY) {
    give_all(-1, 0);
    return;
  }
  if (R.temperature == 0.f || R.top_k == 1 || R.top_p <= 0.f) {
    give_all(static_cast<int>(~static_cast<uint32_t>(best)), 1);
    return;
  }
  const Term e = term_of(logit_of(max_key), R.temperature, L.table);
  const Bracketed bracketed = bracket_row<HALF>(L, list, row, V, R, e, logit_of(max_key), finite);
  // ---- top-k: the k-th largest key, eight bits at a time
  Border border{kNegInf + 1, 0x7fffffff};
  if (bracketed.there) border = bracketed.border;
  if (!bracketed.there && R.top_k > 0 && static_cast<unsigned long long>(R.top_k) < finite) {
    uint32_t prefix = 0;
    unsigned left = static_cast<unsigned>(R.top_k);
    for (int shift = 24; shift >= 0; shift -= 8) {
      __syncthreads();
      if (tid < 256) S.count[tid] = 0;
      __syncthreads();
      for (int v = tid; v < V; v += kThreads) {
        const uint32_t k = key_of(load_logit<HALF>(row, v));
        if (shift == 24 || (k >> (shift + 8)) == (prefix >> (shift + 8))) atomicAdd(&S.count[(k >> shift) & 255u], 1u);
      }
      __syncthreads();
      if (tid == 0) {
        unsigned n = left;
        int b = 255;
        while (b > 0 && S.count[b] < n) n -= S.count[b--];
        S.pick = b;
        S.left = n;
      }
      __syncthreads();
      prefix |= S.pick << shift;
      left = S.left;
    }
    border = Border{prefix, static_cast<int>(left)};
  }
  const Border by_count = border;
  // ---- top-p: bit by bit by sums in fixed point, which only lead the way; the sum above the key it comes to is fp64 and decides
  if (!bracketed.there && R.top_p < 1.f) {
    double mine = 0.0;
    for (int v = tid; v < V; v += kThreads) {
      const float x = load_logit<HALF>(row, v);
      const uint32_t k = key_of(x);
      if (k > by_count.key || (k == by_count.key && by_count.ties == 0x7fffffff)) mine += e(x);
    }
    double total = block_sum(S, mine);
    if (by_count.ties != 0x7fffffff) total += by_count.ties * e(logit_of(by_count.key));
    const double target = static_cast<double>(R.top_p) * total;
    const double scale = ldexp(1.0, 62 - (32 - __clz(V)));
    uint32_t prefix = 0;
    double left = target;
    for (int shift = 24; shift >= 0; shift -= 8) {
      __syncthreads();
      if (tid < 256) S.mass[tid] = 0;
      __syncthreads();
      for (int v = tid; v < V; v += kThreads) {
        const float x = load_logit<HALF>(row, v);
        const uint32_t k = key_of(x);
        if (k > kNegInf && k >= by_count.key && (shift == 24 || (k >> (shift + 8)) == (prefix >> (shift + 8))))
          atomicAdd(&S.mass[(k >> shift) & 255u], static_cast<unsigned long long>(e(x) * scale));
      }
      __syncthreads();
      if (tid == 0) {
        double n = left;
        int b = 255, last = 255;
        for (; b >= 0; --b) {
          if (S.mass[b] == 0) continue;
          last = b;
          const double m = static_cast<double>(S.mass[b]) / scale;
          if (m >= n) break;
          n -= m;
        }
        S.pick = b < 0 ? last : b;
        S.above = b < 0 ? 0.0 : n;
      }
      __syncthreads();
      prefix |= S.pick << shift;
      left = S.above;
    }
    // The border's key has to have  above < target <= above + all of it: else to its neighbour on that side, and, where that is
    // not enough (tails of tokens too light for the fixed point), by halves.
    uint32_t key = prefix, low = kNegInf, high = max_key + 1;   // (the border lies between the last two)
    Border by_sum = by_count;
    for (int tries = 0; tries < 48; ++tries) {
      double sum = 0.0;
      unsigned long long equal = 0, up = 0xffffffffu, down = 0;
      for (int v = tid; v < V; v += kThreads) {
        const float x = load_logit<HALF>(row, v);
        const uint32_t k = key_of(x);
        if (k > key) {
          sum += e(x);
          up = min(up, static_cast<unsigned long long>(k));
        } else if (k == key) {
          ++equal;
        } else if (k >= by_count.key) {
          down = max(down, static_cast<unsigned long long>(k));
        }
      }
      sum = block_sum(S, sum);
      equal = block_sum_u(S, equal);
      if (key == by_count.key && by_count.ties != 0x7fffffff) equal = by_count.ties;
      up = 0xffffffffu - block_max_u(S, 0xffffffffu - up);
      down = block_max_u(S, down);
      const double one = e(logit_of(key)), all = sum + static_cast<double>(equal) * one;
      if (sum >= target && up != 0xffffffffu) {
        low = key;
        key = tries < 4 || high - low < 4 ? static_cast<uint32_t>(up) : low + (high - low) / 2;
      } else if (all < target && down > kNegInf) {
        high = key;
        key = tries < 4 || high - low < 4 ? static_cast<uint32_t>(down) : low + (high - low) / 2;
      } else if (equal == 0) {
        key = static_cast<uint32_t>(up);
      } else {
        double n = ceil((target - sum) / one);
        if (!(n >= 1.0)) n = 1.0;
        unsigned long long m = n < static_cast<double>(equal) ? static_cast<unsigned long long>(n) : equal;
        while (m > 1 && sum + static_cast<double>(m - 1) * one >= target) --m;
        while (m < equal && sum + static_cast<double>(m) * one < target) ++m;
        by_sum = Border{key, static_cast<int>(m > 0 ? m : 1)};
        break;
      }
    }
    if (less(by_sum, border)) border = by_sum;
  }
  // ---- min-p
  const Border by_size{min_p_key(e, R.temperature, R.min_p, max_key), 0x7fffffff};
  bool counted = bracketed.there;
  if (less(by_size, border)) { border = by_size; counted = false; }
  if (static_cast<double>(R.min_p) > 1.0) { border = Border{max_key, 1}; counted = false; }

  // ---- how many are kept, and the index up to which tokens with the border's key are
  unsigned long long above = 0, equal = 0;
  int cut = V;
  if (counted) {
    above = bracketed.kept;
    cut = bracketed.cut;
  } else {
    for (int v = tid; v < V; v += kThreads) {
      const uint32_t k = key_of(load_logit<HALF>(row, v));
      above += k > border.key ? 1 : 0;
      equal += k == border.key ? 1 : 0;
    }
    above = block_sum_u(S, above);
    equal = block_sum_u(S, equal);
  }
  if (equal > static_cast<unsigned long long>(border.ties)) {
    // index of the ties-th: stretches of tokens per thread, counted in order
    const int stretch = (V + kThreads - 1) / kThreads, v0 = min(tid * stretch, V), v1 = min(v0 + stretch, V);
    unsigned mine = 0;
    for (int v = v0; v < v1; ++v) mine += key_of(load_logit<HALF>(row, v)) == border.key ? 1 : 0;
    unsigned incl = mine;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const unsigned x = __shfl_up_sync(0xffffffffu, incl, o);
      if (lane >= o) incl += x;
    }
    __syncthreads();
    if (lane == 31) S.u[warp] = incl;
    __syncthreads();
    for (int w = 0; w < warp; ++w) incl += static_cast<unsigned>(S.u[w]);
    unsigned n = incl - mine;
    const unsigned ties = static_cast<unsigned>(border.ties);
    if (n < ties && incl >= ties) {
      for (int v = v0; v < v1; ++v)
        if (key_of(load_logit<HALF>(row, v)) == border.key && ++n == ties) { S.cut = v; break; }
    }
    __syncthreads();
    cut = S.cut;
    equal = ties;
  }
  if (tid == 0 && A.kept_out) A.kept_out[s] = static_cast<int>(above + equal);
  if (d1 <= d0) return;

  // ---- sums of the kept tokens, segment by segment
  auto kept_term = [&](int v) -> double {
    if (v >= V) return 0.0;
    const float x = load_logit<HALF>(row, v);
    const uint32_t k = key_of(x);
    return k > border.key || (k == border.key && v <= cut) ? e(x) : 0.0;
  };
  const int n_seg = (V + kSeg - 1) / kSeg;
  for (int g = warp; g < n_seg; g += kWarps) {
    double sum = 0.0;
    for (int x = lane; x < kSeg; x += 32) sum += kept_term(g * kSeg + x);
    sum = warp_sum_d(sum);
    if (lane == 0) S.seg[g] = sum;
  }
  __syncthreads();
  if (warp == 0) {
    double run = 0.0;
    for (int g0 = 0; g0 < n_seg; g0 += 32) {
      const double incl = warp_scan_d(g0 + lane < n_seg ? S.seg[g0 + lane] : 0.0, lane) + run;
      if (g0 + lane < n_seg) S.seg[g0 + lane] = incl;
      run = __shfl_sync(0xffffffffu, incl, 31);
    }
  }
  __syncthreads();
  const double total = S.seg[n_seg - 1];
  for (int64_t d = d0 + warp; d < d1; d += kWarps) {
    const float u = A.uniforms[d];
    const double target = (u < 1.f ? fmaxf(u, 0.f) : 1.f) * total;
    int lo = 0, hi = n_seg;                                    // the first segment whose end exceeds the target
    while (lo < hi) {
      const int mid = (lo + hi) >> 1;
      if (S.seg[mid] > target) hi = mid; else lo = mid + 1;
    }
    if (lo == n_seg) {                                         // none: the last one that adds something
      lo = n_seg - 1;
      while (lo > 0 && !(S.seg[lo] > S.seg[lo - 1])) --lo;
    }
    double run = lo > 0 ? S.seg[lo - 1] : 0.0;
    int token = -1, last = -1;
    for (int x = 0; x < kSeg && token < 0; x += 32) {
      const int v = lo * kSeg + x + lane;
      const double t = kept_term(v);
      const double incl = warp_scan_d(t, lane) + run;
      const unsigned over = __ballot_sync(0xffffffffu, t > 0.0 && incl > target), any = __ballot_sync(0xffffffffu, t > 0.0);
      if (over) token = lo * kSeg + x + __ffs(over) - 1;
      if (any) last = lo * kSeg + x + 31 - __clz(any);
      run = __shfl_sync(0xffffffffu, incl, 31);
    }
    if (lane == 0) {
      A.tokens_out[d] = token >= 0 ? token : last;             // (the two sums of a segment may differ in their last bits)
      if (A.seq_out) A.seq_out[d] = s;
    }
  }
  __syncthreads();
}

// The rows that were split, from the lists of their parts, and all that a list was not enough for.
struct FinishShared {
  union {
    unsigned long long list[kCap];
    WholeShared whole;
  };
  ListShared S;
};
template <bool HALF>
__global__ void __launch_bounds__(kListThreads, 2) finish_rows_kernel(const __grid_constant__ Args A) {
  ss::grid_dependency_enter();
  static_assert(kThreads == kListThreads, "the threads of a list go through whole rows");
  extern __shared__ __align__(16) unsigned char smem[];
  FinishShared& M = *reinterpret_cast<FinishShared*>(smem);
  const int tid = threadIdx.x;
  M.S.count[tid] = 0;
  for (int x = 0; x < 3; ++x) M.S.part[x][tid] = 0;
  make_table(M.S.table);
  __syncthreads();
  for (int s = A.whole_rows + blockIdx.x; s < A.n_seq; s += gridDim.x) {
    const int64_t d0 = __ldg(A.draw_offsets + s), d1 = __ldg(A.draw_offsets + s + 1);
    if (d1 <= d0 && !A.kept_out) continue;
    const RowParams R = row_params(A, s);
    const Part* parts = A.part + static_cast<int64_t>(s - A.whole_rows) * A.parts;
    const bool add_up = kind_of(R, A.vocab).add_up;
    // a lane a part (every warp for itself): counts, sums, in the order of the parts
    const int lane = tid & 31, warp = tid >> 5;
    const bool has = lane < A.parts;
    const unsigned m = has ? parts[lane].n : 0;
    unsigned first = m;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const unsigned up = __shfl_up_sync(0xffffffffu, first, o);
      if (lane >= o) first += up;
    }
    const unsigned n = __shfl_sync(0xffffffffu, first, 31);
    first -= m;
    const bool fits = __all_sync(0xffffffffu, m <= kPartCap) && n <= kCap;
    float mx = has ? parts[lane].max : -INFINITY;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) mx = max_nan(mx, __shfl_xor_sync(0xffffffffu, mx, o));
    // (the largest base is that of all: a part far below it adds nothing, and no factor exceeds 1)
    const float low = warp_max(has ? parts[lane].low : kLowest), base = warp_max(has ? parts[lane].base : -INFINITY);
    const double mine = has && add_up ? parts[lane].sum * exp2(static_cast<double>(parts[lane].base) - static_cast<double>(base)) : 0.0;
    const double z = warp_sum_d(mine);
    const double far = warp_sum_d(mine != 0.0 ? mine * fabs(static_cast<double>(parts[lane].max) * quick_c(R) - parts[lane].base) : 0.0) / z;
    if (fits) {
      for (int p = warp; p < A.parts; p += kListWarps) {
        const unsigned count = __shfl_sync(0xffffffffu, m, p), to = __shfl_sync(0xffffffffu, first, p);
        for (unsigned i = lane; i < count; i += 32) M.list[to + i] = parts[p].list[i];
      }
    }
    __syncthreads();
    const bool done = list_row<HALF>(A, M.S, M.list, s, d0, d1, R, fits ? static_cast<int>(n) : 0, fits, low, mx, z, base, far);
    __syncthreads();
    if (!done) {
      whole_row<HALF>(A, M.whole, M.S, M.list, s);
      __syncthreads();
    }
  }
  // the marks of 32 rows of this block at a time
  for (int64_t s0 = blockIdx.x; s0 < A.whole_rows; s0 += static_cast<int64_t>(gridDim.x) * 32) {
    const int64_t mine = s0 + static_cast<int64_t>(tid & 31) * gridDim.x;
    unsigned marked = __ballot_sync(0xffffffffu, mine < A.whole_rows && A.marks[mine] != 0);
    for (; marked; marked &= marked - 1) {
      whole_row<HALF>(A, M.whole, M.S, M.list, static_cast<int>(s0 + static_cast<int64_t>(__ffs(marked) - 1) * gridDim.x));
      __syncthreads();
    }
  }
}

static int32_t check(const ss_sample_desc_t* d) {
  if (!d || d->struct_size != sizeof(ss_sample_desc_t) || d->flags) return SS_ERR_INVALID_ARG;
  if (d->n_seq < 0 || d->vocab < 1 || d->row_stride < d->vocab) return SS_ERR_INVALID_ARG;
  if (d->logits_type != SS_LOGITS_FP32 && d->logits_type != SS_LOGITS_BF16) return SS_ERR_INVALID_ARG;
  if (d->vocab > kMaxVocab) return SS_ERR_UNSUPPORTED;
  return SS_OK;
}
static size_t carve(const ss_sample_desc_t* d, void* base, Args* A) {
  Carver c(base);
  A->marks = c.take<int32_t>(static_cast<size_t>(d->n_seq) + 1);
  A->part = c.take<Part>(2 * static_cast<size_t>(sm_count_of_current_device()));
  return c.off;
}
template <typename Kernel>
static int32_t prepare(Kernel kernel, size_t smem, bool (&done)[kDeviceSlots]) {
  const int slot = current_device_slot();
  if (slot >= 0 && done[slot]) return SS_OK;
  if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(smem)) != cudaSuccess) {
    (void)cudaGetLastError();
    return SS_ERR_CUDA;
  }
  if (slot >= 0) done[slot] = true;
  return SS_OK;
}
// Whole rounds of a row per block, what is left over in parts (of 4096 tokens at least; none where they would be only one), then the
// kernel that finishes what these leave.
template <bool HALF>
static int32_t launch(Args A, cudaStream_t st) {
  static bool done_rows[kDeviceSlots] = {false}, done_finish[kDeviceSlots] = {false};
  int32_t rc = prepare(list_rows_kernel<HALF>, sizeof(RowsShared), done_rows);
  if (rc == SS_OK) rc = prepare(finish_rows_kernel<HALF>, sizeof(FinishShared), done_finish);
  if (rc != SS_OK) return rc;
  const int blocks = 2 * sm_count_of_current_device();
  A.whole_rows = A.n_seq / blocks * blocks;
  int rest = A.n_seq - A.whole_rows;
  A.parts = rest > 0 && A.vocab > kCap ? blocks / rest : 1;
  if (A.parts > A.vocab / 4096) A.parts = A.vocab / 4096;
  if (A.parts > 32) A.parts = 32;                              // (a lane each)
  if (A.parts < 2) {
    A.parts = 1;
    A.whole_rows = A.n_seq;
    rest = 0;
  }
  const int grid = A.whole_rows >= blocks ? blocks : A.whole_rows > rest * A.parts ? A.whole_rows : rest * A.parts;
  SS_LAUNCH(list_rows_kernel<HALF>, grid, kListThreads, sizeof(RowsShared), st, A);
  const int finish = A.n_seq < blocks ? A.n_seq : blocks;      // (two blocks an SM here as well)
  SS_LAUNCH(finish_rows_kernel<HALF>, finish, kListThreads, sizeof(FinishShared), st, A);
  return SS_OK;
}

}  // namespace filtered
}  // namespace ss

extern "C" int32_t ss_filtered_sample_workspace_bytes(const ss_sample_desc_t* desc, size_t* out_bytes) {
  using namespace ss::filtered;
  if (!out_bytes) return SS_ERR_INVALID_ARG;
  const int32_t rc = check(desc);
  if (rc != SS_OK) return rc;
  Args A = {};
  *out_bytes = carve(desc, nullptr, &A);
  return SS_OK;
}

extern "C" int32_t ss_filtered_sample(const ss_sample_desc_t* d, void* workspace, size_t workspace_bytes, void* stream) {
  using namespace ss::filtered;
  const int32_t rc = check(d);
  if (rc != SS_OK) return rc;
  if (!workspace || reinterpret_cast<uintptr_t>(workspace) % ss::kAlign) return SS_ERR_INVALID_ARG;
  Args A = {};
  if (workspace_bytes < carve(d, workspace, &A)) return SS_ERR_WORKSPACE_TOO_SMALL;
  if (d->n_seq == 0) return SS_OK;
  if (!d->logits || !d->draw_offsets) return SS_ERR_INVALID_ARG;
  if (reinterpret_cast<uintptr_t>(d->logits) % (d->logits_type == SS_LOGITS_BF16 ? 2 : 4)) return SS_ERR_UNSUPPORTED;
  A.logits = d->logits;
  A.draw_offsets = d->draw_offsets;
  A.uniforms = d->uniforms;
  A.temperature = d->temperature;
  A.top_k = d->top_k;
  A.top_p = d->top_p;
  A.min_p = d->min_p;
  A.tokens_out = d->tokens_out;
  A.seq_out = d->seq_out;
  A.kept_out = d->kept_out;
  A.row_stride = d->row_stride;
  A.temperature_all = d->temperature_all;
  A.top_p_all = d->top_p_all;
  A.min_p_all = d->min_p_all;
  A.top_k_all = d->top_k_all;
  A.n_seq = d->n_seq;
  A.vocab = d->vocab;
  return d->logits_type == SS_LOGITS_BF16 ? launch<true>(A, ss::as_stream(stream)) : launch<false>(A, ss::as_stream(stream));
}
