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
constexpr int kThreads = 1024, kWarps = kThreads / 32;         // of a block that goes through whole rows
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

struct Border {
  uint32_t key;                                // tokens above it are kept,
  int ties;                                    // and so many with exactly this key
};
__device__ __forceinline__ bool less(const Border& a, const Border& b) { return a.key > b.key || (a.key == b.key && a.ties < b.ties); }

struct Term {                                  // e_v of a row
  double max, inv_t;
  __device__ __forceinline__ double operator()(float x) const { return exp((static_cast<double>(x) - max) * inv_t); }
};
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
__device__ void whole_row(const Args& A, WholeShared& S, int s) {
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
  Term e;
  e.max = static_cast<double>(logit_of(max_key));
  e.inv_t = 1.0 / static_cast<double>(R.temperature);
  // ---- top-k: the k-th largest key, eight bits at a time
  Border border{kNegInf + 1, 0x7fffffff};
  if (R.top_k > 0 && static_cast<unsigned long long>(R.top_k) < finite) {
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
  if (R.top_p < 1.f) {
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
  if (less(by_size, border)) border = by_size;
  if (static_cast<double>(R.min_p) > 1.0) border = Border{max_key, 1};

  // ---- how many are kept, and the index up to which tokens with the border's key are
  unsigned long long above = 0, equal = 0;
  for (int v = tid; v < V; v += kThreads) {
    const uint32_t k = key_of(load_logit<HALF>(row, v));
    above += k > border.key ? 1 : 0;
    equal += k == border.key ? 1 : 0;
  }
  above = block_sum_u(S, above);
  equal = block_sum_u(S, equal);
  int cut = V;
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

template <bool HALF>
__global__ void __launch_bounds__(kThreads) whole_rows_kernel(const __grid_constant__ Args A) {
  ss::grid_dependency_enter();
  __shared__ WholeShared S;
  for (int s = blockIdx.x; s < A.n_seq; s += gridDim.x) {
    whole_row<HALF>(A, S, s);
    __syncthreads();
  }
}

static int32_t check(const ss_sample_desc_t* d) {
  if (!d || d->struct_size != sizeof(ss_sample_desc_t) || d->flags) return SS_ERR_INVALID_ARG;
  if (d->n_seq < 0 || d->vocab < 1 || d->row_stride < d->vocab) return SS_ERR_INVALID_ARG;
  if (d->logits_type != SS_LOGITS_FP32 && d->logits_type != SS_LOGITS_BF16) return SS_ERR_INVALID_ARG;
  if (d->vocab > kMaxVocab) return SS_ERR_UNSUPPORTED;
  return SS_OK;
}
static size_t workspace_bytes_of(const ss_sample_desc_t* d) { return align_up(sizeof(int32_t) * (static_cast<size_t>(d->n_seq) + 64)); }

}  // namespace filtered
}  // namespace ss

extern "C" int32_t ss_filtered_sample_workspace_bytes(const ss_sample_desc_t* desc, size_t* out_bytes) {
  using namespace ss::filtered;
  if (!out_bytes) return SS_ERR_INVALID_ARG;
  const int32_t rc = check(desc);
  if (rc != SS_OK) return rc;
  *out_bytes = workspace_bytes_of(desc);
  return SS_OK;
}

extern "C" int32_t ss_filtered_sample(const ss_sample_desc_t* d, void* workspace, size_t workspace_bytes, void* stream) {
  using namespace ss::filtered;
  const int32_t rc = check(d);
  if (rc != SS_OK) return rc;
  if (!workspace || reinterpret_cast<uintptr_t>(workspace) % ss::kAlign) return SS_ERR_INVALID_ARG;
  if (workspace_bytes < workspace_bytes_of(d)) return SS_ERR_WORKSPACE_TOO_SMALL;
  if (d->n_seq == 0) return SS_OK;
  if (!d->logits || !d->draw_offsets) return SS_ERR_INVALID_ARG;
  if (reinterpret_cast<uintptr_t>(d->logits) % (d->logits_type == SS_LOGITS_BF16 ? 2 : 4)) return SS_ERR_UNSUPPORTED;
  Args A = {};
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
  const int sms = ss::sm_count_of_current_device();
  const int grid = d->n_seq < 2 * sms ? d->n_seq : 2 * sms;
  if (d->logits_type == SS_LOGITS_BF16) {
    SS_LAUNCH(whole_rows_kernel<true>, grid, kThreads, 0, ss::as_stream(stream), A);
  } else {
    SS_LAUNCH(whole_rows_kernel<false>, grid, kThreads, 0, ss::as_stream(stream), A);
  }
  return SS_OK;
}
