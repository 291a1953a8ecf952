// ss_logit_rules: penalties of repeated tokens, biases and grammar masks on rows of logits.
//
//   x -> x / r or x * r where the token is in the prompt or the history, - frequency * count - presence, + bias; -inf where not allowed
//
// A block takes a chunk of kChunk tokens of a row.  It counts the chunk's tokens of the row's prompt and history in shared memory (a word
// a token: the count, its top bit for the prompt), notes the last bias entry of each, and then goes once through the chunk's logits, 16
// bytes at a time, with the words beside them.
#include "common.cuh"

namespace ss {
namespace rules {

constexpr int kThreads = 512;
constexpr int kChunk = 8192;                   // tokens of a block
constexpr int kSlack = 8;                      // the first block of a row also has what lies in front of a 16-byte boundary
constexpr uint32_t kInPrompt = 0x80000000u;

struct List { const int32_t* tokens; const int64_t* offsets; const int32_t* of; int n; };
struct Args {
  const void* logits;
  void* out;
  int64_t row_stride, out_stride, mask_stride;
  int vocab, chunks;
  List history, prompts, bias;
  const float* bias_values;
  const uint32_t* masks;
  const int32_t* mask_of;
  int n_masks;
  const float *repetition, *frequency, *presence;
  float repetition_all, frequency_all, presence_all;
};

struct Range { int64_t lo, hi; };
// What row s has of a list: entries [lo, hi).
__device__ __forceinline__ Range range_of(const List& L, int s) {
  if (!L.offsets) return {0, 0};
  const int i = L.of ? __ldg(L.of + s) : s;
  if (i < 0 || i >= L.n) return {0, 0};
  return {__ldg(L.offsets + i), __ldg(L.offsets + i + 1)};
}

template <typename T> __device__ __forceinline__ float to_float(T x);
template <> __device__ __forceinline__ float to_float(float x) { return x; }
template <> __device__ __forceinline__ float to_float(__nv_bfloat16 x) { return __bfloat162float(x); }
template <typename T> __device__ __forceinline__ T from_float(float x);
template <> __device__ __forceinline__ float from_float(float x) { return x; }
template <> __device__ __forceinline__ __nv_bfloat16 from_float(float x) { return __float2bfloat16_rn(x); }

struct Row { float r, frequency, presence; };

// f(token of the chunk, entry) for every entry of [lo, hi) whose token is one of the chunk's (whole block).
template <typename F>
__device__ __forceinline__ void for_tokens(const int32_t* tokens, Range e, int first, int count, F f) {
  constexpr int kAhead = 8;
  for (int64_t i0 = e.lo + threadIdx.x; i0 < e.hi; i0 += kAhead * kThreads) {
    int t[kAhead];
#pragma unroll
    for (int x = 0; x < kAhead; ++x) {
      const int64_t i = i0 + static_cast<int64_t>(x) * kThreads;
      t[x] = i < e.hi ? __ldg(tokens + i) - first : -1;
    }
#pragma unroll
    for (int x = 0; x < kAhead; ++x)
      if (static_cast<unsigned>(t[x]) < static_cast<unsigned>(count)) f(t[x], i0 + static_cast<int64_t>(x) * kThreads);
  }
}

__device__ __forceinline__ float ruled(float x, const Row& R, uint32_t seen, const float* bias) {
  if (seen) x = x > 0.f ? __fdiv_rn(x, R.r) : x * R.r;
  const uint32_t c = seen & ~kInPrompt;
  if (c) x = fmaf(-R.frequency, static_cast<float>(c), x) - R.presence;
  if (bias) x += __ldg(bias);
  return x;
}

template <typename T, bool BIAS>
__global__ void __launch_bounds__(kThreads) rules_kernel(const __grid_constant__ Args A) {
  ss::grid_dependency_enter();
  extern __shared__ uint4 table4[];            // the words of the chunk's tokens, then (BIAS) the last bias entry of each, plus 1
  uint32_t* seen = reinterpret_cast<uint32_t*>(table4);
  uint32_t* entry = seen + kChunk + kSlack;
  constexpr int kVec = 16 / sizeof(T);
  const int tid = threadIdx.x;
  const int row = blockIdx.x / A.chunks, chunk = blockIdx.x - row * A.chunks;
  const T* in = static_cast<const T*>(A.logits) + row * A.row_stride;
  T* out = static_cast<T*>(A.out) + row * A.out_stride;
  const bool same = static_cast<const void*>(in) == static_cast<const void*>(out);

  // this block's tokens: from the row's first 16-byte boundary on in chunks, what lies in front of it with the first
  const int head = min(A.vocab, static_cast<int>((16 - (reinterpret_cast<uintptr_t>(in) & 15)) & 15) / static_cast<int>(sizeof(T)));
  const int first = chunk == 0 ? 0 : head + chunk * kChunk, end = min(A.vocab, head + (chunk + 1) * kChunk);
  const int count = end - first;
  if (count <= 0) return;
  const bool vectors = ((reinterpret_cast<uintptr_t>(in) ^ reinterpret_cast<uintptr_t>(out)) & 15) == 0;

  const Range history = range_of(A.history, row), prompt = range_of(A.prompts, row), bias = BIAS ? range_of(A.bias, row) : Range{0, 0};
  const int mask_row = A.masks ? (A.mask_of ? __ldg(A.mask_of + row) : row) : -1;
  const uint32_t* mask = mask_row >= 0 && mask_row < A.n_masks ? A.masks + mask_row * A.mask_stride : nullptr;
  Row R;
  R.r = A.repetition ? __ldg(A.repetition + row) : A.repetition_all;
  R.frequency = A.frequency ? __ldg(A.frequency + row) : A.frequency_all;
  R.presence = A.presence ? __ldg(A.presence + row) : A.presence_all;
  if (!(R.r > 0.f)) R.r = 1.f;
  const bool penal = (R.r != 1.f && (history.lo < history.hi || prompt.lo < prompt.hi)) ||
                     ((R.frequency != 0.f || R.presence != 0.f) && history.lo < history.hi);
  const bool biased = BIAS && bias.lo < bias.hi;
  if (same && !penal && !biased && !mask) return;
  const float* values = A.bias_values + bias.lo;

  if (penal) {
    for (int i = tid; i < (count + 3) / 4; i += kThreads) table4[i] = make_uint4(0, 0, 0, 0);
  }
  if (biased) {
    for (int i = tid; i < (count + 3) / 4; i += kThreads) reinterpret_cast<uint4*>(entry)[i] = make_uint4(0, 0, 0, 0);
  }
  __syncthreads();
  if (penal) {
    for_tokens(A.history.tokens, history, first, count, [&](int t, int64_t) { atomicAdd(seen + t, 1u); });
    if (R.r != 1.f) for_tokens(A.prompts.tokens, prompt, first, count, [&](int t, int64_t) { atomicOr(seen + t, kInPrompt); });
  }
  if (biased) for_tokens(A.bias.tokens, bias, first, count, [&](int t, int64_t i) { atomicMax(entry + t, static_cast<uint32_t>(i - bias.lo) + 1u); });
  __syncthreads();

  auto word_of = [&](int t) { return penal ? seen[t] : 0u; };
  auto entry_of = [&](int t) { return biased ? entry[t] : 0u; };
  auto allowed = [&](int token) { return !mask || ((__ldg(mask + (token >> 5)) >> (token & 31)) & 1u); };
  auto one = [&](int t) {                      // token first + t by itself
    const uint32_t w = word_of(t), b = entry_of(t);
    const bool yes = allowed(first + t);
    if (same && !w && !b && yes) return;
    const float x = to_float<T>(in[first + t]);
    out[first + t] = from_float<T>(yes ? ruled(x, R, w, b ? values + (b - 1) : nullptr) : -INFINITY);
  };
  const int before = chunk == 0 ? min(head, count) : 0;        // tokens in front of the vectors
  const int n_vec = vectors ? (count - before) / kVec : 0;
  for (int v = tid; v < n_vec; v += kThreads) {
    const int t0 = before + v * kVec;
    uint32_t w[kVec], b[kVec], any = 0;
#pragma unroll
    for (int x = 0; x < kVec; ++x) {
      w[x] = word_of(t0 + x);
      b[x] = entry_of(t0 + x);
      any |= w[x] | b[x];
    }
    uint32_t bits = (1u << kVec) - 1u;
    if (mask) {
      const int token = first + t0, at = token >> 5, sh = token & 31;
      uint32_t m = __ldg(mask + at) >> sh;
      if (sh > 32 - kVec) m |= __ldg(mask + at + 1) << (32 - sh);
      bits &= m;
    }
    const bool all = bits == (1u << kVec) - 1u;
    if (same && all && !any) continue;
    uint4 raw = *reinterpret_cast<const uint4*>(in + first + t0);
    if (any || !all) {
      T* e = reinterpret_cast<T*>(&raw);
#pragma unroll
      for (int x = 0; x < kVec; ++x) {
        if (!((bits >> x) & 1u)) e[x] = from_float<T>(-INFINITY);
        else if (w[x] | b[x]) e[x] = from_float<T>(ruled(to_float<T>(e[x]), R, w[x], b[x] ? values + (b[x] - 1) : nullptr));
      }
    }
    *reinterpret_cast<uint4*>(out + first + t0) = raw;
  }
  for (int t = tid; t < before; t += kThreads) one(t);
  for (int t = before + n_vec * kVec + tid; t < count; t += kThreads) one(t);
}

template <typename T, bool BIAS>
static int32_t launch(const Args& A, unsigned blocks, cudaStream_t st) {
  constexpr int kSmem = (kChunk + kSlack) * 4 * (BIAS ? 2 : 1);
  static bool done[kDeviceSlots] = {false};
  const int slot = current_device_slot();
  if (slot < 0 || !done[slot]) {
    if (cudaFuncSetAttribute(rules_kernel<T, BIAS>, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmem) != cudaSuccess) {
      (void)cudaGetLastError();
      return SS_ERR_CUDA;
    }
    if (slot >= 0) done[slot] = true;
  }
  SS_LAUNCH((rules_kernel<T, BIAS>), blocks, kThreads, kSmem, st, A);
  return SS_OK;
}

}  // namespace rules
}  // namespace ss

extern "C" int32_t ss_logit_rules(const ss_logit_rules_t* r, void* stream) {
  using namespace ss::rules;
  if (!r || r->struct_size != sizeof(ss_logit_rules_t) || r->flags) return SS_ERR_INVALID_ARG;
  if (r->n_seq < 0 || r->vocab < 0 || r->n_prompts < 0 || r->n_biases < 0 || r->n_masks < 0) return SS_ERR_INVALID_ARG;
  if (r->logits_type != SS_LOGITS_FP32 && r->logits_type != SS_LOGITS_BF16) return SS_ERR_INVALID_ARG;
  if (r->row_stride < r->vocab || r->out_row_stride < r->vocab) return SS_ERR_INVALID_ARG;
  if (r->vocab > 2097152) return SS_ERR_UNSUPPORTED;
  if (r->n_seq == 0 || r->vocab == 0) return SS_OK;
  if (!r->logits || !r->out || (r->out == r->logits && r->out_row_stride != r->row_stride)) return SS_ERR_INVALID_ARG;
  const int size = r->logits_type == SS_LOGITS_BF16 ? 2 : 4;
  if (reinterpret_cast<uintptr_t>(r->logits) % size || reinterpret_cast<uintptr_t>(r->out) % size) return SS_ERR_INVALID_ARG;
  if ((r->history && !r->history_offsets) || (r->prompts && !r->prompt_offsets) || ((r->bias_tokens || r->bias_values) && !r->bias_offsets))
    return SS_ERR_INVALID_ARG;
  if ((r->bias_tokens != nullptr) != (r->bias_values != nullptr)) return SS_ERR_INVALID_ARG;
  if (r->masks && r->mask_stride < (r->vocab + 31) / 32) return SS_ERR_INVALID_ARG;
  Args A = {};
  A.logits = r->logits;
  A.out = r->out;
  A.row_stride = r->row_stride;
  A.out_stride = r->out_row_stride;
  A.mask_stride = r->mask_stride;
  A.vocab = r->vocab;
  A.chunks = (r->vocab + kChunk - 1) / kChunk;
  A.history = {r->history, r->history ? r->history_offsets : nullptr, nullptr, r->n_seq};
  A.prompts = {r->prompts, r->prompts ? r->prompt_offsets : nullptr, r->prompt_of, r->n_prompts};
  A.bias = {r->bias_tokens, r->bias_tokens ? r->bias_offsets : nullptr, r->bias_of, r->n_biases};
  A.bias_values = r->bias_values;
  A.masks = r->masks;
  A.mask_of = r->mask_of;
  A.n_masks = r->n_masks;
  A.repetition = r->repetition;
  A.frequency = r->frequency;
  A.presence = r->presence;
  A.repetition_all = r->repetition_all;
  A.frequency_all = r->frequency_all;
  A.presence_all = r->presence_all;
  const int64_t blocks = static_cast<int64_t>(r->n_seq) * A.chunks;
  if (blocks > 0x7fffffffLL) return SS_ERR_UNSUPPORTED;
  cudaStream_t st = ss::as_stream(stream);
  const unsigned n = static_cast<unsigned>(blocks);
  if (r->logits_type == SS_LOGITS_BF16) return A.bias.offsets ? launch<__nv_bfloat16, true>(A, n, st) : launch<__nv_bfloat16, false>(A, n, st);
  return A.bias.offsets ? launch<float, true>(A, n, st) : launch<float, false>(A, n, st);
}
