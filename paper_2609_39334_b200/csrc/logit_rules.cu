// ss_logit_rules: penalties of repeated tokens, biases and grammar masks on rows of logits.
//
//   x -> x / r or x * r where the token is in the prompt or the history, - frequency * count - presence, + bias; -inf where not allowed
//
// Few tokens of a vocabulary have rules, so the work is split:
//   rules_copy_kernel   every logit as it is, or -inf; 16 bytes at a time (not launched in place without masks).  Bound: HBM
//   rules_list_kernel   the tokens of a row's lists: counted in a table in shared memory, then each written once, from the input.  Short lists in
//                       a hash table by one block of the row's, longer ones in windows of the vocabulary by all of them.  Bound: latency, and
//                       behind a large copy the scattered sectors (a million for 922 rows: 72 us of the call's 274, the copy 160 at 7 TB/s)
// (One kernel with a table for each chunk of a row, rules applied to the vectors as they pass by: 516 us for 922 rows of 151936 with lists of
// 1000 tokens, where three in five warps meet a token with rules and then divide for all of them; the lists gone through twice around the
// copy: 580, a chunk's phases one after the other.)
#include "common.cuh"

namespace ss {
namespace rules {

constexpr int kCopyThreads = 256, kCopyAhead = 8;              // vectors of a thread
constexpr int kThreads = 512;
constexpr int kTable = 49152;                  // bytes of shared memory of the list kernel
constexpr int kSlots = 4096;                   // of the hash table: a token, its word, its bias entry
constexpr int kMostHashed = 2816;              // entries of a row's lists that it takes
constexpr int64_t kMostEntries = 0x7fffffff - 4 * kThreads;    // of a list; a thread's next quad has to fit 32 bits
constexpr int kPartTokens = kTable / 4;        // a row has a block of the list kernel for so many tokens of the vocabulary, or fewer blocks
static_assert(kSlots * 12 <= kTable && kTable / 4 / kThreads <= 32, "tables");

struct List { const int32_t* tokens; const int64_t* offsets; const int32_t* of; int n; };
struct Args {
  const void* logits;
  void* out;
  int64_t row_stride, out_stride, mask_stride;
  int vocab, chunk, chunks, parts;
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
  const int64_t lo = __ldg(L.offsets + i), hi = __ldg(L.offsets + i + 1);
  return {lo, hi < lo ? lo : hi};
}
__device__ __forceinline__ const uint32_t* mask_of_row(const Args& A, int row) {
  if (!A.masks) return nullptr;
  const int m = A.mask_of ? __ldg(A.mask_of + row) : row;
  return m >= 0 && m < A.n_masks ? A.masks + m * A.mask_stride : nullptr;
}
__device__ __forceinline__ bool allowed(const uint32_t* mask, int token) { return !mask || ((__ldg(mask + (token >> 5)) >> (token & 31)) & 1u); }

template <typename T> __device__ __forceinline__ float to_float(T x);
template <> __device__ __forceinline__ float to_float(float x) { return x; }
template <> __device__ __forceinline__ float to_float(__nv_bfloat16 x) { return __bfloat162float(x); }
template <typename T> __device__ __forceinline__ T from_float(float x);
template <> __device__ __forceinline__ float from_float(float x) { return x; }
template <> __device__ __forceinline__ __nv_bfloat16 from_float(float x) { return __float2bfloat16_rn(x); }

template <typename T>
__global__ void __launch_bounds__(kCopyThreads) rules_copy_kernel(const __grid_constant__ Args A) {
  ss::grid_dependency_enter();
  constexpr int kVec = 16 / sizeof(T);
  const int row = blockIdx.x / A.chunks, chunk = blockIdx.x - row * A.chunks, tid = threadIdx.x;
  const T* in = static_cast<const T*>(A.logits) + row * A.row_stride;
  T* out = static_cast<T*>(A.out) + row * A.out_stride;
  const bool same = static_cast<const void*>(in) == static_cast<const void*>(out);
  const uint32_t* mask = mask_of_row(A, row);
  if (same && !mask) return;
  // this block's tokens: from the row's first 16-byte boundary on in chunks, what lies in front of it with the first
  const int head = min(A.vocab, static_cast<int>((16 - (reinterpret_cast<uintptr_t>(in) & 15)) & 15) / static_cast<int>(sizeof(T)));
  const int first = head + chunk * A.chunk, end = min(A.vocab, first + A.chunk);
  const int n_vec = ((reinterpret_cast<uintptr_t>(in) ^ reinterpret_cast<uintptr_t>(out)) & 15) == 0 && end > first ? (end - first) / kVec : 0;
  uint4 raw[kCopyAhead];
#pragma unroll
  for (int x = 0; x < kCopyAhead; ++x)
    if (tid + x * kCopyThreads < n_vec) raw[x] = *reinterpret_cast<const uint4*>(in + first + (tid + x * kCopyThreads) * kVec);
#pragma unroll
  for (int x = 0; x < kCopyAhead; ++x) {
    const int v = tid + x * kCopyThreads, token = first + v * kVec;
    if (v >= n_vec) continue;
    if (mask) {
      const int at = token >> 5, sh = token & 31;
      uint32_t bits = __ldg(mask + at) >> sh;
      if (sh > 32 - kVec) bits |= __ldg(mask + at + 1) << (32 - sh);
      uint32_t* e = reinterpret_cast<uint32_t*>(&raw[x]);
#pragma unroll
      for (int y = 0; y < 4; ++y) {
        if (sizeof(T) == 4) {
          e[y] = (bits >> y) & 1u ? e[y] : 0xff800000u;        // -inf
        } else {
          const uint32_t keep = ((bits >> (2 * y)) & 1u ? 0xffffu : 0u) | ((bits >> (2 * y)) & 2u ? 0xffff0000u : 0u);
          e[y] = (e[y] & keep) | (0xff80ff80u & ~keep);
        }
      }
      if (same && (~bits & ((1u << kVec) - 1u)) == 0) continue;
    }
    *reinterpret_cast<uint4*>(out + token) = raw[x];
  }
  auto copy = [&](int token) {
    const bool yes = allowed(mask, token);
    if (!same || !yes) out[token] = yes ? in[token] : from_float<T>(-INFINITY);
  };
  if (chunk == 0 && tid < head) copy(tid);
  for (int t = first + n_vec * kVec + tid; t < end; t += kCopyThreads) copy(t);
}

struct Row { float r, frequency, presence; };
// A token's logit by its rules: how often it is in the history, whether it is in the prompt, its bias or null.
__device__ __forceinline__ float ruled(float x, const Row& R, uint32_t count, bool in_prompt, const float* bias) {
  if (count || in_prompt) x = x > 0.f ? __fdiv_rn(x, R.r) : x * R.r;
  if (count) x = fmaf(-R.frequency, static_cast<float>(count), x) - R.presence;
  if (bias) x += __ldg(bias);
  return x;
}

constexpr uint32_t kInPrompt = 0x80000000u;    // the top bit of a token's word; the rest: how often it is in the history

// (Its code runs once or twice a block, so it is short: nothing is unrolled but the four tokens of a load, one loop goes through all three lists and
// serves both tables.  With a loop for each, four loads ahead, the call took 21 us for eight rows instead of 15.  Three blocks fit an SM beside their
// tables; bounded to three it has 40 registers instead of 23, and takes as long.)
template <typename T>
__global__ void __launch_bounds__(kThreads, 4) rules_list_kernel(const __grid_constant__ Args A) {
  ss::grid_dependency_enter();
  extern __shared__ uint4 smem[];
  __shared__ uint16_t list[kTable / 4];
  __shared__ int n_found;
  const int row = blockIdx.x / A.parts, part = blockIdx.x - row * A.parts, tid = threadIdx.x, lane = tid & 31;
  Range range[3] = {range_of(A.history, row), range_of(A.prompts, row), range_of(A.bias, row)};
  Row R;
  R.r = A.repetition ? __ldg(A.repetition + row) : A.repetition_all;
  R.frequency = A.frequency ? __ldg(A.frequency + row) : A.frequency_all;
  R.presence = A.presence ? __ldg(A.presence + row) : A.presence_all;
  if (!(R.r > 0.f)) R.r = 1.f;
  if (R.r == 1.f) range[1].hi = range[1].lo;   // (lists without an effect are none)
  if (R.r == 1.f && R.frequency == 0.f && R.presence == 0.f) range[0].hi = range[0].lo;
  const int64_t entries = range[0].hi - range[0].lo + (range[1].hi - range[1].lo) + (range[2].hi - range[2].lo);
  const bool hashed = entries <= kMostHashed, biased = range[2].lo < range[2].hi;
  if (entries == 0 || (hashed && part > 0)) return;
  const T* in = static_cast<const T*>(A.logits) + row * A.row_stride;
  T* out = static_cast<T*>(A.out) + row * A.out_stride;
  const uint32_t* mask = mask_of_row(A, row);
  const float* values = A.bias_values + range[2].lo;

  // Words of tokens, the last bias entry plus 1 of each, and (hashed) which tokens they are.  Hashed: one window, the vocabulary.
  const int window = hashed ? A.vocab : kTable / (biased ? 8 : 4), places = hashed ? kSlots : window, each = places / kThreads;
  uint32_t* word = reinterpret_cast<uint32_t*>(smem);
  uint32_t* entry = word + places;
  int* key = reinterpret_cast<int*>(entry + places);
  for (int64_t first64 = static_cast<int64_t>(part) * window; first64 < A.vocab; first64 += static_cast<int64_t>(A.parts) * window) {
    const int first = static_cast<int>(first64);
    // (In 64 bits: of min(window, A.vocab - first) in 32, signed or not, nvcc 12.9 made code for a bound of three blocks that went on with the first
    // window's number in the last one, and so wrote tokens behind the vocabulary behind the row.  This is right with either bound.)
    const uint32_t count = static_cast<uint32_t>(min(static_cast<int64_t>(window), A.vocab - first64));
#pragma unroll 1
    for (int i = tid; i < kTable / 16; i += kThreads) smem[i] = hashed && i >= 2 * kSlots / 4 ? make_uint4(~0u, ~0u, ~0u, ~0u) : make_uint4(0, 0, 0, 0);
    if (tid == 0) n_found = 0;
    __syncthreads();
    // entry i of list `kind`, whose token is the window's d-th
    auto note = [&](int kind, uint32_t d, int i) {
      if (hashed) {                            // (fewer tokens than slots: it ends)
        const int token = static_cast<int>(d);
        d = (d * 2654435769u) >> 20;
        static_assert(kSlots == 1 << 12, "bits of a slot");
        for (;; d = (d + 1) & (kSlots - 1)) {
          const int was = atomicCAS(key + d, -1, token);
          if (was == -1 || was == token) break;
        }
      }
      if (kind == 0) atomicAdd(word + d, 1u);
      else if (kind == 2) atomicMax(entry + d, static_cast<uint32_t>(i) + 1u);
      else if (!(word[d] & kInPrompt)) atomicOr(word + d, kInPrompt);
    };
#pragma unroll 1
    for (int kind = 0; kind < 3; ++kind) {
      const int32_t* tokens = (kind == 0 ? A.history.tokens : kind == 1 ? A.prompts.tokens : A.bias.tokens) + range[kind].lo;
      const int n = static_cast<int>(min(range[kind].hi - range[kind].lo, kMostEntries));
      // quads on 16-byte boundaries; the first and the last may reach over the list's ends, and take the tokens that are there
      const int skew = static_cast<int>((reinterpret_cast<uintptr_t>(tokens) & 15) / 4);
#pragma unroll 1
      for (int i0 = 4 * tid - skew; i0 < n; i0 += 4 * kThreads) {
        int q[4];
        if (i0 >= 0 && i0 + 4 <= n) {
          const int4 v = __ldg(reinterpret_cast<const int4*>(tokens + i0));
          q[0] = v.x; q[1] = v.y; q[2] = v.z; q[3] = v.w;
        } else {
#pragma unroll
          for (int y = 0; y < 4; ++y) q[y] = i0 + y >= 0 && i0 + y < n ? __ldg(tokens + i0 + y) : -1;
        }
        // (a token in front of the window, or none, comes out as a large difference)
        uint32_t hit = 0;
#pragma unroll
        for (int y = 0; y < 4; ++y) hit |= (static_cast<uint32_t>(q[y]) - static_cast<uint32_t>(first) < count ? 1u : 0u) << y;
        for (; hit; hit &= hit - 1) {
          const int y = __ffs(hit) - 1;
          note(kind, static_cast<uint32_t>((y & 2 ? (y & 1 ? q[3] : q[2]) : (y & 1 ? q[1] : q[0])) - first), i0 + y);
        }
      }
    }
    __syncthreads();

    // ---- the places that hold something, on a list, so that no thread works on a token without rules beside others
    uint32_t found = 0;
#pragma unroll 1
    for (int x = 0; x < each; ++x) {
      const int at = x * kThreads + tid;
      found |= (word[at] || ((hashed || biased) && entry[at]) ? 1u : 0u) << x;
    }
    int n = __popc(found), incl = n;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int up = __shfl_up_sync(0xffffffffu, incl, o);
      if (lane >= o) incl += up;
    }
    int base = 0;
    if (lane == 31) base = atomicAdd(&n_found, incl);
    int to = __shfl_sync(0xffffffffu, base, 31) + incl - n;
    for (; found; found &= found - 1) list[to++] = static_cast<uint16_t>((__ffs(found) - 1) * kThreads + tid);
    __syncthreads();
    // ---- their tokens' logits, once (in place: what is allowed is as it was)
    n = n_found;
#pragma unroll 2
    for (int i = tid; i < n; i += kThreads) {
      const int at = list[i], token = hashed ? key[at] : first + at;
      const uint32_t w = word[at], b = hashed || biased ? entry[at] : 0u;
      const T x = in[token];
      if (allowed(mask, token))
        out[token] = from_float<T>(ruled(to_float<T>(x), R, w & ~kInPrompt, (w & kInPrompt) != 0, b ? values + (b - 1) : nullptr));
    }
    __syncthreads();
  }
}

template <typename T>
static int32_t launch(const Args& A, int64_t rows, bool copy, bool lists, cudaStream_t st) {
  if (copy) SS_LAUNCH(rules_copy_kernel<T>, static_cast<unsigned>(rows * A.chunks), kCopyThreads, 0, st, A);
  if (!lists) return SS_OK;
  static bool done[kDeviceSlots] = {false};
  const int slot = current_device_slot();
  if (slot < 0 || !done[slot]) {
    if (cudaFuncSetAttribute(rules_list_kernel<T>, cudaFuncAttributeMaxDynamicSharedMemorySize, kTable) != cudaSuccess) {
      (void)cudaGetLastError();
      return SS_ERR_CUDA;
    }
    if (slot >= 0) done[slot] = true;
  }
  SS_LAUNCH(rules_list_kernel<T>, static_cast<unsigned>(rows * A.parts), kThreads, kTable, st, A);
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
  A.chunk = kCopyThreads * kCopyAhead * 16 / size;
  A.chunks = (r->vocab + A.chunk - 1) / A.chunk;
  // (of a row with short lists all blocks but one leave at once, which costs where there are many)
  A.parts = (r->vocab + kPartTokens - 1) / kPartTokens;
  while (A.parts > 1 && static_cast<int64_t>(r->n_seq) * A.parts > 16LL * ss::sm_count_of_current_device()) A.parts = (A.parts + 1) / 2;
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
  if (static_cast<int64_t>(r->n_seq) * (A.chunks > A.parts ? A.chunks : A.parts) > 0x7fffffffLL) return SS_ERR_UNSUPPORTED;
  cudaStream_t st = ss::as_stream(stream);
  const bool copy = r->out != r->logits || r->masks, lists = A.history.offsets || A.prompts.offsets || A.bias.offsets;
  return r->logits_type == SS_LOGITS_BF16 ? launch<__nv_bfloat16>(A, r->n_seq, copy, lists, st) : launch<float>(A, r->n_seq, copy, lists, st);
}
