// The next token of each row of logits.
//
// With m the row's largest logit and T its temperature, token i weighs
//   w_i = exp((x_i - m) / T),
// in whole multiples of 2^-44 (64-bit integers): sums of weights are then exact,
// whatever their order, and so is every comparison of a sum with top-p's share or
// with the random number.  The kept tokens are the first ones in the order of
// falling logit, equal ones by rising index; such a set is told by the least key
// in it and how many tokens of that key it has (struct Cut), and the search for
// it goes down the key's bits, 11 at a time, with sums of counts or weights by
// digit in LDS.
//
// One workgroup takes a row.
#include "../../include/entropyinfer.h"
#include "ei_internal.h"

#include <limits.h>
#include <math.h>

namespace ei {
namespace {

constexpr int kThreads = 1024;
constexpr int kWaves = kThreads / kWave;
constexpr int kDigitBits = 11, kDigits = 1 << kDigitBits;
constexpr int kMaxVocab = 1 << 19;   // sums of weights: 2^19 * 2^44 = 2^63
constexpr double kOne = 0x1p44;

struct SampleArgs {
  const void* logits;
  int rows, vocab;
  int64_t stride;
  const float *u, *temperature;
  const int32_t* top_k;
  const float *top_p, *min_p;
  int32_t* tokens;
  float* logprobs;
};

// Logits in their order as unsigned numbers: 0 for -inf and NaN (no token there),
// -0 the same as 0.
__device__ __forceinline__ uint32_t key_of(float x) {
  const uint32_t b = __float_as_uint(x + 0.0f);
  if (!(x > -INFINITY)) return 0;
  return b & 0x80000000u ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float logit_of(uint32_t key) {
  return __uint_as_float(key & 0x80000000u ? key & 0x7fffffffu : ~key);
}

template <int FMT>
__device__ __forceinline__ uint32_t key_at(const SampleArgs& a, int64_t row, int i) {
  if constexpr (FMT == EI_LOGITS_BF16)
    return key_of(__uint_as_float((uint32_t)((const uint16_t*)a.logits)[row * a.stride + i] << 16));
  else
    return key_of(((const float*)a.logits)[row * a.stride + i]);
}

struct Weights {
  float top;       // the largest logit
  double per_t;    // 1 / T
  __device__ __forceinline__ double real(uint32_t key) const {
    const float x = logit_of(key);
    if (x == top) return 1.0;
    return top == INFINITY ? 0.0 : exp(((double)x - (double)top) * per_t);
  }
  __device__ __forceinline__ uint64_t of(uint32_t key) const {
    return (uint64_t)(real(key) * kOne + 0.5);
  }
};

struct Shared {
  uint64_t sums[kDigits];
  uint64_t wave_sum[kWaves];
  uint64_t found_above, found_at;
  uint32_t wave_max[kWaves];
  int found, wave_count[kWaves];
};

__device__ __forceinline__ uint64_t wave_sum_u64(uint64_t v) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o);
  return v;
}
__device__ __forceinline__ uint64_t wave_up_to_u64(uint64_t v, int lane) {
#pragma unroll
  for (int o = 1; o < kWave; o <<= 1) {
    const uint64_t t = __shfl_up(v, o);
    if (lane >= o) v += t;
  }
  return v;
}
__device__ __forceinline__ uint64_t block_sum(Shared& sm, uint64_t v) {
  v = wave_sum_u64(v);
  __syncthreads();
  if (threadIdx.x % kWave == 0) sm.wave_sum[threadIdx.x / kWave] = v;
  __syncthreads();
  uint64_t s = 0;
#pragma unroll
  for (int w = 0; w < kWaves; ++w) s += sm.wave_sum[w];
  return s;
}
// The sum over this thread and those before it.
__device__ __forceinline__ uint64_t block_up_to(Shared& sm, uint64_t v) {
  const int wave = threadIdx.x / kWave;
  v = wave_up_to_u64(v, threadIdx.x % kWave);
  __syncthreads();
  if (threadIdx.x % kWave == kWave - 1) sm.wave_sum[wave] = v;
  __syncthreads();
  for (int w = 0; w < wave; ++w) v += sm.wave_sum[w];
  return v;
}

// The tokens above `key` and the first `count` of those that have it.
struct Cut {
  uint32_t key;
  uint64_t count;
};

// The shortest run of tokens, in their order, of the tokens within `in` whose
// values (1 each, or their weights) add up to `want` (1 at least, and at most the
// sum of all).
template <int FMT, class Value>
__device__ Cut find_cut(Shared& sm, const SampleArgs& a, int64_t row, Cut in, uint64_t want,
                        Value value) {
  uint32_t prefix = 0;
  uint64_t above = 0;
  constexpr int kLow = FMT == EI_LOGITS_BF16 ? 16 : 0;   // (a bf16 key's low bits follow its sign)
  for (int bits = 32; bits > kLow;) {
    const int step = min(bits - kLow, kDigitBits), shift = bits - step;
    for (int d = threadIdx.x; d < kDigits; d += kThreads) sm.sums[d] = 0;
    __syncthreads();
    auto add = [&](uint32_t key, uint64_t v) {
      if (bits < 32 && key >> bits != prefix) return;
      atomicAdd((unsigned long long*)&sm.sums[(key >> shift) & ((1u << step) - 1)],
                (unsigned long long)v);
    };
    for (int i = threadIdx.x; i < a.vocab; i += kThreads) {
      const uint32_t key = key_at<FMT>(a, row, i);
      if (key > in.key) add(key, value(key));
    }
    if (threadIdx.x == 0 && in.key != 0) add(in.key, in.count * value(in.key));
    __syncthreads();
    // digits from the largest down, two a thread
    const int d1 = kDigits - 1 - 2 * (int)threadIdx.x, d0 = d1 - 1;
    const uint64_t s1 = sm.sums[d1], s0 = sm.sums[d0];
    const uint64_t end = above + block_up_to(sm, s1 + s0), mid = end - s0, begin = mid - s1;
    if (begin < want && want <= mid) {
      sm.found = d1;
      sm.found_above = begin;
    } else if (mid < want && want <= end) {
      sm.found = d0;
      sm.found_above = mid;
    }
    __syncthreads();
    prefix = bits < 32 ? prefix << step | (uint32_t)sm.found : (uint32_t)sm.found;
    above = sm.found_above;
    bits = shift;
    __syncthreads();
  }
  Cut c;
  c.key = kLow ? prefix << kLow | (prefix >> 15 ? 0u : 0xffffu) : prefix;
  const uint64_t v = value(c.key);
  c.count = (want - above + v - 1) / v;
  return c;
}

template <int FMT>
__global__ __launch_bounds__(kThreads) void sample_kernel(SampleArgs a, int64_t row0) {
  __shared__ Shared sm;
  const int64_t row = row0 + blockIdx.x;
  const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
  uint32_t top = 0;
  for (int i = threadIdx.x; i < a.vocab; i += kThreads) top = max(top, key_at<FMT>(a, row, i));
  top = wave_max_u32_f(top);
  if (lane == 0) sm.wave_max[wave] = top;
  __syncthreads();
  for (int w = 0; w < kWaves; ++w) top = max(top, sm.wave_max[w]);
  auto answer = [&](int token, float logprob) {
    a.tokens[row] = token;
    if (a.logprobs) a.logprobs[row] = logprob;
  };
  if (top == 0) {
    if (threadIdx.x == 0) answer(-1, -INFINITY);
    return;
  }
  const float t = a.temperature ? a.temperature[row] : 1.0f;
  const bool greedy = !(t > 0.0f);
  const Weights w{logit_of(top), greedy ? 1.0 : 1.0 / (double)t};
  Cut cut{0, 0};
  double least = 0.0;
  if (greedy) {
    cut = Cut{top, 1};
  } else {
    const int k = a.top_k ? a.top_k[row] : 0;
    if (k > 0 && k < a.vocab) {
      uint64_t there = 0;
      for (int i = threadIdx.x; i < a.vocab; i += kThreads) there += key_at<FMT>(a, row, i) != 0;
      there = block_sum(sm, there);
      if ((uint64_t)k < there)
        cut = find_cut<FMT>(sm, a, row, cut, (uint64_t)k, [](uint32_t) { return (uint64_t)1; });
    }
    const float p = a.top_p ? a.top_p[row] : 1.0f;
    if (p < 1.0f) {
      uint64_t total = 0;
      for (int i = threadIdx.x; i < a.vocab; i += kThreads) {
        const uint32_t key = key_at<FMT>(a, row, i);
        if (key > cut.key) total += w.of(key);
      }
      total = block_sum(sm, total) + (cut.key ? cut.count * w.of(cut.key) : 0);
      const double want = ceil((double)p * (double)total);
      cut = find_cut<FMT>(sm, a, row, cut, want < 1.0 ? 1 : (uint64_t)want,
                          [&](uint32_t key) { return w.of(key); });
    }
    const float least_p = a.min_p ? a.min_p[row] : 0.0f;
    if (least_p > 0.0f) least = fmin((double)least_p, 1.0);
  }
  auto weight = [&](uint32_t key) -> uint64_t { return w.real(key) >= least ? w.of(key) : 0; };
  // the tokens by index, a run of them per thread
  const uint64_t w_cut = cut.key ? weight(cut.key) : 0;
  const int per = (a.vocab + kThreads - 1) / kThreads;
  const int i0 = min((int)threadIdx.x * per, a.vocab), i1 = min(i0 + per, a.vocab);
  uint64_t mass = 0, equal = 0;
  for (int i = i0; i < i1; ++i) {
    const uint32_t key = key_at<FMT>(a, row, i);
    if (key > cut.key) mass += weight(key);
    equal += key != 0 && key == cut.key;
  }
  const uint64_t equal_end = block_up_to(sm, equal), equal_begin = equal_end - equal;
  auto kept = [&](uint64_t before) { return before < cut.count ? before : cut.count; };
  mass += (kept(equal_end) - kept(equal_begin)) * w_cut;
  const uint64_t end = block_up_to(sm, mass), begin = end - mass;
  const uint64_t total = block_sum(sm, mass);
  float u = a.u[row];
  u = u > 0.0f ? fminf(u, 0x1.fffffep-1f) : 0.0f;
  const uint64_t want = (uint64_t)((double)u * (double)total);
  if (begin <= want && want < end) {
    uint64_t sum = begin, same = equal_begin;
    for (int i = i0; i < i1; ++i) {
      const uint32_t key = key_at<FMT>(a, row, i);
      if (key > cut.key) sum += weight(key);
      else if (key != 0 && key == cut.key && same++ < cut.count) sum += w_cut;
      if (sum > want) {
        const double x = logit_of(key) == w.top ? 0.0
                             : ((double)logit_of(key) - (double)w.top) * w.per_t;
        answer(i, (float)(x - log((double)total / kOne)));
        break;
      }
    }
  }
}

constexpr int64_t kMaxGrid = (1ll << 31) / kThreads;
bool aligned(const void* p, uintptr_t a) { return ((uintptr_t)p & (a - 1)) == 0; }

}  // namespace
}  // namespace ei

extern "C" size_t ei_sample_workspace_bytes(int32_t, int32_t, int32_t) { return 0; }

extern "C" ei_status ei_sample_tokens(const void* logits, int32_t format, int32_t rows,
                                      int32_t vocab, int64_t row_stride, const float* u,
                                      const float* temperature, const int32_t* top_k,
                                      const float* top_p, const float* min_p, int32_t* tokens,
                                      float* logprobs, void* workspace, size_t workspace_bytes,
                                      void* stream) {
  if (format != EI_LOGITS_BF16 && format != EI_LOGITS_FP32) return EI_ERR_SHAPE;
  if (rows < 0 || vocab < 0 || row_stride < vocab) return EI_ERR_SHAPE;
  if (vocab > ei::kMaxVocab) return EI_ERR_UNSUPPORTED;
  if (rows > 0 && row_stride > INT64_MAX / 8 / rows) return EI_ERR_SHAPE;
  if (rows == 0) return EI_OK;
  if ((vocab > 0 && !logits) || !u || !tokens) return EI_ERR_NULL;
  if (!ei::aligned(logits, format == EI_LOGITS_BF16 ? 2 : 4) || !ei::aligned(u, 4) ||
      !ei::aligned(temperature, 4) || !ei::aligned(top_k, 4) || !ei::aligned(top_p, 4) ||
      !ei::aligned(min_p, 4) || !ei::aligned(tokens, 4) || !ei::aligned(logprobs, 4))
    return EI_ERR_UNSUPPORTED;
  (void)workspace;
  (void)workspace_bytes;
  const ei::SampleArgs a{logits, rows, vocab, row_stride, u,      temperature,
                         top_k,  top_p, min_p, tokens,    logprobs};
  for (int64_t r = 0; r < rows; r += ei::kMaxGrid) {
    const dim3 grid((unsigned)(rows - r < ei::kMaxGrid ? rows - r : ei::kMaxGrid));
    if (format == EI_LOGITS_BF16)
      hipLaunchKernelGGL((ei::sample_kernel<EI_LOGITS_BF16>), grid, dim3(ei::kThreads), 0,
                         (hipStream_t)stream, a, r);
    else
      hipLaunchKernelGGL((ei::sample_kernel<EI_LOGITS_FP32>), grid, dim3(ei::kThreads), 0,
                         (hipStream_t)stream, a, r);
  }
  return hipGetLastError() == hipSuccess ? EI_OK : EI_ERR_LAUNCH;
}
