// The next token of each row of logits.
//
// With m the row's largest logit and T its temperature, token i weighs
//   w_i = exp((x_i - m) / T),
// in whole multiples of 2^-44 (64-bit integers): sums of weights are then exact,
// whatever their order, and so is every comparison of a sum with top-p's share or
// with the random number.  The kept tokens are the first ones in the order of
// falling logit, equal ones by rising index; such a set is told by the least key
// in it and how many tokens of that key it has (struct Cut).
//
//  sample_scan_kernel   each part of a row: its largest logit
//  sample_weigh_kernel  each part: its weights by pieces of 512 tokens or, for a
//                       row with top-k or top-p, counts and weights by distance
//                       from the largest (bins)
//  sample_pick_kernel   a workgroup a row: the bin that the cut lies in, the cut
//                       among that bin's tokens, the token
#include "../../include/entropyinfer.h"
#include "ei_internal.h"

#include <limits.h>
#include <math.h>

namespace ei {
namespace {

constexpr int kPartThreads = 256;
constexpr int kPartWaves = kPartThreads / kWave;
constexpr int kThreads = 1024;       // of sample_pick_kernel
constexpr int kWaves = kThreads / kWave;
constexpr int kDigitBits = 11, kDigits = 1 << kDigitBits;
constexpr int kMaxVocab = 1 << 19;   // sums of weights: 2^19 * 2^44 = 2^63
constexpr double kOne = 0x1p44;
constexpr int kPiece = 8 * kWave;    // tokens a wave takes at once
constexpr int kMaxPieces = kMaxVocab / kPiece + 1;
constexpr int kMaxParts = 64;
constexpr int kBins = 512;           // the last one: all that lies further off
constexpr int kList = 4096;

struct PartInfo {
  float top, sum;      // the largest logit; the sum of the finite ones, and how many
  int finite, pad;
};
struct SampleArgs {
  const void* logits;
  int rows, vocab;
  int64_t stride;
  const float *u, *temperature;
  const int32_t* top_k;
  const float *top_p, *min_p;
  int32_t* tokens;
  float* logprobs;
  int parts, part_pieces;      // of a row; pieces of a part
  int pieces;                  // of a row
  PartInfo* part;              // [rows][parts]
  uint64_t* piece_sums;        // [rows][pieces]
  uint64_t* bin_sums;          // [rows][kBins]
  uint32_t* bin_counts;        // [rows][kBins]
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

// A row in pieces of 512 tokens; lane l has 8 of them in a row, 16 bytes aligned: piece
// q's are the tokens 512 q - skip + 8 l .. + 7, skip being how far the row's first token
// lies behind such a boundary.
template <int FMT>
struct Row {
  const char* at;      // of token -skip
  int skip, vocab;
  __device__ __forceinline__ Row(const SampleArgs& a, int64_t row) {
    constexpr int kSize = FMT == EI_LOGITS_BF16 ? 2 : 4;
    const char* p = (const char*)a.logits + row * a.stride * kSize;
    skip = (int)((uintptr_t)p % (8 * kSize)) / kSize;
    at = p - skip * kSize;
    vocab = a.vocab;
  }
  // token number of element 0
  __device__ __forceinline__ int index(int piece, int lane) const {
    return piece * kPiece + 8 * lane - skip;
  }
  // -inf where there is none
  __device__ __forceinline__ void load(int piece, int lane, float (&x)[8]) const {
    const int i0 = index(piece, lane);
    const int64_t e0 = (int64_t)piece * kPiece + 8 * lane;
    if (i0 >= 0 && i0 + 8 <= vocab) {
      if constexpr (FMT == EI_LOGITS_BF16) {
        const uint4 w = *(const uint4*)(at + e0 * 2);
        const uint32_t ww[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          x[2 * e] = bf16_lo(ww[e]);
          x[2 * e + 1] = bf16_hi(ww[e]);
        }
      } else {
        const float4 u = ((const float4*)(at + e0 * 4))[0], v = ((const float4*)(at + e0 * 4))[1];
        x[0] = u.x; x[1] = u.y; x[2] = u.z; x[3] = u.w;
        x[4] = v.x; x[5] = v.y; x[6] = v.z; x[7] = v.w;
      }
      return;
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      x[e] = -INFINITY;
      if (i0 + e >= 0 && i0 + e < vocab) {
        if constexpr (FMT == EI_LOGITS_BF16)
          x[e] = __uint_as_float((uint32_t)((const uint16_t*)at)[e0 + e] << 16);
        else
          x[e] = ((const float*)at)[e0 + e];
      }
    }
  }
};

// 2^y for y <= 0, as a whole multiple of 2^-44: y = n + f, |f| <= 1/2, and 2^f by its
// power series up to f^12 (the rest is below 2^-52).
__device__ __forceinline__ uint64_t steps_of_exp2(double y) {
  y = fmax(y, -46.0);
  const double big = 0x1.8p52;
  const double z = y + big;
  const double f = y - (z - big);
  double p = 0x1.0p0;
  constexpr double kLn2 = 0.693147180559945309417232121458;
  constexpr double c1 = kLn2, c2 = c1 * kLn2 / 2, c3 = c2 * kLn2 / 3, c4 = c3 * kLn2 / 4,
                   c5 = c4 * kLn2 / 5, c6 = c5 * kLn2 / 6, c7 = c6 * kLn2 / 7, c8 = c7 * kLn2 / 8,
                   c9 = c8 * kLn2 / 9, c10 = c9 * kLn2 / 10, c11 = c10 * kLn2 / 11,
                   c12 = c11 * kLn2 / 12;
  p = fma(c12, f, c11);
  p = fma(p, f, c10);
  p = fma(p, f, c9);
  p = fma(p, f, c8);
  p = fma(p, f, c7);
  p = fma(p, f, c6);
  p = fma(p, f, c5);
  p = fma(p, f, c4);
  p = fma(p, f, c3);
  p = fma(p, f, c2);
  p = fma(p, f, c1);
  p = fma(p, f, 1.0);
  // times 2^n, then rounded to steps of 2^-44 by adding 2^8 (whose last place they are)
  const uint64_t b = __builtin_bit_cast(uint64_t, p) +
                     ((uint64_t)(uint32_t)__builtin_bit_cast(uint64_t, z) << 52);
  return __builtin_bit_cast(uint64_t, __builtin_bit_cast(double, b) + 0x1p8) -
         __builtin_bit_cast(uint64_t, 0x1p8);
}

struct Weights {
  float top;             // the largest logit
  double per_t;          // log2(e) / T
  uint64_t least;        // min_p in steps: lighter ones are not kept
  __device__ __forceinline__ uint64_t of(float x) const {
    // (top is more than -inf; beside an infinite one all others weigh nothing)
    if (!(x > -INFINITY)) return 0;
    if (top == INFINITY) return x == top ? (uint64_t)kOne : 0;
    return steps_of_exp2(((double)x - (double)top) * per_t);
  }
  __device__ __forceinline__ uint64_t kept(float x) const {
    const uint64_t w = of(x);
    return w >= least ? w : 0;
  }
};

struct Settings {
  bool greedy, cuts;     // cuts: top-k or top-p
  int k;                 // 0: no limit
  float p;               // 1: no limit
  Weights w;
};
__device__ __forceinline__ Settings settings_of(const SampleArgs& a, int64_t row, float top) {
  Settings s;
  const float t = a.temperature ? a.temperature[row] : 1.0f;
  s.greedy = !(t > 0.0f);
  const int k = a.top_k ? a.top_k[row] : 0;
  s.k = k > 0 && k < a.vocab ? k : 0;
  const float p = a.top_p ? a.top_p[row] : 1.0f;
  s.p = p < 1.0f ? p : 1.0f;
  s.cuts = !s.greedy && (s.k > 0 || s.p < 1.0f);
  const float m = a.min_p ? a.min_p[row] : 0.0f;
  s.w.top = top;
  s.w.per_t = s.greedy || t == INFINITY ? 0.0 : 1.4426950408889634 / (double)t;
  s.w.least = m > 0.0f ? (uint64_t)(fmin((double)m, 1.0) * kOne) : 0;
  return s;
}

__device__ __forceinline__ uint64_t wave_sum_u64(uint64_t v) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o);
  return v;
}
__device__ __forceinline__ float wave_sum_f32(float v) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o);
  return v;
}
template <class T>
__device__ __forceinline__ T wave_up_to(T v, int lane) {
#pragma unroll
  for (int o = 1; o < kWave; o <<= 1) {
    const T t = __shfl_up(v, o);
    if (lane >= o) v += t;
  }
  return v;
}

// ----------------------------------------------------------------------------
// Scan
// ----------------------------------------------------------------------------
template <int FMT>
__global__ __launch_bounds__(kPartThreads) void sample_scan_kernel(SampleArgs a, int64_t unit0) {
  __shared__ PartInfo sm[kPartWaves];
  const int64_t unit = unit0 + blockIdx.x;
  const int64_t row = unit / a.parts;
  const int part = (int)(unit % a.parts);
  const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
  if (part == 0)
    for (int b = threadIdx.x; b < kBins; b += kPartThreads) {
      a.bin_sums[row * kBins + b] = 0;
      a.bin_counts[row * kBins + b] = 0;
    }
  const Row<FMT> r(a, row);
  const int q0 = part * a.part_pieces, q1 = min(q0 + a.part_pieces, a.pieces);
  float top = -INFINITY, sum = 0.0f;
  int finite = 0;
  for (int q = q0 + wave; q < q1; q += kPartWaves) {
    float x[8];
    r.load(q, lane, x);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      top = fmaxf(top, x[e]);
      const bool in = fabsf(x[e]) < 0x1p64f;    // (masks of a type's lowest value apart)
      sum += in ? x[e] : 0.0f;
      finite += in ? 1 : 0;
    }
  }
  top = wave_max_f32_dpp(top);
  sum = wave_sum_f32(sum);
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) finite += __shfl_xor(finite, o);
  if (lane == 0) sm[wave] = PartInfo{top, sum, finite, 0};
  __syncthreads();
  if (threadIdx.x == 0) {
    PartInfo p = sm[0];
#pragma unroll
    for (int w = 1; w < kPartWaves; ++w) {
      p.top = fmaxf(p.top, sm[w].top);
      p.sum += sm[w].sum;
      p.finite += sm[w].finite;
    }
    a.part[unit] = p;
  }
}

// A row's parts, together, in their order (64 lanes call this).
__device__ __forceinline__ PartInfo row_info(const SampleArgs& a, int64_t row) {
  const int lane = threadIdx.x % kWave;
  PartInfo p{-INFINITY, 0.0f, 0, 0};
  if (lane < a.parts) p = a.part[row * a.parts + lane];
  p.top = wave_max_f32_dpp(p.top);
  p.sum = wave_sum_f32(p.sum);
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) p.finite += __shfl_xor(p.finite, o);
  return p;
}

// Bins of the distance from the largest logit: finer than needed for the list of
// one to be short.  Their range is 16 T, beyond which lies next to no weight, or,
// for top-k, what lies above the mean.
struct Bins {
  float top, scale;
  __device__ __forceinline__ Bins(const Settings& s, const PartInfo& p) {
    top = p.top;
    const float spread = p.finite > 0 ? top - p.sum / (float)p.finite : 0.0f;
    const float range = s.k > 0 ? spread : 16.0f * 1.4426950408889634f / (float)s.w.per_t;
    scale = (float)(kBins - 1) / range;
    if (!(scale > 0.0f && scale < 0x1p100f)) scale = 0.0f;    // (all in the last one)
  }
  __device__ __forceinline__ int of(float x) const {
    const float d = (top - x) * scale;
    return scale > 0.0f && d < (float)(kBins - 1) ? (int)d : kBins - 1;
  }
};

// ----------------------------------------------------------------------------
// Weigh
// ----------------------------------------------------------------------------
template <int FMT>
__global__ __launch_bounds__(kPartThreads) void sample_weigh_kernel(SampleArgs a, int64_t unit0) {
  __shared__ unsigned long long sums[kBins];
  __shared__ uint32_t counts[kBins];
  const int64_t unit = unit0 + blockIdx.x;
  const int64_t row = unit / a.parts;
  const int part = (int)(unit % a.parts);
  const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
  const PartInfo info = row_info(a, row);
  if (info.top == -INFINITY) return;
  const Settings s = settings_of(a, row, info.top);
  if (s.greedy) return;
  const Row<FMT> r(a, row);
  const int q0 = part * a.part_pieces, q1 = min(q0 + a.part_pieces, a.pieces);
  if (!s.cuts) {
    for (int q = q0 + wave; q < q1; q += kPartWaves) {
      float x[8];
      r.load(q, lane, x);
      uint64_t sum = 0;
#pragma unroll
      for (int e = 0; e < 8; ++e) sum += s.w.kept(x[e]);
      sum = wave_sum_u64(sum);
      if (lane == 0) a.piece_sums[row * a.pieces + q] = sum;
    }
    return;
  }
  for (int b = threadIdx.x; b < kBins; b += kPartThreads) {
    sums[b] = 0;
    counts[b] = 0;
  }
  __syncthreads();
  const Bins bins(s, info);
  const bool weigh = s.p < 1.0f;
  uint64_t far = 0;
  uint32_t n_far = 0;
  for (int q = q0 + wave; q < q1; q += kPartWaves) {
    float x[8];
    r.load(q, lane, x);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      if (!(x[e] > -INFINITY)) continue;
      const uint64_t w = weigh ? s.w.of(x[e]) : 0;
      const int b = bins.of(x[e]);
      if (b == kBins - 1) {
        far += w;
        ++n_far;
      } else {
        if (weigh) atomicAdd(&sums[b], (unsigned long long)w);
        atomicAdd(&counts[b], 1u);
      }
    }
  }
  far = wave_sum_u64(far);
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) n_far += __shfl_xor(n_far, o);
  if (lane == 0 && n_far) {
    atomicAdd(&sums[kBins - 1], (unsigned long long)far);
    atomicAdd(&counts[kBins - 1], n_far);
  }
  __syncthreads();
  for (int b = threadIdx.x; b < kBins; b += kPartThreads)
    if (counts[b]) {
      atomicAdd((unsigned long long*)&a.bin_sums[row * kBins + b], sums[b]);
      atomicAdd(&a.bin_counts[row * kBins + b], counts[b]);
    }
}

// ----------------------------------------------------------------------------
// Pick
// ----------------------------------------------------------------------------
// The tokens above `key` and the first `count` of those that have it.
struct Cut {
  uint32_t key;
  uint64_t count;
};

struct PickSmem {
  uint64_t digits[kDigits];      // (pieces' sums, too)
  uint64_t bin_sum[kBins];       // of the bin and those before it
  uint32_t bin_count[kBins];
  uint32_t key[kList];
  int index[kList];
  uint64_t wave_sum[kWaves];
  uint32_t wave_bits[2][kWaves];
  int found, listed, first_bin;
  uint64_t found_above;
  uint32_t equal[kMaxPieces];
};
static_assert(kMaxPieces <= kDigits, "pieces' sums lie in `digits`");

__device__ __forceinline__ uint64_t block_sum(PickSmem& sm, uint64_t v) {
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
__device__ __forceinline__ uint64_t block_up_to(PickSmem& sm, uint64_t v) {
  const int wave = threadIdx.x / kWave;
  v = wave_up_to(v, threadIdx.x % kWave);
  __syncthreads();
  if (threadIdx.x % kWave == kWave - 1) sm.wave_sum[wave] = v;
  __syncthreads();
  for (int w = 0; w < wave; ++w) v += sm.wave_sum[w];
  return v;
}

// The shortest run of tokens, in their order, of those that `each` gives (within `in`)
// whose values (1 each, or their weights) add up to `want` (1 at least, at most the sum
// of all).  The search goes down the keys' bits from the highest that differ, 11 at a
// time, with sums of the values by digit.
template <class Each, class Value>
__device__ Cut find_cut(PickSmem& sm, Cut in, uint64_t want, Each each, Value value) {
  const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
  uint32_t any = 0, all = ~0u;
  each([&](uint32_t key) {
    if (key >= in.key) {
      any |= key;
      all &= key;
    }
  });
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) {
    any |= __shfl_xor(any, o);
    all &= __shfl_xor(all, o);
  }
  __syncthreads();
  if (lane == 0) {
    sm.wave_bits[0][wave] = any;
    sm.wave_bits[1][wave] = all;
  }
  __syncthreads();
  for (int w = 0; w < kWaves; ++w) {
    any |= sm.wave_bits[0][w];
    all &= sm.wave_bits[1][w];
  }
  int bits = any == all ? 0 : 32 - __builtin_clz(any ^ all);      // that differ
  uint32_t prefix = bits < 32 ? all >> bits : 0;
  // (a bf16 key's low bits follow from its sign; those of one sign are all alike)
  uint64_t above = 0;
  while (bits > 0) {
    const int step = min(bits, kDigitBits), shift = bits - step;
    for (int d = threadIdx.x; d < kDigits; d += kThreads) sm.digits[d] = 0;
    __syncthreads();
    auto add = [&](uint32_t key, uint64_t v) {
      if (bits < 32 && key >> bits != prefix) return;
      atomicAdd((unsigned long long*)&sm.digits[(key >> shift) & ((1u << step) - 1)],
                (unsigned long long)v);
    };
    each([&](uint32_t key) {
      if (key > in.key) add(key, value(key));
    });
    if (threadIdx.x == 0 && in.key != 0) add(in.key, in.count * value(in.key));
    __syncthreads();
    // digits from the largest down, two a thread
    const int d1 = kDigits - 1 - 2 * (int)threadIdx.x, d0 = d1 - 1;
    const uint64_t s1 = sm.digits[d1], s0 = sm.digits[d0];
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
  c.key = prefix;
  const uint64_t v = value(c.key);
  c.count = (want - above + v - 1) / v;
  return c;
}

template <int FMT>
__global__ __launch_bounds__(kThreads) void sample_pick_kernel(SampleArgs a, int64_t row0) {
  __shared__ PickSmem sm;
  const int64_t row = row0 + blockIdx.x;
  const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
  const Row<FMT> r(a, row);
  const PartInfo info = row_info(a, row);
  auto answer = [&](int token, double logprob) {
    a.tokens[row] = token;
    if (a.logprobs) a.logprobs[row] = (float)logprob;
  };
  if (info.top == -INFINITY) {
    if (threadIdx.x == 0) answer(-1, -INFINITY);
    return;
  }
  const Settings s = settings_of(a, row, info.top);
  if (s.greedy) {
    // the first part that has it
    const float top = lane < a.parts ? a.part[row * a.parts + lane].top : -INFINITY;
    const int part = __builtin_ctzll(__builtin_amdgcn_ballot_w64(top == info.top));
    const int q0 = part * a.part_pieces, q1 = min(q0 + a.part_pieces, a.pieces);
    uint32_t at = UINT_MAX;
    for (int q = q0 + wave; q < q1; q += kWaves) {
      float x[8];
      r.load(q, lane, x);
#pragma unroll
      for (int e = 7; e >= 0; --e)
        if (x[e] == info.top) at = min(at, (uint32_t)(r.index(q, lane) + e));
    }
    at = wave_min_u32_f(at);
    if (lane == 0) sm.wave_bits[0][wave] = at;
    __syncthreads();
    if (threadIdx.x == 0) {
      for (int w = 0; w < kWaves; ++w) at = min(at, sm.wave_bits[0][w]);
      answer((int)at, 0.0);
    }
    return;
  }
  float u = a.u[row];
  u = u > 0.0f ? fminf(u, 0x1.fffffep-1f) : 0.0f;
  auto log_share = [&](float x, uint64_t total) -> double {
    const double y = x == s.w.top ? 0.0 : ((double)x - (double)s.w.top) * s.w.per_t;
    return y * 0.6931471805599453 - log((double)total * (1.0 / kOne));
  };

  Cut cut{0, 0};
  if (s.cuts) {
    const Bins bins(s, info);
    // sums over the bins from the largest logit on
    const int b = threadIdx.x;
    const uint64_t own_count = b < kBins ? a.bin_counts[row * kBins + b] : 0;
    const uint64_t own_sum = b < kBins ? a.bin_sums[row * kBins + b] : 0;
    const uint64_t count_to = block_up_to(sm, own_count), sum_to = block_up_to(sm, own_sum);
    if (b < kBins) {
      sm.bin_count[b] = (uint32_t)count_to;
      sm.bin_sum[b] = sum_to;
    }
    if (threadIdx.x == 0) {
      sm.listed = 0;
      sm.first_bin = kBins;
    }
    __syncthreads();
    auto counts_before = [&](int bin) { return bin ? sm.bin_count[bin - 1] : 0u; };
    auto sums_before = [&](int bin) { return bin ? sm.bin_sum[bin - 1] : (uint64_t)0; };
    // the first bin up to which the values reach `want`
    auto bin_of = [&](bool reached_before, bool reached) -> int {
      __syncthreads();
      if (b < kBins && !reached_before && reached) sm.found = b;
      __syncthreads();
      return sm.found;
    };
    // The row's tokens of bins `first` .. `last`, where the list holds so many, as
    // (key, index) in no order.
    int first_listed = kBins, last_listed = -1;
    auto list = [&](int bin) -> bool {      // whether it has that bin's
      if (bin >= first_listed && bin <= last_listed) return true;
      if (bin == kBins - 1 || sm.bin_count[bin] - counts_before(bin) > kList) return false;
      // the first bin from which on they fit
      __syncthreads();
      if (threadIdx.x == 0) sm.listed = 0;
      if (b <= bin && sm.bin_count[bin] - counts_before(b) <= kList &&
          (b == 0 || sm.bin_count[bin] - counts_before(b - 1) > kList))
        sm.first_bin = b;
      __syncthreads();
      first_listed = sm.first_bin;
      last_listed = bin;
      for (int q = wave; q < a.pieces; q += kWaves) {
        float x[8];
        r.load(q, lane, x);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          if (!(x[e] > -INFINITY)) continue;
          const int at = bins.of(x[e]);
          if (at < first_listed || at > last_listed) continue;
          const int to = atomicAdd(&sm.listed, 1);
          if (to < kList) {        // (always)
            sm.key[to] = key_of(x[e]);
            sm.index[to] = r.index(q, lane) + e;
          }
        }
      }
      __syncthreads();
      return true;
    };
    auto cut_in = [&](int bin, Cut in, uint64_t want, auto value) -> Cut {
      if (list(bin)) {
        const int n = sm.listed;
        return find_cut(sm, in, want, [&](auto use) {
          for (int i = threadIdx.x; i < n; i += kThreads)
            if (bins.of(logit_of(sm.key[i])) == bin) use(sm.key[i]);
        }, value);
      }
      return find_cut(sm, in, want, [&](auto use) {
        for (int q = wave; q < a.pieces; q += kWaves) {
          float x[8];
          r.load(q, lane, x);
#pragma unroll
          for (int e = 0; e < 8; ++e)
            if (x[e] > -INFINITY && bins.of(x[e]) == bin) use(key_of(x[e]));
        }
      }, value);
    };
    int cut_bin = kBins;
    if (s.k > 0 && (uint32_t)s.k < sm.bin_count[kBins - 1]) {
      const uint32_t k = (uint32_t)s.k;
      cut_bin = bin_of(count_to - own_count >= k, count_to >= k);
      cut = cut_in(cut_bin, cut, k - counts_before(cut_bin), [](uint32_t) { return (uint64_t)1; });
    }
    if (s.p < 1.0f) {
      auto weight = [&](uint32_t key) { return s.w.of(logit_of(key)); };
      uint64_t total = sm.bin_sum[kBins - 1], before = total;
      if (cut_bin < kBins) {
        // the cut bin's kept weight
        before = sums_before(cut_bin);
        uint64_t sum = 0;
        if (cut_bin <= last_listed) {
          for (int i = threadIdx.x; i < sm.listed; i += kThreads)
            if (sm.key[i] > cut.key && bins.of(logit_of(sm.key[i])) == cut_bin) sum += weight(sm.key[i]);
        } else {
          for (int q = wave; q < a.pieces; q += kWaves) {
            float x[8];
            r.load(q, lane, x);
#pragma unroll
            for (int e = 0; e < 8; ++e)
              if (x[e] > -INFINITY && bins.of(x[e]) == cut_bin && key_of(x[e]) > cut.key)
                sum += s.w.of(x[e]);
          }
        }
        total = before + block_sum(sm, sum) + cut.count * weight(cut.key);
      }
      const double real = ceil((double)s.p * (double)total);
      const uint64_t want = real < 1.0 ? 1 : (uint64_t)real;
      if (before < want && cut_bin < kBins) {
        cut = cut_in(cut_bin, cut, want - before, weight);
      } else {
        cut_bin = bin_of(sum_to - own_sum >= want, sum_to >= want);
        cut = cut_in(cut_bin, Cut{0, 0}, want - sums_before(cut_bin), weight);
      }
    }
    // All kept ones in the list, and few: each thread has one, and adds up those of
    // lesser index.
    if (first_listed == 0 && cut_bin < kBins && cut_bin <= last_listed &&
        sm.bin_count[cut_bin] <= kThreads) {
      const int n = sm.listed;
      int mine = -1;
      uint32_t key = 0;
      uint64_t w = 0;
      // (more are listed than the bins up to the cut's hold only where top-p cut again)
      __syncthreads();
      if (threadIdx.x == 0) sm.found = 0;
      __syncthreads();
      for (int i = threadIdx.x; i < n; i += kThreads) {
        const uint32_t have = sm.key[i];
        bool in = have > cut.key;
        if (have == cut.key) {
          uint64_t rank = 0;
          for (int j = 0; j < n; ++j) rank += sm.key[j] == have && sm.index[j] < sm.index[i];
          in = rank < cut.count;
        }
        if (in) {
          const int to = atomicAdd(&sm.found, 1);
          sm.digits[to] = (uint64_t)(uint32_t)sm.index[i] << 32 | have;
        }
      }
      __syncthreads();
      const int m = sm.found;
      if ((int)threadIdx.x < m) {
        mine = (int)(sm.digits[threadIdx.x] >> 32);
        key = (uint32_t)sm.digits[threadIdx.x];
        w = s.w.kept(logit_of(key));
      }
      const uint64_t total = block_sum(sm, w);
      sm.digits[kThreads + threadIdx.x] = w;
      __syncthreads();
      const uint64_t want = (uint64_t)((double)u * (double)total);
      if (w > 0) {
        uint64_t before = 0;
        for (int j = 0; j < m; ++j)
          before += (int)(sm.digits[j] >> 32) < mine ? sm.digits[kThreads + j] : 0;
        if (before <= want && want < before + w) answer(mine, log_share(logit_of(key), total));
      }
      return;
    }
  }

  // The pieces' kept weights, then the piece that u times their total lies in.
  __syncthreads();
  const uint64_t w_cut = cut.key ? s.w.kept(logit_of(cut.key)) : 0;
  if (!s.cuts) {
    for (int q = threadIdx.x; q < a.pieces; q += kThreads) {
      sm.digits[q] = a.piece_sums[row * a.pieces + q];
      sm.equal[q] = 0;
    }
  } else {
    for (int q = wave; q < a.pieces; q += kWaves) {
      float x[8];
      r.load(q, lane, x);
      uint64_t sum = 0;
      uint32_t equal = 0;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const uint32_t key = key_of(x[e]);
        if (key > cut.key) sum += s.w.kept(x[e]);
        equal += key != 0 && key == cut.key;
      }
      sum = wave_sum_u64(sum);
#pragma unroll
      for (int o = 32; o > 0; o >>= 1) equal += __shfl_xor(equal, o);
      if (lane == 0) {
        sm.digits[q] = sum;
        sm.equal[q] = equal;
      }
    }
  }
  __syncthreads();
  auto kept = [&](uint64_t before) { return before < cut.count ? before : cut.count; };
  // two pieces a thread (kMaxPieces of them at most)
  const int qa = 2 * (int)threadIdx.x, qb = qa + 1;
  const uint64_t ea = qa < a.pieces ? sm.equal[qa] : 0, eb = qb < a.pieces ? sm.equal[qb] : 0;
  const uint64_t equal_end = block_up_to(sm, ea + eb), equal_mid = equal_end - eb;
  const uint64_t equal_begin = equal_mid - ea;
  const uint64_t ma = (qa < a.pieces ? sm.digits[qa] : 0) + (kept(equal_mid) - kept(equal_begin)) * w_cut;
  const uint64_t mb = (qb < a.pieces ? sm.digits[qb] : 0) + (kept(equal_end) - kept(equal_mid)) * w_cut;
  const uint64_t end = block_up_to(sm, ma + mb), mid = end - mb, begin = mid - ma;
  const uint64_t total = block_sum(sm, ma + mb);
  const uint64_t want = (uint64_t)((double)u * (double)total);
  __syncthreads();
  if (begin <= want && want < end) {
    const bool second = mid <= want;
    sm.found = second ? qb : qa;
    sm.found_above = second ? mid : begin;
    sm.digits[0] = second ? equal_mid : equal_begin;
  }
  __syncthreads();
  if (wave != 0) return;
  const int q = sm.found;      // (of one wave)
  float x[8];
  r.load(q, lane, x);
  uint32_t same = 0;
  uint64_t sum = 0;
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const uint32_t key = key_of(x[e]);
    if (key > cut.key) sum += s.w.kept(x[e]);
    same += key != 0 && key == cut.key;
  }
  const uint64_t same0 = sm.digits[0] + (wave_up_to(same, lane) - same);
  sum += (kept(same0 + same) - kept(same0)) * w_cut;
  uint64_t run = sm.found_above + wave_up_to(sum, lane) - sum;
  if (!(run <= want && want < run + sum)) return;
  uint64_t n_same = same0;
  for (int e = 0; e < 8; ++e) {
    const uint32_t key = key_of(x[e]);
    if (key > cut.key) run += s.w.kept(x[e]);
    else if (key != 0 && key == cut.key && n_same++ < cut.count) run += w_cut;
    if (run > want) {
      answer(r.index(q, lane) + e, log_share(x[e], total));
      return;
    }
  }
}

// ----------------------------------------------------------------------------
// Host side
// ----------------------------------------------------------------------------
constexpr int64_t kMaxGrid = (1ll << 31) / kThreads;
bool aligned(const void* p, uintptr_t a) { return ((uintptr_t)p & (a - 1)) == 0; }

struct SamplePlan {
  int pieces, parts, part_pieces;
  size_t at_bins, at_counts, at_pieces, bytes;
};
// Parts of a row: as many as give the chip 1024 workgroups, of 4 pieces at least.
SamplePlan sample_plan(int rows, int vocab) {
  SamplePlan p{};
  p.pieces = (vocab + 7 + kPiece - 1) / kPiece;      // (the first may start 7 tokens early)
  int parts = 1024 / rows;
  const int most = (p.pieces + kPartWaves - 1) / kPartWaves;
  parts = parts > kMaxParts ? kMaxParts : parts < 1 ? 1 : parts;
  parts = parts > most ? most : parts;
  p.part_pieces = (p.pieces + parts - 1) / parts;
  p.parts = (p.pieces + p.part_pieces - 1) / p.part_pieces;
  auto up = [](size_t n) { return (n + 255) / 256 * 256; };
  p.at_bins = up((size_t)rows * p.parts * sizeof(PartInfo));
  p.at_counts = p.at_bins + (size_t)rows * kBins * sizeof(uint64_t);
  p.at_pieces = p.at_counts + (size_t)rows * kBins * sizeof(uint32_t);
  p.bytes = p.at_pieces + (size_t)rows * p.pieces * sizeof(uint64_t);
  return p;
}

template <int FMT>
void launch_sample(const SampleArgs& a, hipStream_t stream) {
  const int64_t units = (int64_t)a.rows * a.parts;
  constexpr int64_t most = (1ll << 31) / kPartThreads;
  for (int64_t u = 0; u < units; u += most)
    hipLaunchKernelGGL((sample_scan_kernel<FMT>), dim3((unsigned)(units - u < most ? units - u : most)),
                       dim3(kPartThreads), 0, stream, a, u);
  for (int64_t u = 0; u < units; u += most)
    hipLaunchKernelGGL((sample_weigh_kernel<FMT>), dim3((unsigned)(units - u < most ? units - u : most)),
                       dim3(kPartThreads), 0, stream, a, u);
  for (int64_t r = 0; r < a.rows; r += kMaxGrid)
    hipLaunchKernelGGL((sample_pick_kernel<FMT>),
                       dim3((unsigned)(a.rows - r < kMaxGrid ? a.rows - r : kMaxGrid)),
                       dim3(kThreads), 0, stream, a, r);
}

bool valid(int32_t rows, int32_t vocab, int32_t format) {
  return (format == EI_LOGITS_BF16 || format == EI_LOGITS_FP32) && rows >= 0 && vocab >= 0;
}

}  // namespace
}  // namespace ei

extern "C" size_t ei_sample_workspace_bytes(int32_t rows, int32_t vocab, int32_t format) {
  if (!ei::valid(rows, vocab, format) || vocab > ei::kMaxVocab || rows == 0) return 0;
  return ei::sample_plan(rows, vocab).bytes;
}

extern "C" ei_status ei_sample_tokens(const void* logits, int32_t format, int32_t rows,
                                      int32_t vocab, int64_t row_stride, const float* u,
                                      const float* temperature, const int32_t* top_k,
                                      const float* top_p, const float* min_p, int32_t* tokens,
                                      float* logprobs, void* workspace, size_t workspace_bytes,
                                      void* stream) {
  if (!ei::valid(rows, vocab, format) || row_stride < vocab) return EI_ERR_SHAPE;
  if (vocab > ei::kMaxVocab) return EI_ERR_UNSUPPORTED;
  if (rows > 0 && row_stride > INT64_MAX / 8 / rows) return EI_ERR_SHAPE;
  if (rows == 0) return EI_OK;
  if ((vocab > 0 && !logits) || !u || !tokens) return EI_ERR_NULL;
  if (!ei::aligned(logits, format == EI_LOGITS_BF16 ? 2 : 4) || !ei::aligned(u, 4) ||
      !ei::aligned(temperature, 4) || !ei::aligned(top_k, 4) || !ei::aligned(top_p, 4) ||
      !ei::aligned(min_p, 4) || !ei::aligned(tokens, 4) || !ei::aligned(logprobs, 4))
    return EI_ERR_UNSUPPORTED;
  const ei::SamplePlan p = ei::sample_plan(rows, vocab);
  if (!workspace || workspace_bytes < p.bytes) return EI_ERR_WORKSPACE;
  if (!ei::aligned(workspace, 16)) return EI_ERR_UNSUPPORTED;
  char* ws = (char*)workspace;
  const ei::SampleArgs a{logits, rows, vocab, row_stride, u, temperature, top_k, top_p, min_p,
                         tokens, logprobs, p.parts, p.part_pieces, p.pieces, (ei::PartInfo*)ws,
                         (uint64_t*)(ws + p.at_pieces), (uint64_t*)(ws + p.at_bins),
                         (uint32_t*)(ws + p.at_counts)};
  if (format == EI_LOGITS_BF16) ei::launch_sample<EI_LOGITS_BF16>(a, (hipStream_t)stream);
  else ei::launch_sample<EI_LOGITS_FP32>(a, (hipStream_t)stream);
  return hipGetLastError() == hipSuccess ? EI_OK : EI_ERR_LAUNCH;
}
