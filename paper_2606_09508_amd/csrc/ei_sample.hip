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
// bf16: the weights of a row's values from a table in LDS.
//  sample_row_kernel      a workgroup a row, all steps
// or, where there are few rows, several workgroups a row:
//  sample_tops_kernel     each part of a row: its largest logit
//  sample_counts_kernel   each part of a row with top-k or top-p: the tokens of each value
//  sample_weights_kernel  the cut; each part: the kept weights of each 512 tokens
//  sample_token_kernel    a workgroup a row: the 512 that u lies in, the token
//
// fp32: a weight computed for each logit.
//  sample_scan_kernel   each part of a row: its largest logit
//  sample_bins_kernel   each part of a row with top-k or top-p: counts or weights by
//                       distance from the largest logit
//  sample_cut_kernel    a workgroup for each of those rows: the bin that the cut
//                       lies in, the cut among that bin's tokens, and the token
//                       where few are kept
//  sample_weigh_kernel  each part: the kept weights of each 2048 tokens
//  sample_pick_kernel   a workgroup a row: the 2048 that u lies in, the token
//
// Measured (a captured call, us): 256 rows of 128256 in bf16 34 to 36 (65 MB: 13 at a
// copy's rate), 64 of them with all settings mixed 36, one with top-p 24; in fp32 73, 76
// and 35; 12 masked rows of 32001 36 to 45.  Of the 256 bf16 rows' 35 the largest logits
// take 13 (HBM at a copy's rate), the tables 1, the weights 18 (the rows from HBM once
// more, vector instructions issued in 0.64 of all cycles, LDS reading entries in 0.24 and
// conflicts in 0.14: each overlaps the others in part), the token 3.  Calls of few rows are
// bound by the launches and the steps of the cut, which follow one another.
#include "../../include/entropyinfer.h"
#include "ei_internal.h"

#include <limits.h>
#include <math.h>

namespace ei {
namespace {

constexpr int kPartThreads = 256;
constexpr int kPartWaves = kPartThreads / kWave;
constexpr int kThreads = 1024;       // of sample_cut_kernel
constexpr int kWaves = kThreads / kWave;
constexpr int kDigitBits = 11, kDigits = 1 << kDigitBits;
constexpr int kMaxVocab = 1 << 19;   // sums of weights: 2^19 * 2^44 = 2^63
constexpr double kOne = 0x1p44;
constexpr int kPiece = 8 * kWave;    // tokens a wave takes at once
constexpr int kBlockPieces = 4;      // pieces whose weights are summed together
constexpr int kMaxBlocks = (kMaxVocab / kPiece + 1 + kBlockPieces - 1) / kBlockPieces;
constexpr int kPickThreads = 512;
static_assert(kMaxBlocks <= kPickThreads, "a thread for each");
constexpr int kFew = 256;            // kept tokens that sample_cut_kernel picks from
constexpr int kMaxParts = 64;
constexpr int kBins = 512;           // the last one: all that lies further off
constexpr int kList = 4096;
constexpr int kCUs = 256;

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
  int parts, part_blocks;      // of a row; blocks of a part
  int blocks;                  // of a row
  PartInfo* part;              // [rows][parts]
  struct RowCut* cut;          // [rows], of those with top-k or top-p
  uint64_t* sums;              // [rows][blocks]: kept weights above the cut's key (bf16: of pieces)
  uint32_t* equal;             // [rows][blocks]: tokens of that key
  uint64_t* bin_sums;          // [rows][kBins]
  uint32_t* bin_counts;        // [rows][kBins]
  // of bf16 rows in several workgroups
  float* tops;                 // [rows][parts]
  struct RowState* state;      // [rows]
  uint32_t* counts;            // [rows][kTable]
};

// The tokens above `key` and the first `count` of those that have it.
struct Cut {
  uint32_t key;
  uint64_t count;
};
struct RowCut {
  Cut cut;
  int done, pad[3];
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

// A row in pieces of 512 tokens; lane l has the 8 from 512 q + 8 l on of piece q.  Loads
// are of 16 bytes, aligned to an element only.
template <int FMT>
struct Row {
  const char* at;
  int vocab;
  __device__ __forceinline__ Row(const SampleArgs& a, int64_t row) {
    at = (const char*)a.logits + row * a.stride * (FMT == EI_LOGITS_BF16 ? 2 : 4);
    vocab = a.vocab;
  }
  __device__ __forceinline__ static int index(int piece, int lane) { return piece * kPiece + 8 * lane; }
  __device__ __forceinline__ static uint4 load16(const void* p) {
    uint4 w;
    __builtin_memcpy(&w, p, 16);
    return w;
  }
  // (bf16 as it is)
  __device__ __forceinline__ uint4 load_full(int piece, int lane) const {
    return load16((const uint16_t*)at + index(piece, lane));
  }
  // -inf where there is none
  __device__ __forceinline__ uint4 load_raw(int piece, int lane) const {
    const int i0 = index(piece, lane);
    const uint16_t* p = (const uint16_t*)at + i0;
    if (i0 + 8 <= vocab) return load16(p);
    uint64_t w[2] = {0, 0};
#pragma unroll 1
    for (int e = 7; e >= 0; --e) {
      const uint64_t v = i0 + e < vocab ? p[e] : 0xff80u;
      w[1] = w[1] << 16 | w[0] >> 48;
      w[0] = w[0] << 16 | v;
    }
    return make_uint4((uint32_t)w[0], (uint32_t)(w[0] >> 32), (uint32_t)w[1], (uint32_t)(w[1] >> 32));
  }
  // fp32
  __device__ __forceinline__ void load(int piece, int lane, float (&x)[8]) const {
    const int i0 = index(piece, lane);
    const float* p = (const float*)at + i0;
    if (i0 + 8 <= vocab) {
      const uint4 u = load16(p), v = load16(p + 4);
      const uint32_t w[8] = {u.x, u.y, u.z, u.w, v.x, v.y, v.z, v.w};
#pragma unroll
      for (int e = 0; e < 8; ++e) x[e] = __uint_as_float(w[e]);
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) x[e] = i0 + e < vocab ? p[e] : -INFINITY;
    }
  }
  // four pieces one behind the other
  __device__ __forceinline__ void load_block(int block, int lane, float (&x)[kBlockPieces][8]) const {
#pragma unroll
    for (int q = 0; q < kBlockPieces; ++q) load(block * kBlockPieces + q, lane, x[q]);
  }
};

// 2^y for y <= 0 (more counts as 0, NaN as -inf), as a whole multiple of 2^-44: y =
// n + f, |f| <= 1/2, and 2^f by its power series up to f^12 (the rest is below 2^-52).
// In 64 bits, which cost a lane as many cycles as 32; the series' factors lie in scalar
// registers (as constants the compiler moves each to a vector register first).
struct Series {
  double c[13];
  __device__ __forceinline__ Series() {
    double f = 1.0;
#pragma unroll
    for (int i = 1; i <= 12; ++i) {
      f *= 0.693147180559945309417232121458 / i;
      c[i] = f;
      asm("" : "+s"(c[i]));
    }
  }
  __device__ __forceinline__ uint64_t steps_of_exp2(double y) const {
    y = fmin(fmax(y, -46.0), 0.0);
    const double big = 0x1.8p52;
    const double z = y + big;
    const double f = y - (z - big);
    double p = fma(c[12], f, c[11]);
#pragma unroll
    for (int i = 10; i >= 1; --i) p = fma(p, f, c[i]);
    p = fma(p, f, 1.0);
    // times 2^n, then rounded to steps of 2^-44 by adding 2^8 (whose last place they are)
    const uint64_t b = __builtin_bit_cast(uint64_t, p) +
                       ((uint64_t)((uint32_t)__builtin_bit_cast(uint64_t, z) << 20) << 32);
    return __builtin_bit_cast(uint64_t, __builtin_bit_cast(double, b) + 0x1p8) -
           __builtin_bit_cast(uint64_t, 0x1p8);
  }
};

struct Weights {
  double top;            // the largest logit; an infinite one as 10^300
  double per_t;          // log2(e) / T; beside an infinite logit 1
  uint64_t least;        // min_p in steps: lighter ones are not kept
  Series series;
  // (x = -inf: y is that or NaN; x = +inf: y is that)
  __device__ __forceinline__ uint64_t of(float x) const {
    return series.steps_of_exp2(((double)x - top) * per_t);
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
// As the caller gives them.  (Asked for by themselves, before the largest logit is known.)
struct Given {
  float t, p, m;
  int k;
  __device__ __forceinline__ Given(const SampleArgs& a, int64_t row)
      : t(a.temperature ? a.temperature[row] : 1.0f), p(a.top_p ? a.top_p[row] : 1.0f),
        m(a.min_p ? a.min_p[row] : 0.0f), k(a.top_k ? a.top_k[row] : 0) {}
};
__device__ __forceinline__ Settings settings_of(const SampleArgs& a, const Given& given, float top) {
  Settings s;
  const float t = given.t, p = given.p, m = given.m;
  const int k = given.k;
  s.greedy = !(t > 0.0f);
  s.k = k > 0 && k < a.vocab ? k : 0;
  s.p = p < 1.0f ? p : 1.0f;
  s.cuts = !s.greedy && (s.k > 0 || s.p < 1.0f);
  s.w.top = top == INFINITY ? 1e300 : (double)top;
  s.w.per_t = s.greedy || top == INFINITY ? 1.0 : 1.4426950408889634 / (double)t;
  s.w.least = m > 0.0f ? (uint64_t)(fmin((double)m, 1.0) * kOne) : 0;
  return s;
}

__device__ __forceinline__ uint64_t wave_sum_u64(uint64_t v) {
#define EI_ADD_DPP(ctrl)                                                              \
  v += (uint64_t)EI_DPP_U32((uint32_t)(v >> 32), ctrl, 0xF, false) << 32 |            \
       EI_DPP_U32((uint32_t)v, ctrl, 0xF, false)
  EI_ADD_DPP(0xB1);     // quad_perm [1,0,3,2]
  EI_ADD_DPP(0x4E);     // quad_perm [2,3,0,1]
  EI_ADD_DPP(0x141);    // row_half_mirror
  EI_ADD_DPP(0x140);    // row_mirror
#undef EI_ADD_DPP
  uint64_t s = 0;
#pragma unroll
  for (int l = 0; l < kWave; l += 16)
    s += (uint64_t)rl_u32((uint32_t)(v >> 32), l) << 32 | rl_u32((uint32_t)v, l);
  return s;
}
__device__ __forceinline__ float wave_sum_f32(float v) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o);
  return v;
}
// ----------------------------------------------------------------------------
// Scan
// ----------------------------------------------------------------------------
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
  const Row<EI_LOGITS_FP32> r(a, row);
  const int b0 = part * a.part_blocks, b1 = min(b0 + a.part_blocks, a.blocks);
  float top = -INFINITY, sum = 0.0f;
  int finite = 0;
  for (int b = b0 + wave; b < b1; b += kPartWaves) {
    float x[kBlockPieces][8];
    r.load_block(b, lane, x);
#pragma unroll
    for (int q = 0; q < kBlockPieces; ++q)
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        top = fmaxf(top, x[q][e]);
        const bool in = fabsf(x[q][e]) < 0x1p64f;    // (masks of a type's lowest value apart)
        sum += in ? x[q][e] : 0.0f;
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
    scale = top < INFINITY ? (float)(kBins - 1) / range : 0.0f;
    if (!(scale > 0.0f && scale < 0x1p100f)) scale = 0.0f;    // (all in the last one)
  }
  __device__ __forceinline__ int of(float x) const {
    const float d = (top - x) * scale;
    return scale > 0.0f && d < (float)(kBins - 1) ? (int)d : kBins - 1;
  }
};

// ----------------------------------------------------------------------------
// Bins
// ----------------------------------------------------------------------------
__global__ __launch_bounds__(kPartThreads) void sample_bins_kernel(SampleArgs a, int64_t unit0) {
  __shared__ unsigned long long sums[kBins];
  __shared__ uint32_t counts[kBins];
  const int64_t unit = unit0 + blockIdx.x;
  const int64_t row = unit / a.parts;
  const int part = (int)(unit % a.parts);
  const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
  const PartInfo info = row_info(a, row);
  if (info.top == -INFINITY) return;
  const Settings s = settings_of(a, Given(a, row), info.top);
  if (!s.cuts) return;
  const Row<EI_LOGITS_FP32> r(a, row);
  const int b0 = part * a.part_blocks, b1 = min(b0 + a.part_blocks, a.blocks);
  for (int b = threadIdx.x; b < kBins; b += kPartThreads) {
    sums[b] = 0;
    counts[b] = 0;
  }
  __syncthreads();
  const Bins bins(s, info);
  // top-k alone needs counts, top-p alone weights
  auto pass = [&](auto weigh, auto count) {
    uint64_t far = 0;
    uint32_t n_far = 0;
    for (int b = b0 + wave; b < b1; b += kPartWaves) {
      float x[kBlockPieces][8];
      r.load_block(b, lane, x);
#pragma unroll
      for (int q = 0; q < kBlockPieces; ++q)
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const float v = x[q][e];
          const uint64_t w = weigh() ? s.w.of(v) : 0;
          const int bin = bins.of(v);
          if (bin == kBins - 1) {
            far += w;
            n_far += v > -INFINITY ? 1 : 0;
          } else {
            if (weigh()) atomicAdd(&sums[bin], (unsigned long long)w);
            if (count()) atomicAdd(&counts[bin], 1u);
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
  };
  auto yes = []() { return true; };
  auto no = []() { return false; };
  if (s.k == 0) pass(yes, no);
  else if (s.p < 1.0f) pass(yes, yes);
  else pass(no, yes);
  __syncthreads();
  for (int b = threadIdx.x; b < kBins; b += kPartThreads) {
    if (sums[b]) atomicAdd((unsigned long long*)&a.bin_sums[row * kBins + b], sums[b]);
    if (counts[b]) atomicAdd(&a.bin_counts[row * kBins + b], counts[b]);
  }
}

// ----------------------------------------------------------------------------
// Cut
// ----------------------------------------------------------------------------
struct PickSmem {
  uint64_t digits[kDigits];
  uint64_t bin_sum[kBins];       // of the bin and those before it
  uint32_t bin_count[kBins];
  uint32_t key[kList];
  int index[kList];
  uint64_t wave_sum[kWaves];
  uint32_t wave_bits[2][kWaves];
  int found, listed, first_bin;
  uint64_t found_above;
};

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
  v = wave_incl_scan_u64(v);
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

__device__ __forceinline__ void answer(const SampleArgs& a, int64_t row, int token, double logprob) {
  a.tokens[row] = token;
  if (a.logprobs) a.logprobs[row] = (float)logprob;
}
// The random number's place among the weights.
__device__ __forceinline__ uint64_t want_of(const SampleArgs& a, int64_t row, uint64_t total) {
  float u = a.u[row];
  u = u > 0.0f ? fminf(u, 0x1.fffffep-1f) : 0.0f;
  return (uint64_t)((double)u * (double)total);
}
__device__ __forceinline__ double log_share(const Settings& s, float x, uint64_t total) {
  const double y = fmin(((double)x - s.w.top) * s.w.per_t, 0.0);
  return y * 0.6931471805599453 - log((double)total * (1.0 / kOne));
}

__global__ __launch_bounds__(kThreads) void sample_cut_kernel(SampleArgs a, int64_t row0) {
  __shared__ PickSmem sm;
  const int64_t row = row0 + blockIdx.x;
  const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
  const Row<EI_LOGITS_FP32> r(a, row);
  const PartInfo info = row_info(a, row);
  if (info.top == -INFINITY) return;
  const Settings s = settings_of(a, Given(a, row), info.top);
  if (!s.cuts) return;
  // all of the row's logits, with their indexes
  auto each_logit = [&](auto use) {
    // (a piece at a time: four of them, unrolled, spend 57 us instead of 39 on 12 rows of
    // 32001, mostly waiting for code)
    const int pieces = (a.vocab + kPiece - 1) / kPiece;
#pragma unroll 1
    for (int q = wave; q < pieces; q += kWaves) {
      float x[8];
      r.load(q, lane, x);
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if (x[e] > -INFINITY) use(x[e], r.index(q, lane) + e);
    }
  };

  Cut cut{0, 0};
  {
    const Bins bins(s, info);
    // sums over the bins from the largest logit on
    const int b = threadIdx.x;
    const uint64_t own_sum = b < kBins ? a.bin_sums[row * kBins + b] : 0;
    uint64_t own_count = b < kBins ? a.bin_counts[row * kBins + b] : 0;
    if (s.k == 0 && b < kBins - 1) {
      // At most so many, by the least weight that a logit of the bin has (a hundredth
      // of T further off is far more than its distance was rounded by).
      const double y = ((double)(b + 1) / (double)bins.scale) * s.w.per_t + 0.015;
      const uint64_t least = s.w.series.steps_of_exp2(-y);
      own_count = least ? own_sum / least : own_sum ? kMaxVocab : 0;
    }
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
      each_logit([&](float x, int index) {
        const int at = bins.of(x);
        if (at < first_listed || at > last_listed) return;
        const int to = atomicAdd(&sm.listed, 1);
        if (to < kList) {        // (always)
          sm.key[to] = key_of(x);
          sm.index[to] = index;
        }
      });
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
        each_logit([&](float x, int) {
          if (bins.of(x) == bin) use(key_of(x));
        });
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
          each_logit([&](float x, int) {
            if (bins.of(x) == cut_bin && key_of(x) > cut.key) sum += s.w.of(x);
          });
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
    if (first_listed == 0 && cut_bin <= last_listed) {
      const int n = sm.listed;
      uint64_t same = 0;
      __syncthreads();
      if (threadIdx.x == 0) sm.found = 0;
      __syncthreads();
      for (int i = threadIdx.x; i < n; i += kThreads) {
        const uint32_t key = sm.key[i];
        if (key < cut.key) continue;
        same += key == cut.key;
        const int to = atomicAdd(&sm.found, 1);
        if (to < kFew) sm.digits[to] = (uint64_t)(uint32_t)sm.index[i] << 32 | key;
      }
      same = block_sum(sm, same);
      const int m = sm.found;
      if (m <= kFew) {
        uint32_t key = 0;
        int mine = 0;
        uint64_t w = 0;
        if ((int)threadIdx.x < m) {
          mine = (int)(sm.digits[threadIdx.x] >> 32);
          key = (uint32_t)sm.digits[threadIdx.x];
          uint64_t rank = 0;
          if (key == cut.key && same > cut.count)
            for (int j = 0; j < m; ++j)
              rank += (uint32_t)sm.digits[j] == key && (int)(sm.digits[j] >> 32) < mine;
          if (key > cut.key || rank < cut.count) w = s.w.kept(logit_of(key));
          sm.digits[kFew + threadIdx.x] = w;
        }
        const uint64_t total = block_sum(sm, w);
        const uint64_t want = want_of(a, row, total);
        if (w > 0) {
          uint64_t before = 0;
          for (int j = 0; j < m; ++j)
            before += (int)(sm.digits[j] >> 32) < mine ? sm.digits[kFew + j] : 0;
          if (before <= want && want < before + w)
            answer(a, row, mine, log_share(s, logit_of(key), total));
        }
        if (threadIdx.x == 0) a.cut[row].done = 1;
        return;
      }
    }
  }
  if (threadIdx.x == 0) a.cut[row] = RowCut{cut, 0, {}};
}

// ----------------------------------------------------------------------------
// Weigh
// ----------------------------------------------------------------------------
__global__ __launch_bounds__(kPartThreads) void sample_weigh_kernel(SampleArgs a, int64_t unit0) {
  const int64_t unit = unit0 + blockIdx.x;
  const int64_t row = unit / a.parts;
  const int part = (int)(unit % a.parts);
  const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
  const PartInfo info = row_info(a, row);
  if (info.top == -INFINITY) return;
  const Settings s = settings_of(a, Given(a, row), info.top);
  if (s.greedy) return;
  const Row<EI_LOGITS_FP32> r(a, row);
  const int b0 = part * a.part_blocks, b1 = min(b0 + a.part_blocks, a.blocks);
  if (!s.cuts) {
    for (int b = b0 + wave; b < b1; b += kPartWaves) {
      float x[kBlockPieces][8];
      r.load_block(b, lane, x);
      uint64_t sum = 0;
#pragma unroll
      for (int q = 0; q < kBlockPieces; ++q)
#pragma unroll
        for (int e = 0; e < 8; ++e) sum += s.w.kept(x[q][e]);
      sum = wave_sum_u64(sum);
      if (lane == 0) a.sums[row * a.blocks + b] = sum;
    }
    return;
  }
  const RowCut rc = a.cut[row];
  if (rc.done) return;
  const uint32_t cut = rc.cut.key;
  for (int b = b0 + wave; b < b1; b += kPartWaves) {
    float x[kBlockPieces][8];
    r.load_block(b, lane, x);
    uint64_t sum = 0;
    uint32_t equal = 0;
#pragma unroll
    for (int q = 0; q < kBlockPieces; ++q)
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const uint32_t key = key_of(x[q][e]);
        if (key > cut) sum += s.w.kept(x[q][e]);
        equal += key != 0 && key == cut;
      }
    sum = wave_sum_u64(sum);
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) equal += __shfl_xor(equal, o);
    if (lane == 0) {
      a.sums[row * a.blocks + b] = sum;
      a.equal[row * a.blocks + b] = equal;
    }
  }
}

// ----------------------------------------------------------------------------
// Pick
// ----------------------------------------------------------------------------
constexpr int kPickWaves = kPickThreads / kWave;

__global__ __launch_bounds__(kPickThreads) void sample_pick_kernel(SampleArgs a, int64_t row0) {
  __shared__ uint64_t wave_sum[2][kPickWaves];
  __shared__ uint32_t wave_min[kPickWaves];
  __shared__ uint64_t found_above, found_equal;
  __shared__ int found;
  const int64_t row = row0 + blockIdx.x;
  const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
  const Row<EI_LOGITS_FP32> r(a, row);
  const PartInfo info = row_info(a, row);
  if (info.top == -INFINITY) {
    if (threadIdx.x == 0) answer(a, row, -1, -INFINITY);
    return;
  }
  const Settings s = settings_of(a, Given(a, row), info.top);
  if (s.greedy) {
    // in the first part that has it
    const float top = lane < a.parts ? a.part[row * a.parts + lane].top : -INFINITY;
    const int part = __builtin_ctzll(__builtin_amdgcn_ballot_w64(top == info.top));
    const int b0 = part * a.part_blocks, b1 = min(b0 + a.part_blocks, a.blocks);
    uint32_t at = UINT_MAX;
    for (int q = b0 * kBlockPieces + wave; q < b1 * kBlockPieces; q += kPickWaves) {
      float x[8];
      r.load(q, lane, x);
#pragma unroll
      for (int e = 7; e >= 0; --e)
        if (x[e] == info.top) at = min(at, (uint32_t)(r.index(q, lane) + e));
    }
    at = wave_min_u32_f(at);
    if (lane == 0) wave_min[wave] = at;
    __syncthreads();
    if (threadIdx.x == 0) {
      for (int w = 0; w < kPickWaves; ++w) at = min(at, wave_min[w]);
      answer(a, row, (int)at, 0.0);
    }
    return;
  }
  Cut cut{0, 0};
  if (s.cuts) {
    const RowCut rc = a.cut[row];
    if (rc.done) return;
    cut = rc.cut;
  }
  const uint64_t w_cut = cut.key ? s.w.kept(logit_of(cut.key)) : 0;
  auto kept = [&](uint64_t before) { return before < cut.count ? before : cut.count; };
  // the sum over this thread and those before it
  auto up_to = [&](int which, uint64_t v, uint64_t& total) -> uint64_t {
    v = wave_incl_scan_u64(v);
    if (lane == kWave - 1) wave_sum[which][wave] = v;
    __syncthreads();
    total = 0;
    for (int w = 0; w < kPickWaves; ++w) {
      if (w < wave) v += wave_sum[which][w];
      total += wave_sum[which][w];
    }
    return v;
  };
  const bool in = (int)threadIdx.x < a.blocks;
  const int64_t at = row * a.blocks + threadIdx.x;
  const uint64_t equal = in && cut.key ? a.equal[at] : 0;
  uint64_t total, equals;
  const uint64_t equal_end = up_to(0, equal, equals), equal_begin = equal_end - equal;
  const uint64_t sum = (in ? a.sums[at] : 0) + (kept(equal_end) - kept(equal_begin)) * w_cut;
  const uint64_t end = up_to(1, sum, total), want = want_of(a, row, total);
  if (end - sum <= want && want < end) {
    found = (int)threadIdx.x;
    found_above = end - sum;
    found_equal = equal_begin;
  }
  __syncthreads();
  if (wave != 0) return;
  uint64_t run = found_above, same = found_equal;
  const int b = found;
  for (int q = b * kBlockPieces; q < (b + 1) * kBlockPieces; ++q) {
    float x[8];
    r.load(q, lane, x);
    uint32_t n_same = 0;
    uint64_t mine = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const uint32_t key = key_of(x[e]);
      if (key > cut.key) mine += s.w.kept(x[e]);
      n_same += key != 0 && key == cut.key;
    }
    const uint64_t same_end = same + wave_incl_scan_u32(n_same), same_begin = same_end - n_same;
    mine += (kept(same_end) - kept(same_begin)) * w_cut;
    const uint64_t mine_end = run + wave_incl_scan_u64(mine);
    uint64_t to = mine_end - mine;
    if (to <= want && want < mine_end) {
      uint64_t n = same_begin;
      for (int e = 0; e < 8; ++e) {
        const uint32_t key = key_of(x[e]);
        if (key > cut.key) to += s.w.kept(x[e]);
        else if (key != 0 && key == cut.key && n++ < cut.count) to += w_cut;
        if (to > want) {
          answer(a, row, r.index(q, lane) + e, log_share(s, x[e], total));
          break;
        }
      }
    }
    run = __shfl(mine_end, kWave - 1);
    same = __shfl(same_end, kWave - 1);
    if (want < run) return;
  }
}

// ----------------------------------------------------------------------------
// A row of bf16 in one workgroup
//
// bf16 has few values between the largest logit and where weights vanish, so the
// weights come from a table in LDS by the bits of the logit: the 16 binades up to the
// largest logit, and those up to the farthest negative one that weighs something.
// The tokens counted by the same bits tell the cuts of top-k and top-p exactly, in
// one scan over the table: its entries are single values.  Values nearer to 0 than
// the tables reach (2^-16 of their ends) are rare: their weights are computed one by
// one, and a cut among them is searched for in the row.
// ----------------------------------------------------------------------------
constexpr int kMaxPieces = kMaxVocab / kPiece + 1;
constexpr int kSide = 2047;                        // table entries of a sign
constexpr int kTable = 2 * (kSide + 1);            // (the last of each: weight 0)

typedef short s16x2 __attribute__((ext_vector_type(2)));
typedef unsigned short u16x2 __attribute__((ext_vector_type(2)));

struct RowSmem {
  PickSmem pick;
  uint64_t weight[kTable];
  uint32_t count[kTable + kWave];      // (the last 64: of logits without an entry)
  uint64_t piece_sum[kMaxPieces];
  float wave_top[kWaves];
  int small_count, found;
  uint64_t small_sum, found_before, found_weight, found_count;
  uint64_t wave_sums[kWaves][2];
};

// The magnitude bits of a bf16 number, those of `x` (>= 0) rounded up.
__device__ __forceinline__ int bits_above(double x) {
  if (!(x < 3e38)) return 0x7f7f;
  const uint32_t b = __float_as_uint((float)fmax(x, 0.0)) >> 16;
  return min((int)b + 2, 0x7f7f);     // (the conversion may have rounded down)
}

// What several workgroups of a row have in common.
struct RowState {
  Cut cut;
  uint64_t small_sum;
  uint32_t small_count;
  uint32_t split;
};

struct RowWork {
  const SampleArgs& a;
  RowSmem& sm;
  const int64_t row;
  const Row<EI_LOGITS_BF16> r;
  const int lane, wave, full, pieces;
  int q0, q1;                  // this wave's pieces
  Settings s;
  int base_p, base_n;
  Cut cut;
  bool split;                  // not all tokens of the cut's key are kept

  __device__ __forceinline__ RowWork(const SampleArgs& a_, RowSmem& sm_, int64_t row_)
      : a(a_), sm(sm_), row(row_), r(a_, row_), lane(threadIdx.x % kWave), wave(threadIdx.x / kWave),
        full(a_.vocab / kPiece), pieces((a_.vocab + kPiece - 1) / kPiece), cut{0, 0}, split(false) {
    take(0, 1);
  }
  // The workgroup's are part `part` of `parts`; a wave's lie one behind the other.
  __device__ __forceinline__ void take(int part, int parts) {
    const int of_part = (pieces + parts - 1) / parts, per = (of_part + kWaves - 1) / kWaves;
    const int p0 = min(part * of_part, pieces), p1 = min(p0 + of_part, pieces);
    q0 = min(p0 + wave * per, p1);
    q1 = min(q0 + per, p1);
  }

  // All of them: use(words, piece), four loads under way while four pieces are used.
  // (The row is read again for each pass, from the caches: in registers, 64 a thread,
  // the passes have to be unrolled, and waiting for code that runs once took most of
  // the time, 62 us for a row of 128256.)
  template <class Use>
  __device__ __forceinline__ void each_piece(Use use) const {
    constexpr int kAhead = 4;
    uint4 next[kAhead];
    const int qf = min(q1, full);
    auto ask = [&](int q) {
      if (q + kAhead <= qf)
#pragma unroll
        for (int i = 0; i < kAhead; ++i) next[i] = r.load_full(q + i, lane);
    };
    int q = q0;
    ask(q);
#pragma unroll 1
    for (; q + kAhead <= qf; q += kAhead) {
      uint4 now[kAhead];
#pragma unroll
      for (int i = 0; i < kAhead; ++i) now[i] = next[i];
      ask(q + kAhead);
#pragma unroll
      for (int i = 0; i < kAhead; ++i) {
        const uint32_t words[4] = {now[i].x, now[i].y, now[i].z, now[i].w};
        use(words, q + i);
      }
    }
#pragma unroll 1
    for (; q < q1; ++q) {
      const uint4 now = r.load_raw(q, lane);
      const uint32_t words[4] = {now.x, now.y, now.z, now.w};
      use(words, q);
    }
  }
  __device__ __forceinline__ static uint32_t bits_of(const uint32_t (&words)[4], int e) {
    return e & 1 ? words[e / 2] >> 16 : words[e / 2] & 0xffffu;
  }
  __device__ __forceinline__ static float value(uint32_t bits) { return __uint_as_float(bits << 16); }

  __device__ __forceinline__ float largest() {
    float top = -INFINITY;
    each_piece([&](const uint32_t (&words)[4], int) {
#pragma unroll
      for (int w = 0; w < 4; ++w) top = fmaxf(top, fmaxf(bf16_lo(words[w]), bf16_hi(words[w])));
    });
    top = wave_max_f32_dpp(top);
    if (lane == 0) sm.wave_top[wave] = top;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < kWaves; ++w) top = fmaxf(top, sm.wave_top[w]);
    return top;
  }

  // The first token of the largest logit.
  __device__ __forceinline__ void take_largest(float top) {
    uint32_t at = UINT_MAX;
    each_piece([&](const uint32_t (&words)[4], int q) {
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if (value(bits_of(words, e)) == top) at = min(at, (uint32_t)(r.index(q, lane) + e));
    });
    at = wave_min_u32_f(at);
    if (lane == 0) sm.pick.wave_bits[0][wave] = at;
    __syncthreads();
    if (threadIdx.x == 0) {
      for (int w = 0; w < kWaves; ++w) at = min(at, sm.pick.wave_bits[0][w]);
      answer(a, row, (int)at, 0.0);
    }
  }

  // The tables: entry i of a sign is the magnitude base - i.  Negative logits past
  // 46 binary places below the top weigh nothing.
  __device__ __forceinline__ void place_tables(const Settings& settings, float top) {
    s = settings;
    base_p = max(top > 0.0f ? (int)(__float_as_uint(top) >> 16) : 0, kSide);
    base_n = max(bits_above(46.0 / s.w.per_t - s.w.top), kSide);
  }
  __device__ __forceinline__ uint32_t bits_at(int entry) const {
    return entry > kSide ? 0x8000u | (uint32_t)(base_n - (entry - kSide - 1))
                         : (uint32_t)(base_p - entry);
  }
  __device__ __forceinline__ void clear_counts() {
    for (int i = threadIdx.x; i < kTable; i += kThreads) sm.count[i] = 0;
    if (threadIdx.x == 0) {
      sm.small_count = 0;
      sm.small_sum = 0;
    }
  }
  __device__ __forceinline__ void fill_weights() {
    for (int i = threadIdx.x; i < kTable; i += kThreads)
      sm.weight[i] = (i & kSide) < kSide ? s.w.of(value(bits_at(i))) : 0;
  }

  // (the entry, as it is; kSide and more: nearer to 0 than the table, below zero:
  // weighs nothing, NaN and -inf among them)
  __device__ __forceinline__ int off_of(uint32_t bits) const {
    return (bits & 0x8000u ? base_n : base_p) - (int)(bits & 0x7fffu);
  }
  // The entries of two logits (the last of their sign where they have none), 8 times
  // each, in 16-bit pairs; `off`: theirs.
  __device__ __forceinline__ uint32_t entries_of(uint32_t word, s16x2& off) const {
    const uint32_t base_p2 = (uint32_t)base_p * 0x10001u, base_n2 = (uint32_t)base_n * 0x10001u;
    const uint32_t sign = __builtin_bit_cast(uint32_t, __builtin_bit_cast(s16x2, word) >> 15);
    const uint32_t base = (sign & base_n2) | (~sign & base_p2);
    off = __builtin_bit_cast(s16x2, base) - __builtin_bit_cast(s16x2, word & 0x7fff7fffu);
    const u16x2 at = __builtin_elementwise_min(__builtin_bit_cast(u16x2, off), u16x2{kSide, kSide});
    const uint32_t entry = (sign & (uint32_t)((kSide + 1) * 0x10001)) | __builtin_bit_cast(uint32_t, at);
    return entry << 3;
  }
  __device__ __forceinline__ static bool any_small(s16x2 most) { return most.x >= kSide || most.y >= kSide; }
  // those nearer to 0 than the tables, of a thread's piece: use(bits)
  template <class Use>
  __device__ __forceinline__ void each_small_of(const uint32_t (&words)[4], Use use) const {
    const uint32_t w0 = words[0], w1 = words[1], w2 = words[2], w3 = words[3];
#pragma unroll 1
    for (int e = 0; e < 8; ++e) {
      const uint32_t w = e < 4 ? e < 2 ? w0 : w1 : e < 6 ? w2 : w3;
      const uint32_t bits = e & 1 ? w >> 16 : w & 0xffffu;
      if (off_of(bits) >= kSide) use(bits);
    }
  }

  // The tokens of each entry.
  __device__ __forceinline__ void count() {
    uint64_t small_sum = 0;
    int small_count = 0;
    each_piece([&](const uint32_t (&words)[4], int) {
      s16x2 most = {-1, -1};
#pragma unroll
      for (int w = 0; w < 4; ++w) {
        s16x2 off;
        const uint32_t at = entries_of(words[w], off);
        most = __builtin_elementwise_max(most, off);
        // (the lanes without an entry count apart, each for itself)
        constexpr uint32_t kNone = 8 * kSide;
        const uint32_t lo = at & 0xffffu, hi = at >> 16;
        atomicAdd(&sm.count[(lo & kNone) == kNone ? kTable + lane : lo >> 3], 1u);
        atomicAdd(&sm.count[(hi & kNone) == kNone ? kTable + lane : hi >> 3], 1u);
      }
      if (any_small(most))
        each_small_of(words, [&](uint32_t bits) {
          ++small_count;
          small_sum += s.w.of(value(bits));
        });
    });
    if (small_count) {
      atomicAdd(&sm.small_count, small_count);
      atomicAdd((unsigned long long*)&sm.small_sum, (unsigned long long)small_sum);
    }
  }

  // The cut of top-k and top-p, from the counts and weights; the pieces taken are the
  // whole row's.
  __device__ __forceinline__ void find() {
    // the values in their order, four a thread: positive, near 0, negative
    constexpr int kEach = kTable / kThreads;
    auto place_of = [](int at) { return at <= kSide ? at : kSide + 1 + (2 * kSide - at); };
    uint32_t counts[kEach];
    uint64_t weights[kEach], n_all = 0, w_all = 0;
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
      const int at = (int)threadIdx.x * kEach + i, place = place_of(min(at, 2 * kSide));
      counts[i] = at == kSide ? (uint32_t)sm.small_count : at > 2 * kSide ? 0 : sm.count[place];
      weights[i] = at == kSide ? sm.small_sum : counts[i] * sm.weight[place];
      n_all += counts[i];
      w_all += weights[i];
    }
    // (both sums at once)
    uint64_t n_to = wave_incl_scan_u64(n_all), w_to = wave_incl_scan_u64(w_all), total_n = 0, total_w = 0;
    if (lane == kWave - 1) {
      sm.wave_sums[wave][0] = n_to;
      sm.wave_sums[wave][1] = w_to;
    }
    __syncthreads();
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
      const uint64_t n = sm.wave_sums[w][0], v = sm.wave_sums[w][1];
      n_to += w < wave ? n : 0;
      w_to += w < wave ? v : 0;
      total_n += n;
      total_w += v;
    }
    auto each_small = [&](auto use) {
#pragma unroll 1
      for (int q = q0; q < q1; ++q) {
        const uint4 again = r.load_raw(q, lane);
        const uint32_t words[4] = {again.x, again.y, again.z, again.w};
        each_small_of(words, [&](uint32_t bits) { use(key_of(value(bits))); });
      }
    };
    auto weight = [&](uint32_t key) { return s.w.of(logit_of(key)); };
    uint64_t cut_before = 0;
    int cut_at = -1;
    uint64_t same = 0;         // tokens of the cut's key
    // top-k by counts, then top-p by weights
#pragma unroll 1
    for (int stage = 0; stage < 2; ++stage) {
      const bool by_count = stage == 0;
      // (the tokens past all that weigh something need no cut)
      if (by_count ? s.k == 0 || (uint64_t)s.k >= total_n : s.p >= 1.0f) continue;
      uint64_t want = (uint64_t)s.k;
      if (!by_count) {
        if (cut_at >= 0) {       // the weight of top-k's tokens
          uint64_t mine = 0;
          if (cut_at == kSide)
            each_small([&](uint32_t key) {
              if (key > cut.key) mine += weight(key);
            });
          total_w = cut_before + block_sum(sm.pick, mine) + cut.count * weight(cut.key);
        }
        const double real = ceil((double)s.p * (double)total_w);
        want = real < 1.0 ? 1 : (uint64_t)real;
      }
      Cut in{0, 0};
      if (cut_at >= 0 && cut_before < want) {      // in the same entry
        in = cut;
        want -= cut_before;
      } else {
        // the entry at which the values reach `want`, and what lies before it
        uint64_t before = by_count ? n_to - n_all : w_to - w_all;
        uint64_t weight_before = w_to - w_all;
        __syncthreads();
        const uint64_t end = before + (by_count ? n_all : w_all);
        if (before < want && want <= end)
#pragma unroll
          for (int i = 0; i < kEach; ++i) {
            const uint64_t v = by_count ? counts[i] : weights[i];
            if (before < want && want <= before + v) {
              sm.found = place_of((int)threadIdx.x * kEach + i);
              sm.found_before = before;
              sm.found_weight = weight_before;
              sm.found_count = counts[i];
            }
            before += v;
            weight_before += weights[i];
          }
        __syncthreads();
        cut_at = sm.found;
        want -= sm.found_before;
        cut_before = sm.found_weight;
        same = sm.found_count;
      }
      if (cut_at == kSide) {
        cut = find_cut(sm.pick, in, want, each_small,
                       [&](uint32_t key) { return by_count ? (uint64_t)1 : weight(key); });
      } else {
        // (by counts nothing is to be divided)
        if (!by_count) want = (want + sm.weight[cut_at] - 1) / sm.weight[cut_at];
        cut = Cut{key_of(value(bits_at(cut_at))), want};
      }
    }
    if (cut.key) split = cut_at == kSide || cut.count < same;
    __syncthreads();
  }

  // What is not kept weighs nothing.  The cut's own key, where its tokens are split,
  // weighs kSame: a piece's sum (2^53 at most) then counts them above it.
  static constexpr int kSameBit = 54;
  static constexpr uint64_t kSame = (uint64_t)1 << kSameBit;
  static_assert(kPiece <= 1 << (63 - kSameBit), "512 of them");
  __device__ __forceinline__ uint64_t left_of(uint32_t key, uint64_t w) const {
    return split && key == cut.key ? kSame : key < cut.key || w < s.w.least ? 0 : w;
  }
  __device__ __forceinline__ uint64_t small_weight(uint32_t bits) const {
    return left_of(key_of(value(bits)), s.w.of(value(bits)));
  }
  __device__ __forceinline__ void keep() {
    for (int i = threadIdx.x; i < kTable; i += kThreads)
      if ((i & kSide) < kSide) sm.weight[i] = left_of(key_of(value(bits_at(i))), sm.weight[i]);
  }

  // The kept weights of each piece.
  __device__ __forceinline__ void weigh(uint64_t* piece_sum) const {
    const float least = cut.key ? logit_of(cut.key) : -INFINITY;
    each_piece([&](const uint32_t (&words)[4], int q) {
      uint64_t sum = 0;
      bool some = true;
      if (cut.key) {
        float most = -INFINITY;
#pragma unroll
        for (int w = 0; w < 4; ++w) most = fmaxf(most, fmaxf(bf16_lo(words[w]), bf16_hi(words[w])));
        some = __builtin_amdgcn_ballot_w64(most >= least) != 0;
      }
      if (some) {
        s16x2 most = {-1, -1};
#pragma unroll
        for (int w = 0; w < 4; ++w) {
          s16x2 off;
          const uint32_t at = entries_of(words[w], off);
          most = __builtin_elementwise_max(most, off);
          sum += *(const uint64_t*)((const char*)sm.weight + (at & 0xffffu));
          sum += *(const uint64_t*)((const char*)sm.weight + (at >> 16));
        }
        if (any_small(most))
          each_small_of(words, [&](uint32_t bits) { sum += small_weight(bits); });
        sum = wave_sum_u64(sum);
      }
      if (lane == 0) piece_sum[q] = sum;
    });
  }

  // The token, from the pieces' sums.
  template <bool TABLE>        // whether the table of weights is there
  __device__ __forceinline__ void pick(const uint64_t* piece_sum) {
    const uint64_t w_cut = split ? s.w.kept(logit_of(cut.key)) : 0;
    auto kept = [&](uint64_t before) { return before < cut.count ? before : cut.count; };
    // two pieces a thread
    const int qa = 2 * (int)threadIdx.x, qb = qa + 1;
    const uint64_t pa = qa < pieces ? piece_sum[qa] : 0, pb = qb < pieces ? piece_sum[qb] : 0;
    const uint64_t ea = pa >> kSameBit, eb = pb >> kSameBit;
    const uint64_t equal_end = split ? block_up_to(sm.pick, ea + eb) : 0, equal_mid = equal_end - eb;
    const uint64_t equal_begin = equal_mid - ea;
    const uint64_t ma = (pa & (kSame - 1)) + (kept(equal_mid) - kept(equal_begin)) * w_cut;
    const uint64_t mb = (pb & (kSame - 1)) + (kept(equal_end) - kept(equal_mid)) * w_cut;
    const uint64_t end = block_up_to(sm.pick, ma + mb), mid = end - mb, begin = mid - ma;
    uint64_t total = 0;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) total += sm.pick.wave_sum[w];
    const uint64_t want = want_of(a, row, total);
    if (begin <= want && want < end) {
      const bool second = mid <= want;
      sm.found = second ? qb : qa;
      sm.found_before = second ? mid : begin;
      sm.found_count = second ? equal_mid : equal_begin;
    }
    __syncthreads();
    if (wave != 0) return;
    const int q = sm.found;
    const uint4 again = r.load_raw(q, lane);
    const uint32_t words[4] = {again.x, again.y, again.z, again.w};
    uint64_t mine[8], all = 0;
    uint32_t n_same = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const uint32_t bits = bits_of(words, e);
      const int off = off_of(bits);
      const int entry = (int)(bits >> 15) * (kSide + 1) + (int)min((uint32_t)off, (uint32_t)kSide);
      mine[e] = !TABLE || off >= kSide ? small_weight(bits) : sm.weight[entry];
      n_same += (uint32_t)(mine[e] >> kSameBit);
    }
    uint64_t same = sm.found_count + wave_incl_scan_u32(n_same) - n_same;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      if (mine[e] >> kSameBit) mine[e] = same++ < cut.count ? w_cut : 0;
      all += mine[e];
    }
    uint64_t run = sm.found_before + wave_incl_scan_u64(all) - all;
    if (!(run <= want && want < run + all)) return;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const uint32_t bits = bits_of(words, e);
      if (run <= want && want < run + mine[e])
        answer(a, row, r.index(q, lane) + e, log_share(s, value(bits), total));
      run += mine[e];
    }
  }
};

__global__ __launch_bounds__(kThreads) void sample_row_kernel(SampleArgs a, int64_t row0) {
  __shared__ RowSmem sm;
  const int64_t row = row0 + blockIdx.x;
  RowWork work(a, sm, row);
  const Given given(a, row);
  const float top = work.largest();
  if (top == -INFINITY) {
    if (threadIdx.x == 0) answer(a, row, -1, -INFINITY);
    return;
  }
  const Settings s = settings_of(a, given, top);
  if (s.greedy) {
    work.take_largest(top);
    return;
  }
  work.place_tables(s, top);
  work.fill_weights();
  work.clear_counts();
  __syncthreads();
  if (s.cuts) {
    work.count();
    __syncthreads();
    work.find();
  }
  work.keep();
  __syncthreads();
  work.weigh(sm.piece_sum);
  __syncthreads();
  work.pick<true>(sm.piece_sum);
}

// ----------------------------------------------------------------------------
// A row of bf16 in several workgroups: the same steps, a launch up to each result that
// all of them need.  (The cut and the token by the last workgroup of a row to be done,
// in the launches before, took 270 us for 64 rows: its fences write back and discard
// an XCD's L2 for each wave.)
// ----------------------------------------------------------------------------
__device__ __forceinline__ float row_top(const SampleArgs& a, int64_t row) {
  const int lane = threadIdx.x % kWave;
  return wave_max_f32_dpp(lane < a.parts ? a.tops[row * a.parts + lane] : -INFINITY);
}

__global__ __launch_bounds__(kThreads) void sample_tops_kernel(SampleArgs a, int64_t unit0) {
  __shared__ RowSmem sm;
  const int64_t unit = unit0 + blockIdx.x, row = unit / a.parts;
  const int part = (int)(unit % a.parts);
  RowWork work(a, sm, row);
  work.take(part, a.parts);
  for (int i = part * kThreads + threadIdx.x; i < kTable; i += a.parts * kThreads)
    a.counts[row * kTable + i] = 0;
  if (part == 0 && threadIdx.x == 0) a.state[row] = RowState{};
  const float top = work.largest();
  if (threadIdx.x == 0) a.tops[unit] = top;
}

__global__ __launch_bounds__(kThreads) void sample_counts_kernel(SampleArgs a, int64_t unit0) {
  __shared__ RowSmem sm;
  const int64_t unit = unit0 + blockIdx.x, row = unit / a.parts;
  const Given given(a, row);
  const float top = row_top(a, row);
  if (top == -INFINITY) return;
  const Settings s = settings_of(a, given, top);
  if (!s.cuts) return;
  RowState& state = a.state[row];
  RowWork work(a, sm, row);
  work.take((int)(unit % a.parts), a.parts);
  work.place_tables(s, top);
  work.clear_counts();
  __syncthreads();
  work.count();
  __syncthreads();
  uint32_t* counts = a.counts + row * kTable;
  for (int i = threadIdx.x; i < kTable; i += kThreads)
    if (sm.count[i]) atomicAdd(&counts[i], sm.count[i]);
  if (threadIdx.x == 0 && sm.small_count) {
    atomicAdd(&state.small_count, (uint32_t)sm.small_count);
    atomicAdd((unsigned long long*)&state.small_sum, (unsigned long long)sm.small_sum);
  }
}

__global__ __launch_bounds__(kThreads) void sample_weights_kernel(SampleArgs a, int64_t unit0) {
  __shared__ RowSmem sm;
  const int64_t unit = unit0 + blockIdx.x, row = unit / a.parts;
  const int part = (int)(unit % a.parts);
  const Given given(a, row);
  constexpr int kEach = kTable / kThreads;
  uint32_t count[kEach] = {};
  if (a.top_k || a.top_p)
#pragma unroll
    for (int i = 0; i < kEach; ++i) count[i] = a.counts[row * kTable + i * kThreads + threadIdx.x];
  const float top = row_top(a, row);
  if (top == -INFINITY) {
    if (part == 0 && threadIdx.x == 0) answer(a, row, -1, -INFINITY);
    return;
  }
  const Settings s = settings_of(a, given, top);
  RowWork work(a, sm, row);
  if (s.greedy) {
    // in the first part that has it
    const float mine = work.lane < a.parts ? a.tops[row * a.parts + work.lane] : -INFINITY;
    if (part != (int)__builtin_ctzll(__builtin_amdgcn_ballot_w64(mine == top))) return;
    work.take(part, a.parts);
    work.take_largest(top);
    return;
  }
  work.place_tables(s, top);
  work.fill_weights();
  if (s.cuts) {        // each workgroup finds the cut by itself
    RowState& state = a.state[row];
#pragma unroll
    for (int i = 0; i < kEach; ++i) sm.count[i * kThreads + threadIdx.x] = count[i];
    if (threadIdx.x == 0) {
      sm.small_count = (int)state.small_count;
      sm.small_sum = state.small_sum;
    }
    __syncthreads();
    work.find();
    if (part == 0 && threadIdx.x == 0) {
      state.cut = work.cut;
      state.split = work.split;
    }
  }
  work.take(part, a.parts);
  work.keep();         // (a thread's entries are those that it filled)
  __syncthreads();
  work.weigh(a.sums + row * (int64_t)work.pieces);
}

__global__ __launch_bounds__(kThreads) void sample_token_kernel(SampleArgs a, int64_t row0) {
  __shared__ RowSmem sm;
  const int64_t row = row0 + blockIdx.x;
  const Given given(a, row);
  const float top = row_top(a, row);
  if (top == -INFINITY) return;
  const Settings s = settings_of(a, given, top);
  if (s.greedy) return;
  RowWork work(a, sm, row);
  work.place_tables(s, top);
  if (s.cuts) {
    work.cut = a.state[row].cut;
    work.split = a.state[row].split != 0;
  }
  work.pick<false>(a.sums + row * (int64_t)work.pieces);
}

// ----------------------------------------------------------------------------
// Host side
// ----------------------------------------------------------------------------
bool aligned(const void* p, uintptr_t a) { return ((uintptr_t)p & (a - 1)) == 0; }

struct SamplePlan {
  int blocks, parts, part_blocks;
  size_t at_cuts, at_bins, at_counts, at_sums, at_equal, at_state, bytes;
};
size_t up(size_t n) { return (n + 255) / 256 * 256; }
// fp32.  Parts of a row: as many as give the chip 1024 workgroups, of a block a wave at
// least.
SamplePlan fp32_plan(int rows, int vocab) {
  SamplePlan p{};
  const int tokens = kBlockPieces * kPiece;
  p.blocks = (vocab + tokens - 1) / tokens;
  if (p.blocks < 1) p.blocks = 1;
  int parts = 1024 / rows;
  const int most = (p.blocks + kPartWaves - 1) / kPartWaves;
  parts = parts > kMaxParts ? kMaxParts : parts < 1 ? 1 : parts;
  parts = parts > most ? most : parts;
  p.part_blocks = (p.blocks + parts - 1) / parts;
  p.parts = (p.blocks + p.part_blocks - 1) / p.part_blocks;
  p.at_cuts = up((size_t)rows * p.parts * sizeof(PartInfo));
  p.at_bins = p.at_cuts + up((size_t)rows * sizeof(RowCut));
  p.at_counts = p.at_bins + (size_t)rows * kBins * sizeof(uint64_t);
  p.at_sums = p.at_counts + (size_t)rows * kBins * sizeof(uint32_t);
  p.at_equal = p.at_sums + (size_t)rows * p.blocks * sizeof(uint64_t);
  p.bytes = p.at_equal + (size_t)rows * p.blocks * sizeof(uint32_t);
  return p;
}
// bf16.  A workgroup a row, or, of long rows, as many as the chip has CUs for, of a piece
// a wave at least.  In one and in several, us a call: 1 x 128256 (top-p) 33, 24; 32 rows
// of it 46, 32; 128 50, 45; 1 x 80000 26, 24; 1 x 65536 23, 23; 32 32, 29; but 1 x 50257
// 22, 24; 1 x 32001 18, 24.
SamplePlan bf16_plan(int rows, int vocab) {
  SamplePlan p{};
  const int pieces = (vocab + kPiece - 1) / kPiece;
  const int most = pieces / kWaves;
  p.parts = kCUs / rows;
  p.parts = p.parts > most ? most : p.parts;
  p.parts = p.parts > kMaxParts ? kMaxParts : p.parts;
  if (p.parts < 2 || pieces < 8 * kWaves) {
    p.parts = 1;
    return p;
  }
  p.at_sums = up((size_t)rows * p.parts * sizeof(float));
  p.at_state = p.at_sums + (size_t)rows * pieces * sizeof(uint64_t);
  p.at_counts = p.at_state + (size_t)rows * sizeof(RowState);
  p.bytes = p.at_counts + (size_t)rows * kTable * sizeof(uint32_t);
  return p;
}
SamplePlan sample_plan(int rows, int vocab, int format) {
  return format == EI_LOGITS_BF16 ? bf16_plan(rows, vocab) : fp32_plan(rows, vocab);
}

template <class Kernel>
void launch(Kernel kernel, const SampleArgs& a, int64_t groups, int threads, hipStream_t stream) {
  const int64_t most = (1ll << 31) / threads;
  for (int64_t u = 0; u < groups; u += most)
    hipLaunchKernelGGL(kernel, dim3((unsigned)(groups - u < most ? groups - u : most)),
                       dim3((unsigned)threads), 0, stream, a, u);
}
void launch_bf16(const SampleArgs& a, hipStream_t stream) {
  if (a.parts == 1) {
    launch(sample_row_kernel, a, a.rows, kThreads, stream);
    return;
  }
  const int64_t units = (int64_t)a.rows * a.parts;
  launch(sample_tops_kernel, a, units, kThreads, stream);
  if (a.top_k || a.top_p) launch(sample_counts_kernel, a, units, kThreads, stream);
  launch(sample_weights_kernel, a, units, kThreads, stream);
  launch(sample_token_kernel, a, a.rows, kThreads, stream);
}
void launch_fp32(const SampleArgs& a, hipStream_t stream) {
  const int64_t units = (int64_t)a.rows * a.parts;
  launch(sample_scan_kernel, a, units, kPartThreads, stream);
  if (a.top_k || a.top_p) {
    launch(sample_bins_kernel, a, units, kPartThreads, stream);
    launch(sample_cut_kernel, a, a.rows, kThreads, stream);
  }
  launch(sample_weigh_kernel, a, units, kPartThreads, stream);
  launch(sample_pick_kernel, a, a.rows, kPickThreads, stream);
}

bool valid(int32_t rows, int32_t vocab, int32_t format) {
  return (format == EI_LOGITS_BF16 || format == EI_LOGITS_FP32) && rows >= 0 && vocab >= 0;
}

}  // namespace
}  // namespace ei

extern "C" size_t ei_sample_workspace_bytes(int32_t rows, int32_t vocab, int32_t format) {
  if (!ei::valid(rows, vocab, format) || vocab > ei::kMaxVocab || rows == 0) return 0;
  return ei::sample_plan(rows, vocab, format).bytes;
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
  const ei::SamplePlan p = ei::sample_plan(rows, vocab, format);
  if (p.bytes && (!workspace || workspace_bytes < p.bytes)) return EI_ERR_WORKSPACE;
  if (!ei::aligned(workspace, 16)) return EI_ERR_UNSUPPORTED;
  char* ws = (char*)workspace;
  const ei::SampleArgs a{logits, rows, vocab, row_stride, u, temperature, top_k, top_p, min_p,
                         tokens, logprobs, p.parts, p.part_blocks, p.blocks, (ei::PartInfo*)ws,
                         (ei::RowCut*)(ws + p.at_cuts), (uint64_t*)(ws + p.at_sums),
                         (uint32_t*)(ws + p.at_equal), (uint64_t*)(ws + p.at_bins),
                         (uint32_t*)(ws + p.at_counts), (float*)ws, (ei::RowState*)(ws + p.at_state),
                         (uint32_t*)(ws + p.at_counts)};
  if (format == EI_LOGITS_BF16) ei::launch_bf16(a, (hipStream_t)stream);
  else ei::launch_fp32(a, (hipStream_t)stream);
  return hipGetLastError() == hipSuccess ? EI_OK : EI_ERR_LAUNCH;
}
