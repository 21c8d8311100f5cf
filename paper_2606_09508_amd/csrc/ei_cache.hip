// A paged cache of keys and values in 8 bits, and the attention that reads it.
//
// A page holds P tokens of every KV head ([KV head][P][128] codes, e4m3 or
// int8) and one fp32 scale per KV head; an element is code * scale.
//
//  store_kernel    new tokens into their sequences' pages
//  attend_kernel   the sequences' newest tokens over their pages
//  combine_kernel  joins the parts of a sequence's keys
//  copy_kernel     pages to other pages, over all layers of a cache
#include "../../include/entropyinfer.h"
#include "ei_internal.h"

#include <limits.h>
#include <math.h>

namespace ei {
namespace {

constexpr int kThreads = 256;
constexpr int kWaves = kThreads / kWave;

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x2 __attribute__((ext_vector_type(2)));

__device__ __forceinline__ uint32_t pack_bf16x2(float lo, float hi) {
  const f32x2 x = {lo, hi};
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(x, bf16x2));
}

// ----------------------------------------------------------------------------
// Where the tokens of sequence s lie in the packed tensors: `cu` (clamped to
// the tensor, so that no list leads out of it), or T / S tokens each.
// ----------------------------------------------------------------------------
struct Tokens {
  const int32_t* cu;
  int T, S, each;
};
__device__ __forceinline__ void seq_rows(const Tokens& t, int s, int& first, int& count) {
  if (!t.cu) {
    first = s * t.each;
    count = t.each;
    return;
  }
  first = min(max(t.cu[s], 0), t.T);
  count = max(min(max(t.cu[s + 1], 0), t.T) - first, 0);
}

// Work items of sequences whose lengths only the device knows.  With `cu`,
// sequence s owns the slots floor(cu[s] * num / den) + add * s up to the next
// one's first, which is floor(n_s * num / den) + add of them or one more.
__device__ __forceinline__ int64_t slot_of(const Tokens& t, int s, int num, int den, int add) {
  return (int64_t)min(max(t.cu[s], 0), t.T) * num / den + (int64_t)add * s;
}
// The sequence that owns `slot`, and the slot's number in it.
__device__ __forceinline__ void find_slot(const Tokens& t, int slot, int per_seq, int num, int den,
                                          int add, int& s, int& i) {
  if (!t.cu) {
    s = slot / per_seq;
    i = slot % per_seq;
    return;
  }
  int lo = 0, hi = t.S - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) / 2;
    if (slot_of(t, mid, num, den, add) <= slot) lo = mid; else hi = mid - 1;
  }
  s = lo;
  i = (int)(slot - slot_of(t, lo, num, den, add));
}

struct Pages {
  uint8_t *k, *v;
  float *ks, *vs;
  const int32_t* table;
  int n_pages, max_pages, Hkv, P;
};
// The page of table column c of sequence s, -1 where it is none.
__device__ __forceinline__ int page_at(const Pages& pg, int s, int c) {
  if (c < 0 || c >= pg.max_pages) return -1;
  const int p = pg.table[(int64_t)s * pg.max_pages + c];
  return (unsigned)p < (unsigned)pg.n_pages ? p : -1;
}

// ----------------------------------------------------------------------------
// Store.  One workgroup takes one page of one KV head and one of K and V: the
// largest magnitude of the new rows (as integers: bf16 magnitudes are ordered
// like their bits), the scale, the codes; each element is read once and kept
// in registers in between.  Where the page held rows of the sequence already
// and the scale grows, those are rounded again: by powers of two, so an e4m3
// code changes only where it leaves the normal range, and int8 errors of all
// roundings together stay below one step (1/2 + 1/4 + ...).
// ----------------------------------------------------------------------------
template <int FMT>
constexpr float kCodeMax = FMT == EI_CACHE_E4M3 ? 448.0f : 127.0f;

// The least power of two with a / 2^e <= kCodeMax, 2^-126 at least, for the
// bf16 magnitude bits a < 0x7f80: the code range ends at 1.75 * 2^8 (e4m3) or
// (2 - 2^-6) * 2^6 (int8), so the significand decides between two exponents.
template <int FMT>
__device__ __forceinline__ float scale_of(uint32_t a) {
  const uint32_t top = FMT == EI_CACHE_E4M3 ? 0x60u : 0x7eu;   // its 7 fraction bits
  const int e = (int)(a >> 7) - (FMT == EI_CACHE_E4M3 ? 8 : 6) + ((a & 0x7fu) > top ? 1 : 0);
  return __uint_as_float((uint32_t)max(e, 1) << 23);
}

__device__ __forceinline__ uint32_t e4m3x4(float a, float b, float c, float d) {
  int w = 0;
  w = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, w, false);
  w = __builtin_amdgcn_cvt_pk_fp8_f32(c, d, w, true);
  return (uint32_t)w;
}
template <int FMT>
__device__ __forceinline__ uint32_t encode4(float a, float b, float c, float d) {
  if constexpr (FMT == EI_CACHE_E4M3) return e4m3x4(a, b, c, d);
  auto one = [](float x) { return (uint32_t)(int)rintf(x) & 0xffu; };
  return one(a) | one(b) << 8 | one(c) << 16 | one(d) << 24;
}
template <int FMT>
__device__ __forceinline__ void decode4(uint32_t w, float (&f)[4]) {
  if constexpr (FMT == EI_CACHE_E4M3) {
    const f32x2 lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, false);
    const f32x2 hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, true);
    f[0] = lo.x; f[1] = lo.y; f[2] = hi.x; f[3] = hi.y;
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) f[i] = (float)(int8_t)(w >> (8 * i));
  }
}

// P / 16 chunks of 8 elements per thread.
template <int FMT, int P>
__global__ __launch_bounds__(kThreads) void store_kernel(const uint16_t* __restrict__ k,
                                                         const uint16_t* __restrict__ v, Tokens tk,
                                                         const int32_t* __restrict__ lengths,
                                                         Pages pg, int per_seq, int64_t unit0) {
  constexpr int CH = P * kHeadDim / 8 / kThreads;
  __shared__ uint32_t part[kWaves];
  const int64_t unit = unit0 + blockIdx.x;
  const int side = (int)(unit & 1);
  const int h = (int)((unit >> 1) % pg.Hkv);
  int s, i, first, n;
  find_slot(tk, (int)((unit >> 1) / pg.Hkv), per_seq, 1, P, 2, s, i);
  seq_rows(tk, s, first, n);
  const int64_t begin = (int64_t)lengths[s] - n;      // position of the first new token
  const int64_t from = begin > 0 ? begin : 0;         // (tokens before position 0 are dropped)
  const int64_t c = from / P + i;
  const int r0 = i == 0 ? (int)(from % P) : 0;        // the page's new rows: r0 .. r1 - 1
  const int64_t left = begin + n - c * P;
  const int r1 = (int)(left < P ? left : P);
  if (n == 0 || left <= r0 || c >= pg.max_pages) return;
  const int page = page_at(pg, s, (int)c);
  if (page < 0) return;
  const int64_t hp = (int64_t)page * pg.Hkv + h;
  float* sp = (side ? pg.vs : pg.ks) + hp;
  uint8_t* dst = (side ? pg.v : pg.k) + hp * P * kHeadDim;
  const uint16_t* src = (side ? v : k) +
                        ((int64_t)h * tk.T + first + (c * P - begin)) * kHeadDim;   // row 0
  const float s_old = r0 > 0 ? *sp : 0.0f;
  uint4 w[CH];
  uint32_t top = 0;
#pragma unroll
  for (int j = 0; j < CH; ++j) {
    const int ch = threadIdx.x + j * kThreads, r = ch >> 4;
    if (r >= r0 && r < r1) {
      w[j] = *(const uint4*)(src + (int64_t)ch * 8);
      const uint32_t ww[4] = {w[j].x, w[j].y, w[j].z, w[j].w};
#pragma unroll
      for (int e = 0; e < 4; ++e)
        top = max(top, max(ww[e] & 0x7fffu, (ww[e] >> 16) & 0x7fffu));
    }
  }
  top = wave_max_u32_f(top);
  if (threadIdx.x % kWave == 0) part[threadIdx.x / kWave] = top;
  __syncthreads();   // (and every thread has read the old scale)
#pragma unroll
  for (int j = 0; j < kWaves; ++j) top = max(top, part[j]);
  const bool bad = top >= 0x7f80u || s_old != s_old;
  const float sc = bad ? NAN : fmaxf(s_old, scale_of<FMT>(top));
  const float inv = bad ? 0.0f : 1.0f / sc;
  if (threadIdx.x == 0) *sp = sc;
  const float again = s_old * inv;
#pragma unroll
  for (int j = 0; j < CH; ++j) {
    const int ch = threadIdx.x + j * kThreads, r = ch >> 4;
    uint2* at = (uint2*)(dst + (int64_t)ch * 8);
    if (r < r0) {
      if (!bad && again != 1.0f) {
        float a[4], b[4];
        const uint2 o = *at;
        decode4<FMT>(o.x, a);
        decode4<FMT>(o.y, b);
        *at = make_uint2(encode4<FMT>(a[0] * again, a[1] * again, a[2] * again, a[3] * again),
                         encode4<FMT>(b[0] * again, b[1] * again, b[2] * again, b[3] * again));
      }
    } else if (r < r1) {
      const uint32_t ww[4] = {w[j].x, w[j].y, w[j].z, w[j].w};
      float f[8];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        f[2 * e] = bad ? 0.0f : bf16_lo(ww[e]) * inv;
        f[2 * e + 1] = bad ? 0.0f : bf16_hi(ww[e]) * inv;
      }
      *at = make_uint2(encode4<FMT>(f[0], f[1], f[2], f[3]), encode4<FMT>(f[4], f[5], f[6], f[7]));
    }
  }
}

// ----------------------------------------------------------------------------
// Attention.  The rows of a (sequence, KV head) are its new tokens times the
// G query heads of the group; a workgroup takes 16 of them over a part of the
// sequence's keys, its four waves every fourth step of 32 keys.  Per step
//   S^T = K Q^T        2 x 4  MFMA 16x16x32 (keys on M, rows on N)
//   O^T += V^T P^T     8      MFMA 16x16x32 (dims on M)
// straight from registers.  Operand layouts (lane l, j = l % 16, g = l / 16):
//   A[i][k]: i = j, k = 8g .. 8g+7      B[k][n]: n = j, k = 8g .. 8g+7
//   D[i][n]: n = j, i = 4g + r, r = 0..3
// The order of k is free as long as both operands share it.  K: a lane loads
// the bytes 64a + 16g .. +15 (a = 0, 1) of key 16u + j.  The S^T results it
// then holds are those of row j and the keys 16u + 4g + r, which are the 8
// keys of its B operand of the second product; it loads V's bytes 8j .. 8j+7 of
// the same keys, so operand i of 8 is V[those keys][8j + i] and D's dims are
// 8 (4g + r) + i.  Nothing crosses lanes but the row maxima, taken only when
// a score outgrows the running maximum.
// Codes become bf16 exactly (int8 has 7 bits and a sign, e4m3 4); the scale of K multiplies the
// fp32 scores, V's the fp32 probabilities, which are rounded to bf16 for the matrix cores as in
// the prompt's attention.
// ----------------------------------------------------------------------------
constexpr int kRows = 16;
constexpr int kKeys = 32;
constexpr float kFastLimit = 0x1p32f;
constexpr float kRescaleThreshold = 8.0f;

// Codes 2w, 2w + 1 of a word as packed bf16.
template <int FMT, bool HI>
__device__ __forceinline__ uint32_t widen2(uint32_t x) {
  if constexpr (FMT == EI_CACHE_E4M3) {
    return __builtin_bit_cast(uint32_t,
                              __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(x, 1.0f, HI));
  } else {
    const int lo = (int8_t)(x >> (HI ? 16 : 0)), hi = (int8_t)(x >> (HI ? 24 : 8));
    return pack_bf16x2((float)lo, (float)hi);
  }
}
template <int FMT>
__device__ __forceinline__ bf16x8 widen8(uint32_t x, uint32_t y) {
  return __builtin_bit_cast(bf16x8, make_uint4(widen2<FMT, false>(x), widen2<FMT, true>(x),
                                               widen2<FMT, false>(y), widen2<FMT, true>(y)));
}

struct Part {          // of a row: sums against the maximum m (base 2)
  float m, l;
};

template <int FMT, int P>
__global__ __launch_bounds__(kThreads) void attend_kernel(
    const uint16_t* __restrict__ q, Tokens tk, const int32_t* __restrict__ lengths, Pages pg,
    int Hq, int per_seq, int n_split, float sc_log2, uint16_t* __restrict__ o,
    Part* __restrict__ part_ml, float* __restrict__ part_o, int64_t unit0) {
  __shared__ float sm[kWaves][kRows], sl[kWaves][kRows];
  __shared__ __attribute__((aligned(16))) float so[kWaves][kRows * kHeadDim];
  const int G = Hq / pg.Hkv;
  const int64_t unit = unit0 + blockIdx.x;
  const int split = (int)(unit % n_split);
  const int64_t item = unit / n_split;
  const int kvh = (int)(item % pg.Hkv);
  int s, tile, first, n;
  find_slot(tk, (int)(item / pg.Hkv), per_seq, G, kRows, 1, s, tile);
  seq_rows(tk, s, first, n);
  const int row0 = tile * kRows;
  if (row0 >= n * G) return;
  const int lane = threadIdx.x % kWave, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const int j = lane & 15, g = lane >> 4;
  const int len = (int)min((int64_t)max(lengths[s], 0), (int64_t)pg.max_pages * P);

  // this lane's row: token and head; its last visible key
  const int row = row0 + j;
  const bool real = row < n * G;
  const int t = min(row, n * G - 1) / G, head = kvh * G + min(row, n * G - 1) % G;
  const int pos = lengths[s] - n + t;   // (rows past the last one repeat it)
  const int64_t qrow = (int64_t)head * tk.T + first + t;
  // the tile's keys: those its last row sees
  const int last = lengths[s] - n + min(row0 + kRows - 1, n * G - 1) / G;
  const int keys = max(min(last + 1, len), 0);
  const int steps = (keys + kKeys - 1) / kKeys;
  const int per = (steps + n_split - 1) / n_split;
  const int step0 = split * per, step1 = min(step0 + per, steps);

  bf16x8 qf[4];
#pragma unroll
  for (int a = 0; a < 4; ++a)   // dims 64 (a / 2) + 16 g + 8 (a % 2) ..
    qf[a] = __builtin_bit_cast(
        bf16x8, *(const uint4*)(q + qrow * kHeadDim + 64 * (a >> 1) + 16 * g + 8 * (a & 1)));

  f32x4 oacc[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) oacc[i] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
  float m_i = -INFINITY, l_i = 0.0f;

  for (int st = step0 + wave; st < step1; st += kWaves) {
    const int k0 = st * kKeys;
    const int page = page_at(pg, s, k0 / P);
    if (page < 0) continue;
    const int64_t hp = (int64_t)page * pg.Hkv + kvh;
    const uint8_t* kp = pg.k + (hp * P + k0 % P) * kHeadDim;
    const uint8_t* vp = pg.v + (hp * P + k0 % P) * kHeadDim;
    uint4 kw[2][2];
    uint2 vw[2][4];
#pragma unroll
    for (int u = 0; u < 2; ++u)
#pragma unroll
      for (int a = 0; a < 2; ++a)
        kw[u][a] = *(const uint4*)(kp + (16 * u + j) * kHeadDim + 64 * a + 16 * g);
#pragma unroll
    for (int u = 0; u < 2; ++u)
#pragma unroll
      for (int r = 0; r < 4; ++r)
        vw[u][r] = *(const uint2*)(vp + (16 * u + 4 * g + r) * kHeadDim + 8 * j);
    const float kf = pg.ks[hp] * sc_log2, vf = pg.vs[hp];
    f32x4 sacc[2];
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      sacc[u] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
      for (int a = 0; a < 2; ++a) {
        sacc[u] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(widen8<FMT>(kw[u][a].x, kw[u][a].y),
                                                          qf[2 * a], sacc[u], 0, 0, 0);
        sacc[u] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(widen8<FMT>(kw[u][a].z, kw[u][a].w),
                                                          qf[2 * a + 1], sacc[u], 0, 0, 0);
      }
    }
    float x[8];
    bool seen[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const int key = k0 + 16 * (e >> 2) + 4 * g + (e & 3);
      seen[e] = key <= pos && key < len;
      x[e] = seen[e] ? sacc[e >> 2][e & 3] * kf : -INFINITY;
    }
    // rows behind the sequence's end hold anything, NaN codes included
    if (k0 + kKeys > len) {
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if (k0 + 16 * (e >> 2) + 4 * g + (e & 3) >= len) vw[e >> 2][e & 3] = make_uint2(0u, 0u);
    }
    float p[8], lsum;
    auto probs = [&](float mneg) {
      lsum = 0.0f;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        p[e] = __builtin_amdgcn_exp2f(x[e] + mneg);
        lsum += p[e];
      }
    };
    bool kept = false;
    if (__builtin_amdgcn_ballot_w64(m_i == -INFINITY) == 0) {
      probs(-m_i);
      kept = __builtin_amdgcn_ballot_w64(!(lsum <= kFastLimit)) == 0;
    }
    if (!kept) {
      float mx = x[0];
#pragma unroll
      for (int e = 1; e < 8; ++e) mx = fmaxf(mx, x[e]);
      mx = fmaxf(mx, __shfl_xor(mx, 16));
      mx = fmaxf(mx, __shfl_xor(mx, 32));
      if (__builtin_amdgcn_ballot_w64(mx > m_i + kRescaleThreshold) != 0) {
        const float m_new = fmaxf(m_i, mx);
        const float alpha = m_new == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f(m_i - m_new);
        l_i *= alpha;
#pragma unroll
        for (int i = 0; i < 8; ++i) oacc[i] *= alpha;
        m_i = m_new;
      }
      probs(m_i == -INFINITY ? 0.0f : -m_i);
    }
    l_i += lsum;
    uint32_t pw[4];
#pragma unroll
    for (int e = 0; e < 4; ++e)
      pw[e] = pack_bf16x2(seen[2 * e] ? p[2 * e] * vf : 0.0f,
                          seen[2 * e + 1] ? p[2 * e + 1] * vf : 0.0f);
    const bf16x8 pf = __builtin_bit_cast(bf16x8, make_uint4(pw[0], pw[1], pw[2], pw[3]));
    // byte i of keys (0, 1), (2, 3) of each half, next to each other
#pragma unroll
    for (int half = 0; half < 2; ++half) {     // dims 8j + 4 half ..
      uint32_t pr[2][2][2];                    // [u][key pair][dims 0-1, 2-3]
#pragma unroll
      for (int u = 0; u < 2; ++u)
#pragma unroll
        for (int c = 0; c < 2; ++c) {
          const uint32_t a = half ? vw[u][2 * c].y : vw[u][2 * c].x;
          const uint32_t b = half ? vw[u][2 * c + 1].y : vw[u][2 * c + 1].x;
          pr[u][c][0] = __builtin_amdgcn_perm(b, a, 0x05010400u);
          pr[u][c][1] = __builtin_amdgcn_perm(b, a, 0x07030602u);
        }
#pragma unroll
      for (int w = 0; w < 2; ++w) {
        const bf16x8 v0 = __builtin_bit_cast(
            bf16x8, make_uint4(widen2<FMT, false>(pr[0][0][w]), widen2<FMT, false>(pr[0][1][w]),
                               widen2<FMT, false>(pr[1][0][w]), widen2<FMT, false>(pr[1][1][w])));
        const bf16x8 v1 = __builtin_bit_cast(
            bf16x8, make_uint4(widen2<FMT, true>(pr[0][0][w]), widen2<FMT, true>(pr[0][1][w]),
                               widen2<FMT, true>(pr[1][0][w]), widen2<FMT, true>(pr[1][1][w])));
        oacc[4 * half + 2 * w] =
            __builtin_amdgcn_mfma_f32_16x16x32_bf16(v0, pf, oacc[4 * half + 2 * w], 0, 0, 0);
        oacc[4 * half + 2 * w + 1] =
            __builtin_amdgcn_mfma_f32_16x16x32_bf16(v1, pf, oacc[4 * half + 2 * w + 1], 0, 0, 0);
      }
    }
  }

  // merge the waves
  l_i += __shfl_xor(l_i, 16);
  l_i += __shfl_xor(l_i, 32);
  if (g == 0) {
    sm[wave][j] = m_i;
    sl[wave][j] = l_i;
  }
#pragma unroll
  for (int r = 0; r < 4; ++r) {
    float* at = &so[wave][j * kHeadDim + 8 * (4 * g + r)];
    *(float4*)at = make_float4(oacc[0][r], oacc[1][r], oacc[2][r], oacc[3][r]);
    *(float4*)(at + 4) = make_float4(oacc[4][r], oacc[5][r], oacc[6][r], oacc[7][r]);
  }
  __syncthreads();
  const int mr = threadIdx.x >> 4, md = (threadIdx.x & 15) * 8;   // row, dims
  float m = sm[0][mr];
#pragma unroll
  for (int w = 1; w < kWaves; ++w) m = fmaxf(m, sm[w][mr]);
  float l = 0.0f, acc[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) acc[e] = 0.0f;
#pragma unroll
  for (int w = 0; w < kWaves; ++w) {
    const float f = sm[w][mr] == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(sm[w][mr] - m);
    l += f * sl[w][mr];
#pragma unroll
    for (int e = 0; e < 8; ++e) acc[e] += f * so[w][mr * kHeadDim + md + e];
  }
  if (row0 + mr >= n * G) return;
  if (n_split > 1) {
    const int64_t pr = unit * kRows + mr;
    if (md == 0) part_ml[pr] = Part{m, l};
#pragma unroll
    for (int e = 0; e < 8; e += 4)
      *(float4*)(part_o + pr * kHeadDim + md + e) =
          make_float4(acc[e], acc[e + 1], acc[e + 2], acc[e + 3]);
    return;
  }
  const float inv = l == 0.0f ? 0.0f : 1.0f / l;
  const int mt = (row0 + mr) / G, mh = kvh * G + (row0 + mr) % G;
  *(uint4*)(o + ((int64_t)mh * tk.T + first + mt) * kHeadDim + md) =
      make_uint4(pack_bf16x2(acc[0] * inv, acc[1] * inv), pack_bf16x2(acc[2] * inv, acc[3] * inv),
                 pack_bf16x2(acc[4] * inv, acc[5] * inv), pack_bf16x2(acc[6] * inv, acc[7] * inv));
}

// The parts of each row joined, in order.
__global__ __launch_bounds__(kThreads) void combine_kernel(
    Tokens tk, int Hq, int Hkv, int per_seq, int n_split, const Part* __restrict__ part_ml,
    const float* __restrict__ part_o, uint16_t* __restrict__ o, int64_t item0) {
  const int G = Hq / Hkv;
  const int64_t item = item0 + blockIdx.x;
  const int kvh = (int)(item % Hkv);
  int s, tile, first, n;
  find_slot(tk, (int)(item / Hkv), per_seq, G, kRows, 1, s, tile);
  seq_rows(tk, s, first, n);
  const int mr = threadIdx.x >> 4, md = (threadIdx.x & 15) * 8;
  const int row = tile * kRows + mr;
  if (row >= n * G) return;
  float m = -INFINITY;
  for (int w = 0; w < n_split; ++w) m = fmaxf(m, part_ml[(item * n_split + w) * kRows + mr].m);
  float l = 0.0f, acc[8] = {};
  for (int w = 0; w < n_split; ++w) {
    const int64_t pr = (item * n_split + w) * kRows + mr;
    const Part ml = part_ml[pr];
    const float f = ml.m == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(ml.m - m);
    l += f * ml.l;
#pragma unroll
    for (int e = 0; e < 8; ++e) acc[e] += f * part_o[pr * kHeadDim + md + e];
  }
  const float inv = l == 0.0f ? 0.0f : 1.0f / l;
  *(uint4*)(o + ((int64_t)(kvh * G + row % G) * tk.T + first + row / G) * kHeadDim + md) =
      make_uint4(pack_bf16x2(acc[0] * inv, acc[1] * inv), pack_bf16x2(acc[2] * inv, acc[3] * inv),
                 pack_bf16x2(acc[4] * inv, acc[5] * inv), pack_bf16x2(acc[6] * inv, acc[7] * inv));
}

// ----------------------------------------------------------------------------
// Copy.  One workgroup moves 16 KB of K or of V of a page of a layer.
// ----------------------------------------------------------------------------
constexpr int kCopyBytes = 16 * 1024;

__global__ __launch_bounds__(kThreads) void copy_kernel(Pages pg, int64_t n_moves, int parts,
                                                        const int32_t* __restrict__ src,
                                                        const int32_t* __restrict__ dst,
                                                        int64_t unit0) {
  int64_t u = unit0 + blockIdx.x;
  const int part = (int)(u % parts);
  u /= parts;
  const bool is_v = u & 1;
  u >>= 1;
  const int64_t move = u % n_moves, layer = u / n_moves;
  const int a = src[move], b = dst[move];
  if ((unsigned)a >= (unsigned)pg.n_pages || (unsigned)b >= (unsigned)pg.n_pages || a == b) return;
  const int64_t page_bytes = (int64_t)pg.Hkv * pg.P * kHeadDim;
  const int64_t base = layer * pg.n_pages;
  uint8_t* t = is_v ? pg.v : pg.k;
  const uint4* from = (const uint4*)(t + (base + a) * page_bytes);
  uint4* to = (uint4*)(t + (base + b) * page_bytes);
  const int64_t c0 = (int64_t)part * (kCopyBytes / 16), chunks = page_bytes / 16;
  uint4 w[kCopyBytes / 16 / kThreads];
#pragma unroll
  for (int j = 0; j < kCopyBytes / 16 / kThreads; ++j) {
    const int64_t c = c0 + threadIdx.x + j * kThreads;
    if (c < chunks) w[j] = from[c];
  }
#pragma unroll
  for (int j = 0; j < kCopyBytes / 16 / kThreads; ++j) {
    const int64_t c = c0 + threadIdx.x + j * kThreads;
    if (c < chunks) to[c] = w[j];
  }
  if (part == 0) {
    float* f = is_v ? pg.vs : pg.ks;
    for (int h = threadIdx.x; h < pg.Hkv; h += kThreads)
      f[(base + b) * pg.Hkv + h] = f[(base + a) * pg.Hkv + h];
  }
}

// ----------------------------------------------------------------------------
// Host side
// ----------------------------------------------------------------------------
constexpr int64_t kMaxGrid = (1ll << 31) / kThreads;   // threads of a launch: 32 bits
unsigned launch_grid(int64_t left) { return (unsigned)(left < kMaxGrid ? left : kMaxGrid); }

bool aligned(const void* p, uintptr_t a) { return ((uintptr_t)p & (a - 1)) == 0; }
ei_status from_hip(hipError_t e) { return e == hipSuccess ? EI_OK : EI_ERR_LAUNCH; }

ei_status check_shape(const ei_cache_shape& c) {
  if (c.n_pages < 0 || c.n_kv_heads <= 0 || c.head_dim <= 0) return EI_ERR_SHAPE;
  if (c.format != EI_CACHE_E4M3 && c.format != EI_CACHE_INT8) return EI_ERR_SHAPE;
  if (c.head_dim != kHeadDim || (c.page_len != 64 && c.page_len != 128)) return EI_ERR_UNSUPPORTED;
  if ((int64_t)c.n_pages * c.n_kv_heads > INT_MAX) return EI_ERR_SHAPE;
  return EI_OK;
}
ei_status check_pages(const ei_cache_pages& p) {
  if (!p.k || !p.v || !p.k_scale || !p.v_scale) return EI_ERR_NULL;
  if (!aligned(p.k, 16) || !aligned(p.v, 16) || !aligned(p.k_scale, 4) || !aligned(p.v_scale, 4))
    return EI_ERR_UNSUPPORTED;
  return EI_OK;
}
ei_status check_tokens(int32_t n_tokens, const int32_t* cu, int32_t n_seqs, int32_t max_pages) {
  if (n_tokens < 0 || n_seqs < 0 || max_pages < 0) return EI_ERR_SHAPE;
  if (!cu && n_seqs > 0 && n_tokens % n_seqs) return EI_ERR_SHAPE;
  return EI_OK;
}
Pages pages_of(const ei_cache_shape& c, const ei_cache_pages& p, const int32_t* table, int cols) {
  return Pages{(uint8_t*)p.k, (uint8_t*)p.v, p.k_scale, p.v_scale, table,
               c.n_pages, cols,          c.n_kv_heads, c.page_len};
}

struct AttendPlan {
  int per_seq, n_split;
  int64_t items;
  size_t ml_bytes, bytes;
};
// n_split: enough workgroups for the chip, at least 256 keys each.
AttendPlan attend_plan(int Hq, int n_tokens, bool ragged, int n_seqs, int max_pages,
                       const ei_cache_shape& c) {
  const int64_t G = Hq / c.n_kv_heads;
  AttendPlan p{};
  int64_t slots;
  if (ragged) {
    slots = (int64_t)n_tokens * G / kRows + n_seqs;
  } else {
    p.per_seq = (int)((n_tokens / n_seqs * G + kRows - 1) / kRows);
    slots = (int64_t)n_seqs * p.per_seq;
  }
  p.items = slots * c.n_kv_heads;
  const int64_t most = ((int64_t)max_pages * c.page_len + 255) / 256;
  int64_t sp = p.items > 0 ? (1024 + p.items - 1) / p.items : 1;
  if (sp > most) sp = most;
  p.n_split = (int)(sp < 1 ? 1 : sp);
  if (p.n_split > 1) {
    const size_t rows = (size_t)p.items * p.n_split * kRows;
    p.ml_bytes = (rows * sizeof(Part) + 255) / 256 * 256;
    p.bytes = p.ml_bytes + rows * kHeadDim * sizeof(float);
  }
  return p;
}

}  // namespace
}  // namespace ei

extern "C" {

ei_status ei_cache_store(const uint16_t* k, const uint16_t* v, int32_t n_tokens,
                         const int32_t* cu_seqlens, int32_t n_seqs, const int32_t* lengths,
                         const int32_t* page_table, int32_t max_pages, ei_cache_shape shape,
                         ei_cache_pages pages, void* stream) {
  ei_status st = ei::check_shape(shape);
  if (st != EI_OK) return st;
  if ((st = ei::check_tokens(n_tokens, cu_seqlens, n_seqs, max_pages)) != EI_OK) return st;
  const int P = shape.page_len;
  const int64_t each = n_seqs ? n_tokens / n_seqs : 0;
  const int64_t per_seq = (each + P - 2) / P + 1;
  const int64_t slots =
      cu_seqlens ? (int64_t)n_tokens / P + 2 * (int64_t)n_seqs : (int64_t)n_seqs * per_seq;
  if (slots > INT_MAX) return EI_ERR_SHAPE;
  if (n_tokens == 0 || n_seqs == 0 || max_pages == 0 || shape.n_pages == 0) return EI_OK;
  if (!k || !v || !lengths || !page_table) return EI_ERR_NULL;
  if ((st = ei::check_pages(pages)) != EI_OK) return st;
  if (!ei::aligned(k, 16) || !ei::aligned(v, 16) || !ei::aligned(lengths, 4) ||
      !ei::aligned(page_table, 4) || !ei::aligned(cu_seqlens, 4))
    return EI_ERR_UNSUPPORTED;
  const ei::Tokens tk{cu_seqlens, n_tokens, n_seqs, (int)each};
  const ei::Pages pg = ei::pages_of(shape, pages, page_table, max_pages);
  const int64_t units = slots * shape.n_kv_heads * 2;
  hipStream_t s0 = (hipStream_t)stream;
  for (int64_t u = 0; u < units; u += ei::kMaxGrid) {
    const dim3 grid(ei::launch_grid(units - u)), block(ei::kThreads);
#define EI_STORE(F, PL)                                                                        \
  hipLaunchKernelGGL((ei::store_kernel<F, PL>), grid, block, 0, s0, k, v, tk, lengths, pg,     \
                     (int)per_seq, u)
    if (shape.format == EI_CACHE_E4M3) {
      if (P == 64) EI_STORE(EI_CACHE_E4M3, 64); else EI_STORE(EI_CACHE_E4M3, 128);
    } else {
      if (P == 64) EI_STORE(EI_CACHE_INT8, 64); else EI_STORE(EI_CACHE_INT8, 128);
    }
#undef EI_STORE
  }
  return ei::from_hip(hipGetLastError());
}

size_t ei_cache_attn_workspace_bytes(int32_t n_q_heads, int32_t n_tokens, int32_t packed,
                                     int32_t n_seqs, int32_t max_pages, ei_cache_shape shape) {
  if (ei::check_shape(shape) != EI_OK || n_q_heads <= 0 || n_q_heads % shape.n_kv_heads ||
      n_tokens <= 0 || n_seqs <= 0 || max_pages <= 0 || (!packed && n_tokens % n_seqs))
    return 0;
  return ei::attend_plan(n_q_heads, n_tokens, packed != 0, n_seqs, max_pages, shape).bytes;
}

ei_status ei_cache_attn(const uint16_t* q, int32_t n_q_heads, int32_t n_tokens,
                        const int32_t* cu_seqlens, int32_t n_seqs, const int32_t* lengths,
                        const int32_t* page_table, int32_t max_pages, ei_cache_shape shape,
                        ei_cache_pages pages, float softmax_scale, uint16_t* o, void* workspace,
                        size_t workspace_bytes, void* stream) {
  ei_status st = ei::check_shape(shape);
  if (st != EI_OK && st != EI_ERR_UNSUPPORTED) return st;
  if (n_q_heads <= 0 || n_q_heads % shape.n_kv_heads) return EI_ERR_SHAPE;
  if (!(softmax_scale > 0.0f && softmax_scale <= 3.402823466e38f)) return EI_ERR_SHAPE;
  if (st != EI_OK) return st;
  if ((st = ei::check_tokens(n_tokens, cu_seqlens, n_seqs, max_pages)) != EI_OK) return st;
  if ((int64_t)n_tokens * n_q_heads > INT_MAX || (int64_t)max_pages * shape.page_len > INT_MAX)
    return EI_ERR_SHAPE;
  if (n_tokens == 0 || n_seqs == 0) return EI_OK;
  const ei::AttendPlan pl = ei::attend_plan(n_q_heads, n_tokens, cu_seqlens != nullptr, n_seqs,
                                            max_pages, shape);
  if (pl.items > INT_MAX) return EI_ERR_SHAPE;
  if (!q || !o || !lengths || !page_table) return EI_ERR_NULL;
  if ((st = ei::check_pages(pages)) != EI_OK) return st;
  if (!ei::aligned(q, 16) || !ei::aligned(o, 16) || !ei::aligned(lengths, 4) ||
      !ei::aligned(page_table, 4) || !ei::aligned(cu_seqlens, 4))
    return EI_ERR_UNSUPPORTED;
  if (pl.bytes && (!workspace || workspace_bytes < pl.bytes)) return EI_ERR_WORKSPACE;
  if (!ei::aligned(workspace, 16)) return EI_ERR_UNSUPPORTED;
  const ei::Tokens tk{cu_seqlens, n_tokens, n_seqs, n_tokens / n_seqs};
  const ei::Pages pg = ei::pages_of(shape, pages, page_table, max_pages);
  const float sc_log2 = (float)((double)softmax_scale * 1.4426950408889634);
  ei::Part* ml = (ei::Part*)workspace;
  float* po = (float*)((char*)workspace + pl.ml_bytes);
  const int64_t units = pl.items * pl.n_split;
  hipStream_t s0 = (hipStream_t)stream;
  for (int64_t u = 0; u < units; u += ei::kMaxGrid) {
    const dim3 grid(ei::launch_grid(units - u)), block(ei::kThreads);
#define EI_ATTEND(F, PL)                                                                       \
  hipLaunchKernelGGL((ei::attend_kernel<F, PL>), grid, block, 0, s0, q, tk, lengths, pg,       \
                     n_q_heads, pl.per_seq, pl.n_split, sc_log2, o, ml, po, u)
    if (shape.format == EI_CACHE_E4M3) {
      if (shape.page_len == 64) EI_ATTEND(EI_CACHE_E4M3, 64); else EI_ATTEND(EI_CACHE_E4M3, 128);
    } else {
      if (shape.page_len == 64) EI_ATTEND(EI_CACHE_INT8, 64); else EI_ATTEND(EI_CACHE_INT8, 128);
    }
#undef EI_ATTEND
  }
  if (pl.n_split > 1)
    for (int64_t u = 0; u < pl.items; u += ei::kMaxGrid)
      hipLaunchKernelGGL(ei::combine_kernel, dim3(ei::launch_grid(pl.items - u)),
                         dim3(ei::kThreads), 0, s0, tk, n_q_heads, shape.n_kv_heads, pl.per_seq,
                         pl.n_split, ml, po, o, u);
  return ei::from_hip(hipGetLastError());
}

ei_status ei_cache_copy(ei_cache_shape shape, int32_t n_layers, ei_cache_pages pages,
                        const int32_t* src, const int32_t* dst, int32_t n, void* stream) {
  ei_status st = ei::check_shape(shape);
  if (st != EI_OK) return st;
  if (n_layers < 0 || n < 0) return EI_ERR_SHAPE;
  if (n_layers == 0 || n == 0 || shape.n_pages == 0) return EI_OK;
  if (!src || !dst) return EI_ERR_NULL;
  if ((st = ei::check_pages(pages)) != EI_OK) return st;
  if (!ei::aligned(src, 4) || !ei::aligned(dst, 4)) return EI_ERR_UNSUPPORTED;
  const int64_t page_bytes = (int64_t)shape.n_kv_heads * shape.page_len * ei::kHeadDim;
  const int64_t parts = (page_bytes + ei::kCopyBytes - 1) / ei::kCopyBytes;
  if (parts > INT_MAX || parts * 2 * n > (int64_t)INT_MAX * 1024 / n_layers) return EI_ERR_SHAPE;
  const int64_t units = parts * 2 * n * n_layers;
  const ei::Pages pg = ei::pages_of(shape, pages, nullptr, 0);
  for (int64_t u = 0; u < units; u += ei::kMaxGrid)
    hipLaunchKernelGGL(ei::copy_kernel, dim3(ei::launch_grid(units - u)), dim3(ei::kThreads), 0,
                       (hipStream_t)stream, pg, (int64_t)n, (int)parts, src, dst, u);
  return ei::from_hip(hipGetLastError());
}

}  // extern "C"
