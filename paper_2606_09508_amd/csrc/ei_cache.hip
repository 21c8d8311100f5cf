// A paged cache of keys and values in 8 bits, and the attention that reads it.
//
// A page holds P tokens of every KV head ([KV head][P][128] codes, e4m3 or
// int8) and one fp32 scale per KV head; an element is code * scale.
//
//  store_kernel         new tokens into their sequences' pages
//  attend_kernel        the sequences' newest tokens over their pages, where the
//                       tables are short: a workgroup per item
//  attend_share_kernel  the same for tables of any length, the keys dealt out
//  combine_kernel       joins the parts of an item's keys that it leaves
//  copy_kernel          pages to other pages, over all layers of a cache
//
// All are bound by HBM once the calls are large (a copy of 1 GiB runs at 5.14
// TB/s, nontemporal reads of 2 GB at 7.1, ordinary ones at 6.2), by their chain
// of dependent loads when they are small:
//   store, 32768 tokens of 8 heads:            40 us, 5.1 TB/s (one token of each
//                                              of 64 sequences: 4.6 us)
//   attention, 32 heads over 8 KV heads,
//     8 sequences of up to 131072 tokens:      245 + 5 us, 6.6 TB/s
//     32 sequences of 131 to 7974 tokens:      47 + 5 us, 5.6 TB/s
//     1 sequence of 1000 tokens, 4 heads:      9 us
//   64 heads, 6 of about 13000, 4 new, int8:   37 + 5 us, 4.2 TB/s
//   copy, 150 pages of 128 tokens, 32 layers:  411 us, 6.1 TB/s
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

// Loads and stores of data that a launch touches once.
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
__device__ __forceinline__ uint4 load_once4(const void* p) {
  return __builtin_bit_cast(uint4, __builtin_nontemporal_load((const u32x4*)p));
}
__device__ __forceinline__ void store_once4(void* p, uint4 w) {
  __builtin_nontemporal_store(__builtin_bit_cast(u32x4, w), (u32x4*)p);
}

// Entry i of a list that the kernel only reads: where the lanes share i, through
// the scalar cache.  (Vector loads return in order, behind the keys that all waves
// of the CU have asked for.)
template <class T>
__device__ __forceinline__ T entry(const T* list, int64_t i) {
  return ((const __attribute__((address_space(4))) T*)list)[i];
}

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
  first = min(max(entry(t.cu, s), 0), t.T);
  count = max(min(max(entry(t.cu, s + 1), 0), t.T) - first, 0);
}

// Work items of sequences whose lengths only the device knows.  With `cu`,
// sequence s owns the slots floor(cu[s] * num / den) + add * s up to the next
// one's first, which is floor(n_s * num / den) + add of them or one more.
// (T * num and the slots of all sequences are below 2^31, or the call is refused.)
__device__ __forceinline__ int slot_of(const Tokens& t, int s, int num, int den, int add) {
  return (int)((unsigned)(min(max(entry(t.cu, s), 0), t.T) * num) / (unsigned)den) + add * s;
}
// The sequence that owns `slot`, and the slot's number in it (below zero for the
// slots of the rows before the first sequence, which are nobody's).
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
  i = slot - slot_of(t, lo, num, den, add);
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
  const int p = entry(pg.table, (int64_t)s * pg.max_pages + c);
  return (unsigned)p < (unsigned)pg.n_pages ? p : -1;
}

// ----------------------------------------------------------------------------
// Store.  One workgroup takes a page of one KV head, K and V: the largest
// magnitude of the new rows (as integers: bf16 magnitudes are ordered like
// their bits), the scale, the codes; each element is read once and kept in
// registers in between.  Where the page held rows of the sequence already and
// the scale grows, those are rounded again: by powers of two, so an e4m3 code
// changes only where it leaves the normal range, and int8 errors of all
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

// P / 16 chunks of 8 elements of K and of V per thread.
template <int FMT, int P>
__global__ __launch_bounds__(kThreads) void store_kernel(const uint16_t* __restrict__ k,
                                                         const uint16_t* __restrict__ v, Tokens tk,
                                                         const int32_t* __restrict__ lengths,
                                                         Pages pg, int per_seq, int64_t unit0) {
  constexpr int CH = P * kHeadDim / 8 / kThreads;
  __shared__ uint32_t part[2][kWaves];
  const int64_t unit = unit0 + blockIdx.x;
  const int h = (int)(unit % pg.Hkv);
  int s, i, first, n;
  find_slot(tk, (int)(unit / pg.Hkv), per_seq, 1, P, 2, s, i);
  seq_rows(tk, s, first, n);
  const int64_t begin = (int64_t)entry(lengths, s) - n;      // position of the first new token
  const int64_t from = begin > 0 ? begin : 0;         // (tokens before position 0 are dropped)
  const int64_t c = from / P + i;
  const int r0 = i == 0 ? (int)(from % P) : 0;        // the page's new rows: r0 .. r1 - 1
  const int64_t left = begin + n - c * P;
  const int r1 = (int)(left < P ? left : P);
  if (i < 0 || n == 0 || left <= r0 || c >= pg.max_pages) return;
  const int page = page_at(pg, s, (int)c);
  if (page < 0) return;
  const int64_t hp = (int64_t)page * pg.Hkv + h;
  const int64_t src = ((int64_t)h * tk.T + first + (c * P - begin)) * kHeadDim;   // row 0
  float* const scales[2] = {pg.ks + hp, pg.vs + hp};
  const float s_old[2] = {r0 > 0 ? *scales[0] : 0.0f, r0 > 0 ? *scales[1] : 0.0f};
  uint4 w[2][CH];
#pragma unroll
  for (int side = 0; side < 2; ++side)
#pragma unroll
    for (int j = 0; j < CH; ++j) {
      const int ch = threadIdx.x + j * kThreads, r = ch >> 4;
      w[side][j] = r >= r0 && r < r1 ? load_once4((side ? v : k) + src + (int64_t)ch * 8)
                                     : make_uint4(0u, 0u, 0u, 0u);
    }
#pragma unroll
  for (int side = 0; side < 2; ++side) {
    uint32_t top = 0;
#pragma unroll
    for (int j = 0; j < CH; ++j) {
      const uint32_t ww[4] = {w[side][j].x, w[side][j].y, w[side][j].z, w[side][j].w};
#pragma unroll
      for (int e = 0; e < 4; ++e)
        top = max(top, max(ww[e] & 0x7fffu, (ww[e] >> 16) & 0x7fffu));
    }
    top = wave_max_u32_f(top);
    if (threadIdx.x % kWave == 0) part[side][threadIdx.x / kWave] = top;
  }
  __syncthreads();   // (and every thread has read the old scales)
#pragma unroll
  for (int side = 0; side < 2; ++side) {
    uint32_t top = part[side][0];
#pragma unroll
    for (int j = 1; j < kWaves; ++j) top = max(top, part[side][j]);
    const bool bad = top >= 0x7f80u || s_old[side] != s_old[side];
    const float sc = bad ? NAN : fmaxf(s_old[side], scale_of<FMT>(top));
    const float inv = bad ? 0.0f : 1.0f / sc;
    if (threadIdx.x == 0) *scales[side] = sc;
    const float again = s_old[side] * inv;
    uint8_t* dst = (side ? pg.v : pg.k) + hp * P * kHeadDim;
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
        const uint32_t ww[4] = {w[side][j].x, w[side][j].y, w[side][j].z, w[side][j].w};
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
}

// ----------------------------------------------------------------------------
// Attention.  The rows of a (sequence, KV head) are its new tokens times the
// G query heads of the group; 16 of them (or 32, RT = 2) are an item.  A wave takes
// an item's keys 32 at a time.  Per step and 16 rows
//   S^T = K Q^T        2 x 4  MFMA 16x16x32 (keys on M, rows on N)
//   O^T += V^T P^T     2 x 8  MFMA 16x16x32 (dims on M)
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
// Codes become bf16 exactly (int8 has 7 bits and a sign, e4m3 4); the scale of
// K multiplies the fp32 scores, V's the fp32 probabilities, which go to the
// matrix cores as the sum of two bf16 numbers (16 bits).
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
// An item (16 RT rows of a sequence and KV head) whose keys several waves
// share, left for combine_kernel by the one with its first key.  Its parts in
// the order of the keys: at first_slot and at 2 (worker + 1) ..: n_waves of
// them (waves of the first workgroup); n_groups at 2 kWaves group ..
// (workgroups after it); the rest at 2 last .. (waves of the last one).
// parts = 0: none.
struct SplitItem {
  int s, kvh, row0, parts, first_slot, n_waves, group, n_groups, last, pad[3];
};

struct AttendArgs {
  const uint16_t* q;
  uint16_t* o;
  Tokens tk;
  const int32_t* lengths;
  Pages pg;
  int Hq;
  float sc_log2;
  Part* part_ml;
  float* part_o;
  SplitItem* split;
};

// What a wave has of its 16 RT rows: lane l holds row j = l % 16 of each tile,
// the dims 8 (4g + r) + i of oacc[.][i][r], and its own keys' part of l.
template <int RT>
struct WaveSums {
  float m[RT], l[RT];
  f32x4 o[RT][8];
};

// The rows row0 .. row0 + 16 RT - 1 of sequence s (n tokens from packed row
// `first` on, seq_len of them in the cache) over every `stride`-th step of 32
// keys from the w-th on, of the keys key0 .. key1 - 1.
template <int FMT, int P, int RT>
__device__ __forceinline__ void attend_steps(const AttendArgs& a, int s, int kvh, int row0,
                                             int first, int n, int seq_len, int key0, int key1,
                                             int w, int stride, WaveSums<RT>& ws) {
  const int G = a.Hq / a.pg.Hkv, rows = n * G;
  const int lane = threadIdx.x % kWave;
  const int j = lane & 15, g = lane >> 4;

  bf16x8 qf[RT][4];
  // this lane's rows: the last key each sees, -1 for none (rows past the last repeat it)
  int pos[RT];
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) {
    const int row = min(row0 + kRows * rt + j, rows - 1);
    pos[rt] = max(max(seq_len, 0) - n + row / G, -1);
    const uint16_t* qp =
        a.q + ((int64_t)(kvh * G + row % G) * a.tk.T + first + row / G) * kHeadDim + 16 * g;
#pragma unroll
    for (int c = 0; c < 4; ++c)   // dims 64 (c / 2) + 16 g + 8 (c % 2) ..
      qf[rt][c] = __builtin_bit_cast(bf16x8, *(const uint4*)(qp + 64 * (c >> 1) + 8 * (c & 1)));
  }
  const int pos_min = max(seq_len, 0) - n + row0 / G;

#pragma unroll
  for (int rt = 0; rt < RT; ++rt) {
    ws.m[rt] = -INFINITY;
    ws.l[rt] = 0.0f;
#pragma unroll
    for (int i = 0; i < 8; ++i) ws.o[rt][i] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
  }

  const uint32_t koff = (uint32_t)(j * kHeadDim + 16 * g), voff = (uint32_t)(4 * g * kHeadDim + 8 * j);
  // A step's operands.  The next step's are asked for as soon as this one's have
  // been read out of their registers, so K is on its way during the softmax and
  // the second product, V during the next step's first.  (Deeper pipelines, of
  // up to four steps a wave, were slower wherever all CUs work: 8 sequences of
  // up to 128k tokens 251 us, with a second step in flight 256, with two 259.)
  uint4 kw[2][2];
  uint2 vw[2][4];
  // The loads go through buffer descriptors of the step's rows, of no length
  // where there is no step to load for (such a load fetches nothing): loads
  // behind a branch the compiler would wait for at once.
  constexpr int kOnce = 2;   // nontemporal
  auto rows_of = [&](uint8_t* base, int page, int k0, bool real) {
    const int64_t at = real ? (((int64_t)page * a.pg.Hkv + kvh) * P + k0 % P) * kHeadDim : 0;
    return __builtin_amdgcn_make_buffer_rsrc(base + at, 0, real ? kKeys * kHeadDim : 0, 0x00027000);
  };
  auto load_k = [&](int page, int k0, bool real) {
    const auto rsrc = rows_of(a.pg.k, page, k0, real);
#pragma unroll
    for (int u = 0; u < 2; ++u)
#pragma unroll
      for (int c = 0; c < 2; ++c)
        kw[u][c] = __builtin_bit_cast(uint4, __builtin_amdgcn_raw_buffer_load_b128(
            rsrc, (int)koff + 16 * u * kHeadDim + 64 * c, 0, kOnce));
  };
  auto load_v = [&](int page, int k0, bool real) {
    const auto rsrc = rows_of(a.pg.v, page, k0, real);
#pragma unroll
    for (int u = 0; u < 2; ++u)
#pragma unroll
      for (int r = 0; r < 4; ++r)
        vw[u][r] = __builtin_bit_cast(uint2, __builtin_amdgcn_raw_buffer_load_b64(
            rsrc, (int)voff + (16 * u + r) * kHeadDim, 0, kOnce));
  };

  // `k_read` and `v_read` run once K and V have been read out.
  auto compute = [&](int k0, float kf, float vf, auto k_read, auto v_read) {
    f32x4 sacc[RT][2];
#pragma unroll
    for (int u = 0; u < 2; ++u) {
#pragma unroll
      for (int rt = 0; rt < RT; ++rt) sacc[rt][u] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
      for (int c = 0; c < 2; ++c) {
        const bf16x8 k_lo = widen8<FMT>(kw[u][c].x, kw[u][c].y);
        const bf16x8 k_hi = widen8<FMT>(kw[u][c].z, kw[u][c].w);
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) {
          sacc[rt][u] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k_lo, qf[rt][2 * c], sacc[rt][u], 0, 0, 0);
          sacc[rt][u] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k_hi, qf[rt][2 * c + 1], sacc[rt][u], 0, 0, 0);
        }
      }
    }
    k_read();
    // steps that reach past a row's last key (the others see every key); the
    // asm statements keep the compiler from doing their work in every step
    const bool edge = k0 + kKeys - 1 > pos_min || k0 + kKeys > key1;
    if (k0 + kKeys > key1) {
      int left = key1 - k0 - 4 * g;
      asm volatile("" : "+v"(left));
      // rows behind the sequence's end hold anything, NaN codes included
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if (16 * (e >> 2) + (e & 3) >= left) vw[e >> 2][e & 3] = make_uint2(0u, 0u);
    }
    // the probabilities times V's scale as the sum of two bf16 numbers: one
    // alone would double the variance that the output's rounding has, and the
    // matrix cores have the time
    bf16x8 p_hi[RT], p_lo[RT];
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
      const int lim = min(pos[rt], key1 - 1) - k0 - 4 * g;
      auto place = [](int e) { return 16 * (e >> 2) + (e & 3); };
      auto hide = [&](float (&x)[8]) {
        int most = lim;
        asm volatile("" : "+v"(most));
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = place(e) <= most ? x[e] : 0.0f;
      };
      auto score = [&](int e) { return sacc[rt][e >> 2][e & 3]; };
      float p[8], lsum;
      auto probs = [&](float mneg) {
#pragma unroll
        for (int e = 0; e < 8; ++e) p[e] = __builtin_amdgcn_exp2f(fmaf(score(e), kf, mneg));
        if (edge) hide(p);
        lsum = ((p[0] + p[1]) + (p[2] + p[3])) + ((p[4] + p[5]) + (p[6] + p[7]));
      };
      bool kept = false;
      if (__builtin_amdgcn_ballot_w64(ws.m[rt] == -INFINITY) == 0) {
        probs(-ws.m[rt]);
        kept = __builtin_amdgcn_ballot_w64(!(lsum <= kFastLimit)) == 0;
      }
      if (!kept) {
        float mx = -INFINITY;
#pragma unroll
        for (int e = 0; e < 8; ++e) mx = fmaxf(mx, place(e) <= lim ? score(e) * kf : -INFINITY);
        mx = fmaxf(mx, __shfl_xor(mx, 16));
        mx = fmaxf(mx, __shfl_xor(mx, 32));
        if (__builtin_amdgcn_ballot_w64(mx > ws.m[rt] + kRescaleThreshold) != 0) {
          const float m_new = fmaxf(ws.m[rt], mx);
          const float alpha = m_new == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f(ws.m[rt] - m_new);
          ws.l[rt] *= alpha;
#pragma unroll
          for (int i = 0; i < 8; ++i) ws.o[rt][i] *= alpha;
          ws.m[rt] = m_new;
        }
        probs(ws.m[rt] == -INFINITY ? 0.0f : -ws.m[rt]);
      }
      ws.l[rt] += lsum;
#pragma unroll
      for (int e = 0; e < 8; ++e) p[e] *= vf;
      if (edge) hide(p);   // (a masked probability is 0, but V's scale may be NaN)
      uint32_t hi[4], lo[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        hi[e] = pack_bf16x2(p[2 * e], p[2 * e + 1]);
        lo[e] = pack_bf16x2(p[2 * e] - bf16_lo(hi[e]), p[2 * e + 1] - bf16_hi(hi[e]));
      }
      p_hi[rt] = __builtin_bit_cast(bf16x8, make_uint4(hi[0], hi[1], hi[2], hi[3]));
      p_lo[rt] = __builtin_bit_cast(bf16x8, make_uint4(lo[0], lo[1], lo[2], lo[3]));
    }
    // byte i of keys (0, 1), (2, 3) of each half, next to each other
#pragma unroll
    for (int half = 0; half < 2; ++half) {     // dims 8j + 4 half ..
      uint32_t pr[2][2][2];                    // [u][key pair][dims 0-1, 2-3]
#pragma unroll
      for (int u = 0; u < 2; ++u)
#pragma unroll
        for (int c = 0; c < 2; ++c) {
          const uint32_t x = half ? vw[u][2 * c].y : vw[u][2 * c].x;
          const uint32_t y = half ? vw[u][2 * c + 1].y : vw[u][2 * c + 1].x;
          pr[u][c][0] = __builtin_amdgcn_perm(y, x, 0x05010400u);
          pr[u][c][1] = __builtin_amdgcn_perm(y, x, 0x07030602u);
        }
#pragma unroll
      for (int i2 = 0; i2 < 2; ++i2) {
        const bf16x8 v0 = __builtin_bit_cast(
            bf16x8, make_uint4(widen2<FMT, false>(pr[0][0][i2]), widen2<FMT, false>(pr[0][1][i2]),
                               widen2<FMT, false>(pr[1][0][i2]), widen2<FMT, false>(pr[1][1][i2])));
        const bf16x8 v1 = __builtin_bit_cast(
            bf16x8, make_uint4(widen2<FMT, true>(pr[0][0][i2]), widen2<FMT, true>(pr[0][1][i2]),
                               widen2<FMT, true>(pr[1][0][i2]), widen2<FMT, true>(pr[1][1][i2])));
        const int i = 4 * half + 2 * i2;
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) {
          ws.o[rt][i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v0, p_hi[rt], ws.o[rt][i], 0, 0, 0);
          ws.o[rt][i + 1] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v1, p_hi[rt], ws.o[rt][i + 1], 0, 0, 0);
          ws.o[rt][i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v0, p_lo[rt], ws.o[rt][i], 0, 0, 0);
          ws.o[rt][i + 1] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v1, p_lo[rt], ws.o[rt][i + 1], 0, 0, 0);
        }
      }
    }
    v_read();
  };

  // The wave's steps.  Pages are looked up two steps ahead, scales one.
  const int steps = (key1 - key0 + kKeys - 1) / kKeys;
  const int mine = (steps - w + stride - 1) / stride;
  if (mine > 0) {
    auto key_of = [&](int i) { return key0 + kKeys * (w + stride * min(i, mine - 1)); };
    // (the table has room for the keys: a step's column is one of it)
    const int64_t row = (int64_t)s * a.pg.max_pages;
    auto number_of = [&](int i) { return entry(a.pg.table, row + key_of(i) / P); };
    auto page_of = [&](int number) { return (unsigned)number < (unsigned)a.pg.n_pages ? number : -1; };
    // (where there is no page any scale will do, but a cache of none has no scales)
    const float* const some = (const float*)a.lengths;
    const float* const k_scales = a.pg.n_pages ? a.pg.ks : some;
    const float* const v_scales = a.pg.n_pages ? a.pg.vs : some;
    auto scale_at = [&](int page) { return page < 0 ? 0 : (int64_t)page * a.pg.Hkv + kvh; };
    int page = page_of(number_of(0)), number = number_of(1);
    float kf = entry(k_scales, scale_at(page)), vf = entry(v_scales, scale_at(page));
    load_k(page, key_of(0), page >= 0);
    load_v(page, key_of(0), page >= 0);
    for (int i = 0; i < mine; ++i) {
      // (scalar loads are waited for all together: here, for those of the step before)
      asm volatile("" : "+s"(number), "+s"(kf), "+s"(vf));
      const int next = page_of(number);
      number = number_of(i + 2);
      const float kf_next = entry(k_scales, scale_at(next)), vf_next = entry(v_scales, scale_at(next));
      const bool real = i + 1 < mine && next >= 0;
      // (keys on no page: zeros at places that no row sees)
      compute(page >= 0 ? key_of(i) : INT_MAX - 2 * kKeys, page >= 0 ? kf * a.sc_log2 : 0.0f,
              page >= 0 ? vf : 0.0f, [&]() { load_k(next, key_of(i + 1), real); },
              [&]() { load_v(next, key_of(i + 1), real); });
      page = next;
      kf = kf_next;
      vf = vf_next;
    }
  }
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) {
    ws.l[rt] += __shfl_xor(ws.l[rt], 16);
    ws.l[rt] += __shfl_xor(ws.l[rt], 32);
  }
}

// 8 dims of an output row.
__device__ __forceinline__ void store_dims(const AttendArgs& a, int kvh, int row, int first, int d,
                                           const float (&x)[8], float l) {
  const int G = a.Hq / a.pg.Hkv;
  const float inv = l == 0.0f ? 0.0f : 1.0f / l;
  *(uint4*)(a.o + ((int64_t)(kvh * G + row % G) * a.tk.T + first + row / G) * kHeadDim + d) =
      make_uint4(pack_bf16x2(x[0] * inv, x[1] * inv), pack_bf16x2(x[2] * inv, x[3] * inv),
                 pack_bf16x2(x[4] * inv, x[5] * inv), pack_bf16x2(x[6] * inv, x[7] * inv));
}

// Keys of sequence s that the table has room for.
template <int P>
__device__ __forceinline__ int keys_of(const AttendArgs& a, int s) {
  return (int)min((int64_t)max(entry(a.lengths, s), 0), (int64_t)a.pg.max_pages * P);
}

// The sums of a workgroup's waves over different keys of the same rows, joined
// in LDS; `out` gets row (in the item), dims d .. d + 7 of it, m, l and the sums.
template <int WAVES>
struct MergeSmem {
  static constexpr int kPitch = kHeadDim + 4;   // (a row's start moves on by 4 banks)
  float m[WAVES][kRows], l[WAVES][kRows];
  __attribute__((aligned(16))) float o[WAVES][kRows * kPitch];
};
template <int RT, int WAVES, class Out>
__device__ __forceinline__ void merge_waves(MergeSmem<WAVES>& sm, const WaveSums<RT>& ws, int rows,
                                            Out out) {
  constexpr int kPitch = MergeSmem<WAVES>::kPitch;
  const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave, j = lane & 15, g = lane >> 4;
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) {
    if (rt > 0) __syncthreads();   // (the rows before have been read)
    if (g == 0) {
      sm.m[wave][j] = ws.m[rt];
      sm.l[wave][j] = ws.l[rt];
    }
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      float* at = &sm.o[wave][j * kPitch + 8 * (4 * g + r)];
      *(float4*)at = make_float4(ws.o[rt][0][r], ws.o[rt][1][r], ws.o[rt][2][r], ws.o[rt][3][r]);
      *(float4*)(at + 4) = make_float4(ws.o[rt][4][r], ws.o[rt][5][r], ws.o[rt][6][r], ws.o[rt][7][r]);
    }
    __syncthreads();
    const int mr = threadIdx.x >> 4, md = (threadIdx.x & 15) * 8;   // row, dims
    if (mr < kRows && kRows * rt + mr < rows) {
      float m = sm.m[0][mr];
#pragma unroll
      for (int w = 1; w < WAVES; ++w) m = fmaxf(m, sm.m[w][mr]);
      float l = 0.0f, acc[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) acc[e] = 0.0f;
#pragma unroll
      for (int w = 0; w < WAVES; ++w) {
        const float f = sm.m[w][mr] == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(sm.m[w][mr] - m);
        l += f * sm.l[w][mr];
#pragma unroll
        for (int e = 0; e < 8; ++e) acc[e] += f * sm.o[w][mr * kPitch + md + e];
      }
      out(kRows * rt + mr, md, m, l, acc);
    }
  }
}

// 8 dims of a part's row.
template <int RT>
__device__ __forceinline__ void store_part(const AttendArgs& a, int slot, int row, int d, float m,
                                           float l, const float (&x)[8]) {
  const int64_t pr = (int64_t)slot * (kRows * RT) + row;
  if (d == 0) a.part_ml[pr] = Part{m, l};
  float* at = a.part_o + pr * kHeadDim + d;
  *(float4*)at = make_float4(x[0], x[1], x[2], x[3]);
  *(float4*)(at + 4) = make_float4(x[4], x[5], x[6], x[7]);
}

constexpr int attend_occupancy(int rt) { return rt == 1 ? 3 : 2; }   // waves a SIMD holds

// Short tables: a workgroup per item, its waves merged through LDS.
template <int FMT, int P, int RT, int WAVES>
__global__ __launch_bounds__(WAVES* kWave, attend_occupancy(RT)) void attend_kernel(AttendArgs a, int per_seq,
                                                                int64_t item0) {
  __shared__ MergeSmem<WAVES> sm;
  const int64_t item = item0 + blockIdx.x;
  const int G = a.Hq / a.pg.Hkv, kvh = (int)(item % a.pg.Hkv);
  int s, tile, first, n;
  find_slot(a.tk, (int)(item / a.pg.Hkv), per_seq, G, kRows * RT, 1, s, tile);
  seq_rows(a.tk, s, first, n);
  const int row0 = tile * kRows * RT, rows = n * G;
  if (tile < 0 || row0 >= rows) return;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  WaveSums<RT> ws;
  attend_steps<FMT, P, RT>(a, s, kvh, row0, first, n, entry(a.lengths, s), 0, keys_of<P>(a, s), wave,
                           WAVES, ws);
  merge_waves<RT>(sm, ws, rows - row0, [&](int r, int d, float, float l, const float (&x)[8]) {
    store_dims(a, kvh, row0 + r, first, d, x, l);
  });
}

// Long tables, whose sequences may be of any lengths: the items' steps dealt out
// over the waves of the launch.  With the items one behind the other (by
// sequence, KV head and row tile), each kItemCost steps longer than it is (what
// a wave waits for before an item's first step), every wave takes a run of
// them, all equally long (but see elder_share): a last part of an item, whole
// items, a first part of one.  Whole items are written out, parts left for
// combine_kernel: nothing in here waits for another wave, except where the runs
// of a workgroup's waves lie in one item: they then share the item's steps and
// leave one part.
//
// Each wave adds the sequences up for itself.  Two waves a SIMD are what HBM
// needs (with three, equal runs: 8 sequences of up to 128k tokens 245.6 -> 248.6 us,
// 200 of 1000 to 4000 150 -> 156).  A workgroup per item instead
// (as for short tables) is 3% faster on 128 sequences of about 2000 tokens, all
// alike (96 / 99 us), and far slower on others (256 of 200 to 8000: 243 / 203).
constexpr int kCus = 256;
constexpr int kShareGroups = 2 * kCus;
constexpr int kItemCost = 5;    // (7: 128 ragged sequences 78.5 -> 79.5 us, 64 of them the same)
constexpr int kShareLeast = 4;   // steps and costs a wave takes at least
// The first workgroup of a CU gets its loads before the second one's: with equal
// runs its waves end first, and what is left does not fill HBM.  Wave priorities
// change nothing.  So where every CU has two, the first half of the workgroups
// takes runs longer than the average by a sixth, with 32 rows, whose arithmetic
// goes to the first one's waves too, by a third (attention alone, equal / sixth /
// third: 6 sequences of 13000, 32 rows, int8 40.7 / 38.9 / 36.6 us, e4m3 40.0 / 38.4 /
// 36.4, 16 of 500 to 8000 33.6 / 32.9 / 30.9; 16 rows, equal / sixth: 40 of 300 to
// 6000 18.1 / 17.5; 8 of up to 128k 245.4 / 244.2; 256 of 200 to 8000 188.7 / 187.6; an
// eighth or a fifth within 1% of that; the loser: 16 of 4000 to 16000, two tiles of
// 32 rows each, a call 113.6 / - / 114.9), unless equal runs are whole items (as many
// sequences of one length as make it so: 256 of 4096 and 8 KV heads 322 / 341).
// That workgroups 0 .. 255 are the CUs' first is how the launch fills the chip, and
// only the balance rests on it.
constexpr int elder_share(int rt) { return rt == 1 ? 6 : 3; }

// A value that all lanes share, in scalar registers.
__device__ __forceinline__ int64_t uniform(int64_t x) {
  const uint32_t lo = __builtin_amdgcn_readfirstlane((uint32_t)x);
  const uint32_t hi = __builtin_amdgcn_readfirstlane((uint32_t)((uint64_t)x >> 32));
  return (int64_t)((uint64_t)hi << 32 | lo);
}

template <int FMT, int P, int RT>
__global__ __launch_bounds__(kThreads, attend_occupancy(RT)) void attend_share_kernel(AttendArgs a) {
  __shared__ MergeSmem<kWaves> sm;
  const int G = a.Hq / a.pg.Hkv, lane = threadIdx.x % kWave;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const int group = (int)blockIdx.x, worker = group * kWaves + wave;
  const int workers = (int)gridDim.x * kWaves;
  int steps = 0, tiles = 0;   // of the sequence that cost_of or look was last called for
  auto cost = [&]() { return (int64_t)(steps + kItemCost) * tiles * a.pg.Hkv; };
  auto cost_of = [&](int s) -> int64_t {
    int first, n;
    seq_rows(a.tk, s, first, n);
    steps = (keys_of<P>(a, s) + kKeys - 1) / kKeys;
    tiles = (n * G + kRows * RT - 1) / (kRows * RT);
    return cost();
  };
  // of 64 sequences: the costs up to each lane's
  auto up_to = [&](int64_t x) -> int64_t {
#pragma unroll
    for (int o = 1; o < kWave; o <<= 1) {
      const int64_t up = __shfl_up(x, o);
      if (lane >= o) x += up;
    }
    return x;
  };
  // the first 64 sequences stay in registers
  const int64_t my_cost = lane < a.tk.S ? cost_of(lane) : 0;
  const int my_steps = steps, my_tiles = tiles;
  const int64_t my_end = up_to(my_cost);
  int64_t total = uniform(__shfl(my_end, kWave - 1));
  if (a.tk.S > kWave) {
    int64_t rest = 0;
    for (int s = kWave + lane; s < a.tk.S; s += kWave) rest += cost_of(s);
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) rest += __shfl_xor(rest, o);
    total += uniform(rest);
  }
  auto look = [&](int s) {   // (s the same in all lanes)
    if (s < kWave) {
      steps = __builtin_amdgcn_readlane(my_steps, s);
      tiles = __builtin_amdgcn_readlane(my_tiles, s);
    } else {
      cost_of(s);
    }
  };
  if (lane == 0) a.split[worker].parts = 0;
  // the sequence that unit u < total lies in, and the unit it starts at
  int s;
  int64_t start;
  auto find = [&](int64_t u) {
    int64_t before = 0;
    for (s = 0; s < a.tk.S; s += kWave) {
      const int64_t own = s == 0 ? my_cost : s + lane < a.tk.S ? cost_of(s + lane) : 0;
      const int64_t incl = s == 0 ? my_end : up_to(own);
      const uint64_t past = __builtin_amdgcn_ballot_w64(before + incl > u);
      if (past != 0) {
        const int at = (int)__builtin_ctzll(past);
        start = uniform(__shfl(before + incl - own, at));
        s = __builtin_amdgcn_readfirstlane(s + at);
        return;
      }
      before += uniform(__shfl(incl, kWave - 1));
    }
  };
  // worker w's run: bound(w) .. bound(w + 1) - 1 (less what lies past the total)
  const int64_t even = (total + workers - 1) / workers;
  const int whole0 = __builtin_amdgcn_readlane(my_steps, 0) + kItemCost;
  const bool whole_items = total == even * workers && even % whole0 == 0;
  const int elders = workers == kShareGroups * kWaves && even > kShareLeast && !whole_items
                         ? workers / 2 : 0;
  const int64_t elder = even + even / elder_share(RT);
  const int64_t per = elders ? (total - elders * elder + elders - 1) / elders
                             : even < kShareLeast ? kShareLeast : even;
  auto bound = [&](int w) -> int64_t {
    return min(w, elders) * elder + max(w - elders, 0) * per;
  };
  auto owner = [&](int64_t u) -> int {
    const int64_t rest = u - elders * elder;
    return rest < 0 ? (int)(u / elder) : elders + (int)(rest / per);
  };
  const int64_t g0 = bound(group * kWaves), g1 = min(bound((group + 1) * kWaves), total);
  if (g0 >= g1) return;
  // The units u .. end - 1 of the item that unit u lies in (after look(s)).
  struct Run {
    int item, st0, st1;     // of the sequence; its steps
    int64_t base, next;     // the item's first unit, the one behind it
    bool none, full;
  };
  auto run_at = [&](int64_t u, int64_t end) -> Run {
    const int whole = steps + kItemCost;
    const int off = (int)(u - start), at = off % whole;
    const int to = (int)min((int64_t)whole, at + (end - u));
    Run r;
    r.item = off / whole;
    r.st0 = max(at - kItemCost, 0);
    r.st1 = max(to - kItemCost, 0);
    r.base = u - at;
    r.next = r.base + whole;
    // without steps it is none (an item without keys counts with its last unit)
    r.none = steps == 0 ? to < whole : r.st0 == r.st1;
    r.full = r.st0 == 0 && r.st1 == steps;
    return r;
  };
  // Leaves the list of an item's parts, the first of which is at `slot`, left
  // by wave w0 or, with `joint`, by this workgroup's waves together.
  auto leave_item = [&](const Run& r, int kvh, int row0, int slot, int w0, bool joint) {
    const int last = owner(r.next - 1), last_group = last / kWaves;
    const int64_t last_end = min(bound((last_group + 1) * kWaves), total);
    SplitItem it{};
    it.s = s;
    it.kvh = kvh;
    it.row0 = row0;
    it.first_slot = slot;
    it.group = group + 1;
    it.n_waves = joint ? 1 : min((group + 1) * kWaves - 1, last) - w0 + 1;
    it.last = last_group * kWaves;
    int n_last = 0;
    if (last_group > group) {
      const bool joint_last = last_end <= r.next;
      it.n_groups = last_group - group - 1 + (joint_last ? 1 : 0);
      n_last = joint_last ? 0 : last - it.last + 1;
    }
    it.parts = it.n_waves + it.n_groups + n_last;
    a.split[w0] = it;
  };

  find(g0);
  if (s >= a.tk.S) return;
  look(s);
  // whether the workgroup's waves go together, their runs being of one item
  const bool joint = g1 <= run_at(g0, g1).next;
  const int64_t u0 = joint ? g0 : bound(worker), u1 = joint ? g1 : min(bound(worker + 1), total);
  if (u0 >= u1) return;
  if (!joint && wave > 0) {
    find(u0);
    if (s >= a.tk.S) return;
    look(s);
  }
  for (int64_t u = u0; u < u1 && s < a.tk.S;) {
    if (u >= start + cost()) {   // (also past sequences without new tokens: they cost nothing)
      start += cost();
      if (++s < a.tk.S) cost_of(s);
      continue;
    }
    const Run r = run_at(u, u1);
    const int first_worker = joint ? group * kWaves : worker;
    const int slot = 2 * first_worker + (u == u0 ? 0 : 1);
    u = r.next;
    if (r.none) continue;
    int first, n;
    seq_rows(a.tk, s, first, n);
    const int kvh = r.item / tiles, row0 = r.item % tiles * kRows * RT;
    if (!r.full && r.st0 == 0 && lane == 0 && (!joint || wave == 0))
      leave_item(r, kvh, row0, slot, first_worker, joint);
    WaveSums<RT> ws;
    attend_steps<FMT, P, RT>(a, s, kvh, row0, first, n, entry(a.lengths, s), r.st0 * kKeys,
                             min(r.st1 * kKeys, keys_of<P>(a, s)), joint ? wave : 0,
                             joint ? kWaves : 1, ws);
    auto store = [&](int row, int d, float m, float l, const float (&x)[8]) {
      if (r.full) store_dims(a, kvh, row0 + row, first, d, x, l);
      else store_part<RT>(a, slot, row, d, m, l, x);
    };
    if (joint) {
      merge_waves<RT>(sm, ws, n * G - row0, store);
    } else {
      const int j = lane & 15, g = lane >> 4;
#pragma unroll
      for (int rt = 0; rt < RT; ++rt) {
        const int row = kRows * rt + j;
        if (row0 + row >= n * G) continue;
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          float x[8];
#pragma unroll
          for (int i = 0; i < 8; ++i) x[i] = ws.o[rt][i][q];
          store(row, 8 * (4 * g + q), ws.m[rt], ws.l[rt], x);
        }
      }
    }
  }
}

// The parts of a shared item joined, in the order of their keys.  A workgroup
// looks after 8 rows of the items that `per` workers left, up to four items at
// once: a group of 16 lanes adds up a row's 128 dims over every stripes-th part,
// then the stripes are added up in order.
constexpr int kCombineThreads = 512;
constexpr int kCombineLanes = 16;
constexpr int kCombineRows = 8;
constexpr int kCombineItems = 4;
// Workers a workgroup looks after, at most.  A workgroup that finds no item costs
// its dispatch (8 waves), one that finds several shares its groups among them: so
// kWaves, and twice as many while four in five then find one (4 / 8 / 16 / 32
// workers, us: 48 items of 32 rows 7.1 / 7.4 / 6.1 / 5.4, 128 of them 7.2 / 6.8 / 7.6,
// 256 items of 4 rows 4.7 / 5.4).
constexpr int kCombineWorkers = 32;
static_assert(kCombineWorkers <= kWave, "a lane reads what each of them left");
constexpr int kCombineAhead = 4;   // parts in flight per group (2 / 4 / 8: 40 sequences 6.1 / 5.1 us,
                                   // 64 4.7 / 4.7 / 5.5)
static_assert(kCombineThreads / kCombineLanes / kCombineItems >= kCombineRows,
              "a group for each row of an item");
__global__ __launch_bounds__(kCombineThreads) void combine_kernel(AttendArgs a, int tile_rows,
                                                                  int workers, int per) {
  constexpr int kGroupBits = 5, kGroups = 1 << kGroupBits;
  static_assert(kGroups == kCombineThreads / kCombineLanes, "groups of 16 lanes");
  constexpr int kHalves = kHeadDim / (4 * kCombineLanes);   // four dims of each a lane
  __shared__ float sm_m[kGroups], sm_l[kGroups];
  __shared__ __attribute__((aligned(16))) float sm_o[kGroups][kHeadDim];
  const int G = a.Hq / a.pg.Hkv, lane = threadIdx.x % kWave;
  const int grp = threadIdx.x / kCombineLanes, d = (threadIdx.x % kCombineLanes) * 4;
  const int worker0 = (int)blockIdx.x * per;
  SplitItem left{};   // of worker worker0 + lane
  if (lane < per && worker0 + lane < workers) left = a.split[worker0 + lane];
  uint64_t todo = __builtin_amdgcn_ballot_w64(left.parts > 0);
  const int items = __builtin_popcountll(todo);
  if (items == 0) return;
  // items at once: 1, 2 or 4, each with an equal share of the groups
  const int many = items < 3 ? items - 1 : 2, mine = kGroups >> many;
  const int ahead = __builtin_amdgcn_readfirstlane(grp >> (kGroupBits - many));
  const int at = grp & (mine - 1), r0 = (int)blockIdx.y * kCombineRows;
  for (int p = 0; p < items; p += 1 << many) {
    uint64_t mask = todo;
    for (int i = 0; i < 1 << many; ++i) {
      if (i < ahead) mask &= mask - 1;
      todo &= todo - 1;
    }
    const int w = mask ? (int)__builtin_ctzll(mask) : 0;
    auto of = [&](int x) { return __builtin_amdgcn_readlane(x, w); };
    const int parts = mask ? of(left.parts) : 0, s = of(left.s), kvh = of(left.kvh);
    const int row0 = of(left.row0), first_slot = of(left.first_slot), n_waves = of(left.n_waves);
    const int group = of(left.group), n_groups = of(left.n_groups), last = of(left.last);
    int first = 0, n = 0;
    if (parts > 0) seq_rows(a.tk, s, first, n);   // (else nothing of it is set)
    const int rows = parts > 0 ? min(min(n * G - row0, tile_rows) - r0, kCombineRows) : 0;
    auto slot_row = [&](int p, int r) -> int64_t {
      int slot = first_slot;
      if (p >= n_waves + n_groups) slot = 2 * (last + p - n_waves - n_groups);
      else if (p >= n_waves) slot = 2 * kWaves * (group + p - n_waves);
      else if (p > 0) slot = 2 * (worker0 + w + p);
      return (int64_t)slot * tile_rows + r0 + r;
    };
    // rows by the power of two above them, the rest of the groups in stripes
    const int bits = rows > 4 ? 3 : rows > 2 ? 2 : rows > 1 ? 1 : 0, lanes_r = 1 << bits;
    const int stripes = mine >> bits, stripe = at >> bits, r = at & (lanes_r - 1);
    float m = -INFINITY, l = 0.0f;
    float4 acc[kHalves];
#pragma unroll
    for (int h = 0; h < kHalves; ++h) acc[h] = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
    auto add = [&](float4 (&sum)[kHalves], float f, const float4 (&x)[kHalves], float g) {
#pragma unroll
      for (int h = 0; h < kHalves; ++h) {
        sum[h].x = sum[h].x * f + x[h].x * g;
        sum[h].y = sum[h].y * f + x[h].y * g;
        sum[h].z = sum[h].z * f + x[h].z * g;
        sum[h].w = sum[h].w * f + x[h].w * g;
      }
    };
    if (r < rows)
      for (int p0 = stripe; p0 < parts; p0 += stripes * kCombineAhead) {
        Part ml[kCombineAhead];
        float4 x[kCombineAhead][kHalves];
#pragma unroll
        for (int k = 0; k < kCombineAhead; ++k) {
          const int64_t pr = slot_row(min(p0 + k * stripes, parts - 1), r);
          ml[k] = a.part_ml[pr];
#pragma unroll
          for (int h = 0; h < kHalves; ++h)
            x[k][h] = *(const float4*)(a.part_o + pr * kHeadDim + 4 * kCombineLanes * h + d);
        }
#pragma unroll
        for (int k = 0; k < kCombineAhead; ++k) {
          if (p0 + k * stripes >= parts) break;
          const float mn = fmaxf(m, ml[k].m);
          const float f = m == mn ? 1.0f : __builtin_amdgcn_exp2f(m - mn);
          const float g = ml[k].m == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(ml[k].m - mn);
          l = l * f + ml[k].l * g;
          add(acc, f, x[k], g);
          m = mn;
        }
      }
    if (p > 0) __syncthreads();   // (the sums before have been read)
    if (d == 0) {
      sm_m[grp] = m;
      sm_l[grp] = l;
    }
#pragma unroll
    for (int h = 0; h < kHalves; ++h) *(float4*)&sm_o[grp][4 * kCombineLanes * h + d] = acc[h];
    __syncthreads();
    if (stripe != 0 || r >= rows) continue;
    for (int k = 1; k < stripes; ++k) m = fmaxf(m, sm_m[grp + k * lanes_r]);
    l = 0.0f;
#pragma unroll
    for (int h = 0; h < kHalves; ++h) acc[h] = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
    for (int k = 0; k < stripes; ++k) {
      const int from = grp + k * lanes_r;
      const float g = sm_m[from] == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(sm_m[from] - m);
      float4 x[kHalves];
#pragma unroll
      for (int h = 0; h < kHalves; ++h) x[h] = *(const float4*)&sm_o[from][4 * kCombineLanes * h + d];
      l += sm_l[from] * g;
      add(acc, 1.0f, x, g);
    }
    const float inv = l == 0.0f ? 0.0f : 1.0f / l;
    const int row = row0 + r0 + r;
    uint16_t* at_row = a.o + ((int64_t)(kvh * G + row % G) * a.tk.T + first + row / G) * kHeadDim + d;
#pragma unroll
    for (int h = 0; h < kHalves; ++h)
      *(uint2*)(at_row + 4 * kCombineLanes * h) =
          make_uint2(pack_bf16x2(acc[h].x * inv, acc[h].y * inv),
                     pack_bf16x2(acc[h].z * inv, acc[h].w * inv));
  }
}

// ----------------------------------------------------------------------------
// Copy.  One workgroup moves 4 KB of K or of V of a page of a layer,
// past the caches (150 pages of 32 layers, 2.5 GB read and written: 4 KB each 432
// us, 8 KB 460, 16 KB 482; 8 KB with ordinary stores 484).
// ----------------------------------------------------------------------------
constexpr int kCopyBytes = 4 * 1024;

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
    if (c < chunks) w[j] = load_once4(from + c);
  }
#pragma unroll
  for (int j = 0; j < kCopyBytes / 16 / kThreads; ++j) {
    const int64_t c = c0 + threadIdx.x + j * kThreads;
    if (c < chunks) store_once4(to + c, w[j]);
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
ei_status check_pages(const ei_cache_shape& c, const ei_cache_pages& p) {
  if (c.n_pages == 0) return EI_OK;   // nothing to point at
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

// A table of no more keys: one workgroup per item.  (It reads about 50 KB per us,
// whatever its waves; dealt out, with the second kernel: 1 sequence of 1500 tokens
// 13.7 / 10 + 4 us, 32 of 1900 21.8 / 26 + 5, 100 of up to 1900 49.5 / 41 + 5; tables
// of 3900 here / dealt out: 1 28 / 10 + 4, 32 41 / 45 + 5, 100 of up to 3900 96 / 72 + 6.
// The width alone decides, and is off by up to a fifth on either side of it: 100 of
// up to 1900 lose 3 us by it, 32 of 3900 nine.)
constexpr int kShortKeys = 2048;
constexpr int kShortWaves = 4;     // (8 / 16: 1 of 1000 9.2 -> 9.2 / 10.8 us, 200 51 -> 59 / 72)

struct AttendPlan {
  int rt, per_seq, item_rows;   // item_rows: of an item, at most
  int groups;                   // workgroups of the shared launch, 0: one per item
  int64_t items;
  size_t ml_bytes, split_bytes, bytes;
  bool fits;
};
AttendPlan attend_plan(int Hq, int n_tokens, bool ragged, int n_seqs, int max_pages,
                       const ei_cache_shape& c) {
  const int64_t G = Hq / c.n_kv_heads;
  AttendPlan p{};
  // rows of a tile: 16, or 32 where a sequence has more than 16 (on average)
  p.rt = (int64_t)n_tokens * G > (int64_t)kRows * n_seqs ? 2 : 1;
  const int tile = p.item_rows = kRows * p.rt;
  int64_t slots, tiles;   // row tiles of all sequences, of one
  if (ragged) {
    slots = (int64_t)n_tokens * G / tile + n_seqs;
    tiles = (int64_t)n_tokens * G / tile + 1;
  } else {
    tiles = (n_tokens / n_seqs * G + tile - 1) / tile;
    p.per_seq = (int)tiles;
    if (n_tokens / n_seqs * G < tile) p.item_rows = (int)(n_tokens / n_seqs * G);
    slots = n_seqs * tiles;
  }
  p.items = slots * c.n_kv_heads;
  const int64_t keys = (int64_t)max_pages * c.page_len;
  const int64_t cost = keys / kKeys + kItemCost;   // of an item, at most
  p.fits = p.items <= INT_MAX && cost <= INT_MAX / (tiles * c.n_kv_heads);
  if (keys > kShortKeys && p.fits) {
    const int64_t waves = (p.items * cost + kShareLeast - 1) / kShareLeast;
    const int64_t most = (waves + kWaves - 1) / kWaves;
    p.groups = (int)(most < kShareGroups ? most : kShareGroups);
    const size_t workers = (size_t)p.groups * kWaves, rows = workers * 2 * tile;
    p.split_bytes = (workers * sizeof(SplitItem) + 255) / 256 * 256;
    p.ml_bytes = (rows * sizeof(Part) + 255) / 256 * 256;
    p.bytes = p.split_bytes + p.ml_bytes + rows * kHeadDim * sizeof(float);
  }
  return p;
}

template <int FMT, int P, int RT>
void launch_attend_t(const AttendPlan& pl, const AttendArgs& a, hipStream_t stream) {
  if (pl.groups) {
    hipLaunchKernelGGL((attend_share_kernel<FMT, P, RT>), dim3((unsigned)pl.groups),
                       dim3(kThreads), 0, stream, a);
    const unsigned row_blocks = (unsigned)((pl.item_rows + kCombineRows - 1) / kCombineRows);
    const int workers = pl.groups * kWaves;
    int per = kWaves;
    while (per < kCombineWorkers && pl.items * (5 * per) <= 2 * workers) per *= 2;
    hipLaunchKernelGGL(combine_kernel, dim3((unsigned)((workers + per - 1) / per), row_blocks),
                       dim3(kCombineThreads), 0, stream, a, kRows * RT, workers, per);
    return;
  }
  constexpr int64_t kMost = (1ll << 31) / (kShortWaves * kWave);
  for (int64_t i = 0; i < pl.items; i += kMost)
    hipLaunchKernelGGL((attend_kernel<FMT, P, RT, kShortWaves>),
                       dim3((unsigned)(pl.items - i < kMost ? pl.items - i : kMost)),
                       dim3(kShortWaves * kWave), 0, stream, a, pl.per_seq, i);
}
template <int FMT, int P>
void launch_attend(const AttendPlan& pl, const AttendArgs& a, hipStream_t stream) {
  if (pl.rt == 1) launch_attend_t<FMT, P, 1>(pl, a, stream);
  else launch_attend_t<FMT, P, 2>(pl, a, stream);
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
  if ((st = ei::check_pages(shape, pages)) != EI_OK) return st;
  if (!ei::aligned(k, 16) || !ei::aligned(v, 16) || !ei::aligned(lengths, 4) ||
      !ei::aligned(page_table, 4) || !ei::aligned(cu_seqlens, 4))
    return EI_ERR_UNSUPPORTED;
  const ei::Tokens tk{cu_seqlens, n_tokens, n_seqs, (int)each};
  const ei::Pages pg = ei::pages_of(shape, pages, page_table, max_pages);
  const int64_t units = slots * shape.n_kv_heads;
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
  if ((int64_t)n_tokens * n_q_heads > INT_MAX || (int64_t)max_pages * shape.page_len > INT_MAX)
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
  if (!pl.fits) return EI_ERR_SHAPE;
  if (!q || !o || !lengths || (!page_table && max_pages > 0)) return EI_ERR_NULL;
  if ((st = ei::check_pages(shape, pages)) != EI_OK) return st;
  if (!ei::aligned(q, 16) || !ei::aligned(o, 16) || !ei::aligned(lengths, 4) ||
      !ei::aligned(page_table, 4) || !ei::aligned(cu_seqlens, 4))
    return EI_ERR_UNSUPPORTED;
  if (pl.bytes && (!workspace || workspace_bytes < pl.bytes)) return EI_ERR_WORKSPACE;
  if (!ei::aligned(workspace, 16)) return EI_ERR_UNSUPPORTED;
  const ei::Tokens tk{cu_seqlens, n_tokens, n_seqs, n_tokens / n_seqs};
  const ei::Pages pg = ei::pages_of(shape, pages, page_table, max_pages);
  char* ws = (char*)workspace;
  const ei::AttendArgs a{q, o, tk, lengths, pg, n_q_heads,
                         (float)((double)softmax_scale * 1.4426950408889634),
                         (ei::Part*)(ws + pl.split_bytes),
                         (float*)(ws + pl.split_bytes + pl.ml_bytes), (ei::SplitItem*)ws};
  hipStream_t s0 = (hipStream_t)stream;
  if (shape.format == EI_CACHE_E4M3) {
    if (shape.page_len == 64) ei::launch_attend<EI_CACHE_E4M3, 64>(pl, a, s0);
    else ei::launch_attend<EI_CACHE_E4M3, 128>(pl, a, s0);
  } else {
    if (shape.page_len == 64) ei::launch_attend<EI_CACHE_INT8, 64>(pl, a, s0);
    else ei::launch_attend<EI_CACHE_INT8, 128>(pl, a, s0);
  }
  return ei::from_hip(hipGetLastError());
}

ei_status ei_cache_copy(ei_cache_shape shape, int32_t n_layers, ei_cache_pages pages,
                        const int32_t* src, const int32_t* dst, int32_t n, void* stream) {
  ei_status st = ei::check_shape(shape);
  if (st != EI_OK) return st;
  if (n_layers < 0 || n < 0) return EI_ERR_SHAPE;
  if (n_layers == 0 || n == 0 || shape.n_pages == 0) return EI_OK;
  if (!src || !dst) return EI_ERR_NULL;
  if ((st = ei::check_pages(shape, pages)) != EI_OK) return st;
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
