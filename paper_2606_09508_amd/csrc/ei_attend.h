// What the kernels that read the paged 8-bit cache share: where tokens and pages
// lie, the attention of 16 or 32 rows over steps of 32 keys, the join of its
// sums, and the host's checks.
#pragma once

#include "../../include/entropyinfer.h"
#include "ei_internal.h"

#include <limits.h>
#include <math.h>

namespace ei {
namespace {

constexpr int kAttendThreads = 256;
constexpr int kAttendWaves = kAttendThreads / kWave;

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
constexpr int kAttendRows = 16;
constexpr int kAttendKeys = 32;
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
// them (waves of the first workgroup); n_groups at 2 kAttendWaves group ..
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
    const int row = min(row0 + kAttendRows * rt + j, rows - 1);
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
    return __builtin_amdgcn_make_buffer_rsrc(base + at, 0, real ? kAttendKeys * kHeadDim : 0, 0x00027000);
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
    const bool edge = k0 + kAttendKeys - 1 > pos_min || k0 + kAttendKeys > key1;
    if (k0 + kAttendKeys > key1) {
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
  const int steps = (key1 - key0 + kAttendKeys - 1) / kAttendKeys;
  const int mine = (steps - w + stride - 1) / stride;
  if (mine > 0) {
    auto key_of = [&](int i) { return key0 + kAttendKeys * (w + stride * min(i, mine - 1)); };
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
      compute(page >= 0 ? key_of(i) : INT_MAX - 2 * kAttendKeys, page >= 0 ? kf * a.sc_log2 : 0.0f,
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
  float m[WAVES][kAttendRows], l[WAVES][kAttendRows];
  __attribute__((aligned(16))) float o[WAVES][kAttendRows * kPitch];
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
    if (mr < kAttendRows && kAttendRows * rt + mr < rows) {
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
      out(kAttendRows * rt + mr, md, m, l, acc);
    }
  }
}

// 8 dims of a part's row.
template <int RT>
__device__ __forceinline__ void store_part(const AttendArgs& a, int slot, int row, int d, float m,
                                           float l, const float (&x)[8]) {
  const int64_t pr = (int64_t)slot * (kAttendRows * RT) + row;
  if (d == 0) a.part_ml[pr] = Part{m, l};
  float* at = a.part_o + pr * kHeadDim + d;
  *(float4*)at = make_float4(x[0], x[1], x[2], x[3]);
  *(float4*)(at + 4) = make_float4(x[4], x[5], x[6], x[7]);
}

constexpr int attend_occupancy(int rt) { return rt == 1 ? 3 : 2; }   // waves a SIMD holds

// ----------------------------------------------------------------------------
// Host side
// ----------------------------------------------------------------------------
constexpr int64_t kMaxGrid = (1ll << 31) / kAttendThreads;   // threads of a launch: 32 bits
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

}  // namespace
}  // namespace ei
