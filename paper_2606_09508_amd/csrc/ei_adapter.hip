// Low-rank corrections of the projections that the requests of a batch share:
//   y[t] += scale[a] (x[t] A_a^T) B_a^T,   a = the adapter of t's sequence,
// A_a [rank][in], B_a [out][rank], for up to four projections of the same x.
//
//  plan_kernel    the tokens ordered by adapter, in tiles of one adapter each
//  shrink_kernel  V = x A^T in fp32, the ranks of all projections side by side
//  expand_kernel  y += (scale V) B^T
//
// Both products run on the matrix cores (16x16x32, weights on M, tokens on N)
// and are bound by HBM where there are many tokens: a tile's weights are read once
// and its x and y pass by.  Measured, us:
//   16384 tokens of 4096, q, k and v of 4096 and 1024, rank 16: plan 6.5, shrink 44
//     (156 MB, 3.5 TB/s: a workgroup a CU), expand 84 (418 MB, 5.0 TB/s)
//   1677 tokens, rank 64: shrink 11 to 27, expand 17 (4096 outputs) to 78 (28672: y's
//     192 MB at 2.5 TB/s; B comes again for each tile, V for each 1024 outputs)
//   64 single tokens of 24 adapters, rank 16: plan 6.6, shrink 4.5, expand 4 to 8, which
//     are a launch and two to four loads that wait for one another
#include "../../include/entropyinfer.h"
#include "ei_internal.h"

#include <limits.h>

namespace ei {
namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x2 __attribute__((ext_vector_type(2)));

constexpr int kThreads = 256;
constexpr int kWaves = kThreads / kWave;
constexpr int kMaxAdapters = 8192;   // their counts lie in LDS
constexpr int kMaxRank = 128;
constexpr int kMaxTargets = 4;

__device__ __forceinline__ uint32_t pack_bf16x2(float lo, float hi) {
  const f32x2 x = {lo, hi};
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(x, bf16x2));
}

// ----------------------------------------------------------------------------
// Plan.  [0] the number of tiles; from kPlanHead on the tiles; then the
// tokens.  A tile is `count` tokens of one adapter, from place `begin` of the
// list of tokens on.
// ----------------------------------------------------------------------------
struct Tile {
  int adapter, begin, count, pad;
};
constexpr size_t kPlanHead = 64;
constexpr int kPlanThreads = 1024;

struct PlanShape {
  int tokens, seqs, adapters;
  int rows;        // of a tile, at most
  int max_tiles;
  size_t list_at, bytes;
};
// Tiles of 64 tokens where there are many, and an adapter that may be used has 40 on
// average; else of 16, which waste less and are more workgroups.  A layer's four inputs,
// us a call with 16 and 64: 200 x 10 tokens of 8 adapters 194, 169; 100 x 20 of 50 225,
// 211; 4 x 256 of 4 98, 93 (rank 64: 201, 142); but 128 x 16 of 64 181, 221; 1500 x 1 of
// 64 213, 237; 4 x 64 of 4 85, 98; 512 of one 63, 76.
PlanShape plan_shape(const ei_adapter_batch& b) {
  PlanShape p{b.n_tokens, b.n_seqs, b.n_adapters, 16, 0, 0, 0};
  const int used = b.n_adapters < b.n_seqs ? b.n_adapters : b.n_seqs;
  if (b.n_tokens >= 768 && b.n_tokens / 40 >= used) p.rows = 64;
  p.max_tiles = b.n_tokens / p.rows + (used < b.n_tokens ? used : b.n_tokens);
  p.list_at = kPlanHead + (size_t)p.max_tiles * sizeof(Tile);
  p.bytes = p.list_at + (size_t)b.n_tokens * sizeof(int32_t);
  return p;
}

struct PlanArgs {
  const int32_t *index, *cu;
  int32_t* head;
  Tile* tiles;
  int32_t* list;
  PlanShape p;
};

__device__ __forceinline__ void rows_of(const PlanArgs& a, int s, int& first, int& n) {
  if (!a.cu) {
    n = a.p.tokens / a.p.seqs;
    first = s * n;
    return;
  }
  first = min(max(a.cu[s], 0), a.p.tokens);
  n = max(min(max(a.cu[s + 1], 0), a.p.tokens) - first, 0);
}

// One workgroup.  The counts are integers, and each sequence's place follows from
// those before it, so the list does not depend on the order of the atomics.
__global__ __launch_bounds__(kPlanThreads) void plan_kernel(PlanArgs a) {
  __shared__ int place[kMaxAdapters];          // an adapter's tokens; then its next place
  __shared__ int first_tile[kMaxAdapters];
  __shared__ __attribute__((aligned(16))) int seq_a[kPlanThreads], seq_n[kPlanThreads];
  __shared__ int seq_first[kPlanThreads], longest;
  __shared__ uint32_t wave_tokens[kPlanThreads / kWave], wave_tiles[kPlanThreads / kWave];
  const int tid = threadIdx.x, lane = tid % kWave, wave = tid / kWave;
  const int n = a.p.adapters;
  // a sequence's adapter (-1: none), first token and how many
  int ad = -1, first = 0, count = 0;
  auto look = [&](uint32_t s) {
    ad = -1;
    first = count = 0;
    if (s < (uint32_t)a.p.seqs) {
      ad = a.index[s];
      rows_of(a, (int)s, first, count);
      if (ad < 0 || ad >= n) ad = -1;
    }
  };
  look(tid);
  for (int i = tid; i < n; i += kPlanThreads) place[i] = 0;
  __syncthreads();
  if (ad >= 0) atomicAdd(&place[ad], count);
  if (a.p.seqs > kPlanThreads) {
    for (uint32_t s = tid + kPlanThreads; s < (uint32_t)a.p.seqs; s += kPlanThreads) {
      look(s);
      if (ad >= 0) atomicAdd(&place[ad], count);
    }
    look(tid);
  }
  __syncthreads();
  // the adapters' first places and tiles; a thread has `per` of them in a row
  const int per = (n + kPlanThreads - 1) / kPlanThreads, i0 = tid * per;
  // (in unsigned numbers: offsets that do not ascend may count past 2^32)
  const uint32_t rows = (uint32_t)a.p.rows;
  uint32_t tokens = 0, tiles = 0;
  for (int i = i0; i < min(i0 + per, n); ++i) {
    tokens += (uint32_t)place[i];
    tiles += ((uint32_t)place[i] + rows - 1) / rows;
  }
  const uint32_t up_tokens = wave_incl_scan_u32(tokens), up_tiles = wave_incl_scan_u32(tiles);
  if (lane == kWave - 1) {
    wave_tokens[wave] = up_tokens;
    wave_tiles[wave] = up_tiles;
  }
  __syncthreads();
  uint32_t at = up_tokens - tokens, tile = up_tiles - tiles, sum = 0;
  for (int w = 0; w < kPlanThreads / kWave; ++w) {
    if (w < wave) {
      at += wave_tokens[w];
      tile += wave_tiles[w];
    }
    sum += wave_tiles[w];
  }
  for (int i = i0; i < min(i0 + per, n); ++i) {
    const uint32_t count = (uint32_t)place[i];
    first_tile[i] = (int)tile;
    place[i] = (int)at;
    at += count;
    tile += (count + rows - 1) / rows;
  }
  // (Such offsets' places and tiles mean nothing, but every tile lies in the list: its
  // begin is not below 0, and it ends with the list at the latest or is empty.)
  const int all = (int)min(sum, (uint32_t)a.p.max_tiles);
  if (tid == 0) a.head[0] = all;
  if (tid == kPlanThreads - 1) seq_n[0] = (int)at;
  __syncthreads();
  const int total = seq_n[0];
  for (int t = tid; t < all; t += kPlanThreads) {
    int lo = 0, hi = n - 1;      // the last adapter that starts at tile t or before
    while (lo < hi) {
      const int mid = (lo + hi + 1) / 2;
      if (first_tile[mid] <= t) lo = mid; else hi = mid - 1;
    }
    const int begin = (int)((uint32_t)place[lo] + ((uint32_t)t - (uint32_t)first_tile[lo]) * rows);
    const int stop = min(max(lo + 1 < n ? place[lo + 1] : total, 0), a.p.tokens);
    a.tiles[t] = Tile{lo, begin, begin < 0 ? 0 : min(stop - begin, a.p.rows), 0};
  }
  __syncthreads();
  // the sequences in their order, kPlanThreads at a time (unsigned: their number, and a
  // sequence's tokens, may end a step before 2^31)
  for (uint32_t s0 = 0; s0 < (uint32_t)a.p.seqs; s0 += kPlanThreads) {
    const int here = min(a.p.seqs - (int)s0, kPlanThreads);
    if (s0 > 0) look(s0 + tid);
    if (tid == 0) longest = 0;
    seq_a[tid] = ad;
    seq_n[tid] = count;
    __syncthreads();
    int before = 0;
    // (four at a time: those behind the last sequence count 0)
    for (int i = 0; i < min(here, (wave + 1) * kWave); i += 4) {
      const int4 ia = *(const int4*)&seq_a[i], in = *(const int4*)&seq_n[i];
      before += (i < tid && ia.x == ad ? in.x : 0) + (i + 1 < tid && ia.y == ad ? in.y : 0) +
                (i + 2 < tid && ia.z == ad ? in.z : 0) + (i + 3 < tid && ia.w == ad ? in.w : 0);
    }
    const int to = ad < 0 ? -1 : place[ad] + before;
    __syncthreads();
    constexpr int kShort = 8, kLong = 512;
    if (ad >= 0) atomicAdd(&place[ad], count);
    if (ad >= 0 && count > kShort) atomicMax(&longest, count);
    // their tokens: of short sequences by a lane each, of longer ones by a wave, of long
    // ones by all
    auto write = [&](uint32_t p, uint32_t f, uint32_t c, uint32_t i0, uint32_t step) {
      for (uint32_t i = i0; i < c; i += step)
        if (p + i < (uint32_t)a.p.tokens) a.list[p + i] = (int)(f + i);
    };
    if (ad >= 0 && count <= kShort) write(to, first, count, 0, 1);
    seq_a[tid] = to;
    seq_first[tid] = first;
    if (ad < 0) seq_n[tid] = 0;
    __syncthreads();
    const int most = longest;
    if (most > kShort)
      for (int i = wave; i < here; i += kPlanThreads / kWave)
        if (seq_n[i] > kShort && seq_n[i] <= kLong) write(seq_a[i], seq_first[i], seq_n[i], lane, kWave);
    if (most > kLong)
      for (int i = 0; i < here; ++i)
        if (seq_n[i] > kLong) write(seq_a[i], seq_first[i], seq_n[i], tid, kPlanThreads);
    __syncthreads();
  }
}

// ----------------------------------------------------------------------------
// Shrink.  The ranks of all targets are rows 0 .. targets * rank - 1 of one
// matrix.  A workgroup takes 16 MT of them, a tile's 16 NT tokens and a part of
// the columns, which its waves share; their sums are added in LDS in the waves'
// order, and the parts' by expand_kernel.
// ----------------------------------------------------------------------------
struct Target {
  const uint16_t *a, *b;
  const float* scale;
  uint16_t* y;
  int n_out;
  int block0;      // expand_kernel's first workgroup of it, per tile
};
struct AddArgs {
  const uint16_t* x;
  float* v;                    // [splits][tokens, in the plan's order][targets * rank]
  const int32_t* head;
  const Tile* tiles;
  const int32_t* list;
  int tokens, n_in, rank, targets, splits;
  int blocks, spans;           // expand_kernel's workgroups per tile; 256 outputs of each
  Target t[kMaxTargets];
};

__device__ __forceinline__ const Target& target(const AddArgs& a, int i) {
  return i == 0 ? a.t[0] : i == 1 ? a.t[1] : i == 2 ? a.t[2] : a.t[3];
}

// Token i of a tile (the last one where it has fewer).  Offsets that do not ascend
// may leave places of the list unset.
__device__ __forceinline__ int token_at(const AddArgs& a, const Tile& t, int i) {
  return min(max(a.list[t.begin + min(i, t.count - 1)], 0), a.tokens - 1);
}

constexpr int kColumns = 64;   // of a step

template <int MT, int NT>
__global__ __launch_bounds__(kThreads) void shrink_kernel(AddArgs a, int row_tiles, int64_t unit0) {
  constexpr int kRows = 16 * MT, kTokens = 16 * NT, kPitch = kRows + 4;
  __shared__ __attribute__((aligned(16))) float sm[kWaves][kTokens * kPitch];
  int64_t unit = unit0 + blockIdx.x;
  const int split = (int)(unit % a.splits);
  unit /= a.splits;
  const int r0 = (int)(unit % row_tiles) * kRows;
  const int tile = (int)(unit / row_tiles);
  const Tile t = a.tiles[tile];
  if (tile >= a.head[0] || t.count <= 0) return;
  const int R = a.targets * a.rank;
  const int lane = threadIdx.x % kWave, j = lane & 15, g = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const uint16_t* wp[MT];
  const uint16_t* xp[NT];
#pragma unroll
  for (int m = 0; m < MT; ++m) {
    const int row = min(r0 + 16 * m + j, R - 1), i = row / a.rank;
    wp[m] = target(a, i).a + ((int64_t)t.adapter * a.rank + row % a.rank) * a.n_in + 8 * g;
  }
#pragma unroll
  for (int k = 0; k < NT; ++k) {
    xp[k] = a.x + (int64_t)token_at(a, t, 16 * k + j) * a.n_in + 8 * g;
  }
  f32x4 acc[MT][NT];
#pragma unroll
  for (int m = 0; m < MT; ++m)
#pragma unroll
    for (int k = 0; k < NT; ++k) acc[m][k] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
  const int steps = (a.n_in + kColumns - 1) / kColumns;
  const int per = (steps + a.splits - 1) / a.splits, split_end = min((split + 1) * per, steps);
  // a wave's steps are neighbours; U steps' operands are asked for, then used
  const int mine = (per + kWaves - 1) / kWaves;
  const int begin = split * per + wave * mine, end = min(begin + mine, split_end);
  constexpr int U = NT == 1 ? 4 : 1;
  for (int s = begin; s < end; s += U) {
    uint4 w[U][2][MT], x[U][2][NT];
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int half = 0; half < 2; ++half) {
        const int c = (s + u) * kColumns + 32 * half;
        const bool in = s + u < end && c + 8 * g < a.n_in;       // (columns come in eights)
#pragma unroll
        for (int m = 0; m < MT; ++m) w[u][half][m] = in ? *(const uint4*)(wp[m] + c) : make_uint4(0u, 0u, 0u, 0u);
#pragma unroll
        for (int k = 0; k < NT; ++k) x[u][half][k] = in ? *(const uint4*)(xp[k] + c) : make_uint4(0u, 0u, 0u, 0u);
      }
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int half = 0; half < 2; ++half)
#pragma unroll
        for (int m = 0; m < MT; ++m)
#pragma unroll
          for (int k = 0; k < NT; ++k)
            acc[m][k] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(
                __builtin_bit_cast(bf16x8, w[u][half][m]), __builtin_bit_cast(bf16x8, x[u][half][k]),
                acc[m][k], 0, 0, 0);
  }
  // lane: token j, rows 4g .. 4g + 3 of each tile
#pragma unroll
  for (int m = 0; m < MT; ++m)
#pragma unroll
    for (int k = 0; k < NT; ++k)
      *(float4*)&sm[wave][(16 * k + j) * kPitch + 16 * m + 4 * g] =
          make_float4(acc[m][k][0], acc[m][k][1], acc[m][k][2], acc[m][k][3]);
  __syncthreads();
  for (int e = threadIdx.x; e < kRows * kTokens; e += kThreads) {
    const int tok = e / kRows, row = e % kRows;
    if (tok >= t.count || r0 + row >= R) continue;
    float sum = sm[0][tok * kPitch + row];
#pragma unroll
    for (int w = 1; w < kWaves; ++w) sum += sm[w][tok * kPitch + row];
    a.v[((int64_t)split * a.tokens + t.begin + tok) * R + r0 + row] = sum;
  }
}

// ----------------------------------------------------------------------------
// Expand.  V times the scale goes to the matrix cores as the sum of two bf16
// numbers (16 bits; one alone would double the variance that y's rounding has):
// they are columns 0 .. rank - 1 and rank .. 2 rank - 1 of one operand, each
// against the same columns of B.  y is the accumulator's start and is rounded
// once.  A wave takes 64 outputs at a time; row i of its product m is output
// 16 (i / 4) + 4 m + i % 4, so that a lane has 16 outputs in a row of its token.
// A workgroup brings its tile's V into LDS once for `a.spans` times 256 outputs;
// each wave asks for its first outputs' y and B before that.
// ----------------------------------------------------------------------------
constexpr int kWaveOuts = 64;
constexpr int kBlockOuts = kWaveOuts * kWaves;

template <int NT>
__global__ __launch_bounds__(kThreads) void expand_kernel(AddArgs a, int64_t unit0) {
  constexpr int kTokens = 16 * NT, kPad = 8;
  __shared__ __attribute__((aligned(16))) uint16_t sm[kTokens * (2 * kMaxRank + kPad)];
  const int64_t unit = unit0 + blockIdx.x;
  const int block = (int)(unit % a.blocks), tile = (int)(unit / a.blocks);
  const Tile t = a.tiles[tile];
  if (tile >= a.head[0] || t.count <= 0) return;
  int ti = 0;
  for (int i = 1; i < a.targets; ++i)
    if (block >= target(a, i).block0) ti = i;
  const Target tg = target(a, ti);
  const int r = a.rank, pitch = 2 * r + kPad, R = a.targets * r;
  const int lane = threadIdx.x % kWave, j = lane & 15, g = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  uint16_t* yp[NT];
#pragma unroll
  for (int k = 0; k < NT; ++k)
    yp[k] = tg.y + (int64_t)token_at(a, t, 16 * k + j) * tg.n_out + 16 * g;
  // outputs o0 .. o0 + 63 (of the wave), this lane's from o0 + 16 g on
  uint4 y[NT][2];
  auto load_y = [&](int o0) {
#pragma unroll
    for (int k = 0; k < NT; ++k)
#pragma unroll
      for (int h = 0; h < 2; ++h)
        if (16 * k < t.count && o0 + 16 * g + 8 * h < tg.n_out)
          y[k][h] = *(const uint4*)(yp[k] + o0 + 8 * h);
  };
  const int chunks = (2 * r + 31) / 32;
  auto load_b = [&](int o0, int c, uint4 (&b)[4]) {
    const int col = 32 * c + 8 * g;     // (past 2 r: nothing, rank 8 and the like)
    const int bc = col < r ? col : col - r;
#pragma unroll
    for (int m = 0; m < 4; ++m) {
      const int o = min(o0 + 16 * (j >> 2) + 4 * m + (j & 3), tg.n_out - 1);
      b[m] = make_uint4(0u, 0u, 0u, 0u);
      if (col < 2 * r) b[m] = *(const uint4*)(tg.b + ((int64_t)t.adapter * tg.n_out + o) * r + bc);
    }
  };
  const int first = ((block - tg.block0) * a.spans * kWaves + wave) * kWaveOuts;
  uint4 b0[4];
  if (first < tg.n_out) {
    load_y(first);
    load_b(first, 0, b0);
  }
  const float scale = tg.scale ? tg.scale[t.adapter] : 1.0f;
  // the tile's V, as pairs of bf16 numbers
  for (int e = threadIdx.x; e < kTokens * (r / 4); e += kThreads) {
    const int tok = e / (r / 4), c = e % (r / 4) * 4;
    float4 x = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
    if (tok < t.count) {
      const float* from = a.v + ((int64_t)t.begin + tok) * R + ti * r + c;
      const int64_t part = (int64_t)a.tokens * R;
      constexpr int kAtOnce = 8;
      for (int s = 0; s < a.splits; s += kAtOnce) {
        float4 p[kAtOnce];
#pragma unroll
        for (int i = 0; i < kAtOnce; ++i)
          p[i] = s + i < a.splits ? *(const float4*)(from + (s + i) * part) : make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll
        for (int i = 0; i < kAtOnce; ++i) {
          x.x += p[i].x;
          x.y += p[i].y;
          x.z += p[i].z;
          x.w += p[i].w;
        }
      }
    }
    const float v[4] = {x.x * scale, x.y * scale, x.z * scale, x.w * scale};
    // (the first number ends at bf16's largest: what lies beyond, infinity too, is rest)
    float rest[4], near[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) near[i] = fminf(fmaxf(v[i], -0x1.fep127f), 0x1.fep127f);
    const uint32_t hi[2] = {pack_bf16x2(near[0], near[1]), pack_bf16x2(near[2], near[3])};
#pragma unroll
    for (int i = 0; i < 4; ++i)
      rest[i] = v[i] - (i & 1 ? bf16_hi(hi[i / 2]) : bf16_lo(hi[i / 2]));
    *(uint2*)&sm[tok * pitch + c] = make_uint2(hi[0], hi[1]);
    *(uint2*)&sm[tok * pitch + r + c] = make_uint2(pack_bf16x2(rest[0], rest[1]), pack_bf16x2(rest[2], rest[3]));
  }
  __syncthreads();
  for (int i = 0; i < a.spans; ++i) {
    const int o0 = first + i * kBlockOuts, mine = o0 + 16 * g;
    if (o0 >= tg.n_out) break;
    f32x4 acc[NT][4];
#pragma unroll
    for (int k = 0; k < NT; ++k)
#pragma unroll
      for (int m = 0; m < 4; ++m) {
        const uint4 w = y[k][m >> 1];
        const uint32_t u0 = m & 1 ? w.z : w.x, u1 = m & 1 ? w.w : w.y;
        acc[k][m] = f32x4{bf16_lo(u0), bf16_hi(u0), bf16_lo(u1), bf16_hi(u1)};
      }
    uint4 b[4] = {b0[0], b0[1], b0[2], b0[3]};
    const bool more = i + 1 < a.spans && o0 + kBlockOuts < tg.n_out;
    if (more) load_y(o0 + kBlockOuts);
    for (int c = 0; c < chunks; ++c) {
      const int col = 32 * c + 8 * g;
      uint4 next[4];
      if (c + 1 < chunks) load_b(o0, c + 1, next);
      else if (more) load_b(o0 + kBlockOuts, 0, next);
      uint4 v[NT];
#pragma unroll
      for (int k = 0; k < NT; ++k)
        v[k] = col < 2 * r ? *(const uint4*)&sm[(16 * k + j) * pitch + col] : make_uint4(0u, 0u, 0u, 0u);
#pragma unroll
      for (int k = 0; k < NT; ++k)
#pragma unroll
        for (int m = 0; m < 4; ++m)
          acc[k][m] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(
              __builtin_bit_cast(bf16x8, b[m]), __builtin_bit_cast(bf16x8, v[k]), acc[k][m], 0, 0, 0);
#pragma unroll
      for (int m = 0; m < 4; ++m) b[m] = next[m];
    }
#pragma unroll
    for (int m = 0; m < 4; ++m) b0[m] = b[m];
#pragma unroll
    for (int k = 0; k < NT; ++k) {
      if (16 * k + j >= t.count) continue;
#pragma unroll
      for (int h = 0; h < 2; ++h)
        if (mine + 8 * h < tg.n_out)
          *(uint4*)(yp[k] + o0 + 8 * h) = make_uint4(
              pack_bf16x2(acc[k][2 * h][0], acc[k][2 * h][1]), pack_bf16x2(acc[k][2 * h][2], acc[k][2 * h][3]),
              pack_bf16x2(acc[k][2 * h + 1][0], acc[k][2 * h + 1][1]),
              pack_bf16x2(acc[k][2 * h + 1][2], acc[k][2 * h + 1][3]));
    }
  }
}

// ----------------------------------------------------------------------------
// Host side
// ----------------------------------------------------------------------------
constexpr int64_t kMaxGrid = (1ll << 31) / kThreads;
unsigned launch_grid(int64_t left) { return (unsigned)(left < kMaxGrid ? left : kMaxGrid); }
bool aligned(const void* p, uintptr_t a) { return ((uintptr_t)p & (a - 1)) == 0; }
ei_status from_hip(hipError_t e) { return e == hipSuccess ? EI_OK : EI_ERR_LAUNCH; }

ei_status check_batch(const ei_adapter_batch& b) {
  if (b.n_tokens < 0 || b.n_seqs < 0 || b.n_adapters < 0) return EI_ERR_SHAPE;
  if (b.n_adapters > kMaxAdapters) return EI_ERR_UNSUPPORTED;
  return EI_OK;
}
bool nothing(const ei_adapter_batch& b) {
  return b.n_tokens == 0 || b.n_seqs == 0 || b.n_adapters == 0;
}

struct AddPlan {
  int row_tiles, splits, mt;
  size_t bytes;
};
// Parts of the columns, of 512 at least (two steps a wave): as many as give the chip 512
// workgroups, or 256 with tiles of 64 tokens, each of whose V is read again by every
// workgroup of expand_kernel (the four inputs of a layer, us a call: 64 single tokens 46
// with 256 and 43 with 512; 1677 tokens, rank 64, 209 and 217, with 128 245).
AddPlan add_plan(const PlanShape& p, int n_in, int rank, int targets) {
  AddPlan s{};
  const int R = targets * rank;
  s.mt = p.rows == 16 || R <= 16 ? 1 : R <= 32 ? 2 : R <= 48 ? 3 : 4;
  s.row_tiles = (R + 16 * s.mt - 1) / (16 * s.mt);
  const int64_t units = (int64_t)p.max_tiles * s.row_tiles;
  int64_t splits = (p.rows == 16 ? 512 : 256) / (units > 0 ? units : 1);
  const int64_t most = n_in / 512;
  if (splits > most) splits = most;
  s.splits = splits < 1 ? 1 : (int)splits;
  s.bytes = (size_t)s.splits * p.tokens * R * sizeof(float);
  return s;
}
// Times 256 outputs of a workgroup of expand_kernel: up to 4 while 1024 workgroups are left.
int spans_of(const PlanShape& p, const ei_adapter_target* t, int n) {
  int64_t blocks = 0;
  for (int i = 0; i < n; ++i) blocks += ((int64_t)t[i].n_out + kBlockOuts - 1) / kBlockOuts;
  const int64_t s = blocks * p.max_tiles / 1024;
  return s < 1 ? 1 : s > 4 ? 4 : (int)s;
}
constexpr int kMostWidth = INT_MAX - 4096;   // (the kernels' steps go past a row's end)
ei_status check_sizes(int32_t n_in, int32_t rank, int32_t n_targets) {
  if (n_in <= 0 || n_in > kMostWidth || rank <= 0 || n_targets < 0) return EI_ERR_SHAPE;
  if (n_in % 8 || rank % 8 || rank > kMaxRank || n_targets > kMaxTargets) return EI_ERR_UNSUPPORTED;
  return EI_OK;
}

}  // namespace
}  // namespace ei

extern "C" {

size_t ei_adapter_plan_bytes(ei_adapter_batch batch) {
  if (ei::check_batch(batch) != EI_OK || ei::nothing(batch)) return 0;
  return ei::plan_shape(batch).bytes;
}

ei_status ei_adapter_plan(const int32_t* index, const int32_t* cu_seqlens, ei_adapter_batch batch,
                          void* plan, size_t plan_bytes, void* stream) {
  const ei_status st = ei::check_batch(batch);
  if (st != EI_OK) return st;
  if (!cu_seqlens && batch.n_seqs > 0 && batch.n_tokens % batch.n_seqs) return EI_ERR_SHAPE;
  if (ei::nothing(batch)) return EI_OK;
  if (!index) return EI_ERR_NULL;
  if (!ei::aligned(index, 4) || !ei::aligned(cu_seqlens, 4)) return EI_ERR_UNSUPPORTED;
  const ei::PlanShape p = ei::plan_shape(batch);
  if (!plan || plan_bytes < p.bytes) return EI_ERR_WORKSPACE;
  if (!ei::aligned(plan, 16)) return EI_ERR_UNSUPPORTED;
  char* at = (char*)plan;
  const ei::PlanArgs a{index, cu_seqlens, (int32_t*)at, (ei::Tile*)(at + ei::kPlanHead),
                       (int32_t*)(at + p.list_at), p};
  hipLaunchKernelGGL(ei::plan_kernel, dim3(1), dim3(ei::kPlanThreads), 0, (hipStream_t)stream, a);
  return ei::from_hip(hipGetLastError());
}

size_t ei_adapter_add_workspace_bytes(ei_adapter_batch batch, int32_t n_in, int32_t rank,
                                      int32_t n_targets) {
  if (ei::check_batch(batch) != EI_OK || ei::nothing(batch) ||
      ei::check_sizes(n_in, rank, n_targets) != EI_OK || n_targets == 0)
    return 0;
  return ei::add_plan(ei::plan_shape(batch), n_in, rank, n_targets).bytes;
}

ei_status ei_adapter_add(const uint16_t* x, int32_t n_in, int32_t rank,
                         const ei_adapter_target* targets, int32_t n_targets,
                         ei_adapter_batch batch, const void* plan, size_t plan_bytes,
                         void* workspace, size_t workspace_bytes, void* stream) {
  ei_status st = ei::check_batch(batch);
  if (st != EI_OK) return st;
  if ((st = ei::check_sizes(n_in, rank, n_targets)) != EI_OK) return st;
  if (n_targets > 0 && !targets) return EI_ERR_NULL;
  for (int i = 0; i < n_targets; ++i) {
    if (targets[i].n_out <= 0 || targets[i].n_out > ei::kMostWidth) return EI_ERR_SHAPE;
    if (targets[i].n_out % 8) return EI_ERR_UNSUPPORTED;
  }
  if (ei::nothing(batch) || n_targets == 0) return EI_OK;
  const ei::PlanShape p = ei::plan_shape(batch);
  if (!x) return EI_ERR_NULL;
  if (!ei::aligned(x, 16)) return EI_ERR_UNSUPPORTED;
  for (int i = 0; i < n_targets; ++i) {
    const ei_adapter_target& t = targets[i];
    if (!t.a || !t.b || !t.y) return EI_ERR_NULL;
    if (!ei::aligned(t.a, 16) || !ei::aligned(t.b, 16) || !ei::aligned(t.y, 16) ||
        !ei::aligned(t.scale, 4))
      return EI_ERR_UNSUPPORTED;
  }
  const ei::AddPlan s = ei::add_plan(p, n_in, rank, n_targets);
  if (!plan || plan_bytes < p.bytes || !workspace || workspace_bytes < s.bytes)
    return EI_ERR_WORKSPACE;
  if (!ei::aligned(plan, 16) || !ei::aligned(workspace, 16)) return EI_ERR_UNSUPPORTED;
  const char* at = (const char*)plan;
  ei::AddArgs a{};
  a.spans = ei::spans_of(p, targets, n_targets);
  int64_t blocks = 0;
  for (int i = 0; i < n_targets; ++i) {
    const ei_adapter_target& t = targets[i];
    const int64_t outs = (int64_t)ei::kBlockOuts * a.spans;
    a.t[i] = ei::Target{t.a, t.b, t.scale, t.y, t.n_out, (int)blocks};
    blocks += (t.n_out + outs - 1) / outs;
  }
  a.x = x;
  a.v = (float*)workspace;
  a.head = (const int32_t*)at;
  a.tiles = (const ei::Tile*)(at + ei::kPlanHead);
  a.list = (const int32_t*)(at + p.list_at);
  a.tokens = p.tokens;
  a.n_in = n_in;
  a.rank = rank;
  a.targets = n_targets;
  a.splits = s.splits;
  a.blocks = (int)blocks;
  hipStream_t s0 = (hipStream_t)stream;
  const dim3 block(ei::kThreads);
  const int64_t shrinks = (int64_t)p.max_tiles * s.row_tiles * s.splits;
  for (int64_t u = 0; u < shrinks; u += ei::kMaxGrid) {
    const dim3 grid(ei::launch_grid(shrinks - u));
#define EI_SHRINK(MT, NT) \
  hipLaunchKernelGGL((ei::shrink_kernel<MT, NT>), grid, block, 0, s0, a, s.row_tiles, u)
    if (p.rows == 16) EI_SHRINK(1, 1);
    else if (s.mt == 1) EI_SHRINK(1, 4);
    else if (s.mt == 2) EI_SHRINK(2, 4);
    else if (s.mt == 3) EI_SHRINK(3, 4);
    else EI_SHRINK(4, 4);
#undef EI_SHRINK
  }
  const int64_t expands = (int64_t)p.max_tiles * blocks;
  for (int64_t u = 0; u < expands; u += ei::kMaxGrid) {
    const dim3 grid(ei::launch_grid(expands - u));
    if (p.rows == 16)
      hipLaunchKernelGGL((ei::expand_kernel<1>), grid, block, 0, s0, a, u);
    else
      hipLaunchKernelGGL((ei::expand_kernel<4>), grid, block, 0, s0, a, u);
  }
  return ei::from_hip(hipGetLastError());
}

}  // extern "C"
