// Attention over the paged cache for sequences that share their first pages.
//
// A group's sequences name the same pages in their first `shared` columns.  The
// keys there are read once for all new tokens of the group, the keys behind them
// for each sequence by itself, and the sums are joined.
//
//  shared_plan_kernel   how many pages a group shares in earnest (none that a new
//                       token of it lies in or before), and where the work of
//                       groups and sequences starts
//  shared_wide_kernel   where a group has many rows: the groups' keys, tiles of 64
//                       or 128 rows against keys in LDS, then the sequences' own keys
//  shared_steps_kernel  where they have few, both: 16 or 32 rows against keys in
//                       registers, as cache attention
//  shared_join_kernel   a row's parts joined
//
// Work is counted in units, the items (rows of a group or sequence and a KV head)
// one behind the other, and dealt out in runs of equal length.  A worker leaves a
// part of every item that its run touches at slot (item + worker): both only grow
// along the units, so no two parts meet, and items + workers slots suffice.
//
// Measured, us (plan, keys, join):
//   64 sequences behind 32768 keys, 32 heads over 8:   5.9 + 71.5 + 7.0; 57 of the 71.5
//       are the shared keys, 34 GFLOP at 600 TFLOP/s, matrix cores busy 0.27 of the time
//   16 behind 8192, the same heads:                    5.2 + 21 + 6.9
//   9, 5 and 17 behind 2048 to 12288, 4 new tokens
//     each, 64 over 8, int8:                           6.0 + 71.6 + 10.2
//   2 behind 960, 4 heads over 1:                      5.5 + 7.3 + 4.1
#include "ei_attend.h"

namespace ei {
namespace {

constexpr int kThreads = kAttendThreads, kWaves = kAttendWaves;
constexpr int kRows = kAttendRows, kKeys = kAttendKeys;
constexpr int kPlanThreads = 1024;
constexpr int kWideThreads = 512;
constexpr int kWideWaves = kWideThreads / kWave;
constexpr int kWideKeys = 128;        // of a step
constexpr int kWideWorkers = 256;     // one a CU
constexpr int kWideCost = 1;          // units of an item before its steps, unless runs are whole
constexpr int kWideLeast = 2;         // units of a run, at least
constexpr int kStepsGroups = 512;     // workgroups, two a CU
static_assert(kStepsGroups * kWaves == kWideWorkers * kWideWaves, "the same waves");
constexpr int kStepsCost = 5;
constexpr int kStepsLeast = 8;        // half of it where not a quarter of the waves would have one

typedef _Float16 half8 __attribute__((ext_vector_type(8)));
typedef _Float16 half2 __attribute__((ext_vector_type(2)));
typedef float f32x16 __attribute__((ext_vector_type(16)));

struct Totals {
  int64_t wide_per, steps_per;       // units of a run
  int64_t group_units, seq_units;
  int32_t bad;                       // lists that count more items than there is room for
  int32_t wide_cost, pad[6];         // units of a wide item before its steps
};
struct GroupInfo {      // its shared keys; n = 0 where there are none
  int first, n, pages, lead;
  int64_t unit;
  int item, pad;
};
struct SeqInfo {        // its own keys
  int group, key0, item, pad;
  int64_t unit;
  int first, n;
};

struct SharedArgs {
  AttendArgs a;             // (part_ml and part_o: the parts of shared_steps_kernel)
  const int32_t *group_seqs, *shared_pages;
  int n_groups;
  int wide_rows;            // of a tile, 0: groups' keys go to shared_steps_kernel
  int steps_rows;
  int steps_workers;
  int64_t wide_items, steps_items;   // slots there are, less the workers
  Totals* totals;
  GroupInfo* groups;
  SeqInfo* seqs;
  Part* wide_ml;
  float* wide_o;
};

// Steps of a group's items.
__device__ __forceinline__ int64_t group_steps(const SharedArgs& x, int pages) {
  const int64_t keys = (int64_t)pages * x.a.pg.P;
  return x.wide_rows ? (keys + kWideKeys - 1) / kWideKeys : keys / kKeys;
}
// Whether items of so many steps are whole runs when all workers have the same: an item's
// cost in units would then only push the runs off the items' ends.  Without and with
// this, 32 heads over 8, us a call: 16 sequences behind 8192 keys 35, 33; 16 behind 16384
// 40, 36; 64 behind 32768 79, 77; but 64 behind 8192 51, 52 and 64 behind 4096 44, 47.  A
// page more, where it does not apply, is no jump: 8256 32, 16448 37, 33024 79.
__device__ __forceinline__ bool whole_runs(int64_t units, int64_t steps) {
  const int64_t per = units / kWideWorkers;
  return per >= kWideLeast && units % kWideWorkers == 0 && steps % per == 0;
}
__device__ __forceinline__ int group_cost(const SharedArgs& x, bool whole) {
  return !x.wide_rows ? kStepsCost : whole ? 0 : kWideCost;
}

__device__ __forceinline__ int64_t block_before(int64_t* sums, int64_t v, int64_t& total) {
  // the sum over the threads before this one, and over all
  const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
  const int64_t up = (int64_t)wave_incl_scan_u64((uint64_t)v);
  __syncthreads();
  if (lane == kWave - 1) sums[wave] = up;
  __syncthreads();
  int64_t before = up - v;
  total = 0;
  for (int w = 0; w < kPlanThreads / kWave; ++w) {
    if (w < wave) before += sums[w];
    total += sums[w];
  }
  return before;
}

// units, items: of shared_steps_kernel (with the groups' where it has those too).
__device__ __forceinline__ void finish_totals(const SharedArgs& x, Totals t, int64_t units,
                                              int64_t items) {
  // (Offsets that do not ascend may name tokens or sequences twice.)
  t.bad |= items > x.steps_items;
  if (t.bad) t.group_units = units = 0;
  t.seq_units = units;
  const int64_t w = (t.group_units + kWideWorkers - 1) / kWideWorkers;
  const int64_t n = (units + x.steps_workers - 1) / x.steps_workers;
  t.wide_per = w > kWideLeast ? w : kWideLeast;
  // (half: 16 sequences of about 250 keys of their own 35.0 -> 32.5 us a call; always
  // half: 32 of about 1000, 32 rows each, 79 -> 84)
  const int least = units < (int64_t)x.steps_workers * kStepsLeast / 4 ? kStepsLeast / 2 : kStepsLeast;
  t.steps_per = n > least ? n : least;
  *x.totals = t;
}

__global__ __launch_bounds__(kPlanThreads) void shared_plan_kernel(SharedArgs x) {
  __shared__ int64_t sums[kPlanThreads / kWave];
  const AttendArgs& a = x.a;
  const int S = a.tk.S, P = a.pg.P, G = a.Hq / a.pg.Hkv;
  const int tid = threadIdx.x, lane = tid % kWave, wave = tid / kWave;
  for (int s = tid; s < S; s += kPlanThreads) {
    SeqInfo q{};
    q.group = -1;
    seq_rows(a.tk, s, q.first, q.n);
    x.seqs[s] = q;
  }
  __syncthreads();
  for (int g = wave; g < x.n_groups; g += kPlanThreads / kWave) {
    const int b = min(max(x.group_seqs[g], 0), S), e = min(max(x.group_seqs[g + 1], 0), S);
    int pages = min(max(x.shared_pages[g], 0), a.pg.max_pages);
    GroupInfo q{};
    if (b < e) {
      for (int s = b + lane; s < e; s += kWave) {
        int first, n;
        seq_rows(a.tk, s, first, n);
        if (n > 0) pages = min(pages, max(max(a.lengths[s], 0) - n, 0) / P);
      }
      pages = (int)wave_min_u32_f((uint32_t)pages);
      int n0, end, n1;
      seq_rows(a.tk, b, q.first, n0);
      seq_rows(a.tk, e - 1, end, n1);
      q.n = pages > 0 ? max(end + n1 - q.first, 0) : 0;
      q.pages = pages;
      q.lead = b;
      if (q.n > 0)
        for (int s = b + lane; s < e; s += kWave) {
          x.seqs[s].group = g;
          x.seqs[s].key0 = pages * P;
        }
    }
    if (lane == 0) x.groups[g] = q;
  }
  __syncthreads();
  const int tile = x.wide_rows ? x.wide_rows : x.steps_rows;
  int64_t units = 0, items = 0;
  for (int g0 = 0; g0 < x.n_groups; g0 += kPlanThreads) {
    const int g = g0 + tid;
    int64_t u = 0, it = 0, all_u, all_it;
    if (g < x.n_groups && x.groups[g].n > 0) {
      it = ((int64_t)x.groups[g].n * G + tile - 1) / tile * a.pg.Hkv;
      u = it * group_steps(x, x.groups[g].pages);
    }
    const int64_t bu = block_before(sums, u, all_u), bi = block_before(sums, it, all_it);
    if (g < x.n_groups) {
      x.groups[g].unit = units + bu;
      x.groups[g].item = (int)(items + bi);
    }
    units += all_u;
    items += all_it;
  }
  // (each thread has its own groups' units: the ones it wrote)
  bool whole = true;
  for (int g = tid; g < x.n_groups; g += kPlanThreads)
    whole &= x.groups[g].n == 0 || whole_runs(units, group_steps(x, x.groups[g].pages));
  const int cost = group_cost(x, __syncthreads_and(whole));
  for (int g = tid; g < x.n_groups; g += kPlanThreads)
    x.groups[g].unit += (int64_t)cost * x.groups[g].item;
  Totals t{};
  t.wide_cost = cost;
  t.group_units = units += cost * items;
  if (x.wide_rows) {
    t.bad = items > x.wide_items;
    units = items = 0;
  }
  for (int s0 = 0; s0 < S; s0 += kPlanThreads) {
    const int s = s0 + tid;
    int64_t u = 0, it = 0, all_u, all_it;
    if (s < S) {
      const int64_t keys = min((int64_t)max(a.lengths[s], 0), (int64_t)a.pg.max_pages * P);
      it = ((int64_t)x.seqs[s].n * G + x.steps_rows - 1) / x.steps_rows * a.pg.Hkv;
      u = it * ((max(keys - x.seqs[s].key0, (int64_t)0) + kKeys - 1) / kKeys + kStepsCost);
    }
    const int64_t bu = block_before(sums, u, all_u), bi = block_before(sums, it, all_it);
    if (s < S) {
      x.seqs[s].unit = units + bu;
      x.seqs[s].item = (int)(items + bi);
    }
    units += all_u;
    items += all_it;
  }
  if (tid == 0) finish_totals(x, t, units, items);
}

// The same for up to 256 sequences and groups, a thread each, with one round trip to
// memory and back (of 8.4 us, the other's, most is its seven).
constexpr int kFewThreads = 256;
__global__ __launch_bounds__(kFewThreads) void shared_plan_few_kernel(SharedArgs x) {
  constexpr int W = kFewThreads / kWave;
  __shared__ int g_first[kFewThreads + 1], g_pages[kFewThreads];
  __shared__ int s_first[kFewThreads], s_end[kFewThreads];
  __shared__ int64_t units_of[W];
  __shared__ int64_t items_of[W];
  const AttendArgs& a = x.a;
  const int S = a.tk.S, P = a.pg.P, G = a.Hq / a.pg.Hkv, n_groups = x.n_groups;
  const int t = threadIdx.x, lane = t % kWave, wave = t / kWave;
  int first = 0, n = 0, length = 0;
  if (t < S) {
    length = a.lengths[t];
    if (a.tk.cu) {
      first = min(max(a.tk.cu[t], 0), a.tk.T);
      n = max(min(max(a.tk.cu[t + 1], 0), a.tk.T) - first, 0);
    } else {
      n = a.tk.each;
      first = t * n;
    }
  }
  s_first[t] = first;
  s_end[t] = first + n;
  if (n_groups > 0) {
    if (t <= n_groups) g_first[t] = min(max(x.group_seqs[t], 0), S);
    if (t == 0 && n_groups == kFewThreads) g_first[n_groups] = min(max(x.group_seqs[n_groups], 0), S);
    if (t < n_groups) g_pages[t] = min(max(x.shared_pages[t], 0), a.pg.max_pages);
  }
  __syncthreads();
  // a sequence's group, if any
  int group = -1;
  if (t < S && n_groups > 0) {
    int lo = 0, hi = n_groups - 1;
    while (lo < hi) {
      const int mid = (lo + hi + 1) / 2;
      if (g_first[mid] <= t) lo = mid; else hi = mid - 1;
    }
    if (g_first[lo] <= t && t < g_first[lo + 1]) group = lo;
    if (group >= 0 && n > 0) atomicMin(&g_pages[group], max(max(length, 0) - n, 0) / P);
  }
  __syncthreads();
  GroupInfo gi{};
  if (t < n_groups) {
    const int b = g_first[t], e = g_first[t + 1];
    if (b < e) {
      gi.first = s_first[b];
      gi.pages = g_pages[t];
      gi.lead = b;
      gi.n = gi.pages > 0 ? max(s_end[e - 1] - gi.first, 0) : 0;
    }
  }
  SeqInfo si{};
  si.group = group >= 0 && g_pages[group] > 0 ? group : -1;
  si.key0 = si.group >= 0 ? g_pages[group] * P : 0;
  si.first = first;
  si.n = n;
  auto sum_before = [&](int64_t& u, int64_t& it, int64_t& all_u, int64_t& all_it) {
    const int64_t uu = (int64_t)wave_incl_scan_u64((uint64_t)u);
    const int64_t ii = (int64_t)wave_incl_scan_u64((uint64_t)it);
    __syncthreads();
    if (lane == kWave - 1) {
      units_of[wave] = uu;
      items_of[wave] = ii;
    }
    __syncthreads();
    u = uu - u;
    it = ii - it;
    all_u = all_it = 0;
#pragma unroll
    for (int w = 0; w < W; ++w) {
      if (w < wave) {
        u += units_of[w];
        it += items_of[w];
      }
      all_u += units_of[w];
      all_it += items_of[w];
    }
  };
  const int tile = x.wide_rows ? x.wide_rows : x.steps_rows;
  int64_t units, items, all_u, all_it;
  {
    items = ((int64_t)gi.n * G + tile - 1) / tile * a.pg.Hkv;
    units = items * group_steps(x, gi.pages);
  }
  sum_before(units, items, all_u, all_it);
  const int cost =
      group_cost(x, __syncthreads_and(gi.n == 0 || whole_runs(all_u, group_steps(x, gi.pages))));
  gi.unit = units + cost * items;
  gi.item = (int)items;
  all_u += cost * all_it;
  Totals total{};
  total.wide_cost = cost;
  total.group_units = all_u;
  int64_t base_u = all_u, base_it = all_it;
  if (x.wide_rows) {
    total.bad = all_it > x.wide_items;
    base_u = base_it = 0;
  }
  {
    const int64_t keys = min((int64_t)max(length, 0), (int64_t)a.pg.max_pages * P);
    items = ((int64_t)n * G + x.steps_rows - 1) / x.steps_rows * a.pg.Hkv;
    units = items * ((max(keys - si.key0, (int64_t)0) + kKeys - 1) / kKeys + kStepsCost);
  }
  sum_before(units, items, all_u, all_it);
  si.unit = base_u + units;
  si.item = (int)(base_it + items);
  if (t < n_groups) x.groups[t] = gi;
  if (t < S) x.seqs[t] = si;
  if (t == 0) finish_totals(x, total, base_u + all_u, base_it + all_it);
}

// The last of n elements of a list whose unit is at most u.
template <class Info>
__device__ __forceinline__ int at_unit(const Info* list, int n, int64_t u) {
  int lo = 0, hi = n - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) / 2;
    if (entry(&list->unit, (int64_t)mid * (sizeof(Info) / 8)) <= u) lo = mid; else hi = mid - 1;
  }
  return lo;
}
template <class Info>
__device__ __forceinline__ Info info_at(const Info* list, int i) {
  static_assert(sizeof(Info) == 32, "read as four words of 64 bits");
  uint64_t w[4];
#pragma unroll
  for (int k = 0; k < 4; ++k) w[k] = entry((const uint64_t*)list, (int64_t)i * 4 + k);
  return __builtin_bit_cast(Info, w);
}

// ----------------------------------------------------------------------------
// Steps of 32 keys in registers: a wave takes a run of the sequences' own keys,
// behind the groups' where those have few rows (then in a launch of their own).
// ----------------------------------------------------------------------------
template <int FMT, int P, int RT>
__device__ __forceinline__ void steps_run(const SharedArgs& x, int worker) {
  const AttendArgs& a = x.a;
  const int G = a.Hq / a.pg.Hkv, lane = threadIdx.x % kWave, j = lane & 15, g4 = lane >> 4;
  const int64_t per = entry(&x.totals->steps_per, 0), total = entry(&x.totals->seq_units, 0);
  const int64_t groups = x.wide_rows ? 0 : entry(&x.totals->group_units, 0);
  int64_t u = worker * per;
  const int64_t u1 = min(u + per, total);
  if (u >= u1) return;
  int g = u < groups ? at_unit(x.groups, x.n_groups, u) : x.n_groups;
  int s = u < groups ? 0 : at_unit(x.seqs, a.tk.S, u);
  while (u < u1 && s < a.tk.S) {
    const bool is_group = u < groups;
    int first, n, lead, seq_len, key0, key1, item0;
    int64_t start;
    if (is_group) {
      const GroupInfo q = info_at(x.groups, g);
      first = q.first; n = q.n; lead = q.lead; key0 = 0; key1 = q.pages * P;
      item0 = q.item; start = q.unit;
      seq_len = INT_MAX / 2;      // (every row sees all of them)
    } else {
      const SeqInfo q = info_at(x.seqs, s);
      first = q.first; n = q.n; lead = s; key0 = q.key0; seq_len = entry(a.lengths, s);
      key1 = keys_of<P>(a, s);
      item0 = q.item; start = q.unit;
    }
    const int tiles = (n * G + kRows * RT - 1) / (kRows * RT);
    const int steps = (max(key1 - key0, 0) + kKeys - 1) / kKeys, whole = steps + kStepsCost;
    const int64_t off = u - start;
    const int item = (int)(off / whole), at = (int)(off % whole);
    if (n == 0 || item >= tiles * a.pg.Hkv) {
      if (is_group) ++g; else ++s;
      if (is_group && g >= x.n_groups) break;      // (the units of groups end with the last one)
      continue;
    }
    const int to = (int)min((int64_t)whole, at + (u1 - u));
    u += to - at;
    const int st0 = max(at - kStepsCost, 0), st1 = max(to - kStepsCost, 0);
    const int kvh = item / tiles, row0 = item % tiles * kRows * RT;
    WaveSums<RT> ws;
    attend_steps<FMT, P, RT>(a, lead, kvh, row0, first, n, seq_len, key0 + kKeys * st0,
                             min(key0 + kKeys * st1, max(key1, key0)), 0, 1, ws);
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
      const int row = kRows * rt + j;
      if (row0 + row >= n * G) continue;
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        float v[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = ws.o[rt][i][q];
        store_part<RT>(a, item0 + item + worker, row, 8 * (4 * g4 + q), ws.m[rt], ws.l[rt], v);
      }
    }
  }
}

template <int FMT, int P, int RT>
__global__ __launch_bounds__(kThreads, attend_occupancy(RT)) void shared_steps_kernel(SharedArgs x) {
  steps_run<FMT, P, RT>(x, __builtin_amdgcn_readfirstlane(threadIdx.x / kWave) * (int)gridDim.x +
                               (int)blockIdx.x);
}

// ----------------------------------------------------------------------------
// Wide tiles.  8 waves: RW of them have 32 rows each, KW = 8 / RW share the 128
// keys of a step.  K lies in LDS as bf16 [key][dim], V as fp16 [dim][key].
//   S^T = K Q^T        MFMA 32x32x16 bf16 (keys on M, rows on N)
//   O^T += V^T P^T     MFMA 32x32x16 f16 (dims on M)
// Operand layouts (lane l, j = l % 32, h = l / 32): A[i][k]: i = j, k = 8h .. 8h+7;
// B[k][n]: n = j, the same k; D[i][n]: n = j, i = 8 (r / 4) + 4h + r % 4, r < 16.  A
// lane's scores of 16 keys are thus its B operand of the second product where V's
// operand takes the keys 4h .. 4h+3 and 8+4h .. 8+4h+3 of them.
//
// Both formats' codes are exact in bf16 and in fp16.  The probabilities enter the
// second product as one fp16 number each (11 bits, against 8 of bf16; rounding them
// costs a tenth of what the output's rounding to bf16 does): e = 2^(x + E - M) with x
// the score (base 2), E the exponent of V's scale, and M a running maximum of x + E,
// less 8, that may trail by 6 more: e is at most 2^14, and what fp16 loses lies 2^-32
// below the row's largest.  A scale's significand, 1 from cache_store, is multiplied
// in where it is not.
//
// What a key weighs has nothing to do with V's scale, and a page of zeros has one of
// 2^-126: l = sum of 2^(x - ml) has a running maximum of its own, ml, of x alone, that
// may trail by 14.  A page's part of it is that of e times 2^(M - E - ml), or, where
// that is past 2^64 (e may have lost keys that weigh 2^-62), summed from the scores.
// At an item's end O is brought to ml.
// ----------------------------------------------------------------------------
constexpr float kWideLimit = 0x1p14f;
constexpr float kWideHead = 8.0f;
constexpr float kWideGap = 64.0f;

template <int FMT, bool HI>
__device__ __forceinline__ uint32_t half2_of(uint32_t x) {
  if constexpr (FMT == EI_CACHE_E4M3) {
    return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(x, 1.0f, HI));
  } else {
    // 1024 + 128 + code, by the bits, less 1152
    const uint32_t w = __builtin_amdgcn_perm(0x64646464u, x ^ 0x80808080u,
                                             HI ? 0x04030402u : 0x04010400u);
    const half2 d = __builtin_bit_cast(half2, w) - half2{(_Float16)1152.0f, (_Float16)1152.0f};
    return __builtin_bit_cast(uint32_t, d);
  }
}
__device__ __forceinline__ uint32_t pack_half2(float lo, float hi) {
  const f32x2 x = {lo, hi};
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(x, half2));
}

// Rows of 272 bytes for a key, of 264 for a dim: the lanes of a read, a row each, then
// lie at banks of their own, and all of a wave's reads have one address and constant
// offsets from it.
constexpr int kKeyPitch = kHeadDim * 2 + 16, kDimPitch = kWideKeys * 2 + 8;
struct __attribute__((aligned(16))) WideSmem {
  uint8_t k[2][kWideKeys * kKeyPitch];
  uint8_t v[2][kHeadDim * kDimPitch];
};

template <int FMT, int P, int RW>
__device__ __forceinline__ void wide_run(const SharedArgs& x, WideSmem& sm) {
  constexpr int KW = kWideWaves / RW, KT = kWideKeys / KW / 32;   // key tiles of a wave
  constexpr int kRowsOf = 32 * RW;
  const AttendArgs& a = x.a;
  const int G = a.Hq / a.pg.Hkv, lane = threadIdx.x % kWave, j = lane & 31, h = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const int rw = wave % RW, kw = wave / RW;
  const int64_t per = entry(&x.totals->wide_per, 0), total = entry(&x.totals->group_units, 0);
  const int cost = entry(&x.totals->wide_cost, 0);
  const int worker = (int)blockIdx.x;
  int64_t u = worker * per;
  const int64_t u1 = min(u + per, total);
  if (u >= u1) return;
  int g = at_unit(x.groups, x.n_groups, u);
  for (; u < u1 && g < x.n_groups; ) {
    const GroupInfo q = info_at(x.groups, g);
    const int tiles = (q.n * G + kRowsOf - 1) / kRowsOf;
    const int steps = (int)(((int64_t)q.pages * P + kWideKeys - 1) / kWideKeys);
    const int whole = steps + cost;
    const int64_t off = u - q.unit;
    const int item = (int)(off / whole), at = (int)(off % whole);
    if (q.n == 0 || item >= tiles * a.pg.Hkv) {    // (a group without units, or behind this one)
      ++g;
      continue;
    }
    const int to = (int)min((int64_t)whole, at + (u1 - u));
    u += to - at;
    const int st0 = max(at - cost, 0), st1 = max(to - cost, 0);
    const int kvh = item / tiles, row0 = item % tiles * kRowsOf, rows = q.n * G;
    const int64_t table_row = (int64_t)q.lead * a.pg.max_pages;

    bf16x8 qf[8];
    {
      const int row = min(row0 + 32 * rw + j, rows - 1);
      const uint16_t* qp = a.q + ((int64_t)(kvh * G + row % G) * a.tk.T + q.first + row / G) * kHeadDim;
#pragma unroll
      for (int c = 0; c < 8; ++c)
        qf[c] = __builtin_bit_cast(bf16x8, *(const uint4*)(qp + 16 * c + 8 * h));
      // (waited for here: in the loop a wait for them is one for the codes on their way)
#pragma unroll
      for (int c = 0; c < 8; ++c) asm volatile("" : "+v"(qf[c]));
    }
    float M = -INFINITY, ml = -INFINITY, l = 0.0f;
    f32x16 o[4];
#pragma unroll
    for (int m = 0; m < 4; ++m)
#pragma unroll
      for (int r = 0; r < 16; ++r) o[m][r] = 0.0f;

    // the page of a step's 64 keys number `half`, -1 for none; its first of those keys
    const int keys = q.pages * P;
    auto number_of = [&](int st, int half) -> int {
      const int64_t key = min((int64_t)st * kWideKeys + 64 * half, (int64_t)keys - 64);
      return entry(a.pg.table, table_row + key / P);
    };
    auto page_of = [&](int number, int st, int half) -> int {
      const bool in = st < st1 && st * kWideKeys + 64 * half < keys;
      return in && (unsigned)number < (unsigned)a.pg.n_pages ? number : -1;
    };
    auto rows_of = [&](const uint8_t* base, int page, int half) -> const uint8_t* {
      const int first = P == kWideKeys ? 64 * half : 0;
      return base + (((int64_t)page * a.pg.Hkv + kvh) * P + first) * kHeadDim;
    };
    // K: a thread has 16 dims of a key of each half.  V: 8 dims (number v_dims) of 4 keys
    // (number v_keys); a wave has 32 keys and 64 dims, the 32 lanes that write together
    // 4 by 8 of them, each at banks of its own (with 2 by 16 a step took 1500 of 6500
    // cycles more).
    const uint32_t k_off = threadIdx.x * 16;
    const int v_dims = 8 * (wave & 1) + (lane & 3) + 4 * (lane >> 5), v_half = wave / 4;
    const int v_keys = 8 * (wave >> 1) + (lane >> 2 & 7);
    const uint32_t v_off = (uint32_t)((v_keys & 15) * 4 * kHeadDim + 8 * v_dims);
    uint4 kr[2] = {};
    uint2 vr[4] = {};
    auto load = [&](int p0, int p1) {
      if (p0 >= 0) kr[0] = *(const uint4*)(rows_of(a.pg.k, p0, 0) + k_off);
      if (p1 >= 0) kr[1] = *(const uint4*)(rows_of(a.pg.k, p1, 1) + k_off);
      const int page = v_half ? p1 : p0;
      if (page >= 0) {
        const uint8_t* v = rows_of(a.pg.v, page, v_half);
#pragma unroll
        for (int r = 0; r < 4; ++r) vr[r] = *(const uint2*)(v + v_off + r * kHeadDim);
      }
    };
    auto stage = [&](int buf) {
      uint8_t* k_to = sm.k[buf] + threadIdx.x / 8 * kKeyPitch + threadIdx.x % 8 * 32;
#pragma unroll
      for (int half = 0; half < 2; ++half) {
        *(bf16x8*)(k_to + 64 * half * kKeyPitch) = widen8<FMT>(kr[half].x, kr[half].y);
        *(bf16x8*)(k_to + 64 * half * kKeyPitch + 16) = widen8<FMT>(kr[half].z, kr[half].w);
      }
      uint8_t* v_to = sm.v[buf] + v_dims * 8 * kDimPitch + v_keys * 8;
#pragma unroll
      for (int word = 0; word < 2; ++word) {
        uint32_t pr[2][2];      // [keys 0-1, 2-3][dims 0-1, 2-3]: bytes of two keys side by side
#pragma unroll
        for (int c = 0; c < 2; ++c) {
          const uint32_t w0 = word ? vr[2 * c].y : vr[2 * c].x;
          const uint32_t w1 = word ? vr[2 * c + 1].y : vr[2 * c + 1].x;
          pr[c][0] = __builtin_amdgcn_perm(w1, w0, 0x05010400u);
          pr[c][1] = __builtin_amdgcn_perm(w1, w0, 0x07030602u);
        }
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          uint8_t* to = v_to + (4 * word + 2 * i) * kDimPitch;
          *(uint2*)to = make_uint2(half2_of<FMT, false>(pr[0][i]), half2_of<FMT, false>(pr[1][i]));
          *(uint2*)(to + kDimPitch) =
              make_uint2(half2_of<FMT, true>(pr[0][i]), half2_of<FMT, true>(pr[1][i]));
        }
      }
    };

    const int my_half = kw * (32 * KT) / 64;
    auto scale_at = [&](int page) { return page < 0 ? 0 : (int64_t)page * a.pg.Hkv + kvh; };
    // (where there is no page any scale will do, but a cache of none has no scales)
    const float* const some = (const float*)a.lengths;
    const float* const k_scales = a.pg.n_pages ? a.pg.ks : some;
    const float* const v_scales = a.pg.n_pages ? a.pg.vs : some;
    f32x16 s[KT];
    auto scores = [&](int buf) {
#pragma unroll
      for (int t = 0; t < KT; ++t)
#pragma unroll
        for (int r = 0; r < 16; ++r) s[t][r] = 0.0f;
      const uint8_t* k_at = sm.k[buf] + (32 * KT * kw + j) * kKeyPitch + 16 * h;
      bf16x8 kk[2][KT];
      auto read = [&](int c) {
#pragma unroll
        for (int t = 0; t < KT; ++t)
          kk[c & 1][t] = *(const bf16x8*)(k_at + 32 * t * kKeyPitch + 32 * c);
      };
      read(0);
#pragma unroll
      for (int c = 0; c < 8; ++c) {
        if (c + 1 < 8) read(c + 1);
        __builtin_amdgcn_sched_barrier(0);      // (an operand is on its way while one is used)
#pragma unroll
        for (int t = 0; t < KT; ++t)
          s[t] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kk[c & 1][t], qf[c], s[t], 0, 0, 0);
      }
    };
    auto sums = [&](int buf, float k_scale, float vf) {
      const float kf = k_scale * a.sc_log2;
      // V's scale as sig * 2^E (E = -126 for zeros and what is nearer to them, 0 for
      // infinities and NaN)
      const int ve = (int)(__float_as_uint(vf) >> 23 & 0xffu);
      const int ce = ve == 0xff ? 127 : min(max(ve, 1), 253);
      const float E = (float)(ce - 127);
      const float sig = vf * __uint_as_float((uint32_t)(254 - ce) << 23);
      float e[KT][16], sum;
      auto probs = [&](float c) {
        float part[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int t = 0; t < KT; ++t)
#pragma unroll
          for (int r = 0; r < 16; ++r) {
            e[t][r] = __builtin_amdgcn_exp2f(fmaf(s[t][r], kf, c));
            part[r % 4] += e[t][r];
          }
        sum = (part[0] + part[1]) + (part[2] + part[3]);
      };
      probs(E - M);
      float gap = M - ml - E, part = sum * __builtin_amdgcn_exp2f(gap);
      const bool fits = sum <= kWideLimit && part <= kWideLimit && gap <= kWideGap;
      if (__builtin_amdgcn_ballot_w64(!fits) != 0) {
        float mx = -INFINITY;
#pragma unroll
        for (int t = 0; t < KT; ++t)
#pragma unroll
          for (int r = 0; r < 16; ++r) mx = fmaxf(mx, s[t][r] * kf);
        mx = fmaxf(mx, __shfl_xor(mx, 32));
        const float ml_new = fmaxf(ml, mx), m_new = fmaxf(M, mx + E - kWideHead);
        const bool none = m_new == -INFINITY;      // (and ml_new with it)
        const float alpha = none ? 1.0f : __builtin_amdgcn_exp2f(M - m_new);
        l *= none ? 1.0f : __builtin_amdgcn_exp2f(ml - ml_new);
#pragma unroll
        for (int m = 0; m < 4; ++m) o[m] *= alpha;
        M = m_new;
        ml = ml_new;
        probs(none ? 0.0f : E - M);
        gap = none ? 0.0f : M - ml - E;
        part = sum * __builtin_amdgcn_exp2f(gap);
        if (__builtin_amdgcn_ballot_w64(gap > kWideGap) != 0) {
          part = 0.0f;
#pragma unroll
          for (int t = 0; t < KT; ++t)
#pragma unroll
            for (int r = 0; r < 16; ++r)
              part += __builtin_amdgcn_exp2f(fmaf(s[t][r], kf, none ? 0.0f : -ml));
        }
      }
      l += part;
      if (sig != 1.0f) {
#pragma unroll
        for (int t = 0; t < KT; ++t)
#pragma unroll
          for (int r = 0; r < 16; ++r) e[t][r] *= sig;
      }
      const uint8_t* v_at = sm.v[buf] + j * kDimPitch + 64 * KT * kw + 8 * h;
      uint2 vv[2][4][2];
      auto read = [&](int i) {
#pragma unroll
        for (int m = 0; m < 4; ++m) {
          vv[i & 1][m][0] = *(const uint2*)(v_at + 32 * m * kDimPitch + 32 * i);
          vv[i & 1][m][1] = *(const uint2*)(v_at + 32 * m * kDimPitch + 32 * i + 16);
        }
      };
      read(0);
#pragma unroll
      for (int i = 0; i < 2 * KT; ++i) {       // 16 keys each
        const float(&x)[16] = e[i / 2];
        const int r = 8 * (i & 1);
        const half8 p = __builtin_bit_cast(
            half8, make_uint4(pack_half2(x[r], x[r + 1]), pack_half2(x[r + 2], x[r + 3]),
                              pack_half2(x[r + 4], x[r + 5]), pack_half2(x[r + 6], x[r + 7])));
        if (i + 1 < 2 * KT) read(i + 1);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int m = 0; m < 4; ++m) {
          const uint2 lo = vv[i & 1][m][0], hi = vv[i & 1][m][1];
          o[m] = __builtin_amdgcn_mfma_f32_32x32x16_f16(
              __builtin_bit_cast(half8, make_uint4(lo.x, lo.y, hi.x, hi.y)), p, o[m], 0, 0, 0);
        }
      }
    };

    // While the matrix cores multiply a step's K, its successor's codes, asked for one
    // step earlier, are converted into the other buffer: that costs as much as the
    // step's softmax (a step 6200 cycles with it before the barrier, not beside).  Pages
    // are looked up two steps ahead, scales one.
    int p0 = page_of(number_of(st0, 0), st0, 0), p1 = page_of(number_of(st0, 1), st0, 1), buf = 0;
    int n0 = number_of(st0 + 1, 0), n1 = number_of(st0 + 1, 1);
    load(p0, p1);
    int mine = my_half ? p1 : p0;
    float ks = entry(k_scales, scale_at(mine)), vs = entry(v_scales, scale_at(mine));
    p0 = page_of(n0, st0 + 1, 0);
    p1 = page_of(n1, st0 + 1, 1);
    n0 = number_of(st0 + 2, 0);
    n1 = number_of(st0 + 2, 1);
    if (st0 < st1) {
      stage(0);
      load(p0, p1);
    }
    for (int st = st0; st < st1; ++st, buf ^= 1) {
      __syncthreads();      // (this step's codes are there; the other buffer has been read)
      const int next = my_half ? p1 : p0;
      const float ks_next = entry(k_scales, scale_at(next)), vs_next = entry(v_scales, scale_at(next));
      p0 = page_of(n0, st + 2, 0);
      p1 = page_of(n1, st + 2, 1);
      n0 = number_of(st + 3, 0);
      n1 = number_of(st + 3, 1);
      const bool early = wave < kWideWaves / 2;
      if (mine >= 0 && early) scores(buf);
      if (st + 1 < st1) {
        stage(buf ^ 1);
        load(p0, p1);
      }
      if (mine >= 0 && !early) scores(buf);
      if (mine >= 0) sums(buf, ks, vs);
      mine = next;
      ks = ks_next;
      vs = vs_next;
    }
    l += __shfl_xor(l, 32);
    // (2^(M - ml) may be past fp32 where its half is not)
    const float to_ml = M == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(0.5f * (M - ml));
#pragma unroll
    for (int m = 0; m < 4; ++m) o[m] = o[m] * to_ml * to_ml;
    M = ml;
    // the sums of the waves with the same rows, by halves
    float* const ex = (float*)&sm;
#pragma unroll
    for (int half = KW / 2; half > 0; half >>= 1) {
      __syncthreads();
      float* const to_wave = ex + ((kw - half) * RW + rw) * (66 * kWave) + lane;
      if (kw >= half && kw < 2 * half) {
        to_wave[0] = M;
        to_wave[kWave] = l;
#pragma unroll
        for (int m = 0; m < 4; ++m)
#pragma unroll
          for (int r = 0; r < 16; ++r) to_wave[(2 + 16 * m + r) * kWave] = o[m][r];
      }
      __syncthreads();
      if (kw < half) {
        const float* from = ex + (kw * RW + rw) * (66 * kWave) + lane;
        const float m2 = from[0], l2 = from[kWave], mm = fmaxf(M, m2);
        const float f = M == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(M - mm);
        const float f2 = m2 == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(m2 - mm);
        M = mm;
        l = l * f + l2 * f2;
#pragma unroll
        for (int m = 0; m < 4; ++m)
#pragma unroll
          for (int r = 0; r < 16; ++r) o[m][r] = o[m][r] * f + from[(2 + 16 * m + r) * kWave] * f2;
      }
    }
    __syncthreads();
    const int row = 32 * rw + j;
    if (kw == 0 && row0 + row < rows) {
      const int64_t pr = ((int64_t)q.item + item + worker) * kRowsOf + row;
      if (h == 0) x.wide_ml[pr] = Part{M, l};
      float* to_row = x.wide_o + pr * kHeadDim + 4 * h;
#pragma unroll
      for (int m = 0; m < 4; ++m)
#pragma unroll
        for (int r = 0; r < 4; ++r)
          *(float4*)(to_row + 32 * m + 8 * r) =
              make_float4(o[m][4 * r], o[m][4 * r + 1], o[m][4 * r + 2], o[m][4 * r + 3]);
    }
  }
}

// A workgroup's run of the groups' keys, then its waves' runs of the sequences' own.
// (Two launches instead: the second one's start, and the first one's uneven end, come
// on top.)
template <int FMT, int P, int RW, int RT>
__global__ __launch_bounds__(kWideThreads, 2) void shared_wide_kernel(SharedArgs x) {
  __shared__ WideSmem sm;
  wide_run<FMT, P, RW>(x, sm);
  // (where the runs are fewer than the waves: over the CUs, from the one without groups'
  // keys on)
  steps_run<FMT, P, RT>(x, __builtin_amdgcn_readfirstlane(threadIdx.x / kWave) * kWideWorkers +
                               kWideWorkers - 1 - (int)blockIdx.x);
}

// ----------------------------------------------------------------------------
// A row's parts: a wave, 16 lanes with eight dims each for every fourth part, the
// fours then joined in order.  A workgroup has 4 heads of a token.
// ----------------------------------------------------------------------------
constexpr int kJoinRows = kWaves;

struct RowParts {       // parts `first` .. `first` + n - 1 of a row, `pitch` rows apart
  const Part* ml;
  const float* o;
  int64_t first;
  int pitch, n;
};

__global__ __launch_bounds__(kThreads) void shared_join_kernel(SharedArgs x, int64_t unit0) {
  const AttendArgs& a = x.a;
  const int G = a.Hq / a.pg.Hkv, blocks = (a.Hq + kJoinRows - 1) / kJoinRows;
  const int64_t unit = unit0 + blockIdx.x;
  const int t = (int)(unit / blocks);
  const int head = (int)(unit % blocks) * kJoinRows +
                   __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  int s = 0;
  if (!a.tk.cu) {
    s = t / a.tk.each;
  } else {
    int hi = a.tk.S - 1;
    while (s < hi) {
      const int mid = (s + hi + 1) / 2;
      if (entry(a.tk.cu, mid) <= t) s = mid; else hi = mid - 1;
    }
  }
  const SeqInfo q = info_at(x.seqs, s);
  if (t < q.first || t >= q.first + q.n || entry(&x.totals->bad, 0)) return;
  if (head >= a.Hq) return;
  const int kvh = head / G, lane = threadIdx.x % kWave, d = lane % 16 * 8, stripe = lane / 16;
  // the parts of an item whose units are [begin, begin + whole): its workers' slots
  auto parts_of = [&](const Part* ml, const float* o, int tile_rows, int64_t unit, int item, int n,
                      int row, int whole, int64_t per) {
    const int tiles = (n * G + tile_rows - 1) / tile_rows, at = kvh * tiles + row / tile_rows;
    const int64_t begin = unit + (int64_t)at * whole;
    const int64_t w0 = begin / per, w1 = (begin + whole - 1) / per;
    return RowParts{ml, o, (item + at + w0) * tile_rows + row % tile_rows, tile_rows,
                    (int)(w1 - w0) + 1};
  };
  const int64_t keys = min((int64_t)max(entry(a.lengths, s), 0), (int64_t)a.pg.max_pages * a.pg.P);
  const int own_steps = (int)((max(keys - q.key0, (int64_t)0) + kKeys - 1) / kKeys);
  const int64_t steps_per = entry(&x.totals->steps_per, 0);
  const RowParts own = parts_of(a.part_ml, a.part_o, x.steps_rows, q.unit, q.item, q.n,
                                (t - q.first) * G + head % G, own_steps + kStepsCost, steps_per);
  RowParts common{};
  if (q.group >= 0) {
    const GroupInfo g = info_at(x.groups, q.group);
    const int row = (t - g.first) * G + head % G;
    const int64_t gkeys = (int64_t)g.pages * a.pg.P;
    if (t >= g.first && t < g.first + g.n)
      common = x.wide_rows
          ? parts_of(x.wide_ml, x.wide_o, x.wide_rows, g.unit, g.item, g.n, row,
                     (int)((gkeys + kWideKeys - 1) / kWideKeys) + entry(&x.totals->wide_cost, 0),
                     entry(&x.totals->wide_per, 0))
          : parts_of(a.part_ml, a.part_o, x.steps_rows, g.unit, g.item, g.n, row,
                     (int)(gkeys / kKeys) + kStepsCost, steps_per);
  }
  float m = -INFINITY, l = 0.0f, acc[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) acc[i] = 0.0f;
  auto add = [&](float m2, float l2, const float (&v)[8]) {
    const float mn = fmaxf(m, m2);
    const float f = m == mn ? 1.0f : __builtin_amdgcn_exp2f(m - mn);
    const float g = m2 == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(m2 - mn);
    l = l * f + l2 * g;
#pragma unroll
    for (int i = 0; i < 8; ++i) acc[i] = acc[i] * f + v[i] * g;
    m = mn;
  };
  constexpr int kAhead = 3;
  const int all = common.n + own.n;
  for (int p0 = stripe; p0 < all; p0 += 4 * kAhead) {
    Part ml[kAhead];
    float4 v[kAhead][2];
#pragma unroll
    for (int k = 0; k < kAhead; ++k) {
      const int p = min(p0 + 4 * k, all - 1);
      const RowParts& r = p < common.n ? common : own;
      const int64_t at = r.first + (int64_t)(p < common.n ? p : p - common.n) * r.pitch;
      ml[k] = r.ml[at];
      v[k][0] = *(const float4*)(r.o + at * kHeadDim + d);
      v[k][1] = *(const float4*)(r.o + at * kHeadDim + d + 4);
    }
#pragma unroll
    for (int k = 0; k < kAhead; ++k)
      if (p0 + 4 * k < all) {
        const float x[8] = {v[k][0].x, v[k][0].y, v[k][0].z, v[k][0].w,
                            v[k][1].x, v[k][1].y, v[k][1].z, v[k][1].w};
        add(ml[k].m, ml[k].l, x);
      }
  }
#pragma unroll
  for (int o = 16; o <= 32; o <<= 1) {
    const float m2 = __shfl_xor(m, o), l2 = __shfl_xor(l, o);
    float v[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = __shfl_xor(acc[i], o);
    add(m2, l2, v);
  }
  const float inv = l == 0.0f ? 0.0f : 1.0f / l;
  if (stripe == 0)
    *(uint4*)(a.o + ((int64_t)head * a.tk.T + t) * kHeadDim + d) =
        make_uint4(pack_bf16x2(acc[0] * inv, acc[1] * inv), pack_bf16x2(acc[2] * inv, acc[3] * inv),
                   pack_bf16x2(acc[4] * inv, acc[5] * inv), pack_bf16x2(acc[6] * inv, acc[7] * inv));
}

// ----------------------------------------------------------------------------
// Host side
// ----------------------------------------------------------------------------
struct SharedPlan {
  int wide_rows, rt, groups;       // workgroups of four waves that take the steps
  int64_t items, wide_items;
  bool fits;
  size_t at_groups, at_seqs, at_wide_ml, at_wide_o, at_ml, at_o, bytes;
};
SharedPlan shared_plan(int Hq, int n_tokens, int n_seqs, int n_groups, int max_pages,
                       const ei_cache_shape& c) {
  SharedPlan p{};
  const int64_t G = Hq / c.n_kv_heads, rows = n_tokens * G;
  // Rows of a group and a KV head on average: tiles in LDS from 33 on, of 128 rows from
  // 65 on.  Without, with 64, with 128, us a call: 8 groups of 4096 keys, 32 rows 44, 45,
  // 50; 48 rows 56, 51, 54; 96 rows 82, 77, 70; 4 groups of 16384, 64 rows 75, 56, 63; 96
  // rows 100, 87, 70; one group of 8192, 16 rows 26, 28, 28; 64 rows 35, 33, 33; 128 rows
  // 41, 37, 37.
  const int64_t of_group = n_groups ? rows / n_groups : 0;
  p.wide_rows = of_group > 64 ? 128 : of_group > 32 ? 64 : 0;
  p.rt = rows > (int64_t)kRows * n_seqs ||
                 (!p.wide_rows && n_groups && rows > (int64_t)kRows * n_groups) ? 2 : 1;
  const int64_t tile = kRows * p.rt, most_keys = (int64_t)max_pages * c.page_len;
  int64_t items = (rows / tile + n_seqs) * c.n_kv_heads;
  const int64_t cost = most_keys / kKeys + 1 + kStepsCost;
  int64_t wide_items = 0;
  if (p.wide_rows) wide_items = (rows / p.wide_rows + n_groups) * c.n_kv_heads;
  else items += (rows / tile + n_groups) * c.n_kv_heads;
  p.items = items;
  p.wide_items = wide_items;
  p.fits = items <= INT_MAX / 2 && wide_items <= INT_MAX / 2 && rows <= INT_MAX / 2;
  if (!p.fits) return p;
  const int64_t waves = items > INT64_MAX / cost ? INT64_MAX : items * cost / (kStepsLeast / 2) + 1;
  p.groups = (int)(waves / kWaves + 1 < kStepsGroups ? waves / kWaves + 1 : kStepsGroups);
  if (p.wide_rows) p.groups = kStepsGroups;      // (as many waves as shared_wide_kernel has)
  auto up = [](size_t n) { return (n + 255) / 256 * 256; };
  const size_t slots = ((size_t)items + (size_t)p.groups * kWaves) * tile;
  const size_t wide = p.wide_rows ? ((size_t)wide_items + kWideWorkers) * p.wide_rows : 0;
  p.at_groups = up(sizeof(Totals));
  p.at_seqs = p.at_groups + up(n_groups * sizeof(GroupInfo));
  p.at_wide_ml = p.at_seqs + up(n_seqs * sizeof(SeqInfo));
  p.at_wide_o = p.at_wide_ml + up(wide * sizeof(Part));
  p.at_ml = p.at_wide_o + wide * kHeadDim * sizeof(float);
  p.at_o = p.at_ml + up(slots * sizeof(Part));
  p.bytes = p.at_o + slots * kHeadDim * sizeof(float);
  return p;
}

template <int FMT, int P>
void launch_shared(const SharedPlan& pl, const SharedArgs& x, hipStream_t stream) {
  if (x.a.tk.S <= kFewThreads && x.n_groups <= kFewThreads)
    hipLaunchKernelGGL(shared_plan_few_kernel, dim3(1), dim3(kFewThreads), 0, stream, x);
  else
    hipLaunchKernelGGL(shared_plan_kernel, dim3(1), dim3(kPlanThreads), 0, stream, x);
#define EI_WIDE(RW, RT) \
  hipLaunchKernelGGL((shared_wide_kernel<FMT, P, RW, RT>), dim3(kWideWorkers), dim3(kWideThreads), 0, stream, x)
#define EI_STEPS(RT) \
  hipLaunchKernelGGL((shared_steps_kernel<FMT, P, RT>), dim3((unsigned)pl.groups), dim3(kThreads), 0, stream, x)
  if (pl.wide_rows == 128) {
    if (pl.rt == 1) EI_WIDE(4, 1); else EI_WIDE(4, 2);
  } else if (pl.wide_rows == 64) {
    if (pl.rt == 1) EI_WIDE(2, 1); else EI_WIDE(2, 2);
  } else {
    if (pl.rt == 1) EI_STEPS(1); else EI_STEPS(2);
  }
#undef EI_WIDE
#undef EI_STEPS
  const int64_t units = (int64_t)x.a.tk.T * ((x.a.Hq + kJoinRows - 1) / kJoinRows);
  for (int64_t u = 0; u < units; u += kMaxGrid)
    hipLaunchKernelGGL(shared_join_kernel, dim3(launch_grid(units - u)), dim3(kThreads), 0, stream,
                       x, u);
}

}  // namespace
}  // namespace ei

extern "C" {

size_t ei_cache_attn_shared_workspace_bytes(int32_t n_q_heads, int32_t n_tokens, int32_t n_seqs,
                                            int32_t n_groups, int32_t max_pages,
                                            ei_cache_shape shape) {
  if (ei::check_shape(shape) != EI_OK || n_q_heads <= 0 || n_q_heads % shape.n_kv_heads ||
      n_tokens <= 0 || n_seqs <= 0 || n_groups < 0 || max_pages < 0)
    return 0;
  if ((int64_t)n_tokens * n_q_heads > INT_MAX || (int64_t)max_pages * shape.page_len > INT_MAX)
    return 0;
  return ei::shared_plan(n_q_heads, n_tokens, n_seqs, n_groups, max_pages, shape).bytes;
}

ei_status ei_cache_attn_shared(const uint16_t* q, int32_t n_q_heads, int32_t n_tokens,
                               const int32_t* cu_seqlens, int32_t n_seqs, const int32_t* lengths,
                               const int32_t* page_table, int32_t max_pages,
                               const int32_t* group_seqs, const int32_t* shared_pages,
                               int32_t n_groups, ei_cache_shape shape, ei_cache_pages pages,
                               float softmax_scale, uint16_t* o, void* workspace,
                               size_t workspace_bytes, void* stream) {
  ei_status st = ei::check_shape(shape);
  if (st != EI_OK && st != EI_ERR_UNSUPPORTED) return st;
  if (n_q_heads <= 0 || n_q_heads % shape.n_kv_heads || n_groups < 0) return EI_ERR_SHAPE;
  if (!(softmax_scale > 0.0f && softmax_scale <= 3.402823466e38f)) return EI_ERR_SHAPE;
  if (st != EI_OK) return st;
  if ((st = ei::check_tokens(n_tokens, cu_seqlens, n_seqs, max_pages)) != EI_OK) return st;
  if ((int64_t)n_tokens * n_q_heads > INT_MAX || (int64_t)max_pages * shape.page_len > INT_MAX)
    return EI_ERR_SHAPE;
  if (n_tokens == 0 || n_seqs == 0) return EI_OK;
  const ei::SharedPlan pl = ei::shared_plan(n_q_heads, n_tokens, n_seqs, n_groups, max_pages, shape);
  if (!pl.fits) return EI_ERR_SHAPE;
  if (!q || !o || !lengths || (!page_table && max_pages > 0)) return EI_ERR_NULL;
  if (n_groups > 0 && (!group_seqs || !shared_pages)) return EI_ERR_NULL;
  if ((st = ei::check_pages(shape, pages)) != EI_OK) return st;
  if (!ei::aligned(q, 16) || !ei::aligned(o, 16) || !ei::aligned(lengths, 4) ||
      !ei::aligned(page_table, 4) || !ei::aligned(cu_seqlens, 4) || !ei::aligned(group_seqs, 4) ||
      !ei::aligned(shared_pages, 4))
    return EI_ERR_UNSUPPORTED;
  if (!workspace || workspace_bytes < pl.bytes) return EI_ERR_WORKSPACE;
  if (!ei::aligned(workspace, 16)) return EI_ERR_UNSUPPORTED;
  char* ws = (char*)workspace;
  const ei::Tokens tk{cu_seqlens, n_tokens, n_seqs, n_tokens / n_seqs};
  const ei::Pages pg = ei::pages_of(shape, pages, page_table, max_pages);
  const ei::AttendArgs a{q, o, tk, lengths, pg, n_q_heads,
                         (float)((double)softmax_scale * 1.4426950408889634),
                         (ei::Part*)(ws + pl.at_ml), (float*)(ws + pl.at_o), nullptr};
  const ei::SharedArgs x{a, group_seqs, shared_pages, n_groups, pl.wide_rows, ei::kRows * pl.rt,
                         pl.groups * ei::kWaves, pl.wide_items, pl.items, (ei::Totals*)ws,
                         (ei::GroupInfo*)(ws + pl.at_groups), (ei::SeqInfo*)(ws + pl.at_seqs),
                         (ei::Part*)(ws + pl.at_wide_ml), (float*)(ws + pl.at_wide_o)};
  hipStream_t s0 = (hipStream_t)stream;
  if (shape.format == EI_CACHE_E4M3) {
    if (shape.page_len == 64) ei::launch_shared<EI_CACHE_E4M3, 64>(pl, x, s0);
    else ei::launch_shared<EI_CACHE_E4M3, 128>(pl, x, s0);
  } else {
    if (shape.page_len == 64) ei::launch_shared<EI_CACHE_INT8, 64>(pl, x, s0);
    else ei::launch_shared<EI_CACHE_INT8, 128>(pl, x, s0);
  }
  return ei::from_hip(hipGetLastError());
}

}  // extern "C"
