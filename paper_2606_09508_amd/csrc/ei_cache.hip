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
#include "ei_attend.h"

namespace ei {
namespace {

constexpr int kThreads = 256;
constexpr int kWaves = kThreads / kWave;
constexpr int kRows = 16;      // of a tile
constexpr int kKeys = 32;      // of a step
static_assert(kThreads == kAttendThreads && kRows == kAttendRows && kKeys == kAttendKeys,
              "as the code that they share takes them");

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
