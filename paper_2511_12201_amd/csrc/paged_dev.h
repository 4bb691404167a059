// Device code that the attention kernels on a paged cache share: the rows of a pair, and how the work is cut.
//
// An item is up to tm consecutive query rows of a pair (sequence, KV head); it walks the cache rows that its last query row
// sees, in units of `unit` rows, and counts `over` units more for what it costs to take it up (2048 tokens on as many rows: the
// workgroup with the first, short items of a pair had six of them and took 97 us where the others took 50).  All units of all items,
// item after item, are one line that is cut into as many equal spans as there are workgroups: every workgroup does the same amount of
// work whatever the lengths are, and the lengths stay on the device.  A workgroup that has all units of an item writes its output
// rows; otherwise it leaves a partial state (maximum, sum, weighted rows) in one of its two slots (its span's first item: slot 2 w,
// another one: it can only be the last: 2 w + 1), and the paged_combine kernels join the slots of an item in the order of the units:
// equal inputs, equal bits.  The workgroup that has an item's first unit writes down which spans share it.
#pragma once

#include "paged.h"

namespace omni {

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;
typedef unsigned long long u64;

struct AttnParams {
  const void* Q;
  void* O;
  float* lse;
  Pages pg;
  const int *row_end, *new_cnt;
  const float* acc_in;
  float* acc_out;
  Chunk c;
  int tm, unit, tiles_per_pair, n_items;   // items: tiles_per_pair of every pair
  int over;                                // units that stand for what taking up an item costs
  int n_wgs, min_share;                    // workgroups, units that a span has at least
  float* part_o;                           // [2 n_wgs, tm, D]
  float* part_ml;                          // [2 n_wgs, tm, 2]: maximum (times scale log2 e), sum
  float* logits;                           // [pairs, cap / 32, M of a full chunk, 32] scores times scale log2 e, -inf: not seen
  int4* joins;                             // [n_items] of items that are split: first span, last span, slot of the first
  int w_blocks;                            // the pass for the weights: blocks of a pair,
  int4* w_joins;                           // [pairs, w_blocks] as joins,
  float* w_part;                           // slots of parts
};

// Query rows and cache rows of a pair: row r is token r / G, head r % G of the group; how many rows a query row sees.
struct PairView {
  int pair, b, g, cnt, end, M;
  __device__ __forceinline__ PairView(const AttnParams& p, int pair_, int cnt_, int end_) : pair(pair_), cnt(cnt_), end(end_) {
    b = pair / p.c.Hkv;
    g = pair - b * p.c.Hkv;
    M = cnt * p.c.G;
  }
  __device__ __forceinline__ PairView(const AttnParams& p, int pair_)
      : PairView(p, pair_, clampi(p.new_cnt[pair_ / p.c.Hkv], 0, p.c.n_new), clampi(p.row_end[pair_], 0, rows_cap(p.pg))) {}
  // the view of a pair that the whole wavefront works on: addresses and bounds made of it stay in scalar registers
  __device__ static __forceinline__ PairView uniform(const AttnParams& p, int pair) {
    PairView w(p, pair);
    w.cnt = __builtin_amdgcn_readfirstlane(w.cnt);
    w.end = __builtin_amdgcn_readfirstlane(w.end);
    w.M = __builtin_amdgcn_readfirstlane(w.M);
    return w;
  }
  __device__ __forceinline__ int visible(const AttnParams& p, int t) const { return p.c.causal ? max(end - cnt + t + 1, 0) : end; }
};

// Units of an item that starts at query row r0: what the workgroup that takes a part of it pays besides the tiles, then the tiles.
__device__ __forceinline__ int item_units(const AttnParams& p, const PairView& w, int r0) {
  if (r0 >= w.M) return 0;
  const int keys = w.visible(p, (min(r0 + p.tm, w.M) - 1) / p.c.G);
  return p.over + max(1, cdiv(keys, p.unit));
}
__device__ __forceinline__ int item_units(const AttnParams& p, int item) {
  const int pair = item / p.tiles_per_pair;
  return item_units(p, PairView(p, pair), (item - pair * p.tiles_per_pair) * p.tm);
}

__device__ __forceinline__ u64 wave_uniform(u64 v) {
  return ((u64)(unsigned)__builtin_amdgcn_readfirstlane((int)(v >> 32)) << 32) | (unsigned)__builtin_amdgcn_readfirstlane((int)v);
}

// Spans of the line of units: workgroup w of n has [start(w), start(w + 1)), the first total % n one unit more than the others.
struct Spans {
  u64 total, each, more;
  int n;
  __device__ __forceinline__ void cut(u64 units, int wgs, int min_share) {
    total = units = wave_uniform(units);
    n = (int)max(1ull, min((u64)wgs, (units >> 32) == 0 ? (u64)((unsigned)units / (unsigned)min_share) : (u64)wgs));
    each = (units >> 32) == 0 ? (u64)((unsigned)units / (unsigned)n) : units / n;
    more = units - each * n;
  }
  __device__ __forceinline__ u64 start(int w) const { return each * w + min((u64)w, more); }
  __device__ __forceinline__ int owner(u64 at) const {
    const u64 long_ones = more * (each + 1);
    if (total >> 32) return (int)(at < long_ones ? at / (each + 1) : more + (at - long_ones) / each);
    return at < long_ones ? (int)((unsigned)at / (unsigned)(each + 1)) : (int)more + (int)((unsigned)(at - long_ones) / (unsigned)each);
  }
};

struct Scan {
  u64 wave[16];
  u64 at, at_last;
  int item, last;
};

// Neighbouring spans go to one XCD (workgroup b runs on XCD b % 8): they share a pair, and often the place in it.
__device__ __forceinline__ int span_of(int b, int n) {
  const int each = n / 8;
  return b < each * 8 ? b % 8 * each + b / 8 : b;
}

struct Segment {
  PairView w;
  int item, r0, u0, u1, slot;
  bool whole;
  u64 total;                                             // units of all items
};

// Walks a workgroup's span: f(segment) for its part of every item in it.  All threads call it.  Up to 64 items (a few sequences of
// few tokens, where the start counts) every wavefront finds its place by itself, one item a lane that keeps the item's lengths (loaded
// anew for every use they cost 2 of the 7 us of a token on 4109 rows); more are added up by the workgroup.
template <int THREADS, typename F>
__device__ __forceinline__ void for_segments(const AttnParams& p, Scan& s, F f) {
  Spans sp;
  u64 begin, end, at_item, at_last;                      // the span, where its first and its last item begin
  int item, last, w;
  int lane_cnt = 0, lane_end = 0;
  if (__builtin_expect(p.n_items <= 64, true)) {
    int mine = 0;
    if (lane_id() < p.n_items) {
      const int pair = lane_id() / p.tiles_per_pair;
      const PairView v(p, pair);
      mine = item_units(p, v, (lane_id() - pair * p.tiles_per_pair) * p.tm);
      lane_cnt = v.cnt;
      lane_end = v.end;
    }
    const u64 inc = wave_scan((u64)mine);
    sp.cut(__shfl(inc, 63, 64), p.n_wgs, p.min_share);
    if (sp.total == 0 || (int)blockIdx.x >= sp.n) return;
    w = span_of(blockIdx.x, sp.n);
    begin = sp.start(w);
    end = sp.start(w + 1);
    item = __ffsll((unsigned long long)__ballot(inc > begin)) - 1;
    last = __ffsll((unsigned long long)__ballot(inc >= end)) - 1;
    at_item = __shfl(inc - mine, item, 64);
    at_last = __shfl(inc - mine, last, 64);
  } else {
    const int per = cdiv(p.n_items, THREADS), first = min((int)threadIdx.x * per, p.n_items);
    u64 own = 0;
    for (int i = first; i < min(first + per, p.n_items); ++i) own += item_units(p, i);
    const u64 inc = wave_scan(own);
    if ((threadIdx.x & 63) == 63) s.wave[threadIdx.x >> 6] = inc;
    __syncthreads();
    u64 at = inc - own, total = 0;
#pragma unroll
    for (int v = 0; v < THREADS / 64; ++v) {
      if (v < (int)(threadIdx.x >> 6)) at += s.wave[v];
      total += s.wave[v];
    }
    sp.cut(total, p.n_wgs, p.min_share);
    if (sp.total == 0 || (int)blockIdx.x >= sp.n) return;
    w = span_of(blockIdx.x, sp.n);
    begin = sp.start(w);
    end = sp.start(w + 1);
    if (begin < at + own && end > at) {
      for (int i = first; at < end && i < min(first + per, p.n_items); ++i) {
        const int n = item_units(p, i);
        if (begin >= at && begin < at + n) {
          s.item = i;
          s.at = at;
        }
        if (end > at && end <= at + n) {
          s.last = i;
          s.at_last = at;
        }
        at += n;
      }
    }
    __syncthreads();
    item = s.item;
    last = s.last;
    at_item = s.at;
    at_last = s.at_last;
  }
  // The part of the last item first, then the others in their order: the parts that begin with an item's first rows, then those that
  // end with its last, so that neighbouring workgroups, which are on one XCD, walk the rows of a pair side by side whatever the spans
  // are, and a row comes from its L2 for all but the first of them (2048 tokens on 65536 rows: 0.8 GB from beyond the L2s where items
  // in their order take 7.0, and 1684 us for 1712).
  item = __builtin_amdgcn_readfirstlane(item);
  last = __builtin_amdgcn_readfirstlane(last);
  at_item = wave_uniform(at_item);
  at_last = wave_uniform(at_last);
  for (int next = item < last ? last : item; next >= 0;) {
    const int it = next, pair = it / p.tiles_per_pair, r0 = (it - pair * p.tiles_per_pair) * p.tm;
    const PairView view = p.n_items <= 64 ? PairView(p, pair, __builtin_amdgcn_readlane(lane_cnt, it & 63), __builtin_amdgcn_readlane(lane_end, it & 63))
                                          : PairView::uniform(p, pair);
    const int units = __builtin_amdgcn_readfirstlane(item_units(p, view, r0));
    const u64 at = it == last ? at_last : at_item;
    if (it == last) {
      next = item < last ? item : -1;
    } else {
      at_item += units;
      next = it + 1 < last ? it + 1 : -1;
    }
    if (units == 0) continue;
    const int from = at < begin ? (int)(begin - at) : 0, to = (int)min((u64)units, end - at);
    Segment seg{view, it, r0, max(from - p.over, 0), to - p.over, 2 * w + (at <= begin ? 0 : 1), false, sp.total};
    seg.whole = seg.u0 == 0 && to == units;
    if (seg.u1 > seg.u0) {
      if (seg.u0 == 0 && threadIdx.x == 0)               // who joins the item finds its slots here (whole: first span = last)
        p.joins[it] = int4{w, seg.whole ? w : sp.owner(at + units - 1), seg.slot, 0};
      f(seg);
    }
  }
}

// S^T = K Q^T of 32 cache rows and 32 query rows in fp32.  A 32x32x2 instruction adds two products to every score, element e of the lane
// halves' elements [h D/2, (h + 1) D/2).  A score is a sum of sums of 32 products: one chain of D/2 additions rounds as often at the
// size of the whole (one token on 3370 rows of 128 elements: 1.2e-6 of the output's norm, so 5.3e-7; 256 tokens on 8192 rows 263 / 268 us,
// with weights 421 / 436).  Attention and weights form their
// scores here, so that a weight and the log-sum-exp that it is taken against are of the same scores.
//   operands(e, k, q): elements e .. e + 3 of the lane's half
template <int D, typename F>
__device__ __forceinline__ f32x16 scores_f32(F operands) {
  constexpr int kChain = 16;
  f32x16 total, part;
#pragma unroll
  for (int e0 = 0; e0 < D / 2; e0 += kChain) {
#pragma unroll
    for (int i = 0; i < 16; ++i) part[i] = 0.f;
#pragma unroll
    for (int e = e0; e < e0 + kChain; e += 4) {
      f32x4 k, q;
      operands(e, k, q);
#pragma unroll
      for (int x = 0; x < 4; ++x) part = __builtin_amdgcn_mfma_f32_32x32x2f32(k[x], q[x], part, 0, 0, 0);
    }
#pragma unroll
    for (int i = 0; i < 16; ++i) total[i] = e0 ? total[i] + part[i] : part[i];
  }
  return total;
}

// Output row r of a pair and its place in the log-sum-exps.
__device__ __forceinline__ long long out_row(const AttnParams& p, const PairView& w, int r, long long& at_lse) {
  const int t = r / p.c.G, head = w.g * p.c.G + r % p.c.G;
  at_lse = ((long long)w.b * p.c.Hq + head) * p.c.n_new + t;
  return w.b * p.c.qs[0] + head * p.c.qs[1] + (long long)t * p.c.qs[2];
}

// paged_attn.hip
int launch_combine(const AttnParams& p, int dtype, hipStream_t st);
// paged_f32.hip
int launch_attn_f32(const AttnParams& p, hipStream_t st);
// paged_weights.hip
int launch_weights(const AttnParams& p, int dtype, hipStream_t st);
struct WeightPlan {
  int n_wgs, blocks;
  size_t part_floats;
};
WeightPlan weight_plan(int dtype, int cap);

}  // namespace omni
