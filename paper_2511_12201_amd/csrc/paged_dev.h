// Device code that the attention kernels on a paged cache share: the rows of a pair, and how the work is cut.
//
// An item is up to tm consecutive query rows of a pair (sequence, KV head); it walks the cache rows that its last query row
// sees, in units of `unit` rows.  All units of all items, item after item, are one line that is cut into as many equal spans as
// there are workgroups: every workgroup does the same amount of work whatever the lengths are, and the lengths stay on the
// device.  A workgroup that has all units of an item writes its output rows; otherwise it leaves a partial state (maximum, sum,
// weighted rows) in one of its two slots (its span's first item: slot 2 w, another one: it can only be the last: 2 w + 1), and
// paged_combine_kernel joins the slots of an item in the order of the units: equal inputs, equal bits.  The workgroup that has an
// item's first unit writes down which spans share it.
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
  __device__ __forceinline__ PairView(const AttnParams& p, int pair_) : pair(pair_) {
    b = pair / p.c.Hkv;
    g = pair - b * p.c.Hkv;
    cnt = clampi(p.new_cnt[b], 0, p.c.n_new);
    end = clampi(p.row_end[pair], 0, rows_cap(p.pg));
    M = cnt * p.c.G;
  }
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

__device__ __forceinline__ int item_units(const AttnParams& p, int item) {
  const PairView w(p, item / p.tiles_per_pair);
  const int r0 = item % p.tiles_per_pair * p.tm;
  if (r0 >= w.M) return 0;
  const int keys = w.visible(p, (min(r0 + p.tm, w.M) - 1) / p.c.G);
  return max(1, cdiv(keys, p.unit));
}

// Spans of the line of units: workgroup w of n has [start(w), start(w + 1)).
struct Spans {
  u64 total;
  int n;
  __device__ __forceinline__ u64 start(int w) const { return total * (u64)w / (u64)n; }
  __device__ __forceinline__ int owner(u64 at) const { return (int)(((at + 1) * (u64)n + total - 1) / total) - 1; }
};

struct Scan {
  u64 wave[16];
  u64 at;
  int item;
};

// Every thread: units of its run of consecutive items; returns the units in front of the run, total of all.
template <int THREADS>
__device__ __forceinline__ u64 scan_items(const AttnParams& p, Scan& s, int& first, int& per, u64& own, Spans& sp) {
  per = cdiv(p.n_items, THREADS);
  first = min((int)threadIdx.x * per, p.n_items);
  own = 0;
  for (int i = first; i < min(first + per, p.n_items); ++i) own += item_units(p, i);
  const u64 inc = wave_scan(own);
  if ((threadIdx.x & 63) == 63) s.wave[threadIdx.x >> 6] = inc;
  __syncthreads();
  u64 before = inc - own;
  sp.total = 0;
#pragma unroll
  for (int v = 0; v < THREADS / 64; ++v) {
    if (v < (int)(threadIdx.x >> 6)) before += s.wave[v];
    sp.total += s.wave[v];
  }
  sp.n = (int)max(1ull, min((u64)p.n_wgs, sp.total / p.min_share));
  return before;
}

struct Segment {
  int item, pair, r0, u0, u1, slot;
  bool whole;
};

// Walks a workgroup's span: f(segment) for its part of every item in it.  All threads call it.
// Neighbouring spans go to one XCD (workgroup b runs on XCD b % 8): they share a pair, and often the place in it.
__device__ __forceinline__ int span_of(int b, int n) {
  const int each = n / 8;
  return b < each * 8 ? b % 8 * each + b / 8 : b;
}

template <int THREADS, typename F>
__device__ __forceinline__ void for_segments(const AttnParams& p, Scan& s, F f) {
  int first, per;
  u64 own;
  Spans sp;
  u64 at = scan_items<THREADS>(p, s, first, per, own, sp);
  if (sp.total == 0 || (int)blockIdx.x >= sp.n) return;
  const int w = span_of(blockIdx.x, sp.n);
  const u64 begin = sp.start(w), end = sp.start(w + 1);
  if (begin >= at && begin < at + own) {
    int i = first;
    for (;; ++i) {
      const int n = item_units(p, i);
      if (begin < at + n) break;
      at += n;
    }
    s.item = i;
    s.at = begin - at;
  }
  __syncthreads();
  int item = __builtin_amdgcn_readfirstlane(s.item), off = __builtin_amdgcn_readfirstlane((int)s.at);
  for (u64 pos = begin; pos < end; ++item) {
    const int units = __builtin_amdgcn_readfirstlane(item_units(p, item));
    if (units == 0) continue;
    const int take = (int)min((u64)(units - off), end - pos);
    Segment seg;
    seg.item = item;
    seg.pair = item / p.tiles_per_pair;
    seg.r0 = item % p.tiles_per_pair * p.tm;
    seg.u0 = off;
    seg.u1 = off + take;
    seg.slot = 2 * w + (pos == begin ? 0 : 1);
    seg.whole = off == 0 && take == units;
    if (off == 0 && threadIdx.x == 0)                    // who joins the item finds its slots here (whole: first span = last)
      p.joins[item] = int4{w, seg.whole ? w : sp.owner(pos + units - 1), seg.slot, 0};
    f(seg);
    pos += take;
    off = 0;
  }
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
