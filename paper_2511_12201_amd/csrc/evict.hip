// Eviction from a paged cache by accumulated attention weight (omni_paged_evict).
//
// Per (sequence, KV head) pair the rows are ranked by a 32-bit key (spared rows above every weight, the weights in order, NaN as
// -inf) and the `keep` largest stay, equal keys by lowest row.  The key at the cut is found by histograms in LDS of 11 bits
// of the keys at a time; then the rows are counted in order, which splits the ties and numbers the holes and the rows that move into
// them.  Rows are only copied where they have to: a row that stays in front of the new end stays where it is.
//
// The selection has to read 8 bytes a row, the moves 4 rows' bytes each; what bounds a small call is the chain of dependent steps.
//  * Up to 16384 rows a pair (evict_small_kernel): one workgroup a pair, its keys in registers throughout, one launch and one for
//    the moves; where a pair can have few moves the workgroup makes them itself and the second launch is left out.  16 of 8192 rows,
//    32 pairs: 9.5 us, of which 2 are the rows' loads and 1.3 the moves (three fixed digits, rows in the order of the threads and
//    what is counted in that order by ballots: 14).
//  * More: the pair's rows in front of the new end and those behind it are cut into chunks, a workgroup each: three launches for
//    the digits (every chunk leaves its histogram, the next launch finds the bin), one for the lists, one for the moves.  98304 of
//    131072 rows leave, 8 pairs: 5.2 + 6.4 + 6.1 + 10.2 + 39 us, the last at the rate of a copy.
#include <algorithm>

#include "evict_cut.h"
#include "paged.h"

namespace omni {

namespace {

constexpr int kSmallRows = 16384, kSmallThreads = 1024;
constexpr int kFewMoves = 256;                 // moves that the workgroup of a pair makes itself
constexpr int kBins = 2048;
constexpr int kChunks = 40, kChunkThreads = 512, kChunkRows = 8;     // 38 whole chunks of at most 4096 rows: 155k rows in one round

struct EvictParams {
  Pages pg;
  int Hkv, row_bytes, budget, n_sink, n_recent, move_here;
  const int *seq_len, *row_end, *row_pos;
  const float* acc;
  int *row_cnt, *pos_out;
  float* acc_out;
  int* moves;                    // [pairs]
  int2* list;                    // [pairs, cap / 2] (from, to)
  int *hist, *coarse, *above;    // many rows: [3][pairs, kChunks, kBins], [3][pairs, kChunks, 64], [pairs, kChunks]
  int* cut;                      // [pairs, 4] digits found and rows wanted of the last one
};

__device__ __forceinline__ unsigned rank_key(float acc, bool spared) {
  if (spared) return 0xffffffffu;
  return acc != acc ? float_key(-INFINITY) : float_key(acc + 0.f);       // -0 and 0 are one weight
}

// The rows of a pair.
struct PairRows {
  int cap, n, keep, recent, n_sink;
  const int* pos;
  const float* acc;
  int* pos_out;
  float* acc_out;
  int2* list;
  __device__ __forceinline__ PairRows(const EvictParams& p, int pair) {
    cap = rows_cap(p.pg);
    n = clampi(p.row_end[pair], 0, cap);
    keep = min(n, p.budget);
    recent = (int)std::max((long long)p.seq_len[pair / p.Hkv] - p.n_recent, -(1ll << 31));
    n_sink = p.n_sink;
    const long long at = (long long)pair * cap;
    pos = p.row_pos + at;
    acc = p.acc + at;
    pos_out = p.pos_out + at;
    acc_out = p.acc_out + at;
    list = p.list + (long long)pair * (cap / 2);
  }
  __device__ __forceinline__ unsigned key(float a, int q) const { return rank_key(a, q < n_sink || q >= recent); }
};

// digit 0, 1, 2 of a key, from the top: 11, 11 and 10 bits
__device__ __forceinline__ int digit_of(unsigned key, int d) { return d == 0 ? key >> 21 : d == 1 ? key >> 10 & 2047 : key & 1023; }
__device__ __forceinline__ bool same_above(unsigned key, unsigned prefix, int d) { return d == 0 || (d == 1 ? (key ^ prefix) >> 21 : (key ^ prefix) >> 10) == 0; }
__device__ __forceinline__ unsigned with_digit(unsigned prefix, int bin, int d) { return prefix | (unsigned)bin << (d == 0 ? 21 : d == 1 ? 10 : 0); }

// One key a lane into the histogram; lanes that all meet in one bin (weights that are all zero) add once.
__device__ __forceinline__ void count_key(int* hist, int bin, bool counts) {
  const unsigned long long who = __ballot(counts);
  if (who == 0) return;
  const int first = __builtin_amdgcn_readlane(bin, __ffsll(who) - 1);
  if (__ballot(counts && bin != first) == 0) {
    if (lane_id() == 0) atomicAdd(&hist[first], __popcll(who));
  } else if (counts) {
    atomicAdd(&hist[bin], 1);
  }
}

// Largest of the wavefront's values, in every lane.
__device__ __forceinline__ unsigned wave_umax(unsigned v) {
  v = max(v, dpp_or_zero<0x111, 0xf>(v));
  v = max(v, dpp_or_zero<0x112, 0xf>(v));
  v = max(v, dpp_or_zero<0x114, 0xf>(v));
  v = max(v, dpp_or_zero<0x118, 0xf>(v));
  v = max(v, dpp_or_zero<0x142, 0xa>(v));
  v = max(v, dpp_or_zero<0x143, 0xc>(v));
  return (unsigned)__builtin_amdgcn_readlane((int)v, 63);
}

// From a histogram in LDS; all threads of evict_small_kernel call it.
__device__ __forceinline__ Found find_bin(const int* hist, int need, int* wave_sums, int* out) {
  constexpr int PER = kBins / kSmallThreads, kWaves = kSmallThreads / 64;
  int own = 0, h[PER];
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    h[i] = hist[kBins - 1 - ((int)threadIdx.x * PER + i)];       // from the largest key down
    own += h[i];
  }
  const int inc = (int)wave_scan((unsigned)own), wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
  if (lane_id() == 63) wave_sums[wave] = inc;
  __syncthreads();
  const int sums = (int)wave_scan((unsigned)(lane_id() < kWaves ? wave_sums[lane_id()] : 0));
  int before = inc - own + (wave ? __builtin_amdgcn_readlane(sums, wave - 1) : 0);
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    if (before < need && need <= before + h[i]) {
      out[0] = kBins - 1 - ((int)threadIdx.x * PER + i);
      out[1] = need - before;
      out[2] = h[i];
    }
    before += h[i];
  }
  __syncthreads();
  return Found{out[0], out[1], out[2]};
}

// K and V of moved rows and what they carry; LANES lanes a row.
template <int LANES, typename LIST>
__device__ __forceinline__ void move_rows(const EvictParams& p, const PairRows& w, const LIST& list, int pair, int moves, int first, int step, int lane) {
  const int per = p.row_bytes / 16;
  for (int i = first; i < moves; i += step) {
    const int2 m = list[i];
    if (lane == 0) {
      w.pos_out[m.y] = w.pos[m.x];                       // rows behind `keep` are never written: in place is as good
      w.acc_out[m.y] = w.acc[m.x];
    }
    const int from = pool_row(p.pg, pair, m.x), to = pool_row(p.pg, pair, m.y);
    if (from < 0 || to < 0) continue;
    for (int c = lane; c < per; c += LANES) {
      // nobody reads them there again (131072 rows to 32768: 76.4 / 72.6 us)
      const u32x4 k = __builtin_nontemporal_load(static_cast<const u32x4*>(p.pg.K) + (long long)from * per + c);
      const u32x4 v = __builtin_nontemporal_load(static_cast<const u32x4*>(p.pg.V) + (long long)from * per + c);
      static_cast<u32x4*>(p.pg.K)[(long long)to * per + c] = k;
      static_cast<u32x4*>(p.pg.V)[(long long)to * per + c] = v;
    }
  }
}

// ------------------------------------------------------------------ up to kSmallRows rows a pair.  grid: pairs

typedef int i32x4_4 __attribute__((ext_vector_type(4), aligned(4)));
typedef float f32x4_4 __attribute__((ext_vector_type(4), aligned(4)));

// Sum of the values in front of a thread's, and of all; all threads of evict_small_kernel call it.
struct Before {
  unsigned before, all;
};
__device__ __forceinline__ Before scan_threads(unsigned v, int wave, unsigned* sums) {
  constexpr int kWaves = kSmallThreads / 64;
  const unsigned inc = wave_scan(v);
  if (lane_id() == 63) sums[wave] = inc;
  __syncthreads();
  const int s = (int)wave_scan(lane_id() < kWaves ? sums[lane_id()] : 0u);
  return Before{inc - v + (wave ? (unsigned)__builtin_amdgcn_readlane(s, wave - 1) : 0u), (unsigned)__builtin_amdgcn_readlane(s, kWaves - 1)};
}

// R neighbouring rows a thread: what has to be counted in the order of the rows are bits of one register, and one sum over the threads.
template <int R>
__global__ __launch_bounds__(kSmallThreads) void evict_small_kernel(EvictParams p) {
  __shared__ int hist[3][kBins];
  __shared__ int sums[kSmallThreads / 64], out[3];
  __shared__ unsigned tie_sums[kSmallThreads / 64], move_sums[kSmallThreads / 64];
  __shared__ int2 few[kFewMoves];                        // the list of the moves, where the workgroup makes them itself
  __shared__ unsigned long long cand[kRanked], bound;
  __shared__ int n_cand;
  __shared__ unsigned ends[2][2];                        // of the keys of a bin: the largest, and of their complements
  const int pair = blockIdx.x, tid = threadIdx.x, lane = lane_id(), wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const PairRows w(p, pair);
  const int j0 = tid * R;
  auto bits = [&](int rows) { return (1u << clampi(rows - j0, 0, R)) - 1; };
  const unsigned live = bits(w.n), front = bits(w.keep);
  unsigned key[R];
  int pos[R];
  float acc[R];
#pragma unroll
  for (int k = 0; k < R; k += 4) {
    if (j0 + k + 4 <= w.n) {
      const i32x4_4 q = *reinterpret_cast<const i32x4_4*>(w.pos + j0 + k);
      const f32x4_4 a = *reinterpret_cast<const f32x4_4*>(w.acc + j0 + k);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        pos[k + e] = q[e];
        acc[k + e] = a[e];
      }
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        pos[k + e] = live >> (k + e) & 1u ? w.pos[j0 + k + e] : 0;
        acc[k + e] = live >> (k + e) & 1u ? w.acc[j0 + k + e] : 0.f;
      }
    }
  }
  for (int i = tid; i < 3 * kBins; i += kSmallThreads) hist[0][i] = 0;
  if (tid < 4) ends[tid / 2][tid % 2] = 0;
  if (tid == 0) n_cand = 0;
#pragma unroll
  for (int k = 0; k < R; ++k) asm volatile("" : "+v"(pos[k]), "+v"(acc[k]));     // loaded here: later waits would be for the stores, too
  // what the rows of `rows` in front of the new end carry
  auto keep_rows = [&](unsigned rows) {
#pragma unroll
    for (int k = 0; k < R; k += 4) {
      if ((rows >> k & 15u) == 15u) {
        *reinterpret_cast<i32x4_4*>(w.pos_out + j0 + k) = i32x4_4{pos[k], pos[k + 1], pos[k + 2], pos[k + 3]};
        *reinterpret_cast<f32x4_4*>(w.acc_out + j0 + k) = f32x4_4{acc[k], acc[k + 1], acc[k + 2], acc[k + 3]};
      } else {
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if (rows >> (k + e) & 1u) {
            w.pos_out[j0 + k + e] = pos[k + e];
            w.acc_out[j0 + k + e] = acc[k + e];
          }
      }
    }
  };
  int movers = 0;
  unsigned kept = live;
  if (w.keep < w.n) {
#pragma unroll
    for (int k = 0; k < R; ++k) key[k] = w.key(acc[k], pos[k]);
    auto ranked = [&](int k) { return (unsigned long long)key[k] << 32 | ~(unsigned)(j0 + k); };
    auto inside = [&](const KeyRange& r, int k) { return (live >> k & 1u) && r.holds(key[k]); };
    __syncthreads();
    const KeyCut cut = find_cut(
        w.keep,
        [&](int level, const KeyRange& r, int need) {
          if (wave * 64 * R < w.n) {
#pragma unroll
            for (int k = 0; k < R; ++k) count_key(hist[level], r.bin_of(key[k]), inside(r, k));
          }
          __syncthreads();
          const Found f = find_bin(hist[level], need, sums, out);
          return Found{__builtin_amdgcn_readfirstlane(f.bin), __builtin_amdgcn_readfirstlane(f.left), __builtin_amdgcn_readfirstlane(f.count)};
        },
        [&](int level, const KeyRange& r, unsigned& smallest, unsigned& largest) {
          unsigned top = 0, bottom = 0;
#pragma unroll
          for (int k = 0; k < R; ++k) {
            const bool in = inside(r, k);
            top = max(top, in ? key[k] : 0u);
            bottom = max(bottom, in ? ~key[k] : 0u);
          }
          top = wave_umax(top);
          bottom = wave_umax(bottom);
          if (lane == 0) {
            atomicMax(&ends[level][0], top);
            atomicMax(&ends[level][1], bottom);
          }
          __syncthreads();
          largest = (unsigned)__builtin_amdgcn_readfirstlane((int)ends[level][0]);
          smallest = (unsigned)__builtin_amdgcn_readfirstlane((int)~ends[level][1]);
        });
    unsigned long long least = (unsigned long long)cut.range.base << 32;         // a row stays if ranked >= least
    if (!cut.equal && cut.count != cut.need) {           // few: the last to stay is the one that need - 1 of them are larger than
#pragma unroll
      for (int k = 0; k < R; ++k)
        if (inside(cut.range, k)) {
          const int at = atomicAdd(&n_cand, 1);
          if (at < kRanked) cand[at] = ranked(k);        // cut.count of them; the list keeps its size by itself
        }
      __syncthreads();
      constexpr int kParts = kSmallThreads / kRanked;
      const int i = tid / kParts;
      const unsigned long long own = i < cut.count ? cand[i] : 0;
      int larger = 0;
      for (int c = tid % kParts; c < cut.count; c += kParts) larger += cand[c] > own;
#pragma unroll
      for (int o = kParts / 2; o > 0; o >>= 1) larger += __shfl_xor(larger, o, 64);
      if (tid % kParts == 0 && i < cut.count && larger == cut.need - 1) bound = own;
      __syncthreads();
      least = bound;
    }
    unsigned stay = 0;
    if (!cut.equal) {
#pragma unroll
      for (int k = 0; k < R; ++k) stay |= ranked(k) >= least ? 1u << k : 0u;
    } else {
      unsigned tie = 0;
#pragma unroll
      for (int k = 0; k < R; ++k) {
        stay |= key[k] > cut.range.base ? 1u << k : 0u;
        tie |= key[k] == cut.range.base ? 1u << k : 0u;
      }
      tie &= live;
      int more = cut.need - (int)scan_threads(__popc(tie), wave, tie_sums).before;
#pragma unroll
      for (int k = 0; k < R; ++k) {
        const unsigned one = tie & 1u << k;
        stay |= more > 0 ? one : 0u;
        more -= one != 0;
      }
    }
    stay &= live;
    const unsigned hole = front & ~stay, mover = stay & ~front;
    // 16 bits each: a pair has at most 16384 rows
    const Before b = scan_threads(__popc(hole) | __popc(mover) << 16, wave, move_sums);
    movers = min((int)(b.all >> 16), (int)(b.all & 0xffffu));           // as many as there are holes; no list is longer
    auto list_rows = [&](int2* list) {
      int at_hole = (int)(b.before & 0xffffu), at_mover = (int)(b.before >> 16);
#pragma unroll
      for (int k = 0; k < R; ++k) {
        if ((hole >> k & 1u) && at_hole < movers) list[at_hole++].y = j0 + k;
        if ((mover >> k & 1u) && at_mover < movers) list[at_mover++].x = j0 + k;
      }
    };
    if (p.move_here) list_rows(few);
    else list_rows(w.list);
    kept = stay & front;
    __syncthreads();
  }
  if (tid == 0) {
    p.row_cnt[pair] = w.keep;
    p.moves[pair] = movers;
  }
  if (p.move_here) move_rows<16>(p, w, few, pair, movers, tid / 16, kSmallThreads / 16, tid % 16);
  keep_rows(kept);                                       // last: nothing waits for these stores
}

// ------------------------------------------------------------------ more rows.  grid: (kChunks, pairs)

// Chunk c of a pair: rows [begin, end), all in front of the new end or all behind it.
__device__ __forceinline__ void chunk_rows(const PairRows& w, int c, int& begin, int& end) {
  const int size = cdiv(w.n, kChunks - 2), front = cdiv(w.keep, max(size, 1));
  begin = c < front ? c * size : w.keep + (c - front) * size;
  end = c < front ? min(begin + size, w.keep) : min(begin + size, w.n);
  end = max(begin, end);
}

// One entry of `hist` per (digit, pair, chunk, bin), of `coarse` per (digit, pair, chunk, 32 bins), of `above` per (pair, chunk).
constexpr int kFine = kBins / 64;
__device__ __forceinline__ int* chunk_hist(const EvictParams& p, int d, int pair, int c) {
  return p.hist + (((long long)d * gridDim.y + pair) * kChunks + c) * kBins;
}
__device__ __forceinline__ int* chunk_coarse(const EvictParams& p, int d, int pair, int c) {
  return p.coarse + (((long long)d * gridDim.y + pair) * kChunks + c) * 64;
}

// The bin of digit d that holds the need-th largest key, and how many of it are wanted, from the chunks' histograms: the 32 bins first
// that hold it, then the bin.  (All bins of all chunks are 320 KB a workgroup: 12.5 us for a launch of 320 workgroups that takes 6
// so.)  Wavefront v reads chunks v, v + 8, .. and keeps their counts: with them it knows how many keys of
// such a chunk lie above the bin.  All threads call `find`.
struct DigitCut {
  static constexpr int kWaves = kChunkThreads / 64, kOwn = kChunks / kWaves;
  static_assert(kOwn * kWaves == kChunks && kFine == 32, "");
  int wide[kOwn], fine[(kOwn + 1) / 2];                  // fine: chunk k of the wavefront in lanes 32 (k % 2) .. + 31
  int bin, left;
  __device__ __forceinline__ void find(const EvictParams& p, int d, int pair, int need, int (*part)[64]) {
    const int lane = lane_id(), wave = threadIdx.x >> 6;
    int s = 0;
#pragma unroll
    for (int k = 0; k < kOwn; ++k) wide[k] = chunk_coarse(p, d, pair, wave + k * kWaves)[lane];
#pragma unroll
    for (int k = 0; k < kOwn; ++k) s += wide[k];
    part[wave][lane] = s;
    __syncthreads();
    // a lane a bin, the largest first: the lane in which the keys so far reach `need`
    int n = 0;
#pragma unroll
    for (int v = 0; v < kWaves; ++v) n += part[v][63 - lane];
    int inc = (int)wave_scan((unsigned)n);
    int at = __ffsll((unsigned long long)__ballot(inc >= need)) - 1;
    const int group = 63 - at;
    need -= __shfl(inc - n, at, 64);
    s = 0;
#pragma unroll
    for (int k = 0; k < (kOwn + 1) / 2; ++k) {
      const int own = 2 * k + lane / 32;
      fine[k] = own < kOwn ? chunk_hist(p, d, pair, wave + own * kWaves)[group * kFine + lane % 32] : 0;
    }
#pragma unroll
    for (int k = 0; k < (kOwn + 1) / 2; ++k) s += fine[k];
    __syncthreads();                                     // everyone has read `part`
    part[wave][lane] = s;
    __syncthreads();
    n = 0;
#pragma unroll
    for (int v = 0; v < 2 * kWaves; ++v) n += part[v / 2][v % 2 * 32 + 31 - lane % 32];
    if (lane >= 32) n = 0;
    inc = (int)wave_scan((unsigned)n);
    at = __ffsll((unsigned long long)__ballot(inc >= need)) - 1;
    left = need - __shfl(inc - n, at, 64);
    bin = group * kFine + 31 - at;
  }
  // keys above the bin of the wavefront's chunk k, and in it
  __device__ __forceinline__ int2 chunk(int k) const {
    const int lane = lane_id(), at = bin % kFine;
    const int n = (lane > bin / kFine ? wide[k] : 0) + (lane / 32 == k % 2 && lane % 32 > at ? fine[k / 2] : 0);
    return int2{(int)__shfl(wave_scan((unsigned)n), 63, 64), __shfl(fine[k / 2], k % 2 * 32 + at, 64)};
  }
};

// Histogram of digit D among the keys that share the digits found so far.
template <int D>
__global__ __launch_bounds__(kChunkThreads) void evict_digit_kernel(EvictParams p) {
  __shared__ __attribute__((aligned(16))) int hist[kBins];
  __shared__ int part[kChunkThreads / 64][64];
  const int pair = blockIdx.y, tid = threadIdx.x;
  const PairRows w(p, pair);
  if (w.keep == w.n) return;
  int begin, end;
  chunk_rows(w, blockIdx.x, begin, end);
  float acc[kChunkRows];
  int pos[kChunkRows];
  auto load = [&](int j0) {
#pragma unroll
    for (int k = 0; k < kChunkRows; ++k) {
      const int j = j0 + k * kChunkThreads + tid;
      acc[k] = j < end ? w.acc[j] : 0.f;
      pos[k] = j < end ? w.pos[j] : 0;
    }
  };
  load(begin);                                           // on their way while the digit before is found
  unsigned prefix = 0;
  if constexpr (D > 0) {
    const int need = D == 1 ? w.keep : p.cut[pair * 4 + 1];
    prefix = D == 1 ? 0u : (unsigned)p.cut[pair * 4];
    const int so_far = D == 1 ? 0 : p.above[pair * kChunks + blockIdx.x];
    DigitCut digit;
    digit.find(p, D - 1, pair, need, part);
    prefix = with_digit(prefix, digit.bin, D - 1);
    if (blockIdx.x == 0 && tid == 0) {                   // for the next launch; digits of different launches do not meet
      p.cut[pair * 4 + (D == 1 ? 0 : 2)] = (int)prefix;
      p.cut[pair * 4 + (D == 1 ? 1 : 3)] = digit.left;
    }
#pragma unroll
    for (int k = 0; k < DigitCut::kOwn; ++k) {           // keys of this chunk above the bin
      if (tid / 64 + k * DigitCut::kWaves != (int)blockIdx.x) continue;
      const int n = digit.chunk(k).x;
      if (lane_id() == 0) p.above[pair * kChunks + blockIdx.x] = so_far + n;
    }
  }
  for (int i = tid; i < kBins; i += kChunkThreads) hist[i] = 0;
  __syncthreads();
  for (int j0 = begin; j0 < end; j0 += kChunkRows * kChunkThreads) {
    if (j0 != begin) load(j0);
#pragma unroll
    for (int k = 0; k < kChunkRows; ++k) {
      const unsigned key = w.key(acc[k], pos[k]);
      count_key(hist, digit_of(key, D), j0 + k * kChunkThreads + tid < end && same_above(key, prefix, D));
    }
  }
  __syncthreads();
  static_assert(kBins == 4 * kChunkThreads, "four bins a thread, 32 of 8 lanes");
  const i32x4 h = *reinterpret_cast<const i32x4*>(hist + tid * 4);
  *reinterpret_cast<i32x4*>(chunk_hist(p, D, pair, blockIdx.x) + tid * 4) = h;
  const int n = (int)wave_scan((unsigned)(h[0] + h[1] + h[2] + h[3])), before = __shfl(n, (tid & 56) - 1, 64);
  if (tid % 8 == 7) chunk_coarse(p, D, pair, blockIdx.x)[tid / 8] = n - ((tid & 63) > 7 ? before : 0);
}

// Lists of holes and movers, and what the rows that stay carry.  A chunk's first places follow from the histograms: the rows of
// a chunk above the cut, and its ties.
__global__ __launch_bounds__(kChunkThreads) void evict_lists_kernel(EvictParams p) {
  constexpr int kWaves = kChunkThreads / 64, R = kChunkRows, kRound = R * kChunkThreads;
  static_assert(R * kWaves == 64, "a lane a cell");
  __shared__ int part[kWaves][64], above[kChunks], ties[kChunks], start[3];
  __shared__ unsigned cell[2][64];
  const int pair = blockIdx.y, tid = threadIdx.x, lane = lane_id(), wave = tid >> 6;
  const PairRows w(p, pair);
  int begin, end;
  chunk_rows(w, blockIdx.x, begin, end);
  if (w.keep == w.n) {
    for (int j = begin + tid; j < end; j += kChunkThreads) {
      w.pos_out[j] = w.pos[j];
      w.acc_out[j] = w.acc[j];
    }
    if (blockIdx.x == 0 && tid == 0) {
      p.row_cnt[pair] = w.n;                             // the count as it was, cut to its range: a chunk that reads it later gets the same
      p.moves[pair] = 0;
    }
    return;
  }
  float acc[R];
  int pos[R];
  auto load = [&](int j0) {
#pragma unroll
    for (int k = 0; k < R; ++k) {
      const int j = j0 + k * kChunkThreads + tid;
      acc[k] = j < end ? w.acc[j] : 0.f;
      pos[k] = j < end ? w.pos[j] : 0;
    }
  };
  load(begin);
  int higher[DigitCut::kOwn];                            // rows above the digits before, of the wavefront's chunks
#pragma unroll
  for (int k = 0; k < DigitCut::kOwn; ++k) higher[k] = p.above[pair * kChunks + wave + k * kWaves];
  DigitCut digit;
  digit.find(p, 2, pair, p.cut[pair * 4 + 3], part);
  const unsigned cut = with_digit((unsigned)p.cut[pair * 4 + 2], digit.bin, 2);
  const int need = digit.left;
#pragma unroll
  for (int k = 0; k < DigitCut::kOwn; ++k) {
    const int2 n = digit.chunk(k);
    if (lane == 0) {
      above[wave + k * kWaves] = n.x + higher[k];
      ties[wave + k * kWaves] = n.y;
    }
  }
  __syncthreads();
  if (wave == 0) {                                       // a lane a chunk
    const int c = min(lane, kChunks - 1);
    int b, e;
    chunk_rows(w, c, b, e);
    const int t_own = lane < kChunks ? ties[c] : 0, t = (int)wave_scan((unsigned)t_own) - t_own;
    const int stay = lane < kChunks ? above[c] + min(max(need - t, 0), t_own) : 0;
    const int h_own = lane < kChunks && b < w.keep ? e - b - stay : 0, m_own = lane < kChunks && b >= w.keep ? stay : 0;
    const int h = (int)wave_scan((unsigned)h_own), m = (int)wave_scan((unsigned)m_own);
    if (lane == (int)blockIdx.x) {
      start[0] = t;
      start[1] = h - h_own;
      start[2] = m - m_own;
    }
    if (blockIdx.x == 0 && lane == 63) p.moves[pair] = m;
  }
  __syncthreads();
  int tie0 = start[0], place0 = begin < w.keep ? start[1] : start[2];
  const bool front = begin < w.keep;                     // holes in front of the new end, movers behind it
  const unsigned long long below = (1ull << lane) - 1;
  for (int j0 = begin; j0 < end; j0 += kRound) {
    if (j0 != begin) load(j0);
#pragma unroll
    for (int k = 0; k < R; ++k) asm volatile("" : "+v"(pos[k]), "+v"(acc[k]));   // loaded here: later waits would be for the stores, too
    unsigned long long tie[R];
#pragma unroll
    for (int k = 0; k < R; ++k) {
      tie[k] = __ballot(j0 + k * kChunkThreads + tid < end && w.key(acc[k], pos[k]) == cut);
      if (lane == 0) cell[0][k * kWaves + wave] = __popcll(tie[k]);
    }
    __syncthreads();
    unsigned own = cell[0][lane], inc = wave_scan(own);
    unsigned stay = 0;
    unsigned long long listed[R];
#pragma unroll
    for (int k = 0; k < R; ++k) {
      const int j = j0 + k * kChunkThreads + tid;
      const int before = tie0 + (int)__shfl(inc - own, k * kWaves + wave, 64) + __popcll(tie[k] & below);
      const unsigned key = w.key(acc[k], pos[k]);
      const bool s = j < end && (key > cut || (key == cut && before < need));
      if (s) stay |= 1u << k;
      listed[k] = __ballot(j < end && s != front);
      if (lane == 0) cell[1][k * kWaves + wave] = __popcll(listed[k]);
    }
    tie0 += (int)__shfl(inc, 63, 64);
    __syncthreads();
    own = cell[1][lane];
    inc = wave_scan(own);
#pragma unroll
    for (int k = 0; k < R; ++k) {
      const int j = j0 + k * kChunkThreads + tid;
      const int at = place0 + (int)__shfl(inc - own, k * kWaves + wave, 64) + __popcll(listed[k] & below);
      if (listed[k] >> lane & 1ull) {
        if (front) w.list[at].y = j;
        else w.list[at].x = j;
      }
      if (front && (stay >> k & 1u)) {
        w.pos_out[j] = pos[k];
        w.acc_out[j] = acc[k];
      }
    }
    place0 += (int)__shfl(inc, 63, 64);
  }
}

// The rows that change places, and the new counts: row_cnt may be row_end, which the launches before read.  grid: (blocks, pairs)
constexpr int kMoveThreads = 256;
template <int LANES>
__global__ __launch_bounds__(kMoveThreads) void evict_move_kernel(EvictParams p) {
  const int pair = blockIdx.y;
  const PairRows w(p, pair);
  constexpr int kRows = kMoveThreads / LANES;
  if (blockIdx.x == 0 && threadIdx.x == 0) p.row_cnt[pair] = w.keep;
  move_rows<LANES>(p, w, w.list, pair, p.moves[pair], blockIdx.x * kRows + threadIdx.x / LANES, gridDim.x * kRows, threadIdx.x % LANES);
}

void carve(EvictParams& p, int pairs, int cap, Arena& a) {
  p.moves = a.take<int>(pairs);
  p.list = a.take<int2>((size_t)pairs * (cap / 2));
  if (cap > kSmallRows) {
    p.cut = a.take<int>((size_t)pairs * 4);
    p.hist = a.take<int>((size_t)3 * pairs * kChunks * kBins);
    p.coarse = a.take<int>((size_t)3 * pairs * kChunks * 64);
    p.above = a.take<int>((size_t)pairs * kChunks);
  }
}

}  // namespace

size_t paged_evict_ws(int pairs, int cap) {
  EvictParams p{};
  Arena a(nullptr);
  carve(p, pairs, cap, a);
  return a.used();
}

int run_paged_evict(int B, int Hkv, int D, int dtype, const Pages& pg, int budget, int n_sink, int n_recent, const int* seq_len,
                    const int* row_end, const int* row_pos, const float* acc, int* row_cnt, int* pos_out, float* acc_out,
                    void* ws, hipStream_t st) {
  const int pairs = B * Hkv, cap = rows_cap(pg);
  EvictParams p{};
  Arena a(ws);
  carve(p, pairs, cap, a);
  p.pg = pg; p.Hkv = Hkv; p.row_bytes = D * (dtype == OMNI_BF16 ? 2 : 4); p.budget = budget; p.n_sink = n_sink;
  p.n_recent = n_recent; p.seq_len = seq_len;
  p.row_end = row_end; p.row_pos = row_pos; p.acc = acc; p.row_cnt = row_cnt; p.pos_out = pos_out; p.acc_out = acc_out;
  const int most = std::min({cap / 2, budget, std::max(0, cap - budget)});       // moves of a pair
  if (cap <= kSmallRows) {
    p.move_here = most <= kFewMoves;
    if (cap <= 4 * kSmallThreads) evict_small_kernel<4><<<pairs, kSmallThreads, 0, st>>>(p);
    else if (cap <= 8 * kSmallThreads) evict_small_kernel<8><<<pairs, kSmallThreads, 0, st>>>(p);
    else evict_small_kernel<16><<<pairs, kSmallThreads, 0, st>>>(p);
    OMNI_LAUNCH_CHECK();
    if (p.move_here) return OMNI_OK;
  } else {
    const dim3 grid(kChunks, pairs);
    evict_digit_kernel<0><<<grid, kChunkThreads, 0, st>>>(p);
    OMNI_LAUNCH_CHECK();
    evict_digit_kernel<1><<<grid, kChunkThreads, 0, st>>>(p);
    OMNI_LAUNCH_CHECK();
    evict_digit_kernel<2><<<grid, kChunkThreads, 0, st>>>(p);
    OMNI_LAUNCH_CHECK();
    evict_lists_kernel<<<grid, kChunkThreads, 0, st>>>(p);
    OMNI_LAUNCH_CHECK();
  }
  if (most == 0) return OMNI_OK;
  const int lanes = p.row_bytes / 16;
  const dim3 grid(std::max(1, std::min(cdiv(most, kMoveThreads / lanes), 4096 / pairs)), pairs);
  if (lanes == 8) evict_move_kernel<8><<<grid, kMoveThreads, 0, st>>>(p);
  else if (lanes == 16) evict_move_kernel<16><<<grid, kMoveThreads, 0, st>>>(p);
  else evict_move_kernel<32><<<grid, kMoveThreads, 0, st>>>(p);
  OMNI_LAUNCH_CHECK();
  return OMNI_OK;
}

}  // namespace omni
