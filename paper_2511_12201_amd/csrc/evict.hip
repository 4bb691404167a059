// Eviction from a paged cache by accumulated attention weight (omni_paged_evict).
//
// Per (sequence, KV head) pair the rows are ranked by a 32-bit key (spared rows above every weight, the weights in order, NaN
// below them) and the `keep` largest stay, equal keys by lowest row.  The key at the cut is found digit by digit (11, 11 and 10
// bits) with histograms in LDS; then the rows are counted in order, which splits the ties and numbers the holes and the rows that
// move into them.  Rows are only copied where they have to: a row that stays in front of the new end stays where it is.
//
// The selection has to read 8 bytes a row, the moves 4 rows' bytes each; what bounds a small call is the chain of dependent steps.
//  * Up to 16384 rows a pair (evict_small_kernel): one workgroup a pair, its keys in registers throughout, one launch and one for
//    the moves; where a pair can have few moves the workgroup makes them itself and the second launch is left out.
//  * More: the pair's rows in front of the new end and those behind it are cut into chunks, a workgroup each: three launches for
//    the digits (every chunk leaves its histogram, the next launch adds them up), one for the lists, one for the moves.
#include <algorithm>

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
  int *hist, *total, *above;     // many rows: [3][pairs, kChunks, kBins], [2][pairs, kBins], [pairs, kChunks]
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
  const int first = __shfl(bin, __ffsll((unsigned long long)who) - 1, 64);
  if (__all(!counts || bin == first)) {
    if (lane_id() == 0) atomicAdd(&hist[first], __popcll(who));
  } else if (counts) {
    atomicAdd(&hist[bin], 1);
  }
}

// The bin that holds the need-th largest key, how many of it are wanted, and whether that is all of it; hist in LDS, all threads
// call it.
struct Found {
  int bin, left, all;
};
template <int THREADS>
__device__ __forceinline__ Found find_bin(const int* hist, int need, int* wave_sums, int* out) {
  constexpr int PER = kBins / THREADS, kWaves = THREADS / 64;
  int own = 0, h[PER];
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    h[i] = hist[kBins - 1 - ((int)threadIdx.x * PER + i)];       // from the largest key down
    own += h[i];
  }
  const int inc = (int)wave_scan((unsigned)own), wave = threadIdx.x >> 6;
  if (lane_id() == 63) wave_sums[wave] = inc;
  __syncthreads();
  const int sums = (int)wave_scan((unsigned)(lane_id() < kWaves ? wave_sums[lane_id()] : 0));
  int before = inc - own + (wave ? __shfl(sums, wave - 1, 64) : 0);
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    if (before < need && need <= before + h[i]) {
      out[0] = kBins - 1 - ((int)threadIdx.x * PER + i);
      out[1] = need - before;
      out[2] = need == before + h[i];
    }
    before += h[i];
  }
  __syncthreads();
  return Found{out[0], out[1], out[2]};
}

// K and V of moved rows and what they carry; LANES lanes a row.
template <int LANES>
__device__ __forceinline__ void move_rows(const EvictParams& p, const PairRows& w, int pair, int moves, int first, int step, int lane) {
  const int per = p.row_bytes / 16;
  for (int i = first; i < moves; i += step) {
    const int2 m = w.list[i];
    if (lane == 0) {
      w.pos_out[m.y] = w.pos[m.x];                       // rows behind `keep` are never written: in place is as good
      w.acc_out[m.y] = w.acc[m.x];
    }
    const int from = pool_row(p.pg, pair, m.x), to = pool_row(p.pg, pair, m.y);
    if (from < 0 || to < 0) continue;
    for (int c = lane; c < per; c += LANES) {
      const u32x4 k = static_cast<const u32x4*>(p.pg.K)[(long long)from * per + c], v = static_cast<const u32x4*>(p.pg.V)[(long long)from * per + c];
      static_cast<u32x4*>(p.pg.K)[(long long)to * per + c] = k;
      static_cast<u32x4*>(p.pg.V)[(long long)to * per + c] = v;
    }
  }
}

// ------------------------------------------------------------------ up to kSmallRows rows a pair.  grid: pairs

// R rows a thread: row k * kSmallThreads + thread.
template <int R>
__global__ __launch_bounds__(kSmallThreads) void evict_small_kernel(EvictParams p) {
  constexpr int kWaves = kSmallThreads / 64, kCells = R * kWaves, CPL = kCells / 64;   // cells (k, wavefront) in the order of the rows
  __shared__ int hist[3][kBins];
  __shared__ int sums[kWaves], out[3];
  __shared__ __attribute__((aligned(16))) unsigned cell[2][kCells];
  const int pair = blockIdx.x, tid = threadIdx.x, lane = lane_id(), wave = tid >> 6;
  const PairRows w(p, pair);
  unsigned key[R];
  int pos[R];
  float acc[R];
#pragma unroll
  for (int k = 0; k < R; ++k) {
    const int j = k * kSmallThreads + tid;
    pos[k] = j < w.n ? w.pos[j] : 0;
    acc[k] = j < w.n ? w.acc[j] : 0.f;
  }
  int movers = 0;
  if (w.keep < w.n) {
    for (int i = tid; i < 3 * kBins; i += kSmallThreads) hist[0][i] = 0;
#pragma unroll
    for (int k = 0; k < R; ++k) key[k] = w.key(acc[k], pos[k]);
    unsigned cut = 0;
    int need = w.keep;
    __syncthreads();
    for (int d = 0; d < 3; ++d) {
#pragma unroll
      for (int k = 0; k < R; ++k) {
        if (k * kSmallThreads + wave * 64 < w.n)         // wave-uniform
          count_key(hist[d], digit_of(key[k], d), k * kSmallThreads + tid < w.n && same_above(key[k], cut, d));
      }
      __syncthreads();
      const Found f = find_bin<kSmallThreads>(hist[d], need, sums, out);
      cut = with_digit(cut, f.bin, d);
      need = f.left;
      if (f.all) {                                       // every key from here on stays, whatever its other digits
        need = 0x7fffffff;
        break;
      }
    }
    // in front of a thread's cell k: the counts of the cells before; 16 bits each for two kinds (a pair has at most 16384 rows)
    unsigned base[CPL];
    auto scan_cells = [&](const unsigned* c) {
      unsigned sum = 0;
#pragma unroll
      for (int i = 0; i < CPL; ++i) {
        base[i] = sum;
        sum += c[lane * CPL + i];
      }
      const unsigned before = wave_scan(sum) - sum;
#pragma unroll
      for (int i = 0; i < CPL; ++i) base[i] += before;
    };
    auto before_cell = [&](int k) {
      unsigned v = base[0];                              // cell k * kWaves + wave is piece wave % CPL of lane (k * kWaves + wave) / CPL
#pragma unroll
      for (int i = 1; i < CPL; ++i) v = wave % CPL == i ? base[i] : v;
      return __shfl(v, (k * kWaves + wave) / CPL, 64);
    };
    const unsigned long long below = (1ull << lane) - 1;
    unsigned stay = 0;
    if (need == 0x7fffffff) {
#pragma unroll
      for (int k = 0; k < R; ++k)
        if (k * kSmallThreads + tid < w.n && key[k] >= cut) stay |= 1u << k;
    } else {
#pragma unroll
      for (int k = 0; k < R; ++k) {
        const unsigned long long b = __ballot(k * kSmallThreads + tid < w.n && key[k] == cut);
        if (lane == 0) cell[0][k * kWaves + wave] = __popcll(b);
      }
      __syncthreads();
      scan_cells(cell[0]);
#pragma unroll
      for (int k = 0; k < R; ++k) {
        const int j = k * kSmallThreads + tid;
        const bool tie = j < w.n && key[k] == cut;
        const unsigned long long b = __ballot(tie);
        const int before = (int)before_cell(k) + __popcll(b & below);
        if (j < w.n && (key[k] > cut || (tie && before < need))) stay |= 1u << k;
      }
    }
#pragma unroll
    for (int k = 0; k < R; ++k) {
      const int j = k * kSmallThreads + tid;
      const bool s = stay >> k & 1u;
      const unsigned long long bh = __ballot(j < w.keep && !s), bm = __ballot(j >= w.keep && s);
      if (lane == 0) cell[1][k * kWaves + wave] = (unsigned)__popcll(bh) | (unsigned)__popcll(bm) << 16;
    }
    __syncthreads();
    scan_cells(cell[1]);
#pragma unroll
    for (int k = 0; k < R; ++k) {
      const int j = k * kSmallThreads + tid;
      const bool s = stay >> k & 1u, hole = j < w.keep && !s, mover = j >= w.keep && s;
      const unsigned long long bh = __ballot(hole), bm = __ballot(mover);
      const unsigned before = before_cell(k);
      if (hole) w.list[(before & 0xffffu) + __popcll(bh & below)].y = j;
      if (mover) w.list[(before >> 16) + __popcll(bm & below)].x = j;
      if (j < w.keep && s) {
        w.pos_out[j] = pos[k];
        w.acc_out[j] = acc[k];
      }
      if (k == R - 1 && wave == kWaves - 1 && lane == 0) out[0] = (int)(before >> 16) + __popcll(bm);
    }
    __syncthreads();
    movers = out[0];
  } else {
#pragma unroll
    for (int k = 0; k < R; ++k) {
      const int j = k * kSmallThreads + tid;
      if (j < w.n) {
        w.pos_out[j] = pos[k];
        w.acc_out[j] = acc[k];
      }
    }
  }
  if (tid == 0) {
    p.row_cnt[pair] = w.keep;
    p.moves[pair] = movers;
  }
  if (p.move_here) move_rows<16>(p, w, pair, movers, tid / 16, kSmallThreads / 16, tid % 16);
}

// ------------------------------------------------------------------ more rows.  grid: (kChunks, pairs)

// Chunk c of a pair: rows [begin, end), all in front of the new end or all behind it.
__device__ __forceinline__ void chunk_rows(const PairRows& w, int c, int& begin, int& end) {
  const int size = cdiv(w.n, kChunks - 2), front = cdiv(w.keep, max(size, 1));
  begin = c < front ? c * size : w.keep + (c - front) * size;
  end = c < front ? min(begin + size, w.keep) : min(begin + size, w.n);
  end = max(begin, end);
}

// One entry of `hist` per (digit, pair, chunk, bin), of `total` per (digit 1 or 2, pair, bin), of `above` per (pair, chunk).
__device__ __forceinline__ int* chunk_hist(const EvictParams& p, int d, int pair, int c) {
  return p.hist + (((long long)d * gridDim.y + pair) * kChunks + c) * kBins;
}
__device__ __forceinline__ int* pair_total(const EvictParams& p, int d, int pair) { return p.total + ((long long)(d - 1) * gridDim.y + pair) * kBins; }

// Digit d of all chunks of the pair into LDS: the chunks' histograms added up (digit 0), or what they have added to the pair's.
__device__ __forceinline__ void load_total(const EvictParams& p, int d, int pair, int* hist) {
  for (int i = threadIdx.x * 4; i < kBins; i += kChunkThreads * 4) {
    i32x4 s = {0, 0, 0, 0};
    if (d == 0) {
      const int* src = chunk_hist(p, 0, pair, 0) + i;
#pragma unroll 20
      for (int c = 0; c < kChunks; ++c) s += *reinterpret_cast<const i32x4*>(src + c * kBins);
    } else {
      s = *reinterpret_cast<const i32x4*>(pair_total(p, d, pair) + i);
    }
    *reinterpret_cast<i32x4*>(hist + i) = s;
  }
  __syncthreads();
}

// Histogram of digit D among the keys that share the digits found so far.  Digit 0 also clears the pair's totals of the other two.
template <int D>
__global__ __launch_bounds__(kChunkThreads) void evict_digit_kernel(EvictParams p) {
  constexpr int kWaves = kChunkThreads / 64;
  __shared__ __attribute__((aligned(16))) int hist[kBins];
  __shared__ int sums[kWaves], out[3];
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
    load_total(p, D - 1, pair, hist);
    const Found f = find_bin<kChunkThreads>(hist, need, sums, out);
    prefix = with_digit(prefix, f.bin, D - 1);
    if (blockIdx.x == 0 && tid == 0) {                   // for the next launch; digits of different launches do not meet
      p.cut[pair * 4 + (D == 1 ? 0 : 2)] = (int)prefix;
      p.cut[pair * 4 + (D == 1 ? 1 : 3)] = f.left;
    }
    // keys of this chunk above the bin
    const int* own = chunk_hist(p, D - 1, pair, blockIdx.x);
    int n = 0;
    for (int i = tid; i < kBins; i += kChunkThreads) n += i > f.bin ? own[i] : 0;
    n = wave_sum(n);
    if (lane_id() == 0) sums[tid >> 6] = n;
    __syncthreads();
    if (tid == 0) {
      n = D == 1 ? 0 : p.above[pair * kChunks + blockIdx.x];
      for (int v = 0; v < kWaves; ++v) n += sums[v];
      p.above[pair * kChunks + blockIdx.x] = n;
    }
  } else if (blockIdx.x == 0) {
    for (int i = tid; i < kBins; i += kChunkThreads) pair_total(p, 1, pair)[i] = pair_total(p, 2, pair)[i] = 0;
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
  int* dst = chunk_hist(p, D, pair, blockIdx.x);
  for (int i = tid * 4; i < kBins; i += kChunkThreads * 4) {
    const i32x4 h = *reinterpret_cast<const i32x4*>(hist + i);
    *reinterpret_cast<i32x4*>(dst + i) = h;
    if constexpr (D > 0) {                               // integers: the order of the additions does not matter
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (h[e]) atomicAdd(pair_total(p, D, pair) + i + e, h[e]);
    }
  }
}

// Lists of holes and movers, and what the rows that stay carry.  A chunk's first places follow from the histograms: the rows of
// a chunk above the cut, and its ties.
__global__ __launch_bounds__(kChunkThreads) void evict_lists_kernel(EvictParams p) {
  constexpr int kWaves = kChunkThreads / 64, R = kChunkRows, kRound = R * kChunkThreads;
  static_assert(R * kWaves == 64, "a lane a cell");
  __shared__ __attribute__((aligned(16))) int hist[kBins];
  __shared__ int sums[kWaves], out[3], above[kChunks], ties[kChunks], start[3];
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
  load_total(p, 2, pair, hist);
  const Found f = find_bin<kChunkThreads>(hist, p.cut[pair * 4 + 3], sums, out);
  const unsigned cut = with_digit((unsigned)p.cut[pair * 4 + 2], f.bin, 2);
  const int need = f.left;
  // rows above the cut and ties of every chunk: a wavefront takes every kWaves-th chunk (the last digit has 1024 bins)
  constexpr int kOwn = kChunks / kWaves;
  static_assert(kOwn * kWaves == kChunks, "");
  int higher[kOwn], equal[kOwn];
#pragma unroll
  for (int k = 0; k < kOwn; ++k) {                       // all loads first
    const int* h = chunk_hist(p, 2, pair, wave + k * kWaves);
    higher[k] = 0;
#pragma unroll
    for (int i = lane * 4; i < 1024; i += 256) {
      const i32x4 x = *reinterpret_cast<const i32x4*>(h + i);
#pragma unroll
      for (int e = 0; e < 4; ++e) higher[k] += i + e > f.bin ? x[e] : 0;
    }
    equal[k] = h[f.bin];
  }
#pragma unroll
  for (int k = 0; k < kOwn; ++k) {
    const int c = wave + k * kWaves, n = (int)__shfl(wave_scan((unsigned)higher[k]), 63, 64);
    if (lane == 0) {
      above[c] = n + p.above[pair * kChunks + c];
      ties[c] = equal[k];
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
  move_rows<LANES>(p, w, pair, p.moves[pair], blockIdx.x * kRows + threadIdx.x / LANES, gridDim.x * kRows, threadIdx.x % LANES);
}

void carve(EvictParams& p, int pairs, int cap, Arena& a) {
  p.moves = a.take<int>(pairs);
  p.list = a.take<int2>((size_t)pairs * (cap / 2));
  if (cap > kSmallRows) {
    p.cut = a.take<int>((size_t)pairs * 4);
    p.hist = a.take<int>((size_t)3 * pairs * kChunks * kBins);
    p.total = a.take<int>((size_t)2 * pairs * kBins);
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
