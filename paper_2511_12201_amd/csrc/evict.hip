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
constexpr int kChunks = 32, kChunkThreads = 512;

struct EvictParams {
  Pages pg;
  int Hkv, row_bytes, budget, n_sink, n_recent, move_here;
  const int *seq_len, *row_end, *row_pos;
  const float* acc;
  int *row_cnt, *pos_out;
  float* acc_out;
  int* moves;                    // [pairs]
  int2* list;                    // [pairs, cap / 2] (from, to)
  int *hist, *cut;               // many rows: [3][pairs, kChunks, kBins]; [pairs, 4] digits found and rows wanted of the last one
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
    recent = p.seq_len[pair / p.Hkv] - p.n_recent;
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

// The bin that holds the need-th largest key, and how many of it are wanted; hist in LDS, all threads call it.
template <int THREADS>
__device__ __forceinline__ void find_bin(const int* hist, int need, int* wave_sums, int* out, int& bin, int& left) {
  constexpr int PER = kBins / THREADS;
  int own = 0, h[PER];
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    h[i] = hist[kBins - 1 - ((int)threadIdx.x * PER + i)];       // from the largest key down
    own += h[i];
  }
  const int inc = (int)wave_scan((unsigned)own);
  if (lane_id() == 63) wave_sums[threadIdx.x >> 6] = inc;
  __syncthreads();
  int before = inc - own;
  for (int v = 0; v < (int)(threadIdx.x >> 6); ++v) before += wave_sums[v];
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    if (before < need && need <= before + h[i]) {
      out[0] = kBins - 1 - ((int)threadIdx.x * PER + i);
      out[1] = need - before;
    }
    before += h[i];
  }
  __syncthreads();
  bin = out[0];
  left = out[1];
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
  constexpr int kWaves = kSmallThreads / 64, kCells = R * kWaves;        // (k, wavefront) in the order of the rows
  __shared__ int hist[kBins];
  __shared__ int sums[kWaves], out[2];
  __shared__ unsigned cell[kCells], cell_wave[kWaves];
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
#pragma unroll
    for (int k = 0; k < R; ++k) key[k] = w.key(acc[k], pos[k]);
    unsigned cut = 0;
    int need = w.keep;
    for (int d = 0; d < 3; ++d) {
      for (int i = tid; i < kBins; i += kSmallThreads) hist[i] = 0;
      __syncthreads();
#pragma unroll
      for (int k = 0; k < R; ++k) {
        if (k * kSmallThreads + wave * 64 < w.n)         // wave-uniform
          count_key(hist, digit_of(key[k], d), k * kSmallThreads + tid < w.n && same_above(key[k], cut, d));
      }
      __syncthreads();
      int bin;
      find_bin<kSmallThreads>(hist, need, sums, out, bin, need);
      cut = with_digit(cut, bin, d);
      __syncthreads();
    }
    // exclusive counts of the cells, in order; a cell holds two counts of 16 bits (a pair has at most 16384 rows)
    auto scan_cells = [&]() {
      __syncthreads();
      unsigned own = tid < kCells ? cell[tid] : 0u;
      const unsigned inc = wave_scan(own);
      if (lane == 63) cell_wave[wave] = inc;
      __syncthreads();
      unsigned before = inc - own;
      for (int v = 0; v < wave; ++v) before += cell_wave[v];
      if (tid < kCells) cell[tid] = before;
      __syncthreads();
    };
    const unsigned long long below = (1ull << lane) - 1;
#pragma unroll
    for (int k = 0; k < R; ++k) {
      const unsigned long long b = __ballot(k * kSmallThreads + tid < w.n && key[k] == cut);
      if (lane == 0) cell[k * kWaves + wave] = __popcll(b);
    }
    scan_cells();
    unsigned stay = 0;
#pragma unroll
    for (int k = 0; k < R; ++k) {
      const int j = k * kSmallThreads + tid;
      const bool tie = j < w.n && key[k] == cut;
      const unsigned long long b = __ballot(tie);
      if (j < w.n && (key[k] > cut || (tie && (int)cell[k * kWaves + wave] + __popcll(b & below) < need))) stay |= 1u << k;
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < R; ++k) {
      const int j = k * kSmallThreads + tid;
      const bool s = stay >> k & 1u;
      const unsigned long long bh = __ballot(j < w.keep && !s), bm = __ballot(j >= w.keep && s);
      if (lane == 0) cell[k * kWaves + wave] = (unsigned)__popcll(bh) | (unsigned)__popcll(bm) << 16;
    }
    scan_cells();
#pragma unroll
    for (int k = 0; k < R; ++k) {
      const int j = k * kSmallThreads + tid;
      const bool s = stay >> k & 1u, hole = j < w.keep && !s, mover = j >= w.keep && s;
      const unsigned long long bh = __ballot(hole), bm = __ballot(mover);
      const unsigned before = cell[k * kWaves + wave];
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

// The histogram of a digit added up over the chunks of the pair into LDS.
__device__ __forceinline__ void sum_hist(const EvictParams& p, int d, int pair, int* hist) {
  const int* src = p.hist + ((long long)d * gridDim.y + pair) * kChunks * kBins;
  for (int i = threadIdx.x * 4; i < kBins; i += kChunkThreads * 4) {
    i32x4 s = {0, 0, 0, 0};
#pragma unroll 8
    for (int c = 0; c < kChunks; ++c) s += *reinterpret_cast<const i32x4*>(src + c * kBins + i);
    *reinterpret_cast<i32x4*>(hist + i) = s;
  }
  __syncthreads();
}

// Histogram of digit D among the keys that share the digits found so far.
template <int D>
__global__ __launch_bounds__(kChunkThreads) void evict_digit_kernel(EvictParams p) {
  __shared__ __attribute__((aligned(16))) int hist[kBins];
  __shared__ int sums[kChunkThreads / 64], out[2];
  const int pair = blockIdx.y, tid = threadIdx.x;
  const PairRows w(p, pair);
  if (w.keep == w.n) return;
  unsigned prefix = 0;
  if constexpr (D > 0) {
    int need = D == 1 ? w.keep : p.cut[pair * 4 + 1];
    prefix = D == 1 ? 0u : (unsigned)p.cut[pair * 4];
    sum_hist(p, D - 1, pair, hist);
    int bin;
    find_bin<kChunkThreads>(hist, need, sums, out, bin, need);
    prefix = with_digit(prefix, bin, D - 1);
    if (blockIdx.x == 0 && tid == 0) {                   // for the next launch; digits of different launches do not meet
      p.cut[pair * 4 + (D == 1 ? 0 : 2)] = (int)prefix;
      p.cut[pair * 4 + (D == 1 ? 1 : 3)] = need;
    }
    __syncthreads();
  }
  for (int i = tid; i < kBins; i += kChunkThreads) hist[i] = 0;
  __syncthreads();
  int begin, end;
  chunk_rows(w, blockIdx.x, begin, end);
  for (int j0 = begin; j0 < end; j0 += kChunkThreads) {
    const int j = j0 + tid;
    const unsigned k = j < end ? w.key(w.acc[j], w.pos[j]) : 0u;
    count_key(hist, digit_of(k, D), j < end && same_above(k, prefix, D));
  }
  __syncthreads();
  int* dst = p.hist + (((long long)D * gridDim.y + pair) * kChunks + blockIdx.x) * kBins;
  for (int i = tid * 4; i < kBins; i += kChunkThreads * 4) *reinterpret_cast<i32x4*>(dst + i) = *reinterpret_cast<const i32x4*>(hist + i);
}

// Lists of holes and movers, and what the rows that stay carry.  A chunk's first places follow from the histograms: the rows of
// a chunk above the cut, and its ties.
__global__ __launch_bounds__(kChunkThreads) void evict_lists_kernel(EvictParams p) {
  constexpr int kWaves = kChunkThreads / 64;
  __shared__ __attribute__((aligned(16))) int hist[kBins];
  __shared__ int sums[kWaves], out[2], above[kChunks], ties[kChunks], start[3];
  __shared__ int wave_tie[kWaves], wave_hole[kWaves], wave_move[kWaves];
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
      p.row_cnt[pair] = w.keep;
      p.moves[pair] = 0;
    }
    return;
  }
  int need = p.cut[pair * 4 + 3];
  unsigned cut = (unsigned)p.cut[pair * 4 + 2];
  sum_hist(p, 2, pair, hist);
  int bin;
  find_bin<kChunkThreads>(hist, need, sums, out, bin, need);
  cut = with_digit(cut, bin, 2);
  // rows above the cut and ties of every chunk: a wavefront takes every kWaves-th chunk
  for (int c = wave; c < kChunks; c += kWaves) {
    int n = 0;
    for (int d = 0; d < 3; ++d) {
      const int* h = p.hist + (((long long)d * gridDim.y + pair) * kChunks + c) * kBins;
      for (int i = digit_of(cut, d) + 1 + lane; i < kBins; i += 64) n += h[i];
    }
    n = wave_sum(n);
    if (lane == 0) {
      above[c] = n;
      ties[c] = p.hist[((2ll * gridDim.y + pair) * kChunks + c) * kBins + digit_of(cut, 2)];
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
    if (blockIdx.x == 0 && lane == 63) {
      p.row_cnt[pair] = w.keep;
      p.moves[pair] = m;
    }
  }
  __syncthreads();
  int tie0 = start[0], hole0 = start[1], move0 = start[2];
  const unsigned long long below = (1ull << lane) - 1;
  for (int j0 = begin; j0 < end; j0 += kChunkThreads) {
    const int j = j0 + tid;
    const float a = j < end ? w.acc[j] : 0.f;
    const int q = j < end ? w.pos[j] : 0;
    const unsigned k = w.key(a, q);
    const bool tie = j < end && k == cut;
    const unsigned long long bt = __ballot(tie);
    if (lane == 0) wave_tie[wave] = __popcll(bt);
    __syncthreads();
    int before = tie0 + __popcll(bt & below);
#pragma unroll
    for (int v = 0; v < kWaves; ++v) {
      if (v < wave) before += wave_tie[v];
      tie0 += wave_tie[v];
    }
    const bool stays = j < end && (k > cut || (tie && before < need));
    const bool hole = j < end && j < w.keep && !stays, mover = stays && j >= w.keep;
    const unsigned long long bh = __ballot(hole), bm = __ballot(mover);
    if (lane == 0) {
      wave_hole[wave] = __popcll(bh);
      wave_move[wave] = __popcll(bm);
    }
    __syncthreads();
    int ih = hole0 + __popcll(bh & below), im = move0 + __popcll(bm & below);
#pragma unroll
    for (int v = 0; v < kWaves; ++v) {
      if (v < wave) {
        ih += wave_hole[v];
        im += wave_move[v];
      }
      hole0 += wave_hole[v];
      move0 += wave_move[v];
    }
    if (hole) w.list[ih].y = j;
    if (mover) w.list[im].x = j;
    if (stays && j < w.keep) {
      w.pos_out[j] = q;
      w.acc_out[j] = a;
    }
    // the next round's first barrier comes after everyone has read wave_tie; wave_hole and wave_move are written after it
  }
}

// The rows that change places.  grid: (blocks, pairs)
constexpr int kMoveThreads = 256;
template <int LANES>
__global__ __launch_bounds__(kMoveThreads) void evict_move_kernel(EvictParams p) {
  const int pair = blockIdx.y;
  const PairRows w(p, pair);
  constexpr int kRows = kMoveThreads / LANES;
  move_rows<LANES>(p, w, pair, p.moves[pair], blockIdx.x * kRows + threadIdx.x / LANES, gridDim.x * kRows, threadIdx.x % LANES);
}

void carve(EvictParams& p, int pairs, int cap, Arena& a) {
  p.moves = a.take<int>(pairs);
  p.list = a.take<int2>((size_t)pairs * (cap / 2));
  if (cap > kSmallRows) {
    p.cut = a.take<int>((size_t)pairs * 4);
    p.hist = a.take<int>((size_t)3 * pairs * kChunks * kBins);
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
