// Eviction from a paged cache by accumulated attention weight (omni_paged_evict).
//
// Per (sequence, KV head) pair the rows are ranked by a 32-bit key (spared rows above every weight, the weights in order, NaN
// below them) and the `keep` largest stay, equal keys by lowest row.  The key at the cut is found byte by byte with histograms in
// LDS; then the rows are walked once in order, which splits the ties and numbers the holes and the rows that move into them.
// Rows are only copied where they have to: a row that stays in front of the new end stays where it is.
#include <algorithm>

#include "paged.h"

namespace omni {

namespace {

constexpr int kThreads = 1024;
constexpr int kWaves = kThreads / 64;

struct EvictParams {
  Pages pg;
  int Hkv, budget, n_sink, n_recent;
  const int *seq_len, *row_end, *row_pos;
  const float* acc;
  int *row_cnt, *pos_out;
  float* acc_out;
  int* moves;                    // [pairs]
  int2* list;                    // [pairs, cap / 2] (from, to)
};

__device__ __forceinline__ unsigned rank_key(float acc, bool spared) {
  if (spared) return 0xffffffffu;
  return acc != acc ? float_key(-INFINITY) : float_key(acc + 0.f);       // -0 and 0 are one weight
}

// grid: pairs
__global__ __launch_bounds__(kThreads) void evict_select_kernel(EvictParams p) {
  __shared__ int hist[256];
  __shared__ unsigned sPrefix;
  __shared__ int sNeed, sWave[kWaves], sWave2[kWaves], sWave3[kWaves];
  const int pair = blockIdx.x, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int cap = rows_cap(p.pg);
  const int n = clampi(p.row_end[pair], 0, cap), keep = min(n, p.budget);
  const int* pos = p.row_pos + (long long)pair * cap;
  const float* acc = p.acc + (long long)pair * cap;
  const int recent = p.seq_len[pair / p.Hkv] - p.n_recent;
  auto key_of = [&](int j) { return rank_key(acc[j], pos[j] < p.n_sink || pos[j] >= recent); };

  if (keep < n) {
    unsigned prefix = 0;
    int need = keep;                                   // rows still wanted among those that share the prefix
    for (int shift = 24; shift >= 0; shift -= 8) {
      if (tid < 256) hist[tid] = 0;
      __syncthreads();
      for (int j = tid; j < n; j += kThreads) {
        const unsigned k = key_of(j);
        if (shift == 24 || (k >> (shift + 8)) == (prefix >> (shift + 8))) atomicAdd(&hist[(k >> shift) & 255], 1);
      }
      __syncthreads();
      if (tid == 0) {
        int left = need, v = 255;
        while (v > 0 && hist[v] < left) left -= hist[v--];
        sPrefix = prefix | ((unsigned)v << shift);
        sNeed = left;
      }
      __syncthreads();
      prefix = sPrefix;
      need = sNeed;
    }
    // rows in order: ties up to `need`, holes in front of `keep`, movers behind it
    int ties = 0, holes = 0, movers = 0;
    int2* list = p.list + (long long)pair * (cap / 2);
    for (int j0 = 0; j0 < n; j0 += kThreads) {
      const int j = j0 + tid;
      const unsigned k = j < n ? key_of(j) : 0u;
      const bool tie = j < n && k == prefix;
      const unsigned long long bt = __ballot(tie);
      if (lane == 0) sWave[wave] = __popcll(bt);
      __syncthreads();
      int before = ties + __popcll(bt & ((1ull << lane) - 1)), all = 0;
      for (int v = 0; v < kWaves; ++v) {
        if (v < wave) before += sWave[v];
        all += sWave[v];
      }
      ties += all;
      const bool stays = j < n && (k > prefix || (tie && before < need));
      const bool hole = j < keep && !stays, mover = j >= keep && stays;
      const unsigned long long bh = __ballot(hole), bm = __ballot(mover);
      if (lane == 0) {
        sWave2[wave] = __popcll(bh);
        sWave3[wave] = __popcll(bm);
      }
      __syncthreads();
      int ih = holes + __popcll(bh & ((1ull << lane) - 1)), im = movers + __popcll(bm & ((1ull << lane) - 1));
      for (int v = 0; v < kWaves; ++v) {
        if (v < wave) {
          ih += sWave2[v];
          im += sWave3[v];
        }
        holes += sWave2[v];
        movers += sWave3[v];
      }
      if (hole) list[ih].y = j;
      if (mover) list[im].x = j;
      if (j < keep && stays) {
        p.pos_out[(long long)pair * cap + j] = pos[j];
        p.acc_out[(long long)pair * cap + j] = acc[j];
      }
    }
    if (tid == 0) p.moves[pair] = movers;
    __syncthreads();
    for (int i = tid; i < movers; i += kThreads) {     // what the moved rows carry; rows behind `keep` are never written
      const int2 m = list[i];
      p.pos_out[(long long)pair * cap + m.y] = pos[m.x];
      p.acc_out[(long long)pair * cap + m.y] = acc[m.x];
    }
  } else {
    for (int j = tid; j < n; j += kThreads) {
      p.pos_out[(long long)pair * cap + j] = pos[j];
      p.acc_out[(long long)pair * cap + j] = acc[j];
    }
    if (tid == 0) p.moves[pair] = 0;
  }
  if (tid == 0) p.row_cnt[pair] = keep;
}

// The rows that change places, K and V.  grid: (blocks, pairs)
template <int ROW_BYTES>
__global__ __launch_bounds__(256) void evict_move_kernel(EvictParams p) {
  constexpr int LPR = ROW_BYTES / 16, RPB = 256 / LPR;
  const int pair = blockIdx.y, cap = rows_cap(p.pg), moves = p.moves[pair];
  const int2* list = p.list + (long long)pair * (cap / 2);
  for (int i = blockIdx.x * RPB + threadIdx.x / LPR; i < moves; i += gridDim.x * RPB) {
    const int from = pool_row(p.pg, pair, list[i].x), to = pool_row(p.pg, pair, list[i].y);
    if (from < 0 || to < 0) continue;
    const long long s = (long long)from * LPR + threadIdx.x % LPR, d = (long long)to * LPR + threadIdx.x % LPR;
    const u32x4 k = static_cast<const u32x4*>(p.pg.K)[s], v = static_cast<const u32x4*>(p.pg.V)[s];
    static_cast<u32x4*>(p.pg.K)[d] = k;
    static_cast<u32x4*>(p.pg.V)[d] = v;
  }
}

}  // namespace

size_t paged_evict_ws(int pairs, int cap) {
  Arena a(nullptr);
  a.take<int>(pairs);
  a.take<int2>((size_t)pairs * (cap / 2));
  return a.used();
}

int run_paged_evict(int B, int Hkv, int D, int dtype, const Pages& pg, int budget, int n_sink, int n_recent, const int* seq_len,
                    const int* row_end, const int* row_pos, const float* acc, int* row_cnt, int* pos_out, float* acc_out,
                    void* ws, hipStream_t st) {
  const int pairs = B * Hkv, cap = rows_cap(pg);
  EvictParams p{};
  Arena a(ws);
  p.moves = a.take<int>(pairs);
  p.list = a.take<int2>((size_t)pairs * (cap / 2));
  p.pg = pg; p.Hkv = Hkv; p.budget = budget; p.n_sink = n_sink; p.n_recent = n_recent; p.seq_len = seq_len;
  p.row_end = row_end; p.row_pos = row_pos; p.acc = acc; p.row_cnt = row_cnt; p.pos_out = pos_out; p.acc_out = acc_out;
  evict_select_kernel<<<pairs, kThreads, 0, st>>>(p);
  OMNI_LAUNCH_CHECK();
  const int bytes = D * (dtype == OMNI_BF16 ? 2 : 4);
  const dim3 grid(std::max(1, std::min(cdiv(cap / 2, 256 / (bytes / 16)), 4096 / pairs)), pairs);
  if (bytes == 128) evict_move_kernel<128><<<grid, 256, 0, st>>>(p);
  else if (bytes == 256) evict_move_kernel<256><<<grid, 256, 0, st>>>(p);
  else evict_move_kernel<512><<<grid, 256, 0, st>>>(p);
  OMNI_LAUNCH_CHECK();
  return OMNI_OK;
}

}  // namespace omni
