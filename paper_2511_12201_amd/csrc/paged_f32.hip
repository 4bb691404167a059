// omni_paged_attn in fp32, on the fp32 32x32x2 matrix instructions.
//
// S^T = K Q^T and O^T = V^T P^T: a lane owns one query row; lane half h takes the elements [h D/2, (h + 1) D/2) of the first
// product's sum, so that a lane reads its half of a K row 16 bytes at a time, and the accumulators of S^T are the second product's
// B operand as they stand (register i holds row 8 (i / 4) + 4 h + i % 4).  Two divisions of labour: four wavefronts of 32 query rows
// that share 32-row tiles of the cache, or, for pairs of at most 32 query rows, four wavefronts that take 32-row tiles of their own
// and join their states.  The matrix instructions bound it (64 cycles each, D of them per 32 x 32 tile): 256 tokens of 28 heads on 8192
// rows of 128 elements 268 us, 112 TFLOP/s of the 154 that a large product reaches.
#include "paged_dev.h"

namespace omni {

namespace {

constexpr int kWaves = 4, kThreads = kWaves * 64;

// SPLIT: the wavefronts split the cache rows (unit 128, tm 32), else the query rows (unit 32, tm 128)
template <int D, bool SPLIT>
__global__ __launch_bounds__(kThreads, SPLIT ? 1 : 2) void paged_attn_f32_kernel(AttnParams p) {
  constexpr int PITCH = D + 4, TILE = 32 * PITCH, NB = D / 32;
  constexpr int LOADERS = SPLIT ? 64 : kThreads;         // threads that stage a tile
  constexpr int CPR = D / 4, NL = 32 * CPR / LOADERS;    // 16-byte pieces of a row, of a tile per loader
  __shared__ __attribute__((aligned(16))) float sK[(SPLIT ? kWaves : 1) * TILE], sV[(SPLIT ? kWaves : 1) * TILE];
  __shared__ Scan scan;
  __shared__ float sM[kWaves][32], sL[kWaves][32];
  const Chunk& c = p.c;
  const int wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6)), lane = lane_id(), ln = lane & 31, h = lane >> 5;
  float* tk = sK + (SPLIT ? wave * TILE : 0);
  float* tv = sV + (SPLIT ? wave * TILE : 0);
  const int loader = SPLIT ? lane : (int)threadIdx.x;
  const float c2 = c.scale * kLog2e;

  for_segments<kThreads>(p, scan, [&](const Segment& seg) {
    const PairView w = seg.w;
    const int r = seg.r0 + (SPLIT ? 0 : wave * 32) + ln;
    const bool real = r < w.M;
    const int rc = min(r, w.M - 1);
    const int vis = w.visible(p, rc / c.G);
    long long at_lse;
    const long long at_row = out_row(p, w, rc, at_lse);
    float q[D / 2];
    const float* src = static_cast<const float*>(p.Q) + at_row + h * (D / 2);
#pragma unroll
    for (int k = 0; k < D / 2; k += 4) {
      const f32x4 x = *reinterpret_cast<const f32x4*>(src + k);
#pragma unroll
      for (int e = 0; e < 4; ++e) q[k + e] = x[e];
    }
    f32x16 o[NB];
#pragma unroll
    for (int db = 0; db < NB; ++db)
#pragma unroll
      for (int i = 0; i < 16; ++i) o[db][i] = 0.f;
    float m = -INFINITY, l = 0.f;

    f32x4 ak[NL], av[NL];
    unsigned there_next = 0u;
    // rows of the next tile into registers; what is not there as zeros, so that no weight of 0 meets a NaN
    auto fetch = [&](int j0) {
      const int row_mine = j0 + ln < w.end ? pool_row(p.pg, w.pair, j0 + ln) : -1;
      there_next = (unsigned)__ballot(row_mine >= 0);
#pragma unroll
      for (int i = 0; i < NL; ++i) {
        const int piece = i * LOADERS + loader;
        const int row = __shfl(row_mine, piece / CPR, 64);
        ak[i] = av[i] = f32x4{0.f, 0.f, 0.f, 0.f};
        if (row >= 0) {
          const long long at = (long long)row * D + piece % CPR * 4;
          ak[i] = *reinterpret_cast<const f32x4*>(static_cast<const float*>(p.pg.K) + at);
          av[i] = *reinterpret_cast<const f32x4*>(static_cast<const float*>(p.pg.V) + at);
        }
      }
    };
    const int step = SPLIT ? kWaves : 1;
    const int first = seg.u0 * step + (SPLIT ? wave : 0), last = seg.u1 * step;
    fetch(first * 32);
    for (int tile = first; tile < last; tile += step) {
      const int j0 = tile * 32;
      __syncthreads();                                   // (SPLIT: the same number of trips for every wavefront)
#pragma unroll
      for (int i = 0; i < NL; ++i) {
        const int piece = i * LOADERS + loader;
        *reinterpret_cast<f32x4*>(tk + piece / CPR * PITCH + piece % CPR * 4) = ak[i];
        *reinterpret_cast<f32x4*>(tv + piece / CPR * PITCH + piece % CPR * 4) = av[i];
      }
      const unsigned there = there_next >> (4 * h);
      __syncthreads();
      if (tile + step < last) fetch(j0 + 32 * step);
      f32x16 s = scores_f32<D>([&](int e, f32x4& kv, f32x4& qv) {
        kv = *reinterpret_cast<const f32x4*>(tk + ln * PITCH + h * (D / 2) + e);
        qv = f32x4{q[e], q[e + 1], q[e + 2], q[e + 3]};
      });
      float mx = m;
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const int key = 8 * (i / 4) + i % 4;             // + 4 h
        s[i] = j0 + 4 * h + key < vis && ((there >> key) & 1u) ? s[i] * c2 : -INFINITY;
        mx = fmaxf(mx, s[i]);
      }
      mx = pair_max(mx);
      const float ref = mx == -INFINITY ? 0.f : mx;
      const float alpha = fast_exp2(m - ref);
      float sum = 0.f;
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        s[i] = fast_exp2(s[i] - ref);
        sum += s[i];
      }
      l = fmaf(l, alpha, sum);
      m = mx;
#pragma unroll
      for (int db = 0; db < NB; ++db) {
#pragma unroll
        for (int i = 0; i < 16; ++i) o[db][i] *= alpha;
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          const float v = tv[(8 * (i / 4) + 4 * h + i % 4) * PITCH + db * 32 + ln];
          o[db] = __builtin_amdgcn_mfma_f32_32x32x2f32(v, s[i], o[db], 0, 0, 0);
        }
      }
    }
    float total = pair_sum(l);
    if constexpr (SPLIT) {                               // join the wavefronts in their order, through the tiles' space
      __syncthreads();
      if (h == 0) {
        sM[wave][ln] = m;
        sL[wave][ln] = total;
      }
      __syncthreads();
      float top = sM[0][ln];
#pragma unroll
      for (int v = 1; v < kWaves; ++v) top = fmaxf(top, sM[v][ln]);
      const float ref = top == -INFINITY ? 0.f : top, mine = fast_exp2(m - ref);
      total = 0.f;
#pragma unroll
      for (int v = 0; v < kWaves; ++v) total = fmaf(sL[v][ln], fast_exp2(sM[v][ln] - ref), total);
      m = top;
#pragma unroll
      for (int db = 0; db < NB; ++db)
#pragma unroll
        for (int i = 0; i < 16; i += 4)
          *reinterpret_cast<f32x4*>(tk + ln * PITCH + db * 32 + 2 * i + 4 * h) =
              f32x4{o[db][i] * mine, o[db][i + 1] * mine, o[db][i + 2] * mine, o[db][i + 3] * mine};
      __syncthreads();
      if (wave == 0) {
#pragma unroll
        for (int db = 0; db < NB; ++db)
#pragma unroll
          for (int i = 0; i < 16; i += 4) {
            f32x4 x = *reinterpret_cast<const f32x4*>(sK + ln * PITCH + db * 32 + 2 * i + 4 * h);
#pragma unroll
            for (int v = 1; v < kWaves; ++v) x += *reinterpret_cast<const f32x4*>(sK + v * TILE + ln * PITCH + db * 32 + 2 * i + 4 * h);
#pragma unroll
            for (int e = 0; e < 4; ++e) o[db][i + e] = x[e];
          }
      }
      __syncthreads();                                   // the next segment's tiles take the space
      if (wave != 0) return;
    }
    if (!real) return;
    if (seg.whole) {
      const float inv = total == 0.f ? 0.f : 1.f / total;
      float* dst = static_cast<float*>(p.O) + at_row;
#pragma unroll
      for (int db = 0; db < NB; ++db)
#pragma unroll
        for (int i = 0; i < 16; i += 4)
          *reinterpret_cast<f32x4*>(dst + db * 32 + 2 * i + 4 * h) = f32x4{o[db][i] * inv, o[db][i + 1] * inv, o[db][i + 2] * inv, o[db][i + 3] * inv};
      if (h == 0) p.lse[at_lse] = total == 0.f ? -INFINITY : (m + log2f(total)) * kLn2;
    } else {
      const long long at = (long long)seg.slot * p.tm + r - seg.r0;
#pragma unroll
      for (int db = 0; db < NB; ++db)
#pragma unroll
        for (int i = 0; i < 16; i += 4)
          *reinterpret_cast<f32x4*>(p.part_o + at * D + db * 32 + 2 * i + 4 * h) = f32x4{o[db][i], o[db][i + 1], o[db][i + 2], o[db][i + 3]};
      if (h == 0) *reinterpret_cast<f32x2*>(p.part_ml + at * 2) = f32x2{m, total};
    }
  });
}

}  // namespace

int launch_attn_f32(const AttnParams& p, hipStream_t st) {
  if (p.tm == 32) {
    if (p.c.D == 128) paged_attn_f32_kernel<128, true><<<p.n_wgs, kThreads, 0, st>>>(p);
    else paged_attn_f32_kernel<64, true><<<p.n_wgs, kThreads, 0, st>>>(p);
  } else {
    if (p.c.D == 128) paged_attn_f32_kernel<128, false><<<p.n_wgs, kThreads, 0, st>>>(p);
    else paged_attn_f32_kernel<64, false><<<p.n_wgs, kThreads, 0, st>>>(p);
  }
  OMNI_LAUNCH_CHECK();
  return OMNI_OK;
}

}  // namespace omni
