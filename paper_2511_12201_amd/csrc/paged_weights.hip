// The weight that every cache row collects by a step of omni_paged_attn.
#include "paged_dev.h"

namespace omni {

namespace {

constexpr int kWaves = 4, kThreads = kWaves * 64, kRows = kWaves * 32;

// Where the weights of a block of cache rows go: straight to acc_out, or, where the query rows are split, to a plane of their
// own, and paged_weights_sum_kernel adds the planes in their order.
__device__ __forceinline__ void put_weight(const AttnParams& p, const PairView& w, int j, float v) {
  const long long at = (long long)w.pair * rows_cap(p.pg) + j;
  if (p.w_splits > 1) p.w_part[(long long)blockIdx.z * p.c.B * p.c.Hkv * rows_cap(p.pg) + at] = v;
  else p.acc_out[at] = (p.acc_in ? p.acc_in[at] : 0.f) + v;
}
// The tiles of `rows` query rows that this workgroup goes through: those whose last token sees cache row j0, its share of them.
__device__ __forceinline__ void tile_range(const AttnParams& p, const PairView& w, int j0, int rows, int& begin, int& end) {
  const int t_first = p.c.causal ? max(0, j0 - (w.end - w.cnt)) : 0;
  const int first = (int)min((long long)t_first * p.c.G, (long long)w.M) / rows, n = cdiv(w.M, rows) - first;
  begin = first + (int)((long long)n * blockIdx.z / p.w_splits);
  end = first + (int)((long long)n * (blockIdx.z + 1) / p.w_splits);
}

// fp32.  Weights from the finished log-sum-exps: a wavefront owns 32 cache rows, the query rows pass by.
// grid: (blocks of kRows cache rows, pairs, splits of the query rows)
template <int D>
__global__ __launch_bounds__(kThreads) void paged_weights_f32_kernel(AttnParams p) {
  __shared__ __attribute__((aligned(16))) float sQ[32 * (D + 4)];
  __shared__ float sL[32];
  __shared__ int sVis[32];
  const Chunk& c = p.c;
  const PairView w(p, blockIdx.y);
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, ln = lane & 31, h = lane >> 5;
  const int j0 = blockIdx.x * kRows + wave * 32;
  if ((int)blockIdx.x * kRows >= w.end) return;
  const int row = j0 + ln < w.end ? pool_row(p.pg, w.pair, j0 + ln) : -1;
  const unsigned there = (unsigned)__ballot(row >= 0) >> (4 * h);
  float k[D / 2];
#pragma unroll
  for (int e = 0; e < D / 2; ++e) k[e] = 0.f;
  if (row >= 0) {
    const float* src = static_cast<const float*>(p.pg.K) + (long long)row * D + h * (D / 2);
#pragma unroll
    for (int e = 0; e < D / 2; e += 4) {
      const f32x4 x = *reinterpret_cast<const f32x4*>(src + e);
#pragma unroll
      for (int i = 0; i < 4; ++i) k[e + i] = x[i];
    }
  }
  const float c2 = c.scale * kLog2e;
  float sum[16];
#pragma unroll
  for (int i = 0; i < 16; ++i) sum[i] = 0.f;
  constexpr int CPR = D / 4;
  int t0, t1;
  tile_range(p, w, blockIdx.x * kRows, 32, t0, t1);
  for (int r0 = t0 * 32; r0 < t1 * 32; r0 += 32) {
    __syncthreads();
    for (int i = threadIdx.x; i < 32 * CPR; i += kThreads) {
      const int r = r0 + i / CPR;
      f32x4 x = {0.f, 0.f, 0.f, 0.f};
      long long at_lse;
      if (r < w.M) x = *reinterpret_cast<const f32x4*>(static_cast<const float*>(p.Q) + out_row(p, w, r, at_lse) + i % CPR * 4);
      *reinterpret_cast<f32x4*>(sQ + (i / CPR) * (D + 4) + i % CPR * 4) = x;
    }
    if (threadIdx.x < 32) {
      const int r = r0 + threadIdx.x;
      float lse = -INFINITY;
      long long at_lse;
      if (r < w.M) {
        out_row(p, w, r, at_lse);
        lse = p.lse[at_lse];
      }
      sL[threadIdx.x] = lse * kLog2e;
      sVis[threadIdx.x] = lse > -INFINITY ? w.visible(p, r / c.G) : 0;
    }
    __syncthreads();
    f32x16 s;
#pragma unroll
    for (int i = 0; i < 16; ++i) s[i] = 0.f;
#pragma unroll
    for (int e = 0; e < D / 2; e += 4) {
      const f32x4 q = *reinterpret_cast<const f32x4*>(sQ + ln * (D + 4) + h * (D / 2) + e);
#pragma unroll
      for (int x = 0; x < 4; ++x) s = __builtin_amdgcn_mfma_f32_32x32x2f32(k[e + x], q[x], s, 0, 0, 0);
    }
    const int vis = sVis[ln];
    const float ref = sL[ln];
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      const int key = 8 * (i / 4) + i % 4;
      if (j0 + 4 * h + key < vis && ((there >> key) & 1u)) sum[i] += fast_exp2(fmaf(s[i], c2, -ref));
    }
  }
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    float v = sum[i];
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor(v, o, 64);
    const int j = j0 + 8 * (i / 4) + 4 * h + i % 4;
    if (ln == 0 && j < w.end) put_weight(p, w, j, v);
  }
}

// bf16, many query rows.  A wavefront keeps 64 cache rows as fragments in registers and its 64 sums per lane-half; tiles of 64 query
// rows pass through LDS, two buffers, one barrier a tile.  Per 64 x 32 weights a wavefront issues 16 matrix instructions (512 cycles)
// and 32 times scale, 2^x and sum (768 cycles): the vector ALU bounds it, two wavefronts per SIMD overlap the two.
constexpr int kBfKeys = 64, kBfRows = kWaves * kBfKeys, kBfQ = 64;
template <int D>
__global__ __launch_bounds__(kThreads, 2) void paged_weights_bf16_kernel(AttnParams p) {
  constexpr int RB = D * 2, QP = RB + 16, CPR = D / 8, KS = D / 16, NL = kBfQ * CPR / kThreads;
  __shared__ __attribute__((aligned(16))) unsigned char sQ[2][kBfQ * QP];
  __shared__ long long sAt[2][kBfQ];
  __shared__ float sRef[4][kBfQ];
  __shared__ int sVis[4][kBfQ];
  const Chunk& c = p.c;
  const PairView w = PairView::uniform(p, blockIdx.y);
  if ((int)blockIdx.x * kBfRows >= w.end) return;
  const int wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6)), lane = lane_id(), ln = lane & 31, h = lane >> 5;
  const int j0 = blockIdx.x * kBfRows + wave * kBfKeys;
  const u16* Kp = static_cast<const u16*>(p.pg.K);
  const float c2 = c.scale * kLog2e;
  bf16x8 kf[2][KS];
  unsigned there[2];
#pragma unroll
  for (int kb = 0; kb < 2; ++kb) {
    const int j = j0 + kb * 32 + ln, row = j < w.end ? pool_row(p.pg, w.pair, j) : -1;
    there[kb] = (unsigned)__ballot(row >= 0);
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
      u32x4 raw = {0u, 0u, 0u, 0u};
      if (row >= 0) raw = *reinterpret_cast<const u32x4*>(Kp + (long long)row * D + ks * 16 + h * 8);
      kf[kb][ks] = __builtin_bit_cast(bf16x8, raw);
    }
  }
  const bool all_there = (there[0] & there[1]) == 0xffffffffu;
  float sum[2][16];
#pragma unroll
  for (int kb = 0; kb < 2; ++kb)
#pragma unroll
    for (int i = 0; i < 16; ++i) sum[kb][i] = 0.f;

  int t0, t1;
  tile_range(p, w, blockIdx.x * kBfRows, kBfQ, t0, t1);
  // Where the rows of a tile lie and what they see, by the first wavefront: its rows advance by a tile per call of meta_load, and what
  // it loads is written down a tile later, when it has arrived (a wait for it in between would be one for the query rows, too).
  int meta_t = (t0 * kBfQ + (int)threadIdx.x) / c.G, meta_h = (t0 * kBfQ + (int)threadIdx.x) - meta_t * c.G;
  const int step_t = kBfQ / c.G, step_h = kBfQ - step_t * c.G;
  long long m_at = 0;
  float m_lse = 0.f;
  int m_vis = 0;
  auto meta_load = [&](int tile) {
    if (threadIdx.x < kBfQ) {
      const bool real = tile < t1 && meta_t < w.cnt;
      const int t = real ? meta_t : 0, head = w.g * c.G + (real ? meta_h : 0);
      m_at = w.b * c.qs[0] + head * c.qs[1] + t * c.qs[2];
      m_lse = p.lse[((long long)w.b * c.Hq + head) * c.n_new + t];
      m_vis = real ? w.visible(p, t) : 0;
      meta_t += step_t;
      meta_h += step_h;
      if (meta_h >= c.G) {
        meta_h -= c.G;
        ++meta_t;
      }
    }
  };
  auto meta_write = [&](int tile) {
    if (threadIdx.x < kBfQ) {
      sAt[tile & 1][threadIdx.x] = m_at;
      sRef[tile & 3][threadIdx.x] = m_lse > -INFINITY ? m_lse * kLog2e : 0.f;
      sVis[tile & 3][threadIdx.x] = m_lse > -INFINITY ? m_vis : 0;
    }
  };
  u32x4 raw[NL];
  auto load = [&](int tile) {
#pragma unroll
    for (int i = 0; i < NL; ++i) {
      const int piece = i * kThreads + threadIdx.x;
      raw[i] = *reinterpret_cast<const u32x4*>(static_cast<const u16*>(p.Q) + sAt[tile & 1][piece / CPR] + piece % CPR * 8);
    }
  };
  if (t0 < t1) {
    meta_load(t0);
    meta_write(t0);
    meta_load(t0 + 1);
    meta_write(t0 + 1);
    __syncthreads();
    load(t0);
    meta_load(t0 + 2);
    __syncthreads();
  }
  // Scores of 32 query rows under the weights of the 32 before: each matrix instruction is followed by its share of the vector work.
  // (One after the other the two wavefronts of a SIMD, which the barrier keeps in step, are in the same phase: 223 us / W_US for 500 new
  // tokens in four sequences of 8200 to 16400 rows.)
  float ref_a = 0.f, ref_b = 0.f;
  f32x16 sa[2], sb[2];
#pragma unroll
  for (int kb = 0; kb < 2; ++kb)
#pragma unroll
    for (int i = 0; i < 16; ++i) sb[kb][i] = -INFINITY;
  auto add_weights = [&](const f32x16 (&s)[2], int x, float ref) { sum[x / 16][x % 16] += fast_exp2(fmaf(s[x / 16][x % 16], c2, -ref)); };
  auto block = [&](int tile, int qb, f32x16 (&s)[2], float& ref, const f32x16 (&old)[2], float old_ref) {
    const unsigned char* q = &sQ[tile & 1][(qb * 32 + ln) * QP + h * 16];
    const f32x16 zero16 = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    bf16x8 qf[2] = {*reinterpret_cast<const bf16x8*>(q), *reinterpret_cast<const bf16x8*>(q + 32)};
    constexpr int PER = 16 / KS;                         // weights per matrix instruction: 2 KS of them, 32 weights
#pragma unroll
    for (int x = 0; x < 2 * KS; ++x) {
      const int kb = x % 2, ks = x / 2;
      __builtin_amdgcn_sched_barrier(0);
      s[kb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf[kb][ks], qf[ks % 2], ks == 0 ? zero16 : s[kb], 0, 0, 0);
      if (kb == 1 && ks + 2 < KS) qf[ks % 2] = *reinterpret_cast<const bf16x8*>(q + (ks + 2) * 32);
#pragma unroll
      for (int e = 0; e < PER; ++e) {
        add_weights(old, x * PER + e, old_ref);
        asm volatile("" : "+v"(sum[(x * PER + e) / 16][(x * PER + e) % 16]));      // here, not behind the branch below
      }
    }
    __builtin_amdgcn_sched_barrier(0);
    ref = sRef[tile & 3][qb * 32 + ln];
    const int rel = sVis[tile & 3][qb * 32 + ln] - j0;
    if (!all_there || __any(rel < kBfKeys)) {
#pragma unroll
      for (int kb = 0; kb < 2; ++kb)
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          const int key = kb * 32 + 8 * (i / 4) + 4 * h + i % 4;
          if (key >= rel || !((there[kb] >> (key & 31)) & 1u)) s[kb][i] = -INFINITY;
        }
    }
  };
  for (int tile = t0; tile < t1; ++tile) {
#pragma unroll
    for (int i = 0; i < NL; ++i) {
      const int piece = i * kThreads + threadIdx.x;
      *reinterpret_cast<u32x4*>(&sQ[tile & 1][piece / CPR * QP + piece % CPR * 16]) = raw[i];
    }
    meta_write(tile + 2);
    if (tile + 1 < t1) load(tile + 1);
    meta_load(tile + 3);
    __syncthreads();
    block(tile, 0, sa, ref_a, sb, ref_b);
    block(tile, 1, sb, ref_b, sa, ref_a);
  }
#pragma unroll
  for (int x = 0; x < 32; ++x) add_weights(sb, x, ref_b);
#pragma unroll
  for (int kb = 0; kb < 2; ++kb)
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      float v = sum[kb][i];
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) v += __shfl_xor(v, o, 64);
      const int j = j0 + kb * 32 + 8 * (i / 4) + 4 * h + i % 4;
      if (ln == 0 && j < w.end) put_weight(p, w, j, v);
    }
}

// The planes of split query rows.  grid: (blocks of cache rows, pairs)
__global__ __launch_bounds__(kThreads) void paged_weights_sum_kernel(AttnParams p) {
  const PairView w(p, blockIdx.y);
  const int j = blockIdx.x * kThreads + threadIdx.x;
  if (j >= w.end) return;
  const long long at = (long long)w.pair * rows_cap(p.pg) + j, plane = (long long)p.c.B * p.c.Hkv * rows_cap(p.pg);
  float v = 0.f;
  for (int s = 0; s < p.w_splits; ++s) v += p.w_part[s * plane + at];
  p.acc_out[at] = (p.acc_in ? p.acc_in[at] : 0.f) + v;
}

// The same from scores that the pass over the cache has kept (few query rows): a wavefront takes 32 cache rows at a time, two
// query rows per load.  grid: (blocks of cache rows, pairs)
constexpr int kLogitBlocks = 16;                         // 32-row blocks of a workgroup
__global__ __launch_bounds__(kThreads) void paged_weights_logits_kernel(AttnParams p) {
  __shared__ float sL[32];
  const PairView w(p, blockIdx.y);
  const int first = blockIdx.x * kLogitBlocks;
  if (first * 32 >= w.end) return;
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, ln = lane & 31, h = lane >> 5;
  const int mfull = p.c.G * p.c.n_new, cap = rows_cap(p.pg);
  if (threadIdx.x < 32) {
    long long at_lse;
    float ref = 0.f;                                     // a query row that sees nothing: its scores are -inf, its weights 0
    if ((int)threadIdx.x < w.M) {
      out_row(p, w, threadIdx.x, at_lse);
      const float lse = p.lse[at_lse];
      if (lse > -INFINITY) ref = lse * kLog2e;
    }
    sL[threadIdx.x] = ref;
  }
  __syncthreads();
  for (int block = first + wave; block < min(first + kLogitBlocks, cdiv(w.end, 32)); block += kWaves) {
    const float* src = p.logits + ((long long)w.pair * cdiv(cap, 32) + block) * mfull * 32 + lane;
    const int j = block * 32 + ln;
    const long long at = (long long)w.pair * cap + j;
    const float before = h == 0 && j < w.end && p.acc_in ? p.acc_in[at] : 0.f;
    float sum = 0.f;
#pragma unroll 4
    for (int r = 0; r < w.M; r += 2)
      if (r + h < w.M) sum += fast_exp2(src[r * 32] - sL[r + h]);
    sum = pair_sum(sum);
    if (h == 0 && j < w.end) p.acc_out[at] = before + sum;
  }
}

}  // namespace

// Workgroups enough for the chip: where the cache rows give few, the query rows are split, a tile or more each.
int weight_splits(const Chunk& c, int dtype, int cap) {
  const long long blocks = (long long)c.B * c.Hkv * cdiv(cap, dtype == OMNI_BF16 ? kBfRows : kRows);
  const int tiles = cdiv(c.G * c.n_new, dtype == OMNI_BF16 ? kBfQ : 32);
  return (int)max(1ll, min(min((1535 + blocks) / blocks, 16ll), (long long)tiles));
}

int launch_weights(const AttnParams& p, int dtype, hipStream_t st) {
  const int pairs = p.c.B * p.c.Hkv, cap = rows_cap(p.pg);
  if (p.logits) {
    paged_weights_logits_kernel<<<dim3(cdiv(cap, 32 * kLogitBlocks), pairs), kThreads, 0, st>>>(p);
  } else if (dtype == OMNI_BF16) {
    const dim3 grid(cdiv(cap, kBfRows), pairs, p.w_splits);
    if (p.c.D == 128) paged_weights_bf16_kernel<128><<<grid, kThreads, 0, st>>>(p);
    else paged_weights_bf16_kernel<64><<<grid, kThreads, 0, st>>>(p);
  } else {
    const dim3 grid(cdiv(cap, kRows), pairs, p.w_splits);
    if (p.c.D == 128) paged_weights_f32_kernel<128><<<grid, kThreads, 0, st>>>(p);
    else paged_weights_f32_kernel<64><<<grid, kThreads, 0, st>>>(p);
  }
  OMNI_LAUNCH_CHECK();
  if (p.w_splits > 1) {
    paged_weights_sum_kernel<<<dim3(cdiv(cap, kThreads), pairs), kThreads, 0, st>>>(p);
    OMNI_LAUNCH_CHECK();
  }
  return OMNI_OK;
}

}  // namespace omni
