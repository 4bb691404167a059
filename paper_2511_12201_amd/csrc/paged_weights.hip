// The weight that every cache row collects by a step of omni_paged_attn.
#include "paged_dev.h"

namespace omni {

namespace {

template <typename T>
__device__ __forceinline__ float to_f32(T x);
template <>
__device__ __forceinline__ float to_f32<float>(float x) { return x; }
template <>
__device__ __forceinline__ float to_f32<u16>(u16 x) { return bf16_bits_to_f32(x); }

constexpr int kWaves = 4, kThreads = kWaves * 64, kRows = kWaves * 32;

// Weights from the finished log-sum-exps: a wavefront owns 32 cache rows, all query rows of the pair pass by.
// grid: (blocks of kRows cache rows, pairs)
template <typename T, int D>
__global__ __launch_bounds__(kThreads) void paged_weights_f32_kernel(AttnParams p) {
  __shared__ float sQ[32 * (D + 4)], sL[32];
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
    const T* src = static_cast<const T*>(p.pg.K) + (long long)row * D + h * (D / 2);
#pragma unroll
    for (int e = 0; e < D / 2; ++e) k[e] = to_f32<T>(src[e]);
  }
  const float c2 = c.scale * kLog2e;
  float sum[16];
#pragma unroll
  for (int i = 0; i < 16; ++i) sum[i] = 0.f;
  constexpr int E = Elem<T>::kPer16B, CPR = D / E;
  for (int r0 = 0; r0 < w.M; r0 += 32) {
    __syncthreads();
    for (int i = threadIdx.x; i < 32 * CPR; i += kThreads) {
      const int r = r0 + i / CPR, cc = i % CPR, t = r / c.G, head = w.g * c.G + r % c.G;
      u32x4 raw = {0u, 0u, 0u, 0u};
      if (r < w.M)
        raw = *reinterpret_cast<const u32x4*>(static_cast<const T*>(p.Q) + w.b * c.qs[0] + head * c.qs[1] + t * c.qs[2] + cc * E);
      float x[E];
      unpack16(raw, x, (const T*)nullptr);
#pragma unroll
      for (int e = 0; e < E; ++e) sQ[(i / CPR) * (D + 4) + cc * E + e] = x[e];
    }
    if (threadIdx.x < 32) {
      const int r = r0 + threadIdx.x, t = r / c.G, head = w.g * c.G + r % c.G;
      const float lse = r < w.M ? p.lse[((long long)w.b * c.Hq + head) * c.n_new + t] : -INFINITY;
      sL[threadIdx.x] = lse * kLog2e;
      sVis[threadIdx.x] = lse > -INFINITY ? w.visible(p, t) : 0;
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
    if (ln == 0 && j < w.end) {
      const long long at = (long long)w.pair * rows_cap(p.pg) + j;
      p.acc_out[at] = (p.acc_in ? p.acc_in[at] : 0.f) + v;
    }
  }
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

int launch_weights(const AttnParams& p, int dtype, hipStream_t st) {
  const int pairs = p.c.B * p.c.Hkv, cap = rows_cap(p.pg);
  if (p.logits) {
    paged_weights_logits_kernel<<<dim3(cdiv(cap, 32 * kLogitBlocks), pairs), kThreads, 0, st>>>(p);
  } else if (dtype == OMNI_BF16) {
    if (p.c.D == 128) paged_weights_f32_kernel<u16, 128><<<dim3(cdiv(cap, kRows), pairs), kThreads, 0, st>>>(p);
    else paged_weights_f32_kernel<u16, 64><<<dim3(cdiv(cap, kRows), pairs), kThreads, 0, st>>>(p);
  } else {
    if (p.c.D == 128) paged_weights_f32_kernel<float, 128><<<dim3(cdiv(cap, kRows), pairs), kThreads, 0, st>>>(p);
    else paged_weights_f32_kernel<float, 64><<<dim3(cdiv(cap, kRows), pairs), kThreads, 0, st>>>(p);
  }
  OMNI_LAUNCH_CHECK();
  return OMNI_OK;
}

}  // namespace omni
