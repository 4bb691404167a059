// Attention of a chunk of new tokens over a paged cache (omni_paged_attn), and the weight that every row collects by it.
//
// The query heads of a KV head share its rows, so the unit of work is a pair (sequence, KV head) with G * new_cnt query rows:
// row r is token r / G, head r % G of the group.  Both products are formed transposed, S^T = K Q^T and O^T = V^T P^T: a lane
// owns one query row, the softmax statistics are per-lane scalars and the accumulators of S^T are the B operand of the second
// product as they stand.  Running maximum and sum, one pass over the rows; rows that are not there (behind the last one, or on a
// page that is missing) are read as zeros and masked.
#include "paged.h"

namespace omni {

namespace {

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;

struct AttnParams {
  const void* Q;
  void* O;
  float* lse;
  Pages pg;
  const int *row_end, *new_cnt;
  const float* acc_in;
  float* acc_out;
  Chunk c;
};

// Query rows and cache rows of a pair, and how many rows a query row sees.
struct PairView {
  int pair, b, g, cnt, end, M;
  __device__ __forceinline__ PairView(const AttnParams& p, int pair_) : pair(pair_) {
    b = pair / p.c.Hkv;
    g = pair - b * p.c.Hkv;
    cnt = clampi(p.new_cnt[b], 0, p.c.n_new);
    end = clampi(p.row_end[pair], 0, rows_cap(p.pg));
    M = cnt * p.c.G;
  }
  __device__ __forceinline__ int visible(const AttnParams& p, int t) const { return p.c.causal ? max(end - cnt + t + 1, 0) : end; }
};

template <typename T>
__device__ __forceinline__ float to_f32(T x);
template <>
__device__ __forceinline__ float to_f32<float>(float x) { return x; }
template <>
__device__ __forceinline__ float to_f32<u16>(u16 x) { return bf16_bits_to_f32(x); }

// Rows [j0, j0 + ROWS) of a pair as fp32 into LDS, pitch D + 4; what is not there as zeros.  Returns nothing; `there` gets a bit
// per row (ROWS = 32).
template <typename T, int D, int THREADS>
__device__ __forceinline__ void stage_rows(const Pages& pg, const void* store, int pair, int end, int j0, float* dst) {
  constexpr int E = Elem<T>::kPer16B, CPR = D / E;
  for (int i = threadIdx.x; i < 32 * CPR; i += THREADS) {
    const int r = i / CPR, c = i % CPR, j = j0 + r;
    const int row = j < end ? pool_row(pg, pair, j) : -1;
    float x[E];
    u32x4 raw = {0u, 0u, 0u, 0u};
    if (row >= 0) raw = *reinterpret_cast<const u32x4*>(static_cast<const T*>(store) + (long long)row * D + c * E);
    unpack16(raw, x, (const T*)nullptr);
#pragma unroll
    for (int e = 0; e < E; e += 4) *reinterpret_cast<f32x4*>(dst + r * (D + 4) + c * E + e) = f32x4{x[e], x[e + 1], x[e + 2], x[e + 3]};
  }
}

constexpr int kWaves = 4, kThreads = kWaves * 64, kRows = kWaves * 32;

// grid: (blocks of kRows query rows, pairs)
template <typename T, int D>
__global__ __launch_bounds__(kThreads) void paged_attn_f32_kernel(AttnParams p) {
  __shared__ float sK[32 * (D + 4)], sV[32 * (D + 4)];
  __shared__ unsigned sThere;
  const Chunk& c = p.c;
  const PairView w(p, blockIdx.y);
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, ln = lane & 31, h = lane >> 5;
  const int r = blockIdx.x * kRows + wave * 32 + ln;
  const int t = r / c.G, head = w.g * c.G + r % c.G;
  const bool in_chunk = t < c.n_new, real = t < w.cnt;
  const int vis = real ? w.visible(p, t) : 0;
  const int r_last = min((int)(blockIdx.x + 1) * kRows, w.M) - 1;
  const int keys = r_last >= (int)blockIdx.x * kRows ? w.visible(p, r_last / c.G) : 0;

  float q[D / 2];
#pragma unroll
  for (int k = 0; k < D / 2; ++k) q[k] = 0.f;
  const long long qoff = w.b * c.qs[0] + head * c.qs[1] + (long long)t * c.qs[2];
  if (real) {
    const T* src = static_cast<const T*>(p.Q) + qoff + h * (D / 2);
#pragma unroll
    for (int k = 0; k < D / 2; ++k) q[k] = to_f32<T>(src[k]);
  }
  const float c2 = c.scale * kLog2e;
  f32x16 o[D / 32];
#pragma unroll
  for (int db = 0; db < D / 32; ++db)
#pragma unroll
    for (int i = 0; i < 16; ++i) o[db][i] = 0.f;
  float m = -INFINITY, l = 0.f;

  for (int j0 = 0; j0 < keys; j0 += 32) {
    __syncthreads();
    stage_rows<T, D, kThreads>(p.pg, p.pg.K, w.pair, w.end, j0, sK);
    stage_rows<T, D, kThreads>(p.pg, p.pg.V, w.pair, w.end, j0, sV);
    if (wave == 0) {
      const bool is = lane < 32 && j0 + lane < w.end && pool_row(p.pg, w.pair, j0 + lane) >= 0;
      const unsigned bits = (unsigned)__ballot(is);
      if (lane == 0) sThere = bits;
    }
    __syncthreads();
    f32x16 s;
#pragma unroll
    for (int i = 0; i < 16; ++i) s[i] = 0.f;
#pragma unroll
    for (int k = 0; k < D / 2; k += 4) {
      const f32x4 kv = *reinterpret_cast<const f32x4*>(sK + ln * (D + 4) + h * (D / 2) + k);
#pragma unroll
      for (int e = 0; e < 4; ++e) s = __builtin_amdgcn_mfma_f32_32x32x2f32(kv[e], q[k + e], s, 0, 0, 0);
    }
    const unsigned there = sThere >> (4 * h);
    float mx = m;
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      const int key = 8 * (i / 4) + i % 4;                        // + 4 h
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
    for (int db = 0; db < D / 32; ++db) {
#pragma unroll
      for (int i = 0; i < 16; ++i) o[db][i] *= alpha;
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const float v = sV[(8 * (i / 4) + 4 * h + i % 4) * (D + 4) + db * 32 + ln];
        o[db] = __builtin_amdgcn_mfma_f32_32x32x2f32(v, s[i], o[db], 0, 0, 0);
      }
    }
  }
  if (!in_chunk) return;
  const float total = pair_sum(l), inv = total > 0.f ? 1.f / total : 0.f;
  T* dst = static_cast<T*>(p.O) + qoff;
#pragma unroll
  for (int db = 0; db < D / 32; ++db)
#pragma unroll
    for (int i = 0; i < 16; ++i) Elem<T>::store(dst + db * 32 + 8 * (i / 4) + 4 * h + i % 4, o[db][i] * inv);
  if (h == 0) p.lse[((long long)w.b * c.Hq + head) * c.n_new + t] = total > 0.f ? (m + log2f(total)) * kLn2 : -INFINITY;
}

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

template <typename T, int D>
int launch(const AttnParams& p, hipStream_t st) {
  const int pairs = p.c.B * p.c.Hkv;
  paged_attn_f32_kernel<T, D><<<dim3(cdiv(p.c.G * p.c.n_new, kRows), pairs), kThreads, 0, st>>>(p);
  OMNI_LAUNCH_CHECK();
  if (p.acc_out) {
    paged_weights_f32_kernel<T, D><<<dim3(cdiv(rows_cap(p.pg), kRows), pairs), kThreads, 0, st>>>(p);
    OMNI_LAUNCH_CHECK();
  }
  return OMNI_OK;
}

}  // namespace

size_t paged_attn_ws(const Chunk& c, int dtype, int weight_rows) { return 256; }

int run_paged_attn(const Chunk& c, int dtype, const void* Q, const Pages& pg, const int* row_end, const int* new_cnt, void* O,
                   float* lse, const float* acc_in, float* acc_out, void* ws, hipStream_t st) {
  AttnParams p{};
  p.Q = Q; p.O = O; p.lse = lse; p.pg = pg; p.row_end = row_end; p.new_cnt = new_cnt; p.acc_in = acc_in; p.acc_out = acc_out;
  p.c = c;
  if (dtype == OMNI_BF16) return c.D == 128 ? launch<u16, 128>(p, st) : launch<u16, 64>(p, st);
  return c.D == 128 ? launch<float, 128>(p, st) : launch<float, 64>(p, st);
}

}  // namespace omni
