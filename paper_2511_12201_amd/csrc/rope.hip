// Rotary positions: omni_rope (forward and backward on a layer's Q and K) and omni_paged_append (a chunk's Q and K turned, K and
// V stored in the pages).
//
// A pair (u, v) of a head becomes (u cos a - v sin a, u sin a + v cos a), a = position * frequency.  Every element is read and
// written once, so memory bounds it; the angle belongs to (token, pair) and serves all heads.  A thread therefore owns eight
// pairs of one token, forms their cosines and sines once and walks over the heads: 16 elements of a head at a time, 16 bytes a
// load.  The angle is kept in turns: position * (frequency / 2 pi) in 64 bits, of which the fraction goes on in 32.  65536 tokens of 32
// heads of 128 elements in bf16: 193 us, 5.6 TB/s in and out, where a copy reaches 5.1.
#include <algorithm>

#include "paged.h"

namespace omni {

namespace {

constexpr int kThreads = 256;
constexpr double kInvTwoPi = 0.15915494309189535;

struct RopeParams {
  const void *Q, *K, *V;
  void *Qout, *Kout;
  Pages pg;
  const int* pos;                // omni_rope: [B, N] or null; append: [B], position of a chunk's first token
  const int *new_cnt, *row_cnt;  // append
  int *row_end, *row_pos;
  float* acc;
  int B, Hq, Hkv, N, rot, heads_per_block;   // rot 0: K goes to the pages as it is
  float sign, out_scale;
  long long qs[3], ks[3];
  double f[64];                  // turns per position of a pair
};

// 8 neighbours, 16 bytes (bf16) or two times 16 (fp32).  ONCE: what passes by does not push out what the caches hold.
template <bool ONCE>
__device__ __forceinline__ void load8(const u16* p, float (&x)[8]) {
  const u32x4* q = reinterpret_cast<const u32x4*>(p);
  u32x4 raw;
  if constexpr (ONCE) raw = __builtin_nontemporal_load(q);
  else raw = *q;
  unpack16(raw, x, p);
}
template <bool ONCE>
__device__ __forceinline__ void load8(const float* p, float (&x)[8]) {
  const f32x4 a = *reinterpret_cast<const f32x4*>(p), b = *reinterpret_cast<const f32x4*>(p + 4);
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    x[e] = a[e];
    x[4 + e] = b[e];
  }
}
template <bool ONCE>
__device__ __forceinline__ void store8(u16* p, const float (&x)[8]) {
  const u32x4 raw = {pack_bf16x2(x[0], x[1]), pack_bf16x2(x[2], x[3]), pack_bf16x2(x[4], x[5]), pack_bf16x2(x[6], x[7])};
  if constexpr (ONCE) __builtin_nontemporal_store(raw, reinterpret_cast<u32x4*>(p));
  else *reinterpret_cast<u32x4*>(p) = raw;
}
template <bool ONCE>
__device__ __forceinline__ void store8(float* p, const float (&x)[8]) {
  *reinterpret_cast<f32x4*>(p) = f32x4{x[0], x[1], x[2], x[3]};
  *reinterpret_cast<f32x4*>(p + 4) = f32x4{x[4], x[5], x[6], x[7]};
}

// grid: (blocks of tokens, blocks of heads, B); a block's threads: D / 16 chunks of each of its tokens
template <typename T, int D, bool INTER, bool APPEND, bool ONCE>
__global__ __launch_bounds__(kThreads) void rope_kernel(RopeParams p) {
  constexpr int CPT = D / 16;
  const int b = blockIdx.z;
  const int n = blockIdx.x * (kThreads / CPT) + threadIdx.x / CPT, c = threadIdx.x % CPT;
  if (n >= p.N) return;
  const int h_begin = blockIdx.y * p.heads_per_block;
  const int n_heads = p.Hq + (APPEND ? 2 : 1) * p.Hkv;
  const int h_end = min(h_begin + p.heads_per_block, n_heads);

  int cnt = p.N, cap = 0;
  if constexpr (APPEND) {
    cnt = clampi(p.new_cnt[b], 0, p.N);
    cap = rows_cap(p.pg);
    if (n == 0 && c == 0)
      for (int h = max(h_begin, p.Hq); h < min(h_end, p.Hq + p.Hkv); ++h) {
        const int pair = b * p.Hkv + h - p.Hq;
        const int have = clampi(p.row_cnt[pair], 0, cap);
        p.row_end[pair] = cnt > cap - have ? cap : have + cnt;
      }
    if (n >= cnt) return;
  }
  int position = n;
  if constexpr (APPEND) position = (int)((unsigned)p.pos[b] + (unsigned)n);
  else if (p.pos) position = p.pos[(long long)b * p.N + n];

  // where the chunk's two runs of eight lie, in the two halves of what is turned or of what is not: neighbouring threads have
  // neighbouring runs.  Turned, they are the members of eight pairs, or (pairs side by side) two times four pairs.
  const bool turned = c < p.rot / 16;
  const int at0 = turned ? 8 * c : p.rot + 8 * (c - p.rot / 16), at1 = at0 + (turned ? p.rot : D - p.rot) / 2;
  float cs[8], sn[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    cs[e] = 1.f;
    sn[e] = 0.f;
  }
  if (turned) {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const double turns = (double)position * p.f[INTER ? 4 * c + (e < 4 ? e : p.rot / 4 + e - 4) : 8 * c + e];
      float s, co;
      sincospif(2.f * (float)(turns - rint(turns)), &s, &co);
      cs[e] = co * p.out_scale;
      sn[e] = s * p.out_scale * p.sign;
    }
  }
  auto turn = [&](float (&a)[8], float (&d)[8]) {
    if (!turned) return;
    if constexpr (INTER) {
#pragma unroll
      for (int e = 0; e < 8; e += 2) {
        const float u = a[e], v = a[e + 1], w = d[e], x = d[e + 1];
        a[e] = u * cs[e / 2] - v * sn[e / 2];
        a[e + 1] = u * sn[e / 2] + v * cs[e / 2];
        d[e] = w * cs[4 + e / 2] - x * sn[4 + e / 2];
        d[e + 1] = w * sn[4 + e / 2] + x * cs[4 + e / 2];
      }
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float u = a[e], v = d[e];
        a[e] = u * cs[e] - v * sn[e];
        d[e] = u * sn[e] + v * cs[e];
      }
    }
  };

  for (int h = h_begin; h < h_end; ++h) {
    const T* src;
    T* dst;
    bool rotate = true;
    if (h < p.Hq) {
      const long long off = b * p.qs[0] + h * p.qs[1] + n * p.qs[2];
      if (APPEND && !p.Q) continue;
      src = static_cast<const T*>(p.Q) + off;
      dst = static_cast<T*>(p.Qout) + off;
    } else if constexpr (!APPEND) {
      const long long off = b * p.ks[0] + (h - p.Hq) * p.ks[1] + n * p.ks[2];
      src = static_cast<const T*>(p.K) + off;
      dst = static_cast<T*>(p.Kout) + off;
    } else {
      const bool is_v = h >= p.Hq + p.Hkv;
      const int g = h - p.Hq - (is_v ? p.Hkv : 0), pair = b * p.Hkv + g;
      const long long j = (long long)clampi(p.row_cnt[pair], 0, cap) + n;
      if (j >= cap) continue;
      if (!is_v && c == 0) {
        p.row_pos[(long long)pair * cap + j] = position;
        if (p.acc) p.acc[(long long)pair * cap + j] = 0.f;
      }
      const int row = pool_row(p.pg, pair, (int)j);
      if (row < 0) continue;
      src = static_cast<const T*>(is_v ? p.V : p.K) + b * p.ks[0] + g * p.ks[1] + n * p.ks[2];
      dst = static_cast<T*>(is_v ? p.pg.V : p.pg.K) + (long long)row * D;
      rotate = !is_v;
    }
    float a[8], d[8];
    load8<ONCE>(src + at0, a);
    load8<ONCE>(src + at1, d);
    if (rotate) turn(a, d);
    store8<ONCE>(dst + at0, a);
    store8<ONCE>(dst + at1, d);
  }
}

template <bool APPEND>
int launch(RopeParams& p, int dtype, int D, bool inter, hipStream_t st) {
  const int n_heads = p.Hq + (APPEND ? 2 : 1) * p.Hkv;
  const int blocks = cdiv(p.N, kThreads / (D / 16));
  // A thread walks over the heads with its angles in hand; where the tokens alone do not fill the chip (1024 workgroups), the heads
  // are split and the angles formed again.  us all heads in one thread / split: 1024 tokens of 4 heads in fp32 5.9 / 4.4, one token of
  // eight sequences, 36 heads to the pages, 19.7 / 5.2, 13312 tokens 56 / 51.
  p.heads_per_block = (int)std::max(1ll, std::min((long long)n_heads, (long long)n_heads * blocks * p.B / 1024));
  const dim3 grid(blocks, cdiv(n_heads, p.heads_per_block), p.B);
  // Beyond what the L2s hold (32 MB, in and out) the rows pass by once: 65536 tokens of 32 heads 205 / 194 us, 13312 tokens to the
  // pages 56 / 52.  Not where a line of 128 bytes takes two instructions (fp32, short heads, heads turned in part: 108 / 123).
  const bool once = dtype == OMNI_BF16 && D == 128 && p.rot == D && (long long)p.B * p.N * n_heads * D * 4 > 64ll << 20;
#define OMNI_ROPE(T, DD, I, O)                                  \
  if (D == DD && inter == I && once == O) rope_kernel<T, DD, I, APPEND, O><<<grid, kThreads, 0, st>>>(p)
#define OMNI_ROPE_T(T)                                          \
  OMNI_ROPE(T, 64, false, false); else OMNI_ROPE(T, 64, true, false); else OMNI_ROPE(T, 128, false, false); else OMNI_ROPE(T, 128, true, false)
  if (dtype == OMNI_BF16) {
    OMNI_ROPE(u16, 128, false, true);
    else OMNI_ROPE(u16, 128, true, true);
    else OMNI_ROPE_T(u16);
  } else {
    OMNI_ROPE_T(float);
  }
#undef OMNI_ROPE_T
#undef OMNI_ROPE
  OMNI_LAUNCH_CHECK();
  return OMNI_OK;
}

void set_plan(RopeParams& p, const omni_rope_desc& r, bool backward) {
  p.rot = r.rot_dim;
  p.sign = backward ? -1.f : 1.f;
  p.out_scale = r.out_scale;
  for (int i = 0; i < r.rot_dim / 2; ++i) p.f[i] = r.inv_freq[i] * kInvTwoPi;
}

}  // namespace

int run_rope(const omni_rope_desc& r, const Layer& L, int dtype, const void* Q, const void* K, const int* pos, bool backward,
             void* Qout, void* Kout, hipStream_t st) {
  RopeParams p{};
  set_plan(p, r, backward);
  p.Q = Q; p.K = K; p.Qout = Qout; p.Kout = Kout; p.pos = pos;
  p.B = L.B; p.Hq = L.Hq; p.Hkv = L.Hkv; p.N = L.N;
  for (int k = 0; k < 3; ++k) {
    p.qs[k] = L.qs[k];
    p.ks[k] = L.ks[k];
  }
  return launch<false>(p, dtype, L.D, r.interleaved != 0, st);
}

int run_paged_append(const Chunk& c, int dtype, const omni_rope_desc* r, const void* Q, const void* K, const void* V,
                     const Pages& pg, const int* pos, const int* new_cnt, const int* row_cnt, void* Qout, int* row_end,
                     int* row_pos, float* acc, hipStream_t st) {
  RopeParams p{};
  if (r) set_plan(p, *r, false);
  p.Q = Q; p.K = K; p.V = V; p.Qout = Qout; p.pg = pg; p.pos = pos; p.new_cnt = new_cnt; p.row_cnt = row_cnt;
  p.row_end = row_end; p.row_pos = row_pos; p.acc = acc;
  p.B = c.B; p.Hq = c.Hq; p.Hkv = c.Hkv; p.N = c.n_new;
  for (int k = 0; k < 3; ++k) {
    p.qs[k] = c.qs[k];
    p.ks[k] = c.ks[k];
  }
  return launch<true>(p, dtype, c.D, r && r->interleaved, st);
}

}  // namespace omni
