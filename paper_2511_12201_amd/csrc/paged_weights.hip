// The weight that every cache row collects by a step of omni_paged_attn.
#include "paged_dev.h"

namespace omni {

namespace {

constexpr int kWaves = 4, kThreads = kWaves * 64, kRows = kWaves * 32;

// Work: a block of `keys` cache rows of a pair with the tiles of `rows` query rows whose last token sees its first row.  As in the
// attention kernels all (block, tile) units are one line cut into equal spans; a workgroup that has all tiles of a block writes
// its weights, else it leaves its part in a slot, and paged_weights_join_kernel adds the parts in their order.
struct PairBlocks {
  int tiles, whole, blocks, base;        // tiles of the pair; blocks that every token sees from the first row on; all blocks
  __device__ __forceinline__ PairBlocks(const AttnParams& p, const PairView& w, int keys, int rows) {
    tiles = cdiv(w.M, rows);
    blocks = w.M ? cdiv(w.end, keys) : 0;
    base = p.c.causal ? max(w.end - w.cnt, 0) : w.end;
    whole = min(blocks, base / keys + 1);
  }
  // first tile of a block behind `whole`: token j0 - base is the first one that sees row j0
  __device__ __forceinline__ int first_tile(const AttnParams& p, int block, int keys, int rows) const {
    return (int)((long long)max(block * keys - base, 0) * p.c.G / rows);
  }
  __device__ __forceinline__ u64 units(const AttnParams& p, int keys, int rows) const {
    u64 n = (u64)whole * tiles;
    for (int k = whole; k < blocks; ++k) n += tiles - first_tile(p, k, keys, rows);
    return n;
  }
};

struct WeightSegment {
  int pair, block, t0, t1, slot;
  bool whole;
};

template <int THREADS, typename F>
__device__ __forceinline__ void for_weight_segments(const AttnParams& p, Scan& s, int keys, int rows, F f) {
  const int pairs = p.c.B * p.c.Hkv, per = cdiv(pairs, THREADS);
  const int first = min((int)threadIdx.x * per, pairs);
  u64 own = 0;
  for (int i = first; i < min(first + per, pairs); ++i) own += PairBlocks(p, PairView(p, i), keys, rows).units(p, keys, rows);
  const u64 inc = wave_scan(own);
  if ((threadIdx.x & 63) == 63) s.wave[threadIdx.x >> 6] = inc;
  __syncthreads();
  u64 at = inc - own, total = 0;
#pragma unroll
  for (int v = 0; v < THREADS / 64; ++v) {
    if (v < (int)(threadIdx.x >> 6)) at += s.wave[v];
    total += s.wave[v];
  }
  Spans sp;
  sp.cut(total, gridDim.x, 1);
  if (total == 0 || (int)blockIdx.x >= sp.n) return;
  const int w = span_of(blockIdx.x, sp.n);
  const u64 begin = sp.start(w), end = sp.start(w + 1);
  if (begin >= at && begin < at + own) {
    for (int i = first;; ++i) {
      const u64 n = PairBlocks(p, PairView(p, i), keys, rows).units(p, keys, rows);
      if (begin < at + n) {
        s.item = i;
        break;
      }
      at += n;
    }
    s.at = begin - at;
  }
  __syncthreads();
  int pair = __builtin_amdgcn_readfirstlane(s.item);
  u64 off = wave_uniform(s.at);
  for (u64 pos = begin; pos < end; ++pair, off = 0) {
    const PairView view = PairView::uniform(p, pair);
    const PairBlocks pb(p, view, keys, rows);
    int block = 0, t = 0;
    if (pb.blocks == 0) continue;
    if (off < (u64)pb.whole * pb.tiles) {
      block = (int)(off / pb.tiles);
      t = (int)(off - (u64)block * pb.tiles);
    } else {
      off -= (u64)pb.whole * pb.tiles;
      block = pb.whole;
      for (int n; off >= (u64)(n = pb.tiles - pb.first_tile(p, block, keys, rows)); ++block) off -= n;
      t = pb.first_tile(p, block, keys, rows) + (int)off;
    }
    for (; block < pb.blocks && pos < end; ++block) {
      const int t_first = block < pb.whole ? 0 : pb.first_tile(p, block, keys, rows);
      if (t < t_first) t = t_first;
      const int take = (int)min((u64)(pb.tiles - t), end - pos);
      WeightSegment seg{pair, block, t, t + take, 2 * w + (pos == begin ? 0 : 1), t == t_first && t + take == pb.tiles};
      if (t == t_first && threadIdx.x == 0)
        p.w_joins[(long long)pair * p.w_blocks + block] = int4{w, seg.whole ? w : sp.owner(pos + (pb.tiles - t) - 1), seg.slot, 0};
      f(seg, view);
      pos += take;
      t = 0;
    }
  }
}

// Sum over the 32 lanes of a half wavefront, on the vector ALU; every lane gets it.
__device__ __forceinline__ float half_lanes_sum(float v) {
  v = row_lanes_sum<16>(v);
  const u32x2 r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return __uint_as_float(r.x) + __uint_as_float(r.y);
}

// A row's sum of this workgroup's tiles.
__device__ __forceinline__ void put_weight(const AttnParams& p, const WeightSegment& seg, int keys, int at_block, int j, float v) {
  if (seg.whole) {
    const long long at = (long long)seg.pair * rows_cap(p.pg) + j;
    p.acc_out[at] = (p.acc_in ? p.acc_in[at] : 0.f) + v;
  } else {
    p.w_part[(long long)seg.slot * keys + at_block] = v;
  }
}

// fp32.  A wavefront keeps 32 cache rows as operands in registers; tiles of 32 query rows pass through LDS, the next one on its way in
// registers.  The matrix instructions bound it (D / 2 of 64 cycles per 32 x 32 weights).
template <int D>
__global__ __launch_bounds__(kThreads) void paged_weights_f32_kernel(AttnParams p) {
  constexpr int CPR = D / 4, NL = 32 * CPR / kThreads, PITCH = D + 4;
  __shared__ __attribute__((aligned(16))) float sQ[32 * PITCH];
  __shared__ float sL[32];
  __shared__ int sVis[32];
  __shared__ Scan scan;
  const Chunk& c = p.c;
  const int wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6)), lane = lane_id(), ln = lane & 31, h = lane >> 5;
  const float c2 = c.scale * kLog2e;
  for_weight_segments<kThreads>(p, scan, kRows, 32, [&](const WeightSegment& seg, const PairView& w) {
    f32x4 next[NL];
    float next_lse = -INFINITY;
    int next_vis = 0;
    auto load = [&](int r0) {                            // rows behind the last one as zeros, and nothing to see
      long long at_lse;
#pragma unroll
      for (int i = 0; i < NL; ++i) {
        const int piece = i * kThreads + threadIdx.x, r = r0 + piece / CPR;
        next[i] = f32x4{0.f, 0.f, 0.f, 0.f};
        if (r < w.M) next[i] = *reinterpret_cast<const f32x4*>(static_cast<const float*>(p.Q) + out_row(p, w, r, at_lse) + piece % CPR * 4);
      }
      if (threadIdx.x < 32) {
        const int r = r0 + threadIdx.x;
        next_lse = -INFINITY;
        if (r < w.M) {
          out_row(p, w, r, at_lse);
          next_lse = p.lse[at_lse];
        }
        next_vis = r < w.M ? w.visible(p, r / c.G) : 0;
      }
    };
    load(seg.t0 * 32);
    const int j0 = seg.block * kRows + wave * 32;
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
    float sum[16];
#pragma unroll
    for (int i = 0; i < 16; ++i) sum[i] = 0.f;
    for (int tile = seg.t0; tile < seg.t1; ++tile) {
      __syncthreads();
#pragma unroll
      for (int i = 0; i < NL; ++i) {
        const int piece = i * kThreads + threadIdx.x;
        *reinterpret_cast<f32x4*>(sQ + piece / CPR * PITCH + piece % CPR * 4) = next[i];
      }
      if (threadIdx.x < 32) {
        sL[threadIdx.x] = next_lse * kLog2e;
        sVis[threadIdx.x] = next_lse == -INFINITY ? 0 : next_vis;
      }
      __syncthreads();
      if (tile + 1 < seg.t1) load((tile + 1) * 32);
      const f32x16 s = scores_f32<D>([&](int e, f32x4& kv, f32x4& qv) {
        kv = f32x4{k[e], k[e + 1], k[e + 2], k[e + 3]};
        qv = *reinterpret_cast<const f32x4*>(sQ + ln * PITCH + h * (D / 2) + e);
      });
      const int vis = sVis[ln];
      const float ref = sL[ln];
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const int key = 8 * (i / 4) + i % 4;             // + 4 h
        if (j0 + 4 * h + key < vis && ((there >> key) & 1u)) sum[i] += fast_exp2(fmaf(s[i], c2, -ref));
      }
    }
    float own = 0.f;                                     // lane ln of a half takes the sum of register ln
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      const float v = half_lanes_sum(sum[i]);
      own = ln == i ? v : own;
    }
    const int in_block = wave * 32 + 8 * (ln / 4) + 4 * h + ln % 4, j = seg.block * kRows + in_block;
    if (ln < 16 && j < w.end) put_weight(p, seg, kRows, in_block, j, own);
  });
}

// bf16, many query rows.  A wavefront keeps 64 cache rows as fragments in registers and its sums per lane half; tiles of 64 query
// rows go from memory straight into a ring of four LDS stages, three on their way while one is worked on, one barrier a tile.  The
// scores of 32 query rows are formed under the weights of the 32 before: per 64 x 32 weights a wavefront issues 16 matrix
// instructions (512 cycles) and 32 times scale, 2^x and sum (950 cycles with the four that each 2^x takes): the vector ALU bounds it.
// 500 new tokens in four sequences of 8200 to 16400 rows: 196 us, 114 if nothing but those instructions counted; the rest is what a
// block of cache rows costs to take up (11 us of the 65 us that its tiles take) and the second workgroup of a CU, which works alone
// once the first, older one is through.
constexpr int kBfKeys = 64, kBfRows = kWaves * kBfKeys, kBfQ = 64, kBfStages = 4;
template <int D>
__global__ __launch_bounds__(kThreads, 2) void paged_weights_bf16_kernel(AttnParams p) {
  constexpr int RB = D * 2, CPR = D / 8, KS = D / 16, RPI = 1024 / RB, NL = kBfQ * RB / 1024 / kWaves, LPT = NL + 1;
  constexpr int kTileBytes = kBfQ * RB;
  __shared__ __attribute__((aligned(1024))) unsigned char sQ[kBfStages * kTileBytes];
  __shared__ __attribute__((aligned(256))) float sLse[kBfStages][kWaves][kBfQ];       // a copy per wavefront: its own loads
  __shared__ Scan scan;
  const Chunk& c = p.c;
  const int wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6)), lane = lane_id(), ln = lane & 31, h = lane >> 5;
  const u16* Kp = static_cast<const u16*>(p.pg.K);
  const unsigned q_base = (unsigned)(size_t)(__attribute__((address_space(3))) unsigned char*)sQ;
  const unsigned lse_base = (unsigned)(size_t)(__attribute__((address_space(3))) float*)&sLse[0][wave][0];
  const float c2 = c.scale * kLog2e;
  // Steps of kCopyRows rows and of a tile: heads of the group, elements, elements where the head passes the last one.
  constexpr int kCopyRows = kWaves * RPI;
  const int copy_dh = kCopyRows % c.G, stat_dh = kBfQ % c.G;
  const long long copy_step = copy_dh * c.qs[1] + kCopyRows / c.G * c.qs[2], copy_wrap = copy_step - c.G * c.qs[1] + c.qs[2];
  const long long stat_step = (long long)stat_dh * c.n_new + kBfQ / c.G, stat_wrap = stat_step - (long long)c.G * c.n_new + 1;
  // the piece of its row that a lane copies: rows change the places of their pieces as in the attention kernels
  const int in_tile = wave * RPI + lane / CPR, piece = (lane % CPR) ^ (D == 128 ? in_tile & 15 : in_tile >> 1 & 7);
  typedef __attribute__((address_space(3))) bf16x8* lds_eights;
  for_weight_segments<kThreads>(p, scan, kBfRows, kBfQ, [&](const WeightSegment& seg, const PairView& w) {
    const int j0 = seg.block * kBfRows + wave * kBfKeys, t0 = seg.t0, t1 = seg.t1;
    // The row that this lane copies next and the log-sum-exp it copies next: place, and head of the group, moved on by fixed steps of
    // tokens and heads.  Rows behind the last one are copied from the pair's first.
    const u16* q_first = static_cast<const u16*>(p.Q) + w.b * c.qs[0] + w.g * c.G * c.qs[1] + piece * 8;
    const float* lse_first = p.lse + ((long long)w.b * c.Hq + w.g * c.G) * c.n_new;
    int copy_row = t0 * kBfQ + wave * RPI + lane / CPR, stat_row = t0 * kBfQ + lane;
    int copy_h = copy_row % c.G, stat_h = stat_row % c.G;
    const u16* copy_at = q_first + copy_h * c.qs[1] + copy_row / c.G * c.qs[2];
    const float* stat_at = lse_first + (long long)stat_h * c.n_new + stat_row / c.G;
    auto issue = [&](int tile) {
      const int stage = tile % kBfStages;
#pragma unroll
      for (int i = 0; i < NL; ++i) {
        gload_lds16(copy_row < w.M ? copy_at : q_first, q_base + stage * kTileBytes + (i * kWaves + wave) * 1024);
        copy_row += kCopyRows;
        copy_h += copy_dh;
        const bool wrap = copy_h >= c.G;
        copy_h -= wrap ? c.G : 0;
        copy_at += wrap ? copy_wrap : copy_step;
      }
      gload_lds4(stat_row < w.M ? stat_at : lse_first, lse_base + stage * (kWaves * kBfQ * 4));
      stat_row += kBfQ;
      stat_h += stat_dh;
      const bool wrap = stat_h >= c.G;
      stat_h -= wrap ? c.G : 0;
      stat_at += wrap ? stat_wrap : stat_step;
    };
    __syncthreads();                                     // the segment before is done with the ring
    wait_vmcnt<0>();                                     // nothing older is counted below
    issue(t0);
    issue(t0 + 1);                                       // tiles behind the last one: nobody reads them
    issue(t0 + 2);
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
#pragma unroll
    for (int kb = 0; kb < 2; ++kb)
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) asm volatile("" : "+v"(kf[kb][ks]));          // loaded here, not waited for in the loop
    // from this tile on every query row sees all of this wavefront's 64 rows: token j0 + 63 - (end - cnt) sees the last one
    const int clear_t = c.causal ? max(0, j0 + kBfKeys - 1 - (w.end - w.cnt)) : 0;
    const int clear = (int)min(((long long)clear_t * c.G + kBfQ - 1) / kBfQ, (long long)t1);
    float sum[2][16];
#pragma unroll
    for (int kb = 0; kb < 2; ++kb)
#pragma unroll
      for (int i = 0; i < 16; ++i) sum[kb][i] = 0.f;
    float ref_a = 0.f, ref_b = 0.f;
    f32x16 sa[2], sb[2];
#pragma unroll
    for (int kb = 0; kb < 2; ++kb)
#pragma unroll
      for (int i = 0; i < 16; ++i) sb[kb][i] = -INFINITY;
    auto add_weights = [&](const f32x16 (&s)[2], int x, float ref) { sum[x / 16][x % 16] += fast_exp2(fmaf(s[x / 16][x % 16], c2, -ref)); };
    auto block = [&](int tile, int qb, f32x16 (&s)[2], float& ref, const f32x16 (&old)[2], float old_ref) {
      const int stage = tile % kBfStages;
      const unsigned q = q_base + stage * kTileBytes + (qb * 32 + ln) * RB + ((h ^ (D == 128 ? ln & 15 : ln >> 1 & 7)) * 16);
      const f32x16 zero16 = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
      auto frag = [&](int ks) { return *(lds_eights)(size_t)(q ^ (ks * 32)); };
      bf16x8 qf[2] = {frag(0), frag(1)};
      constexpr int PER = 16 / KS;                       // weights per matrix instruction: 2 KS of them, 32 weights
#pragma unroll
      for (int x = 0; x < 2 * KS; ++x) {
        const int kb = x % 2, ks = x / 2;
        __builtin_amdgcn_sched_barrier(0);
        s[kb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf[kb][ks], qf[ks % 2], ks == 0 ? zero16 : s[kb], 0, 0, 0);
        if (kb == 1 && ks + 2 < KS) qf[ks % 2] = frag(ks + 2);
#pragma unroll
        for (int e = 0; e < PER; ++e) {
          add_weights(old, x * PER + e, old_ref);
          asm volatile("" : "+v"(sum[(x * PER + e) / 16][(x * PER + e) % 16]));      // here, not behind the branch below
        }
      }
      __builtin_amdgcn_sched_barrier(0);
      const float lse = sLse[stage][wave][qb * 32 + ln];
      ref = lse * kLog2e;
      if ((tile + 1) * kBfQ > w.M || !(lse > -INFINITY)) {
        // behind the last row, or a row that sees nothing: no weights; NaN: a NaN for every row that is not masked below
        const bool none = tile * kBfQ + qb * 32 + ln >= w.M || lse == -INFINITY;
        if (none || lse != lse) {
          ref = 0.f;
#pragma unroll
          for (int x = 0; x < 32; ++x) s[x / 16][x % 16] = none ? -INFINITY : lse;
        }
      }
      if (tile < clear) {
        const int rel = w.visible(p, (tile * kBfQ + qb * 32 + ln) / c.G) - j0 - 4 * h;
#pragma unroll
        for (int kb = 0; kb < 2; ++kb)
#pragma unroll
          for (int i = 0; i < 16; ++i)
            if (kb * 32 + 8 * (i / 4) + i % 4 >= rel) s[kb][i] = -INFINITY;
      }
    };
    for (int tile = t0; tile < t1; ++tile) {
      wait_vmcnt<2 * LPT>();                             // this wavefront's share of the tile has landed
      __syncthreads();                                   // and everyone's; the tile before is done with, its stage is free
      issue(tile + 3);
      block(tile, 0, sa, ref_a, sb, ref_b);
      block(tile, 1, sb, ref_b, sa, ref_a);
    }
    wait_vmcnt<0>();                                     // no copy is on its way into a ring that is not this segment's any more
#pragma unroll
    for (int x = 0; x < 32; ++x) add_weights(sb, x, ref_b);
    // lane ln of a half takes the sum of its row: block ln / 16, register ln % 16
    float own = 0.f;
#pragma unroll
    for (int kb = 0; kb < 2; ++kb)
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const float v = half_lanes_sum(sum[kb][i]);
        own = ln == kb * 16 + i ? v : own;
      }
    const int in_block = wave * kBfKeys + ln / 16 * 32 + 8 * (ln % 16 / 4) + 4 * h + ln % 4, j = seg.block * kBfRows + in_block;
    // a row that is not there entered as zeros: nobody attends it
    if (j < w.end) put_weight(p, seg, kBfRows, in_block, j, (ln < 16 ? there[0] : there[1]) >> (in_block & 31) & 1u ? own : 0.f);
  });
}

// Blocks whose tiles were split, and pairs without new tokens.  grid: (blocks of KEYS rows, pairs)
template <int KEYS>
__global__ __launch_bounds__(KEYS) void paged_weights_join_kernel(AttnParams p) {
  const PairView w(p, blockIdx.y);
  const int j = blockIdx.x * KEYS + threadIdx.x;
  if (j >= w.end) return;
  float v = 0.f;
  if (w.M) {
    const int4 join = p.w_joins[(long long)blockIdx.y * p.w_blocks + blockIdx.x];
    if (join.x == join.y) return;                        // one workgroup had all of it and wrote the rows
    for (int i = join.x; i <= join.y; ++i) v += p.w_part[(long long)(i == join.x ? join.z : 2 * i) * KEYS + threadIdx.x];
  }
  const long long at = (long long)blockIdx.y * rows_cap(p.pg) + j;
  p.acc_out[at] = (p.acc_in ? p.acc_in[at] : 0.f) + v;
}

// The same from scores that the pass over the cache has kept (few query rows).  A block of 32 cache rows is M rows of 32 scores: a lane
// takes 4 neighbours, so that one load is 8 query rows, and a wavefront works on four blocks at once; memory bounds it (117 MB in
// 30 us).  The scores are read once and as such (470 MB of four tokens: 623 / 586 us for the call).
// grid: (blocks of cache rows, pairs)
constexpr int kLogitBlocks = 4 * kWaves;                 // 32-row blocks of a workgroup
__global__ __launch_bounds__(kThreads) void paged_weights_logits_kernel(AttnParams p) {
  __shared__ float sL[32];
  const PairView w = PairView::uniform(p, blockIdx.y);
  if ((int)blockIdx.x * kLogitBlocks * 32 >= w.end) return;
  const int wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6)), lane = lane_id(), r0 = lane / 8, quad = lane % 8;
  const int mfull = p.c.G * p.c.n_new, cap = rows_cap(p.pg), blocks = cdiv(w.end, 32);
  const int first = blockIdx.x * kLogitBlocks + wave * 4;
  // the first eight rows' scores and the weights so far are on their way while the log-sum-exps arrive
  f32x4 x[4], sum[4];
  auto load = [&](int r) {
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      x[k] = f32x4{-INFINITY, -INFINITY, -INFINITY, -INFINITY};
      if (first + k < blocks && r < w.M)
        x[k] = __builtin_nontemporal_load(
            reinterpret_cast<const f32x4*>(p.logits + (((long long)w.pair * cdiv(cap, 32) + first + k) * mfull + r) * 32 + quad * 4));
    }
  };
  load(r0);
  // lanes 0..7 hold the four rows of the first block, 8..15 of the second, ..: block lane / 8 % 4
  const int j = (first + r0 % 4) * 32 + quad * 4;
  const long long at = (long long)w.pair * cap + j;
  f32x4 own = {0.f, 0.f, 0.f, 0.f};
  if (lane < 32 && p.acc_in && j + 3 < w.end) own = *reinterpret_cast<const f32x4*>(p.acc_in + at);
  else if (lane < 32 && p.acc_in)
    for (int e = 0; e < 4; ++e) own[e] = j + e < w.end ? p.acc_in[at + e] : 0.f;
  if (threadIdx.x < 32) {
    long long at_lse;
    float ref = 0.f;                                     // a query row that sees nothing: its scores are -inf, its weights 0
    if ((int)threadIdx.x < w.M) {
      out_row(p, w, threadIdx.x, at_lse);
      const float lse = p.lse[at_lse];
      if (lse != -INFINITY) ref = lse * kLog2e;
    }
    sL[threadIdx.x] = ref;
  }
  __syncthreads();
#pragma unroll
  for (int k = 0; k < 4; ++k) sum[k] = f32x4{0.f, 0.f, 0.f, 0.f};
  for (int r = r0; r < r0 + 32; r += 8) {
    if (r - r0 >= w.M) break;
    if (r != r0) load(r);
    const float ref = sL[r & 31];
#pragma unroll
    for (int k = 0; k < 4; ++k)
#pragma unroll
      for (int e = 0; e < 4; ++e) sum[k][e] += x[k][e] == -INFINITY ? 0.f : fast_exp2(x[k][e] - ref);     // not seen: 0 whatever the token's sum is
  }
  f32x4 mine = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int k = 0; k < 4; ++k)
#pragma unroll
    for (int e = 0; e < 4; ++e) {                        // over the eight rows: lanes 8, 16 and 32 apart
      float v = sum[k][e];
      v += __uint_as_float(dpp_or_zero<0x128, 0xf>(__float_as_uint(v)));
      const u32x2 s = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
      v = pair_sum(__uint_as_float(s.x) + __uint_as_float(s.y));
      mine[e] = r0 % 4 == k ? v : mine[e];
    }
  if (lane < 32) {
    own += mine;
    if (j + 3 < w.end) *reinterpret_cast<f32x4*>(p.acc_out + at) = own;
    else
      for (int e = 0; e < 4; ++e)
        if (j + e < w.end) p.acc_out[at + e] = own[e];
  }
}

}  // namespace

// What the pass needs: workgroups, blocks of a pair (rows_cap / the rows of a block), floats of the slots.
WeightPlan weight_plan(int dtype, int cap) {
  return dtype == OMNI_BF16 ? WeightPlan{512, cdiv(cap, kBfRows), (size_t)2 * 512 * kBfRows}
                            : WeightPlan{768, cdiv(cap, kRows), (size_t)2 * 768 * kRows};
}

int launch_weights(const AttnParams& p, int dtype, hipStream_t st) {
  const int pairs = p.c.B * p.c.Hkv, cap = rows_cap(p.pg);
  if (p.logits) {
    paged_weights_logits_kernel<<<dim3(cdiv(cap, 32 * kLogitBlocks), pairs), kThreads, 0, st>>>(p);
    OMNI_LAUNCH_CHECK();
    return OMNI_OK;
  }
  const WeightPlan pl = weight_plan(dtype, cap);
  const dim3 blocks(pl.blocks, pairs);
  if (dtype == OMNI_BF16) {
    if (p.c.D == 128) paged_weights_bf16_kernel<128><<<pl.n_wgs, kThreads, 0, st>>>(p);
    else paged_weights_bf16_kernel<64><<<pl.n_wgs, kThreads, 0, st>>>(p);
    OMNI_LAUNCH_CHECK();
    paged_weights_join_kernel<kBfRows><<<blocks, kBfRows, 0, st>>>(p);
  } else {
    if (p.c.D == 128) paged_weights_f32_kernel<128><<<pl.n_wgs, kThreads, 0, st>>>(p);
    else paged_weights_f32_kernel<64><<<pl.n_wgs, kThreads, 0, st>>>(p);
    OMNI_LAUNCH_CHECK();
    paged_weights_join_kernel<kRows><<<blocks, kRows, 0, st>>>(p);
  }
  OMNI_LAUNCH_CHECK();
  return OMNI_OK;
}

}  // namespace omni
