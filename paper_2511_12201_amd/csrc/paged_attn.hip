// Attention of a chunk of new tokens over a paged cache (omni_paged_attn) in bf16, and what joins split items in both types.
//
// The query heads of a KV head share its rows, so the unit of work is a pair (sequence, KV head) with G * new_cnt query rows.
// Both products are formed transposed, S^T = K Q^T and O^T = V^T P^T, with 32x32x16 matrix instructions: a lane owns one query
// row, the softmax statistics are per-lane scalars and the accumulators of S^T are the second product's B operand as they stand.
// Running maximum and sum, one pass over the rows.  Rows that are not there (behind the last one, or on a page that is missing)
// enter as zeros and are masked.
//
//  * Few query rows a pair (paged_stream_kernel, at most 32): memory bounds it.  Every wavefront streams 32-row blocks of the
//    cache of its own through LDS; the states of a workgroup's wavefronts meet at an item's end.
//  * Many (paged_tile_kernel): eight wavefronts of 32 query rows share 64-row tiles that go from the pages straight into a ring
//    of four LDS stages, one barrier a tile; the softmax of a tile runs under the matrix instructions of the next.
// The second product takes a weight as two bf16 numbers (17 bits) where memory bounds it, and as one where the matrix instructions do
// (half a step: 2^-8 relative, the errors of many rows average out; two would cost 56 % of 2048 tokens on 65536 rows).  Their sum is
// taken before the rounding, in fp32.  Both kernels take the weights against the largest score so far: the weight of a
// row that stands out is then 1, which bf16 holds, and what one cache row dominates is that row's V.  (A value kept while scores rise
// leaves 2^x of some fraction x there, rounded above the line and not below: V off by its last bit.)
#include "paged_dev.h"

#include <type_traits>

namespace omni {

namespace {

typedef short s16x4 __attribute__((ext_vector_type(4)));

// ------------------------------------------------------------------ few query rows: stream the cache

// A wavefront takes 32 cache rows per trip, K and V straight from the pages into a ring of two LDS stages of its own: while one is
// worked on the other is on its way, 64 to 128 KB per CU in flight, and no barrier in the loop.  (Loads through registers, three
// workgroups a CU, kept less in flight: 131k rows of eight sequences and four KV heads of 128 elements, a token each, took 567 us
// with the weights, 416 now; 327 without them, 6.5 TB/s where a copy, which also writes, reaches 5.1.)  An instruction takes 1024
// bytes, whole rows of one page; the pieces of a row change places as in the tile kernel below.  Blocks with pages that are not there
// go through registers.
constexpr int kStreamWaves = 4, kStreamThreads = kStreamWaves * 64, kStreamRows = 32;

// where the 16-byte pieces of row r of a tile lie: piece c at c ^ swz(r)
template <int D>
__device__ __forceinline__ int swz_k(int row) { return D == 128 ? row & 15 : row >> 1 & 7; }
template <int D>
__device__ __forceinline__ int swz_v(int row) { return D == 128 ? (row & 3) << 2 : (row & 2) << 1; }

template <int D, bool LOGITS>
__global__ __launch_bounds__(kStreamThreads, 1) void paged_stream_kernel(AttnParams p) {
  constexpr int RB = D * 2, CPR = D / 8, RPI = 1024 / RB, NB = D / 32, KS = D / 16;
  constexpr int kKBytes = 32 * RB, kStageBytes = 2 * kKBytes, LPH = kKBytes / 1024;
  constexpr int kStores = LOGITS ? 1 : 0;                // store instructions of a trip, at least
  constexpr int kScoreBytes = 16 * 128;                  // scores of 16 query rows on their way out, of a wavefront
  constexpr int QP = RB + 16;                            // bytes between the queries
  constexpr int OP = 36;                                 // floats between the rows of the merge buffer (32 of the D elements at a time)
  __shared__ __attribute__((aligned(1024))) unsigned char ring[kStreamWaves * 2 * kStageBytes];
  // the queries, which go into registers; with LOGITS then the wavefronts' scores on their way out
  constexpr int kSharedBytes = LOGITS && kStreamWaves * kScoreBytes > 32 * QP ? kStreamWaves * kScoreBytes : 32 * QP;
  __shared__ __attribute__((aligned(16))) unsigned char sQ[kSharedBytes];
  __shared__ float sM[kStreamWaves][32], sL[kStreamWaves][32];
  __shared__ Scan scan;
  static_assert(kStreamWaves * 32 * OP * 4 <= (int)sizeof(ring), "the merge buffer takes the ring's place");
  const Chunk& c = p.c;
  const int wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6)), lane = lane_id(), n = lane & 31, h = lane >> 5;
  const float c2 = c.scale * kLog2e;
  const unsigned own_ring = (unsigned)(size_t)(__attribute__((address_space(3))) unsigned char*)ring + wave * 2 * kStageBytes;
  unsigned char* own_bytes = ring + wave * 2 * kStageBytes;
  const unsigned char* Kpool = static_cast<const unsigned char*>(p.pg.K);
  const unsigned char* Vpool = static_cast<const unsigned char*>(p.pg.V);
  const int in_row = lane / CPR, slot = lane % CPR;
  unsigned src_k[16 / RPI > 1 ? 4 : 1];                  // the K swizzle goes through 16 rows: 16 / RPI patterns
  constexpr int NP = 16 / RPI;
#pragma unroll
  for (int i = 0; i < NP; ++i) src_k[i] = in_row * RB + ((slot ^ swz_k<D>(i * RPI + in_row)) * 16);
  const unsigned src_v = in_row * RB + ((slot ^ swz_v<D>(in_row)) * 16);
  const unsigned frag_k = n * RB + ((h ^ swz_k<D>(n)) * 16);
  const unsigned frag_v = kKBytes + (4 * h + (n & 15) / 4) * RB + ((swz_v<D>((n & 15) / 4) + (n >> 4) * 2) * 16) + (n & 3) * 8;
  typedef __attribute__((address_space(3))) s16x4* lds_quads;
  typedef __attribute__((address_space(3))) bf16x8* lds_eights;
  const unsigned char* qlane = sQ + n * QP + h * 16;

  for_segments<kStreamThreads>(p, scan, [&](const Segment& seg) {
    const PairView w = seg.w;
    const int keys = w.visible(p, (w.M - 1) / c.G);
    const int first = seg.u0 * kStreamWaves + wave, last = min(seg.u1 * kStreamWaves, cdiv(keys, 32));
    // read only while the kernel runs: entries come through the scalar cache, so that no wait for them is one for the copies
    const auto* table = (const __attribute__((address_space(4))) int*)(p.pg.table + (long long)w.pair * p.pg.pages_cap);
    const int page_mask = (1 << p.pg.shift) - 1;
    // table entries of a block's two halves of 16 rows (each inside one page), and the pool row of a half, -1: not there
    auto entry = [&](int block, int half) {
      const int j = block * 32 + half * 16;
      return block < last && j < w.end ? (int)table[j >> p.pg.shift] : -1;
    };
    auto half_row = [&](int block, int half, int page) {
      return (unsigned)page < (unsigned)p.pg.n_pages ? (page << p.pg.shift) + ((block * 32 + half * 16) & page_mask) : -1;
    };
    // Rows pass by once, so they are loaded as such (one token of eight sequences on 131089 rows 378 / 338 us, 6.35 TB/s; with scores 506
    // / 453), unless scores are kept and the infinity cache holds most rows from call to call (131089 rows, 268 MB: 64 / 69).
    const bool once = !LOGITS || seg.total * (kStreamWaves * 32) * (2 * RB) > 320ull << 20;
    // K or V of a block into a stage
    auto issue = [&](auto is_k, int block, int stage, int row_a, int row_b) {
      constexpr bool kIsK = decltype(is_k)::value;
      const unsigned char* pool = kIsK ? Kpool : Vpool;
      const int at = stage * kStageBytes + (kIsK ? 0 : kKBytes);
      const int last_row = w.end - 1 - block * 32;       // of the block
      if (__builtin_expect(row_a >= 0 && row_b >= 0 && last_row >= 31, true)) {
#pragma unroll
        for (int i = 0; i < LPH; ++i) {
          const long long row = (long long)(i * RPI < 16 ? row_a : row_b) + i * RPI % 16;
          if (once) gload_lds16_once(pool + row * RB, kIsK ? src_k[i % NP] : src_v, own_ring + at + i * 1024);
          else gload_lds16(pool + row * RB, kIsK ? src_k[i % NP] : src_v, own_ring + at + i * 1024);
        }
      } else if (row_a >= 0 && (row_b >= 0 || last_row < 16)) {          // the last rows: behind the last one it again, which is masked
#pragma unroll
        for (int i = 0; i < LPH; ++i) {
          const int r = min(i * RPI + in_row, last_row);
          const unsigned piece = (kIsK ? src_k[i % NP] : src_v) - in_row * RB;
          gload_lds16(pool + ((long long)(r < 16 ? row_a : row_b) + r % 16) * RB + piece, own_ring + at + i * 1024);
        }
      } else {                                           // pages that are not there: zeros
#pragma unroll 1
        for (int i = 0; i < LPH; ++i) {
          const int r = i * RPI + in_row, from = r < 16 ? row_a : row_b;
          u32x4 x = {0u, 0u, 0u, 0u};
          if (from >= 0 && block * 32 + r < w.end) x = *reinterpret_cast<const u32x4*>(pool + ((long long)from + r % 16) * RB + slot * 16);
          *reinterpret_cast<u32x4*>(own_bytes + at + r * RB + (slot ^ (kIsK ? swz_k<D>(r) : swz_v<D>(r))) * 16) = x;
        }
        // every copy before ends here: a half that took no load of its own would be missing in the counts of the waits
        wait_vmcnt<0>();
      }
    };
    constexpr std::true_type kKeys{};
    constexpr std::false_type kValues{};
    int row_a = half_row(first, 0, entry(first, 0)), row_b = half_row(first, 1, entry(first, 1));
    __syncthreads();                                     // the last segment's queries and merge buffer are done with
    for (int i = threadIdx.x; i < 32 * CPR; i += kStreamThreads) {
      const int r = i / CPR;
      u32x4 raw = {0u, 0u, 0u, 0u};
      if (r < w.M) {
        long long at_lse;
        raw = *reinterpret_cast<const u32x4*>(static_cast<const u16*>(p.Q) + out_row(p, w, r, at_lse) + i % CPR * 8);
      }
      *reinterpret_cast<u32x4*>(sQ + r * QP + i % CPR * 16) = raw;
    }
    wait_vmcnt<0>();                                     // nothing older is counted below
    // K(0) V(0) K(1) V(1) .. are issued in this order, a block's K two trips ahead as soon as its stage's keys are read, its V as
    // soon as the values are: three halves of a stage or more are always on their way
    const int second = first + kStreamWaves;
    int row_a1 = half_row(second, 0, entry(second, 0)), row_b1 = half_row(second, 1, entry(second, 1));
    if (first < last) {
      issue(kKeys, first, 0, row_a, row_b);
      issue(kValues, first, 0, row_a, row_b);
    }
    if (second < last) {
      issue(kKeys, second, 1, row_a1, row_b1);
      issue(kValues, second, 1, row_a1, row_b1);
    }
    int page_a2 = entry(second + kStreamWaves, 0), page_b2 = entry(second + kStreamWaves, 1);
    const int vis = n < w.M ? w.visible(p, n / c.G) : 0;
    f32x16 o[NB];
#pragma unroll
    for (int db = 0; db < NB; ++db)
#pragma unroll
      for (int i = 0; i < 16; ++i) o[db][i] = 0.f;
    float m = -INFINITY, l = 0.f;
    __syncthreads();
    bf16x8 qf[KS];
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) qf[ks] = *reinterpret_cast<const bf16x8*>(qlane + ks * 32);
    if constexpr (LOGITS) __syncthreads();               // everyone has them
    int stage = 0;
    for (int block = first; block < last; block += kStreamWaves) {
      const unsigned there = ((row_a >= 0 ? 0xffffu : 0u) | (row_b >= 0 ? 0xffff0000u : 0u)) >> (4 * h);
      const bool next = block + kStreamWaves < last, next2 = block + 2 * kStreamWaves < last;
      // K of this block has landed: newer are its V, the next block and, from the second trip on, the stores of at least one trip
      if (!next) wait_vmcnt<LPH>();
      else if (block == first) wait_vmcnt<3 * LPH>();
      else wait_vmcnt<3 * LPH + kStores>();
      const unsigned base = own_ring + stage * kStageBytes;
      f32x16 s;
#pragma unroll
      for (int i = 0; i < 16; ++i) s[i] = 0.f;
      bf16x8 kf[KS];
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) kf[ks] = *(lds_eights)(size_t)((base + frag_k) ^ (ks * 32));
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");      // the keys are read: their stage is free
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf[ks], qf[ks], s, 0, 0, 0);
      const int row_a2 = half_row(block + 2 * kStreamWaves, 0, page_a2), row_b2 = half_row(block + 2 * kStreamWaves, 1, page_b2);
      page_a2 = entry(block + 3 * kStreamWaves, 0);
      page_b2 = entry(block + 3 * kStreamWaves, 1);
      if (next2) issue(kKeys, block + 2 * kStreamWaves, stage, row_a2, row_b2);
      const int rel = min(vis, w.end) - block * 32 - 4 * h;   // rows of this block from here on are not seen
      float mx = m;
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const int key = 8 * (i / 4) + i % 4;             // + 4 h
        s[i] = key < rel && ((there >> key) & 1u) ? s[i] * c2 : -INFINITY;
        mx = fmaxf(mx, s[i]);
      }
      if constexpr (LOGITS) {
        // through LDS, so that a store writes whole lines: rows of 32 scores, 8 of them per instruction (16 bytes a lane straight from
        // the accumulators, a quarter of a line per instruction: no faster here, but the pass that adds them up reads whole lines)
        unsigned char* out = sQ + wave * kScoreBytes;
        float* dst = p.logits + ((long long)w.pair * cdiv(rows_cap(p.pg), 32) + block) * (c.G * c.n_new) * 32;
#pragma unroll
        for (int half = 0; half < 2; ++half) {
          if (half * 16 >= w.M) break;
          if (n / 16 == half) {
#pragma unroll
            for (int i = 0; i < 16; i += 4)
              *reinterpret_cast<f32x4*>(out + n % 16 * 128 + ((i / 2 + h) ^ (n & 7)) * 16) = f32x4{s[i], s[i + 1], s[i + 2], s[i + 3]};
          }
#pragma unroll
          for (int k = 0; k < 2; ++k) {
            const int r = k * 8 + lane / 8;
            if (half * 16 + k * 8 >= w.M) break;
            const f32x4 x = *reinterpret_cast<const f32x4*>(out + r * 128 + ((lane ^ r) & 7) * 16);
            if (half * 16 + r < w.M) *reinterpret_cast<f32x4*>(dst + (half * 16 + r) * 32 + lane % 8 * 4) = x;
          }
        }
      }
      mx = pair_max(mx);
      const float ref = mx == -INFINITY ? 0.f : mx;
      const float alpha = mx == m ? 1.f : fast_exp2(m - ref);
      float sum = 0.f;
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        s[i] = fast_exp2(s[i] - ref);
        sum += s[i];
      }
      l = fmaf(l, alpha, sum);
      m = mx;
      if (__any(alpha != 1.f)) {
#pragma unroll
        for (int db = 0; db < NB; ++db)
#pragma unroll
          for (int i = 0; i < 16; ++i) o[db][i] *= alpha;
      }
      // a weight as two bf16 numbers: the matrix cores have the time here (one token of eight sequences on 131089 rows 325 / 327 us)
      union { bf16x8 v[2]; unsigned u[8]; } pf, rest;
#pragma unroll
      for (int i = 0; i < 16; i += 2) {
        const unsigned u = pf.u[i / 2] = pack_bf16x2(s[i], s[i + 1]);
        rest.u[i / 2] = pack_bf16x2(s[i] - __uint_as_float(u << 16), s[i + 1] - __uint_as_float(u & 0xffff0000u));
      }
      // V of this block has landed: newer are the next block, the K after it and this trip's stores
      if (next2) wait_vmcnt<3 * LPH + kStores>();
      else if (next) wait_vmcnt<2 * LPH>();
      else wait_vmcnt<0>();
      union { s16x4 q[2]; bf16x8 v; } vf[2][NB];
#pragma unroll
      for (int s2 = 0; s2 < 2; ++s2)
#pragma unroll
        for (int db = 0; db < NB; ++db) {
          const unsigned at = ((base + frag_v) ^ (db * 64)) + s2 * 16 * RB;
          vf[s2][db].q[0] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_quads)(size_t)at);
          vf[s2][db].q[1] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_quads)(size_t)(at + 8 * RB));
        }
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");      // and the values
      if (next2) issue(kValues, block + 2 * kStreamWaves, stage, row_a2, row_b2);
#pragma unroll
      for (int s2 = 0; s2 < 2; ++s2)
#pragma unroll
        for (int db = 0; db < NB; ++db) o[db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf[s2][db].v, pf.v[s2], o[db], 0, 0, 0);
#pragma unroll
      for (int s2 = 0; s2 < 2; ++s2)
#pragma unroll
        for (int db = 0; db < NB; ++db) o[db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf[s2][db].v, rest.v[s2], o[db], 0, 0, 0);
      row_a = row_a1;
      row_b = row_b1;
      row_a1 = row_a2;
      row_b1 = row_b2;
      stage ^= 1;
    }
    // join the wavefronts in their order, 32 elements of the rows at a time
    const float own = pair_sum(l);
    if (h == 0) {
      sM[wave][n] = m;
      sL[wave][n] = own;
    }
    __syncthreads();
    float top = sM[0][n];
#pragma unroll
    for (int v = 1; v < kStreamWaves; ++v) top = fmaxf(top, sM[v][n]);
    const float ref = top == -INFINITY ? 0.f : top, mine = fast_exp2(m - ref);
    float total = 0.f;
#pragma unroll
    for (int v = 0; v < kStreamWaves; ++v) total = fmaf(sL[v][n], fast_exp2(sM[v][n] - ref), total);
    const float inv = total == 0.f ? 0.f : 1.f / total;                 // a NaN among the scores stays one
    if (wave == 0 && h == 0 && n < w.M) {
      if (seg.whole) {
        long long at_lse;
        out_row(p, w, n, at_lse);
        p.lse[at_lse] = total == 0.f ? -INFINITY : (top + log2f(total)) * kLn2;
      } else {
        *reinterpret_cast<f32x2*>(p.part_ml + ((long long)seg.slot * kStreamRows + n) * 2) = f32x2{top, total};
      }
    }
    const float by = seg.whole ? mine * inv : mine;
    float* sO = reinterpret_cast<float*>(ring);          // a buffer per group of 32 elements where the ring has the space
    constexpr int kGroup = kStreamWaves * 32 * OP;
    static_assert(NB * kGroup * 4 <= (int)sizeof(ring), "");
#pragma unroll
    for (int db = 0; db < NB; ++db)
#pragma unroll
      for (int i = 0; i < 16; i += 4)
        *reinterpret_cast<f32x4*>(sO + db * kGroup + (wave * 32 + n) * OP + 2 * i + 4 * h) = f32x4{o[db][i] * by, o[db][i + 1] * by, o[db][i + 2] * by, o[db][i + 3] * by};
    __syncthreads();
    for (int i = threadIdx.x; i < w.M * (D / 4); i += kStreamThreads) {
      const int r = i / (D / 4), d = i % (D / 4) * 4, at = d / 32 * kGroup + r * OP + d % 32;
      f32x4 x = *reinterpret_cast<const f32x4*>(sO + at);
#pragma unroll
      for (int v = 1; v < kStreamWaves; ++v) x += *reinterpret_cast<const f32x4*>(sO + at + v * 32 * OP);
      if (seg.whole) {
        long long at_lse;
        u16* dst = static_cast<u16*>(p.O) + out_row(p, w, r, at_lse) + d;
        *reinterpret_cast<uint2*>(dst) = uint2{pack_bf16x2(x[0], x[1]), pack_bf16x2(x[2], x[3])};
      } else {
        *reinterpret_cast<f32x4*>(p.part_o + ((long long)seg.slot * kStreamRows + r) * D + d) = x;
      }
    }
  });
}

int launch_stream(const AttnParams& p, hipStream_t st) {
  if (p.c.D == 128) {
    if (p.logits) paged_stream_kernel<128, true><<<p.n_wgs, kStreamThreads, 0, st>>>(p);
    else paged_stream_kernel<128, false><<<p.n_wgs, kStreamThreads, 0, st>>>(p);
  } else {
    if (p.logits) paged_stream_kernel<64, true><<<p.n_wgs, kStreamThreads, 0, st>>>(p);
    else paged_stream_kernel<64, false><<<p.n_wgs, kStreamThreads, 0, st>>>(p);
  }
  OMNI_LAUNCH_CHECK();
  return OMNI_OK;
}

// ------------------------------------------------------------------ many query rows: tiles in LDS

// 512 threads = 8 wavefronts x 32 query rows.  K and V tiles of 64 rows go from the pages straight into LDS (global_load_lds), row by
// row: an instruction takes 4 (D = 128) or 8 (D = 64) whole rows, which lie in one page (page_rows >= 16), so that a page costs one
// wave-uniform table entry.  A row's 16-byte pieces change places inside the row as they are written (the lanes' addresses do it): K
// piece c of row r goes to c ^ (r % 16) (D = 64: c ^ (r / 2 % 8)), so that the 16 lanes that read one piece of 16 rows meet every
// bank once; V piece c to c ^ 4 (r % 4) (D = 64: c ^ 4 (r / 2 % 2)), so that the transposing reads of 4 rows do.  Ring of four
// stages, so up to three tiles are in flight while one is computed and one barrier per tile is enough; the waits are counted by hand
// (the compiler would wait for every load in flight).  2048 tokens of 28 heads on 65536 rows: 1.65 ms, 1.16 PFLOP/s of the 1.34 that
// a large product reaches; of it the maximum in every tile takes 0.08 (of 0.51 ms on 32768 rows of 64 elements 0.02; voted on at the end
// of a step, not under the second product, 0.04).  Tiles that are not whole (the last one, missing
// pages) are copied through registers with zeros for what is not there.
constexpr int kTileWaves = 8, kTileThreads = kTileWaves * 64, kTileRows = kTileWaves * 32;
constexpr int kTileKeys = 64, kStages = 4;
constexpr int kTab = 2048;                               // page table entries in LDS: 512 tiles of the smallest pages

template <int D>
__global__ __launch_bounds__(kTileThreads, 2) void paged_tile_kernel(AttnParams p) {
  constexpr int kKBytes = kTileKeys * D * 2, kStageBytes = 2 * kKBytes;
  constexpr int LPH = kKBytes / 1024 / kTileWaves, LPT = 2 * LPH;     // load instructions per wavefront: of K, of a tile
  constexpr int RB = D * 2, CPR = D / 8, RPI = 1024 / RB;             // bytes and pieces of a row, rows of a load instruction
  constexpr int NB = D / 32, KS = D / 16;
  constexpr int NQK = 2 * KS, NPV = 4 * NB;                           // matrix instructions of the two products of a tile
  constexpr int kAhead = 2;                                           // fragments are read this many of them ahead
  static_assert(LPH >= 1 && 32 % NQK == 0 && 32 % NPV == 0, "chunking of the copies and of the vector work");
  __shared__ __attribute__((aligned(1024))) unsigned char smem[kStages * kStageBytes];
  __shared__ int sTab[kTab];
  __shared__ int sMissing;
  __shared__ Scan scan;
  const Chunk& c = p.c;
  const int lane = lane_id(), wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6)), ln = lane & 31, h = lane >> 5;
  const float c2 = c.scale * kLog2e;
  const unsigned lds_base = (unsigned)(size_t)(__attribute__((address_space(3))) unsigned char*)smem;
  const unsigned char* Kpool = static_cast<const unsigned char*>(p.pg.K);
  const unsigned char* Vpool = static_cast<const unsigned char*>(p.pg.V);

  // a lane's source inside the rows that an instruction takes (the instruction's first row is a multiple of RPI = 4 or 8; for K
  // the row's low bits beyond that are the wavefront's)
  const int in_row = lane / CPR, slot = lane % CPR;
  const unsigned src_k = in_row * RB + ((slot ^ swz_k<D>(wave * RPI + in_row)) * 16);
  const unsigned src_v = in_row * RB + ((slot ^ swz_v<D>(in_row)) * 16);
  // a lane's fragments: K row ln (+ 32), piece 2 ks + h; V rows 4 h + .. (+ 8, 16 t), 16 bytes of a column group
  const unsigned frag_k = ln * RB + ((h ^ swz_k<D>(ln)) * 16);
  const unsigned frag_v = kKBytes + (4 * h + (ln & 15) / 4) * RB + ((swz_v<D>((ln & 15) / 4) + (ln >> 4) * 2) * 16) + (ln & 3) * 8;
  typedef __attribute__((address_space(3))) s16x4* lds_quads;
  typedef __attribute__((address_space(3))) bf16x8* lds_eights;
  const f32x16 zero16 = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};

  for_segments<kTileThreads>(p, scan, [&](const Segment& seg) {
    const PairView w = seg.w;
    const bool active = seg.r0 + wave * 32 < w.M;        // wave-uniform: the others only copy
    const int rc = min(seg.r0 + wave * 32 + ln, w.M - 1);
    const int qvis = w.visible(p, rc / c.G) - 4 * h;     // compared with rows of a tile that leave out 4 h
    const int seen_by_all = w.visible(p, seg.r0 / c.G);
    bf16x8 qf[KS];
    {
      long long at_lse;
      const u16* q = static_cast<const u16*>(p.Q) + out_row(p, w, rc, at_lse) + h * 8;
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) qf[ks] = *reinterpret_cast<const bf16x8*>(q + ks * 16);
    }

    f32x16 o[NB];
#pragma unroll
    for (int db = 0; db < NB; ++db) o[db] = zero16;
    float m_run = -INFINITY, l_run = 0.f, mc = 0.f;      // the row's largest score so far (mc: times c2, 0 if there is none yet)

    // stretches of the span whose table entries fit the window
    const int tiles_per_window = max(1, (int)min((long long)(kTab - 1) << p.pg.shift >> 6, (long long)0x3fffffff));
    for (int c0 = seg.u0, c1; c0 < seg.u1; c0 = c1) {
      c1 = min(seg.u1, c0 + tiles_per_window);
      const int nt = c1 - c0;
      const int tab0 = (c0 * kTileKeys) >> p.pg.shift;
      const int tab_end = min(cdiv(min(c1 * kTileKeys, w.end), 1 << p.pg.shift), p.pg.pages_cap);
      __syncthreads();                                   // everyone is done with the stretch before
      if (threadIdx.x == 0) sMissing = 0;
      __syncthreads();
      for (int i = threadIdx.x; i < tab_end - tab0; i += kTileThreads) {
        const int page = p.pg.table[(long long)w.pair * p.pg.pages_cap + tab0 + i];
        const bool there = (unsigned)page < (unsigned)p.pg.n_pages;
        sTab[i] = there ? page : -1;
        if (!there) sMissing = 1;
      }
      __syncthreads();
      // the loads of the queries end here: a wait for them inside the loop would wait for the copies in flight, too
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) asm volatile("" : "+v"(qf[ks]));
      const bool missing = __builtin_amdgcn_readfirstlane(sMissing) != 0;
      const int n_plain = missing ? 0 : min(nt, w.end / kTileKeys - c0);              // whole tiles come first
      const int n_full = missing ? 0 : min(seen_by_all / kTileKeys - c0, nt);         // tiles in which nothing is masked

      // a wavefront's share of a tile: LPH times RPI rows, K and V alike; `entry` is their page
      auto first_row = [&](int t, int part) { return (c0 + t) * kTileKeys + (part * kTileWaves + wave) * RPI; };
      auto entry = [&](int t, int part) { return sTab[(first_row(t, part) >> p.pg.shift) - tab0]; };
      auto bytes_at = [&](int t, int part, int page) {
        page = __builtin_amdgcn_readfirstlane(page);
        return (((long long)page << p.pg.shift) + (first_row(t, part) & ((1 << p.pg.shift) - 1))) * RB;
      };
      auto copy_part = [&](int t, int part, bool is_k, long long from) {     // one load instruction
        const unsigned dst = lds_base + (unsigned)(t % kStages) * kStageBytes + (part * kTileWaves + wave) * 1024;
        if (is_k) gload_lds16(Kpool + from, src_k, dst);
        else gload_lds16(Vpool + from, src_v, dst + kKBytes);
      };
      auto row_there = [&](int j) { return j < w.end ? sTab[(j >> p.pg.shift) - tab0] : -1; };
      auto copy_tile = [&](int t) {                      // a tile that is not whole; every load before ends here, as the counts of the waits assume
        unsigned char* dst = smem + (t % kStages) * kStageBytes;
        for (int i = threadIdx.x; i < kTileKeys * CPR; i += kTileThreads) {
          const int row = i / CPR, piece = i % CPR, j = (c0 + t) * kTileKeys + row;
          const int page = row_there(j);
          u32x4 k = {0u, 0u, 0u, 0u}, v = k;
          if (page >= 0) {
            const long long src = (((long long)page << p.pg.shift) + (j & ((1 << p.pg.shift) - 1))) * RB + piece * 16;
            k = *reinterpret_cast<const u32x4*>(Kpool + src);
            v = *reinterpret_cast<const u32x4*>(Vpool + src);
          }
          *reinterpret_cast<u32x4*>(dst + row * RB + (piece ^ swz_k<D>(row)) * 16) = k;
          *reinterpret_cast<u32x4*>(dst + kKBytes + row * RB + (piece ^ swz_v<D>(row)) * 16) = v;
        }
        wait_vmcnt<0>();
      };
      auto issue_tile = [&](int t) {
        if (t < n_plain) {
#pragma unroll
          for (int part = 0; part < LPH; ++part) {
            const long long from = bytes_at(t, part, entry(t, part));
            copy_part(t, part, true, from);
            copy_part(t, part, false, from);
          }
        } else {
          copy_tile(t);
        }
      };
      auto kfrag = [&](unsigned stage, int i) {
        const int kb = i % 2, ks = i / 2;
        return *(lds_eights)(size_t)(lds_base + ((stage + frag_k) ^ (ks * 32)) + kb * 32 * RB);
      };
      auto vfrag = [&](unsigned stage, int i) {
        const int t16 = i / NB, db = i % NB;
        const unsigned at = lds_base + ((stage + frag_v) ^ (db * 64)) + t16 * 16 * RB;
        union { s16x4 q[2]; bf16x8 v; } f;
        f.q[0] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_quads)(size_t)at);
        f.q[1] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_quads)(size_t)(at + 8 * RB));
        return f.v;
      };
      auto rescale = [&](float mloc) {
        const float m_new = fmaxf(m_run, mloc);
        const float m_ref = m_new == -INFINITY ? 0.f : m_new;
        const float alpha = fast_exp2((m_run - m_ref) * c2);
        l_run *= alpha;
#pragma unroll
        for (int db = 0; db < NB; ++db)
#pragma unroll
          for (int i = 0; i < 16; ++i) o[db][i] *= alpha;
        m_run = m_new;
        mc = m_ref * c2;
      };
      auto tile_max = [&](const f32x16 (&sn)[2]) {
        float mloc = sn[0][0];
#pragma unroll
        for (int kb = 0; kb < 2; ++kb)
#pragma unroll
          for (int i = 0; i < 16; i += 2) mloc = fmaxf(fmaxf(sn[kb][i], sn[kb][i + 1]), mloc);
        return mloc;
      };
      auto mask_tile = [&](f32x16 (&sn)[2], int t) {
        const int rel = qvis - (c0 + t) * kTileKeys;
        u64 there = ~0ull;
        if (missing) there = __ballot(row_there((c0 + t) * kTileKeys + lane) >= 0);
        there >>= 4 * h;
#pragma unroll
        for (int kb = 0; kb < 2; ++kb)
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            const int key = kb * 32 + 8 * (i / 4) + i % 4;
            if (key >= rel || !((there >> key) & 1u)) sn[kb][i] = -INFINITY;
          }
        return tile_max(sn);
      };
      auto weights = [&](const f32x16 (&sc)[2], int i, float& sum) {       // two weights, packed
        const float a = fast_exp2(fmaf(sc[i / 16][i % 16], c2, -mc)), b = fast_exp2(fmaf(sc[i / 16][i % 16 + 1], c2, -mc));
        sum += a;
        sum += b;
        return pack_bf16x2(a, b);
      };
      union PFrag { bf16x8 v[4]; unsigned u[16]; };
      // The pages of this wavefront's shares of kGroup tiles, a lane each: a look-up in every step would wait for the fragments on their
      // way (2048 tokens on 65536 rows: 1685 us; looked up a step ahead 1653; so 1628).
      constexpr int kGroup = 64 / LPH;
      int pages = 0;
      auto load_pages = [&](int t) { pages = entry(min(t + lane / LPH, n_plain - 1), lane % LPH); };
      if (n_plain > 0) load_pages(0);

      // One step: weights of tile t from sc and O += V(t) P(t); where there is a tile t + 1, its scores into sn under the
      // weights, and their maximum under the second product.  kSteady: there is one, and tile t + 3 is whole and issued here.
      auto step = [&](auto steady, f32x16 (&sc)[2], f32x16 (&sn)[2], int t) {
        constexpr bool kSteady = decltype(steady)::value;
        const bool has_next = kSteady || t + 1 < nt;
        const unsigned stage = (unsigned)(t % kStages) * kStageBytes, stage_n = (unsigned)((t + 1) % kStages) * kStageBytes;
        PFrag pf;
        float lsum = 0.f;
        long long from[LPH];                             // where the share of tile t + 3 begins
        bf16x8 vf[kAhead];
        constexpr int EQ = 32 / NQK;
        if (has_next) {
          if (kSteady || t + 2 < nt) wait_vmcnt<LPT>();  // this wavefront's share of tile t + 1 has landed
          else wait_vmcnt<0>();
          __syncthreads();                               // and everyone's; tile t - 1 is done with
          if (!kSteady && t + 3 < nt) issue_tile(t + 3);
          __builtin_amdgcn_sched_barrier(0);
          if (kSteady && (t + 3) % kGroup == 0) load_pages(t + 3);
#pragma unroll
          for (int part = 0; kSteady && part < LPH; ++part) from[part] = bytes_at(t + 3, part, __builtin_amdgcn_readlane(pages, (t + 3) % kGroup * LPH + part));
          bf16x8 kf[kAhead];
#pragma unroll
          for (int i = 0; i < kAhead; ++i) kf[i] = kfrag(stage_n, i);
#pragma unroll
          for (int i = 0; i < NQK; ++i) {
            __builtin_amdgcn_sched_barrier(0);
            sn[i % 2] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf[i % kAhead], qf[i / 2], i < 2 ? zero16 : sn[i % 2], 0, 0, 0);
            if (i + kAhead < NQK) kf[i % kAhead] = kfrag(stage_n, i + kAhead);
            else vf[i + kAhead - NQK] = vfrag(stage, i + kAhead - NQK);
#pragma unroll
            for (int e = 0; e < EQ; e += 2) pf.u[(i * EQ + e) / 2] = weights(sc, i * EQ + e, lsum);
            if (kSteady && i * LPH % NQK == 0) copy_part(t + 3, i * LPH / NQK, true, from[i * LPH / NQK]);
          }
        } else {
#pragma unroll
          for (int i = 0; i < kAhead; ++i) vf[i] = vfrag(stage, i);
#pragma unroll
          for (int i = 0; i < 32; i += 2) pf.u[i / 2] = weights(sc, i, lsum);
        }
        l_run += lsum;
        __builtin_amdgcn_s_setprio(0);
        float mloc = -INFINITY;
        constexpr int EV = 64 / NPV;                     // the maximum under the first half of the product, the vote before its end
        bool higher = false;
#pragma unroll
        for (int i = 0; i < NPV; ++i) {
          __builtin_amdgcn_sched_barrier(0);
          o[i % NB] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf[i % kAhead], pf.v[i / NB], o[i % NB], 0, 0, 0);
          if (i + kAhead < NPV) vf[i % kAhead] = vfrag(stage, i + kAhead);
#pragma unroll
          for (int e = 0; i < NPV / 2 && e < EV; e += 2) {
            const int x = i * EV + e;
            mloc = fmaxf(fmaxf(sn[x / 16][x % 16], sn[x / 16][x % 16 + 1]), mloc);
          }
          if (i == NPV * 3 / 4) higher = __any(mloc > m_run);
          if (kSteady && i * LPH % NPV == 0) copy_part(t + 3, i * LPH / NPV, false, from[i * LPH / NPV]);
        }
        __builtin_amdgcn_sched_barrier(0);
        __builtin_amdgcn_s_setprio(1);
        if (has_next) {
          if (t + 1 >= n_full) {
            mloc = mask_tile(sn, t + 1);
            higher = __any(mloc > m_run);
          }
          if (higher) rescale(pair_max(mloc));
        }
      };

      // At the top of step t the tiles up to t + 2 have been issued; after its barrier everyone is done with tile t - 1, whose
      // stage takes tile t + 3.
      wait_vmcnt<0>();                                   // nothing older is counted below
      issue_tile(0);
      if (nt > 1) issue_tile(1);
      if (nt > 2) issue_tile(2);
      if (nt > 2) wait_vmcnt<2 * LPT>();
      else if (nt > 1) wait_vmcnt<LPT>();
      else wait_vmcnt<0>();
      __syncthreads();
      if (active) {
        f32x16 sa[2], sb[2];
        sb[0] = zero16;
        sb[1] = zero16;
#pragma unroll
        for (int i = 0; i < NQK; ++i) sa[i % 2] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kfrag(0, i), qf[i / 2], i < 2 ? zero16 : sa[i % 2], 0, 0, 0);
        const float first = 0 >= n_full ? mask_tile(sa, 0) : tile_max(sa);
        if (__any(first > m_run)) rescale(pair_max(first));
        int t = 0;
        for (; t + 4 < n_plain; t += 2) {
          step(std::true_type{}, sa, sb, t);
          step(std::true_type{}, sb, sa, t + 1);
        }
        for (; t < nt; t += 2) {
          step(std::false_type{}, sa, sb, t);
          if (t + 1 < nt) step(std::false_type{}, sb, sa, t + 1);
        }
      } else {
        for (int t = 0; t + 1 < nt; ++t) {
          if (t + 2 < nt) wait_vmcnt<LPT>();
          else wait_vmcnt<0>();
          __syncthreads();
          if (t + 3 < nt) issue_tile(t + 3);
        }
      }
    }

    // the row's place formed anew: no register holds it across the loop
    const int row_out = seg.r0 + wave * 32 + (loop_lane() & 31);
    const float total = pair_sum(l_run);
    if (row_out >= w.M) return;
    long long at_lse;
    const long long at_row = out_row(p, w, row_out, at_lse);
    const float by = !seg.whole ? 1.f : total == 0.f ? 0.f : 1.f / total;
    const long long at_part = (long long)seg.slot * kTileRows + row_out - seg.r0;
#pragma unroll
    for (int db = 0; db < NB; ++db)
#pragma unroll
      for (int i = 0; i < 16; i += 4) {
        const int d = db * 32 + 2 * i + 4 * h;
        const f32x4 x = {o[db][i] * by, o[db][i + 1] * by, o[db][i + 2] * by, o[db][i + 3] * by};
        if (seg.whole)
          *reinterpret_cast<uint2*>(static_cast<u16*>(p.O) + at_row + d) = uint2{pack_bf16x2(x[0], x[1]), pack_bf16x2(x[2], x[3])};
        else
          *reinterpret_cast<f32x4*>(p.part_o + at_part * D + d) = x;
      }
    if (h == 0) {
      if (seg.whole) p.lse[at_lse] = total == 0.f ? -INFINITY : (m_run * c2 + log2f(total)) * kLn2;
      else *reinterpret_cast<f32x2*>(p.part_ml + at_part * 2) = f32x2{m_run * c2, total};
    }
  });
}

int launch_tiles(const AttnParams& p, hipStream_t st) {
  if (p.c.D == 128) paged_tile_kernel<128><<<p.n_wgs, kTileThreads, 0, st>>>(p);
  else paged_tile_kernel<64><<<p.n_wgs, kTileThreads, 0, st>>>(p);
  OMNI_LAUNCH_CHECK();
  return OMNI_OK;
}

// ------------------------------------------------------------------ items that were split, rows of the padding

// What the two kernels below share: the spans of an item, and where a row's part of a span lies.
struct Join {
  int w0, w1, slot0;
  __device__ __forceinline__ Join(const AttnParams& p, const PairView& w, int item, int r0) {
    const int4 j = r0 < w.M ? p.joins[item] : int4{0, 0, 0, 0};       // an item without rows has no entry
    w0 = __builtin_amdgcn_readfirstlane(j.x);
    w1 = __builtin_amdgcn_readfirstlane(j.y);
    slot0 = __builtin_amdgcn_readfirstlane(j.z);
  }
  __device__ __forceinline__ long long row(const AttnParams& p, int v, int rl) const { return (long long)(v == w0 ? slot0 : 2 * v) * p.tm + rl; }
};

constexpr int kCombineThreads = 256;

// Items of 256 or 128 rows, shared by few spans: 16 lanes a row, four rows a wavefront.  grid: (items, blocks of 16 rows of an item)
template <typename T, int D>
__global__ __launch_bounds__(kCombineThreads) void paged_combine_rows_kernel(AttnParams p) {
  constexpr int E = D / 16;
  const int item = blockIdx.x, pair = item / p.tiles_per_pair, r0 = (item - pair * p.tiles_per_pair) * p.tm;
  const PairView w = PairView::uniform(p, pair);
  const Join join(p, w, item, r0);
  const int rl = blockIdx.y * 16 + threadIdx.x / 16, r = r0 + rl, c = threadIdx.x % 16;
  // one span had all of the item and wrote its rows; rows of the padding get zeros
  if (rl >= p.tm || r >= p.c.G * p.c.n_new || (r < w.M && join.w0 == join.w1)) return;
  long long at_lse;
  T* dst = static_cast<T*>(p.O) + out_row(p, w, r, at_lse) + c * E;
  float m = -INFINITY, l = 0.f, x[E];
#pragma unroll
  for (int e = 0; e < E; ++e) x[e] = 0.f;
  if (r < w.M) {
#pragma unroll 4
    for (int v = join.w0; v <= join.w1; ++v) {           // running maximum: one pass, the loads of four parts at a time
      const long long at = join.row(p, v, rl);
      const f32x2 ml = *reinterpret_cast<const f32x2*>(p.part_ml + at * 2);
      f32x4 y[E / 4];
#pragma unroll
      for (int k = 0; k < E / 4; ++k) y[k] = *reinterpret_cast<const f32x4*>(p.part_o + at * D + c * E + 4 * k);
      const float top = fmaxf(m, ml[0]), ref = top == -INFINITY ? 0.f : top;
      const float old = fast_exp2(m - ref), add = fast_exp2(ml[0] - ref);
      l = l * old + ml[1] * add;
#pragma unroll
      for (int e = 0; e < E; ++e) x[e] = x[e] * old + y[e / 4][e % 4] * add;
      m = top;
    }
  }
  const float inv = l == 0.f ? 0.f : 1.f / l;
#pragma unroll
  for (int e = 0; e < E; ++e) x[e] *= inv;
  if constexpr (sizeof(T) == 2 && E == 8) {
    *reinterpret_cast<u32x4*>(dst) = u32x4{pack_bf16x2(x[0], x[1]), pack_bf16x2(x[2], x[3]), pack_bf16x2(x[4], x[5]), pack_bf16x2(x[6], x[7])};
  } else if constexpr (sizeof(T) == 2) {
    *reinterpret_cast<u32x2*>(dst) = u32x2{pack_bf16x2(x[0], x[1]), pack_bf16x2(x[2], x[3])};
  } else {
#pragma unroll
    for (int k = 0; k < E / 4; ++k) *reinterpret_cast<f32x4*>(dst + 4 * k) = f32x4{x[4 * k], x[4 * k + 1], x[4 * k + 2], x[4 * k + 3]};
  }
  if (c == 0) p.lse[at_lse] = l == 0.f ? -INFINITY : (m + log2f(l)) * kLn2;
}

// Items of up to 32 rows, shared by up to all spans: a workgroup a row, every fourth span a wavefront, the wavefronts in their order.
// grid: (items, rows of an item)
template <typename T, int D>
__global__ __launch_bounds__(kCombineThreads) void paged_combine_spans_kernel(AttnParams p) {
  constexpr int kWaves = kCombineThreads / 64, E = D / 64;
  __shared__ float sX[kWaves][D], sL[kWaves];
  const int item = blockIdx.x, wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6)), lane = lane_id();
  const PairView w = PairView::uniform(p, item / p.tiles_per_pair);
  const Join join(p, w, item, 0);                        // 32 rows: a pair is one item
  const int r = blockIdx.y;
  if (r < w.M && join.w0 == join.w1) return;
  long long at_lse;
  T* dst = static_cast<T*>(p.O) + out_row(p, w, r, at_lse) + lane * E;
  float m = -INFINITY, l = 0.f, x[E];
#pragma unroll
  for (int e = 0; e < E; ++e) x[e] = 0.f;
  if (r < w.M) {
    for (int v = join.w0 + lane; v <= join.w1; v += 64) m = fmaxf(m, p.part_ml[join.row(p, v, r) * 2]);
    m = wave_max(m);
    const float ref = m == -INFINITY ? 0.f : m;
#pragma unroll 8
    for (int v = join.w0 + wave; v <= join.w1; v += kWaves) {
      const long long at = join.row(p, v, r);
      const f32x2 ml = *reinterpret_cast<const f32x2*>(p.part_ml + at * 2);
      const float wgt = fast_exp2(ml[0] - ref);
      l = fmaf(ml[1], wgt, l);
#pragma unroll
      for (int e = 0; e < E; ++e) x[e] = fmaf(p.part_o[at * D + lane * E + e], wgt, x[e]);
    }
  }
#pragma unroll
  for (int e = 0; e < E; ++e) sX[wave][lane * E + e] = x[e];
  if (lane == 0) sL[wave] = l;
  __syncthreads();
  if (wave != 0) return;
#pragma unroll
  for (int v = 1; v < kWaves; ++v) {
    l += sL[v];
#pragma unroll
    for (int e = 0; e < E; ++e) x[e] += sX[v][lane * E + e];
  }
  const float inv = l == 0.f ? 0.f : 1.f / l;
#pragma unroll
  for (int e = 0; e < E; ++e) Elem<T>::store(dst + e, x[e] * inv);
  if (lane == 0) p.lse[at_lse] = l == 0.f ? -INFINITY : (m + log2f(l)) * kLn2;
}

// ------------------------------------------------------------------ which kernel, how many workgroups

struct Plan {
  int tm, unit, over, n_wgs, min_share;
  bool logits;                                           // scores of the pass are kept for the weights
};

// Pairs of at most 32 query rows stream the cache.  us a call, stream / tiles, 28 heads on 4: one token on 131089 rows 53 / 88, four
// tokens on 4109 rows 14 / 23, on 131089 of eight sequences 341 / 405, with weights 587 / 723; 32 heads on 4 of 64 elements, four
// tokens on 4109 rows 13 / 17, on 131089 of eight sequences 177 / 191.  Above, a stream would read the cache twice.
// Workgroups: what the chip holds at once (LDS: one a CU, two of the streams and of the fp32 tiles with their small stages).
Plan make_plan(const Chunk& c, int dtype, int weight_rows) {
  const bool few = c.G * c.n_new <= kStreamRows, bf16 = dtype == OMNI_BF16;
  Plan pl = few ? Plan{32, 128, 0, bf16 && c.D == 64 ? 512 : 256, 1, false}
                : bf16 ? Plan{256, 64, 5, 256, 4, false} : Plan{128, 32, 1, 512, 2, false};
  pl.logits = weight_rows > 0 && bf16 && few;
  return pl;
}

void carve(AttnParams& p, const Plan& pl, int dtype, int weight_rows, void* ws, size_t* bytes) {
  Arena a(ws);
  p.part_o = a.take<float>((size_t)2 * pl.n_wgs * pl.tm * p.c.D);
  p.part_ml = a.take<float>((size_t)2 * pl.n_wgs * pl.tm * 2);
  p.joins = a.take<int4>((size_t)p.c.B * p.c.Hkv * cdiv(p.c.G * p.c.n_new, pl.tm));
  p.logits = pl.logits ? a.take<float>((size_t)p.c.B * p.c.Hkv * cdiv(weight_rows, 32) * p.c.G * p.c.n_new * 32) : nullptr;
  if (weight_rows > 0 && !pl.logits) {
    const WeightPlan wp = weight_plan(dtype, weight_rows);
    p.w_blocks = wp.blocks;
    p.w_joins = a.take<int4>((size_t)p.c.B * p.c.Hkv * wp.blocks);
    p.w_part = a.take<float>(wp.part_floats);
  }
  if (bytes) *bytes = a.used();
}

}  // namespace

int launch_combine(const AttnParams& p, int dtype, hipStream_t st) {
  const int rows = min(p.tm, p.c.G * p.c.n_new);
#define OMNI_COMBINE(T, D)                                                                                          \
  (p.tm == 32 ? paged_combine_spans_kernel<T, D><<<dim3(p.n_items, rows), kCombineThreads, 0, st>>>(p)              \
              : paged_combine_rows_kernel<T, D><<<dim3(p.n_items, cdiv(rows, 16)), kCombineThreads, 0, st>>>(p))
  if (dtype == OMNI_BF16) {
    if (p.c.D == 128) OMNI_COMBINE(u16, 128);
    else OMNI_COMBINE(u16, 64);
  } else {
    if (p.c.D == 128) OMNI_COMBINE(float, 128);
    else OMNI_COMBINE(float, 64);
  }
#undef OMNI_COMBINE
  OMNI_LAUNCH_CHECK();
  return OMNI_OK;
}

size_t paged_attn_ws(const Chunk& c, int dtype, int weight_rows) {
  AttnParams p{};
  p.c = c;
  size_t bytes;
  carve(p, make_plan(c, dtype, weight_rows), dtype, weight_rows, nullptr, &bytes);
  return bytes;
}

int run_paged_attn(const Chunk& c, int dtype, const void* Q, const Pages& pg, const int* row_end, const int* new_cnt, void* O,
                   float* lse, const float* acc_in, float* acc_out, void* ws, hipStream_t st) {
  AttnParams p{};
  p.Q = Q; p.O = O; p.lse = lse; p.pg = pg; p.row_end = row_end; p.new_cnt = new_cnt; p.acc_in = acc_in; p.acc_out = acc_out;
  p.c = c;
  const int weight_rows = acc_out ? rows_cap(pg) : 0;
  const Plan pl = make_plan(c, dtype, weight_rows);
  carve(p, pl, dtype, weight_rows, ws, nullptr);
  p.tm = pl.tm;
  p.unit = pl.unit;
  p.over = pl.over;
  p.n_wgs = pl.n_wgs;
  p.min_share = pl.min_share;
  p.tiles_per_pair = cdiv(c.G * c.n_new, pl.tm);
  p.n_items = c.B * c.Hkv * p.tiles_per_pair;
  int rc;
  if (dtype == OMNI_F32) rc = launch_attn_f32(p, st);
  else if (pl.tm == 32) rc = launch_stream(p, st);
  else rc = launch_tiles(p, st);
  if (rc != OMNI_OK) return rc;
  rc = launch_combine(p, dtype, st);
  if (rc != OMNI_OK || !acc_out) return rc;
  return launch_weights(p, dtype, st);
}

}  // namespace omni
