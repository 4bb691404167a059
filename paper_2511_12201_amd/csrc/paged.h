// What the kernels on a paged cache share (append, attention of a chunk, eviction).
#pragma once

#include "common.h"
#include "kernels.h"

namespace omni {

// A pool of pages and the pages of every (sequence, KV head) pair.
struct Pages {
  void *K, *V;
  const int* table;              // [pairs, pages_cap]; entries outside [0, n_pages): pages that are not there
  int shift, pages_cap, n_pages;
};

__host__ __device__ inline int rows_cap(const Pages& pg) { return pg.pages_cap << pg.shift; }

// Row of the pool that holds row j of a pair (0 <= j < rows_cap), -1 if its page is not there.
__device__ __forceinline__ int pool_row(const Pages& pg, int pair, int j) {
  const int page = pg.table[(long long)pair * pg.pages_cap + (j >> pg.shift)];
  return (unsigned)page < (unsigned)pg.n_pages ? (page << pg.shift) + (j & ((1 << pg.shift) - 1)) : -1;
}

__device__ __forceinline__ int clampi(int x, int lo, int hi) { return min(max(x, lo), hi); }

struct Chunk {
  int B, Hq, Hkv, G, D, n_new, causal;
  float scale;
  long long qs[3], ks[3];
};

// rope.hip
int run_rope(const omni_rope_desc& r, const Layer& L, int dtype, const void* Q, const void* K, const int* pos, bool backward,
             void* Qout, void* Kout, hipStream_t st);
int run_paged_append(const Chunk& c, int dtype, const omni_rope_desc* r, const void* Q, const void* K, const void* V,
                     const Pages& pg, const int* pos, const int* new_cnt, const int* row_cnt, void* Qout, int* row_end,
                     int* row_pos, float* acc, hipStream_t st);

// paged_attn.hip
size_t paged_attn_ws(const Chunk& c, int dtype, int weight_rows);    // weight_rows: rows_cap if weights are wanted, else 0
int run_paged_attn(const Chunk& c, int dtype, const void* Q, const Pages& pg, const int* row_end, const int* new_cnt, void* O,
                   float* lse, const float* acc_in, float* acc_out, void* ws, hipStream_t st);

// evict.hip
size_t paged_evict_ws(int pairs, int cap);
int run_paged_evict(int B, int Hkv, int D, int dtype, const Pages& pg, int budget, int n_sink, int n_recent, const int* seq_len,
                    const int* row_end, const int* row_pos, const float* acc, int* row_cnt, int* pos_out, float* acc_out,
                    void* ws, hipStream_t st);

}  // namespace omni
