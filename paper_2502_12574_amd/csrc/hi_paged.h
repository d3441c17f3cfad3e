// The page pool and the sequences of a step as the kernels take them.
#pragma once
#include <math.h>
#include "hi_device.h"
#include "hi_serve.h"

namespace hi {

struct PagedPool {
  char* pages; float* scales;
  int n_pages, heads, shift, bits;      // shift: log2 of the rows of a page
};
struct PagedSeqs {
  const int* table; const int* past; const int* starts;
  int n_seqs, table_pages, n_rows;
};

// Sequence s as the kernels see it: its first new row and how many (0: left out), its rows in the cache before them.
struct PagedSeq { int first, rows, past; };
__host__ __device__ __forceinline__ PagedSeq paged_seq(int past, int start, int end, int n_rows) {
  PagedSeq q;
  q.first = start < 0 ? 0 : start < n_rows ? start : n_rows;
  const int e = end < 0 ? 0 : end < n_rows ? end : n_rows;
  q.rows = past < 0 || e < q.first ? 0 : e - q.first;
  q.past = past < 0 ? 0 : past;
  return q;
}
__device__ __forceinline__ PagedSeq paged_seq_of(const PagedSeqs& b, int s) {
  return paged_seq(b.past[s], b.starts[s], b.starts[s + 1], b.n_rows);
}

// Sums of the lanes up to this one, inside the register file; the last lane has that of all.
__device__ __forceinline__ int sum_wave(int x) {
#define HI_DPP(ctrl, mask) x += __builtin_amdgcn_update_dpp(0, x, ctrl, mask, 0xf, false)
  HI_DPP(0x111, 0xf); HI_DPP(0x112, 0xf); HI_DPP(0x114, 0xf); HI_DPP(0x118, 0xf);      // 1, 2, 4, 8 lanes up within 16
  HI_DPP(0x142, 0xa); HI_DPP(0x143, 0xc);                                              // the sum of the 16, then of the 32 before
#undef HI_DPP
  return x;
}

// The rows of one head of a page from row r on, as a number of rows behind the pool's start (K; V lies a page's rows further on).
__device__ __forceinline__ int64_t paged_row(const PagedPool& p, int page, int head, int r) {
  return ((((int64_t)page * p.heads + head) * 2) << p.shift) + r;
}

hi_status paged_arguments(const hi_paged_cache* cache, const hi_paged_batch* batch, const char* what, PagedPool& pool, PagedSeqs& seqs);

}  // namespace hi
