// What the kernels of the paged token cache share: the view of one layer's pool and of a batch of sequences, and the mask.
#pragma once
#include "common.cuh"

namespace scalekv {
namespace paged {

// One layer of the pool.  Row r of page `page` for kv head h is row ((page * heads + h) << page_shift) + r of the K rows, of the V
// rows and, where rows are 8-bit codes, of the two arrays of scales.
struct Store {
  char *k_rows, *v_rows;
  float *k_scales, *v_scales;      // q8 only
  int n_pages, heads, page_shift;
  int *status;                     // sticky device status word
};

// A batch: the tokens of sequence b are rows starts[b] .. starts[b + 1] - 1 of the token tensors and the last positions of its
// lengths[b] cache entries.
struct Batch {
  const int *table;                // [n_seqs][table_ld], table_pages of them in use: page of every page_tokens positions
  const int *lengths, *starts;
  int table_ld, table_pages, n_seqs, n_tokens;
};

// [tokens][heads][head_dim] rows, strides in bytes
struct Rows {
  char *ptr;
  long long st, sh;
};

// The grid before this one in the stream has ended, and all that it wrote is there.  First of all in every kernel but for what needs no memory.  What is read
// behind it may have been written while this grid was there already, so nothing goes through the read-only path (__ldg, ld.global.nc), which is for memory that
// nobody writes as long as the grid lives.
__device__ __forceinline__ void wait_for_grid() { asm volatile("griddepcontrol.wait;" ::: "memory"); }
// The grid behind this one may be set up where it finds room.
__device__ __forceinline__ void next_grid() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }

// (a wait that gave up stays on record)
__device__ __forceinline__ void report(int *status) { atomicCAS(status, 0, kDevCheck); }

// Whether the starts of sequence b are out of order: from 0 to n_tokens, none below the one before it.
__device__ __forceinline__ bool starts_wrong(const Batch &bt, int b, int start, int end) {
  return start < 0 || end < start || end > bt.n_tokens || (b == 0 && start != 0) || (b == bt.n_seqs - 1 && end != bt.n_tokens);
}

// Page of position pos of sequence b, or -1 (reported) where the table has none.
__device__ __forceinline__ int page_of(const Store &s, const Batch &bt, int b, int pos) {
  const int i = pos >> s.page_shift;
  int page = -1;
  if (pos >= 0 && i < bt.table_pages) page = bt.table[(size_t)b * bt.table_ld + i];
  if ((unsigned)page >= (unsigned)s.n_pages) { report(s.status); return -1; }
  return page;
}

__device__ __forceinline__ size_t store_row(const Store &s, int page, int head, int pos) {
  return (((size_t)page * s.heads + head) << s.page_shift) + (size_t)(pos & ((1 << s.page_shift) - 1));
}

// Division of 0 <= x < 2^31 by a fixed divisor: x * floor(2^32 / d) / 2^32 is less than 1/2 below x / d, so at most one too small.
struct Divisor {
  unsigned mul;
  int d;
  static Divisor of(int d) { return {(unsigned)((1ull << 32) / (unsigned)d - (d == 1 ? 1 : 0)), d}; }
  __device__ __forceinline__ int div(int x) const {
    int q = (int)__umulhi((unsigned)x, mul);
    return x - q * d >= d ? q + 1 : q;
  }
};

}  // namespace paged
}  // namespace scalekv
