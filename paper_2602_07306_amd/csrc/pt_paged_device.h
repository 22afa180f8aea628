// Device-side helpers of the paged-cache kernels: which sequence a row or a tile of rows belongs to.
#ifndef PT_PAGED_DEVICE_H_
#define PT_PAGED_DEVICE_H_

#include "pt_device.h"
#include "pt_serving.h"

// What a kernel may rely on about one sequence, whatever the arrays say: rows inside the buffers, positions inside the table.
struct paged_seq {
  int first, n, kv;   // first row, rows, positions
};

__device__ __forceinline__ void paged_raise(const pt_paged_rows& b, int bit) {
  if (b.status) atomicOr(b.status, bit);
}

__device__ __forceinline__ paged_seq paged_load_seq(const pt_paged_rows& b, int seq) {
  const int r0 = b.row_start[seq], r1 = b.row_start[seq + 1], kv = b.kv_len[seq];
  paged_seq s;
  s.first = min(max(r0, 0), b.total_rows);
  s.n = min(max(r1, s.first), b.total_rows) - s.first;
  s.n = min(s.n, b.max_q_len);
  s.kv = min(max(kv, 0), b.max_kv_len);
  if (s.first != r0 || s.n != r1 - r0 || s.kv != kv) paged_raise(b, PT_PAGED_BAD_LENGTH);
  return s;
}

// The sequence that row `row` belongs to: how many sequences end at or before it.  64 ends are compared at a time (every lane
// of the wavefront must call this with the same row); n_seqs where the row lies behind the last sequence.
__device__ __forceinline__ int paged_find_row(const pt_paged_rows& b, int row) {
  const int lane = threadIdx.x & 63;
  for (int base = 0; base < b.n_seqs; base += 64) {
    const int i = base + lane;
    const uint64_t ended = __ballot(i < b.n_seqs && b.row_start[i + 1] <= row);
    const int n = min(64, b.n_seqs - base);
    if (ended != (n == 64 ? ~0ull : (1ull << n) - 1)) return base + __popcll(ended);
  }
  return b.n_seqs;
}

// Page of a position, as the table says; page 0 (and a raised status) where that is no page.
__device__ __forceinline__ int paged_checked(const pt_paged_rows& b, int page) {
  if ((unsigned)page < (unsigned)b.n_pages) return page;
  paged_raise(b, PT_PAGED_BAD_PAGE);
  return 0;
}

#endif  // PT_PAGED_DEVICE_H_
