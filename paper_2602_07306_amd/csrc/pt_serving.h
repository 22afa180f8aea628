// Internal declarations of the serving operators (paged cache, page copies, sampling): kernel arguments and launchers.
#ifndef PT_SERVING_H_
#define PT_SERVING_H_

#include "pt_internal.h"

// Bits of pt_paged_batch.status.
enum { PT_PAGED_BAD_PAGE = 1, PT_PAGED_BAD_LENGTH = 2 };

// The batch as the kernels see it: pt_paged_batch with its bounds resolved.
struct pt_paged_rows {
  const int32_t* row_start;
  const int32_t* kv_len;
  const int32_t* pages;
  int64_t pages_stride;
  int32_t* status;
  int32_t n_seqs, total_rows, max_q_len, max_kv_len, n_pages, page_shift;
};

struct pt_append_args {
  pt_paged_rows b;
  const void* q;
  void* q_out;
  const void* k;
  const void* v;
  int64_t q_rs, q_hs, qo_rs, qo_hs, k_rs, k_hs, v_rs, v_hs;   // row and head strides, elements
  void* kc;                                                  // the layer's pages
  void* vc;
  int64_t page_stride, head_stride, token_stride;
  int32_t H, Hkv, hd;
};

// How the rows of a batch's sequences are cut: rows (new row, head of the group) per tile, upper bound of the number of
// tiles, keys per range, upper bound of the number of ranges.
struct pt_paged_cut {
  int32_t tile_rows, tiles, chunk, n_splits;
};

struct pt_paged_attn_args {
  pt_paged_rows b;
  const void* q;
  void* o;
  const void* kc;
  const void* vc;
  int64_t q_rs, q_hs, o_rs, o_hs;
  int64_t page_stride, head_stride, token_stride;
  // What the ranges leave to be joined, class by class (of those that are cut): [cut[c].n_splits][part_rows[c]][H][hd] unscaled sums,
  // then [cut[c].n_splits][part_rows[c]][H] (reference of the exponents in binary orders, sum).
  float* part;
  int32_t part_rows[2];
  int32_t seq_rows;  // > 0: new row i of sequence b is row b * seq_rows + i of class 0's; else rows are those of the batch
  float scale_log2;  // |scale| * log2 e, or 1 where the scale is 0
  float q_sign;      // what the queries are multiplied with for that: 1, -1 or 0
  int32_t causal, H, Hkv, hd;
  // sequences of at most `few` packed rows are cut by cut[0] and go to the kernels that stream keys past few rows; the
  // others by cut[1], to the kernel whose wavefronts share key tiles.  cut[i].tiles is 0 where a class cannot occur.
  int32_t few;
  pt_paged_cut cut[2];
};

struct pt_paged_plan {
  int32_t few;
  pt_paged_cut cut[2];
  int32_t part_rows[2], seq_rows;
  size_t bytes;   // workspace
};

// Elements of the partials of a class that is cut, a multiple of 16 bytes.
__host__ __device__ inline int64_t pt_paged_part_size(int32_t n_splits, int32_t rows, int32_t H, int32_t hd) {
  return n_splits > 1 ? ((int64_t)n_splits * rows * H * (hd + 2) + 3) / 4 * 4 : 0;
}

int pt_launch_paged_append(const pt_append_args& a, const pt_rope* rope, int32_t dtype, hipStream_t s);
int pt_plan_paged_attn(int32_t dtype, int32_t hd, int32_t H, int32_t Hkv, const pt_paged_rows& b, pt_paged_plan* p);
int pt_launch_paged_attn(const pt_paged_attn_args& a, int32_t dtype, hipStream_t s);
int pt_launch_page_copy(const pt_paged_cache& c, const int32_t* pairs, int32_t n, hipStream_t s);
size_t pt_sample_workspace(int32_t rows, int32_t vocab);
struct pt_sample_args {
  const float* logits;
  int64_t row_stride;
  const float* uniform;
  const float* temperature;
  const int32_t* top_k;
  const float* top_p;
  const float* min_p;
  int32_t* out;
  void* ws;
  int32_t rows, vocab;
  int32_t parts, part_len;   // set by the launcher
};
int pt_launch_sample(const pt_sample_args& a, hipStream_t s);

#endif  // PT_SERVING_H_
