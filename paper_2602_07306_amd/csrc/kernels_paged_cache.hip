// Paged cache: appending a step's keys and values with the rotary positions, and copying pages.  Both only move memory;
// what bounds them is HBM for many rows or pages and latency for few.
#include <algorithm>

#include "pt_paged_device.h"

// ------------------------------------------------------------------------------------------------
// Append.  A workgroup owns one row and a range of its heads; a thread owns one unit of a head - VEC pairs of the HALF layout
// (two vectors of VEC elements, r/2 apart), VEC / 2 pairs of the INTERLEAVED one, or VEC copied elements - and keeps its unit
// from head to head, so that a pair's sine and cosine are formed once for all of them.  VEC elements are 16 bytes where
// the rotated part allows it (UNIT), else single pairs.
//
// Angles: turns = p * f / 2 pi in 64 bits (fp64 products run at the rate of unpacked fp32 ones here), of which the whole
// part and then the nearest quarter are taken off; the rest, within an eighth of a turn, goes through the Taylor series of
// sine and cosine in fp32 (first terms left out: 1.8e-9 and 1.2e-10 at pi / 4).
// Measured: 8192 rows of 64 + 16 heads of 128 (336 MB read and written) 62 us, 5.4 TB/s, where a large copy reaches 4.9 to 5.1;
// 64 rows of 128 + 32 heads 5.6 us, two thirds of it launch and the chain row -> sequence -> page -> store.
// ------------------------------------------------------------------------------------------------
__device__ __forceinline__ void sincos_turns(double t, float* s, float* c) {
  t -= rint(t);
  const double quarter = rint(4.0 * t);
  const float x = (float)(t - 0.25 * quarter) * 6.283185307179586f;
  const float z = x * x;
  const float sx = x * fmaf(z, fmaf(z, fmaf(z, fmaf(z, 1.0f / 362880, -1.0f / 5040), 1.0f / 120), -1.0f / 6), 1.0f);
  const float cx = fmaf(z, fmaf(z, fmaf(z, fmaf(z, fmaf(z, -1.0f / 3628800, 1.0f / 40320), -1.0f / 720), 1.0f / 24), -0.5f), 1.0f);
  const int k = (int)quarter & 3;
  const float a = k & 1 ? cx : sx, b = k & 1 ? sx : cx;
  *s = k & 2 ? -a : a;
  *c = (k + 1) & 2 ? -b : b;
}

template <typename T, int VEC>
struct chunk {
  T e[VEC];
};
template <typename T, int VEC>
__device__ __forceinline__ chunk<T, VEC> load_chunk(const T* p) {
  chunk<T, VEC> x;
  if constexpr (VEC * sizeof(T) == 16) {
    *(uint4*)x.e = *(const uint4*)p;
  } else {
#pragma unroll
    for (int i = 0; i < VEC; ++i) x.e[i] = p[i];
  }
  return x;
}
template <typename T, int VEC>
__device__ __forceinline__ void store_chunk(T* p, const chunk<T, VEC>& x) {
  if constexpr (VEC * sizeof(T) == 16) {
    *(uint4*)p = *(const uint4*)x.e;
  } else {
#pragma unroll
    for (int i = 0; i < VEC; ++i) p[i] = x.e[i];
  }
}

enum { ROT_HALF = PT_ROPE_HALF, ROT_INTERLEAVED = PT_ROPE_INTERLEAVED, ROT_NONE = 2 };

// One unit of a head: loaded, turned and stored.  `pairs`: units of pairs (HALF) or of rotated elements (INTERLEAVED).
template <typename T, int VEC, int ROT>
struct rot_unit {
  static constexpr int NP = ROT == ROT_HALF ? VEC : ROT == ROT_INTERLEAVED ? VEC / 2 : 1;   // pairs of a unit
  chunk<T, VEC> x[ROT == ROT_HALF ? 2 : 1];

  __device__ __forceinline__ void load(const T* head, int e0, int e1, bool rotated) {
    x[0] = load_chunk<T, VEC>(head + e0);
    if constexpr (ROT == ROT_HALF) {
      if (rotated) x[1] = load_chunk<T, VEC>(head + e1);
    }
  }
  __device__ __forceinline__ void turn(const float* s, const float* c) {
    if constexpr (ROT != ROT_NONE) {
#pragma unroll
      for (int i = 0; i < NP; ++i) {
        T& ta = ROT == ROT_HALF ? x[0].e[i] : x[0].e[2 * i];
        T& tb = ROT == ROT_HALF ? x[ROT == ROT_HALF ? 1 : 0].e[i] : x[0].e[2 * i + 1];
        const float a = elem<T>::ld(&ta), b = elem<T>::ld(&tb);
        elem<T>::st(&ta, a * c[i] - b * s[i]);
        elem<T>::st(&tb, b * c[i] + a * s[i]);
      }
    }
  }
  __device__ __forceinline__ void store(T* head, int e0, int e1, bool rotated) const {
    store_chunk<T, VEC>(head + e0, x[0]);
    if constexpr (ROT == ROT_HALF) {
      if (rotated) store_chunk<T, VEC>(head + e1, x[1]);
    }
  }
};

// units: per head; rot_units: of them rotated; e1_off: distance of a pair's elements (HALF).  Threads beyond units * slots idle.
template <typename T, int VEC, int ROT>
__global__ void __launch_bounds__(256) paged_append_kernel(const pt_append_args a, const pt_rope rope, int units, int rot_units, int heads_per_block) {
  constexpr int Q_BATCH = 4, KV_BATCH = 2;   // heads whose loads are issued together
  const int row = blockIdx.x, tid = threadIdx.x;
  const int seq = paged_find_row(a.b, row);
  if (seq >= a.b.n_seqs) return;             // behind the last sequence
  const paged_seq sq = paged_load_seq(a.b, seq);
  if (row < sq.first || row >= sq.first + sq.n) return;   // contradictory arrays only
  const int pos = sq.kv - sq.n + (row - sq.first);
  const int slots = 256 / units;
  const int slot = tid / units, u = tid - slot * units;
  if (slot >= slots) return;
  const bool rotated = u < rot_units;
  const int half = rope.rotary_dim / 2;
  // elements of the unit: rotated ones first, then the copied rest of the head
  const int e0 = ROT == ROT_HALF && !rotated ? rope.rotary_dim + (u - rot_units) * VEC : u * VEC;
  const int e1 = e0 + half;
  using unit = rot_unit<T, VEC, ROT>;
  float s[unit::NP], c[unit::NP];
  if (ROT != ROT_NONE && rotated) {
    const float m = (float)rope.magnitude;
#pragma unroll
    for (int i = 0; i < unit::NP; ++i) {
      sincos_turns((double)pos * rope.turns[u * unit::NP + i], &s[i], &c[i]);
      s[i] *= m;
      c[i] *= m;
    }
  }
  const int h0 = blockIdx.y * heads_per_block, h1 = min(h0 + heads_per_block, a.H + a.Hkv);
  const T* q = (const T*)a.q + row * a.q_rs;
  T* q_out = (T*)a.q_out + row * a.qo_rs;
  for (int h = h0 + slot; h < min(h1, a.H); h += slots * Q_BATCH) {
    unit x[Q_BATCH];
#pragma unroll
    for (int i = 0; i < Q_BATCH; ++i)
      if (h + i * slots < min(h1, a.H)) x[i].load(q + (h + i * slots) * a.q_hs, e0, e1, rotated);
#pragma unroll
    for (int i = 0; i < Q_BATCH; ++i)
      if (h + i * slots < min(h1, a.H)) {
        if (rotated) x[i].turn(s, c);
        x[i].store(q_out + (h + i * slots) * a.qo_hs, e0, e1, rotated);
      }
  }
  if (h1 <= a.H || pos < 0) return;          // only queries here, or a row of padding
  const int page = a.b.pages[seq * a.b.pages_stride + (pos >> a.b.page_shift)];
  if ((unsigned)page >= (unsigned)a.b.n_pages) {
    paged_raise(a.b, PT_PAGED_BAD_PAGE);
    return;
  }
  const int64_t at = page * a.page_stride + (pos & ((1 << a.b.page_shift) - 1)) * a.token_stride;
  const T* k = (const T*)a.k + row * a.k_rs;
  const T* v = (const T*)a.v + row * a.v_rs;
  T* kc = (T*)a.kc + at;
  T* vc = (T*)a.vc + at;
  for (int h = max(h0 - a.H, 0) + slot; h < h1 - a.H; h += slots * KV_BATCH) {
    unit x[KV_BATCH], y[KV_BATCH];
#pragma unroll
    for (int i = 0; i < KV_BATCH; ++i)
      if (h + i * slots < h1 - a.H) {
        x[i].load(k + (h + i * slots) * a.k_hs, e0, e1, rotated);
        y[i].load(v + (h + i * slots) * a.v_hs, e0, e1, rotated);
      }
#pragma unroll
    for (int i = 0; i < KV_BATCH; ++i)
      if (h + i * slots < h1 - a.H) {
        if (rotated) x[i].turn(s, c);
        x[i].store(kc + (h + i * slots) * a.head_stride, e0, e1, rotated);
        y[i].store(vc + (h + i * slots) * a.head_stride, e0, e1, rotated);
      }
  }
}

template <typename T, int VEC, int ROT>
static int launch_append(const pt_append_args& a, const pt_rope& r, hipStream_t s) {
  const int rot_units = ROT == ROT_HALF ? r.rotary_dim / 2 / VEC : ROT == ROT_INTERLEAVED ? r.rotary_dim / VEC : 0;
  const int units = rot_units + (a.hd - (ROT == ROT_NONE ? 0 : r.rotary_dim)) / VEC;
  const int slots = 256 / units, heads = a.H + a.Hkv;
  // One workgroup per row takes all heads where there are rows enough to fill the chip; few rows share theirs out, down
  // to one pass of a workgroup.
  const int passes = (heads + slots - 1) / slots;
  const int groups = std::max(1, std::min(passes, (1024 + a.b.total_rows - 1) / a.b.total_rows));
  const int per = ((heads + groups - 1) / groups + slots - 1) / slots * slots;
  hipLaunchKernelGGL((paged_append_kernel<T, VEC, ROT>), dim3((unsigned)a.b.total_rows, (unsigned)((heads + per - 1) / per)), dim3(256), 0, s,
                     a, r, units, rot_units, per);
  PT_HIP_CHECK(hipGetLastError());
  return PT_OK;
}

template <typename T>
static int launch_append_type(const pt_append_args& a, const pt_rope* rope, hipStream_t s) {
  constexpr int VEC = 16 / sizeof(T);
  if (!rope) {
    pt_rope none = {};
    return launch_append<T, VEC, ROT_NONE>(a, none, s);
  }
  if (rope->layout == PT_ROPE_HALF)
    return rope->rotary_dim % (2 * VEC) == 0 ? launch_append<T, VEC, ROT_HALF>(a, *rope, s) : launch_append<T, 1, ROT_HALF>(a, *rope, s);
  return rope->rotary_dim % VEC == 0 ? launch_append<T, VEC, ROT_INTERLEAVED>(a, *rope, s) : launch_append<T, 2, ROT_INTERLEAVED>(a, *rope, s);
}

int pt_launch_paged_append(const pt_append_args& a, const pt_rope* rope, int32_t dtype, hipStream_t s) {
  return dtype == PT_F32 ? launch_append_type<float>(a, rope, s) : launch_append_type<bf16_t>(a, rope, s);
}

// ------------------------------------------------------------------------------------------------
// Page copies.  The pairs travel in the kernel's arguments (as the pointers of pt_track_merge do): no copy to the device,
// no buffer that must outlive the call, and a captured launch keeps its own.  A page of one layer is n_in x n_out stretches of
// `len` 16-byte chunks (one stretch where the strides leave no gap); a workgroup copies 256 * PER of them.
// Stores bypass the caches (what was moved is not read again soon, and a line that is written whole need not be fetched): 2 GB
// of pages, both directions, 594 us with ordinary stores and eight chunks a thread, 411 with these, and with fewer per
// thread 424 (four), 383 (two), 349 (one: 5.8 TB/s).  Small copies are better off with two: 34 MB 4.8 us against 6.0.
// ------------------------------------------------------------------------------------------------
constexpr int COPY_PAIRS = 400;   // 3200 bytes of arguments
typedef uint32_t u32x4_t __attribute__((ext_vector_type(4)));

struct copy_args {
  char* k;
  char* v;
  int64_t layer_bytes, page_bytes, in_bytes, out_bytes;   // strides
  int32_t len, n_in, chunks;     // chunks of a stretch, stretches of the inner level, chunks of a page
  int32_t n_layers, n_pairs, blocks_per_page;
  int2 pair[COPY_PAIRS];
};

template <bool FLAT, int PER>
__global__ void __launch_bounds__(256) page_copy_kernel(const copy_args a) {
  const int64_t total = (int64_t)a.blocks_per_page * 2 * a.n_layers * a.n_pairs;
  for (int64_t w = blockIdx.x; w < total; w += gridDim.x) {
    const int part = (int)(w % a.blocks_per_page);
    int64_t rest = w / a.blocks_per_page;
    char* pool = rest & 1 ? a.v : a.k;
    rest >>= 1;
    const int layer = (int)(rest % a.n_layers);
    const int2 pr = a.pair[rest / a.n_layers];
    pool += layer * a.layer_bytes;
    const char* src = pool + pr.x * a.page_bytes;
    char* dst = pool + pr.y * a.page_bytes;
    u32x4_t x[PER];
    int64_t off[PER];
    const int c0 = part * 256 * PER + threadIdx.x;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      const int ch = c0 + i * 256;
      if (FLAT) {
        off[i] = (int64_t)ch * 16;
      } else {
        const int st = ch / a.len, in = st % a.n_in, out = st / a.n_in;
        off[i] = in * a.in_bytes + out * a.out_bytes + (int64_t)(ch - st * a.len) * 16;
      }
      if (ch < a.chunks) x[i] = *(const u32x4_t*)(src + off[i]);
    }
#pragma unroll
    for (int i = 0; i < PER; ++i)
      if (c0 + i * 256 < a.chunks) __builtin_nontemporal_store(x[i], (u32x4_t*)(dst + off[i]));
  }
}

template <int PER>
static void launch_copy(copy_args& a, bool flat, hipStream_t s) {
  a.blocks_per_page = (a.chunks + 256 * PER - 1) / (256 * PER);
  const int64_t total = (int64_t)a.blocks_per_page * 2 * a.n_layers * a.n_pairs;
  const unsigned grid = (unsigned)std::min<int64_t>(total, 1 << 22);
  if (flat) hipLaunchKernelGGL((page_copy_kernel<true, PER>), dim3(grid), dim3(256), 0, s, a);
  else hipLaunchKernelGGL((page_copy_kernel<false, PER>), dim3(grid), dim3(256), 0, s, a);
}

int pt_launch_page_copy(const pt_paged_cache& c, const int32_t* pairs, int32_t n, hipStream_t s) {
  copy_args a;
  const int64_t es = c.dtype == PT_F32 ? 4 : 2;
  a.k = (char*)c.k;
  a.v = (char*)c.v;
  a.layer_bytes = c.layer_stride * es;
  a.page_bytes = c.page_stride * es;
  // the two levels of a page, smaller stride inside; levels without gaps are one stretch
  int64_t n_in = c.page_size, s_in = c.token_stride, n_out = c.n_kv_heads, s_out = c.head_stride;
  if (s_out < s_in) { std::swap(n_in, n_out); std::swap(s_in, s_out); }
  int64_t len = c.head_dim;
  if (n_in == 1 || s_in == len) { len *= n_in; n_in = 1; }
  if (n_in == 1 && (n_out == 1 || s_out == len)) { len *= n_out; n_out = 1; }
  const int64_t chunks = len * n_in * n_out * es / 16;
  if (chunks > (1 << 30)) return pt_set_error(PT_ERR_INVALID_ARGUMENT, "a page holds more than 16 GiB");
  a.in_bytes = s_in * es;
  a.out_bytes = s_out * es;
  a.len = (int32_t)(len * es / 16);
  a.n_in = (int32_t)n_in;
  a.chunks = (int32_t)chunks;
  a.n_layers = c.n_layers;
  for (int32_t at = 0; at < n; at += COPY_PAIRS) {
    a.n_pairs = std::min(COPY_PAIRS, n - at);
    for (int i = 0; i < a.n_pairs; ++i) a.pair[i] = make_int2(pairs[2 * (at + i)], pairs[2 * (at + i) + 1]);
    const bool flat = n_in == 1 && n_out == 1;
    if (chunks * 2 * a.n_layers * a.n_pairs >= (int64_t)1 << 23) launch_copy<1>(a, flat, s);   // 128 MB and more
    else launch_copy<2>(a, flat, s);
    PT_HIP_CHECK(hipGetLastError());
  }
  return PT_OK;
}
