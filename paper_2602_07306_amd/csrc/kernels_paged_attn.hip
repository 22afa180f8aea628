// Attention of a step's rows over a paged cache: o = softmax(scale q K^T) V per row and head, over the positions that the
// row may see.  One pass over the keys with a running maximum and sum.
//
// Rows of a sequence that share a KV head - its n new rows times the G query heads of the group - are packed into tiles:
// packed row r is new row r / G, head r % G of the group.  A workgroup takes one tile, one KV head and one range of keys; its
// four wavefronts take the range's key tiles in turn and are merged at the end through LDS.  Where one range does not hold all
// keys, each leaves its unscaled sums and statistics to paged_combine_kernel.
#include <algorithm>
#include <type_traits>

#include "pt_paged_device.h"

typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));
typedef short s16x4_t __attribute__((ext_vector_type(4)));
typedef float f32x4_t __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) void* lptr_t;
typedef __attribute__((address_space(3))) s16x4_t* lptr4_t;
typedef const __attribute__((address_space(4))) int32_t* cptr_t;   // what no kernel writes: scalar loads

template <int N, typename F>
__device__ __forceinline__ void static_for(F&& f) {
  if constexpr (N > 0) {
    static_for<N - 1>(f);
    f(std::integral_constant<int, N - 1>{});
  }
}

// Largest of the four lanes that share lane % 16.
__device__ __forceinline__ float max_over_groups(float v) {
  // fmaxf would first pass each exchanged value through an instruction of its own
  auto larger = [](uint32_t x, uint32_t y) {
    float r;
    asm("v_max_f32 %0, %1, %2" : "=v"(r) : "v"(x), "v"(y));
    return r;
  };
  const auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  v = larger(a[0], a[1]);
  const auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return larger(b[0], b[1]);
}

constexpr int PA_MAX_SPLITS = 64;   // a wavefront of the combine holds one range's statistics per lane

// A tile of packed rows: its sequence, its rows, the keys that its last row sees, and in how many ranges they are cut.
struct paged_tile {
  paged_seq sq;
  int seq, row0, nrows, base_pos, vis, nsplit;
};

__device__ __forceinline__ int paged_vis(const pt_paged_attn_args& a, const paged_seq& sq, int last_row) {
  const int pos = sq.kv - sq.n + last_row;
  return pos < 0 ? 0 : a.causal ? pos + 1 : sq.kv;
}

// Rows of a sequence, and whether class WIDE takes it.
template <bool WIDE>
__device__ __forceinline__ bool paged_in_class(const pt_paged_attn_args& a, int n) {
  return n > 0 && (n * (int64_t)(a.H / a.Hkv) > a.few) == WIDE;
}

// Tile `tile` of the class's sequences; false where there are fewer.  Where no sequence has more than one tile, tile and
// sequence are one; otherwise sequences are scanned 64 at a time (wavefront-uniform result).
template <bool WIDE>
__device__ __forceinline__ bool paged_find_tile(const pt_paged_attn_args& a, int tile, paged_tile* t) {
  const int G = a.H / a.Hkv, lane = threadIdx.x & 63;
  const pt_paged_cut& cut = a.cut[WIDE];
  int seq = tile, in_seq = 0;
  if (WIDE || min(a.b.max_q_len * (int64_t)G, (int64_t)a.few) > cut.tile_rows) {
    int before = 0;
    seq = -1;
    for (int base = 0; base < a.b.n_seqs; base += 64) {
      int n = 0;
      if (base + lane < a.b.n_seqs) {
        const int r0 = a.b.row_start[base + lane], r1 = a.b.row_start[base + lane + 1];
        const int first = min(max(r0, 0), a.b.total_rows);
        const int rows = min(min(max(r1, first), a.b.total_rows) - first, a.b.max_q_len);
        if (paged_in_class<WIDE>(a, rows)) n = (int)(((int64_t)rows * G + cut.tile_rows - 1) / cut.tile_rows);
      }
      int sum = n;   // inclusive over the lanes
#pragma unroll
      for (int o = 1; o < 64; o <<= 1) {
        const int up = __shfl_up(sum, o, 64);
        if (lane >= o) sum += up;
      }
      const uint64_t past = __ballot(before + sum > tile);
      if (past) {
        const int l = __ffsll((unsigned long long)past) - 1;
        seq = base + l;
        in_seq = tile - before - (__shfl(sum, l, 64) - __shfl(n, l, 64));
        break;
      }
      before += __shfl(sum, 63, 64);
    }
    if (seq < 0) return false;
  }
  seq = __builtin_amdgcn_readfirstlane(seq);
  in_seq = __builtin_amdgcn_readfirstlane(in_seq);
  t->seq = seq;
  t->sq = paged_load_seq(a.b, seq);
  if (!paged_in_class<WIDE>(a, t->sq.n)) return false;
  t->row0 = in_seq * cut.tile_rows;
  t->nrows = (int)min((int64_t)cut.tile_rows, (int64_t)t->sq.n * G - t->row0);
  if (t->nrows <= 0) return false;
  t->base_pos = t->sq.kv - t->sq.n;
  t->vis = paged_vis(a, t->sq, (t->row0 + t->nrows - 1) / G);
  t->nsplit = max(1, (int)(((int64_t)t->vis + cut.chunk - 1) / cut.chunk));
  return true;
}

// One row by one wavefront, keys k0 .. k1-1, touching no other key: lane = key for the scores, lane = element for the values.
// For rows whose result holds an infinity or a NaN while the keys behind them hold one among their values: a key that the
// mask drops still enters the tile's product, as 0 * V.
template <typename T>
__device__ __forceinline__ void paged_row_alone(const pt_paged_attn_args& a, const T* q, const T* K, const T* V, const int32_t* pages, int k0, int k1,
                                             float* m_out, float* l_out, float acc[4]) {
  const int lane = threadIdx.x & 63;
  float m = -INFINITY, l = 0.f;
#pragma unroll
  for (int i = 0; i < 4; ++i) acc[i] = 0.f;
  for (int base = k0; base < k1; base += 64) {
    const int key = base + lane;
    int64_t off = 0;
    float s = -INFINITY;
    if (key < k1) {
      off = paged_checked(a.b, pages[key >> a.b.page_shift]) * a.page_stride + (key & ((1 << a.b.page_shift) - 1)) * a.token_stride;
      float dot = 0.f;
#pragma unroll 4
      for (int e = 0; e < a.hd; ++e) dot = fmaf(elem<T>::ld(q + e) * a.q_sign, elem<T>::ld(K + off + e), dot);
      s = dot * a.scale_log2;
    }
    const float m_new = fmaxf(m, wave_max(s));
    const float ref = m_new == -INFINITY ? 0.f : m_new;
    const float corr = __builtin_amdgcn_exp2f(m - ref);
    const float p = key < k1 ? __builtin_amdgcn_exp2f(s - ref) : 0.f;
    l = l * corr + wave_sum(p);
    m = m_new;
#pragma unroll
    for (int i = 0; i < 4; ++i) acc[i] *= corr;
    const int nk = min(64, k1 - base);
    for (int kk = 0; kk < nk; ++kk) {
      const float pk = __shfl(p, kk, 64);
      const int64_t o = __shfl((long long)off, kk, 64);
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (lane + 64 * i < a.hd) acc[i] = fmaf(pk, elem<T>::ld(V + o + lane + 64 * i), acc[i]);
    }
  }
  *m_out = m;
  *l_out = l;
}

// Whether a value of the keys from .. to-1 is infinite or no number: lane = key.
template <typename T>
__device__ __forceinline__ bool paged_odd_values(const pt_paged_attn_args& a, const T* V, const int32_t* pages, int from, int to) {
  bool odd = false;
  for (int key = from + (int)(threadIdx.x & 63); key < to; key += 64) {
    const T* v = V + paged_checked(a.b, pages[key >> a.b.page_shift]) * a.page_stride + (key & ((1 << a.b.page_shift) - 1)) * a.token_stride;
    for (int e = 0; e < a.hd; e += 4) {
#pragma unroll
      for (int i = 0; i < 4; ++i) odd |= !(fabsf(elem<T>::ld(v + e + i)) < INFINITY);
    }
  }
  return __any(odd);
}

// A class's partials.
template <bool WIDE>
struct paged_parts {
  float* o;
  float2* ml;
  __device__ __forceinline__ explicit paged_parts(const pt_paged_attn_args& a) {
    o = a.part + (WIDE ? pt_paged_part_size(a.cut[0].n_splits, a.part_rows[0], a.H, a.hd) : 0);
    ml = (float2*)(o + (int64_t)a.cut[WIDE].n_splits * a.part_rows[WIDE] * a.H * a.hd);
  }
  // that of (range, new row i of the tile's sequence, head), counted in heads of rows
  static __device__ __forceinline__ int64_t at(const pt_paged_attn_args& a, const paged_tile& t, int split, int i, int head) {
    const int64_t row = WIDE || a.seq_rows == 0 ? t.sq.first + i : (int64_t)t.seq * a.seq_rows + i;
    return ((int64_t)split * a.part_rows[WIDE] + row) * a.H + head;
  }
};

// Result of one row over one range: the output itself, or a partial for the combine.
template <typename T, bool WIDE>
__device__ __forceinline__ void paged_store_row(const pt_paged_attn_args& a, const paged_tile& t, int split, int i, int head, int lim, float m, float l, float o, int e) {
  if (t.nsplit == 1) {
    // sees nothing: zero; sees only scores of -infinity: 0 / 0
    elem<T>::st((T*)a.o + (t.sq.first + i) * a.o_rs + head * a.o_hs + e, lim <= 0 ? 0.f : o / l);
  } else {
    const paged_parts<WIDE> parts(a);
    const int64_t at = parts.at(a, t, split, i, head);
    parts.o[at * a.hd + e] = o;
    if (e == 0) parts.ml[at] = make_float2(m, l);
  }
}

// Merge of the four wavefronts of a workgroup: red_o [4][R][HD + 4] unscaled sums, red_ml [4][R] statistics.
template <typename T, int HD>
__device__ __forceinline__ void paged_merge(const pt_paged_attn_args& a, const paged_tile& t, int split, int kvh, int k0, int k1,
                                            const float* red_o, const float2* red_ml) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, G = a.H / a.Hkv;
  constexpr int PER = HD / 64;
  for (int r = wave; r < t.nrows; r += 4) {
    const int i = (t.row0 + r) / G, hh = (t.row0 + r) - i * G;
    const int row = t.sq.first + i, head = kvh * G + hh;
    const int lim = paged_vis(a, t.sq, i);
    float m = -INFINITY, l = 0.f, f[4], o[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int w = 0; w < 4; ++w) m = fmaxf(m, red_ml[w * a.cut[0].tile_rows + r].x);
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      const float2 ml = red_ml[w * a.cut[0].tile_rows + r];
      f[w] = ml.x == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(ml.x - m);
      l += f[w] * ml.y;
    }
    bool odd = !(fabsf(l) < INFINITY);
#pragma unroll
    for (int j = 0; j < PER; ++j) {
#pragma unroll
      for (int w = 0; w < 4; ++w) o[j] += f[w] * red_o[(w * a.cut[0].tile_rows + r) * (HD + 4) + lane + 64 * j];
      if (lane + 64 * j < a.hd) odd |= !(fabsf(o[j]) < INFINITY);
    }
    const int64_t hoff = (int64_t)kvh * a.head_stride;
    if (__any(odd) && paged_odd_values<T>(a, (const T*)a.vc + hoff, a.b.pages + t.seq * a.b.pages_stride, max(k0, lim), k1)) {
      paged_row_alone<T>(a, (const T*)a.q + row * a.q_rs + head * a.q_hs, (const T*)a.kc + hoff, (const T*)a.vc + hoff,
                         a.b.pages + t.seq * a.b.pages_stride, k0, min(k1, lim), &m, &l, o);
    }
#pragma unroll
    for (int j = 0; j < PER; ++j)
      if (lane + 64 * j < a.hd) paged_store_row<T, false>(a, t, split, i, head, lim, m, l, o[j], lane + 64 * j);
  }
}

// ------------------------------------------------------------------------------------------------
// bf16.  S^T = K Q^T and O^T = V^T P^T on 16x16x32 MFMAs, so that a query is a lane (lane % 16) of both results and the
// statistics are per lane.  A wavefront's key tile goes straight into its own LDS, K and V as they lie in their pages, 16-byte
// chunks swizzled by row; nothing but the merge waits for another wavefront.  V^T fragments come from the transposing LDS read
// (16 lanes read a 4 x 16 block and receive its columns).
// MFMA contraction order of the second product: lane group g holds, of 32 keys, 4g..4g+3 of the first and of the second
// 16 - what the S^T result leaves in its registers, and what two transposing reads deliver.
// What bounds it is HBM: 64 sequences of 128 to 8192 keys on 16 KV heads of 128, 2.19 GB, 381 us = 5.7 TB/s where a streaming read
// reaches 6.0 to 6.2; tiles of 32 keys instead of 64 there 399.  One workgroup holds 128 KB of tiles at hd = 128.
// NQ: blocks of 16 packed rows.  FULL: hd == HD; otherwise the rest of the LDS rows is zeroed once and never loaded.
// ------------------------------------------------------------------------------------------------
template <int HD>
struct paged_geom {
  static constexpr int ROWB = HD * 2, CH = HD / 8;    // bytes and 16-byte chunks of a row
  static constexpr int RPI = 64 / CH;                 // rows per load instruction of 1024 bytes
  static constexpr int PER16 = 16 / RPI;              // load instructions per 16 keys
  // XOR of a row's chunk numbers.  A 16-byte read of 16 rows at once must meet 16 different chunks (of 256 bytes), a
  // transposing read of 8 rows at once 8 different pairs of chunks: the row's low bits choose the pair, a higher one the half.
  static __device__ __forceinline__ int swz(int row) { return HD == 64 ? (row & 6) | (row >> 3 & 1) : (row & 7) << 1 | (row >> 3 & 1); }
};

// 16 keys of a page into LDS at `lds`: N instructions of 1024 consecutive LDS bytes, 16 per lane, from base + off[i] + LDS_BIAS.
// Instruction i's offset field counts for both sides, so off[i] is short of 1024 (i % 4) (and base of the bias that keeps
// it positive); m0, the LDS address, is set once for four.  Inline assembly because the compiler takes any LDS read to
// depend on such a load of its own and waits for all of them in front of it, that is for the next tile in front of this
// one's first product.  There are no result registers; every wait for these loads is written out.
constexpr int LDS_BIAS = 3 * 1024;
template <int N, bool FULL>
__device__ __forceinline__ void load_keys_to_lds(uint32_t lds, const char* base, const uint32_t (&off)[N], const bool (&on)[N]) {
  if constexpr (FULL && N == 2) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %3\n\tglobal_load_lds_dwordx4 %2, %3 offset:1024"
                 ::"s"(lds), "v"(off[0]), "v"(off[1]), "s"(base) : "memory", "m0");
  } else if constexpr (FULL) {
#pragma unroll
    for (int i = 0; i < N; i += 4)
      asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %5\n\tglobal_load_lds_dwordx4 %2, %5 offset:1024\n\t"
                   "global_load_lds_dwordx4 %3, %5 offset:2048\n\tglobal_load_lds_dwordx4 %4, %5 offset:%6"
                   ::"s"(lds + i * 1024), "v"(off[i]), "v"(off[i + 1]), "v"(off[i + 2]), "v"(off[i + 3]), "s"(base), "n"(LDS_BIAS) : "memory", "m0");
  } else {
#pragma unroll
    for (int i = 0; i < N; ++i)
      if (on[i])
        asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2 offset:%3"
                     ::"s"(lds + i / 4 * 4096), "v"(off[i]), "s"(base), "n"(i % 4 * 1024) : "memory", "m0");
  }
}

// TK: keys of a tile.
template <int HD, int NQ, bool FULL, int TK>
__device__ __forceinline__ void paged_few_rows(const pt_paged_attn_args& a, int block, char* smem) {
#if defined(__HIP_DEVICE_COMPILE__)
  using geo = paged_geom<HD>;
  constexpr int CH = geo::CH, RPI = geo::RPI, PER16 = geo::PER16, TILE_B = TK * geo::ROWB;
  constexpr int NB = TK / 16, KS = HD / 32, HB = HD / 16, NU = TK / 32;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int l16 = lane & 15, g = lane >> 4;
  const int kvh = block % a.Hkv;
  const int rest = block / a.Hkv;
  const int split = rest / a.cut[0].tiles;
  paged_tile t;
  if (!paged_find_tile<false>(a, rest - split * a.cut[0].tiles, &t) || split >= t.nsplit) return;
  const int k0 = split * a.cut[0].chunk, k1 = min(t.vis, k0 + a.cut[0].chunk);
  const int G = a.H / a.Hkv;

  // queries: B operand of S^T, and each one's first key that it does not see
  bf16x8_t qf[NQ][KS];
  int lim[NQ];
#pragma unroll
  for (int n = 0; n < NQ; ++n) {
    const int r = t.row0 + n * 16 + l16, i = r / G, hh = r - i * G;
    const bool real = n * 16 + l16 < t.nrows;
    lim[n] = real ? min(paged_vis(a, t.sq, i), k1) : 0;
    const bf16_t* q = (const bf16_t*)a.q + (t.sq.first + i) * a.q_rs + (kvh * G + hh) * a.q_hs;
#pragma unroll
    for (int kk = 0; kk < KS; ++kk) {
      uint4 w = make_uint4(0, 0, 0, 0);
      if (real && (FULL || kk * 32 + g * 8 < a.hd)) w = *(const uint4*)(q + kk * 32 + g * 8);
      if (a.q_sign != 1.0f) {
        const uint32_t keep = a.q_sign == 0.0f ? 0u : 0xffffffffu, flip = a.q_sign < 0.0f ? 0x80008000u : 0u;
        w.x = (w.x & keep) ^ flip; w.y = (w.y & keep) ^ flip; w.z = (w.z & keep) ^ flip; w.w = (w.w & keep) ^ flip;
      }
      qf[n][kk] = *(const bf16x8_t*)&w;
    }
  }
  const int lim_first = min(paged_vis(a, t.sq, t.row0 / G), k1);   // the row that sees least

  char* kt = smem + wave * 2 * TILE_B;
  char* vt = kt + TILE_B;
  const uint32_t kt_lds = (uint32_t)(uintptr_t)(lptr_t)kt, vt_lds = kt_lds + TILE_B;
  if (!FULL)
    for (int i = lane; i < 2 * TILE_B / 16; i += 64) ((uint4*)kt)[i] = make_uint4(0, 0, 0, 0);
  // a lane's source within 16 keys: its row and swizzled chunk, per load instruction
  uint32_t voff[PER16];
  bool on[PER16];
#pragma unroll
  for (int i = 0; i < PER16; ++i) {
    const int row = i * RPI + lane / CH, c = (lane % CH) ^ geo::swz(row);
    voff[i] = (uint32_t)(row * a.token_stride * 2 + c * 16) + LDS_BIAS - i % 4 * 1024;
    on[i] = FULL || c * 8 < a.hd;
  }
  const cptr_t pages = (cptr_t)(a.b.pages + t.seq * a.b.pages_stride);
  const int mask = (1 << a.b.page_shift) - 1;
  // pages of the tile's blocks of 16 keys (of the range's last key where those are behind it)
  auto page_ids = [&](int kb, int (&id)[NB]) {
#pragma unroll
    for (int j = 0; j < NB; ++j) id[j] = pages[min(kb + 16 * j, k1 - 1) >> a.b.page_shift];
  };
  const char* const k_base = (const char*)a.kc + kvh * a.head_stride * 2 - LDS_BIAS;
  const char* const v_base = (const char*)a.vc + kvh * a.head_stride * 2 - LDS_BIAS;
  const int64_t page_bytes = a.page_stride * 2;
  const uint32_t token_bytes = (uint32_t)a.token_stride * 2;
  auto load_tile = [&](const char* cache, uint32_t lds, int kb, const int (&id)[NB]) {
#pragma unroll
    for (int j = 0; j < NB; ++j) {
      const int page = (unsigned)id[j] < (unsigned)a.b.n_pages ? id[j] : 0;
      const uint32_t slot = ((kb + 16 * j) & mask) * token_bytes;   // page_size * token_stride < 2^31 elements
      load_keys_to_lds<PER16, FULL>(lds + j * PER16 * 1024, cache + (page * page_bytes + slot), voff, on);
    }
  };
  auto report = [&](const int (&id)[NB]) {
    bool bad = false;
#pragma unroll
    for (int j = 0; j < NB; ++j) bad |= (unsigned)id[j] >= (unsigned)a.b.n_pages;
    if (bad) paged_raise(a.b, PT_PAGED_BAD_PAGE);
  };

  f32x4_t acc[NQ][HB];
  float m_run[NQ], l_run[NQ];
#pragma unroll
  for (int n = 0; n < NQ; ++n) {
    m_run[n] = -INFINITY;
    l_run[n] = 0.f;
#pragma unroll
    for (int hb = 0; hb < HB; ++hb) acc[n][hb] = {0.f, 0.f, 0.f, 0.f};
  }
  const float c_log2 = a.scale_log2;
  int kb = k0 + wave * TK;
  int pid[NB];
  if (!FULL) asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");   // the zeros are in LDS
  if (kb < k1) {
    page_ids(kb, pid);
    load_tile(k_base, kt_lds, kb, pid);
    load_tile(v_base, vt_lds, kb, pid);
    report(pid);
    page_ids(min(kb + 4 * TK, k1 - 1), pid);
  }
  for (; kb < k1; kb += 4 * TK) {
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");   // the tile has landed; the wavefront is alone with it
    const bool more = kb + 4 * TK < k1, tail = kb + TK > k1;
    bf16x8_t kf[NB][KS];
#pragma unroll
    for (int b = 0; b < NB; ++b)
#pragma unroll
      for (int kk = 0; kk < KS; ++kk) {
        const int row = b * 16 + l16;
        kf[b][kk] = *(const bf16x8_t*)(kt + row * geo::ROWB + (((kk * 4 + g) ^ geo::swz(row)) * 16));
      }
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    if (more) load_tile(k_base, kt_lds, kb + 4 * TK, pid);
    f32x4_t s[NQ][NB];
#pragma unroll
    for (int b = 0; b < NB; ++b)
#pragma unroll
      for (int n = 0; n < NQ; ++n) {
        s[n][b] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int kk = 0; kk < KS; ++kk) s[n][b] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf[b][kk], qf[n][kk], s[n][b], 0, 0, 0);
      }
    union v_frag {
      s16x4_t h[2];
      uint32_t u[4];
      bf16x8_t v;
    } vf[HB][NU];
#pragma unroll
    for (int hb = 0; hb < HB; ++hb)
#pragma unroll
      for (int u = 0; u < NU; ++u)
#pragma unroll
        for (int x = 0; x < 2; ++x) {
          const int row = 32 * u + 16 * x + 4 * g + (l16 >> 2), c = hb * 2 + ((l16 & 3) >> 1);
          vf[hb][u].h[x] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lptr4_t)(uintptr_t)(vt_lds + row * geo::ROWB + ((c ^ geo::swz(row)) * 16) + (l16 & 1) * 8));
        }
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    if (more) {
      load_tile(v_base, vt_lds, kb + 4 * TK, pid);
      report(pid);
      page_ids(min(kb + 8 * TK, k1 - 1), pid);
    }
    if (tail) {   // cache bytes behind the range are not data: zeroed, so that 0 * x stays 0
#pragma unroll
      for (int u = 0; u < NU; ++u)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const int key = kb + 32 * u + 16 * (j >> 1) + 4 * g + 2 * (j & 1);
          const uint32_t keep = (key < k1 ? 0xffffu : 0u) | (key + 1 < k1 ? 0xffff0000u : 0u);
#pragma unroll
          for (int hb = 0; hb < HB; ++hb) vf[hb][u].u[j] &= keep;
        }
    }
    // s[n][b], register v: key kb + 16 b + 4 g + v, query n * 16 + l16
#pragma unroll
    for (int n = 0; n < NQ; ++n) {
      if (kb + TK > lim_first) {
#pragma unroll
        for (int b = 0; b < NB; ++b)
#pragma unroll
          for (int v = 0; v < 4; ++v)
            if (kb + 16 * b + 4 * g + v >= lim[n]) s[n][b][v] = -INFINITY;
      }
      float mx = -INFINITY;
#pragma unroll
      for (int b = 0; b < NB; ++b)
#pragma unroll
        for (int v = 0; v < 4; ++v) mx = fmaxf(mx, s[n][b][v]);
      mx = max_over_groups(mx);
      const float m_new = fmaxf(m_run[n], mx);
      const float ref = m_new == -INFINITY ? 0.f : m_new;   // no key seen yet
      const float corr = __builtin_amdgcn_exp2f((m_run[n] - ref) * c_log2);
      const float mc = ref * c_log2;
      float psum = 0.f;
#pragma unroll
      for (int b = 0; b < NB; ++b)
#pragma unroll
        for (int v = 0; v < 4; ++v) {
          s[n][b][v] = __builtin_amdgcn_exp2f(fmaf(s[n][b][v], c_log2, -mc));
          psum += s[n][b][v];
        }
      l_run[n] = l_run[n] * corr + psum;
      m_run[n] = m_new;
      if (__any(corr != 1.0f)) {
#pragma unroll
        for (int hb = 0; hb < HB; ++hb) acc[n][hb] *= corr;
      }
      union {
        uint32_t u[4];
        bf16x8_t v;
      } pf[NU];
#pragma unroll
      for (int u = 0; u < NU; ++u)
#pragma unroll
        for (int j = 0; j < 4; ++j) pf[u].u[j] = pack_bf16x2(s[n][2 * u + (j >> 1)][2 * (j & 1)], s[n][2 * u + (j >> 1)][2 * (j & 1) + 1]);
#pragma unroll
      for (int hb = 0; hb < HB; ++hb)
#pragma unroll
        for (int u = 0; u < NU; ++u) acc[n][hb] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf[hb][u].v, pf[u].v, acc[n][hb], 0, 0, 0);
    }
  }
  // merge: the tiles' LDS is free once every wavefront is here
  __syncthreads();
  float* red_o = (float*)smem;                                      // [4][16 NQ][HD + 4]
  float2* red_ml = (float2*)(red_o + 4 * 16 * NQ * (HD + 4));       // [4][16 NQ]
#pragma unroll
  for (int n = 0; n < NQ; ++n) {
    l_run[n] += __shfl_xor(l_run[n], 16, 64);
    l_run[n] += __shfl_xor(l_run[n], 32, 64);
    const int at = (wave * NQ + n) * 16 + l16;
    if (g == 0) red_ml[at] = make_float2(m_run[n] * c_log2, l_run[n]);
#pragma unroll
    for (int hb = 0; hb < HB; ++hb) *(f32x4_t*)(red_o + at * (HD + 4) + hb * 16 + 4 * g) = acc[n][hb];
  }
  __syncthreads();
  paged_merge<bf16_t, HD>(a, t, split, kvh, k0, k1, red_o, red_ml);
#endif
}

template <int HD, int NQ, bool FULL, int TK>
__global__ void __launch_bounds__(256, 1) paged_attn_kernel(const pt_paged_attn_args a) {
  extern __shared__ __attribute__((aligned(1024))) char smem[];
  paged_few_rows<HD, NQ, FULL, TK>(a, blockIdx.x, smem);
}

// ------------------------------------------------------------------------------------------------
// bf16, many rows: four wavefronts of 32 packed rows each share key tiles of 64 (K and V as they lie in their pages, two
// tiles in LDS: one that is read, one on its way).  A wavefront loads the tile's 16 keys of its number - one page - and
// multiplies all 64 with its own rows; MFMA layouts, swizzle and transposing reads as above.  The rows' sums of probabilities
// are one more product, with a row of ones: it costs matrix time that is free and saves as much vector time as the maximum.
// What bounds it: 2048 rows over 16384 keys, 64 heads on 8 KV heads of 128, 1.03 TFLOP, 910 to 975 us by the machine = 1.06 to
// 1.13 PFLOP/s; matrix pipes busy 55 % and vector issue 54 % of the time at 2.0 GHz.  On zeros the same call takes 820 us where
// it takes 975 (the chip gives way with its clock on data).  Of some 950: without loads into LDS 840, without the exponentials
// 795, without LDS reads of operands 857.  Steps:
// no overlap inside a wavefront 1058, units of 32 keys in three stages (below) 955, sums by product 940.  Measured and not
// kept: 64 rows per wavefront, one to a SIMD (1133: scores travel between accumulation and vector registers), eight
// wavefronts to a tile (no change), the search for the maximum spread over the second product (no change at 128, 10 %
// slower at 64), two or eight fragments in flight instead of four (no change).
// ------------------------------------------------------------------------------------------------
template <int HD, bool FULL>
__device__ __forceinline__ void paged_many_rows(const pt_paged_attn_args& a, int block, char* smem) {   // smem: [2][K tile], [2][V tile]
#if defined(__HIP_DEVICE_COMPILE__)
  using geo = paged_geom<HD>;
  constexpr int TK = 64, CH = geo::CH, RPI = geo::RPI, PER16 = geo::PER16, ROWB = geo::ROWB, TILE_B = TK * ROWB;
  constexpr int NB = TK / 16, KS = HD / 32, HB = HD / 16, NU = TK / 32, NQ = 2;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int l16 = lane & 15, g = lane >> 4;
  const int kvh = block % a.Hkv;
  const int rest = block / a.Hkv;
  const int split = rest / a.cut[1].tiles;
  paged_tile t;
  // the last tiles of a sequence see most: they come first
  if (!paged_find_tile<true>(a, a.cut[1].tiles - 1 - (rest - split * a.cut[1].tiles), &t) || split >= t.nsplit) return;
  const int k0 = split * a.cut[1].chunk, k1 = min(t.vis, k0 + a.cut[1].chunk);
  const int G = a.H / a.Hkv;
  const int w0 = wave * NQ * 16;   // the wavefront's first row in the tile

  bf16x8_t qf[NQ][KS];
  int lim[NQ];
#pragma unroll
  for (int n = 0; n < NQ; ++n) {
    const int r = t.row0 + w0 + n * 16 + l16, i = r / G, hh = r - i * G;
    const bool real = w0 + n * 16 + l16 < t.nrows;
    lim[n] = real ? min(paged_vis(a, t.sq, i), k1) : 0;
    const bf16_t* q = (const bf16_t*)a.q + (t.sq.first + i) * a.q_rs + (kvh * G + hh) * a.q_hs;
#pragma unroll
    for (int kk = 0; kk < KS; ++kk) {
      uint4 w = make_uint4(0, 0, 0, 0);
      if (real && (FULL || kk * 32 + g * 8 < a.hd)) w = *(const uint4*)(q + kk * 32 + g * 8);
      if (a.q_sign != 1.0f) {
        const uint32_t keep = a.q_sign == 0.0f ? 0u : 0xffffffffu, flip = a.q_sign < 0.0f ? 0x80008000u : 0u;
        w.x = (w.x & keep) ^ flip; w.y = (w.y & keep) ^ flip; w.z = (w.z & keep) ^ flip; w.w = (w.w & keep) ^ flip;
      }
      qf[n][kk] = *(const bf16x8_t*)&w;
    }
  }
  // the keys that this wavefront's first and last rows see (no row: none)
  const int w_rows = min(NQ * 16, t.nrows - w0);
  const int lim_first = w_rows > 0 ? min(paged_vis(a, t.sq, (t.row0 + w0) / G), k1) : 0;
  const int lim_last = w_rows > 0 ? min(paged_vis(a, t.sq, (t.row0 + w0 + w_rows - 1) / G), k1) : 0;

  const uint32_t lds0 = (uint32_t)(uintptr_t)(lptr_t)smem;
  if (!FULL)
    for (int i = tid; i < 4 * TILE_B / 16; i += 256) ((uint4*)smem)[i] = make_uint4(0, 0, 0, 0);
  uint32_t voff[PER16];
  bool on[PER16];
#pragma unroll
  for (int i = 0; i < PER16; ++i) {
    const int row = i * RPI + lane / CH, c = (lane % CH) ^ geo::swz(row);
    voff[i] = (uint32_t)(row * a.token_stride * 2 + c * 16) + LDS_BIAS - i % 4 * 1024;
    on[i] = FULL || c * 8 < a.hd;
  }
  const cptr_t pages = (cptr_t)(a.b.pages + t.seq * a.b.pages_stride);
  const int mask = (1 << a.b.page_shift) - 1;
  // page of the wavefront's 16 keys of the tile (of the range's last key where those are behind it)
  auto page_id = [&](int kb) { return pages[min(kb + 16 * wave, k1 - 1) >> a.b.page_shift]; };
  const char* const k_base = (const char*)a.kc + kvh * a.head_stride * 2 - LDS_BIAS;
  const char* const v_base = (const char*)a.vc + kvh * a.head_stride * 2 - LDS_BIAS;
  const int64_t page_bytes = a.page_stride * 2;
  const uint32_t token_bytes = (uint32_t)a.token_stride * 2;
  const uint32_t lds_wave = lds0 + wave * 16 * ROWB;
  // where the wavefront's 16 keys of the tile lie, in K as in V
  auto offset_of = [&](int kb, int page) {
    if ((unsigned)page >= (unsigned)a.b.n_pages) {
      paged_raise(a.b, PT_PAGED_BAD_PAGE);
      page = 0;
    }
    const uint32_t slot = ((kb + 16 * wave) & mask) * token_bytes;   // page_size * token_stride < 2^31 elements
    return page * page_bytes + slot;
  };

  // LDS addresses of the fragments of the first 16 keys
  uint32_t ka[KS], va[HB];
#pragma unroll
  for (int kk = 0; kk < KS; ++kk) ka[kk] = lds0 + l16 * ROWB + (((kk * 4 + g) ^ geo::swz(l16)) * 16);
  const int vrow = 4 * g + (l16 >> 2);
#pragma unroll
  for (int hb = 0; hb < HB; ++hb) va[hb] = lds0 + 2 * TILE_B + vrow * ROWB + (((hb * 2 + ((l16 & 3) >> 1)) ^ geo::swz(vrow)) * 16) + (l16 & 1) * 8;
  typedef const __attribute__((address_space(3))) bf16x8_t* lk_t;

  f32x4_t acc[NQ][HB], l_run[NQ];   // l_run: the rounded probabilities' sums, the product with a row of ones
  float m_run[NQ];
  const bf16x8_t ones = {(__bf16)1.0f, (__bf16)1.0f, (__bf16)1.0f, (__bf16)1.0f, (__bf16)1.0f, (__bf16)1.0f, (__bf16)1.0f, (__bf16)1.0f};
#pragma unroll
  for (int n = 0; n < NQ; ++n) {
    m_run[n] = -INFINITY;
    l_run[n] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int hb = 0; hb < HB; ++hb) acc[n][hb] = {0.f, 0.f, 0.f, 0.f};
  }
  const float c_log2 = a.scale_log2;
  constexpr uint32_t K_STAGE = TILE_B, V_LDS = 2 * TILE_B;
  constexpr int UK = 32, UB = UK / 16;        // keys of a unit, in blocks of 16
  constexpr int NS = UB * KS, STEPS = NS + HB;   // operand fragments of a unit: K's, then those of V^T; each feeds NQ MFMAs
  constexpr int PF = 4;                       // fragments in flight between LDS and their MFMAs
  union frag {
    s16x4_t h[2];
    bf16x8_t v;
  };
  // s[n][b], register v: key first + 16 b + 4 g + v, query n * 16 + l16
  auto mask_unit = [&](f32x4_t (&s)[NQ][UB], int first) __attribute__((always_inline)) {
    if (first + UK > lim_first) {
      int key = first + 4 * g;
      asm volatile("" : "+v"(key));   // the keys' numbers are formed here and not in front of the branch
#pragma unroll
      for (int n = 0; n < NQ; ++n)
#pragma unroll
        for (int b = 0; b < UB; ++b)
#pragma unroll
          for (int v = 0; v < 4; ++v)
            if (key + 16 * b + v >= lim[n]) s[n][b][v] = -INFINITY;
    }
  };
  // The reference of the exponentials is a whole binary order, and moves only when the maximum exceeds it by more than 8:
  // until then the probabilities stay below 2^8, which fp32 sums and bf16 operands hold as well.  Moving it multiplies
  // by a power of two, which is exact, for the probabilities (p) that wait for their product too.
  union prob {
    uint32_t u[4];
    bf16x8_t v;
  };
  auto new_reference = [&](const float (&top)[NQ], prob (&p)[NQ]) __attribute__((always_inline)) {
#pragma unroll
    for (int n = 0; n < NQ; ++n) {
      const float mx = max_over_groups(top[n]) * c_log2;
      const bool grow = mx > m_run[n] + 8.0f;
      if (__any(grow)) {
        const float m_new = grow ? ceilf(mx) : m_run[n];
        const float corr = grow ? __builtin_amdgcn_exp2f(m_run[n] - m_new) : 1.0f;
        m_run[n] = m_new;
        l_run[n] *= corr;
#pragma unroll
        for (int hb = 0; hb < HB; ++hb) acc[n][hb] *= corr;
#pragma unroll
        for (int j = 0; j < 4; ++j) p[n].u[j] = pack_bf16x2(__uint_as_float(p[n].u[j] << 16) * corr, __uint_as_float(p[n].u[j] & 0xffff0000u) * corr);
      }
    }
  };
  // Fragment f of a unit into its place of the ring.  K's come block by block of keys inside a step of the head, so that four
  // chains of sums alternate.
  frag fr[PF];
  auto fetch = [&](auto F_, uint32_t k_at, uint32_t v_at) __attribute__((always_inline)) {
    constexpr int f = decltype(F_)::value;
    if constexpr (f < NS) {
      fr[f % PF].v = *(lk_t)(uintptr_t)(ka[f / UB] + k_at + (f % UB) * 16 * ROWB);
    } else {
#pragma unroll
      for (int x = 0; x < 2; ++x) fr[f % PF].h[x] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lptr4_t)(uintptr_t)(va[f - NS] + v_at + 16 * x * ROWB));
    }
  };
  static_assert(STEPS % PF == 0 && NS % PF == 0, "a unit begins at the ring's first place");
  auto fill = [&](uint32_t k_at) __attribute__((always_inline)) { static_for<PF>([&](auto F_) { fetch(F_, k_at, 0); }); };
  // Unit i of 32 keys: its probabilities p_new from its scores s_cur, beside two products that do not depend on them: the
  // scores s_nxt of unit i + 1 and the values of unit i - 1 (p_old; LAG: there is one).  So matrix and vector pipes work
  // side by side inside one wavefront.  k_at, v_at: LDS offsets of the two units; the ring holds the first fragments of
  // K, and with NEXT receives those of the unit at k_next at the end.
  auto unit = [&](auto LAG_, auto NEXT_, f32x4_t (&s_cur)[NQ][UB], f32x4_t (&s_nxt)[NQ][UB], prob (&p_old)[NQ], prob (&p_new)[NQ], uint32_t k_at,
                  uint32_t v_at, uint32_t k_next, int first) __attribute__((always_inline)) {
    constexpr bool LAG = decltype(LAG_)::value, NEXT = decltype(NEXT_)::value;
    constexpr int END = LAG ? STEPS : NS;
    float mc[NQ], top[NQ];
#pragma unroll
    for (int n = 0; n < NQ; ++n) {
      mc[n] = m_run[n] == -INFINITY ? 0.f : m_run[n];
      top[n] = -INFINITY;
    }
    // One MFMA at a time, and behind it its share of the scores: what a wavefront issues right behind an MFMA runs beside it,
    // another MFMA would wait for the first one's end.
    constexpr int SCORES = NQ * UB * 4, SLOTS = END * NQ;
    float half[NQ];
    static_for<SLOTS>([&](auto I_) {
      constexpr int slot = decltype(I_)::value, i = slot / NQ, n = slot % NQ;
      if constexpr (i < NS) {
        constexpr int b = i % UB, kk = i / UB;
        if (kk == 0) s_nxt[n][b] = {0.f, 0.f, 0.f, 0.f};
        s_nxt[n][b] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(fr[i % PF].v, qf[n][kk], s_nxt[n][b], 0, 0, 0);
      } else {
        acc[n][i - NS] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(fr[i % PF].v, p_old[n].v, acc[n][i - NS], 0, 0, 0);
        if constexpr (i == NS) l_run[n] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(ones, p_old[n].v, l_run[n], 0, 0, 0);
      }
      if constexpr (n == NQ - 1 && i + PF < END) fetch(std::integral_constant<int, i + PF>{}, k_at, v_at);
      if constexpr (n == NQ - 1 && i + PF >= END && NEXT) fetch(std::integral_constant<int, i + PF - END>{}, k_next, 0);
      static_for<SCORES>([&](auto J_) {
        constexpr int sc = decltype(J_)::value;
        if constexpr (sc * SLOTS / SCORES == slot) {   // score: query block, key block, register
          constexpr int n = sc / (UB * 4), b = sc / 4 % UB, v = sc % 4;
          float p = __builtin_amdgcn_exp2f(fmaf(s_cur[n][b][v], c_log2, -mc[n]));
          // formed here: the compiler would move all of it behind the last product otherwise
          if constexpr (v % 2 == 0) {
            asm volatile("" : "+v"(p));
            half[n] = p;
          } else {
            p_new[n].u[2 * b + v / 2] = pack_bf16x2(half[n], p);
            asm volatile("" : "+v"(p_new[n].u[2 * b + v / 2]));
          }
        }
      });
      __builtin_amdgcn_sched_barrier(0);
    });
    mask_unit(s_nxt, first + UK);
#pragma unroll
    for (int n = 0; n < NQ; ++n) {
#pragma unroll
      for (int b = 0; b < UB; ++b)
#pragma unroll
        for (int v = 0; v < 4; v += 2) top[n] = fmaxf(fmaxf(top[n], s_nxt[n][b][v]), s_nxt[n][b][v + 1]);
    }
    new_reference(top, p_new);
  };

  // Tile i of the range (two units): K in stage i % 2 of the first half of LDS, V in stage i % 2 of the second; K runs a
  // unit ahead and V a unit behind, so tile i + 1 of K and tile i of V are needed together.
  const int n_tiles = (k1 - k0 + TK - 1) / TK;
  const int own = (max(lim_last - k0, 0) + UK - 1) / UK;   // units that this wavefront's rows see
  if (!FULL) __syncthreads();   // the zeros are in LDS
  int page = 0;                 // of tile i + 2
  int64_t v_off = 0;            // of tile i + 1
  if (n_tiles > 0) {
    const int64_t off = offset_of(k0, page_id(k0));
    load_keys_to_lds<PER16, FULL>(lds_wave, k_base + off, voff, on);
    load_keys_to_lds<PER16, FULL>(lds_wave + V_LDS, v_base + off, voff, on);
    if (n_tiles > 1) {
      v_off = offset_of(k0 + TK, page_id(k0 + TK));
      load_keys_to_lds<PER16, FULL>(lds_wave + K_STAGE, k_base + v_off, voff, on);
    }
    page = page_id(min(k0 + 2 * TK, k1 - 1));
  }
  asm volatile("s_waitcnt vmcnt(0)\n\ts_barrier" ::: "memory");
  f32x4_t s_a[NQ][UB], s_b[NQ][UB];
  prob p_a[NQ], p_b[NQ];
  if (own > 0) {
    float top[NQ];
#pragma unroll
    for (int n = 0; n < NQ; ++n)
#pragma unroll
      for (int b = 0; b < UB; ++b) s_a[n][b] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int i = 0; i < NS; ++i) {
      const bf16x8_t kf = *(lk_t)(uintptr_t)(ka[i % KS] + (i / KS) * 16 * ROWB);
#pragma unroll
      for (int n = 0; n < NQ; ++n) s_a[n][i / KS] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf, qf[n][i % KS], s_a[n][i / KS], 0, 0, 0);
    }
    mask_unit(s_a, k0);
#pragma unroll
    for (int n = 0; n < NQ; ++n) {
      top[n] = -INFINITY;
#pragma unroll
      for (int j = 0; j < 4; ++j) p_b[n].u[j] = 0;
#pragma unroll
      for (int b = 0; b < UB; ++b)
#pragma unroll
        for (int v = 0; v < 4; ++v) top[n] = fmaxf(top[n], s_a[n][b][v]);
    }
    new_reference(top, p_b);
    // unit 0: nothing lags behind it
    fill(UK * ROWB);
    unit(std::false_type{}, std::false_type{}, s_a, s_b, p_b, p_a, UK * ROWB, 0, 0, k0);
  }
  auto tile = [&](auto ODD_, int i) __attribute__((always_inline)) {
    constexpr uint32_t odd = decltype(ODD_)::value * K_STAGE;
    // everything that was asked for is there, here and in the other wavefronts, and nobody reads K of tile i or V of tile
    // i - 1 any more
    asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
    const int kb = k0 + i * TK;
    fill(K_STAGE - odd);
    if (i + 1 < n_tiles) load_keys_to_lds<PER16, FULL>(lds_wave + V_LDS + K_STAGE - odd, v_base + v_off, voff, on);
    if (i + 2 < n_tiles) {
      v_off = offset_of(kb + 2 * TK, page);
      load_keys_to_lds<PER16, FULL>(lds_wave + odd, k_base + v_off, voff, on);
      page = page_id(min(kb + 3 * TK, k1 - 1));
    }
    if (kb + TK > k1) {
      // positions behind the range are not data: their values become 0, so that 0 * x stays 0
      for (int j = (k1 - kb) * CH + tid; j < TK * CH; j += 256) ((uint4*)(smem + V_LDS + odd))[j] = make_uint4(0, 0, 0, 0);
      __syncthreads();
    }
    // units 2 i + 1 and 2 i + 2; past the wavefront's own, scores are masked whatever LDS holds, and one unit more takes the
    // last product
    if (2 * i + 1 <= own) unit(std::true_type{}, std::true_type{}, s_b, s_a, p_a, p_b, K_STAGE - odd, odd, K_STAGE - odd + UK * ROWB, kb + UK);
    if (2 * i + 2 <= own) unit(std::true_type{}, std::false_type{}, s_a, s_b, p_b, p_a, K_STAGE - odd + UK * ROWB, odd + UK * ROWB, 0, kb + TK);
  };
  for (int i = 0; i < n_tiles; i += 2) {   // two stages: their addresses are constants
    tile(std::integral_constant<uint32_t, 0>{}, i);
    if (i + 1 < n_tiles) tile(std::integral_constant<uint32_t, 1>{}, i + 1);
  }
  // acc[n][hb], register v: element 16 hb + 4 g + v of query n * 16 + l16
#pragma unroll
  for (int n = 0; n < NQ; ++n) {
    const float l = l_run[n][0];
    const float m = m_run[n];
    const int r = t.row0 + w0 + n * 16 + l16, i = r / G, head = kvh * G + (r - i * G), row = t.sq.first + i;
    const bool real = w0 + n * 16 + l16 < t.nrows;
    const int see = paged_vis(a, t.sq, i);
    bool odd = !(fabsf(l) < INFINITY);
#pragma unroll
    for (int hb = 0; hb < HB; ++hb)
#pragma unroll
      for (int v = 0; v < 4; ++v) odd |= !(fabsf(acc[n][hb][v]) < INFINITY);
    odd &= real;
    // rows that met an infinity or a NaN among the keys behind them: again, without those
    uint64_t again = __ballot(odd);
    again |= again >> 32;
    again |= again >> 16;
    again &= 0xffff;
    if (again && !paged_odd_values<bf16_t>(a, (const bf16_t*)a.vc + (int64_t)kvh * a.head_stride, a.b.pages + t.seq * a.b.pages_stride,
                                           max(k0, lim_first), min(k1, k0 + own * UK + UK)))
      again = 0;
    if (real && !(again >> l16 & 1)) {   // the others' queries are read once more, and the output may lie over them
      if (t.nsplit == 1) {
        const float inv = see <= 0 ? 0.f : 1.0f / l;
        bf16_t* o = (bf16_t*)a.o + row * a.o_rs + head * a.o_hs + 4 * g;
#pragma unroll
        for (int hb = 0; hb < HB; ++hb)
          if (FULL || hb * 16 + 4 * g < a.hd) {
            uint2 w;
            w.x = pack_bf16x2(acc[n][hb][0] * inv, acc[n][hb][1] * inv);
            w.y = pack_bf16x2(acc[n][hb][2] * inv, acc[n][hb][3] * inv);
            *(uint2*)(o + hb * 16) = w;
          }
      } else {
        const paged_parts<true> parts(a);
        const int64_t at = parts.at(a, t, split, i, head);
#pragma unroll
        for (int hb = 0; hb < HB; ++hb)
          if (FULL || hb * 16 + 4 * g < a.hd) *(f32x4_t*)(parts.o + at * a.hd + hb * 16 + 4 * g) = acc[n][hb];
        if (g == 0) parts.ml[at] = make_float2(m, l);
      }
    }
    for (int j = 0; j < 16; ++j)
      if (again >> j & 1) {
        const int rj = t.row0 + w0 + n * 16 + j, ij = rj / G, hj = kvh * G + (rj - ij * G), rowj = t.sq.first + ij;
        const int limj = paged_vis(a, t.sq, ij);
        const int64_t hoff = (int64_t)kvh * a.head_stride;
        float mj, lj, oj[4];
        paged_row_alone<bf16_t>(a, (const bf16_t*)a.q + rowj * a.q_rs + hj * a.q_hs, (const bf16_t*)a.kc + hoff, (const bf16_t*)a.vc + hoff,
                                a.b.pages + t.seq * a.b.pages_stride, k0, min(k1, limj), &mj, &lj, oj);
#pragma unroll
        for (int e = 0; e < HD / 64; ++e)
          if (lane + 64 * e < a.hd) paged_store_row<bf16_t, true>(a, t, split, ij, hj, limj, mj, lj, oj[e], lane + 64 * e);
      }
  }
#endif
}

template <int HD, bool FULL>
__global__ void __launch_bounds__(256, 2) paged_attn_wide_kernel(const pt_paged_attn_args a) {
  extern __shared__ __attribute__((aligned(1024))) char smem[];
  paged_many_rows<HD, FULL>(a, blockIdx.x, smem);
}

// Decode steps beside chunks in one launch: workgroups of the one kind wait for HBM while those of the other multiply.  Stretches
// of 64 workgroups are dealt to the two kinds in proportion (multiples of the 8 XCDs, so that a KV head stays on its own).
// Two workgroups share a compute unit: the few rows' tiles hold half the keys at hd = 128.  36 decode steps and 4 chunks of
// 400 on 64 heads of 64: 176 us, one kernel behind the other 118 + 72; more of it needs more workgroups to a unit than 159
// registers leave (tiles of 32 keys, three workgroups: 182 to 192).
constexpr int PA_DEAL = 64;
template <int HD, bool FULL>
__global__ void __launch_bounds__(256, 2) paged_attn_both_kernel(const pt_paged_attn_args a, int many, int few) {
  extern __shared__ __attribute__((aligned(1024))) char smem[];
  const int64_t all = many + few;                     // stretches
  const int st = blockIdx.x / PA_DEAL, in = blockIdx.x % PA_DEAL;
  const int before = (int)(st * (int64_t)many / all);   // stretches of the many-row kind in front of this one
  if ((int)((st + 1) * (int64_t)many / all) > before) {
    const int block = before * PA_DEAL + in;
    if (block < a.cut[1].tiles * a.Hkv * a.cut[1].n_splits) paged_many_rows<HD, FULL>(a, block, smem);
  } else {
    const int block = (st - before) * PA_DEAL + in;
    if (block < a.cut[0].tiles * a.Hkv * a.cut[0].n_splits) paged_few_rows<HD, 1, FULL, HD == 128 ? 32 : 64>(a, block, smem);
  }
}

// ------------------------------------------------------------------------------------------------
// fp32 (latency and L2 bound at the sizes it is for), on 16x16x4 MFMAs: 16 packed rows per workgroup, 16 keys per wavefront and step, operands straight from the pages.
// The contraction over the head takes elements 16 j + 4 g + i in step (j, i), so that a lane's operands are 16-byte loads; the
// second product's rows are head elements 64 hb + 4 r + j for the same reason.
// ------------------------------------------------------------------------------------------------
template <int HD>
__global__ void __launch_bounds__(256, 1) paged_attn_f32_kernel(const pt_paged_attn_args a) {
  constexpr int KJ = HD / 16, VH = HD / 64;
  extern __shared__ __attribute__((aligned(1024))) char smem[];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int l16 = lane & 15, g = lane >> 4;
  const int kvh = blockIdx.x % a.Hkv;
  const int rest = blockIdx.x / a.Hkv;
  const int split = rest / a.cut[0].tiles;
  paged_tile t;
  if (!paged_find_tile<false>(a, rest - split * a.cut[0].tiles, &t) || split >= t.nsplit) return;
  const int k0 = split * a.cut[0].chunk, k1 = min(t.vis, k0 + a.cut[0].chunk);
  const int G = a.H / a.Hkv;
  f32x4_t qf[KJ];
  const int r = t.row0 + l16, qi = r / G, hh = r - qi * G;
  const bool real = l16 < t.nrows;
  const int lim = real ? min(paged_vis(a, t.sq, qi), k1) : 0;
  {
    const float* q = (const float*)a.q + (t.sq.first + qi) * a.q_rs + (kvh * G + hh) * a.q_hs;
#pragma unroll
    for (int j = 0; j < KJ; ++j) {
      qf[j] = {0.f, 0.f, 0.f, 0.f};
      if (real && 16 * j + 4 * g < a.hd) qf[j] = *(const f32x4_t*)(q + 16 * j + 4 * g) * a.q_sign;
    }
  }
  const int lim_first = min(paged_vis(a, t.sq, t.row0 / G), k1);
  const int32_t* pages = a.b.pages + t.seq * a.b.pages_stride;
  const int mask = (1 << a.b.page_shift) - 1;
  f32x4_t kf[KJ], vf[VH][4];
  auto load = [&](int kb) {   // a row behind the range is inside its page and unused: zeros for the values
    const int page = paged_checked(a.b, pages[kb >> a.b.page_shift]);
    const int64_t off = page * a.page_stride + (kb & mask) * a.token_stride + kvh * a.head_stride;
    const float* k = (const float*)a.kc + off + l16 * a.token_stride + 4 * g;
    const float* v = (const float*)a.vc + off + 4 * l16;
#pragma unroll
    for (int j = 0; j < KJ; ++j) {
      kf[j] = {0.f, 0.f, 0.f, 0.f};
      if (16 * j + 4 * g < a.hd) kf[j] = *(const f32x4_t*)(k + 16 * j);
    }
#pragma unroll
    for (int h = 0; h < VH; ++h)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        vf[h][i] = {0.f, 0.f, 0.f, 0.f};
        if (64 * h + 4 * l16 < a.hd && kb + 4 * g + i < k1) vf[h][i] = *(const f32x4_t*)(v + (4 * g + i) * a.token_stride + 64 * h);
      }
  };
  f32x4_t acc[VH][4];
#pragma unroll
  for (int h = 0; h < VH; ++h)
#pragma unroll
    for (int j = 0; j < 4; ++j) acc[h][j] = {0.f, 0.f, 0.f, 0.f};
  float m_run = -INFINITY, l_run = 0.f;
  const float c_log2 = a.scale_log2;
  int kb = k0 + wave * 16;
  if (kb < k1) load(kb);
  for (; kb < k1; kb += 64) {
    f32x4_t s = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int j = 0; j < KJ; ++j)
#pragma unroll
      for (int i = 0; i < 4; ++i) s = __builtin_amdgcn_mfma_f32_16x16x4f32(kf[j][i], qf[j][i], s, 0, 0, 0);
    f32x4_t vc[VH][4];
#pragma unroll
    for (int h = 0; h < VH; ++h)
#pragma unroll
      for (int i = 0; i < 4; ++i) vc[h][i] = vf[h][i];
    if (kb + 64 < k1) load(kb + 64);
    if (kb + 16 > lim_first) {
#pragma unroll
      for (int v = 0; v < 4; ++v)
        if (kb + 4 * g + v >= lim) s[v] = -INFINITY;
    }
    float mx = fmaxf(fmaxf(s[0], s[1]), fmaxf(s[2], s[3]));
    mx = max_over_groups(mx);
    const float m_new = fmaxf(m_run, mx);
    const float ref = m_new == -INFINITY ? 0.f : m_new;
    const float corr = __builtin_amdgcn_exp2f((m_run - ref) * c_log2);
    const float mc = ref * c_log2;
    float psum = 0.f;
#pragma unroll
    for (int v = 0; v < 4; ++v) {
      s[v] = __builtin_amdgcn_exp2f(fmaf(s[v], c_log2, -mc));
      psum += s[v];
    }
    l_run = l_run * corr + psum;
    m_run = m_new;
#pragma unroll
    for (int h = 0; h < VH; ++h)
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        acc[h][j] *= corr;
#pragma unroll
        for (int i = 0; i < 4; ++i) acc[h][j] = __builtin_amdgcn_mfma_f32_16x16x4f32(vc[h][i][j], s[i], acc[h][j], 0, 0, 0);
      }
  }
  float* red_o = (float*)smem;
  float2* red_ml = (float2*)(red_o + 4 * 16 * (HD + 4));
  l_run += __shfl_xor(l_run, 16, 64);
  l_run += __shfl_xor(l_run, 32, 64);
  const int at = wave * 16 + l16;
  if (g == 0) red_ml[at] = make_float2(m_run * c_log2, l_run);
#pragma unroll
  for (int h = 0; h < VH; ++h)   // acc[h][j], register v: element 64 h + 16 g + 4 v + j
#pragma unroll
    for (int v = 0; v < 4; ++v) {
      const f32x4_t o = {acc[h][0][v], acc[h][1][v], acc[h][2][v], acc[h][3][v]};
      *(f32x4_t*)(red_o + at * (HD + 4) + 64 * h + 16 * g + 4 * v) = o;
    }
  __syncthreads();
  paged_merge<float, HD>(a, t, split, kvh, k0, k1, red_o, red_ml);
}

// Joins the ranges of a tile's rows, in the ranges' order.  Tiles whose keys fitted one range are done already.  A wavefront takes a
// row, four rows a workgroup; many ranges (SHARE = 4) are shared out to a workgroup's wavefronts, which read eight at a time
// (one sequence of 16000 keys in 63 ranges, attention and joining: 96 us with a wavefront to a row, one range after the other; 29).
template <typename T, bool WIDE, int SHARE>
__device__ __forceinline__ void paged_combine(const pt_paged_attn_args& a, int block, float (*shared)[256]) {
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const pt_paged_cut& cut = a.cut[WIDE];
  const int parts = cut.tile_rows / (4 / SHARE), G = a.H / a.Hkv;
  const int kvh = block % a.Hkv;
  const int rest = block / a.Hkv;
  paged_tile t;
  if (!paged_find_tile<WIDE>(a, rest / parts, &t) || t.nsplit == 1) return;
  const int r = rest % parts * (4 / SHARE) + (SHARE == 4 ? 0 : wave);
  if (r >= t.nrows) return;                         // SHARE = 4: all four wavefronts alike
  const int64_t step = (int64_t)a.part_rows[WIDE] * a.H;
  const int i = (t.row0 + r) / G, head = kvh * G + (t.row0 + r) - i * G, row = t.sq.first + i;
  const paged_parts<WIDE> from(a);
  const int64_t at = from.at(a, t, 0, i, head);
  float2 ml = make_float2(-INFINITY, 0.f);
  if (lane < t.nsplit) ml = from.ml[lane * step + at];
  const float m = wave_max(ml.x);
  const float f = ml.x == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(ml.x - m);
  const float l = wave_sum(f * ml.y);
  const int lim = paged_vis(a, t.sq, i);
  // a wavefront's ranges: consecutive ones
  const int per = (t.nsplit + SHARE - 1) / SHARE, s0 = SHARE == 4 ? min(t.nsplit, wave * per) : 0, s1 = min(t.nsplit, s0 + per);
  float o[4] = {0.f, 0.f, 0.f, 0.f};
  for (int s = s0; s < s1; s += 8) {
#pragma unroll
    for (int u = 0; u < 8; ++u) {
      const float fs = __shfl(f, min(s + u, 63), 64);
#pragma unroll
      for (int j = 0; j < 4; ++j)
        if (s + u < s1 && lane + 64 * j < a.hd) o[j] += fs * from.o[((s + u) * step + at) * a.hd + lane + 64 * j];
    }
  }
  if constexpr (SHARE == 4) {
#pragma unroll
    for (int j = 0; j < 4; ++j) shared[wave][lane + 64 * j] = o[j];
    __syncthreads();
    if (wave > 0) return;
#pragma unroll
    for (int j = 0; j < 4; ++j) o[j] = ((shared[0][lane + 64 * j] + shared[1][lane + 64 * j]) + shared[2][lane + 64 * j]) + shared[3][lane + 64 * j];
  }
#pragma unroll
  for (int j = 0; j < 4; ++j)
    if (lane + 64 * j < a.hd) elem<T>::st((T*)a.o + row * a.o_rs + head * a.o_hs + lane + 64 * j, lim <= 0 ? 0.f : o[j] / l);
}

// The first `few` workgroups join tiles of few rows, the others those of many.
template <typename T, int SHARE>
__global__ void __launch_bounds__(256) paged_combine_kernel(const pt_paged_attn_args a, int few) {
  __shared__ float shared[4][256];
  if ((int)blockIdx.x < few) paged_combine<T, false, SHARE>(a, blockIdx.x, shared);
  else paged_combine<T, true, SHARE>(a, blockIdx.x - few, shared);
}

constexpr int PA_WIDE_ROWS = 128;

// Ranges of keys for `units` workgroups: as many as it takes to have 512 of them, two to a compute unit, each of at least 256 keys (a
// tile of 64 for every wavefront) and at most `longest`.  One range where `single` keys are not exceeded: one sequence of
// 777 keys, 64 heads of 64, takes 8.5 us in one and 5.4 + 3.9 in four with the launch that joins them.
static void paged_ranges(int64_t units, int64_t keys, int64_t single, int64_t longest, pt_paged_cut* c) {
  int64_t splits = keys <= single ? 1 : std::max((512 + units - 1) / units, (keys + longest - 1) / longest);
  splits = std::min<int64_t>(splits, PA_MAX_SPLITS);
  const int64_t chunk = ((keys + splits - 1) / splits + 255) / 256 * 256;
  c->chunk = (int32_t)chunk;
  c->n_splits = (int32_t)((keys + chunk - 1) / chunk);
}

int pt_plan_paged_attn(int32_t dtype, int32_t hd, int32_t H, int32_t Hkv, const pt_paged_rows& b, pt_paged_plan* p) {
  const int64_t G = H / Hkv, rows_max = b.max_q_len * G, keys = std::max(b.max_kv_len, 1);
  if (rows_max > 0x3fffffff) return pt_set_error(PT_ERR_INVALID_ARGUMENT, "max_q_len times the heads of a group is too large");
  const bool wide = dtype == PT_BF16 && hd <= 128 && rows_max > 32;
  // Blocks of 16 packed rows in a tile of the few-row kernels: what the longest sequence needs, or beside longer ones, what a
  // single new row needs; none where a lone sequence is all there is.
  const int64_t few = wide ? (G <= 32 && b.n_seqs > 1 ? G : 0) : rows_max;
  const int nq = dtype == PT_F32 || few <= 16 ? 1 : 2;
  p->cut[0].tile_rows = 16 * nq;
  p->few = wide ? (few > 0 ? 16 * nq : 0) : 0x7fffffff;
  int64_t t0 = wide && few == 0 ? 0 : b.n_seqs, t1 = 0;
  if (!wide && rows_max > 16 * nq)
    t0 = std::min(b.n_seqs * ((rows_max + 16 * nq - 1) / (16 * nq)), b.total_rows * G / (16 * nq) + b.n_seqs);
  if (wide) {
    const int64_t seqs = std::min<int64_t>(b.n_seqs, b.total_rows * G / (p->few + 1));
    t1 = std::min(seqs * ((rows_max + PA_WIDE_ROWS - 1) / PA_WIDE_ROWS), b.total_rows * G / PA_WIDE_ROWS + seqs);
    p->cut[1].tile_rows = PA_WIDE_ROWS;
  }
  p->cut[0].tiles = (int32_t)std::min<int64_t>(t0, 0x7fffffff);
  p->cut[1].tiles = (int32_t)std::min<int64_t>(t1, 0x7fffffff);
  // Few rows, 2048 / 512 workgroups wanted, us: 23 sequences of 1324 to 5606 keys on 8 KV heads of 128 88 / 68, 60 of 1100 to 2000 on
  // 16 169 / 137, 64 of 128 to 8192 on 16 387 / 383; past 8192 keys a range is cut all the same, so that one long sequence among
  // short ones does not end as one workgroup.  The fp32 kernel takes 64 keys at a time where the other takes 256.
  if (t0 > 0) paged_ranges(t0 * Hkv, keys, dtype == PT_F32 ? 256 : 1024, 8192, &p->cut[0]);
  // Many rows: by the number of tiles that the rows make up, not its bound.
  if (t1 > 0) paged_ranges((b.total_rows * G / PA_WIDE_ROWS + 1) * Hkv, keys, 256, keys, &p->cut[1]);
  // workgroups of the two launches: a grid holds less than 2^32 threads, where both kinds run in one each in whole stretches
  int64_t runs = 0, joins = 0;
  for (int c = 0; c < 2; ++c) {
    const int64_t tiles = (c ? t1 : t0) * Hkv;
    runs += (tiles * p->cut[c].n_splits + PA_DEAL - 1) / PA_DEAL * PA_DEAL;
    if (p->cut[c].n_splits > 1) joins += tiles * p->cut[c].tile_rows;
  }
  if (std::max(runs, joins) >= 1 << 24) return pt_set_error(PT_ERR_INVALID_ARGUMENT, "the batch has too many tiles of rows for one call");
  // Partials of each class that is cut.  Beside chunks, the rows of sequences of few rows are a small part of all: they are counted
  // by sequence.  One decode step beside a chunk of 2048 over 16384 keys, 64 heads on 8 KV heads of 128: 4.3 MB, by rows of
  // the batch 2.2 GB.
  p->part_rows[0] = p->part_rows[1] = b.total_rows;
  if (wide && t0 > 0 && b.n_seqs * (p->few / G) < b.total_rows) {
    p->seq_rows = (int32_t)(p->few / G);
    p->part_rows[0] = b.n_seqs * p->seq_rows;
  }
  for (int c = 0; c < 2; ++c) p->bytes += (size_t)pt_paged_part_size(p->cut[c].n_splits, p->part_rows[c], H, hd) * sizeof(float);
  return PT_OK;
}

template <int HD, int NQ, bool FULL, int TK>
static int launch_paged(const pt_paged_attn_args& a, unsigned grid, hipStream_t s) {
  constexpr int LDS = std::max(8 * TK * paged_geom<HD>::ROWB, 4 * 16 * NQ * ((HD + 4) * 4 + 8));
  static_assert(LDS <= 160 * 1024, "LDS of a compute unit");
  auto kern = paged_attn_kernel<HD, NQ, FULL, TK>;
  PT_SET_MAX_LDS_ONCE(kern, LDS);
  hipLaunchKernelGGL(kern, dim3(grid), dim3(256), LDS, s, a);
  return PT_OK;
}
template <int HD, int NQ, int TK>
static int launch_paged_full(const pt_paged_attn_args& a, unsigned grid, hipStream_t s) {
  return a.hd == HD ? launch_paged<HD, NQ, true, TK>(a, grid, s) : launch_paged<HD, NQ, false, TK>(a, grid, s);
}
// Keys of a tile: 64, and 32 where that is 512 bytes a key.  At 256 bytes a key tiles of 64 leave room for one workgroup to a
// compute unit, whose first loads and merge nothing covers; in ranges of up to 1024 keys that costs more than the smaller
// tiles do (67 sequences of 208 to 338 keys on 8 KV heads of 128: 26 us against 20; of 8192 keys: 377 against 399).
template <int HD, int NQ>
static int launch_paged_tile(const pt_paged_attn_args& a, unsigned grid, hipStream_t s) {
  if constexpr (HD == 128) return a.cut[0].chunk <= 1024 ? launch_paged_full<128, NQ, 32>(a, grid, s) : launch_paged_full<128, NQ, 64>(a, grid, s);
  else return launch_paged_full<HD, NQ, HD == 64 ? 64 : 32>(a, grid, s);
}
template <int HD>
static int launch_paged_f32(const pt_paged_attn_args& a, unsigned grid, hipStream_t s) {
  hipLaunchKernelGGL(paged_attn_f32_kernel<HD>, dim3(grid), dim3(256), 4 * 16 * ((HD + 4) * 4 + 8), s, a);
  return PT_OK;
}

template <int HD, bool FULL>
static int launch_wide(const pt_paged_attn_args& a, unsigned grid, hipStream_t s) {
  constexpr int LDS = 4 * 64 * paged_geom<HD>::ROWB;
  auto kern = paged_attn_wide_kernel<HD, FULL>;
  PT_SET_MAX_LDS_ONCE(kern, LDS);
  hipLaunchKernelGGL(kern, dim3(grid), dim3(256), LDS, s, a);
  return PT_OK;
}

template <int HD, bool FULL>
static int launch_both(const pt_paged_attn_args& a, hipStream_t s) {
  constexpr int LDS = 64 * 1024;   // 4 tiles of 64 keys, or 8 of the few rows' own: the same at both widths or less
  static_assert(LDS >= 4 * 64 * paged_geom<HD>::ROWB && LDS >= 8 * (HD == 128 ? 32 : 64) * paged_geom<HD>::ROWB && LDS >= 4 * 16 * ((HD + 4) * 4 + 8), "both kinds fit");
  const int many = (int)(((int64_t)a.cut[1].tiles * a.Hkv * a.cut[1].n_splits + PA_DEAL - 1) / PA_DEAL);
  const int few = (int)(((int64_t)a.cut[0].tiles * a.Hkv * a.cut[0].n_splits + PA_DEAL - 1) / PA_DEAL);
  auto kern = paged_attn_both_kernel<HD, FULL>;
  PT_SET_MAX_LDS_ONCE(kern, LDS);
  hipLaunchKernelGGL(kern, dim3((unsigned)(many + few) * PA_DEAL), dim3(256), LDS, s, a, many, few);
  return PT_OK;
}

int pt_launch_paged_attn(const pt_paged_attn_args& a, int32_t dtype, hipStream_t s) {
  int rc = PT_OK;
  const bool both = a.cut[0].tiles > 0 && a.cut[1].tiles > 0 && a.cut[0].tile_rows == 16;
  if (both) {
    if (a.hd <= 64) rc = a.hd == 64 ? launch_both<64, true>(a, s) : launch_both<64, false>(a, s);
    else rc = a.hd == 128 ? launch_both<128, true>(a, s) : launch_both<128, false>(a, s);
  }
  if (!both && a.cut[1].tiles > 0) {
    const unsigned grid = (unsigned)((int64_t)a.cut[1].tiles * a.Hkv * a.cut[1].n_splits);
    if (a.hd <= 64) rc = a.hd == 64 ? launch_wide<64, true>(a, grid, s) : launch_wide<64, false>(a, grid, s);
    else rc = a.hd == 128 ? launch_wide<128, true>(a, grid, s) : launch_wide<128, false>(a, grid, s);
  }
  if (!rc && !both && a.cut[0].tiles > 0) {
    const unsigned grid = (unsigned)((int64_t)a.cut[0].tiles * a.Hkv * a.cut[0].n_splits);
    const int nq = a.cut[0].tile_rows / 16;
    if (dtype == PT_F32) {
      rc = a.hd <= 64 ? launch_paged_f32<64>(a, grid, s) : a.hd <= 128 ? launch_paged_f32<128>(a, grid, s) : launch_paged_f32<256>(a, grid, s);
    } else if (a.hd <= 64) {
      rc = nq == 1 ? launch_paged_tile<64, 1>(a, grid, s) : launch_paged_tile<64, 2>(a, grid, s);
    } else if (a.hd <= 128) {
      rc = nq == 1 ? launch_paged_tile<128, 1>(a, grid, s) : launch_paged_tile<128, 2>(a, grid, s);
    } else {
      rc = nq == 1 ? launch_paged_tile<256, 1>(a, grid, s) : launch_paged_tile<256, 2>(a, grid, s);
    }
  }
  if (rc) return rc;
  const int share = std::max(a.cut[0].n_splits, a.cut[1].n_splits) > 8 ? 4 : 1;   // wavefronts to a row
  auto joins = [&](int c) { return a.cut[c].n_splits > 1 ? a.cut[c].tiles * a.Hkv * (a.cut[c].tile_rows / (4 / share)) : 0; };   // workgroups
  const int few = joins(0), many = joins(1);
  if (few + many > 0) {
    const dim3 grid((unsigned)(few + many));
    if (dtype == PT_F32) {
      if (share == 4) hipLaunchKernelGGL((paged_combine_kernel<float, 4>), grid, dim3(256), 0, s, a, few);
      else hipLaunchKernelGGL((paged_combine_kernel<float, 1>), grid, dim3(256), 0, s, a, few);
    } else {
      if (share == 4) hipLaunchKernelGGL((paged_combine_kernel<bf16_t, 4>), grid, dim3(256), 0, s, a, few);
      else hipLaunchKernelGGL((paged_combine_kernel<bf16_t, 1>), grid, dim3(256), 0, s, a, few);
    }
  }
  PT_HIP_CHECK(hipGetLastError());
  return PT_OK;
}
