// Sampling one token per row of logits: temperature, top-k, top-p, min-p, inverse of the running sum in order of index.
//
// One workgroup per row.  Weights w = exp((x - max) / T) are formed in fp64 (its products run at the rate of unpacked fp32
// ones on this chip) and held as integers of 2^-S with S = 62 - ceil(log2 vocab), at most 51: sums of integers do not depend
// on their order, so atomics, reductions and scans may run in any, and a row's answer is a function of its inputs alone.
// The kept set of top-k and top-p is a prefix of the order (logit descending, index ascending), so it is described by
// its last element, and only rows of up to SAMPLE_LIST logits are sorted whole.
//   top-k (up to SAMPLE_LIST_K): the k-th largest of the maxima of 256 or 1024 groups of the row is a lower bound of the
//     k-th largest logit; the few logits above it are gathered, sorted in LDS, and everything else happens among them.
//   top-p alone or after a larger k (sample_top_p): fp32 weights by 2048 equal steps of the logit name the step that holds the
//     last kept element; a pass of exact weights checks that and lists the step's members, which are sorted.
//   a larger k, and steps with more members than the list holds (sample_cut): an exact histogram of ones or weights over the
//     steps, whose step is listed and sorted; where it does not fit, further histograms split its range of keys.
//   pick: sixteen wavefronts sum a sixteenth of the range each, the one that holds the target is split again.
// Rows are read from HBM once and from the caches in the later passes.
// What bounds it: fp64 issue (about 45 instructions a weight, every compute unit on its own row) and, for top-k, a chain of
// some fifteen steps between barriers.  256 rows of 32000 (33 MB, 6 us to read): largest logit 14 us, temperature alone 26,
// top-k 40 24, top-k 400 45, top-p 0.95 46; one row of 32000 8.5, 19, 18, 38 and 37.
// Few rows of many logits leave most of the chip idle and one compute unit with all fp64 work of a row: their rows are cut
// into parts first.  sample_part_kernel finds each part's largest logit and its candidates for top-k, sample_sum_kernel each
// wavefront's sum of weights relative to the row's largest; sample_kernel then starts from those.  The sums are the integers
// that a row in one piece is summed by, so a row's token does not depend on how many rows the call has.  64 rows of 130001 by
// temperature 28 us (6.6, 13 and 8.9 in the three).  Which rows have a filter is known on the device only, so the launch of
// sums is there for them too, and costs them 2 us: the largest logit 17 us, top-k 40 31.
#include <algorithm>

#include "pt_device.h"
#include "pt_serving.h"

typedef unsigned long long u64;

constexpr int SAMPLE_BINS = 2048;
constexpr int SAMPLE_U = 1;           // loads in flight of a thread where it forms weights: two cost the registers of the other paths

constexpr int SAMPLE_LIST = 2048;     // gathered elements that fit
constexpr int SAMPLE_LIST_K = 640;    // top-k by gathering: past it 1024 group maxima leave more than the list holds
constexpr uint32_t KEY_NEG_INF = 0x007fffffu;

// Order-preserving integer of a float; both zeros alike, NaN as -infinity.
__device__ __forceinline__ uint32_t key_of(float x) {
  if (!(x == x)) return KEY_NEG_INF;
  const uint32_t b = __float_as_uint(x + 0.0f);
  return b & 0x80000000u ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float of_key(uint32_t k) { return __uint_as_float(k & 0x80000000u ? k ^ 0x80000000u : ~k); }

constexpr int SAMPLE_PARTS = 16;      // of a row at most
constexpr int SAMPLE_PART_K = 192;    // top-k by a part's candidates up to here
constexpr int SAMPLE_PART_LIST = 512; // candidates of a part that fit

// What a part leaves for the row's workgroup.
struct sample_part {
  float max, min;            // largest logit, smallest finite one
  int n, pad;                // candidates found (more than fit: none are there); -1: not asked for
  u64 sum[16];               // weights of each wavefront's stretch, relative to the row's largest logit
  u64 list[SAMPLE_PART_LIST];
};

struct sample_lds {
  u64 list[SAMPLE_LIST];       // histogram or gathered elements (inverted key, index)
  u64 wave[16], total[16];
  u64 value;
  float tmax[1024];
  float wmin[16];
  int n, found;
  uint32_t key, lo, hi;
};

// One row's problem; uniform over the workgroup.
struct sample_row {
  const float* x;
  int V, S;
  float max, top;              // largest logit; the same, or 0 where that is infinite and only its equals count
  bool infinite;
  double c;                    // log2 e / T
  double rounder;              // 1.5 * 2^(52 - S)
  uint32_t tau, tau_idx;       // last element kept by top-k and top-p
  float min_p;
  u64 least;                   // min-p as a weight
  float bin_scale;

  // Weight of a logit, as an integer of 2^-S; 0 for -infinity and NaN.  2^t with t = n + f, |f| <= 1/2: the polynomial of degree
  // 9 through 2^f's values at Chebyshev's nodes, its constant term 1 (relative error 4e-14), n added to the exponent.  Whole
  // numbers come out of sums with 1.5 * 2^k, whose low bits they are: n with k = 52, the weight with k = 52 - S.
  __device__ __forceinline__ double power(float v) const {
    const float x = v == max ? top : infinite ? -INFINITY : v;
    const double t = fmax(((double)x - (double)top) * c, -200.0);   // the clamp also takes NaN: -infinity times 0
    const double shifted = t + 6755399441055744.0;
    const double f = t - (shifted - 6755399441055744.0);
    double p = 1.0203121113055101e-07;
    p = fma(p, f, 1.3255224878933224e-06);
    p = fma(p, f, 1.5252686846120593e-05);
    p = fma(p, f, 0.00015403455852451632);
    p = fma(p, f, 0.0013333558179043103);
    p = fma(p, f, 0.0096181291594025619);
    p = fma(p, f, 0.055504108664760424);
    p = fma(p, f, 0.24022650695812989);
    p = fma(p, f, 0.69314718055994529);
    p = fma(p, f, 1.0);
    return __hiloint2double(__double2hiint(p) + (__double2loint(shifted) << 20), __double2loint(p));
  }
  __device__ __forceinline__ u64 weight(float v) const { return (u64)__double_as_longlong(power(v) + rounder) - (u64)__double_as_longlong(rounder); }
  // any weight at all, and min-p's
  __device__ __forceinline__ bool has_weight(float v) const {
    return v == max || (!infinite && v > -INFINITY && ((double)v - (double)max) * c > -1074.0 && (!(min_p > 0.0f) || power(v) >= (double)min_p));
  }
  __device__ __forceinline__ void set_max(float m) {
    max = m;
    infinite = m == INFINITY;
    top = infinite ? 0.0f : m;
  }
  __device__ __forceinline__ bool in_prefix(uint32_t key, uint32_t i) const { return key > tau || (key == tau && i <= tau_idx); }
  __device__ __forceinline__ int bin(float v) const { return (int)fminf((max - v) * bin_scale, (float)(SAMPLE_BINS - 1)); }
};

// The elements lo .. hi-1 by `threads` threads, 16 bytes at a time whatever the row's alignment: four(index, four logits), and
// one(index, logit) for up to three in front of the 16-byte boundary and up to three behind the last.  U loads of a thread
// are in flight.
template <int U, typename F, typename G>
__device__ __forceinline__ void for_fours(const float* x, int lo, int hi, int tid, int threads, F&& four, G&& one) {
  const int head = min(hi, lo + (int)((16 - ((uintptr_t)(x + lo) & 15)) >> 2 & 3));
  const int n4 = (hi - head) >> 2;
  const float4* x4 = (const float4*)(x + head);
#pragma unroll 1
  for (int j0 = tid; j0 < n4; j0 += U * threads) {
    float4 v[U];
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (j0 + u * threads < n4) v[u] = x4[j0 + u * threads];
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (j0 + u * threads < n4) four(head + 4 * (j0 + u * threads), v[u]);
  }
  const int done = head + 4 * n4;
  const int i = lo + tid < head ? lo + tid : tid >= 4 && done + tid - 4 < hi ? done + tid - 4 : -1;
  if (i >= 0) one(i, x[i]);
}
// f(index, logit) for each; the four calls of a load run interleaved where they are free of branches.
template <int U, typename F>
__device__ __forceinline__ void for_each(const float* x, int lo, int hi, int tid, int threads, F&& f) {
  for_fours<U>(x, lo, hi, tid, threads, [&](int i, float4 v) {
    f(i, v.x);
    f(i + 1, v.y);
    f(i + 2, v.z);
    f(i + 3, v.w);
  }, f);
}

// Lanes exchange through the vector unit's own paths (moves within rows of 16, swaps of rows and halves) and not through LDS,
// whose latency would be that of every step of a scan or sort.
template <int CTRL, int BANKS = 0xf>
__device__ __forceinline__ uint32_t dpp(uint32_t old, uint32_t v) {
  return (uint32_t)__builtin_amdgcn_update_dpp((int)old, (int)v, CTRL, 0xf, BANKS, false);
}
constexpr int DPP_QUAD_SWAP1 = 0xb1, DPP_QUAD_SWAP2 = 0x4e, DPP_ROW_SHL = 0x100, DPP_ROW_SHR = 0x110, DPP_ROW_ROR = 0x120;

// The value of lane ^ J.
template <int J>
__device__ __forceinline__ uint32_t partner32(uint32_t v) {
  if constexpr (J == 1) return dpp<DPP_QUAD_SWAP1>(v, v);
  if constexpr (J == 2) return dpp<DPP_QUAD_SWAP2>(v, v);
  if constexpr (J == 4) return dpp<DPP_ROW_SHR + 4, 0xa>(dpp<DPP_ROW_SHL + 4, 0x5>(v, v), v);
  if constexpr (J == 8) return dpp<DPP_ROW_ROR + 8>(v, v);
  if constexpr (J == 16) {
    const auto r = __builtin_amdgcn_permlane16_swap(v, v, false, false);
    return threadIdx.x & 16 ? r[0] : r[1];
  }
  if constexpr (J == 32) {
    const auto r = __builtin_amdgcn_permlane32_swap(v, v, false, false);
    return threadIdx.x & 32 ? r[0] : r[1];
  }
}
template <int J>
__device__ __forceinline__ u64 partner64(u64 v) {
  return (u64)partner32<J>((uint32_t)(v >> 32)) << 32 | partner32<J>((uint32_t)v);
}
template <int J>
__device__ __forceinline__ void sum_step(u64& v) { v += partner64<J>(v); }
__device__ __forceinline__ u64 wave_sum64(u64 v) {
  sum_step<1>(v); sum_step<2>(v); sum_step<4>(v); sum_step<8>(v); sum_step<16>(v); sum_step<32>(v);
  return v;
}
template <int N>
__device__ __forceinline__ void scan_step(u64& v) {   // plus the value N lanes before, inside a row
  v += (u64)dpp<DPP_ROW_SHR + N>(0, (uint32_t)(v >> 32)) << 32 | dpp<DPP_ROW_SHR + N>(0, (uint32_t)v);
}
__device__ __forceinline__ u64 lane_value64(u64 v, int lane) {   // lane: the same everywhere
  return (u64)(uint32_t)__builtin_amdgcn_readlane((int)(v >> 32), lane) << 32 | (uint32_t)__builtin_amdgcn_readlane((int)v, lane);
}
__device__ __forceinline__ u64 wave_scan64(u64 v) {   // inclusive
  const int lane = threadIdx.x & 63;
  scan_step<1>(v); scan_step<2>(v); scan_step<4>(v); scan_step<8>(v);
  const u64 r0 = lane_value64(v, 15), r1 = lane_value64(v, 31), r2 = lane_value64(v, 47);
  return v + (lane >= 48 ? r0 + r1 + r2 : lane >= 32 ? r0 + r1 : lane >= 16 ? r0 : 0);
}
// One step of a bitonic sort: `index` is compared with index ^ J, ascending where `up`.
template <int J>
__device__ __forceinline__ void sort_step(u64& v, bool up) {
  const u64 o = partner64<J>(v);
  v = (v < o) == (((threadIdx.x & J) == 0) == up) ? v : o;
}
__device__ __forceinline__ void sort_merge32(u64& v, bool up) {   // steps of 32 and less
  sort_step<32>(v, up); sort_step<16>(v, up); sort_step<8>(v, up); sort_step<4>(v, up); sort_step<2>(v, up); sort_step<1>(v, up);
}
// The wavefront's values in ascending order of lanes, or descending.
__device__ __forceinline__ u64 wave_sort64(u64 v, bool up = true) {
  const int lane = threadIdx.x;
  sort_step<1>(v, !(lane & 2));
  sort_step<2>(v, !(lane & 4)); sort_step<1>(v, !(lane & 4));
  sort_step<4>(v, !(lane & 8)); sort_step<2>(v, !(lane & 8)); sort_step<1>(v, !(lane & 8));
  sort_step<8>(v, !(lane & 16)); sort_step<4>(v, !(lane & 16)); sort_step<2>(v, !(lane & 16)); sort_step<1>(v, !(lane & 16));
  sort_step<16>(v, !(lane & 32)); sort_step<8>(v, !(lane & 32)); sort_step<4>(v, !(lane & 32)); sort_step<2>(v, !(lane & 32)); sort_step<1>(v, !(lane & 32));
  sort_merge32(v, up);
  return v;
}
// Inclusive sum over the workgroup's threads; *total the whole.
__device__ __forceinline__ u64 block_scan64(sample_lds& s, u64 v, u64* total) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  v = wave_scan64(v);
  __syncthreads();
  if (lane == 63) s.wave[wave] = v;
  __syncthreads();
  u64 before = 0, all = 0;
#pragma unroll
  for (int w = 0; w < 16; ++w) {
    const u64 x = s.wave[w];
    before += w < wave ? x : 0;
    all += x;
  }
  *total = all;
  return before + v;
}

// Smallest index i at which the running sum of weight(i, logit) exceeds `target(total)`; -1 where the total is 0.  The
// weights are free of branches: four of a thread's run interleaved, where one alone is a chain of twenty dependent
// fp64 operations (130001 weights of a row: 50 us with a branch in front of each, 30 us without).
// The range lo .. hi-1 only, and with `known` for the target t.
template <typename W, typename T>
__device__ int sample_pick_in(sample_lds& s, const sample_row& r, int lo, int hi, bool known, u64 t, W&& weight, T&& target) {
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  while (!known || hi - lo > 1024) {
    const int part = ((hi - lo + 15) / 16 + 255) / 256 * 256;   // whole loads of a wavefront, until the end
    const int a = min(hi, lo + wave * part), b = min(hi, a + part);
    u64 sum = 0;
    for_each<SAMPLE_U>(r.x, a, b, lane, 64, [&](int i, float v) { sum += weight(i, v); });
    sum = wave_sum64(sum);
    __syncthreads();
    if (lane == 0) s.wave[wave] = sum;
    __syncthreads();
    u64 total = 0;
#pragma unroll
    for (int w = 0; w < 16; ++w) total += s.wave[w];
    if (!known) {
      if (total == 0) return -1;
      t = target(total);
      known = true;
    }
    u64 before = 0, run = 0;
    int at = 0;
#pragma unroll
    for (int w = 0; w < 16; ++w) {   // the last part whose start the target reaches
      if (run <= t && s.wave[w] > 0) { at = w; before = run; }
      run += s.wave[w];
    }
    t -= before;
    lo = min(hi, lo + at * part);
    hi = min(hi, lo + part);
  }
  u64 total;
  const u64 w = lo + tid < hi ? weight(lo + tid, r.x[lo + tid]) : 0;
  const u64 c = block_scan64(s, w, &total);
  if (w > 0 && c > t && c - w <= t) s.found = lo + tid;   // one thread: t < total
  __syncthreads();
  const int found = s.found;
  __syncthreads();
  return found;
}
template <typename W, typename T>
__device__ int sample_pick(sample_lds& s, const sample_row& r, W&& weight, T&& target) {
  return sample_pick_in(s, r, 0, r.V, false, 0, weight, target);
}

// Sorts list[0 .. n-1] ascending (bitonic; padded with the largest value to a power of two, 64 at least).  A thread holds the elements
// tid and, of more than 1024, tid + 1024: steps of less than 64 stay in the wavefronts' registers, wider ones go through
// LDS, 10 of 55 for 1024 elements.
typedef __attribute__((address_space(3))) u64 lds64_t;
__device__ __forceinline__ void sample_sort_inline(lds64_t* list, int n) {
  const int tid = threadIdx.x;
  int size = 64;
  while (size < n) size <<= 1;
  const bool busy = (tid & ~63) < size;   // wavefront-uniform
  u64 v[2];
  __syncthreads();
#pragma unroll
  for (int e = 0; e < 2; ++e) {
    const int i = tid + 1024 * e;
    v[e] = i < n ? list[i] : ~0ull;
    if (busy) v[e] = wave_sort64(v[e], size == 64 || !(i & 64));
  }
  for (int k = 128; k <= size; k <<= 1) {
    for (int j = k >> 1; j >= 64; j >>= 1) {
      if (j == 1024) {
        const u64 a = min(v[0], v[1]);
        v[1] = max(v[0], v[1]);
        v[0] = a;
        continue;
      }
      __syncthreads();
      if (busy) {
        list[tid] = v[0];
        if (size > 1024) list[tid + 1024] = v[1];
      }
      __syncthreads();
      if (busy) {
        const bool low = (tid & j) == 0;
        u64 o = list[tid ^ j];
        v[0] = (v[0] < o) == (low == ((tid & k) == 0)) ? v[0] : o;
        if (size > 1024) {
          o = list[(tid ^ j) + 1024];
          v[1] = (v[1] < o) == (low == (((tid + 1024) & k) == 0)) ? v[1] : o;
        }
      }
    }
    if (busy) {
      sort_merge32(v[0], (tid & k) == 0);
      if (size > 1024) sort_merge32(v[1], ((tid + 1024) & k) == 0);
    }
  }
  __syncthreads();
  if (tid < size) list[tid] = v[0];
  if (size > 1024) list[tid + 1024] = v[1];
  __syncthreads();
}
// One copy for the callers: in line everywhere, the kernel's other paths take up to 3 us longer (256 rows of 32000, top-k 40
// 23.5 us against 26.9).  sample_top_p has its own.
__device__ __attribute__((noinline)) void sample_sort_call(lds64_t* list, int n) { sample_sort_inline(list, n); }
__device__ __forceinline__ void sample_sort(sample_lds& s, int n) { sample_sort_call((lds64_t*)s.list, n); }

// A lower bound of the k-th largest logit of a range, k <= SAMPLE_LIST_K: the k-th largest of the maxima that its threads left in
// s.tmax.  256 groups of them (about k (1 + k / 512) logits lie above the bound) are ranked by comparing each with all,
// 1024 are sorted.
__device__ float sample_bound(sample_lds& s, int k) {
  const int tid = threadIdx.x;
  if (k > 192) {
    s.list[tid] = (u64)~key_of(s.tmax[tid]) << 32;
    sample_sort(s, 1024);
    return of_key(~(uint32_t)(s.list[k - 1] >> 32));
  }
  float gm = -INFINITY;
  if (tid < 256) {
#pragma unroll
    for (int j = 0; j < 4; ++j) gm = fmaxf(gm, s.tmax[tid + 256 * j]);
  }
  __syncthreads();
  if (tid < 256) s.tmax[tid] = gm;
  __syncthreads();
  if (tid < 256) {
    int rank = 0;
#pragma unroll 16
    for (int j = 0; j < 256; ++j) {
      const float o = s.tmax[j];
      rank += o > gm || (o == gm && j < tid);
    }
    if (rank == k - 1) s.wmin[0] = gm;
  }
  __syncthreads();
  return s.wmin[0];
}

// Gathers the elements that `take` accepts; their number (the list holds them only if it is at most SAMPLE_LIST).
template <typename F>
__device__ int sample_gather(sample_lds& s, const sample_row& r, int lo, int hi, F&& take) {
  __syncthreads();
  if (threadIdx.x == 0) s.n = 0;
  __syncthreads();
  for_each<2>(r.x, lo, hi, threadIdx.x, 1024, [&](int i, float v) {
    if (take(i, v)) {
      const int at = atomicAdd(&s.n, 1);
      if (at < SAMPLE_LIST) s.list[at] = (u64)~key_of(v) << 32 | (uint32_t)i;
    }
  });
  __syncthreads();
  return s.n;
}

// Bin of a histogram, of which each thread holds two (a, b), in which the running sum reaches target(whole sum), which *need
// receives; *before the sum in front of it.  -1: never.
template <typename T>
__device__ int sample_find_bin(sample_lds& s, u64 a, u64 b, T&& target_of, u64* need, u64* before) {
  const int tid = threadIdx.x;
  u64 total;
  const u64 c = block_scan64(s, a + b, &total);
  if (threadIdx.x == 0) s.found = -1;
  __syncthreads();
  const u64 start = c - a - b, target = target_of(total);
  *need = target;
  if (start < target && start + a >= target) { s.found = 2 * tid; s.value = start; }
  else if (start + a < target && c >= target) { s.found = 2 * tid + 1; s.value = start + a; }
  __syncthreads();
  const int found = s.found;
  *before = s.value;
  __syncthreads();
  return found;
}

// Shortens the kept prefix to the shortest whose values sum to target(sum of all) or more (all of it where they do not).
// ONES: every element counts 1, else its weight.
template <bool ONES, typename T>
__device__ void sample_cut(sample_lds& s, sample_row& r, T&& target_of) {
  const int tid = threadIdx.x;
  auto value = [&](float v) { return ONES ? (u64)1 : r.weight(v); };
  auto kept = [&](int i, float v) { return v > -INFINITY && r.in_prefix(key_of(v), i); };
  auto clear = [&] {
    __syncthreads();
    s.list[tid] = 0;
    s.list[tid + 1024] = 0;
    __syncthreads();
  };
  clear();
  for_each<2>(r.x, 0, r.V, tid, 1024, [&](int i, float v) {
    const u64 x = value(v);   // no branch: see sample_pick
    atomicAdd(&s.list[r.bin(v)], kept(i, v) ? x : 0);
  });
  u64 target, before;
  __syncthreads();
  const int b = sample_find_bin(s, s.list[2 * tid], s.list[2 * tid + 1], target_of, &target, &before);
  if (b < 0) return;
  target -= before;
  const int n = sample_gather(s, r, 0, r.V, [&](int i, float v) { return kept(i, v) && r.bin(v) == b; });
  if (n <= SAMPLE_LIST) {
    sample_sort(s, n);
    const u64 e0 = 2 * tid < n ? s.list[2 * tid] : 0, e1 = 2 * tid + 1 < n ? s.list[2 * tid + 1] : 0;
    const u64 v0 = 2 * tid < n ? value(of_key(~(uint32_t)(e0 >> 32))) : 0, v1 = 2 * tid + 1 < n ? value(of_key(~(uint32_t)(e1 >> 32))) : 0;
    u64 total;
    const u64 c = block_scan64(s, v0 + v1, &total), start = c - v0 - v1;
    if (start < target && c >= target) s.value = start + v0 >= target ? e0 : e1;
    __syncthreads();
    r.tau = ~(uint32_t)(s.value >> 32);
    r.tau_idx = (uint32_t)s.value;
    __syncthreads();
    return;
  }
  // too many in one step of the histogram: split its range of keys until one key is left
  __syncthreads();
  if (tid == 0) { s.lo = 0xffffffffu; s.hi = 0; }
  __syncthreads();
  for_each<2>(r.x, 0, r.V, tid, 1024, [&](int i, float v) {
    if (kept(i, v) && r.bin(v) == b) {
      atomicMin(&s.lo, key_of(v));
      atomicMax(&s.hi, key_of(v));
    }
  });
  __syncthreads();
  uint32_t lo = s.lo, hi = s.hi;
  while (lo < hi) {
    int shift = 0;
    while ((hi - lo) >> shift >= SAMPLE_BINS) ++shift;
    clear();
    for_each<2>(r.x, 0, r.V, tid, 1024, [&](int i, float v) {
      const uint32_t k = key_of(v);
      if (k >= lo && k <= hi && kept(i, v)) atomicAdd(&s.list[(hi - k) >> shift], value(v));
    });
    u64 same;
    __syncthreads();
    const int at = sample_find_bin(s, s.list[2 * tid], s.list[2 * tid + 1], [&](u64) { return target; }, &same, &before);   // reached: the step's values sum to the target or more
    target -= before;
    hi -= (uint32_t)at << shift;
    const uint32_t width = (1u << shift) - 1;
    if (hi - lo > width) lo = hi - width;
  }
  // the first `ties` elements of this key, in order of index
  const u64 one = value(of_key(hi));
  const u64 ties = (target + one - 1) / one;
  const int last = sample_pick(s, r, [&](int i, float v) { return (u64)(key_of(v) == hi && kept(i, v)); }, [&](u64) { return ties - 1; });
  r.tau = hi;
  r.tau_idx = (uint32_t)last;
}

// The answer to a uniform number of 0: the first token of the prefix that has any weight, however small (down to 2^-1074, where
// fp64 ends; as integers of 2^-S most of those are 0).  A call, for it is rare and its registers are not the kernel's.
__device__ __attribute__((noinline)) int sample_first(sample_lds& s, const sample_row& r) {
  __syncthreads();
  if (threadIdx.x == 0) s.n = 0x7fffffff;
  __syncthreads();
  for_each<2>(r.x, 0, r.V, threadIdx.x, 1024, [&](int i, float v) {
    if (r.has_weight(v) && r.in_prefix(key_of(v), i)) atomicMin(&s.n, i);
  });
  __syncthreads();
  return s.n;
}

// Stretch of a range of `n` elements that a wavefront sums: whole loads of a wavefront, until the end.
__device__ __forceinline__ int sample_stretch(int n) { return ((n + 15) / 16 + 255) / 256 * 256; }

// Top-p (of what the prefix holds so far) and the token: with two passes over the row.  The first adds up fp32 weights by
// steps of the logit, which tells the step that the cut falls into, give or take rounding (then its neighbour counts as part
// of it).  The second forms the exact weights: each wavefront's sum over its stretch of the row of what lies above that
// step, the sum of all, and the step's members for the list; with them the step is checked (and the next one tried), the cut is found
// among the sorted members, and the token's stretch is known.  -2: the step holds more than the list, sample_cut finds the
// prefix and sample_pick the token.  64 rows of 130001 logits: 240 us with sample_cut's exact histogram and
// sample_pick, 109 so.
template <typename C, typename T>
__device__ int sample_top_p(sample_lds& s, sample_row& r, bool first, C&& cut_of, T&& target_of) {
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  __syncthreads();
  s.list[tid] = 0;
  s.list[tid + 1024] = 0;
  __syncthreads();
  const float c32 = (float)fmin(r.c, 1e38);
  const bool all = r.tau == 0 && r.tau_idx == 0xffffffffu;   // no prefix yet
  for_each<2>(r.x, 0, r.V, tid, 1024, [&](int i, float v) {
    const float x = v == r.max ? r.top : r.infinite ? -INFINITY : v;
    float w = __builtin_amdgcn_exp2f(fmaxf((x - r.top) * c32, -126.0f));
    if (!all) w = r.in_prefix(key_of(v), i) ? w : 0.f;
    atomicAdd(&s.list[r.bin(v)], (u64)(uint32_t)fmaf(w, 2147483648.0f, 0.5f));   // whole numbers: an LDS sum of floats takes 16 times as long
  });
  __syncthreads();
  u64 need, before;
  const int found = sample_find_bin(s, s.list[2 * tid], s.list[2 * tid + 1], cut_of, &need, &before);
  // The fp32 sums are off by some 2^-20 of what they hold.  Where the cut lies that near to an end of its step, the next step is
  // listed too: another pass would cost 10 us, and one of a hundred rows would need it.
  int first_bin = max(found, 0), last_bin = first_bin;
  if (found >= 0) {
    const u64 slack = (need >> 16) + r.V, mass = s.list[found];
    if (need <= before + slack) first_bin = max(found - 1, 0);
    if (need + slack >= before + mass) last_bin = min(found + 1, SAMPLE_BINS - 1);
  }
  const int len = sample_stretch(r.V), lo = min(r.V, wave * len), hi = min(r.V, lo + len);
  for (int step = 0;;) {
    if (tid == 0) s.n = 0;
    __syncthreads();
    u64 total = 0, above = 0, heavy = 0;   // heavy: above and not dropped by min-p
    const float edge = (float)first_bin, next = (float)(last_bin + 1);   // r.bin(v) < first_bin and <= last_bin without the whole number
    const bool last = last_bin == SAMPLE_BINS - 1, floor_on = r.least > 1;
    // whether a logit lies in the step
    auto add = [&](int i, float v) {
      u64 w = r.weight(v);
      if (!all) w = r.in_prefix(key_of(v), i) ? w : 0;
      const float at = (r.max - v) * r.bin_scale;
      const bool up = at < edge;
      total += w;
      above += up ? w : 0;
      if (floor_on) heavy += up && w >= r.least ? w : 0;
      return !up && (last || at < next) && w > 0;
    };
    auto list = [&](int i, float v) {
      const int to = atomicAdd(&s.n, 1);
      if (to < SAMPLE_LIST) s.list[to] = (u64)~key_of(v) << 32 | (uint32_t)i;
    };
    for_fours<SAMPLE_U>(r.x, lo, hi, lane, 64, [&](int i, float4 v) {
      const bool b0 = add(i, v.x), b1 = add(i + 1, v.y), b2 = add(i + 2, v.z), b3 = add(i + 3, v.w);   // no branch between them
      if (b0) list(i, v.x);
      if (b1) list(i + 1, v.y);
      if (b2) list(i + 2, v.z);
      if (b3) list(i + 3, v.w);
    }, [&](int i, float v) {
      if (add(i, v)) list(i, v);
    });
    above = wave_sum64(above);
    total = wave_sum64(total);
    const u64 mine = floor_on ? wave_sum64(heavy) : above;
    if (lane == 0) {
      s.wave[wave] = above;
      s.total[wave] = total;
    }
    __syncthreads();
    above = total = 0;
#pragma unroll
    for (int q = 0; q < 16; ++q) {
      above += s.wave[q];
      total += s.total[q];
    }
    const int n = s.n;
    if (n > SAMPLE_LIST) return -2;
    const u64 cut = cut_of(total);
    sample_sort_inline((lds64_t*)s.list, n);   // called, all of it takes 7 us longer (256 rows of 32000: 47)
    u64 e[2], w[2];
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const int i = 2 * tid + j;
      e[j] = i < n ? s.list[i] : 0;
      w[j] = i < n ? r.weight(of_key(~(uint32_t)(e[j] >> 32))) : 0;
    }
    u64 inside;
    const u64 c = block_scan64(s, w[0] + w[1], &inside), start = above + c - w[0] - w[1];
    // the cut lies above these steps, or below them: never both ways, for the sums are exact
    if (cut <= above && first_bin > 0 && step <= 0) { step = -1; last_bin = --first_bin; __syncthreads(); continue; }
    if (cut > above + inside && last_bin < SAMPLE_BINS - 1 && step >= 0) { step = 1; first_bin = ++last_bin; __syncthreads(); continue; }
    __syncthreads();
    if (lane == 0) s.wave[wave] = mine;
    if (start < cut && start + w[0] + w[1] >= cut) s.value = start + w[0] >= cut ? e[0] : e[1];
    __syncthreads();
    r.tau = ~(uint32_t)(s.value >> 32);
    r.tau_idx = (uint32_t)s.value;
    if (first) return sample_first(s, r);
#pragma unroll
    for (int j = 0; j < 2; ++j)   // kept members join their stretch
      if (w[j] >= r.least && (j == 0 ? start : start + w[0]) < cut) atomicAdd(&s.wave[(int)(uint32_t)e[j] / len], w[j]);
    __syncthreads();
    u64 kept = 0;
#pragma unroll
    for (int q = 0; q < 16; ++q) kept += s.wave[q];
    const u64 t = target_of(kept);
    u64 run = 0, start_of = 0;
    int at = 0;
#pragma unroll
    for (int q = 0; q < 16; ++q) {   // the last stretch whose start the target reaches
      if (run <= t && s.wave[q] > 0) { at = q; start_of = run; }
      run += s.wave[q];
    }
    __syncthreads();
    const int from = min(r.V, at * len);
    return sample_pick_in(s, r, from, min(r.V, from + len), true, t - start_of, [&](int i, float v) {
      const u64 x = r.weight(v);
      return x >= r.least && r.in_prefix(key_of(v), i) ? x : (u64)0;
    }, [](u64 x) { return x; });
  }
}

// Largest and smallest finite logit of a range; each thread's own largest stays in s.tmax.
__device__ void sample_extremes(sample_lds& s, const float* x, int lo, int hi, float* largest, float* smallest) {
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  float mx = -INFINITY, mn = INFINITY;
  for_each<2>(x, lo, hi, tid, 1024, [&](int, float v) {
    mx = fmaxf(mx, v);
    mn = fminf(mn, v > -INFINITY ? v : INFINITY);
  });
  s.tmax[tid] = mx;
  mn = -wave_max(-mn);
  if (lane == 0) s.wmin[wave] = mn;
  __syncthreads();
  mx = s.tmax[lane];
#pragma unroll
  for (int w = 1; w < 16; ++w) mx = fmaxf(mx, s.tmax[lane + 64 * w]);
  *largest = wave_max(mx) + 0.0f;
#pragma unroll
  for (int w = 0; w < 16; ++w) mn = fminf(mn, s.wmin[w]);
  *smallest = mn;
  __syncthreads();
}

// The row's parameters, without its largest logit.
__device__ __forceinline__ sample_row sample_load_row(const pt_sample_args& a, int row, float temperature, float min_p) {
  sample_row r;
  r.x = a.logits + row * a.row_stride;
  r.V = a.vocab;
  int bits = 0;
  while (bits < 31 && (1 << bits) < r.V) ++bits;
  r.S = min(51, 62 - bits);
  r.rounder = ldexp(1.5, 52 - r.S);
  r.c = 1.4426950408889634 / (double)temperature;
  r.tau = 0;
  r.tau_idx = 0xffffffffu;
  r.min_p = min_p;
  r.least = min_p > 0.0f ? max((u64)1, (u64)fmin(ceil(ldexp((double)min_p, r.S)), ldexp(1.0, r.S))) : 1;
  return r;
}

// One part of a row: a.part_len logits from part * a.part_len on.
__global__ void __launch_bounds__(1024) sample_part_kernel(const pt_sample_args a) {
  __shared__ sample_lds s;
  const int tid = threadIdx.x;
  const int row = blockIdx.x / a.parts, part = blockIdx.x - row * a.parts;
  sample_part* const to = (sample_part*)a.ws + blockIdx.x;
  const float temperature = a.temperature ? a.temperature[row] : 1.0f;
  const int top_k = a.top_k ? a.top_k[row] : 0;
  const sample_row r = sample_load_row(a, row, temperature, 0.0f);
  const int lo = min(r.V, part * a.part_len), hi = min(r.V, lo + a.part_len);
  float mx, mn;
  sample_extremes(s, r.x, lo, hi, &mx, &mn);
  if (tid == 0) {
    to->max = mx;
    to->min = mn;
    to->n = -1;
  }
  if (mx == -INFINITY || !(temperature > 0.0f)) return;
  if (top_k > 0 && top_k < r.V && top_k <= SAMPLE_PART_K) {
    const float bound = sample_bound(s, top_k);
    const int n = sample_gather(s, r, lo, hi, [&](int, float v) { return v >= bound && v > -INFINITY; });
    if (tid == 0) to->n = n;
    if (n <= SAMPLE_PART_LIST && tid < n) to->list[tid] = s.list[tid];
  }
}

// Whether a row has no filter: its parts' sums serve it.
__device__ __forceinline__ bool sample_no_filter(int top_k, float top_p, float min_p, int vocab) {
  return !(top_k > 0 && top_k < vocab) && !(top_p < 1.0f) && !(min_p > 0.0f);
}
// Largest logit of a row from its parts (every lane of a wavefront must call this).
__device__ __forceinline__ float sample_parts_max(const sample_part* parts, int n) {
  const int lane = threadIdx.x & 63;
  return wave_max(lane < n ? parts[lane].max : -INFINITY);
}

// Sums of weights of a part's stretches, of rows without a filter.
__global__ void __launch_bounds__(1024) sample_sum_kernel(const pt_sample_args a) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int row = blockIdx.x / a.parts, part = blockIdx.x - row * a.parts;
  const float temperature = a.temperature ? a.temperature[row] : 1.0f;
  if (!(temperature > 0.0f) || !sample_no_filter(a.top_k ? a.top_k[row] : 0, a.top_p ? a.top_p[row] : 1.0f, a.min_p ? a.min_p[row] : 0.0f, a.vocab)) return;
  sample_part* const parts = (sample_part*)a.ws + row * a.parts;
  sample_row r = sample_load_row(a, row, temperature, 0.0f);
  r.set_max(sample_parts_max(parts, a.parts));
  if (r.max == -INFINITY) return;
  const int lo = min(r.V, part * a.part_len), hi = min(r.V, lo + a.part_len);
  const int len = sample_stretch(hi - lo), from = min(hi, lo + wave * len);
  u64 sum = 0;
  for_each<SAMPLE_U>(r.x, from, min(hi, from + len), lane, 64, [&](int, float v) { sum += r.weight(v); });
  sum = wave_sum64(sum);
  if (lane == 0) parts[part].sum[wave] = sum;
}

// A row without a filter from its parts' sums: which stretch the target falls into, and the token inside it.
template <typename T>
__device__ int sample_from_sums(sample_lds& s, const sample_row& r, const sample_part* parts, const pt_sample_args& a, T&& target_of) {
  const int tid = threadIdx.x;
  const u64 own = tid < a.parts * 16 ? parts[tid >> 4].sum[tid & 15] : 0;
  u64 total;
  const u64 c = block_scan64(s, own, &total), t = target_of(total);
  if (c - own <= t && c > t) {   // one thread: t < total
    s.found = tid;
    s.value = c - own;
  }
  __syncthreads();
  const int at = s.found;
  const u64 before = s.value;
  __syncthreads();
  const int p0 = min(r.V, (at >> 4) * a.part_len), p1 = min(r.V, p0 + a.part_len), len = sample_stretch(p1 - p0);
  const int lo = min(p1, p0 + (at & 15) * len), hi = min(p1, lo + len);
  return sample_pick_in(s, r, lo, hi, true, t - before, [&](int, float v) { return r.weight(v); }, [](u64 x) { return x; });
}

// PARTS: sample_part_kernel and sample_sum_kernel ran before.
template <bool PARTS>
__global__ void __launch_bounds__(1024) sample_kernel(const pt_sample_args a) {
  __shared__ sample_lds s;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int row = blockIdx.x;
  const float temperature = a.temperature ? a.temperature[row] : 1.0f;
  const int top_k = a.top_k ? a.top_k[row] : 0;
  const float top_p = a.top_p ? a.top_p[row] : 1.0f, min_p = a.min_p ? a.min_p[row] : 0.0f;
  const float uniform = a.uniform[row];
  sample_row r = sample_load_row(a, row, temperature, min_p);
  const sample_part* const parts = PARTS ? (const sample_part*)a.ws + row * a.parts : nullptr;
  float mx, mn;
  if constexpr (PARTS) {
    mx = sample_parts_max(parts, a.parts);
    mn = -wave_max(lane < a.parts ? -parts[lane].min : -INFINITY);
  } else {
    sample_extremes(s, r.x, 0, r.V, &mx, &mn);
  }
  if (mx == -INFINITY) {
    if (tid == 0) a.out[row] = -1;
    return;
  }
  r.set_max(mx);
  if (!(temperature > 0.0f)) {   // greedy
    int lo = 0, hi = r.V;
    if constexpr (PARTS) {   // the first part that holds the largest
      const int p = __ffsll((unsigned long long)__ballot(lane < a.parts && parts[lane].max == mx)) - 1;
      lo = min(r.V, p * a.part_len);
      hi = min(r.V, lo + a.part_len);
    }
    if (tid == 0) s.n = 0x7fffffff;
    __syncthreads();
    for_each<2>(r.x, lo, hi, tid, 1024, [&](int i, float v) {
      if (v == r.max) atomicMin(&s.n, i);
    });
    __syncthreads();
    if (tid == 0) a.out[row] = s.n;
    return;
  }
  const bool k_on = top_k > 0 && top_k < r.V, p_on = top_p < 1.0f;
  const double u = uniform > 0.0f ? fmin((double)uniform, 1.0) : 0.0;
  // uniform * total, below the total
  auto target = [&](u64 total) { return min((u64)(u * (double)total), total - 1); };
  auto cut_mass = [&](u64 total) { return max((u64)1, min((u64)ceil(fmax((double)top_p, 0.0) * (double)total), total)); };
  if constexpr (PARTS) {
    if (sample_no_filter(top_k, top_p, min_p, r.V) && u > 0.0) {
      const int token = sample_from_sums(s, r, parts, a, target);
      if (tid == 0) a.out[row] = token;
      return;
    }
  }

  // Among a list: the candidates for a small k, or all of a short row.
  const bool short_row = r.V <= SAMPLE_LIST && (k_on || p_on);
  if (short_row || (k_on && top_k <= SAMPLE_LIST_K)) {
    const int most = k_on ? top_k : r.V;   // how many of the list count
    int n = SAMPLE_LIST + 1;
    if (short_row) {
      n = r.V;
      __syncthreads();
      for (int i = tid; i < n; i += 1024) s.list[i] = (u64)~key_of(r.x[i]) << 32 | (uint32_t)i;
      __syncthreads();
    }
    if (PARTS && !short_row && top_k <= SAMPLE_PART_K) {
      // the parts' candidates, one part behind the other
      const int own = lane < a.parts ? max(parts[lane].n, 0) : 0;
      const bool whole = __all(own <= SAMPLE_PART_LIST);
      int sum = own;
#pragma unroll
      for (int o = 1; o < SAMPLE_PARTS; o <<= 1) {
        const int up = __shfl_up(sum, o, 64);
        if (lane >= o) sum += up;
      }
      const int all = __shfl(sum, SAMPLE_PARTS - 1, 64);
      if (whole && all <= SAMPLE_LIST) {
        n = all;
        for (int p = wave; p < a.parts; p += 16) {
          const int count = __shfl(own, p, 64), first = __shfl(sum, p, 64) - count;
          for (int i = lane; i < count; i += 64) s.list[first + i] = parts[p].list[i];
        }
        __syncthreads();
      }
    }
    if (n > SAMPLE_LIST) {
      if constexpr (PARTS) sample_extremes(s, r.x, 0, r.V, &mx, &mn);   // the threads' maxima
      const float bound = sample_bound(s, top_k);
      n = sample_gather(s, r, 0, r.V, [&](int, float v) { return v >= bound && v > -INFINITY; });
    }
    if (n > 64 && n <= 512 && most <= 64) {
      // the k largest by comparing each with all: the sorts below have a barrier per step
      const u64 mine = tid < n ? s.list[tid] : ~0ull;
      int rank = 0;
      if (tid < n) {
#pragma unroll 8
        for (int j = 0; j < n; ++j) rank += s.list[j] < mine;
      }
      __syncthreads();
      if (tid < n && rank < most) s.list[rank] = mine;
      __syncthreads();
      n = most;
    }
    if (n <= 64) {
      // one wavefront, an element per lane: the same steps without a barrier
      if (wave > 0) return;
      u64 e = lane < n ? s.list[lane] : ~0ull;
      e = wave_sort64(e);
      const int m = min(n, most);
      u64 w = lane < m ? r.weight(of_key(~(uint32_t)(e >> 32))) : 0;
      u64 c = wave_scan64(w);
      u64 total = lane_value64(c, 63);
      const u64 need = p_on ? cut_mass(total) : total;
      if (u == 0.0) {   // see sample_first
        const bool in = lane < m && r.has_weight(of_key(~(uint32_t)(e >> 32))) && (!p_on || c - w < need);
        int token = in ? (int)(uint32_t)e : 0x7fffffff;
#pragma unroll
        for (int o = 32; o > 0; o >>= 1) token = min(token, __shfl_xor(token, o, 64));
        if (lane == 0) a.out[row] = token;
        return;
      }
      if (!(w >= r.least && c - w < need)) {   // least is 1 or more: lanes without an element go too
        e = ~0ull;
        w = 0;
      } else {
        e = e << 32 | ~(uint32_t)(e >> 32);
      }
      e = wave_sort64(e);
      w = e != ~0ull ? r.weight(of_key((uint32_t)e)) : 0;
      c = wave_scan64(w);
      total = lane_value64(c, 63);
      const u64 t = target(total);
      if (w > 0 && c - w <= t && c > t) a.out[row] = (int32_t)(e >> 32);
      return;
    }
    if (n <= SAMPLE_LIST) {
      sample_sort(s, n);
      // two elements per thread, in order; those past k drop out
      const int m = min(n, most);
      u64 e[2], w[2];
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        const int i = 2 * tid + j;
        e[j] = i < m ? s.list[i] : 0;
        w[j] = i < m ? r.weight(of_key(~(uint32_t)(e[j] >> 32))) : 0;
      }
      u64 total;
      const u64 c = block_scan64(s, w[0] + w[1], &total), start = c - w[0] - w[1];
      const u64 need = p_on ? cut_mass(total) : total;
      if (u == 0.0) {   // see sample_first
        if (tid == 0) s.n = 0x7fffffff;
        __syncthreads();
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          const int i = 2 * tid + j;
          if (i < m && r.has_weight(of_key(~(uint32_t)(e[j] >> 32))) && (!p_on || (j == 0 ? start : start + w[0]) < need))
            atomicMin(&s.n, (int)(uint32_t)e[j]);
        }
        __syncthreads();
        if (tid == 0) a.out[row] = s.n;
        return;
      }
      // kept: in front of the target, and heavy enough; back into the list in order of index
      if (tid == 0) s.n = 0;
      __syncthreads();
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        const int i = 2 * tid + j;
        const bool in = i < m && w[j] >= r.least && (j == 0 ? start : start + w[0]) < need;
        if (in) atomicMax(&s.n, i + 1);   // a prefix: weights fall
      }
      __syncthreads();
      n = s.n;
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        const int i = 2 * tid + j;
        if (i < n) s.list[i] = (uint32_t)e[j] * (u64)1 << 32 | ~(uint32_t)(e[j] >> 32);
      }
      __syncthreads();
      sample_sort(s, n);
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        const int i = 2 * tid + j;
        e[j] = i < n ? s.list[i] : 0;
        w[j] = i < n ? r.weight(of_key((uint32_t)e[j])) : 0;
      }
      const u64 c2 = block_scan64(s, w[0] + w[1], &total), start2 = c2 - w[0] - w[1];
      const u64 t = target(total);
      if (start2 <= t && c2 > t) a.out[row] = (int32_t)(start2 + w[0] > t ? e[0] >> 32 : e[1] >> 32);
      return;
    }
  }
  const float span = r.max - mn;
  if (k_on) {
    r.bin_scale = span > 0.0f ? (SAMPLE_BINS - 1) / span : 0.0f;
    sample_cut<true>(s, r, [&](u64) { return (u64)top_k; });
  }
  if (p_on) {
    // mass lies within 40 T of the largest logit; the last step takes what is behind
    r.bin_scale = span > 0.0f ? (SAMPLE_BINS - 1) / fminf(span, 40.0f * temperature) : 0.0f;
    const int token = sample_top_p(s, r, u == 0.0, cut_mass, target);
    if (token != -2) {
      if (tid == 0) a.out[row] = token;
      return;
    }
    sample_cut<false>(s, r, cut_mass);
  }
  int token;
  if (u == 0.0) {
    token = sample_first(s, r);
  } else if (!k_on && !p_on) {
    token = sample_pick(s, r, [&](int, float v) {
      const u64 w = r.weight(v);
      return w >= r.least ? w : (u64)0;
    }, target);
  } else {
    token = sample_pick(s, r, [&](int i, float v) {
      const u64 w = r.weight(v);
      return w >= r.least && r.in_prefix(key_of(v), i) ? w : (u64)0;
    }, target);
  }
  if (tid == 0) a.out[row] = token;
}

// Parts of a row: none where the rows alone fill the chip, or where a part would be below 16384 logits.
static int sample_parts(int32_t rows, int32_t vocab) {
  const int64_t p = std::min<int64_t>(std::min<int64_t>(SAMPLE_PARTS, 256 / rows), vocab / 16384);
  return p < 2 ? 1 : (int)p;
}

size_t pt_sample_workspace(int32_t rows, int32_t vocab) {
  const int parts = sample_parts(rows, vocab);
  return parts == 1 ? 0 : (size_t)rows * parts * sizeof(sample_part);
}

int pt_launch_sample(const pt_sample_args& args, hipStream_t s) {
  pt_sample_args a = args;
  a.parts = sample_parts(a.rows, a.vocab);
  a.part_len = ((a.vocab + a.parts - 1) / a.parts + 1023) / 1024 * 1024;
  if (a.parts > 1) {
    hipLaunchKernelGGL(sample_part_kernel, dim3((unsigned)(a.rows * a.parts)), dim3(1024), 0, s, a);
    hipLaunchKernelGGL(sample_sum_kernel, dim3((unsigned)(a.rows * a.parts)), dim3(1024), 0, s, a);
    hipLaunchKernelGGL(sample_kernel<true>, dim3((unsigned)a.rows), dim3(1024), 0, s, a);
  } else {
    hipLaunchKernelGGL(sample_kernel<false>, dim3((unsigned)a.rows), dim3(1024), 0, s, a);
  }
  PT_HIP_CHECK(hipGetLastError());
  return PT_OK;
}
