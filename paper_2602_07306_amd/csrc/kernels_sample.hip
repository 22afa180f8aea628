// Sampling one token per row of logits: temperature, top-k, top-p, min-p, inverse of the running sum in order of index.
//
// One workgroup per row.  Weights w = exp((x - max) / T) are formed in fp64 (its products run at the rate of unpacked fp32
// ones on this chip) and held as integers of 2^-S with S = 62 - ceil(log2 vocab), at most 52: sums of integers do not depend
// on their order, so atomics, reductions and scans may run in any, and a row's answer is a function of its inputs alone.
// The kept set of top-k and top-p is a prefix of the order (logit descending, index ascending), so it is described by
// its last element; no filter ever sorts a row.
//   top-k (up to SAMPLE_LIST_K): the k-th largest of the maxima of 256 or 1024 groups of the row is a lower bound of the
//     k-th largest logit; the few logits above it are gathered, sorted in LDS, and everything else happens among them.
//   otherwise: a histogram of weights (or of ones) over 2048 equal steps of the logit finds the step that holds the last
//     kept element, its members are gathered and sorted; where they do not fit, further histograms split its range of keys.
//   pick: sixteen wavefronts sum a sixteenth of the range each, the one that holds the target is split again.
// Rows are read from HBM once and from the caches in the later passes.
#include "pt_device.h"
#include "pt_serving.h"

typedef unsigned long long u64;

constexpr int SAMPLE_BINS = 2048;
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

struct sample_lds {
  u64 list[SAMPLE_LIST];       // histogram or gathered elements (inverted key, index)
  u64 wave[16];
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
  float max;
  double c;                    // log2 e / T
  uint32_t tau, tau_idx;       // last element kept by top-k and top-p
  u64 least;                   // min-p as a weight
  float bin_scale;

  // weight of a logit, as an integer of 2^-S
  __device__ __forceinline__ u64 weight(float v) const {
    if (v == max) return (u64)1 << S;
    if (!(v > -INFINITY) || max == INFINITY) return 0;
    const double t = fmax(((double)v - (double)max) * c, -200.0);
    const double n = rint(t);
    const double r = (t - n) * 0.6931471805599453;   // exp(r) by its series, |r| <= 0.347: 6e-15
    double p = 1.0 / 39916800;
    p = fma(p, r, 1.0 / 3628800);
    p = fma(p, r, 1.0 / 362880);
    p = fma(p, r, 1.0 / 40320);
    p = fma(p, r, 1.0 / 5040);
    p = fma(p, r, 1.0 / 720);
    p = fma(p, r, 1.0 / 120);
    p = fma(p, r, 1.0 / 24);
    p = fma(p, r, 1.0 / 6);
    p = fma(p, r, 0.5);
    p = fma(p, r, 1.0);
    p = fma(p, r, 1.0);
    return (u64)(ldexp(p, (int)n + S) + 0.5);
  }
  __device__ __forceinline__ bool in_prefix(uint32_t key, uint32_t i) const { return key > tau || (key == tau && i <= tau_idx); }
  __device__ __forceinline__ int bin(float v) const { return (int)fminf((max - v) * bin_scale, (float)(SAMPLE_BINS - 1)); }
};

// f(index, logit) for the elements lo .. hi-1, by `threads` threads, 16 bytes at a time whatever the row's alignment.
template <typename F>
__device__ __forceinline__ void for_each(const float* x, int lo, int hi, int tid, int threads, F&& f) {
  const int head = min(hi, lo + (int)((16 - ((uintptr_t)(x + lo) & 15)) >> 2 & 3));
  if (lo + tid < head) f(lo + tid, x[lo + tid]);
  const int n4 = (hi - head) >> 2;
  const float4* x4 = (const float4*)(x + head);
  for (int j0 = tid; j0 < n4; j0 += 4 * threads) {
    float4 v[4];
#pragma unroll
    for (int u = 0; u < 4; ++u)
      if (j0 + u * threads < n4) v[u] = x4[j0 + u * threads];
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      if (j0 + u * threads < n4) {
        const int i = head + 4 * (j0 + u * threads);
        f(i, v[u].x);
        f(i + 1, v[u].y);
        f(i + 2, v[u].z);
        f(i + 3, v[u].w);
      }
    }
  }
  const int done = head + 4 * n4;
  if (done + tid < hi) f(done + tid, x[done + tid]);
}

__device__ __forceinline__ u64 wave_sum64(u64 v) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v += (u64)__shfl_xor((long long)v, o, 64);
  return v;
}
__device__ __forceinline__ u64 wave_scan64(u64 v) {   // inclusive
  const int lane = threadIdx.x & 63;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const u64 up = (u64)__shfl_up((long long)v, o, 64);
    if (lane >= o) v += up;
  }
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

// Smallest index i at which the running sum of weight(i, logit) exceeds `target(total)`; -1 where the total is 0.
template <typename W, typename T>
__device__ int sample_pick(sample_lds& s, const sample_row& r, W&& weight, T&& target) {
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  int lo = 0, hi = r.V;
  u64 t = 0;
  bool known = false;
  while (!known || hi - lo > 1024) {
    const int part = ((hi - lo + 15) / 16 + 255) / 256 * 256;   // whole loads of a wavefront, until the end
    const int a = min(hi, lo + wave * part), b = min(hi, a + part);
    u64 sum = 0;
    for_each(r.x, a, b, lane, 64, [&](int i, float v) { sum += weight(i, v); });
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

// Sorts s.list[0 .. n-1] ascending; padded to a power of two with the largest value.
__device__ void sample_sort(sample_lds& s, int n) {
  int size = 2;
  while (size < n) size <<= 1;
  for (int i = n + threadIdx.x; i < size; i += 1024) s.list[i] = ~0ull;
  for (int k = 2; k <= size; k <<= 1)
    for (int j = k >> 1; j > 0; j >>= 1) {
      __syncthreads();
      const int p = threadIdx.x;
      if (p < size / 2) {
        const int i = 2 * p - (p & (j - 1)), l = i + j;
        const u64 a = s.list[i], b = s.list[l];
        if ((a > b) == ((i & k) == 0)) { s.list[i] = b; s.list[l] = a; }
      }
    }
  __syncthreads();
}

// Gathers the elements that `take` accepts; their number (the list holds them only if it is at most SAMPLE_LIST).
template <typename F>
__device__ int sample_gather(sample_lds& s, const sample_row& r, F&& take) {
  __syncthreads();
  if (threadIdx.x == 0) s.n = 0;
  __syncthreads();
  for_each(r.x, 0, r.V, threadIdx.x, 1024, [&](int i, float v) {
    if (take(i, v)) {
      const int at = atomicAdd(&s.n, 1);
      if (at < SAMPLE_LIST) s.list[at] = (u64)~key_of(v) << 32 | (uint32_t)i;
    }
  });
  __syncthreads();
  return s.n;
}

// Bin of s.list (as a histogram) in which the running sum reaches `target`; *before the sum in front of it.  -1: never.
__device__ int sample_find_bin(sample_lds& s, u64 target, u64* before) {
  const int tid = threadIdx.x;
  __syncthreads();
  const u64 a = s.list[2 * tid], b = s.list[2 * tid + 1];
  u64 total;
  const u64 c = block_scan64(s, a + b, &total);
  if (threadIdx.x == 0) s.found = -1;
  __syncthreads();
  const u64 start = c - a - b;
  if (start < target && start + a >= target) { s.found = 2 * tid; s.value = start; }
  else if (start + a < target && c >= target) { s.found = 2 * tid + 1; s.value = start + a; }
  __syncthreads();
  const int found = s.found;
  *before = s.value;
  __syncthreads();
  return found;
}

// Shortens the kept prefix to the shortest whose values sum to `target` or more (all of it where they do not).
// ONES: every element counts 1, else its weight.
template <bool ONES>
__device__ void sample_cut(sample_lds& s, sample_row& r, u64 target) {
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
  for_each(r.x, 0, r.V, tid, 1024, [&](int i, float v) {
    if (kept(i, v)) atomicAdd(&s.list[r.bin(v)], value(v));
  });
  u64 before;
  const int b = sample_find_bin(s, target, &before);
  if (b < 0) return;
  target -= before;
  const int n = sample_gather(s, r, [&](int i, float v) { return kept(i, v) && r.bin(v) == b; });
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
  for_each(r.x, 0, r.V, tid, 1024, [&](int i, float v) {
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
    for_each(r.x, 0, r.V, tid, 1024, [&](int i, float v) {
      const uint32_t k = key_of(v);
      if (k >= lo && k <= hi && kept(i, v)) atomicAdd(&s.list[(hi - k) >> shift], value(v));
    });
    const int at = sample_find_bin(s, target, &before);   // reached: the step's values sum to the target or more
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

__global__ void __launch_bounds__(1024) sample_kernel(const pt_sample_args a) {
  __shared__ sample_lds s;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int row = blockIdx.x;
  sample_row r;
  r.x = a.logits + row * a.row_stride;
  r.V = a.vocab;
  const float temperature = a.temperature ? a.temperature[row] : 1.0f;
  const int top_k = a.top_k ? a.top_k[row] : 0;
  const float top_p = a.top_p ? a.top_p[row] : 1.0f, min_p = a.min_p ? a.min_p[row] : 0.0f;
  const float uniform = a.uniform[row];
  // largest logit, smallest finite one
  float mx = -INFINITY, mn = INFINITY;
  for_each(r.x, 0, r.V, tid, 1024, [&](int, float v) {
    mx = fmaxf(mx, v);
    if (v > -INFINITY) mn = fminf(mn, v);
  });
  s.tmax[tid] = mx;
  mn = -wave_max(-mn);
  if (lane == 0) s.wmin[wave] = mn;
  __syncthreads();
  mx = s.tmax[lane];
#pragma unroll
  for (int w = 1; w < 16; ++w) mx = fmaxf(mx, s.tmax[lane + 64 * w]);
  mx = wave_max(mx);
#pragma unroll
  for (int w = 0; w < 16; ++w) mn = fminf(mn, s.wmin[w]);
  if (mx == -INFINITY) {
    if (tid == 0) a.out[row] = -1;
    return;
  }
  r.max = mx + 0.0f;
  if (!(temperature > 0.0f)) {   // greedy
    __syncthreads();
    if (tid == 0) s.n = 0x7fffffff;
    __syncthreads();
    for_each(r.x, 0, r.V, tid, 1024, [&](int i, float v) {
      if (v == r.max) atomicMin(&s.n, i);
    });
    __syncthreads();
    if (tid == 0) a.out[row] = s.n;
    return;
  }
  int bits = 0;
  while (bits < 31 && (1 << bits) < r.V) ++bits;
  r.S = min(52, 62 - bits);
  r.c = 1.4426950408889634 / (double)temperature;
  r.tau = 0;
  r.tau_idx = 0xffffffffu;
  r.least = min_p > 0.0f ? max((u64)1, (u64)fmin(ceil(ldexp((double)min_p, r.S)), ldexp(1.0, r.S))) : 1;
  const bool k_on = top_k > 0 && top_k < r.V, p_on = top_p < 1.0f;
  const double u = uniform > 0.0f ? fmin((double)uniform, 1.0) : 0.0;
  // uniform * total, below the total
  auto target = [&](u64 total) { return min((u64)(u * (double)total), total - 1); };
  auto cut_mass = [&](u64 total) { return max((u64)1, min((u64)ceil(fmax((double)top_p, 0.0) * (double)total), total)); };

  if (k_on && top_k <= SAMPLE_LIST_K) {
    // a lower bound of the k-th largest: the k-th largest of group maxima
    const int groups = top_k <= 192 ? 256 : 1024;
    float gm = -INFINITY;
    if (tid < groups)
      for (int j = tid; j < 1024; j += groups) gm = fmaxf(gm, s.tmax[j]);
    __syncthreads();
    if (tid < groups) s.tmax[tid] = gm;
    __syncthreads();
    if (tid < groups) {
      int rank = 0;
      for (int j = 0; j < groups; ++j) {
        const float o = s.tmax[j];
        rank += o > gm || (o == gm && j < tid);
      }
      if (rank == top_k - 1) s.wmin[0] = gm;
    }
    __syncthreads();
    const float bound = s.wmin[0];
    int n = sample_gather(s, r, [&](int, float v) { return v >= bound && v > -INFINITY; });
    if (n <= SAMPLE_LIST) {
      sample_sort(s, n);
      // two elements per thread, in order; those past k drop out
      const int m = min(n, top_k);
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
    sample_cut<true>(s, r, (u64)top_k);
  }
  if (p_on) {
    // mass lies within 40 T of the largest logit; the last step takes what is behind
    r.bin_scale = span > 0.0f ? (SAMPLE_BINS - 1) / fminf(span, 40.0f * temperature) : 0.0f;
    u64 sum = 0, total;
    for_each(r.x, 0, r.V, tid, 1024, [&](int i, float v) {
      if (r.in_prefix(key_of(v), i)) sum += r.weight(v);
    });
    block_scan64(s, sum, &total);
    sample_cut<false>(s, r, cut_mass(total));
  }
  const int token = sample_pick(s, r, [&](int i, float v) {
    if (!r.in_prefix(key_of(v), i)) return (u64)0;
    const u64 w = r.weight(v);
    return w >= r.least ? w : (u64)0;
  }, target);
  if (tid == 0) a.out[row] = token;
}

size_t pt_sample_workspace(int32_t, int32_t) { return 0; }

int pt_launch_sample(const pt_sample_args& a, hipStream_t s) {
  hipLaunchKernelGGL(sample_kernel, dim3((unsigned)a.rows), dim3(1024), 0, s, a);
  PT_HIP_CHECK(hipGetLastError());
  return PT_OK;
}
