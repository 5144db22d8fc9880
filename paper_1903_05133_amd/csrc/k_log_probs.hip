// Log probabilities of given labels with entropy and top alternatives, and
// their gradient (include/hieravg.h, hieravg_log_probs).
//
// A row x needs m = max x, Z = sum exp(x - m) and S = sum exp(x - m) (x - m):
// lse = m + log Z, log p_j = (x_j - m) - log Z, entropy = log Z - S / Z.  All
// three are kept in one pass, in float32: where the maximum rises by d, Z takes
// the factor exp(-d), and S that factor and -d times it of Z.  Reading the
// logits once is the bound of large calls, launches that of small ones.
#include <algorithm>
#include <cmath>

#include "ops.h"

namespace hav {

namespace {

constexpr float kLog2e = 1.44269504088896340736f;
// exp of a difference d <= 0, off by (1.25 |d| + 2) 2^-24 of it, most of which
// is the product's rounding: little beside a sum's larger terms, and beside
// results of 16 bits (2^-12 at |d| = 2000, where it is 0).  0 below 2^-126.
__device__ inline float exp_of(float d) { return __builtin_amdgcn_exp2f(d * kLog2e); }
// The same for results that stay float32, off by 4 2^-24: exp2 of the rounded
// product, times 2 to the rest of it.
__device__ inline float exp_close(float d) {
  const float c = d < -150.0f ? -150.0f : d;  // exp(-150) is 0; NaN stays
  const float t = c * kLog2e, rest = fmaf(c, kLog2e, -t) + c * 1.92596303e-8f;  // log2(e) - kLog2e
  const float e = __builtin_amdgcn_exp2f(t);
  return fmaf(e, rest * 0.693147181f, e);
}

struct LogProbArgs {
  const void* x;
  int64_t rows, stride;
  int classes, top;
  const void* labels;
  int label_bytes;
  float *logp, *entropy, *lse, *top_logp;
  int32_t* top_ids;
  int parts, part;  // parts of a row, classes of each
  uint64_t* keys;   // [rows][parts][top] candidates of the parts, if parts > 1
  f32x4* sums;      // [rows][parts] their sums
};

__device__ inline int64_t label_of(const void* labels, int bytes, int64_t r) {
  return bytes == 8 ? ((const int64_t*)labels)[r] : (int64_t)((const int32_t*)labels)[r];
}

// Order of the logits as unsigned integers: NaN above +inf, -0 as 0.
__device__ inline uint32_t order_of(float x) {
  if (x != x) return 0xFFFFFFFEu;  // below the key that no class has
  const uint32_t b = __float_as_uint(x + 0.0f);
  return b & 0x80000000u ? ~b : b | 0x80000000u;
}
// With the index: larger value first, of equal ones the lower index.
__device__ inline uint64_t key_of(float x, uint32_t j) { return (uint64_t)order_of(x) << 32 | (0xFFFFFFFFu - j); }
__device__ inline int class_of(uint64_t key) { return (int)(0xFFFFFFFFu - (uint32_t)key); }

// The partial sums of a part of a row: greatest value m, sum of exp(x - m) and
// of exp(x - m) (x - m).
struct Sums {
  float m, z, s;
};
// The same sums from the greatest value m >= a.m.  exp(d) d is 0 where exp(d)
// is: d may be infinite, or overflow with z.
__device__ inline Sums from_max(const Sums& a, float m) {
  if (a.m == -INFINITY) return {m, a.z, 0.0f};  // nothing, or NaN
  const float d = a.m - m, e = exp_of(d), ed = e == 0.0f ? 0.0f : e * d;
  return {m, e * a.z, e * a.s + ed * a.z};
}
__device__ inline Sums joined(const Sums& a, const Sums& b) {
  const float m = fmaxf(a.m, b.m);
  const Sums x = from_max(a, m), y = from_max(b, m);
  return {m, x.z + y.z, x.s + y.s};
}
// Over the lanes of a wave, in all of them.
__device__ inline Sums joined_wave(Sums a) {
  a = from_max(a, max_over_wave(a.m));
  return {a.m, add_over_wave(a.z), add_over_wave(a.s)};
}

// What a row's sums say: m, log z (NaN without a distribution), entropy.
struct RowStats {
  float m, logz, entropy;
};
__device__ inline RowStats row_stats(const Sums& t) {
  const bool some = t.z > 0.0f && t.m != INFINITY;
  const float logz = some ? logf(t.z) : NAN;
  return {t.m, logz, logz - t.s / t.z};
}
template <class T>
__device__ inline void write_row(const LogProbArgs& a, int64_t r, const T* x, const RowStats& q) {
  if (a.lse) a.lse[r] = q.m + q.logz;
  if (a.entropy) a.entropy[r] = q.entropy;
  if (a.logp) {
    const int64_t y = label_of(a.labels, a.label_bytes, r);
    a.logp[r] = y < 0 ? 0.0f : y >= a.classes ? NAN : to_f32(x[y]) - q.m - q.logz;
  }
}

// ------------------------------------------------------------ few classes
// A row in the registers of L lanes, E classes each; for the top rounds of a
// maximum over the lanes and the lowest index that has it.  Its few
// microseconds are a launch, a load and those rounds one after the other
// (512 x 1000 with five of the top: 6.9 us on the device; 4096 x 10: 3.7).
template <int L>
__device__ inline float max_lanes(float v) {
  if (L == 64) return max_over_wave(v);
  v = fmaxf(v, dpp_f<0xB1>(v));
  v = fmaxf(v, dpp_f<0x4E>(v));
  v = fmaxf(v, dpp_f<0x141>(v));
  return fmaxf(v, dpp_f<0x140>(v));
}
template <int L>
__device__ inline float add_lanes(float v) {
  if (L == 64) return add_over_wave(v);
  v += dpp_f<0xB1>(v);
  v += dpp_f<0x4E>(v);
  v += dpp_f<0x141>(v);
  return v + dpp_f<0x140>(v);
}
template <int L>
__device__ inline uint32_t max_lanes(uint32_t v) {
  return L == 64 ? max_over_wave(v) : max16(v);
}

template <class T, int L, int E>
__global__ __launch_bounds__(256) void k_log_probs_few(LogProbArgs a) {
  constexpr int V = E < 4 ? E : 4;  // consecutive classes of a lane
  const int lane = threadIdx.x & (L - 1);
  const int64_t r = ((int64_t)blockIdx.x * 256 + threadIdx.x) / L;
  const bool on = r < a.rows;  // the lanes of a wave stay together
  const T* x = (const T*)a.x + (on ? r : 0) * a.stride;
  float v[E];
#pragma unroll
  for (int i = 0; i < E / V; ++i) {
    const int j = (i * L + lane) * V;
    if (j + V <= a.classes) {
      const Pack<T, V> p = load_pack<T, V>(x + j);
#pragma unroll
      for (int e = 0; e < V; ++e) v[i * V + e] = to_f32(p.v[e]);
    } else {
#pragma unroll
      for (int e = 0; e < V; ++e) v[i * V + e] = j + e < a.classes ? to_f32(x[j + e]) : -INFINITY;
    }
  }
  float m = -INFINITY;
#pragma unroll
  for (int e = 0; e < E; ++e) m = fmaxf(m, v[e]);
  m = max_lanes<L>(m);
  const float base = m == -INFINITY ? 0.0f : m;
  Sums t = {m, 0.0f, 0.0f};
#pragma unroll
  for (int e = 0; e < E; ++e) {
    const float d = v[e] - base, p = exp_of(d);
    t.z += p;
    t.s += p * fmaxf(d, -200.0f);  // exp(-200) is 0: so is its product with -inf
  }
  t.z = add_lanes<L>(t.z);
  t.s = add_lanes<L>(t.s);
  const RowStats q = row_stats(t);
  if (on && lane == 0) write_row(a, r, x, q);
  if (a.top == 0) return;
  uint32_t ord[E];
#pragma unroll
  for (int e = 0; e < E; ++e) {
    const int j = (e / V * L + lane) * V + e % V;
    ord[e] = j < a.classes ? order_of(v[e]) : 0;  // 0: below every value's
  }
  for (int k = 0; k < a.top; ++k) {
    uint32_t best = 0;
#pragma unroll
    for (int e = 0; e < E; ++e) best = max(best, ord[e]);
    const uint32_t most = max_lanes<L>(best);
    int at = 0;  // of this lane's classes with that value the lowest
#pragma unroll
    for (int e = E - 1; e >= 0; --e)
      if (ord[e] == most) at = e;
    const int j = (at / V * L + lane) * V + at % V;
    const uint32_t low = ~max_lanes<L>(best == most ? ~(uint32_t)j : 0u);
    const bool mine = best == most && (uint32_t)j == low;
    if (mine && on) {
      float xv = v[0];
#pragma unroll
      for (int e = 1; e < E; ++e)
        if (at == e) xv = v[e];
      a.top_ids[r * a.top + k] = j;
      a.top_logp[r * a.top + k] = xv - q.m - q.logz;
    }
#pragma unroll
    for (int e = 0; e < E; ++e)
      if (mine && at == e) ord[e] = 0;
  }
}

// ------------------------------------------------------------ many classes
// One workgroup per part of a row, one pass: TILE = 16 or 32 classes a thread at
// a time (a tile of 4096 or 8192), with the thread's own running maximum and sums, joined at the
// end.  The top: each thread's maximum so far is a different class, so a value
// that `top` of the 256 maxima reach is a lower bound of the top-th class.
// Classes above it (of the first tile: or at it) go to a list in LDS; the bound
// is taken again after 2, 4, 8, .. tiles, so the list grows by about `top`
// entries each time the classes seen double.  At the end each entry counts the
// entries before it, and the first `top` are the answer.  A list that runs over
// (a masked beginning or part, many ties, rising rows) is made again in a second
// reading, of the classes above the exact bound and, as their order is that of
// the index, of each wave's first `top` at it (2048 x 131072 bf16 whose first half
// is -inf: 5692 us by searches, 254 so).  A row with NaN, or a list that runs
// over again, is searched `top` times for the next key.  A list that is nearly
// full and does not run over takes its time in ordering (64 x 131072 bf16 in
// rising order, whose parts are runs of equal values: 165 us, 20 for random rows).
constexpr int kCandidates = 1024;
constexpr int kMaxParts = 64;

struct TopShared {
  uint32_t maxima[256];
  uint64_t list[kCandidates];
  uint32_t bound, count;
  Sums sums[4];
  uint64_t wave_best[4];
};

// The largest value, of those whose order's lower 16 bits are 0, that `top` of the
// maxima (given as orders) reach: a search bit by bit in one wave, by ballots.
// For bf16 from 0 up that is the value itself; below 0, where the order is the
// complement of the bits, the float next above the bf16 value below it, so that
// classes equal to the value that was meant are listed too.  Up to 32 of the top: of the maxima of four threads each, one a
// lane (the bound is reached by 44 classes for 32, as of random values).  EXACT:
// the largest of all values that `top` of the 256 reach.
template <bool EXACT>
__device__ inline float take_bound(TopShared& sh, uint32_t mine, int top) {
  constexpr int kLow = EXACT ? 0 : 16;
  const int tid = threadIdx.x;
  const bool fours = !EXACT && top <= 32;
  if (fours) {
    mine = max(mine, dpp_u<0xB1>(mine));
    mine = max(mine, dpp_u<0x4E>(mine));
    if ((tid & 3) == 0) sh.maxima[tid >> 2] = mine;
  } else {
    sh.maxima[tid] = mine;
  }
  __syncthreads();
  if (tid < 64) {
    uint32_t t = 0;
    if (fours) {
      const uint32_t w = sh.maxima[tid];
      for (int bit = 31; bit >= kLow; --bit) {
        const uint32_t c = t | 1u << bit;
        if (__popcll(__ballot(w >= c)) >= top) t = c;
      }
    } else {
      const u32x4 w = *(const u32x4*)&sh.maxima[4 * tid];
      for (int bit = 31; bit >= kLow; --bit) {
        const uint32_t c = t | 1u << bit;
        const int n = __popcll(__ballot(w[0] >= c)) + __popcll(__ballot(w[1] >= c)) + __popcll(__ballot(w[2] >= c)) +
                      __popcll(__ballot(w[3] >= c));
        if (n >= top) t = c;
      }
    }
    if (tid == 0) sh.bound = t;
  }
  __syncthreads();
  const uint32_t o = sh.bound;
  // below -inf's order (empty threads' maxima): everything
  return o < 0x007FFFFFu ? -INFINITY : __uint_as_float(o & 0x80000000u ? o & 0x7FFFFFFFu : ~o);
}

__device__ inline uint64_t max_wave(uint64_t v) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) {
    const uint64_t w = __shfl_xor((unsigned long long)v, o, 64);
    v = max(v, w);
  }
  return v;
}

// The largest of the workgroup's keys, in every thread.
__device__ inline uint64_t max_group(TopShared& sh, uint64_t v) {
  v = max_wave(v);
  __syncthreads();  // the last result has been read
  if ((threadIdx.x & 63) == 0) sh.wave_best[threadIdx.x >> 6] = v;
  __syncthreads();
  v = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) v = max(v, sh.wave_best[i]);
  return v;
}

// At eight workgroups on a CU 110 to 119 us for 2048 x 131072 bf16 and 20 of the
// top (131 with seven where eight took 119); 102 without the top (5.3 TB/s).
template <class T, int TILE>
__global__ __launch_bounds__(256, 8) void k_log_probs(LogProbArgs a) {
  constexpr int V = sizeof(T) == 4 ? 4 : 8;  // classes per 16 bytes
  __shared__ TopShared sh;
  const int64_t r = blockIdx.x / a.parts;
  const int part = blockIdx.x - (int)(r * a.parts);
  const T* x = (const T*)a.x + r * a.stride;
  const int c0 = part * a.part, c1 = min(c0 + a.part, a.classes);
  const int tid = threadIdx.x;
  const int top = min(a.top, c1 - c0);
  if (tid == 0) sh.count = 0;
  Sums t = {-INFINITY, 0.0f, 0.0f};
  float seen = -INFINITY, bound = 0.0f;
  int tile = 0;
  for (int64_t base = c0; base < c1; base += (256 * TILE), ++tile) {
    float v[TILE];
    if (base + (256 * TILE) <= c1) {  // all loads before the first use
      Pack<T, V> p[TILE / V];
#pragma unroll
      for (int i = 0; i < TILE / V; ++i) p[i] = load_pack<T, V>(x + base + (i * 256 + tid) * V);
#pragma unroll
      for (int i = 0; i < TILE; ++i) v[i] = to_f32(p[i / V].v[i % V]);
    } else {
#pragma unroll
      for (int i = 0; i < TILE / V; ++i) {
        const int64_t j = base + (i * 256 + tid) * V;
        if (j + V <= c1) {
          const Pack<T, V> p = load_pack<T, V>(x + j);
#pragma unroll
          for (int e = 0; e < V; ++e) v[i * V + e] = to_f32(p.v[e]);
        } else {
#pragma unroll
          for (int e = 0; e < V; ++e) v[i * V + e] = j + e < c1 ? to_f32(x[j + e]) : -INFINITY;
        }
      }
    }
    float eight[TILE / 8], m = -INFINITY;  // maxima of eight classes each
#pragma unroll
    for (int g = 0; g < TILE / 8; ++g) {
      eight[g] = v[8 * g];
#pragma unroll
      for (int e = 1; e < 8; ++e) eight[g] = fmaxf(eight[g], v[8 * g + e]);
      m = fmaxf(m, eight[g]);
    }
    seen = fmaxf(seen, m);
    if (m > t.m) t = from_max(t, m);
    const float from = t.m == -INFINITY ? 0.0f : t.m;
#pragma unroll
    for (int e = 0; e < TILE; ++e) {
      const float d = v[e] - from, p = exp_of(d);
      t.z += p;
      t.s += p * fmaxf(d, -200.0f);  // exp(-200) is 0: so is its product with -inf
    }
    if (top > 0) {
      if (tile == 0) bound = take_bound<false>(sh, order_of(seen), top);
      // Later classes at the bound come after `top` that are not below it.
      // Some lane of a wave has one in most tiles: looked for by eights.
#pragma unroll
      for (int g = 0; g < TILE / 8; ++g) {
        if (tile == 0 ? eight[g] >= bound : eight[g] > bound) {
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            const int e = 8 * g + i;
            const int64_t j = base + (e / V * 256 + tid) * V + e % V;
            if ((tile == 0 ? v[e] >= bound : v[e] > bound) && j < c1) {
              const uint32_t at = atomicAdd(&sh.count, 1u);
              if (at < kCandidates) sh.list[at] = key_of(v[e], (uint32_t)j);
            }
          }
        }
      }
      if (tile > 0 && (tile & (tile + 1)) == 0 && base + (256 * TILE) < c1) bound = take_bound<false>(sh, order_of(seen), top);
    }
  }
  // The row's sums.
  t = joined_wave(t);
  if ((tid & 63) == 0) sh.sums[tid >> 6] = t;
  __syncthreads();
  t = sh.sums[0];
#pragma unroll
  for (int i = 1; i < 4; ++i) t = joined(t, sh.sums[i]);
  const RowStats q = row_stats(t);
  if (tid == 0) {
    if (a.parts > 1)
      a.sums[blockIdx.x] = f32x4{t.m, t.z, t.s, 0.0f};
    else
      write_row(a, r, x, q);
  }
  if (a.top == 0) return;
  auto put = [&](int k, uint64_t key) {
    if (a.parts > 1) {
      a.keys[(int64_t)blockIdx.x * a.top + k] = key;
    } else {
      const int j = class_of(key);
      a.top_ids[r * a.top + k] = j;
      a.top_logp[r * a.top + k] = to_f32(x[j]) - q.m - q.logz;
    }
  };
  int n = (int)sh.count;
  if (n > kCandidates && t.z == t.z) {
    bound = take_bound<true>(sh, order_of(seen), top);
    if (tid == 0) sh.count = 0;  // read by every thread before that bound
    __syncthreads();
    int ties = 0;  // of this wave's classes so far
    for (int64_t base = c0; base < c1; base += 256 * V) {
      const int64_t j = base + tid * V;
      float v[V];
      if (j + V <= c1) {
        const Pack<T, V> p = load_pack<T, V>(x + j);
#pragma unroll
        for (int e = 0; e < V; ++e) v[e] = to_f32(p.v[e]);
      } else {
#pragma unroll
        for (int e = 0; e < V; ++e) v[e] = j + e < c1 ? to_f32(x[j + e]) : NAN;
      }
      int before = ties;  // ties of this wave before this class
#pragma unroll
      for (int e = 0; e < V; ++e) {
        const uint64_t tie = __ballot(v[e] == bound);
        before += __popcll(tie & ((1ull << (tid & 63)) - 1));
        ties += __popcll(tie);
      }
#pragma unroll
      for (int e = 0; e < V; ++e) {
        const bool tie = v[e] == bound;
        if (v[e] > bound || (tie && before < top)) {
          const uint32_t at = atomicAdd(&sh.count, 1u);
          if (at < kCandidates) sh.list[at] = key_of(v[e], (uint32_t)(j + e));
        }
        before += tie ? 1 : 0;
      }
    }
    __syncthreads();
    n = (int)sh.count;
  }
  if (n <= kCandidates && n >= top && t.z == t.z) {
    for (int i = tid; i < n; i += 256) {
      const uint64_t key = sh.list[i];
      int before = 0;
      for (int j = 0; j < n; ++j) before += sh.list[j] > key ? 1 : 0;
      if (before < top) put(before, key);
    }
  } else {
    uint64_t last = ~0ull;
    for (int k = 0; k < top; ++k) {
      uint64_t best = 0;
      for (int64_t j = c0 + tid; j < c1; j += 256) {
        const uint64_t key = key_of(to_f32(x[j]), (uint32_t)j);
        if (key < last && key > best) best = key;
      }
      last = max_group(sh, best);
      if (tid == 0) put(k, last);
    }
  }
  if (a.parts > 1)
    for (int k = top + tid; k < a.top; k += 256) a.keys[(int64_t)blockIdx.x * a.top + k] = 0;
}

// The parts of a row together: their sums, and the first `top` of their
// candidates.  These are in falling order within a part, so the largest
// top-th entry of a part, and the least of the parts' entry number
// ceil(top / parts), are reached by `top` candidates: what is not below both is
// listed, and each entry counts the entries before it.
template <class T>
__global__ __launch_bounds__(256) void k_log_probs_join(LogProbArgs a) {
  __shared__ uint64_t list[kMaxParts * HIERAVG_TOP_MAX];
  __shared__ uint64_t most[4], least[4];
  __shared__ uint32_t count;
  const int64_t r = blockIdx.x;
  const T* x = (const T*)a.x + r * a.stride;
  const int tid = threadIdx.x, top = a.top;
  Sums t = {-INFINITY, 0.0f, 0.0f};
  if ((tid & 63) < a.parts) {
    const f32x4 s = a.sums[r * a.parts + (tid & 63)];
    t = Sums{s[0], s[1], s[2]};
  }
  const RowStats q = row_stats(joined_wave(t));
  if (tid == 0) write_row(a, r, x, q);
  if (top == 0) return;
  const uint64_t* keys = a.keys + r * a.parts * top;
  const int n = a.parts * top, step = (top + a.parts - 1) / a.parts;
  if (tid == 0) count = 0;
  uint64_t hi = 0, lo = ~0ull;
  for (int p = tid; p < a.parts; p += 256) {
    hi = max(hi, keys[p * top + top - 1]);
    lo = min(lo, keys[p * top + step - 1]);
  }
  hi = max_wave(hi);
  lo = ~max_wave(~lo);
  if ((tid & 63) == 0) {
    most[tid >> 6] = hi;
    least[tid >> 6] = lo;
  }
  __syncthreads();
  const uint64_t bound = max(max(max(most[0], most[1]), max(most[2], most[3])), min(min(least[0], least[1]), min(least[2], least[3])));
  for (int i = tid; i < n; i += 256) {
    const uint64_t key = keys[i];
    if (key >= bound && key != 0) list[atomicAdd(&count, 1u)] = key;
  }
  __syncthreads();
  const int m = (int)count;
  for (int i = tid; i < m; i += 256) {
    const uint64_t key = list[i];
    int before = 0;
    for (int j = 0; j < m; ++j) before += list[j] > key ? 1 : 0;
    if (before < top) {
      const int j = class_of(key);
      a.top_ids[r * top + before] = j;
      a.top_logp[r * top + before] = to_f32(x[j]) - q.m - q.logz;
    }
  }
}

// ------------------------------------------------------------ the gradient
struct GradArgs {
  const void* x;
  void* grad;
  int64_t rows, stride, grad_stride;
  int classes;
  const void* labels;
  int label_bytes;
  const float *lse, *entropy, *g_logp, *g_entropy;
};

// Elementwise, read once and written once, 16 classes a thread: HBM is the
// bound (2048 x 131072 bf16 with the entropy's part: 187 us, 5.7 TB/s).
//
// lse rounded to float32 makes every p of its row off by |lse| 2^-24.  Past
// kFarLse (4e-6) one workgroup takes the whole row: it sums it again, and where lse is
// this row's own to its rounding, log p is (x - m) - log Z, as in the forward
// (a second reading: 2048 x 131072 bf16 403 us, 1 x 131072 63).  Any other lse is the caller's, and taken as it is.
constexpr int kGradChunk = 256 * 16;
constexpr float kFarLse = 64.0f;
template <class T>
__global__ __launch_bounds__(256) void k_log_probs_grad(GradArgs a) {
  constexpr int V = sizeof(T) == 4 ? 4 : 8;
  const int64_t r = blockIdx.y;
  // A wave without classes (a barrier waits for those that are left).
  if (gridDim.x == 1 && __builtin_amdgcn_readfirstlane((int)threadIdx.x) * V >= a.classes) return;
  const float lse = a.lse[r];
  const int64_t y = a.g_logp ? label_of(a.labels, a.label_bytes, r) : -1;
  float g = a.g_logp && y >= 0 ? a.g_logp[r] : 0.0f;
  const float h = a.g_entropy ? a.g_entropy[r] : 0.0f;
  if (y >= a.classes) g = NAN;
  const bool zero = g == 0.0f && h == 0.0f;
  const float ent = a.g_entropy ? a.entropy[r] : 0.0f;
  const T* x = (const T*)a.x + r * a.stride;
  T* o = (T*)a.grad + r * a.grad_stride;
  // Chunk c of the row by log_p of its logits; none: zeros.
  auto chunk = [&](int64_t c, bool none, auto&& log_p) {
    auto grad = [&](float v, int64_t j) {
      const float l = log_p(v), p = sizeof(T) == 4 ? exp_close(l) : exp_of(l);
      return (j == y ? g : 0.0f) - p * g - (p == 0.0f ? 0.0f : h * p * (l + ent));
    };
#pragma unroll
    for (int i = 0; i < 16 / V; ++i) {
      const int64_t j = c * kGradChunk + (i * 256 + threadIdx.x) * V;
      if (j >= a.classes) break;
      if (j + V <= a.classes) {
        Pack<T, V> p, d;
        if (!none) p = load_pack<T, V>(x + j);
#pragma unroll
        for (int e = 0; e < V; ++e) from_f32(none ? 0.0f : grad(to_f32(p.v[e]), j + e), &d.v[e]);
        store_pack<T, V>(o + j, d);
      } else {
        for (int e = 0; j + e < a.classes; ++e) from_f32(none ? 0.0f : grad(to_f32(x[j + e]), j + e), &o[j + e]);
      }
    }
  };
  if (zero) return chunk(blockIdx.x, true, [](float v) { return v; });
  if (!(fabsf(lse) > kFarLse && fabsf(lse) < INFINITY))
    return chunk(blockIdx.x, false, [&](float v) { return v - lse; });
  if (blockIdx.x != (unsigned)(r % gridDim.x)) return;  // one XCD has every eighth workgroup
  // Each wave for itself: four waves' loads are one from memory.
  Sums t = {-INFINITY, 0.0f, 0.0f};
  for (int64_t base = 0; base < a.classes; base += 64 * 4 * V) {
    Pack<T, V> p[4];
    const int64_t j0 = base + (threadIdx.x & 63) * V;
    float v[4 * V], most = -INFINITY;
    if (base + 64 * 4 * V <= a.classes) {  // all loads before the first use
#pragma unroll
      for (int i = 0; i < 4; ++i) p[i] = load_pack<T, V>(x + j0 + i * 64 * V);
#pragma unroll
      for (int i = 0; i < 4 * V; ++i) v[i] = to_f32(p[i / V].v[i % V]);
    } else {
#pragma unroll
      for (int i = 0; i < 4 * V; ++i) {
        const int64_t j = j0 + (i / V) * 64 * V + i % V;
        v[i] = j < a.classes ? to_f32(x[j]) : -INFINITY;
      }
    }
#pragma unroll
    for (int i = 0; i < 4 * V; ++i) most = fmaxf(most, v[i]);
    if (most > t.m) t = from_max(t, most);
    const float from = t.m == -INFINITY ? 0.0f : t.m;
#pragma unroll
    for (int i = 0; i < 4 * V; ++i) t.z += exp_of(v[i] - from);
  }
  t = joined_wave(t);
  __syncthreads();  // the whole row has been read: o may be x
  const float m = t.m, logz = row_stats(t).logz;
  const bool own = fabsf(lse - (m + logz)) <= 0x1p-22f * fabsf(lse);
  const float base = own ? m : lse, rest = own ? logz : 0.0f;
  for (unsigned c = 0; c < gridDim.x; ++c) chunk(c, false, [&](float v) { return (v - base) - rest; });
}

// How the rows are taken.
struct RowPlan {
  int parts, part, tile;  // 0 parts: few classes
};
constexpr int kFewClasses = 1024, kFewTop = 8;
constexpr int64_t kPartMost = 131072;  // classes that a list's capacity is made for
constexpr int64_t kMostClasses = kPartMost * kMaxParts;

// Few classes in a wave, unless many rounds for the top would take longer than
// a list (512 x 1000, 64 of the top: 41 us).  Else parts of 4096 classes or more
// for up to 2048 workgroups (eight per CU: 1500 x 50001 in one part 40 us, in two
// 52); up to 8192 classes one part, which a second launch to join two would
// outweigh (1 x 5000 in a graph 7.9 against 10.4 us, a call 10.9 against 14.3).
RowPlan plan_rows(int64_t rows, int64_t classes, int top) {
  if (classes <= 64 || (classes <= kFewClasses && top <= kFewTop)) return {0, (int)classes, 0};
  const int64_t least = (classes + kPartMost - 1) / kPartMost;
  const int64_t most = classes <= 8192 ? 1 : std::min<int64_t>((classes + 4095) / 4096, kMaxParts);
  const int64_t parts = std::max({least, int64_t(1), std::min(most, 2048 / rows)});
  // Whole tiles, whose loads are all under way at once, where a part has one.
  // The large tile has more of them under way, the small one less to do before
  // the first bound (2048 x 131072: 119 against 128 us; 4096 x 4096: 22.4 against 17.3).
  const int64_t even = (classes + parts - 1) / parts;
  const int tile = even > 65536 ? 32 : 16;
  const int64_t part = round_up(even, even > 128 * tile ? 256 * tile : 64);
  return {(int)((classes + part - 1) / part), (int)part, tile};
}

int check_logits(const void* logits, int32_t type, int64_t rows, int64_t classes, int64_t stride) {
  if (!known_type(type)) return invalid("unknown element type");
  if (rows < 0 || rows > 0x7FFFFFFF) return invalid("rows must be in [0, 2^31)");
  if (classes < 1 || classes > kMostClasses) return invalid("classes must be in [1, 2^23]");
  if (stride < classes || !addressable(rows, stride, type_bytes(type)))
    return invalid("row_stride must be at least classes, the rows within 2^56 bytes");
  if (rows > 0 && (!logits || !aligned(logits, type_bytes(type))))
    return invalid("logits must be a pointer aligned to its element");
  return HIERAVG_OK;
}

// Whether rows of two matrices share memory; the same rows, and rows that lie
// between the other's, do not.
bool rows_collide(const void* a, int64_t a_stride, const void* b, int64_t b_stride, int64_t rows, int64_t classes, int bytes) {
  const uintptr_t x = (uintptr_t)a, y = (uintptr_t)b, row = (uintptr_t)classes * bytes;
  const uintptr_t sx = (uintptr_t)a_stride * bytes, sy = (uintptr_t)b_stride * bytes, n = (uintptr_t)rows - 1;
  if (x + n * sx + row <= y || y + n * sy + row <= x) return false;
  if (rows == 1 || sx != sy) return x != y || rows > 1;
  const uintptr_t d = (x > y ? x - y : y - x) % sx;
  return x != y && (d < row || d > sx - row);
}

int check_labels(const void* labels, int32_t label_bytes) {
  if (label_bytes != 4 && label_bytes != 8) return invalid("label_bytes must be 4 or 8");
  if (!labels || !aligned(labels, label_bytes)) return invalid("labels must be a pointer aligned to its element");
  return HIERAVG_OK;
}

template <class T>
void launch_log_probs(hipStream_t s, const LogProbArgs& a, const RowPlan& pl) {
  const unsigned grid = (unsigned)(a.rows * pl.parts);
  if (pl.parts == 0) {
    const unsigned g16 = (unsigned)((a.rows + 15) / 16), g64 = (unsigned)((a.rows + 3) / 4);
    if (a.classes <= 16)
      launch(k_log_probs_few<T, 16, 1>, g16, 256, 0, s, a);
    else if (a.classes <= 64)
      launch(k_log_probs_few<T, 16, 4>, g16, 256, 0, s, a);
    else if (a.classes <= 256)
      launch(k_log_probs_few<T, 64, 4>, g64, 256, 0, s, a);
    else
      launch(k_log_probs_few<T, 64, 16>, g64, 256, 0, s, a);
  } else {
    if (pl.tile == 32)
      launch(k_log_probs<T, 32>, grid, 256, 0, s, a);
    else
      launch(k_log_probs<T, 16>, grid, 256, 0, s, a);
  }
  if (a.parts > 1) launch(k_log_probs_join<T>, (unsigned)a.rows, 256, 0, s, a);
}

}  // namespace

}  // namespace hav

using namespace hav;

extern "C" {

size_t hieravg_log_probs_scratch(int64_t rows, int64_t classes, int32_t top) {
  if (rows < 1 || rows > 0x7FFFFFFF || classes < 1 || classes > kMostClasses || top < 0 || top > HIERAVG_TOP_MAX) return 0;
  const RowPlan p = plan_rows(rows, classes, top);
  return p.parts > 1 ? (size_t)rows * p.parts * (sizeof(f32x4) + sizeof(uint64_t) * top) : 0;
}

int hieravg_log_probs(const void* logits, int32_t type, int64_t rows, int64_t classes, int64_t row_stride,
                      const void* labels, int32_t label_bytes, int32_t top, float* logp, float* entropy, float* lse,
                      int32_t* top_ids, float* top_logp, void* scratch, size_t scratch_bytes, void* hip_stream) {
  return guarded([&]() -> int {
    int rc = check_logits(logits, type, rows, classes, row_stride);
    if (rc != HIERAVG_OK) return rc;
    if (top < 0 || top > HIERAVG_TOP_MAX || top > classes)
      return invalid("top must be in [0, min(classes, HIERAVG_TOP_MAX)]");
    if (rows == 0) return HIERAVG_OK;
    if (logp && (rc = check_labels(labels, label_bytes)) != HIERAVG_OK) return rc;
    if (top > 0 && (!top_ids || !top_logp)) return invalid("top > 0 needs top_ids and top_logp");
    const size_t need = hieravg_log_probs_scratch(rows, classes, top);
    if (need && (!scratch || scratch_bytes < need || !aligned(scratch, 16)))
      return invalid("scratch must hold hieravg_log_probs_scratch bytes, 16-byte aligned");
    const RowPlan pl = plan_rows(rows, classes, top);
    LogProbArgs a{logits, rows, row_stride, (int)classes, top, labels, label_bytes, logp, entropy, lse, top_logp, top_ids,
                  pl.parts, pl.part, nullptr, nullptr};
    if (pl.parts > 1) {
      a.sums = (f32x4*)scratch;
      a.keys = (uint64_t*)(a.sums + rows * pl.parts);
    }
    hipStream_t s = (hipStream_t)hip_stream;
    const int64_t step = kMaxGroups / std::max(pl.parts, 1);
    for (int64_t r0 = 0; r0 < rows; r0 += step) {
      LogProbArgs b = a;
      b.x = (const char*)logits + r0 * row_stride * type_bytes(type);
      b.rows = std::min(rows - r0, step);
      b.labels = labels ? (const char*)labels + r0 * label_bytes : nullptr;
      b.logp = logp ? logp + r0 : nullptr;
      b.entropy = entropy ? entropy + r0 : nullptr;
      b.lse = lse ? lse + r0 : nullptr;
      b.top_ids = top_ids ? top_ids + r0 * top : nullptr;
      b.top_logp = top_logp ? top_logp + r0 * top : nullptr;
      if (pl.parts > 1) {
        b.sums = a.sums + r0 * pl.parts;
        b.keys = a.keys + r0 * pl.parts * top;
      }
      if (type == HIERAVG_F32)
        launch_log_probs<float>(s, b, pl);
      else if (type == HIERAVG_F16)
        launch_log_probs<f16_t>(s, b, pl);
      else
        launch_log_probs<bf16_t>(s, b, pl);
    }
    return launched("hieravg_log_probs");
  });
}

int hieravg_log_probs_grad(const void* logits, int32_t type, int64_t rows, int64_t classes, int64_t row_stride,
                           const void* labels, int32_t label_bytes, const float* lse, const float* entropy,
                           const float* g_logp, const float* g_entropy, void* grad, int64_t grad_stride,
                           void* hip_stream) {
  return guarded([&]() -> int {
    int rc = check_logits(logits, type, rows, classes, row_stride);
    if (rc != HIERAVG_OK) return rc;
    if (grad_stride < classes || !addressable(rows, grad_stride, type_bytes(type)))
      return invalid("grad_stride must be at least classes, the rows within 2^56 bytes");
    if (rows == 0) return HIERAVG_OK;
    if (!grad || !aligned(grad, type_bytes(type))) return invalid("grad must be a pointer aligned to its element");
    if (rows_collide(logits, row_stride, grad, grad_stride, rows, classes, type_bytes(type)))
      return invalid("grad must be the logits (same pointer and row stride) or overlap none of their rows");
    if (!lse) return invalid("lse is NULL");
    if (!g_logp && !g_entropy) return invalid("g_logp and g_entropy are both NULL");
    if (g_logp && (rc = check_labels(labels, label_bytes)) != HIERAVG_OK) return rc;
    if (g_entropy && !entropy) return invalid("g_entropy needs entropy");
    GradArgs a{logits, grad, rows, row_stride, grad_stride, (int)classes, labels, label_bytes, lse, entropy, g_logp, g_entropy};
    hipStream_t s = (hipStream_t)hip_stream;
    for (int64_t r0 = 0; r0 < rows; r0 += 65535) {
      GradArgs b = a;
      const int es = type_bytes(type);
      b.x = (const char*)a.x + r0 * row_stride * es;
      b.grad = (char*)a.grad + r0 * grad_stride * es;
      b.labels = labels ? (const char*)labels + r0 * label_bytes : nullptr;
      b.lse = lse + r0;
      b.entropy = entropy ? entropy + r0 : nullptr;
      b.g_logp = g_logp ? g_logp + r0 : nullptr;
      b.g_entropy = g_entropy ? g_entropy + r0 : nullptr;
      const dim3 grid((unsigned)((classes + kGradChunk - 1) / kGradChunk), (unsigned)std::min<int64_t>(rows - r0, 65535));
      if (type == HIERAVG_F32)
        launch(k_log_probs_grad<float>, grid, 256, 0, s, b);
      else if (type == HIERAVG_F16)
        launch(k_log_probs_grad<f16_t>, grid, 256, 0, s, b);
      else
        launch(k_log_probs_grad<bf16_t>, grid, 256, 0, s, b);
    }
    return launched("hieravg_log_probs_grad");
  });
}

int hieravg_scores(hieravg_t h, int32_t replica, int32_t split, int64_t n_rows, int32_t top, float* logp,
                   float* entropy, int32_t* top_ids, float* top_logp) {
  return guarded([&]() -> int {
    if (!logp || !entropy) return invalid("logp or entropy is NULL");
    if (top < 0 || top > HIERAVG_TOP_MAX) return invalid("top must be in [0, min(classes, HIERAVG_TOP_MAX)]");
    if (top > 0 && (!top_ids || !top_logp)) return invalid("top > 0 needs top_ids and top_logp");
    // One chunk's results and scratch, for the call.
    struct Buffer {
      char* p = nullptr;
      ~Buffer() {
        if (p) (void)hipFree(p);
      }
    } buf;
    size_t cap = 0;
    return eval_logits(h, replica, split, n_rows, [&](const LogitRows& r) -> int {
      if (top > r.classes) return invalid("top must be in [0, min(classes, HIERAVG_TOP_MAX)]");
      const size_t rows = (size_t)r.rows, one = (size_t)round_up(4 * rows, 256), many = (size_t)round_up(4 * rows * top, 256);
      const size_t scratch = hieravg_log_probs_scratch(r.rows, r.classes, top), need = 2 * one + 2 * many + scratch;
      hipError_t e = hipSuccess;
      if (cap < need) {  // the first chunk is the largest, but a last one may take more scratch
        if (buf.p) (void)hipFree(buf.p);
        buf.p = nullptr;
        e = hipMalloc((void**)&buf.p, need);
        cap = need;
      }
      if (e == hipSuccess) {
        char *dl = buf.p, *de = dl + one, *di = de + one, *dt = di + many, *ds = dt + many;
        const int rc = hieravg_log_probs(r.logits, HIERAVG_F32, r.rows, r.classes, r.ld, r.labels, 4, top, (float*)dl, (float*)de,
                                         nullptr, (int32_t*)di, (float*)dt, ds, scratch, r.stream);
        if (rc != HIERAVG_OK) return rc;
        const size_t at = (size_t)r.first;
        e = hipMemcpyAsync(logp + at, dl, 4 * rows, hipMemcpyDefault, r.stream);
        if (e == hipSuccess) e = hipMemcpyAsync(entropy + at, de, 4 * rows, hipMemcpyDefault, r.stream);
        if (e == hipSuccess && top) e = hipMemcpyAsync(top_ids + at * top, di, 4 * rows * top, hipMemcpyDefault, r.stream);
        if (e == hipSuccess && top) e = hipMemcpyAsync(top_logp + at * top, dt, 4 * rows * top, hipMemcpyDefault, r.stream);
        if (e == hipSuccess) e = hipStreamSynchronize(r.stream);
      }
      if (e != hipSuccess) {
        set_error(std::string("hieravg_scores: ") + hipGetErrorString(e));
        return HIERAVG_EHIP;
      }
      return HIERAVG_OK;
    });
  });
}

}  // extern "C"
