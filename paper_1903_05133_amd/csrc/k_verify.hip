// Verification of drafted tokens (include/hieravg.h, hieravg_verify_drafts).
//
// Which drafts stand depends on probabilities of single classes: float32 sums
// of all rows, one pass over the logits, decide that unless the two sides of a
// comparison lie within the sums' error of each other; such a one is decided
// from sums in 64 bits.  Which class is drawn depends on where a uniform
// number falls among all sums of a distribution: the one row (or two) of each
// sequence that this concerns is summed in 64 bits.  So the tokens are those
// of the definition, whatever the parts that a row is summed in.
#include <algorithm>
#include <cmath>

#include "ops.h"

namespace hav {

namespace {

constexpr double kLog2e = 1.4426950408889634074;
constexpr int kMostParts = 64;      // a lane each where they are joined
constexpr int64_t kMostClasses = int64_t(1) << 23;

// A part of a row: largest value, sum of exp((x - m) / T), first class with the largest value.
struct Part {
  float m, z;
  int first, pad;
};
// What the decision found: the row whose distribution the token is drawn
// from, and how.
enum Kind { kNothing = 0, kTarget = 1, kDifference = 2, kGreedy = 3 };
struct Decision {
  int row;      // also the number of accepted drafts
  int kind;
  int removed;  // a class that is not drawn (a draft of certainty), or -1
  float m, mq;  // the rows' largest values
  int token;    // kGreedy: the token
  int pad[2];
};

struct VerifyArgs {
  const void *x, *q;  // logits of the target and of the draft model, or NULL
  int64_t stride, q_stride;
  int64_t seqs;
  int drafts, classes;
  const void* tokens_in;
  int token_bytes;
  const float *uniforms, *temperature;
  const int32_t* lengths;
  int32_t *tokens, *accepted;
  float* logp;
  float unsure;      // how far apart the sides of a comparison must be, relative
  int parts, part;   // of the float32 sums
  int fine, fine_part;  // of the sums in 64 bits
  Part *px, *pq;     // [seqs][drafts + 1][parts], [seqs][drafts][parts]
  double2* sums;     // [seqs][fine]: of the target's row, of the draft's
  double* rest;      // [seqs][fine]: of the difference
  Decision* decisions;
};

__device__ inline int drafts_of(const VerifyArgs& a, int64_t b) {
  return a.lengths ? min(max(a.lengths[b], 0), a.drafts) : a.drafts;
}
// log2(e) / T for float32 exponentials; the bounds keep 0 by it and -infinity by
// it as they are.  Past them (T above 1.9e36 or below 1.1e-36) the float32 sums tell
// whether there is a distribution, and nothing of it: 64 bits decide.
__device__ inline float exponent_of(double it) {
  return it > 0.0 ? (float)fmin(fmax(it * kLog2e, 0x1p-120), 0x1p120) : (float)kLog2e;
}
__device__ inline bool in_float32(double it) { return it * kLog2e >= 0x1p-120 && it * kLog2e <= 0x1p120; }
// 1 / T; 0 for the largest class alone.
__device__ inline double inverse_temperature(const VerifyArgs& a, int64_t b) {
  if (!a.temperature) return 1.0;
  const float t = a.temperature[b];
  return t > 0.0f && t < INFINITY ? 1.0 / (double)t : 0.0;
}
__device__ inline int64_t draft_of(const VerifyArgs& a, int64_t b, int i) {
  const int64_t at = b * a.drafts + i;
  return a.token_bytes == 8 ? ((const int64_t*)a.tokens_in)[at] : (int64_t)((const int32_t*)a.tokens_in)[at];
}

// e^t, t <= 0, off by (|t| + 4) 2^-53 of it, from a table (P. T. P. Tang, "Table-driven
// implementation of the exponential function in IEEE floating-point arithmetic",
// 1989): t = k ln 2 / 32 + r, 2^(i/32) from the table and the series of e^r to its sixth power, whose rest is below 2^-57 for
// |r| < 0.0109.  0 below -745; NaN stays.
struct ExpTable {
  double v[32];
};
__constant__ const double kPowers[32] = {  // 2^(i/32)
    0x1p+0, 0x1.059b0d3158574p+0, 0x1.0b5586cf9890fp+0, 0x1.11301d0125b51p+0, 0x1.172b83c7d517bp+0,
    0x1.1d4873168b9aap+0, 0x1.2387a6e756238p+0, 0x1.29e9df51fdee1p+0, 0x1.306fe0a31b715p+0,
    0x1.371a7373aa9cbp+0, 0x1.3dea64c123422p+0, 0x1.44e086061892dp+0, 0x1.4bfdad5362a27p+0,
    0x1.5342b569d4f82p+0, 0x1.5ab07dd485429p+0, 0x1.6247eb03a5585p+0, 0x1.6a09e667f3bcdp+0,
    0x1.71f75e8ec5f74p+0, 0x1.7a11473eb0187p+0, 0x1.82589994cce13p+0, 0x1.8ace5422aa0dbp+0,
    0x1.93737b0cdc5e5p+0, 0x1.9c49182a3f090p+0, 0x1.a5503b23e255dp+0, 0x1.ae89f995ad3adp+0,
    0x1.b7f76f2fb5e47p+0, 0x1.c199bdd85529cp+0, 0x1.cb720dcef9069p+0, 0x1.d5818dcfba487p+0,
    0x1.dfc97337b9b5fp+0, 0x1.ea4afa2a490dap+0, 0x1.f50765b6e4540p+0};
__device__ inline void fill(ExpTable& t) {
  if (threadIdx.x < 32) t.v[threadIdx.x] = kPowers[threadIdx.x];
}
__device__ inline double exp_of(const ExpTable& tab, double t) {
  const double c = t < -800.0 ? -800.0 : t;  // NaN stays
  const double k = rint(c * (32.0 * kLog2e));
  const double r = fma(k, -0x1.62e42fefa39efp-6, c);  // ln 2 / 32
  const int n = (int)k;
  double p = fma(r, 1.0 / 720.0, 1.0 / 120.0);
  p = fma(p, r, 1.0 / 24.0);
  p = fma(p, r, 1.0 / 6.0);
  p = fma(p, r, 0.5);
  p = fma(p, r, 1.0);
  p = fma(p, r, 1.0);
  const double e = ldexp(tab.v[n & 31] * p, n >> 5);
  return t == t ? e : t;
}

// ------------------------------------------------------------ sums of all rows
// A workgroup per part of a row: the running maximum and sum of a thread, joined
// at the end.  Memory is the bound: 576 rows of 131072 bf16 classes 25 us (6.0 TB/s).
template <class T>
__device__ inline void sum_part(const T* x, int c0, int c1, float by, bool find, Part* out) {
  constexpr int V = 16 / sizeof(T), TILE = 16;
  __shared__ Part waves[4];
  const int tid = threadIdx.x;
  float m = -INFINITY, z = 0.0f;
  int first = 0x7FFFFFFF;
  for (int base = c0; base < c1; base += 256 * TILE) {
    float v[TILE];
    if (base + 256 * TILE <= c1) {
      Pack<T, V> p[TILE / V];
#pragma unroll
      for (int i = 0; i < TILE / V; ++i) p[i] = load_pack<T, V>(x + base + (i * 256 + tid) * V);
#pragma unroll
      for (int i = 0; i < TILE; ++i) v[i] = to_f32(p[i / V].v[i % V]);
    } else {
#pragma unroll
      for (int i = 0; i < TILE / V; ++i) {
        const int j = base + (i * 256 + tid) * V;
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
    float most = v[0];
#pragma unroll
    for (int i = 1; i < TILE; ++i) most = fmaxf(most, v[i]);
    if (most > m) {
      z *= __builtin_amdgcn_exp2f((m - most) * by);
      m = most;
      if (find) {
        first = 0x7FFFFFFF;
#pragma unroll
        for (int i = TILE - 1; i >= 0; --i)
          if (v[i] == m) first = base + (i / V * 256 + tid) * V + i % V;
      }
    }
    const float from = m == -INFINITY ? 0.0f : m;
#pragma unroll
    for (int i = 0; i < TILE; ++i) z += __builtin_amdgcn_exp2f((v[i] - from) * by);
  }
  const float top = max_over_wave(m);
  z = m == -INFINITY ? z : z * __builtin_amdgcn_exp2f((m - top) * by);  // NaN without a maximum stays
  z = add_over_wave(z);
  first = m == top ? first : 0x7FFFFFFF;
  if (find) first = (int)~max_over_wave(~(uint32_t)first);
  if ((tid & 63) == 0) waves[tid >> 6] = {top, z, first, 0};
  __syncthreads();
  if (tid == 0) {
    Part r = waves[0];
#pragma unroll
    for (int i = 1; i < 4; ++i) {
      const Part w = waves[i];
      const float most = fmaxf(r.m, w.m);
      const float zr = r.m == -INFINITY ? r.z : r.z * __builtin_amdgcn_exp2f((r.m - most) * by);
      const float zw = w.m == -INFINITY ? w.z : w.z * __builtin_amdgcn_exp2f((w.m - most) * by);
      r.first = min(r.m == most ? r.first : 0x7FFFFFFF, w.m == most ? w.first : 0x7FFFFFFF);
      r.z = zr + zw;
      r.m = most;
    }
    *out = r;
  }
}

template <class T, class Q>
__global__ __launch_bounds__(256) void k_verify_sums(VerifyArgs a) {
  const int rows = a.q ? 2 * a.drafts + 1 : a.drafts + 1;  // of a sequence: the target's, then the draft model's
  const int64_t all = (int64_t)blockIdx.x / a.parts;
  const int part = (int)(blockIdx.x - all * a.parts);
  const int64_t b = all / rows;
  const int r = (int)(all - b * rows), n = drafts_of(a, b);
  const double it = inverse_temperature(a, b);
  const int c0 = part * a.part, c1 = min(c0 + a.part, a.classes);
  const float by = exponent_of(it);
  if (r <= a.drafts) {
    if (r <= n)
      sum_part((const T*)a.x + (b * (a.drafts + 1) + r) * a.stride, c0, c1, by, it == 0.0,
               a.px + (b * (a.drafts + 1) + r) * a.parts + part);
  } else {
    const int i = r - a.drafts - 1;
    if (i < n && it > 0.0)
      sum_part((const Q*)a.q + (b * a.drafts + i) * a.q_stride, c0, c1, by, false,
               a.pq + (b * a.drafts + i) * a.parts + part);
  }
}

// ------------------------------------------------------------ the decision
// A row's parts, a lane each, joined in all lanes of a wave.
__device__ inline Part part_of_lane(const Part* p, int parts) {
  const int lane = threadIdx.x & 63;
  const Part w = p[min(lane, parts - 1)];
  return lane < parts ? w : Part{-INFINITY, 0.0f, 0x7FFFFFFF, 0};
}
__device__ inline Part joined(const Part& w, float by) {
  const float m = max_over_wave(w.m);
  const float z = w.m == -INFINITY ? w.z : w.z * __builtin_amdgcn_exp2f((w.m - m) * by);
  Part r;
  r.m = m;
  r.z = add_over_wave(z);
  r.first = (int)~max_over_wave(~(uint32_t)(w.m == m ? w.first : 0x7FFFFFFF));
  r.pad = 0;
  return r;
}
// The same of a whole short row, by a wave.
template <class T>
__device__ inline Part row_of_wave(const T* x, int classes, float by) {
  const int lane = threadIdx.x & 63;
  float m = -INFINITY, z = 0.0f;
  int first = 0x7FFFFFFF;
  for (int base = 0; base < classes; base += 8 * 64) {
    float v[8], most = -INFINITY;
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = to_f32(x[min(base + i * 64 + lane, classes - 1)]);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      if (base + i * 64 + lane >= classes) v[i] = -INFINITY;
      most = fmaxf(most, v[i]);
    }
    if (most > m) {
      z *= __builtin_amdgcn_exp2f((m - most) * by);
      m = most;
#pragma unroll
      for (int i = 7; i >= 0; --i)
        if (v[i] == m) first = base + i * 64 + lane;
    }
    const float from = m == -INFINITY ? 0.0f : m;
#pragma unroll
    for (int i = 0; i < 8; ++i) z += __builtin_amdgcn_exp2f((v[i] - from) * by);
  }
  return joined({m, z, first, 0}, by);
}
__device__ inline bool has_distribution(const Part& p) { return p.z > 0.0f && p.m < INFINITY; }

struct Shared {
  ExpTable tab;
  double waves[8];
  int status[HIERAVG_DRAFTS_MAX];  // of each draft: 0 not accepted, 1 accepted, 2 not decided yet
  Part p[HIERAVG_DRAFTS_MAX + 1], q[HIERAVG_DRAFTS_MAX];  // the rows
};

// exp((x - m) / T) over a part of a row of T, summed over the workgroup: a
// thread's classes in their order, then a tree that does not change.
template <class T, class F>
__device__ inline double sum_over(Shared& sh, const T* x, int c0, int c1, F&& f) {
  constexpr int V = 16 / sizeof(T);
  double s = 0.0;
  for (int base = c0; base < c1; base += 256 * V) {
    const int j = base + (int)threadIdx.x * V;
    if (j + V <= c1) {
      const Pack<T, V> p = load_pack<T, V>(x + j);
#pragma unroll
      for (int e = 0; e < V; ++e) s += f((double)to_f32(p.v[e]), j + e);
    } else {
#pragma unroll
      for (int e = 0; e < V; ++e)
        if (j + e < c1) s += f((double)to_f32(x[j + e]), j + e);
    }
  }
  s = add_over_wave(s);
  __syncthreads();  // the last sum has been read
  if ((threadIdx.x & 63) == 0) sh.waves[threadIdx.x >> 6] = s;
  __syncthreads();
  return (sh.waves[0] + sh.waves[1]) + (sh.waves[2] + sh.waves[3]);
}

// The deciding row of a sequence from the float32 sums, by a workgroup.  `first`:
// the one that writes the results.  FEW: the sums are taken here.
template <class T, class Q, bool FEW = false>
__device__ inline Decision decide(const VerifyArgs& a, Shared& sh, int64_t b, bool first) {
  const int tid = threadIdx.x, wave = tid >> 6, n = drafts_of(a, b), G = a.drafts;
  const double it = inverse_temperature(a, b);
  const bool greedy = it == 0.0;
  const float by = exponent_of(it);
  const T* x = (const T*)a.x + b * (G + 1) * a.stride;
  const Q* q = (const Q*)a.q + b * G * a.q_stride;
  // The rows' sums and the drafts' comparisons, a wave each.
  const bool with_q = a.q && !greedy;
  for (int i = wave; i <= n; i += 4) {
    const bool draft = i < n;
    Part wp{-INFINITY, 0.0f, 0x7FFFFFFF, 0}, wq = wp;
    if (!FEW) {
      wp = part_of_lane(a.px + (b * (G + 1) + i) * a.parts, a.parts);
      if (with_q && draft) wq = part_of_lane(a.pq + (b * G + i) * a.parts, a.parts);
    }
    const int64_t t = draft ? draft_of(a, b, i) : -1;
    const bool inside = t >= 0 && t < a.classes;
    const double u = (double)a.uniforms[b * (G + 1) + i];
    const float xt = to_f32(x[i * a.stride + (inside ? t : 0)]), qt = with_q && draft ? to_f32(q[i * a.q_stride + (inside ? t : 0)]) : 0.0f;
    Part p, d = wq;
    if (FEW) {
      p = row_of_wave(x + i * a.stride, a.classes, by);
      if (with_q && draft) d = row_of_wave(q + i * a.q_stride, a.classes, by);
    } else {
      p = joined(wp, by);
      d = joined(wq, by);
    }
    int status = 0;
    if (inside && has_distribution(p)) {
      if (greedy) {
        status = t == p.first;
      } else {
        double lhs = u * (double)p.z, rhs = exp_of(sh.tab, ((double)xt - p.m) * it);
        if (with_q) {
          lhs *= exp_of(sh.tab, ((double)qt - d.m) * it);
          rhs *= (double)d.z;
        }
        if (!with_q || has_distribution(d)) status = !in_float32(it) || fabs(lhs - rhs) <= (double)a.unsure * rhs ? 2 : lhs < rhs;
      }
    }
    if ((tid & 63) == 0) {
      sh.p[i] = p;
      if (draft) {
        sh.q[i] = d;
        sh.status[i] = status;
        if (first && inside)  // stays if it is accepted
          a.logp[b * (G + 1) + i] = greedy ? 0.0f : (float)(((double)xt - p.m) * it - log((double)p.z));
      }
    }
  }
  __syncthreads();
  int row = 0;
  for (; row < n; ++row) {
    int s = sh.status[row];
    if (s == 2) {  // the same in all workgroups of the sequence
      const int64_t t = draft_of(a, b, row);
      const Part p = sh.p[row];
      const T* xr = x + row * a.stride;
      auto ex = [&](double v, float m) { return exp_of(sh.tab, (v - m) * it); };
      const double z = sum_over(sh, xr, 0, a.classes, [&](double v, int) { return ex(v, p.m); });
      double lhs = (double)a.uniforms[b * (G + 1) + row] * z, rhs = ex(to_f32(xr[t]), p.m);
      if (first && tid == 0) a.logp[b * (G + 1) + row] = (float)(((double)to_f32(xr[t]) - p.m) * it - log(z));
      if (a.q) {
        const Part d = sh.q[row];
        const Q* qr = q + row * a.q_stride;
        lhs *= ex(to_f32(qr[t]), d.m);
        rhs *= sum_over(sh, qr, 0, a.classes, [&](double v, int) { return ex(v, d.m); });
      }
      s = lhs < rhs;
    }
    if (s == 0) break;
  }
  // The row that the token is drawn from.
  const Part p = sh.p[row];
  const bool refused = row < n;
  Decision d{row, kTarget, -1, p.m, 0.0f, -1, {0, 0}};
  if (!has_distribution(p)) {
    d.kind = kNothing;
  } else if (greedy) {
    d.kind = kGreedy;
    d.token = p.first;
  } else if (refused && a.q) {
    const Part pq = sh.q[row];
    d.kind = has_distribution(pq) ? kDifference : kNothing;
    d.mq = pq.m;
  } else if (refused) {
    const int64_t t = draft_of(a, b, row);
    if (t >= 0 && t < a.classes) d.removed = (int)t;
  }
  if (first) {
    if (tid == 0) a.decisions[b] = d;
    for (int i = tid; i <= G; i += 256)
      if (i != row || d.kind == kNothing) {
        a.tokens[b * (G + 1) + i] = i < row ? (int)draft_of(a, b, i) : -1;
        if (i >= row) a.logp[b * (G + 1) + i] = 0.0f;
      }
    if (tid == 0) a.accepted[b] = row;
  }
  return d;
}

// A workgroup per sequence.
template <class T, class Q>
__global__ __launch_bounds__(256) void k_verify_decide(VerifyArgs a) {
  __shared__ Shared sh;
  fill(sh.tab);
  __syncthreads();
  decide<T, Q>(a, sh, blockIdx.x, true);
}

template <class T, class Q>
__device__ inline double2 fine_sums(const VerifyArgs& a, Shared& sh, const T* x, const Q* q, const Decision& d, double it, int part) {
  const int c0 = part * a.fine_part, c1 = min(c0 + a.fine_part, a.classes);
  double2 s;
  s.x = sum_over(sh, x, c0, c1, [&](double v, int) { return exp_of(sh.tab, (v - d.m) * it); });
  s.y = d.kind == kDifference ? sum_over(sh, q, c0, c1, [&](double v, int) { return exp_of(sh.tab, (v - d.mq) * it); }) : 0.0;
  return s;
}
// max(p - q, 0) of a class from the exponentials, each product rounded by itself:
// equal ones give 0, and every kernel the same bits.
__device__ inline double over_draft(double p, double ip, double q, double iq) {
#pragma clang fp contract(off)
  const double a = p * ip, b = q * iq;
  return fmax(a - b, 0.0);
}
// The sum of that over a part.
template <class T, class Q>
__device__ inline double rest_sum(const VerifyArgs& a, Shared& sh, const T* x, const Q* q, const Decision& d, const double2& z,
                                  double it, int part) {
  const int c0 = part * a.fine_part, c1 = min(c0 + a.fine_part, a.classes);
  const double ix = 1.0 / z.x, iq = 1.0 / z.y;
  return sum_over(sh, x, c0, c1, [&](double v, int j) {
    return over_draft(exp_of(sh.tab, (v - d.m) * it), ix, exp_of(sh.tab, ((double)to_f32(q[j]) - d.mq) * it), iq);
  });
}

// The sums in 64 bits of a part of the deciding row.  HERE: every workgroup finds
// that row by itself, which costs each of them what a launch costs all (64
// sequences, 4096 workgroups: 33 us; a launch for it and then the sums 6.2 + 16.5).
// 17 M exponentials in 16 us, of which about 7 are their 64-bit operations at full
// rate; the waves wait 40 % of their time, for a chain of few loads, table look-ups and sums.
template <class T, class Q, bool HERE>
__global__ __launch_bounds__(256) void k_verify_fine(VerifyArgs a) {
  __shared__ Shared sh;
  const int64_t b = blockIdx.x / a.fine;
  const int part = (int)(blockIdx.x - b * a.fine);
  fill(sh.tab);
  __syncthreads();
  const Decision d = HERE ? decide<T, Q>(a, sh, b, part == 0) : a.decisions[b];
  if (d.kind != kTarget && d.kind != kDifference) return;
  const double it = inverse_temperature(a, b);
  const T* x = (const T*)a.x + (b * (a.drafts + 1) + d.row) * a.stride;
  const Q* q = (const Q*)a.q + (b * a.drafts + d.row) * a.q_stride;
  const double2 s = fine_sums(a, sh, x, q, d, it, part);
  if (threadIdx.x == 0) a.sums[blockIdx.x] = s;
}

// The sums of all parts, in all lanes.
__device__ inline double2 joined_sums(const double2* s, int parts) {
  const int lane = threadIdx.x & 63;
  const double2 v = lane < parts ? s[lane] : double2{0.0, 0.0};
  return {add_over_wave(v.x), add_over_wave(v.y)};
}

// Where the token is drawn from max(p - q, 0): its sum over each part (64
// sequences over 131072 classes: 14 us).
template <class T, class Q>
__global__ __launch_bounds__(256) void k_verify_rest(VerifyArgs a) {
  __shared__ Shared sh;
  const int64_t b = blockIdx.x / a.fine;
  const int part = (int)(blockIdx.x - b * a.fine);
  const Decision d = a.decisions[b];
  if (d.kind != kDifference) return;
  fill(sh.tab);
  __syncthreads();
  const double it = inverse_temperature(a, b);
  const double2 z = joined_sums(a.sums + b * a.fine, a.fine);
  const T* x = (const T*)a.x + (b * (a.drafts + 1) + d.row) * a.stride;
  const Q* q = (const Q*)a.q + (b * a.drafts + d.row) * a.q_stride;
  const double s = rest_sum(a, sh, x, q, d, z, it, part);
  if (threadIdx.x == 0) a.rest[blockIdx.x] = s;
}

// The token: the part that the uniform number falls into, then the thread, then
// the class.  A chain of a few loads and sums over lanes: 6.6 us for one sequence,
// 8.6 for 64.
// At temperature 0.
__device__ inline void put_largest(const VerifyArgs& a, int64_t b, const Decision& d) {
  if (threadIdx.x > 0) return;
  a.tokens[b * (a.drafts + 1) + d.row] = d.token;
  a.logp[b * (a.drafts + 1) + d.row] = 0.0f;
}
// mine_p, mine_rest: the sums of the lane's part.
template <class T, class Q>
__device__ inline void draw(const VerifyArgs& a, Shared& sh, int64_t b, const Decision& d, double it, const double2& z, double mine_p,
                            double mine_rest) {
  __shared__ int found;
  const int tid = threadIdx.x, lane = tid & 63;
  const int64_t at = b * (a.drafts + 1) + d.row;
  const double u = (double)a.uniforms[b * (a.drafts + 1) + a.drafts];
  const T* x = (const T*)a.x + at * a.stride;
  const Q* q = (const Q*)a.q + (b * a.drafts + d.row) * a.q_stride;
  if (tid == 0) found = 0x7FFFFFFF;
  double mine = mine_rest;
  const bool difference = d.kind == kDifference && add_over_wave(mine) > 0.0;  // p = q: from p
  // p alone is drawn from as its exponentials: with a factor, ones that lie
  // at the end of the range would sum to more than they are worth one by one
  const double ix = 1.0 / z.x, iq = 1.0 / z.y;
  __syncthreads();
  // without the removed class, unless nothing else is left
  int removed = difference ? -1 : d.removed;
  // eight classes' weights from j on, 0 from `end` on: the loads go out together
  auto weights = [&](int j, int end, double (&w)[8]) {
    float v[8], o[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      v[e] = to_f32(x[min(j + e, a.classes - 1)]);
      if (difference) o[e] = to_f32(q[min(j + e, a.classes - 1)]);
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      w[e] = exp_of(sh.tab, ((double)v[e] - d.m) * it);
      if (difference) w[e] = over_draft(w[e], ix, exp_of(sh.tab, ((double)o[e] - d.mq) * it), iq);
      if (j + e >= end || j + e == removed) w[e] = 0.0;
    }
  };
  if (!difference) {
    mine = mine_p;
    if (removed >= 0) {
      // that part's sum again, without it
      const int part = removed / a.fine_part, c0 = part * a.fine_part, c1 = min(c0 + a.fine_part, a.classes);
      const double s = sum_over(sh, x, c0, c1, [&](double v, int j) {
        return j == removed ? 0.0 : exp_of(sh.tab, (v - d.m) * it);
      });
      const double kept = mine;
      if (lane == part) mine = s;
      if (!(add_over_wave(mine) > 0.0)) {
        removed = -1;
        mine = kept;
      }
    }
  }
  // The first part whose running sum passes u times the whole: sums in the
  // parts' order.
  double run = mine;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const double up = __shfl_up(run, o, 64);
    if (lane >= o) run += up;
  }
  const double target = u * __shfl(run, 63, 64);
  const uint64_t over = __ballot(run > target && mine > 0.0), some = __ballot(mine > 0.0);
  const int part = over ? __ffsll((unsigned long long)over) - 1 : 63 - __clzll((long long)some);
  const double left = target - (__shfl(run, part, 64) - __shfl(mine, part, 64));
  const int c0 = part * a.fine_part, c1 = min(c0 + a.fine_part, a.classes), each = (c1 - c0 + 255) / 256;
  const int j0 = c0 + tid * each, j1 = min(j0 + each, c1);
  double s = 0.0, w[8];
  int some_class = -1;  // the thread's last with a weight
  for (int j = j0; j < j1; j += 8) {
    weights(j, j1, w);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      s += w[e];
      if (w[e] > 0.0) some_class = j + e;
    }
  }
  // the sums of the threads before
  double up_to = s;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const double up = __shfl_up(up_to, o, 64);
    if (lane >= o) up_to += up;
  }
  __syncthreads();
  if (lane == 63) sh.waves[tid >> 6] = up_to;
  __syncthreads();
  double r = up_to - s;
  for (int i = 0; i < tid >> 6; ++i) r += sh.waves[i];
  if (s > 0.0 && r + s > left) {
    int at_class = 0x7FFFFFFF;
    for (int j = j0; j < j1 && at_class == 0x7FFFFFFF; j += 8) {
      if (each > 8) weights(j, j1, w);  // else as they are
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        r += w[e];
        if (w[e] > 0.0 && r > left) at_class = min(at_class, j + e);
      }
    }
    if (at_class != 0x7FFFFFFF) atomicMin(&found, at_class);
  }
  __syncthreads();
  int token = found;
  if (token == 0x7FFFFFFF) {  // roundings: the part's last class with a weight
    __syncthreads();
    if (tid == 0) found = -1;
    __syncthreads();
    if (some_class >= 0) atomicMax(&found, some_class);
    __syncthreads();
    token = found;
  }
  if (tid == 0) {
    a.tokens[at] = token;
    a.logp[at] = (float)(((double)to_f32(x[token]) - d.m) * it - log(z.x));
  }
}

template <class T, class Q>
__global__ __launch_bounds__(256) void k_verify_draw(VerifyArgs a) {
  __shared__ Shared sh;
  const int64_t b = blockIdx.x;
  const int lane = threadIdx.x & 63;
  const Decision d = a.decisions[b];
  if (d.kind == kNothing) return;
  if (d.kind == kGreedy) return put_largest(a, b, d);
  fill(sh.tab);
  const double2 s = lane < a.fine ? a.sums[b * a.fine + lane] : double2{0.0, 0.0};
  const double rest = d.kind == kDifference && lane < a.fine ? a.rest[b * a.fine + lane] : 0.0;
  draw<T, Q>(a, sh, b, d, inverse_temperature(a, b), {add_over_wave(s.x), add_over_wave(s.y)}, s.x, rest);
}

// Few classes (one part of either kind: up to 2048): all of it by one workgroup for
// each sequence, its four waves one row after the other in steps of 512 classes.  Calls
// in us, of 1 and 64 sequences, beside those of several launches with a workgroup a row:
//   classes   4 drafts             8                    16                   32                   64
//       256   13, 16 (21, 24)      17, 18 (23, 27)      22, 23 (27, 31)      31, 32 (33, 41)      50, 50 (51, 60)
//      1024   15, 16 (20, 23)      18, 19 (22, 26)      24, 26 (26, 30)      36, 38 (32, 40)      61, 72 (47, 62)
//      2048   14, 19 (21, 24)      23, 24 (23, 26)      32, 34 (26, 31)      51, 54 (33, 41)      88, 109 (50, 62)
// So: one step a row, or up to 20 steps a wave.
inline bool in_one_launch(int64_t rows, int64_t classes) {
  const int64_t steps = (classes + 511) / 512;
  return steps == 1 || (rows + 3) / 4 * steps <= 20;
}
template <class T, class Q>
__global__ __launch_bounds__(256) void k_verify_few(VerifyArgs a) {
  __shared__ Shared sh;
  const int64_t b = blockIdx.x;
  const int lane = threadIdx.x & 63;
  fill(sh.tab);
  __syncthreads();
  const Decision d = decide<T, Q, true>(a, sh, b, true);
  if (d.kind == kNothing) return;
  if (d.kind == kGreedy) return put_largest(a, b, d);
  const double it = inverse_temperature(a, b);
  const T* x = (const T*)a.x + (b * (a.drafts + 1) + d.row) * a.stride;
  const Q* q = (const Q*)a.q + (b * a.drafts + d.row) * a.q_stride;
  const double2 z = fine_sums(a, sh, x, q, d, it, 0);
  const double rest = d.kind == kDifference ? rest_sum(a, sh, x, q, d, z, it, 0) : 0.0;
  draw<T, Q>(a, sh, b, d, it, z, lane == 0 ? z.x : 0.0, lane == 0 ? rest : 0.0);
}

struct VerifyPlan {
  int parts, part, fine, fine_part;
  size_t px, pq, sums, rest, decisions, bytes;  // offsets
};

VerifyPlan plan_verify(int64_t seqs, int64_t drafts, int64_t classes, bool q) {
  VerifyPlan p;
  const int64_t rows = seqs * (q ? 2 * drafts + 1 : drafts + 1);
  const int64_t most = std::min<int64_t>((classes + 2047) / 2048, kMostParts);
  const int64_t parts = std::max<int64_t>(1, std::min(most, (2048 + rows - 1) / rows));
  p.part = (int)round_up((classes + parts - 1) / parts, 64);
  p.parts = (int)((classes + p.part - 1) / p.part);
  p.fine_part = (int)round_up((classes + most - 1) / most, 64);
  p.fine = (int)((classes + p.fine_part - 1) / p.fine_part);
  size_t at = 0;
  auto take = [&](size_t n) {
    const size_t o = at;
    at += (size_t)round_up((int64_t)n, 16);
    return o;
  };
  p.px = take((size_t)seqs * (drafts + 1) * p.parts * sizeof(Part));
  p.pq = take(q ? (size_t)seqs * drafts * p.parts * sizeof(Part) : 0);
  p.sums = take((size_t)seqs * p.fine * sizeof(double2));
  p.rest = take(q ? (size_t)seqs * p.fine * sizeof(double) : 0);
  p.decisions = take((size_t)seqs * sizeof(Decision));
  p.bytes = at;
  return p;
}

// Sequences of one set of launches: the largest grid has kMostParts workgroups for each of their rows.
constexpr int64_t kMostSeqs = kMaxGroups / kMostParts / (2 * HIERAVG_DRAFTS_MAX + 1);

bool verifiable(int64_t seqs, int64_t drafts, int64_t classes) {
  return seqs >= 0 && seqs <= 1 << 24 && drafts >= 0 && drafts <= HIERAVG_DRAFTS_MAX && classes >= 1 && classes <= kMostClasses;
}

// Workgroups up to which each decides by itself: one a CU.
constexpr unsigned kDecideHere = 256;

template <class T, class Q>
void launch_verify(hipStream_t s, const VerifyArgs& a) {
  const int64_t of_one = a.q ? 2 * a.drafts + 1 : a.drafts + 1, rows = a.seqs * of_one;
  const unsigned fine = (unsigned)(a.seqs * a.fine);
  if (a.fine == 1 && a.parts == 1 && in_one_launch(of_one, a.classes))
    return launch(k_verify_few<T, Q>, (unsigned)a.seqs, 256, 0, s, a);
  launch(k_verify_sums<T, Q>, (unsigned)(rows * a.parts), 256, 0, s, a);
  if (fine <= kDecideHere) {
    launch(k_verify_fine<T, Q, true>, fine, 256, 0, s, a);
  } else {
    launch(k_verify_decide<T, Q>, (unsigned)a.seqs, 256, 0, s, a);
    launch(k_verify_fine<T, Q, false>, fine, 256, 0, s, a);
  }
  if (a.q && a.drafts > 0) launch(k_verify_rest<T, Q>, fine, 256, 0, s, a);
  launch(k_verify_draw<T, Q>, (unsigned)a.seqs, 256, 0, s, a);
}

template <class T>
void launch_verify(hipStream_t s, const VerifyArgs& a, int32_t q_type) {
  if (!a.q || q_type == HIERAVG_F32)
    launch_verify<T, float>(s, a);
  else if (q_type == HIERAVG_F16)
    launch_verify<T, f16_t>(s, a);
  else
    launch_verify<T, bf16_t>(s, a);
}

}  // namespace

}  // namespace hav

using namespace hav;

extern "C" {

size_t hieravg_verify_drafts_scratch(int64_t seqs, int32_t drafts, int64_t classes, int32_t draft_logits) {
  if (!verifiable(seqs, drafts, classes) || seqs == 0) return 0;
  return plan_verify(std::min(seqs, kMostSeqs), drafts, classes, draft_logits != 0).bytes;
}

int hieravg_verify_drafts(const void* logits, int32_t type, int64_t seqs, int32_t drafts, int64_t classes,
                          int64_t row_stride, const void* draft_logits, int32_t draft_type, int64_t draft_stride,
                          const void* draft_tokens, int32_t token_bytes, const float* uniforms, const int32_t* lengths,
                          const float* temperature, int32_t* tokens, int32_t* accepted, float* logp, void* scratch,
                          size_t scratch_bytes, void* hip_stream) {
  return guarded([&]() -> int {
    if (!known_type(type) || (draft_logits && !known_type(draft_type))) return invalid("unknown element type");
    if (!verifiable(seqs, drafts, classes))
      return invalid("seqs must be in [0, 2^24], drafts in [0, HIERAVG_DRAFTS_MAX], classes in [1, 2^23]");
    if (row_stride < classes || !addressable(seqs * (drafts + 1), row_stride, type_bytes(type)))
      return invalid("row_stride must be at least classes, the rows within 2^56 bytes");
    if (draft_logits && (draft_stride < classes || !addressable(seqs * drafts, draft_stride, type_bytes(draft_type))))
      return invalid("draft_stride must be at least classes, the rows within 2^56 bytes");
    if (token_bytes != 4 && token_bytes != 8) return invalid("token_bytes must be 4 or 8");
    if (seqs == 0) return HIERAVG_OK;
    if (!logits || !aligned(logits, type_bytes(type)) || (draft_logits && !aligned(draft_logits, type_bytes(draft_type))))
      return invalid("logits must be pointers aligned to their element");
    if (drafts > 0 && (!draft_tokens || !aligned(draft_tokens, token_bytes)))
      return invalid("draft_tokens must be a pointer aligned to its element");
    if (!uniforms || !tokens || !accepted || !logp) return invalid("uniforms, tokens, accepted or logp is NULL");
    for (const void* p : {(const void*)uniforms, (const void*)lengths, (const void*)temperature, (const void*)tokens,
                          (const void*)accepted, (const void*)logp})
      if (!aligned(p, 4)) return invalid("uniforms, lengths, temperature, tokens, accepted and logp must be aligned to their element");
    const VerifyPlan p = plan_verify(std::min(seqs, kMostSeqs), drafts, classes, draft_logits != nullptr);
    if (!scratch || scratch_bytes < p.bytes || !aligned(scratch, 16))
      return invalid("scratch must hold hieravg_verify_drafts_scratch bytes, 16-byte aligned");
    // workgroups that still decide read what the first of them writes over
    const Area xa = rows_area(logits, seqs * (drafts + 1), row_stride, classes, type), qa = rows_area(draft_logits, seqs * drafts, draft_stride, classes, draft_type),
               da = block_area(draft_tokens, seqs * drafts * token_bytes), ua = block_area(uniforms, seqs * (drafts + 1) * 4),
               la = block_area(lengths, seqs * 4), ta = block_area(temperature, seqs * 4), tokens_a = block_area(tokens, ua.len),
               accepted_a = block_area(accepted, seqs * 4), logp_a = block_area(logp, ua.len);
    if (meet_any(tokens_a, xa, qa, da, ua, la, ta, accepted_a, logp_a) || meet_any(accepted_a, xa, qa, da, ua, la, ta, logp_a) ||
        meet_any(logp_a, xa, qa, da, ua, la, ta))
      return invalid("tokens, accepted and logp must overlap neither an operand nor each other");
    char* w = (char*)scratch;
    for (int64_t s0 = 0; s0 < seqs; s0 += kMostSeqs) {
      const int64_t row = s0 * (drafts + 1), draft = s0 * drafts;
      VerifyArgs a{};
      a.x = (const char*)logits + row * row_stride * type_bytes(type);
      if (draft_logits && drafts > 0) a.q = (const char*)draft_logits + draft * draft_stride * type_bytes(draft_type);
      a.stride = row_stride;
      a.q_stride = draft_stride;
      a.seqs = std::min(seqs - s0, kMostSeqs);
      a.drafts = drafts;
      a.classes = (int)classes;
      a.tokens_in = drafts > 0 ? (const char*)draft_tokens + draft * token_bytes : nullptr;
      a.token_bytes = token_bytes;
      a.uniforms = uniforms + row;
      a.temperature = temperature ? temperature + s0 : nullptr;
      a.lengths = lengths ? lengths + s0 : nullptr;
      a.tokens = tokens + row;
      a.accepted = accepted + s0;
      a.logp = logp + row;
      a.parts = p.parts;
      a.part = p.part;
      a.fine = p.fine;
      a.fine_part = p.fine_part;
      a.px = (Part*)(w + p.px);
      a.pq = (Part*)(w + p.pq);
      a.sums = (double2*)(w + p.sums);
      a.rest = (double*)(w + p.rest);
      a.decisions = (Decision*)(w + p.decisions);
      // Each side's sum is off by at most (part / 256 + 110) 2^-24 of it: a thread's
      // additions one after the other, a tree's, and the exponentials' own errors,
      // (5 |t| + 3) 2^-24 with |t| <= log classes on average over a distribution.
      a.unsure = 2.5f * ((float)p.part / 256.0f + 110.0f) * 0x1p-24f;
      hipStream_t s = (hipStream_t)hip_stream;
      if (type == HIERAVG_F32)
        launch_verify<float>(s, a, draft_type);
      else if (type == HIERAVG_F16)
        launch_verify<f16_t>(s, a, draft_type);
      else
        launch_verify<bf16_t>(s, a, draft_type);
    }
    return launched("hieravg_verify_drafts");
  });
}

}  // extern "C"
