// Log probabilities of given labels with entropy and top alternatives, and
// their gradient (include/hieravg.h, hieravg_log_probs).
#include <algorithm>
#include <cmath>

#include "ops.h"

namespace hav {

namespace {

struct LogProbArgs {
  const void* x;
  int64_t rows, stride;
  int classes, top;
  const void* labels;
  int label_bytes;
  float *logp, *entropy, *lse, *top_logp;
  int32_t* top_ids;
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

// The partial sums of a part of a row: greatest value m, sum of exp(x - m) and
// of exp(x - m) (x - m).
struct Sums {
  float m, z, s;
};
// The same sums from the greatest value m >= a.m.  exp(d) d is 0 where exp(d)
// is: d may be infinite, or overflow with z.
__device__ inline Sums from_max(const Sums& a, float m) {
  if (a.m == -INFINITY) return {m, a.z, 0.0f};  // nothing, or NaN
  const float d = a.m - m, e = expf(d), ed = e == 0.0f ? 0.0f : e * d;
  return {m, e * a.z, e * a.s + ed * a.z};
}
__device__ inline Sums joined(const Sums& a, const Sums& b) {
  const float m = fmaxf(a.m, b.m);
  const Sums x = from_max(a, m), y = from_max(b, m);
  return {m, x.z + y.z, x.s + y.s};
}

template <class T>
__global__ __launch_bounds__(256) void k_log_probs(LogProbArgs a) {
  __shared__ Sums part[256];
  __shared__ uint64_t keys[256];
  const int64_t r = blockIdx.x;
  const T* x = (const T*)a.x + r * a.stride;
  const int tid = threadIdx.x;
  Sums t = {-INFINITY, 0.0f, 0.0f};
  for (int j = tid; j < a.classes; j += 256) {
    const float v = to_f32(x[j]);
    if (v > t.m) t = from_max(t, v);
    const float d = v - t.m;
    if (!(v == -INFINITY)) {
      const float e = expf(d);
      t.z += e;
      t.s += e > 0.0f ? e * d : e;  // e NaN: NaN
    }
  }
  part[tid] = t;
  __syncthreads();
  if (tid == 0) {
    for (int i = 1; i < 256; ++i) t = joined(t, part[i]);
    const bool none = !(t.z > 0.0f) || t.m == INFINITY;
    const float logz = none ? NAN : logf(t.z), lse = t.m + logz;
    part[0] = {t.m, logz, 0.0f};
    if (a.lse) a.lse[r] = lse;
    if (a.entropy) a.entropy[r] = logz - t.s / t.z;
    if (a.logp) {
      const int64_t y = label_of(a.labels, a.label_bytes, r);
      a.logp[r] = y < 0 ? 0.0f : y >= a.classes ? NAN : to_f32(x[y]) - t.m - logz;
    }
  }
  __syncthreads();
  const float most = part[0].m, logz = part[0].z;
  uint64_t last = ~0ull;
  for (int k = 0; k < a.top; ++k) {
    uint64_t best = 0;
    for (int j = tid; j < a.classes; j += 256) {
      const uint64_t key = key_of(to_f32(x[j]), (uint32_t)j);
      if (key < last && key > best) best = key;
    }
    keys[tid] = best;
    __syncthreads();
    for (int o = 128; o > 0; o >>= 1) {
      if (tid < o) keys[tid] = max(keys[tid], keys[tid + o]);
      __syncthreads();
    }
    last = keys[0];
    __syncthreads();
    if (tid == 0) {
      const int j = (int)(0xFFFFFFFFu - (uint32_t)last);
      a.top_ids[r * a.top + k] = j;
      a.top_logp[r * a.top + k] = to_f32(x[j]) - most - logz;
    }
  }
}

struct GradArgs {
  const void* x;
  void* grad;
  int64_t rows, stride, grad_stride;
  int classes;
  const void* labels;
  int label_bytes;
  const float *lse, *entropy, *g_logp, *g_entropy;
};

template <class T>
__global__ __launch_bounds__(256) void k_log_probs_grad(GradArgs a) {
  const int64_t r = blockIdx.y;
  const int64_t y = a.g_logp ? label_of(a.labels, a.label_bytes, r) : -1;
  float g = a.g_logp && y >= 0 ? a.g_logp[r] : 0.0f;
  const float h = a.g_entropy ? a.g_entropy[r] : 0.0f;
  if (y >= a.classes) g = NAN;
  const bool zero = g == 0.0f && h == 0.0f;
  const float lse = a.lse[r], ent = a.g_entropy ? a.entropy[r] : 0.0f;
  const T* x = (const T*)a.x + r * a.stride;
  T* o = (T*)a.grad + r * a.grad_stride;
  for (int j = blockIdx.x * 256 + threadIdx.x; j < a.classes; j += gridDim.x * 256) {
    float d = 0.0f;
    if (!zero) {
      const float l = to_f32(x[j]) - lse, p = expf(l);
      d = -g * p + (j == y ? g : 0.0f) - h * (p == 0.0f ? 0.0f : p * (l + ent));
    }
    from_f32(d, &o[j]);
  }
}

int check_logits(const void* logits, int32_t type, int64_t rows, int64_t classes, int64_t stride) {
  if (!known_type(type)) return invalid("unknown element type");
  if (rows < 0 || rows > 0x7FFFFFFF) return invalid("rows must be in [0, 2^31)");
  if (classes < 1 || classes >= 0x7FFFFFFF) return invalid("classes must be in [1, 2^31)");
  if (stride < classes) return invalid("row_stride must be at least classes");
  if (rows > 0 && (!logits || !aligned(logits, type_bytes(type))))
    return invalid("logits must be a pointer aligned to its element");
  return HIERAVG_OK;
}

int check_labels(const void* labels, int32_t label_bytes) {
  if (label_bytes != 4 && label_bytes != 8) return invalid("label_bytes must be 4 or 8");
  if (!labels || !aligned(labels, label_bytes)) return invalid("labels must be a pointer aligned to its element");
  return HIERAVG_OK;
}

}  // namespace

}  // namespace hav

using namespace hav;

extern "C" {

size_t hieravg_log_probs_scratch(int64_t rows, int64_t classes, int32_t top) {
  (void)rows;
  (void)classes;
  (void)top;
  return 0;
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
    LogProbArgs a{logits, rows, row_stride, (int)classes, top, labels, label_bytes, logp, entropy, lse, top_logp, top_ids};
    hipStream_t s = (hipStream_t)hip_stream;
    const unsigned grid = (unsigned)rows;
    if (type == HIERAVG_F32)
      launch(k_log_probs<float>, grid, 256, 0, s, a);
    else if (type == HIERAVG_F16)
      launch(k_log_probs<f16_t>, grid, 256, 0, s, a);
    else
      launch(k_log_probs<bf16_t>, grid, 256, 0, s, a);
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
    if (grad_stride < classes) return invalid("grad_stride must be at least classes");
    if (rows == 0) return HIERAVG_OK;
    if (!grad || !aligned(grad, type_bytes(type))) return invalid("grad must be a pointer aligned to its element");
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
      const dim3 grid((unsigned)std::min<int64_t>((classes + 1023) / 1024, 65535), (unsigned)std::min<int64_t>(rows - r0, 65535));
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

}  // extern "C"
