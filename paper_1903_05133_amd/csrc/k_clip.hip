// The norm of many gradients, of each and of all, and their clipping
// (include/hieravg.h, hieravg_grad_norm, hieravg_scale_tensors).  The tensors'
// addresses and sizes are kernel arguments, so that a graph holds them.
#include <algorithm>
#include <cmath>
#include <vector>

#include "ops.h"

namespace hav {

namespace {

constexpr int kPerLaunch = 128;      // tensors
// Elements that one workgroup takes: few, so that those that run at once read one
// stretch of memory (155 M bf16 elements: 74 us, 81 in chunks of 76 000; their
// scaling 94, 100).
constexpr int64_t kChunkLeast = 16384;
constexpr int64_t kChunksMost = 1 << 16;  // from then on chunks grow

struct NormArgs {
  double* parts;     // sum of squares of each chunk
  int32_t* starts;   // first chunk of each tensor
  int64_t chunk;     // elements of a chunk
  int chunk0, tensor0;  // first of this launch
  int count;
  uint32_t first[kPerLaunch];  // first chunk of each tensor, from chunk0
  const void* p[kPerLaunch];
  int64_t n[kPerLaunch];
  uint8_t type[kPerLaunch];
};
struct ScaleArgs {
  const float* factor;
  int64_t chunk;
  int count;
  uint32_t first[kPerLaunch];
  const void* in[kPerLaunch];
  void* out[kPerLaunch];
  int64_t n[kPerLaunch];
  uint8_t type[kPerLaunch];
};

// The tensor that chunk c of a launch belongs to: how many begin at or before
// it, less one; every lane has two of the 128.
__device__ inline int tensor_of(const uint32_t* first, int count, uint32_t c) {
  const int lane = threadIdx.x & 63;
  const bool a = lane < count && first[lane] <= c, b = lane + 64 < count && first[lane + 64] <= c;
  return __popcll(__ballot(a)) + __popcll(__ballot(b)) - 1;
}

// The sum is in 64 bits, where no square of a float32 overflows or vanishes.
// Conversions and additions in 64 bits take longer than the memory (155 M bf16
// elements 88 us, 3.5 TB/s), so in whole steps eight squares are added in float32
// first, in pairs: a product, a sum, two sums of sums, each rounded, so off by 4 2^-24
// of their sum at most (16-bit values, whose squares are exact, by 3), unless one of a
// wave's sixty-four eights has its largest value where squares are not normal numbers.
template <int V>
__device__ inline void add_squares(const float (&x)[V], double (&s)[4]) {
#pragma unroll
  for (int e = 0; e < V; ++e) s[e & 3] = fma((double)x[e], (double)x[e], s[e & 3]);
}
template <int V>
__device__ inline void add_squares_fast(const float (&x)[V], double (&s)[4]) {
  static_assert(V == 8, "pairs of pairs");
  float most = fabsf(x[0]), pair[4];
#pragma unroll
  for (int e = 1; e < V; ++e) most = fmaxf(most, fabsf(x[e]));
#pragma unroll
  for (int e = 0; e < V; e += 2) pair[e / 2] = fmaf(x[e + 1], x[e + 1], x[e] * x[e]);
  // NaN leaves no largest value, but a sum that is none
  const bool odd = !(most <= 0x1p60f) || (most < 0x1p-60f && most > 0.0f);
  if (__any(odd))
    add_squares(x, s);
  else
    s[0] += (double)((pair[0] + pair[1]) + (pair[2] + pair[3]));
}
template <class T>
__device__ inline double square_sum(const T* p, int64_t n) {
  constexpr int V = 16 / sizeof(T), U = 32 / V;  // elements of a load, loads under way
  double s[4] = {0.0, 0.0, 0.0, 0.0};
  int64_t i = 0;
  for (; i + 256 * V * U <= n; i += 256 * V * U) {
    Pack<T, V> v[U];
#pragma unroll
    for (int u = 0; u < U; ++u) v[u] = load_pack<T, V>(p + i + (u * 256 + threadIdx.x) * V);
#pragma unroll
    for (int u = 0; u < U; u += 8 / V) {
      float x[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) x[e] = to_f32(v[u + e / V].v[e % V]);
      add_squares_fast(x, s);
    }
  }
  for (; i < n; i += 256 * V) {
    const int64_t j = i + threadIdx.x * V;
    float x[V];
    if (j + V <= n) {
      const Pack<T, V> v = load_pack<T, V>(p + j);
#pragma unroll
      for (int e = 0; e < V; ++e) x[e] = to_f32(v.v[e]);
    } else {
#pragma unroll
      for (int e = 0; e < V; ++e) {
        x[e] = 0.0f;
        if (j + e < n) x[e] = to_f32(p[j + e]);
      }
    }
    add_squares(x, s);
  }
  return (s[0] + s[1]) + (s[2] + s[3]);
}

// 155 M bf16 elements: 74 us (4.2 TB/s), the waves waiting for memory 85 % of their time.
__global__ __launch_bounds__(256) void k_square_sums(NormArgs a) {
  __shared__ double waves[4];
  const uint32_t c = blockIdx.x;
  const int k = tensor_of(a.first, a.count, c);
  const int64_t at = (int64_t)(c - a.first[k]) * a.chunk, n = min(a.chunk, a.n[k] - at);
  double s;
  if (a.type[k] == HIERAVG_F32)
    s = square_sum((const float*)a.p[k] + at, n);
  else if (a.type[k] == HIERAVG_F16)
    s = square_sum((const f16_t*)a.p[k] + at, n);
  else
    s = square_sum((const bf16_t*)a.p[k] + at, n);
  s = add_over_wave(s);
  if ((threadIdx.x & 63) == 0) waves[threadIdx.x >> 6] = s;
  __syncthreads();
  if (threadIdx.x == 0) {
    a.parts[a.chunk0 + c] = (waves[0] + waves[1]) + (waves[2] + waves[3]);
    if (at == 0) a.starts[a.tensor0 + k] = a.chunk0 + (int)c;
  }
}

// The sums of chunks, of all by the first workgroup and of each tensor by one of
// the others, in an order that does not change.
__device__ inline double sum_parts(const double* parts, int from, int to, int step) {
  double s = 0.0;
  for (int i = from; i < to; i += 8 * step) {
    double v[8];
#pragma unroll
    for (int u = 0; u < 8; ++u) v[u] = parts[min(i + u * step, to - 1)];
#pragma unroll
    for (int u = 0; u < 8; ++u) s += i + u * step < to ? v[u] : 0.0;
  }
  return add_over_wave(s);
}

__global__ __launch_bounds__(1024) void k_join_norms(const double* parts, const int32_t* starts, int chunks, int count,
                                                     double max_norm, float* norms, float* norm, float* factor) {
  __shared__ double waves[16];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int k = (int)blockIdx.x - 1;
  const int from = k < 0 ? 0 : starts[k], to = k >= 0 && k + 1 < count ? starts[k + 1] : chunks;
  double s = sum_parts(parts, from + tid, to, 1024);
  if (lane == 0) waves[wave] = s;
  __syncthreads();
  s = add_over_wave(lane < 16 ? waves[lane] : 0.0);
  if (tid > 0) return;
  const double all = sqrt(s);
  if (k >= 0) {
    norms[k] = (float)all;
  } else {
    if (norm) *norm = (float)all;
    // NaN stays
    if (factor) *factor = all <= max_norm ? 1.0f : (float)(max_norm / all);
  }
}

template <class T>
__device__ inline void scale(const T* in, T* out, int64_t n, float f) {
  constexpr int V = 16 / sizeof(T), U = 4;
  int64_t i = 0;
  for (; i + 256 * V * U <= n; i += 256 * V * U) {
    Pack<T, V> v[U];
#pragma unroll
    for (int u = 0; u < U; ++u) v[u] = load_pack<T, V>(in + i + (u * 256 + threadIdx.x) * V);
#pragma unroll
    for (int u = 0; u < U; ++u) {
#pragma unroll
      for (int e = 0; e < V; ++e) from_f32(to_f32(v[u].v[e]) * f, &v[u].v[e]);
      store_pack(out + i + (u * 256 + threadIdx.x) * V, v[u]);
    }
  }
  for (; i < n; i += 256 * V) {
    const int64_t j = i + threadIdx.x * V;
    if (j + V <= n) {
      Pack<T, V> v = load_pack<T, V>(in + j);
#pragma unroll
      for (int e = 0; e < V; ++e) from_f32(to_f32(v.v[e]) * f, &v.v[e]);
      store_pack(out + j, v);
    } else {
      for (int e = 0; e < V; ++e)
        if (j + e < n) from_f32(to_f32(in[j + e]) * f, out + j + e);
    }
  }
}

// 155 M bf16 elements: 93 us (6.7 TB/s read and written).
__global__ __launch_bounds__(256) void k_scale(ScaleArgs a) {
  const float f = *a.factor;
  const uint32_t c = gridDim.x - 1 - blockIdx.x;  // what the norm read last is still in the caches
  const int k = tensor_of(a.first, a.count, c);
  if (f == 1.0f && a.in[k] == a.out[k]) return;
  const int64_t at = (int64_t)(c - a.first[k]) * a.chunk, n = min(a.chunk, a.n[k] - at);
  if (a.type[k] == HIERAVG_F32)
    scale((const float*)a.in[k] + at, (float*)a.out[k] + at, n, f);
  else if (a.type[k] == HIERAVG_F16)
    scale((const f16_t*)a.in[k] + at, (f16_t*)a.out[k] + at, n, f);
  else
    scale((const bf16_t*)a.in[k] + at, (bf16_t*)a.out[k] + at, n, f);
}

int check_tensors(const hieravg_tensor* t, int32_t count) {
  if (!t || count < 1 || count > 1 << 20) return invalid("no tensors, or more than 2^20");
  int64_t all = 0;
  for (int32_t k = 0; k < count; ++k) {
    if (t[k].n < 0 || t[k].n > (int64_t(1) << 40)) return invalid("a tensor's size is negative or beyond 2^40");
    if (!known_type(t[k].type)) return invalid("unknown element type");
    if (t[k].data && !aligned(t[k].data, type_bytes(t[k].type))) return invalid("a tensor must be aligned to its element");
    all += t[k].n;
  }
  if (all > int64_t(1) << 44) return invalid("more than 2^44 elements");
  return HIERAVG_OK;
}

int64_t elements(const hieravg_tensor& t) { return t.data ? t.n : 0; }

// Elements of a chunk: a multiple of the least, about kChunksMost chunks in all.
int64_t chunk_size(const hieravg_tensor* t, int32_t count) {
  int64_t all = 0;
  for (int32_t k = 0; k < count; ++k) all += elements(t[k]);
  return round_up(std::max<int64_t>(1, (all + kChunksMost - 1) / kChunksMost), kChunkLeast);
}
// Chunks of a tensor, one for an empty one.
int64_t chunks_of(const hieravg_tensor& t, int64_t chunk) { return std::max<int64_t>(1, (elements(t) + chunk - 1) / chunk); }

int64_t all_chunks(const hieravg_tensor* t, int32_t count) {
  const int64_t chunk = chunk_size(t, count);
  int64_t c = 0;
  for (int32_t k = 0; k < count; ++k) c += chunks_of(t[k], chunk);
  return c;
}

// Memory that is read, or written (a tensor scaled in place: only written).
struct Range {
  uintptr_t begin, end;
  bool written;
};
// Whether any range shares memory with a written one.
bool collide(std::vector<Range>& r) {
  std::sort(r.begin(), r.end(), [](const Range& a, const Range& b) { return a.begin < b.begin; });
  uintptr_t read_end = 0, written_end = 0;  // of those that begin before
  for (const Range& x : r) {
    if (x.begin < written_end || (x.written && x.begin < read_end)) return true;
    (x.written ? written_end : read_end) = std::max(x.written ? written_end : read_end, x.end);
  }
  return false;
}

}  // namespace

}  // namespace hav

using namespace hav;

extern "C" {

size_t hieravg_grad_norm_scratch(const hieravg_tensor* grads, int32_t count) {
  if (check_tensors(grads, count) != HIERAVG_OK) return 0;
  return (size_t)all_chunks(grads, count) * sizeof(double) + (size_t)count * sizeof(int32_t);
}

int hieravg_grad_norm(const hieravg_tensor* grads, int32_t count, double max_norm, float* norms, float* norm,
                      float* factor, void* scratch, size_t scratch_bytes, void* hip_stream) {
  return guarded([&]() -> int {
    const int rc = check_tensors(grads, count);
    if (rc != HIERAVG_OK) return rc;
    if (!(max_norm >= 0.0)) return invalid("max_norm must be >= 0 (infinite: no clipping)");
    if (!norms && !norm && !factor) return invalid("norms, norm and factor are all NULL");
    if (!aligned(norms, 4) || !aligned(norm, 4) || !aligned(factor, 4))
      return invalid("norms, norm and factor must be aligned to their element");
    const int64_t chunk = chunk_size(grads, count), chunks = all_chunks(grads, count);
    if (!scratch || scratch_bytes < (size_t)chunks * sizeof(double) + (size_t)count * sizeof(int32_t) || !aligned(scratch, 16))
      return invalid("scratch must hold hieravg_grad_norm_scratch bytes, 16-byte aligned");
    hipStream_t s = (hipStream_t)hip_stream;
    double* parts = (double*)scratch;
    int32_t* starts = (int32_t*)(parts + chunks);
    int64_t c = 0;
    for (int32_t k0 = 0; k0 < count; k0 += kPerLaunch) {
      NormArgs a{};
      a.parts = parts;
      a.starts = starts;
      a.chunk = chunk;
      a.chunk0 = (int)c;
      a.tensor0 = k0;
      a.count = std::min(count - k0, kPerLaunch);
      uint32_t in = 0;
      for (int i = 0; i < a.count; ++i) {
        const hieravg_tensor& t = grads[k0 + i];
        a.first[i] = in;
        a.p[i] = t.data;
        a.n[i] = elements(t);
        a.type[i] = (uint8_t)t.type;
        in += (uint32_t)chunks_of(t, chunk);
      }
      launch(k_square_sums, in, 256, 0, s, a);
      c += in;
    }
    launch(k_join_norms, norms ? 1 + count : 1, 1024, 0, s, parts, starts, (int)chunks, (int)count, max_norm, norms, norm, factor);
    return launched("hieravg_grad_norm");
  });
}

int hieravg_scale_tensors(const hieravg_tensor* in, void* const* out, int32_t count, const float* factor,
                          void* hip_stream) {
  return guarded([&]() -> int {
    const int rc = check_tensors(in, count);
    if (rc != HIERAVG_OK) return rc;
    if (!out || !factor || !aligned(factor, 4)) return invalid("out or factor is NULL or not aligned");
    std::vector<Range> ranges;
    for (int32_t k = 0; k < count; ++k) {
      if (!elements(in[k])) continue;
      if (!out[k] || !aligned(out[k], type_bytes(in[k].type))) return invalid("a result must be a pointer aligned to its element");
      const uintptr_t x = (uintptr_t)in[k].data, y = (uintptr_t)out[k], n = (uintptr_t)in[k].n * type_bytes(in[k].type);
      if (x != y) ranges.push_back({x, x + n, false});
      ranges.push_back({y, y + n, true});
    }
    if (ranges.empty()) return HIERAVG_OK;
    ranges.push_back({(uintptr_t)factor, (uintptr_t)factor + 4, false});
    if (collide(ranges)) return invalid("a result must be its own tensor or overlap no tensor, no other result and not the factor");
    const int64_t chunk = chunk_size(in, count);
    for (int32_t k0 = 0; k0 < count; k0 += kPerLaunch) {
      ScaleArgs a{};
      a.factor = factor;
      a.chunk = chunk;
      uint32_t c = 0;
      for (int32_t k = k0; k < std::min(count, k0 + kPerLaunch); ++k) {
        if (!elements(in[k])) continue;
        a.first[a.count] = c;
        a.in[a.count] = in[k].data;
        a.out[a.count] = out[k];
        a.n[a.count] = in[k].n;
        a.type[a.count] = (uint8_t)in[k].type;
        ++a.count;
        c += (uint32_t)chunks_of(in[k], chunk);
      }
      if (c) launch(k_scale, c, 256, 0, (hipStream_t)hip_stream, a);
    }
    return launched("hieravg_scale_tensors");
  });
}

}  // extern "C"
