// AdamW over many tensors (include/hieravg.h, hieravg_adamw_*): one launch for
// up to 256 tensors, whose gradients' addresses are its arguments (so that a
// graph holds them), while parameters and states stay in a table in device
// memory.
#include <algorithm>
#include <cmath>
#include <new>
#include <utility>
#include <vector>

#include "ops.h"

namespace hav {

namespace {

constexpr uint64_t kTagAdamW = 0x68762e6164616d77ull;  // "hv.adamw"
constexpr int kChunk = 2048;     // elements of a tensor that one workgroup steps at a time
constexpr int kGradsPerLaunch = 256;

// One tensor as the kernels see it.
struct Tensor {
  void* param;
  void* copy;
  int64_t n;
  int64_t state;  // its first element in m and v
  int64_t chunk0; // its first chunk
  int32_t param_type, grad_type, copy_type, pad;
};

// What changes from step to step, in device memory.
struct Hyper {
  double lr;
  int64_t t;         // steps taken
  uint64_t key;      // random stream of step t + 1
  float step, root;  // lr / (1 - beta1^(t+1)), 1 / sqrt(1 - beta2^(t+1))
  float keep;        // 1 - lr * decay
  uint32_t done;     // workgroups of the running launch that have finished
};

struct Betas {
  double beta1, beta2, decay;
  uint64_t seed_key;  // H(seed, tag)
  float b1, b2, c1, c2, eps;  // float32 of beta1, beta2, 1 - beta1, 1 - beta2, eps
};

// x^n by squaring, a few dozen multiplications (pow's hundreds are the longest
// part of a small step): off by n roundings at most, 1e-16 n relative, while
// x^n counts beside 1; the same bits on the host, on the device and after a
// resume.
__host__ __device__ inline double power(double x, int64_t n) {
#pragma clang fp contract(off)
  double p = 1.0;
  for (; n > 0; n >>= 1) {
    if (n & 1) p *= x;
    x *= x;
  }
  return p;
}

__host__ __device__ inline void set_factors(Hyper* h, const Betas& b) {
  h->step = (float)(h->lr / (1.0 - power(b.beta1, h->t + 1)));
  h->root = (float)(1.0 / sqrt(1.0 - power(b.beta2, h->t + 1)));
  h->keep = (float)(1.0 - h->lr * b.decay);
  h->key = hash64(b.seed_key, (uint64_t)(h->t + 1));
}

struct AdamWArgs {
  const Tensor* tensors;
  const int32_t* chunk_tensor;
  Hyper* hyper;
  Betas b;
  void *m, *v;
  uint8_t *m_scales, *v_scales;
  int64_t chunk0, chunks;
  int first;  // first tensor of this launch
  int tick;   // the step's last launch
  const void* grads[kGradsPerLaunch];
};

// Eight consecutive elements of any type as they lie in memory.
struct Raw8 {
  u32x4 lo, hi;  // hi: float32 only
};
__device__ inline Raw8 load_raw8(const void* p, int type, int64_t i) {
  Raw8 r;
  if (type == HIERAVG_F32) {
    __builtin_memcpy(&r, (const float*)p + i, 32);
  } else {
    __builtin_memcpy(&r.lo, (const uint16_t*)p + i, 16);
    r.hi = u32x4{0, 0, 0, 0};
  }
  return r;
}
__device__ inline void unpack8(const Raw8& r, int type, float (&x)[8]) {
  if (type == HIERAVG_F32) {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      x[e] = __uint_as_float(r.lo[e]);
      x[4 + e] = __uint_as_float(r.hi[e]);
    }
  } else if (type == HIERAVG_BF16) {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      x[2 * e] = __uint_as_float(r.lo[e] << 16);
      x[2 * e + 1] = __uint_as_float(r.lo[e] & 0xFFFF0000u);
    }
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      x[2 * e] = to_f32(f16_t{(uint16_t)r.lo[e]});
      x[2 * e + 1] = to_f32(f16_t{(uint16_t)(r.lo[e] >> 16)});
    }
  }
}
__device__ inline uint32_t bits16(float x, int type) { return type == HIERAVG_BF16 ? bf16_bits(x) : f16_bits(x); }
__device__ inline void store8(void* p, int type, int64_t i, const float (&x)[8]) {
  if (type == HIERAVG_F32) {
    __builtin_memcpy((float*)p + i, x, 32);
  } else {
    u32x4 v;
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = bits16(x[2 * e], type) | bits16(x[2 * e + 1], type) << 16;
    __builtin_memcpy((uint16_t*)p + i, &v, 16);
  }
}
// One element, at the end of a tensor.
__device__ inline float load_one(const void* p, int type, int64_t i) {
  return type == HIERAVG_F32 ? ((const float*)p)[i]
                             : type == HIERAVG_F16 ? to_f32(((const f16_t*)p)[i]) : to_f32(((const bf16_t*)p)[i]);
}
__device__ inline void store_one(void* p, int type, int64_t i, float x) {
  if (type == HIERAVG_F32)
    ((float*)p)[i] = x;
  else
    ((uint16_t*)p)[i] = (uint16_t)bits16(x, type);
}

// 2^(byte - 127); NaN for 255.
__device__ inline float scale_of(uint32_t byte) {
  return __uint_as_float(byte == 0 ? 0x00400000u : byte == 255 ? 0x7FC00000u : byte << 23);
}
// 2^-e, -127 <= e <= 127.
__device__ inline float inverse_scale(int e) { return __uint_as_float(e == 127 ? 0x00400000u : (uint32_t)(127 - e) << 23); }

// The least e in [-127, 127] with amax <= (1 + top / 2^23) 2^(e + texp); 0 for amax = 0.
__device__ inline int block_exponent(float amax, uint32_t top, int texp) {
  if (amax == 0.0f) return 0;
  int shift = 0;
  if (amax < 0x1p-100f) {  // subnormals too
    amax *= 0x1p64f;
    shift = 64;
  }
  const uint32_t b = __float_as_uint(amax);
  const int e = (int)(b >> 23) - 127 - shift - texp + ((b & 0x7FFFFF) > top ? 1 : 0);
  return min(max(e, -127), 127);
}

// |y| <= 448 to E4M3 bits, rounded up where the fraction and r / 2^16 pass one.
__device__ inline uint32_t e4m3_random(float y, uint32_t r) {
  const uint32_t b = __float_as_uint(y);
  const float a = fabsf(y);
  const uint32_t c = a >= 0x1p-6f ? (((b & 0x7FFFFFFF) + (r << 4)) >> 20) - (120u << 3)
                                  : (uint32_t)(int)floorf(a * 512.0f + (float)r * 0x1p-16f);
  return c | (b >> 31) << 7;
}
// 0 <= y < 2 to the unsigned code of v.
__device__ inline uint32_t u4f4_random(float y, uint32_t r) {
  const uint32_t c = y >= 0x1p-14f ? ((__float_as_uint(y) + (r << 3)) >> 19) - (112u << 4)
                                   : (uint32_t)(int)floorf(y * 0x1p18f + (float)r * 0x1p-16f);
  return min(c, 255u);
}
__device__ inline float u4f4_value(uint32_t c) {
  return c < 16 ? (float)c * 0x1p-18f : __uint_as_float((c << 19) + (112u << 23));
}

// The first line of the step, each operation rounded by itself: the 8-bit
// codes depend on every bit of m and v.
__device__ inline void moments(const Betas& b, float g, float& m, float& v) {
#pragma clang fp contract(off)
  m = b.b1 * m + b.c1 * g;
  v = b.b2 * v + b.c2 * (g * g);
}

// The hardware's root takes what is below the normal range for 0: times 2^32
// first (below 2^-96), and the root by 2^16.
__device__ inline float root_of(float v) {
  const bool low = v < 0x1p-96f;
  const float r = __builtin_amdgcn_sqrtf(low ? v * 0x1p32f : v);
  return low ? r * 0x1p-16f : r;
}

__device__ inline int64_t round_up_128(int64_t n) { return (n + 127) & ~int64_t(127); }

// What only the host writes, read through the scalar cache.
template <class T>
__device__ inline T scalar_load(const T* p) {
  const auto* q = (const __attribute__((address_space(4))) uint32_t*)(uintptr_t)p;
  uint32_t w[sizeof(T) / 4];
#pragma unroll
  for (unsigned i = 0; i < sizeof(T) / 4; ++i) w[i] = q[i];
  T r;
  __builtin_memcpy(&r, w, sizeof(T));
  return r;
}

// A workgroup takes chunks of 2048 elements of one tensor, a thread eight
// consecutive ones (with 8 bits 16 lanes a block of 128, whose maxima are four
// steps within the lanes).  Memory is the bound: 28 bytes an element with
// float32 parameters, gradients and states; the types are the tensor's, so
// they are uniform branches around 16-byte accesses.  155 M parameters so: 850 us
// (5.1 TB/s); 66 M with 8-bit states, bf16 gradients and copies (16 bytes): 207
// us (5.1 TB/s).  The root (root_of) and the quotient are
// the hardware's, off by one unit in the last place each.
template <bool EIGHT>
__global__ __launch_bounds__(256) void k_adamw(AdamWArgs a) {
  const Hyper h = *a.hyper;
  const int tid = threadIdx.x;
  for (int64_t c = a.chunk0 + blockIdx.x; c < a.chunk0 + a.chunks; c += gridDim.x) {
    const int k = scalar_load(a.chunk_tensor + c);
    const Tensor t = scalar_load(a.tensors + k);
    const void* gp = a.grads[k - a.first];
    if (!gp) continue;
    const int64_t i = (c - t.chunk0) * kChunk + 8 * tid, s = t.state + i;
    const int64_t have = t.n - i;
    // With 8 bits the rest of a tensor's last block steps too, on gradient 0.
    const bool in = EIGHT ? i < round_up_128(t.n) : have > 0;
    float g[8], w[8], m[8], v[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) g[e] = w[e] = m[e] = v[e] = 0.0f;
    if (in) {
      Raw8 rg, rw;
      u32x2 cm, cv;
      uint32_t bm, bv;
      if (have >= 8) {
        rw = load_raw8(t.param, t.param_type, i);
        rg = load_raw8(gp, t.grad_type, i);
      }
      if (EIGHT) {
        cm = *(const u32x2*)((const uint8_t*)a.m + s);
        cv = *(const u32x2*)((const uint8_t*)a.v + s);
        bm = a.m_scales[s >> 7];
        bv = a.v_scales[s >> 7];
      } else if (have >= 8) {
        __builtin_memcpy(m, (const float*)a.m + s, 32);
        __builtin_memcpy(v, (const float*)a.v + s, 32);
      }
      if (have >= 8) {
        unpack8(rw, t.param_type, w);
        unpack8(rg, t.grad_type, g);
      } else {
#pragma unroll
        for (int e = 0; e < 8; ++e)
          if (e < have) {
            w[e] = load_one(t.param, t.param_type, i + e);
            g[e] = load_one(gp, t.grad_type, i + e);
            if (!EIGHT) {
              m[e] = ((const float*)a.m)[s + e];
              v[e] = ((const float*)a.v)[s + e];
            }
          }
      }
      if (EIGHT) {
        const float sm = scale_of(bm), sv = scale_of(bv);
#pragma unroll
        for (int e = 0; e < 8; e += 2) {
          const auto x = e & 2 ? __builtin_amdgcn_cvt_pk_f32_fp8((int)cm[e >> 2], true)
                               : __builtin_amdgcn_cvt_pk_f32_fp8((int)cm[e >> 2], false);
          m[e] = x[0] * sm;
          m[e + 1] = x[1] * sm;
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = u4f4_value((cv[e >> 2] >> (8 * (e & 3))) & 0xFF) * sv;
      }
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        moments(a.b, g[e], m[e], v[e]);
        w[e] = w[e] * h.keep - h.step * m[e] * __builtin_amdgcn_rcpf(root_of(v[e]) * h.root + a.b.eps);
      }
      if (have >= 8) {
        store8(t.param, t.param_type, i, w);
        if (t.copy) store8(t.copy, t.copy_type, i, w);
        if (!EIGHT) {
          __builtin_memcpy((float*)a.m + s, m, 32);
          __builtin_memcpy((float*)a.v + s, v, 32);
        }
      } else {
#pragma unroll
        for (int e = 0; e < 8; ++e)
          if (e < have) {
            store_one(t.param, t.param_type, i + e, w[e]);
            if (t.copy) store_one(t.copy, t.copy_type, i + e, w[e]);
            if (!EIGHT) {
              ((float*)a.m)[s + e] = m[e];
              ((float*)a.v)[s + e] = v[e];
            }
          }
      }
    }
    if (EIGHT) {
      uint32_t bm = 0, bv = 0;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        bm = max(bm, __float_as_uint(m[e]) & 0x7FFFFFFFu);
        bv = max(bv, __float_as_uint(v[e]) & 0x7FFFFFFFu);
      }
      bm = max16(bm);
      bv = max16(bv);
      const bool pm = bm >= 0x7F800000u, pv = bv >= 0x7F800000u;
      const int em = pm ? 0 : block_exponent(__uint_as_float(bm), 0x600000, 8);
      const int ev = pv ? 0 : block_exponent(__uint_as_float(bv), 0x780000, 0);
      if (in) {
        const float im = inverse_scale(em), iv = inverse_scale(ev);
        u32x2 cm = {0, 0}, cv = {0, 0};
        // hash64(key, s/2 + q): the counters of neighbours differ by kGolden
        uint64_t z = h.key + (((uint64_t)s >> 1) + 1) * kGolden;
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          const uint64_t bits = mix64(z);
          z += kGolden;
#pragma unroll
          for (int o = 0; o < 2; ++o) {
            const int e = 2 * q + o;
            const uint32_t r = o ? (uint32_t)(bits >> 32) : (uint32_t)bits;
            uint32_t xm = e4m3_random(m[e] * im, r & 0xFFFF), xv = u4f4_random(v[e] * iv, r >> 16);
            if (v[e] > 0.0f) xv = max(xv, 1u);
            cm[e >> 2] |= xm << (8 * (e & 3));
            cv[e >> 2] |= xv << (8 * (e & 3));
          }
        }
        if (pm) cm = u32x2{0, 0};
        if (pv) cv = u32x2{0, 0};
        *(u32x2*)((uint8_t*)a.m + s) = cm;
        *(u32x2*)((uint8_t*)a.v + s) = cv;
        if ((tid & 15) == 0) {
          a.m_scales[s >> 7] = (uint8_t)(pm ? 255 : em + 127);
          a.v_scales[s >> 7] = (uint8_t)(pv ? 255 : ev + 127);
        }
      }
    }
  }
  if (!a.tick) return;
  // The last workgroup to get here sets the next step's factors: every one has
  // read this step's by then (its values are needed here), and nothing else
  // passes between them, so the count needs no fence.  (With one, whose release
  // writes the L2 back, 4096 workgroups took 1154 us for 155 M parameters.)
  asm volatile("" ::"v"(h.step), "v"(h.root), "v"(h.keep), "v"((uint32_t)h.key), "v"((uint32_t)(h.key >> 32)));
  __syncthreads();
  if (tid == 0) {
    if (__hip_atomic_fetch_add(&a.hyper->done, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == gridDim.x - 1) {
      Hyper* p = a.hyper;
      p->done = 0;
      p->t = h.t + 1;
      set_factors(p, a.b);
    }
  }
}

// lr < 0 or t < 0: as it is.
__global__ void k_set_hyper(Hyper* h, Betas b, double lr, int64_t t) {
  if (lr >= 0.0) h->lr = lr;
  if (t >= 0) h->t = t;
  set_factors(h, b);
}

int64_t state_size(const int64_t* n, int32_t count) {
  int64_t s = 0;
  for (int32_t k = 0; k < count; ++k) {
    if (n[k] < 0 || n[k] > (int64_t(1) << 40)) return -1;
    s += round_up(n[k], kBlock);
    if (s > int64_t(1) << 56) return -1;
  }
  return s;
}

}  // namespace

}  // namespace hav

using namespace hav;

struct hieravg_adamw {
  Betas b{};
  int bits = 32, device = 0;
  void *m = nullptr, *v = nullptr;
  uint8_t *m_scales = nullptr, *v_scales = nullptr;
  std::vector<Tensor> tensors;
  int64_t chunks = 0;
  char* dev = nullptr;  // Hyper, the tensors, the chunks' tensors
  Tensor* d_tensors = nullptr;
  int32_t* d_chunks = nullptr;
};

namespace {

// What the device holds once all that was enqueued has run.
int read_hyper(hieravg_adamw_t h, Hyper* hy, const char* what) {
  hipError_t e = hipDeviceSynchronize();
  if (e == hipSuccess) e = hipMemcpy(hy, h->dev, sizeof(*hy), hipMemcpyDeviceToHost);
  if (e == hipSuccess) return HIERAVG_OK;
  set_error(std::string(what) + ": " + hipGetErrorString(e));
  return HIERAVG_EHIP;
}

}  // namespace

extern "C" {

int64_t hieravg_adamw_state_size(const int64_t* n, int32_t count) {
  if (!n || count < 1) {
    set_error("no tensors");
    return HIERAVG_EINVAL;
  }
  const int64_t s = state_size(n, count);
  if (s < 0) {
    set_error("a tensor's size is negative or beyond 2^40, or all of them are beyond 2^56");
    return HIERAVG_EINVAL;
  }
  return s;
}

hieravg_adamw_t hieravg_adamw_create(const hieravg_adamw_config* cfg, const hieravg_adamw_tensor* tensors,
                                     int32_t count, void* m, void* v, uint8_t* m_scales, uint8_t* v_scales) {
  hieravg_adamw* h = nullptr;
  const int rc = guarded([&]() -> int {
    if (!cfg || !tensors || count < 1) return invalid("no configuration or no tensors");
    if (!(cfg->lr >= 0.0) || !std::isfinite(cfg->lr)) return invalid("lr must be finite and >= 0");
    if (!(cfg->beta1 >= 0.0 && cfg->beta1 < 1.0) || !(cfg->beta2 >= 0.0 && cfg->beta2 < 1.0))
      return invalid("betas must be in [0, 1)");
    // the step multiplies by 1 / eps where the moments are 0
    if (!((float)cfg->eps >= 0x1p-126f) || !std::isfinite((float)cfg->eps))
      return invalid("eps must be a float32 of at least 2^-126");
    if (!(cfg->weight_decay >= 0.0) || !std::isfinite(cfg->weight_decay))
      return invalid("weight_decay must be finite and >= 0");
    if (cfg->state_bits != 8 && cfg->state_bits != 32) return invalid("state_bits must be 8 or 32");
    h = new hieravg_adamw;
    h->bits = cfg->state_bits;
    int64_t state = 0;
    std::vector<int32_t> owner;
    std::vector<std::pair<uintptr_t, uintptr_t>> written;
    for (int32_t k = 0; k < count; ++k) {
      const hieravg_adamw_tensor& t = tensors[k];
      if (t.n < 0 || t.n > (int64_t(1) << 40)) return invalid("a tensor's size is negative or beyond 2^40");
      if (!known_type(t.param_type) || !known_type(t.grad_type) || (t.copy && !known_type(t.copy_type)))
        return invalid("unknown element type");
      if (t.n > 0 && (!t.param || !aligned(t.param, type_bytes(t.param_type))))
        return invalid("a parameter must be a pointer aligned to its element");
      if (t.copy && !aligned(t.copy, type_bytes(t.copy_type))) return invalid("a copy must be aligned to its element");
      const int64_t nc = (t.n + kChunk - 1) / kChunk;
      h->tensors.push_back({t.param, t.copy, t.n, state, (int64_t)owner.size(), t.param_type, t.grad_type, t.copy_type, 0});
      if ((int64_t)owner.size() + nc > 0x7FFFFFFF) return invalid("too many elements");
      owner.insert(owner.end(), (size_t)nc, k);
      if (t.n > 0) {
        const uintptr_t p = (uintptr_t)t.param, c = (uintptr_t)t.copy;
        written.push_back({p, p + (uintptr_t)t.n * type_bytes(t.param_type)});
        if (c) written.push_back({c, c + (uintptr_t)t.n * type_bytes(t.copy_type)});
      }
      state += round_up(t.n, kBlock);
    }
    if (state > 0 && (!m || !v || !aligned(m, 16) || !aligned(v, 16)))
      return invalid("m and v must be pointers aligned to 16 bytes");
    if (state > 0 && h->bits == 8 && (!m_scales || !v_scales)) return invalid("8-bit states need their scales");
    std::sort(written.begin(), written.end());
    for (size_t i = 1; i < written.size(); ++i)
      if (written[i].first < written[i - 1].second) return invalid("parameters and copies must not overlap");
    h->m = m;
    h->v = v;
    h->m_scales = m_scales;
    h->v_scales = v_scales;
    h->chunks = (int64_t)owner.size();
    h->b = {cfg->beta1, cfg->beta2, cfg->weight_decay, hash64(cfg->seed, kTagAdamW), (float)cfg->beta1,
            (float)cfg->beta2, (float)(1.0 - cfg->beta1), (float)(1.0 - cfg->beta2), (float)cfg->eps};
    Hyper hy{};
    hy.lr = cfg->lr;
    set_factors(&hy, h->b);
    const size_t o1 = 256, o2 = o1 + round_up(sizeof(Tensor) * count, 256), bytes = o2 + sizeof(int32_t) * owner.size();
    hipError_t e = hipGetDevice(&h->device);
    if (e == hipSuccess) e = hipMalloc((void**)&h->dev, bytes);
    if (e == hipSuccess) e = hipMemcpy(h->dev, &hy, sizeof(hy), hipMemcpyHostToDevice);
    if (e == hipSuccess) e = hipMemcpy(h->dev + o1, h->tensors.data(), sizeof(Tensor) * count, hipMemcpyHostToDevice);
    if (e == hipSuccess && !owner.empty())
      e = hipMemcpy(h->dev + o2, owner.data(), sizeof(int32_t) * owner.size(), hipMemcpyHostToDevice);
    if (e != hipSuccess) {
      set_error(std::string("hieravg_adamw_create: ") + hipGetErrorString(e));
      return HIERAVG_EHIP;
    }
    h->d_tensors = (Tensor*)(h->dev + o1);
    h->d_chunks = (int32_t*)(h->dev + o2);
    return HIERAVG_OK;
  });
  if (rc == HIERAVG_OK) return h;
  hieravg_adamw_destroy(h);
  return nullptr;
}

int hieravg_adamw_step(hieravg_adamw_t h, const void* const* grads, void* hip_stream) {
  return guarded([&]() -> int {
    if (!h || !grads) return invalid("NULL handle or gradients");
    const int count = (int)h->tensors.size();
    for (int k = 0; k < count; ++k)
      if (grads[k] && !aligned(grads[k], type_bytes(h->tensors[k].grad_type)))
        return invalid("a gradient must be aligned to its element");
    for (int k0 = 0; k0 < count; k0 += kGradsPerLaunch) {
      const int k1 = std::min(count, k0 + kGradsPerLaunch);
      AdamWArgs a;
      a.tensors = h->d_tensors;
      a.chunk_tensor = h->d_chunks;
      a.hyper = (Hyper*)h->dev;
      a.b = h->b;
      a.m = h->m;
      a.v = h->v;
      a.m_scales = h->m_scales;
      a.v_scales = h->v_scales;
      a.chunk0 = h->tensors[k0].chunk0;
      a.chunks = (k1 < count ? h->tensors[k1].chunk0 : h->chunks) - a.chunk0;
      a.first = k0;
      a.tick = k1 == count;
      for (int k = k0; k < k1; ++k) a.grads[k - k0] = grads[k];
      for (int k = k1; k < k0 + kGradsPerLaunch; ++k) a.grads[k - k0] = nullptr;
      // 8192 workgroups loop over the chunks: with one per chunk (75 000 for 155 M
      // parameters) their counts at one address take longer (960 against 864 us;
      // 8-bit 390 against 208), 2048 leave memory less to do (871; 222).  Measured
      // at 155 and 66 M; for fewer chunks than that the counts, 12 ns each, are
      // most of the time (8-bit, 17 M: 106 us, its bytes 53; 4 M: 30, its bytes 13).
      const unsigned grid = (unsigned)std::max<int64_t>(1, std::min<int64_t>(a.chunks, 8192));
      if (h->bits == 8)
        launch(k_adamw<true>, grid, 256, 0, (hipStream_t)hip_stream, a);
      else
        launch(k_adamw<false>, grid, 256, 0, (hipStream_t)hip_stream, a);
    }
    return launched("hieravg_adamw_step");
  });
}

int hieravg_adamw_set_lr(hieravg_adamw_t h, double lr, void* hip_stream) {
  return guarded([&]() -> int {
    if (!h) return invalid("NULL handle");
    if (!(lr >= 0.0) || !std::isfinite(lr)) return invalid("lr must be finite and >= 0");
    launch(k_set_hyper, 1, 1, 0, (hipStream_t)hip_stream, (Hyper*)h->dev, h->b, lr, int64_t(-1));
    return launched("hieravg_adamw_set_lr");
  });
}

int hieravg_adamw_set_steps(hieravg_adamw_t h, int64_t t, void* hip_stream) {
  return guarded([&]() -> int {
    if (!h) return invalid("NULL handle");
    if (t < 0 || t > int64_t(1) << 62) return invalid("the step count must be in [0, 2^62]");
    launch(k_set_hyper, 1, 1, 0, (hipStream_t)hip_stream, (Hyper*)h->dev, h->b, -1.0, t);
    return launched("hieravg_adamw_set_steps");
  });
}

int64_t hieravg_adamw_steps(hieravg_adamw_t h) {
  Hyper hy{};
  const int rc = guarded([&]() -> int { return h ? read_hyper(h, &hy, "hieravg_adamw_steps") : invalid("NULL handle"); });
  return rc == HIERAVG_OK ? hy.t : rc;
}

int hieravg_adamw_lr(hieravg_adamw_t h, double* lr) {
  return guarded([&]() -> int {
    if (!h || !lr) return invalid("NULL handle or lr");
    Hyper hy{};
    const int rc = read_hyper(h, &hy, "hieravg_adamw_lr");
    if (rc == HIERAVG_OK) *lr = hy.lr;
    return rc;
  });
}

void hieravg_adamw_destroy(hieravg_adamw_t h) {
  if (!h) return;
  if (h->dev) (void)hipFree(h->dev);
  delete h;
}

}  // extern "C"
