// Shared by the tensor operators (k_log_probs.hip, k_adamw.hip, k_blocks.hip):
// element types, unaligned vector access, argument checks.
#pragma once

#include <exception>

#include "internal.h"

namespace hav {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

constexpr int kBlock = 128;  // elements per scale
constexpr int64_t kMaxGroups = (int64_t(1) << 24) - 1;  // workgroups of 256 threads: a grid has less than 2^32

struct f16_t {
  uint16_t bits;
};
struct bf16_t {
  uint16_t bits;
};

__device__ inline float to_f32(float x) { return x; }
__device__ inline float to_f32(f16_t x) { return (float)__builtin_bit_cast(_Float16, x.bits); }
__device__ inline float to_f32(bf16_t x) { return __uint_as_float((uint32_t)x.bits << 16); }
// One rounding, to nearest even; NaN stays NaN.
__device__ inline uint16_t bf16_bits(float x) { return __builtin_bit_cast(uint16_t, (__bf16)x); }
__device__ inline uint16_t f16_bits(float x) { return __builtin_bit_cast(uint16_t, (_Float16)x); }
__device__ inline void from_f32(float x, float* o) { *o = x; }
__device__ inline void from_f32(float x, f16_t* o) { o->bits = f16_bits(x); }
__device__ inline void from_f32(float x, bf16_t* o) { o->bits = bf16_bits(x); }

// N elements at any address that suits one element, as one access of their
// whole width (the hardware takes unaligned vector accesses to global memory).
template <class T, int N>
struct Pack {
  T v[N];
};
template <class T, int N>
__device__ inline Pack<T, N> load_pack(const T* p) {
  Pack<T, N> r;
  __builtin_memcpy(&r, p, sizeof(r));
  return r;
}
template <class T, int N>
__device__ inline void store_pack(T* p, const Pack<T, N>& v) {
  __builtin_memcpy(p, &v, sizeof(v));
}

// Over the 64 lanes of a wave, the result in all of them: within 16 lanes by
// lane permutations, the four sixteens through scalar registers.
template <int CTRL>
__device__ inline float dpp_f(float v) {
  return __uint_as_float(dpp_u<CTRL>(__float_as_uint(v)));
}
template <class F>
__device__ inline float over_wave(float v, F&& f) {
  v = f(v, dpp_f<0xB1>(v));
  v = f(v, dpp_f<0x4E>(v));
  v = f(v, dpp_f<0x141>(v));
  v = f(v, dpp_f<0x140>(v));
  const int b = __builtin_bit_cast(int, v);
  auto lane = [&](int l) { return __builtin_bit_cast(float, __builtin_amdgcn_readlane(b, l)); };
  return f(f(lane(0), lane(16)), f(lane(32), lane(48)));
}
__device__ inline float max_over_wave(float v) {
  return over_wave(v, [](float a, float b) { return fmaxf(a, b); });
}
__device__ inline float add_over_wave(float v) {
  return over_wave(v, [](float a, float b) { return a + b; });
}
__device__ inline uint32_t max_over_wave(uint32_t v) {
  v = max16(v);
  auto lane = [&](int l) { return (uint32_t)__builtin_amdgcn_readlane((int)v, l); };
  return max(max(lane(0), lane(16)), max(lane(32), lane(48)));
}

inline bool known_type(int32_t t) { return t == HIERAVG_F32 || t == HIERAVG_F16 || t == HIERAVG_BF16; }
inline int type_bytes(int32_t t) { return t == HIERAVG_F32 ? 4 : 2; }
inline bool aligned(const void* p, uintptr_t n) { return ((uintptr_t)p & (n - 1)) == 0; }

// Whether rows this many elements apart can lie in memory (2^56 bytes; no
// offset then passes 64 bits).
inline bool addressable(int64_t rows, int64_t stride, int bytes) {
  return rows <= 1 || stride <= (int64_t(1) << 56) / bytes / (rows - 1);
}

inline int invalid(const char* msg) {
  set_error(msg);
  return HIERAVG_EINVAL;
}

inline int launched(const char* what) {
  const hipError_t e = hipGetLastError();
  if (e == hipSuccess) return HIERAVG_OK;
  set_error(std::string(what) + " failed to launch: " + hipGetErrorString(e));
  return HIERAVG_EHIP;
}

// The body of a C entry: no exception leaves it.
template <class F>
int guarded(F&& body) {
  try {
    return body();
  } catch (const std::exception&) {
    set_error("out of memory");  // short enough to need none
    return HIERAVG_EHIP;
  }
}

}  // namespace hav
