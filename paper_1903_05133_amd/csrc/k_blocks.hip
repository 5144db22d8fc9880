// Matrices in 8-bit floating point with a scale for each block of 128
// (include/hieravg.h, hieravg_quantize_blocks and hieravg_block_product).
#include <algorithm>

#include "ops.h"

namespace hav {

namespace {

typedef int i32x8 __attribute__((ext_vector_type(8)));

inline int64_t code_pitch(int64_t k) { return round_up(k, kBlock); }
inline int64_t scale_pitch(int64_t k) { return round_up(code_pitch(k) / kBlock, 4); }

// Exponent of a block's scale: the least e with amax <= 448 * 2^e = 1.75 * 2^(e + 8).
__device__ inline int scale_exponent(float amax) {
  if (amax == 0.0f) return 0;
  int shift = 0;
  if (amax < 0x1p-100f) {
    amax *= 0x1p64f;
    shift = 64;
  }
  const uint32_t b = __float_as_uint(amax);
  return max((int)(b >> 23) - 127 - shift - 8 + ((b & 0x7FFFFF) > 0x600000u ? 1 : 0), -127);
}
__device__ inline float inverse_of(int e) { return __uint_as_float((uint32_t)(127 - e) << 23); }  // e <= 120

__device__ inline bool finite(float x) { return (__float_as_uint(x) & 0x7FFFFFFF) < 0x7F800000u; }
__device__ inline uint8_t code_of(float x, float inv) {
  if (!finite(x)) return 0x7F;
  return (uint8_t)__builtin_amdgcn_cvt_pk_fp8_f32(x * inv, 0.0f, 0, false);
}

struct QuantArgs {
  const void* x;
  int64_t rows, cols, stride;
  uint8_t *codes, *scales, *codes_t, *scales_t;
  int64_t pitch, spitch, pitch_t, spitch_t;
  int64_t ctiles;
};

// One workgroup per 128 x 128 tile, in LDS.
template <class T, bool TILES>
__global__ __launch_bounds__(256) void k_quantize(QuantArgs a) {
  __shared__ float t[128][129];
  __shared__ int er[128], ec[128];
  const int64_t i0 = (blockIdx.x / a.ctiles) * 128, j0 = (blockIdx.x % a.ctiles) * 128;
  const int tid = threadIdx.x;
  for (int e = tid; e < 128 * 128; e += 256) {
    const int i = e >> 7, j = e & 127;
    t[i][j] = i0 + i < a.rows && j0 + j < a.cols ? to_f32(((const T*)a.x)[(i0 + i) * a.stride + j0 + j]) : 0.0f;
  }
  __syncthreads();
  {
    const int q = tid & 127;
    float m = 0.0f;
    for (int p = 0; p < 128; ++p) {
      const float v = tid < 128 ? t[q][p] : t[p][q];
      if (finite(v)) m = fmaxf(m, fabsf(v));
    }
    int* e = tid < 128 ? er : ec;
    e[q] = __float_as_int(m);
  }
  __syncthreads();
  if (TILES) {
    float m = 0.0f;
    for (int p = 0; p < 128; ++p) m = fmaxf(m, __int_as_float(er[p]));
    __syncthreads();
    if (tid < 128) er[tid] = ec[tid] = scale_exponent(m);
  } else if (tid < 128) {
    er[tid] = scale_exponent(__int_as_float(er[tid]));
    ec[tid] = scale_exponent(__int_as_float(ec[tid]));
  }
  __syncthreads();
  if (a.codes) {
    for (int e = tid; e < 128 * 128; e += 256) {
      const int i = e >> 7, j = e & 127;
      if (i0 + i < a.rows) a.codes[(i0 + i) * a.pitch + j0 + j] = code_of(t[i][j], inverse_of(er[i]));
    }
    const int64_t kb = j0 >> 7, nb = a.cols + 127 >> 7;
    if (TILES ? tid == 0 : tid < 128 && i0 + tid < a.rows) {
      uint8_t* s = a.scales + (TILES ? i0 >> 7 : i0 + tid) * a.spitch;
      s[kb] = (uint8_t)(er[tid] + 127);
      if (kb == nb - 1)
        for (int64_t p = nb; p < a.spitch; ++p) s[p] = 0;
    }
  }
  if (a.codes_t) {
    for (int e = tid; e < 128 * 128; e += 256) {
      const int j = e >> 7, i = e & 127;
      if (j0 + j < a.cols) a.codes_t[(j0 + j) * a.pitch_t + i0 + i] = code_of(t[i][j], inverse_of(ec[j]));
    }
    const int64_t kb = i0 >> 7, nb = a.rows + 127 >> 7;
    if (TILES ? tid == 0 : tid < 128 && j0 + tid < a.cols) {
      uint8_t* s = a.scales_t + (TILES ? j0 >> 7 : j0 + tid) * a.spitch_t;
      s[kb] = (uint8_t)(ec[tid] + 127);
      if (kb == nb - 1)
        for (int64_t p = nb; p < a.spitch_t; ++p) s[p] = 0;
    }
  }
}

struct ProductArgs {
  const uint8_t *a, *as, *b, *bs;
  int a_shift, b_shift;  // log2 of the rows per scale
  int64_t m, n, pitch, spitch;
  int kb;  // blocks of 128
  void* out;
  int64_t ldo;
  int64_t ntiles;
};

// One wave per 16 x 16 outputs, operands straight from memory.
template <class T>
__global__ __launch_bounds__(64) void k_product(ProductArgs p) {
  const int64_t i0 = (blockIdx.x / p.ntiles) * 16, j0 = (blockIdx.x % p.ntiles) * 16;
  const int lane = threadIdx.x, r = lane & 15, g = lane >> 4;
  const int64_t i = min(i0 + r, p.m - 1), j = min(j0 + r, p.n - 1);
  const uint8_t *pa = p.a + i * p.pitch + 32 * g, *pb = p.b + j * p.pitch + 32 * g;
  const uint8_t *sa = p.as + (i >> p.a_shift) * p.spitch, *sb = p.bs + (j >> p.b_shift) * p.spitch;
  f32x4 acc = {0.0f, 0.0f, 0.0f, 0.0f};
  for (int k = 0; k < p.kb; ++k) {
    const i32x8 x = *(const i32x8*)(pa + 128 * (int64_t)k), y = *(const i32x8*)(pb + 128 * (int64_t)k);
    acc = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(x, y, acc, 0, 0, 0, (int)sa[k], 0, (int)sb[k]);
  }
#pragma unroll
  for (int q = 0; q < 4; ++q)
    if (i0 + 4 * g + q < p.m && j0 + r < p.n) from_f32(acc[q], (T*)p.out + (i0 + 4 * g + q) * p.ldo + j0 + r);
}

}  // namespace

}  // namespace hav

using namespace hav;

extern "C" {

int hieravg_quantize_blocks(const void* x, int32_t type, int64_t rows, int64_t cols, int64_t row_stride,
                            int32_t tiles, uint8_t* codes, uint8_t* scales, uint8_t* codes_t, uint8_t* scales_t,
                            void* hip_stream) {
  return guarded([&]() -> int {
    if (!known_type(type)) return invalid("unknown element type");
    if (rows < 0 || cols < 1 || rows > 0x7FFFFF00 || cols > 0x7FFFFF00)
      return invalid("rows must be in [0, 2^31 - 256], cols in [1, 2^31 - 256]");
    if (row_stride < cols) return invalid("row_stride must be at least cols");
    if (tiles != 0 && tiles != 1) return invalid("tiles must be 0 or 1");
    if ((codes != nullptr) != (scales != nullptr) || (codes_t != nullptr) != (scales_t != nullptr))
      return invalid("codes and scales go together");
    if (!codes && !codes_t) return invalid("no block form asked for");
    if (rows == 0) return HIERAVG_OK;
    if (!x || !aligned(x, type_bytes(type))) return invalid("x must be a pointer aligned to its element");
    if (!aligned(codes, 16) || !aligned(codes_t, 16) || !aligned(scales, 4) || !aligned(scales_t, 4))
      return invalid("codes must be aligned to 16 bytes, scales to 4");
    QuantArgs a{x, rows, cols, row_stride, codes, scales, codes_t, scales_t, code_pitch(cols), scale_pitch(cols),
                code_pitch(rows), scale_pitch(rows), (cols + 127) / 128};
    const int64_t grid = a.ctiles * ((rows + 127) / 128);
    if (grid > 0x7FFFFFFF) return invalid("the matrix has too many blocks");
    hipStream_t s = (hipStream_t)hip_stream;
#define HAV_QUANT(T_)                                                        \
  do {                                                                       \
    if (tiles)                                                               \
      launch(k_quantize<T_, true>, (unsigned)grid, 256, 0, s, a);            \
    else                                                                     \
      launch(k_quantize<T_, false>, (unsigned)grid, 256, 0, s, a);           \
  } while (0)
    if (type == HIERAVG_F32)
      HAV_QUANT(float);
    else if (type == HIERAVG_F16)
      HAV_QUANT(f16_t);
    else
      HAV_QUANT(bf16_t);
#undef HAV_QUANT
    return launched("hieravg_quantize_blocks");
  });
}

size_t hieravg_block_product_scratch(int64_t m, int64_t n, int64_t k) {
  (void)m;
  (void)n;
  (void)k;
  return 0;
}

int hieravg_block_product(const uint8_t* a, const uint8_t* a_scales, int32_t a_tiles, const uint8_t* b,
                          const uint8_t* b_scales, int32_t b_tiles, int64_t m, int64_t n, int64_t k, void* out,
                          int32_t out_type, int64_t out_stride, void* scratch, size_t scratch_bytes,
                          void* hip_stream) {
  return guarded([&]() -> int {
    if (out_type != HIERAVG_F16 && out_type != HIERAVG_BF16)
      return invalid("out_type must be HIERAVG_F16 or HIERAVG_BF16");
    if (m < 0 || n < 0 || k < 1 || m > 0x7FFFFF00 || n > 0x7FFFFF00 || k > 0x7FFFFF00)
      return invalid("m and n must be in [0, 2^31 - 256], k in [1, 2^31 - 256]");
    if ((a_tiles != 0 && a_tiles != 1) || (b_tiles != 0 && b_tiles != 1)) return invalid("tiles must be 0 or 1");
    if (out_stride < n) return invalid("out_stride must be at least n");
    if (m == 0 || n == 0) return HIERAVG_OK;
    if (!a || !b || !a_scales || !b_scales || !out) return invalid("NULL operand");
    if (!aligned(a, 16) || !aligned(b, 16) || !aligned(a_scales, 4) || !aligned(b_scales, 4) || !aligned(out, 2))
      return invalid("codes must be aligned to 16 bytes, scales to 4, out to its element");
    const size_t need = hieravg_block_product_scratch(m, n, k);
    if (need && (!scratch || scratch_bytes < need || !aligned(scratch, 16)))
      return invalid("scratch must hold hieravg_block_product_scratch bytes, 16-byte aligned");
    ProductArgs p{a, a_scales, b, b_scales, a_tiles ? 7 : 0, b_tiles ? 7 : 0, m, n, code_pitch(k), scale_pitch(k),
                  (int)(code_pitch(k) / kBlock), out, out_stride, (n + 15) / 16};
    const int64_t grid = p.ntiles * ((m + 15) / 16);
    if (grid > 0x7FFFFFFF) return invalid("the product has too many tiles");
    if (out_type == HIERAVG_F16)
      launch(k_product<f16_t>, (unsigned)grid, 64, 0, (hipStream_t)hip_stream, p);
    else
      launch(k_product<bf16_t>, (unsigned)grid, 64, 0, (hipStream_t)hip_stream, p);
    return launched("hieravg_block_product");
  });
}

}  // extern "C"
