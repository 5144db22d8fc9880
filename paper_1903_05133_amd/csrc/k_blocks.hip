// Matrices in 8-bit floating point with a scale for each block of 128
// (include/hieravg.h, hieravg_quantize_blocks and hieravg_block_product).
#include <algorithm>
#include <utility>

#include "ops.h"

namespace hav {

namespace {

typedef int i32x2 __attribute__((ext_vector_type(2)));
typedef int i32x4 __attribute__((ext_vector_type(4)));

// A tile's rows of a contraction this long are addressed with 32-bit offsets.
constexpr int64_t kMaxContraction = int64_t(1) << 23;
constexpr int64_t kMostRows = 0x7FFFFF00;

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

constexpr uint32_t kInf = 0x7F800000u;
__device__ inline uint32_t abs_bits(float x) { return __float_as_uint(x) & 0x7FFFFFFFu; }

// The codes of eight values that share a scale, `finite`: all are finite.
__device__ inline u32x2 codes8(const float (&x)[8], float inv, bool finite) {
  int lo = __builtin_amdgcn_cvt_pk_fp8_f32(x[0] * inv, x[1] * inv, 0, false);
  lo = __builtin_amdgcn_cvt_pk_fp8_f32(x[2] * inv, x[3] * inv, lo, true);
  int hi = __builtin_amdgcn_cvt_pk_fp8_f32(x[4] * inv, x[5] * inv, 0, false);
  hi = __builtin_amdgcn_cvt_pk_fp8_f32(x[6] * inv, x[7] * inv, hi, true);
  u32x2 c = {(uint32_t)lo, (uint32_t)hi};
  if (!finite) {
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (abs_bits(x[e]) >= kInf) c[e >> 2] = (c[e >> 2] & ~(0xFFu << (8 * (e & 3)))) | 0x7Fu << (8 * (e & 3));
  }
  return c;
}

// Eight consecutive elements of a row, `have` of which exist (the others 0).
template <class T>
__device__ inline void load8(const T* p, int64_t have, float (&x)[8]) {
  if (have >= 8) {
    const Pack<T, 8> v = load_pack<T, 8>(p);
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = to_f32(v.v[e]);
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = e < have ? to_f32(p[e]) : 0.0f;
  }
}

// The largest finite magnitude (as bits) of x; *any: the largest of all.
__device__ inline uint32_t largest(const float (&x)[8], uint32_t* any) {
  uint32_t m = 0;
#pragma unroll
  for (int e = 0; e < 8; ++e) m = max(m, abs_bits(x[e]));
  *any = m;
  if (m < kInf) return m;
  m = 0;
#pragma unroll
  for (int e = 0; e < 8; ++e) m = max(m, abs_bits(x[e]) < kInf ? abs_bits(x[e]) : 0u);
  return m;
}

struct QuantArgs {
  const void* x;
  int64_t rows, cols, stride;
  uint8_t *codes, *scales, *codes_t, *scales_t;
  int64_t pitch, spitch, pitch_t, spitch_t;
  int64_t ctiles;
};

// 1 x 128 blocks of rows alone: a wave per four blocks of a row (16 lanes a
// block, eight elements a lane), whose four scale bytes are one store.  HBM is
// the bound (308 MB of bf16: 83 us, 5.6 TB/s read and written).
template <class T>
__global__ __launch_bounds__(256) void k_quantize_rows(QuantArgs a) {
  const int lane = threadIdx.x & 63;
  const int64_t quads = a.spitch / 4, unit = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  if (unit >= a.rows * quads) return;
  const int64_t row = unit / quads, quad = unit - row * quads, col = quad * 512 + lane * 8;
  float x[8];
  load8((const T*)a.x + row * a.stride + col, a.cols - col, x);
  uint32_t any;
  const uint32_t m = max16(largest(x, &any));
  const int e = scale_exponent(__uint_as_float(m));
  if (col < a.pitch) *(u32x2*)(a.codes + row * a.pitch + col) = codes8(x, inverse_of(e), any < kInf);
  // blocks past the last: 0
  uint32_t s = col < a.pitch ? (uint32_t)(e + 127) << (8 * (lane >> 4)) : 0;
  s |= __shfl_xor((int)s, 16, 64);
  s |= __shfl_xor((int)s, 32, 64);
  if (lane == 0) *(uint32_t*)(a.scales + row * a.spitch + quad * 4) = s;
}

// Eight rows of eight elements as they lie in memory, 16-bit ones two to a
// register (so that a thread's tile takes 32), and the largest magnitudes of
// its rows and columns as float bits.
typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
__device__ inline uint32_t max2(uint32_t a, uint32_t b) {  // of both halves
  return __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(u16x2, a), __builtin_bit_cast(u16x2, b)));
}
template <class T>
struct Tile8 {
  u32x4 w[8];
  __device__ void load(int i, const T* p, int64_t have) {
    if (have >= 8) {
      __builtin_memcpy(&w[i], p, 16);
    } else {
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const uint32_t lo = 2 * q < have ? p[2 * q].bits : 0, hi = 2 * q + 1 < have ? p[2 * q + 1].bits : 0;
        w[i][q] = lo | hi << 16;
      }
    }
  }
  __device__ float get(int i, int j) const { return to_f32(T{(uint16_t)(w[i][j >> 1] >> (16 * (j & 1)))}); }
  // Returns the largest of all; filter: of the finite ones.
  __device__ uint32_t maxima(uint32_t (&r)[8], uint32_t (&c)[8], bool filter) const {
    uint32_t cm[4] = {0, 0, 0, 0}, all = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      uint32_t m[4], rm = 0;
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        m[q] = w[i][q] & 0x7FFF7FFFu;
        if (filter) {
          if (abs_bits(get(i, 2 * q)) >= kInf) m[q] &= 0xFFFF0000u;
          if (abs_bits(get(i, 2 * q + 1)) >= kInf) m[q] &= 0x0000FFFFu;
        }
        cm[q] = max2(cm[q], m[q]);
        rm = max2(rm, m[q]);
      }
      r[i] = abs_bits(to_f32(T{(uint16_t)max(rm & 0xFFFF, rm >> 16)}));
      all = max(all, r[i]);
    }
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      c[2 * q] = abs_bits(to_f32(T{(uint16_t)cm[q]}));
      c[2 * q + 1] = abs_bits(to_f32(T{(uint16_t)(cm[q] >> 16)}));
    }
    return all;
  }
};
template <>
struct Tile8<float> {
  float x[8][8];
  __device__ void load(int i, const float* p, int64_t have) { load8(p, have, x[i]); }
  __device__ float get(int i, int j) const { return x[i][j]; }
  __device__ uint32_t maxima(uint32_t (&r)[8], uint32_t (&c)[8], bool filter) const {
    uint32_t all = 0;
#pragma unroll
    for (int j = 0; j < 8; ++j) c[j] = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      r[i] = 0;
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const uint32_t b = abs_bits(x[i][j]), m = filter && b >= kInf ? 0 : b;
        r[i] = max(r[i], m);
        c[j] = max(c[j], m);
      }
      all = max(all, r[i]);
    }
    return all;
  }
};

// The other forms: a workgroup per 128 x 128 tile, a thread per 8 x 8 of it in
// registers; the transposed codes go through LDS (33 words a column: the 8-byte
// pieces of a wave spread over all banks).  308 MB of bf16: transposed 93 us
// (5.0 TB/s), both forms 130 (4.7), 128 x 128 blocks 88 (5.2).
template <class T, bool TILES>
__global__ __launch_bounds__(256) void k_quantize_tile(QuantArgs a) {
  __shared__ uint32_t t[128 * 33];
  __shared__ uint32_t cm[4][128];
  const int64_t ti = blockIdx.x / a.ctiles, tj = blockIdx.x - ti * a.ctiles, i0 = ti * 128, j0 = tj * 128;
  const int tid = threadIdx.x, c = tid & 15, rg = tid >> 4, wave = tid >> 6;
  Tile8<T> x;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int64_t row = i0 + 8 * rg + i, col = j0 + 8 * c;
    x.load(i, (const T*)a.x + row * a.stride + col, row < a.rows ? a.cols - col : 0);
  }
  uint32_t rmax[8], cmax[8];
  const bool finite = x.maxima(rmax, cmax, false) < kInf;
  if (!finite) x.maxima(rmax, cmax, true);
  float cinv[8];
  int re[8];
  if (TILES) {
    uint32_t m = 0;
#pragma unroll
    for (int j = 0; j < 8; ++j) m = max(m, cmax[j]);
    m = max16(m);
    m = max(m, (uint32_t)__shfl_xor((int)m, 16, 64));
    m = max(m, (uint32_t)__shfl_xor((int)m, 32, 64));
    if ((tid & 63) == 0) cm[0][wave] = m;
    __syncthreads();
    m = max(max(cm[0][0], cm[0][1]), max(cm[0][2], cm[0][3]));
    const int e = scale_exponent(__uint_as_float(m));
    const float inv = inverse_of(e);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      re[i] = e;
      cinv[i] = inv;
    }
    if (tid == 0) {
      // and zeros behind the last block of a row of scales
      if (a.codes) {
        uint8_t* s = a.scales + ti * a.spitch;
        s[tj] = (uint8_t)(e + 127);
        if (tj == a.ctiles - 1)
          for (int64_t q = tj + 1; q < a.spitch; ++q) s[q] = 0;
      }
      if (a.codes_t) {
        uint8_t* s = a.scales_t + tj * a.spitch_t;
        s[ti] = (uint8_t)(e + 127);
        if (i0 + 128 >= a.rows)
          for (int64_t q = ti + 1; q < a.spitch_t; ++q) s[q] = 0;
      }
    }
  } else {
    if (a.codes) {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        re[i] = scale_exponent(__uint_as_float(max16(rmax[i])));
        const int64_t row = i0 + 8 * rg + i;
        if (c == 0 && row < a.rows) {
          uint8_t* s = a.scales + row * a.spitch;
          s[tj] = (uint8_t)(re[i] + 127);
          if (tj == a.ctiles - 1)
            for (int64_t q = tj + 1; q < a.spitch; ++q) s[q] = 0;
        }
      }
    }
    if (a.codes_t) {
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        uint32_t m = cmax[j];
        m = max(m, (uint32_t)__shfl_xor((int)m, 16, 64));
        m = max(m, (uint32_t)__shfl_xor((int)m, 32, 64));
        if ((tid & 63) < 16) cm[wave][8 * c + j] = m;
      }
      __syncthreads();
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const int q = 8 * c + j;
        const int e = scale_exponent(__uint_as_float(max(max(cm[0][q], cm[1][q]), max(cm[2][q], cm[3][q]))));
        cinv[j] = inverse_of(e);
        if (rg == 0 && j0 + q < a.cols) {
          uint8_t* s = a.scales_t + (j0 + q) * a.spitch_t;
          s[ti] = (uint8_t)(e + 127);
          if (i0 + 128 >= a.rows)
            for (int64_t z = ti + 1; z < a.spitch_t; ++z) s[z] = 0;
        }
      }
    }
  }
  if (a.codes) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int64_t row = i0 + 8 * rg + i;
      float y[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) y[j] = x.get(i, j);
      if (row < a.rows) *(u32x2*)(a.codes + row * a.pitch + j0 + 8 * c) = codes8(y, inverse_of(re[i]), finite);
    }
  }
  if (a.codes_t) {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      float y[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) y[i] = x.get(i, j);
      const u32x2 v = codes8(y, cinv[j], finite);
      uint32_t* o = t + (8 * c + j) * 33 + 2 * rg;
      o[0] = v[0];
      o[1] = v[1];
    }
    __syncthreads();
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const int col = q * 32 + (tid >> 3), w = (tid & 7) * 4;
      const uint32_t* o = t + col * 33 + w;
      if (j0 + col < a.cols) *(u32x4*)(a.codes_t + (j0 + col) * a.pitch_t + i0 + 4 * w) = u32x4{o[0], o[1], o[2], o[3]};
    }
  }
}

// ------------------------------------------------------------ products
// The matrix cores' products of 8-bit floats keep less than float32 does: a
// block's sum is off by 2^-14 to 2^-13 of its largest product (+-448^2 and 126
// products around 1, 16 x 16 x 128: by a third of the sum).  So the
// codes become bf16 times their block's power of two, which is exact from 2^-126
// up to 2^128 and takes an instruction for two, and the products of bf16, whose
// sums are in float32 (the same sum to 0.1 %).  A lane's eight codes of a row
// are an operand; which of the contraction's elements they are does not matter as
// long as both operands take the same.  The weights (b) are the first operand,
// so that a lane ends up with four consecutive columns of a row of the result.
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

// 2^(byte - 127) of byte u of four blocks' scales, 0 for byte 0 and infinity
// for 255, which the conversion reads as 2^-127 and NaN.
__device__ inline float scale_of_byte(int word, int u) {
  return __uint_as_float(((uint32_t)word >> (8 * u) & 0xFFu) << 23);
}
// Codes 2w and 2w + 1 of an operand's eight, which are `codes`.
__device__ inline int two_values(i32x2 codes, int w, float scale) {
  return __builtin_bit_cast(int, w & 1 ? __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((uint32_t)codes[w >> 1], scale, true)
                                       : __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((uint32_t)codes[w >> 1], scale, false));
}
__device__ inline i32x4 eight_values(i32x2 codes, float scale) {
  return i32x4{two_values(codes, 0, scale), two_values(codes, 1, scale), two_values(codes, 2, scale),
               two_values(codes, 3, scale)};
}
__device__ inline f32x16 product32(i32x4 b, i32x4 a, f32x16 c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, b), __builtin_bit_cast(bf16x8, a), c, 0, 0, 0);
}
__device__ inline f32x4 product16(i32x4 b, i32x4 a, f32x4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, b), __builtin_bit_cast(bf16x8, a), c, 0, 0, 0);
}

struct ProductArgs {
  const uint8_t *a, *as, *b, *bs;
  int a_shift, b_shift;  // log2 of the rows per scale
  int64_t m, n, pitch, spitch;
  int kb;  // blocks of 128
  void* out;
  int64_t ldo;
  int tm, tn;        // tiles along m and n
  float* part;       // partial sums [splits][m][n], if splits > 1
  int splits, cps;   // splits of the contraction, blocks of each (a multiple of 4)
  int swap;
};

// The result's type is a template argument: as a value it makes the compiler
// convert both ways and choose (256 results a lane: 2 us a tile).
template <bool F16>
__device__ inline uint16_t out_bits(float x) {
  return F16 ? f16_bits(x) : bf16_bits(x);
}
template <bool F16>
__device__ inline uint32_t pack2(float x, float y) {
  return (uint32_t)out_bits<F16>(x) | (uint32_t)out_bits<F16>(y) << 16;
}

// Workgroup -> tile: consecutive tiles on one XCD, four tile rows of a at a
// time, so that the tiles that run together share panels in that XCD's L2.
__device__ inline void tile_of(const ProductArgs& p, int t, int* ti, int* tj) {
  const int rows = 4, group = t / (rows * p.tn), first = group * rows, have = min(p.tm - first, rows);
  const int in = t - group * rows * p.tn;
  *ti = first + in % have;
  *tj = in / have;
}

// Swizzle of the 16-byte pieces of a 128-byte row in LDS: the 16 lanes that a
// b128 read takes at a time touch every bank once.
__device__ inline int swz(int row) { return (row >> 1) & 7; }

// Eight of a piece's 16 codes.
__device__ inline i32x2 half_of(i32x4 x, int q) { return q & 1 ? i32x2{x[2], x[3]} : i32x2{x[0], x[1]}; }

typedef __attribute__((address_space(3))) void* lds_ptr;
template <int V>
struct Int {
  static constexpr int value = V;
};

// The loads into LDS have landed, in every wave.
__device__ inline void landed() {
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
  __syncthreads();
}

// Large products: 256 x 256 outputs per workgroup, four waves of 128 x 128 (all
// 256 accumulation registers of a lane), 256 rows of each operand at a time in
// LDS as codes, two buffers.  A step is a block of 128, in eighths of 16
// products; beside each product of an eighth two words of operands are made,
// one of b's for the next eighth and one of a's for the next row tile.  The
// second half's codes are read in the first eighth; then, after the one barrier
// of a step, which stands in its middle, where the buffer has been read, the
// next step's first half, and the loads of the step after next start into that
// buffer.
// Needs m, n >= 256: the last tiles start where they are whole, and store what
// no other tile does.
// 8192^3: 700 to 800 us as the card is warm, 1.57 to 1.37 PFLOP/s; 4096^3 95 us,
// 1.45.  The bound is the matrix cores, 77 % busy, at the clock that their power
// leaves (1.75 GHz): the same products from registers reach 1.76 PFLOP/s on
// random operands and 2.46 on zeros.  The products are
// pinned in order, so that what is made beside them stays there.
constexpr int kBigLds = 2 * 512 * 128;
template <bool F16>
__global__ __launch_bounds__(256) void k_product_256(ProductArgs p) {
  constexpr int kStage = 512 * 128;
  extern __shared__ uint8_t lds[];
  const int tid = threadIdx.x, l = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wm = wave >> 1, wn = wave & 1;
  int ti, tj;
  tile_of(p, xcd_remap(blockIdx.x, gridDim.x), &ti, &tj);
  const int64_t i1 = (int64_t)ti * 256, j1 = (int64_t)tj * 256;
  const int64_t i0 = min(i1, p.m - 256), j0 = min(j1, p.n - 256);
  const int x8 = wave * 8 + (l >> 3);
  const uint32_t voff = (uint32_t)x8 * (uint32_t)p.pitch + (((l & 7) ^ swz(x8)) << 4);
  const int rowstep = 32 * (int)p.pitch, klast = (p.kb - 1) * 128;
  const __amdgpu_buffer_rsrc_t qa = buf_rsrc(p.a + i0 * p.pitch, 256 * (uint64_t)p.pitch);
  const __amdgpu_buffer_rsrc_t qb = buf_rsrc(p.b + j0 * p.pitch, 256 * (uint64_t)p.pitch);
  int ks = 0;
  auto dma = [&](int buf, int q) {  // piece q of 16: 32 rows of one operand
    uint8_t* d = lds + buf * kStage + (q * 4 + wave) * 1024;
    __builtin_amdgcn_raw_ptr_buffer_load_lds(q < 8 ? qa : qb, (lds_ptr)d, 16, voff, ks + (q & 7) * rowstep, 0, 0);
  };
  auto stage = [&](int buf) {
#pragma unroll
    for (int q = 0; q < 16; ++q) dma(buf, q);
    ks = min(ks + 128, klast);  // past the end: the last again, never multiplied
  };
  const int r = l & 31, g = l >> 5;
  const uint8_t *pas = p.as + (i0 >> p.a_shift) * p.spitch, *pbs = p.bs + (j0 >> p.b_shift) * p.spitch;
  const int ia = (int)(i0 & ((1 << p.a_shift) - 1)) + wm * 128 + r, ib = (int)(j0 & ((1 << p.b_shift) - 1)) + wn * 128 + r;
  // Four blocks' scales of a lane's rows (one byte each).
  auto scales = [&](int k, int* xa, int* xb) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      xa[i] = *(const int*)(pas + k + (int64_t)((ia + 32 * i) >> p.a_shift) * p.spitch);
      xb[i] = *(const int*)(pbs + k + (int64_t)((ib + 32 * i) >> p.b_shift) * p.spitch);
    }
  };
  f32x16 acc[4][4];
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int j = 0; j < 4; ++j)
#pragma unroll
      for (int e = 0; e < 16; ++e) acc[i][j][e] = 0.0f;
  const int ra = (wm * 128 + r) * 128, rb = (256 + wn * 128 + r) * 128;
  // Pieces 2c + g of a row, c = 0 .. 3, are a lane's 64 codes of a step: eight operands.
  auto piece = [&](const uint8_t* s, int row, int c) { return *(const i32x4*)(s + row + (((2 * c + g) ^ swz(r)) << 4)); };
  int sa[4], sb[4], xa[4], xb[4];
  i32x4 pa[4][4], pb[4][4];  // [row tile][piece]
  i32x4 va[2], vb[2][4];     // operands: a's of this row tile and of the next, b's of this eighth and of the next
  stage(0);
  stage(1);
  scales(0, sa, sb);
  landed();
#pragma unroll
  for (int i = 0; i < 4; ++i) {
#pragma unroll
    for (int c = 0; c < 2; ++c) {
      pa[i][c] = piece(lds, ra + i * 4096, c);
      pb[i][c] = piece(lds, rb + i * 4096, c);
    }
    vb[0][i] = eight_values(half_of(pb[i][0], 0), scale_of_byte(sb[i], 0));
  }
  va[0] = eight_values(half_of(pa[0][0], 0), scale_of_byte(sa[0], 0));
  // na, nb: the words that hold the next step's scales.
  auto step = [&](auto u, auto bc, const int (&na)[4], const int (&nb)[4]) {
    constexpr int U = decltype(u)::value, NU = (U + 1) & 3, BUF = decltype(bc)::value;
    const uint8_t *s = lds + BUF * kStage, *n = lds + (1 - BUF) * kStage;
#pragma unroll
    for (int q = 0; q < 8; ++q) {
      const int nq = (q + 1) & 7;
      if (q == 4) landed();  // the next step's operands; and this step's have been read
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const int slot = 4 * i + j;
          // In the first eighth this step's second half, after the barrier the next step's first.
          if (q == 0) {
            if (slot < 8)
              pb[slot >> 1][2 + (slot & 1)] = piece(s, rb + (slot >> 1) * 4096, 2 + (slot & 1));
            else
              pa[(slot - 8) >> 1][2 + (slot & 1)] = piece(s, ra + ((slot - 8) >> 1) * 4096, 2 + (slot & 1));
          }
          if (q == 4) {
            if (slot < 8)
              pb[slot >> 1][slot & 1] = piece(n, rb + (slot >> 1) * 4096, slot & 1);
            else
              pa[(slot - 8) >> 1][slot & 1] = piece(n, ra + ((slot - 8) >> 1) * 4096, slot & 1);
          }
          if (q == 5) dma(BUF, slot);
          acc[i][j] = product32(vb[q & 1][j], va[i & 1], acc[i][j]);
          vb[nq & 1][i][j] = two_values(half_of(pb[i][nq >> 1], nq), j, q == 7 ? scale_of_byte(nb[i], NU) : scale_of_byte(sb[i], U));
          if (i < 3)
            va[(i + 1) & 1][j] = two_values(half_of(pa[i + 1][q >> 1], q), j, scale_of_byte(sa[i + 1], U));
          else
            va[0][j] = two_values(half_of(pa[0][nq >> 1], nq), j, q == 7 ? scale_of_byte(na[0], NU) : scale_of_byte(sa[0], U));
          __builtin_amdgcn_sched_barrier(0);
        }
    }
    ks = min(ks + 128, klast);
  };
  int k = 0;
  for (; k + 4 <= p.kb; k += 4) {
    scales(min(k + 4, (int)p.spitch - 4), xa, xb);
    step(Int<0>(), Int<0>(), sa, sb);
    step(Int<1>(), Int<1>(), sa, sb);
    step(Int<2>(), Int<0>(), sa, sb);
    step(Int<3>(), Int<1>(), xa, xb);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      sa[i] = xa[i];
      sb[i] = xb[i];
    }
  }
  if (k < p.kb) step(Int<0>(), Int<0>(), sa, sb);
  if (k + 1 < p.kb) step(Int<1>(), Int<1>(), sa, sb);
  if (k + 2 < p.kb) step(Int<2>(), Int<0>(), sa, sb);
  landed();
  // Each wave turns its rows through LDS, 32 at a time, into whole lines of the
  // result; a row's 16-byte pieces are permuted by the row, so that neither side
  // meets a bank twice.
  uint8_t* w = lds + wave * (32 * 256);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
#pragma unroll
    for (int j = 0; j < 4; ++j)
#pragma unroll
      for (int q = 0; q < 4; ++q)
        *(u32x2*)(w + r * 256 + (((4 * j + q) ^ (r & 15)) << 4) + 8 * g) =
            u32x2{pack2<F16>(acc[i][j][4 * q], acc[i][j][4 * q + 1]), pack2<F16>(acc[i][j][4 * q + 2], acc[i][j][4 * q + 3])};
    __builtin_amdgcn_wave_barrier();
#pragma unroll
    for (int q = 0; q < 8; ++q) {
      const int rr = q * 4 + (l >> 4), cc = (l & 15) * 8;
      const u32x4 v = *(const u32x4*)(w + rr * 256 + (((l & 15) ^ (rr & 15)) << 4));
      const int64_t row = i0 + wm * 128 + 32 * i + rr, col = j0 + wn * 128 + cc;
      if (row >= i1) {
        uint16_t* o = (uint16_t*)p.out + row * p.ldo + col;
        if (col >= j1) {
          __builtin_memcpy(o, &v, 16);
        } else {
#pragma unroll
          for (int e = 0; e < 8; ++e)
            if (col + e >= j1) o[e] = (uint16_t)(v[e >> 1] >> (16 * (e & 1)));
        }
      }
    }
    __builtin_amdgcn_wave_barrier();
  }
}

// Ordinary products: 128 x 128 outputs, four waves of 64 x 64, two buffers of
// 256 rows, so that two workgroups share a CU; codes are read and operands made
// under the products before, as in the large ones.  The contraction may be split
// (p.splits): float32 partial sums, which k_product_sum adds in order.
constexpr int kMidLds = 2 * 256 * 128;
template <bool F16>
__global__ __launch_bounds__(256, 2) void k_product_128(ProductArgs p) {
  constexpr int kStage = 256 * 128;
  extern __shared__ uint8_t lds[];
  const int tid = threadIdx.x, l = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wm = wave >> 1, wn = wave & 1;
  const int tiles = p.tm * p.tn, w0 = xcd_remap(blockIdx.x, gridDim.x), split = w0 / tiles;
  int ti, tj;
  tile_of(p, w0 - split * tiles, &ti, &tj);
  const int64_t i0 = (int64_t)ti * 128, j0 = (int64_t)tj * 128;
  const int k0 = split * p.cps, k1 = min(k0 + p.cps, p.kb);
  const int ml = (int)min((int64_t)128, p.m - i0) - 1, nl = (int)min((int64_t)128, p.n - j0) - 1;
  const uint8_t *a0 = p.a + i0 * p.pitch + (int64_t)k0 * 128, *b0 = p.b + j0 * p.pitch + (int64_t)k0 * 128;
  uint32_t ga[4], gb[4];  // rows past the last: the last again
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    const int row = (q * 4 + wave) * 8 + (l >> 3), c = ((l & 7) ^ swz(row)) << 4;
    ga[q] = (uint32_t)min(row, ml) * (uint32_t)p.pitch + c;
    gb[q] = (uint32_t)min(row, nl) * (uint32_t)p.pitch + c;
  }
  const __amdgpu_buffer_rsrc_t qa = buf_rsrc(a0, (uint64_t)(ml + 1) * p.pitch - (uint64_t)k0 * 128);
  const __amdgpu_buffer_rsrc_t qb = buf_rsrc(b0, (uint64_t)(nl + 1) * p.pitch - (uint64_t)k0 * 128);
  int ks = 0;
  const int klast = (k1 - 1 - k0) * 128;
  auto stage = [&](int buf) {
    uint8_t* d = lds + buf * kStage + wave * 1024;
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      __builtin_amdgcn_raw_ptr_buffer_load_lds(qa, (lds_ptr)(d + q * 4096), 16, ga[q], ks, 0, 0);
      __builtin_amdgcn_raw_ptr_buffer_load_lds(qb, (lds_ptr)(d + (4 + q) * 4096), 16, gb[q], ks, 0, 0);
    }
    ks = min(ks + 128, klast);  // past the end: the last again, never multiplied
  };
  const int r = l & 15, g = l >> 4;
  const uint8_t *sa[4], *sb[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    sa[i] = p.as + (min(i0 + wm * 64 + 16 * i + r, p.m - 1) >> p.a_shift) * p.spitch;
    sb[i] = p.bs + (min(j0 + wn * 64 + 16 * i + r, p.n - 1) >> p.b_shift) * p.spitch;
  }
  f32x4 acc[4][4];
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int j = 0; j < 4; ++j) acc[i][j] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
  const int ra = (wm * 64 + r) * 128, rb = (128 + wn * 64 + r) * 128;
  // Pieces g and 4 + g of a row are a lane's 32 codes of a step: four operands.
  auto piece = [&](const uint8_t* s, int row, int c) { return *(const i32x4*)(s + row + (((4 * c + g) ^ swz(r)) << 4)); };
  // Four blocks' scales; the next four are asked for three steps ahead.
  int xa[4], xb[4], na[4], nb[4];
  auto scales = [&](int k) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      na[i] = *(const int*)(sa[i] + k);
      nb[i] = *(const int*)(sb[i] + k);
    }
  };
  scales(k0);
  stage(0);
  stage(1);
  i32x4 pa[4][2], pb[4][2];  // [row tile][piece]
  i32x4 va[2], vb[2][4];     // operands: a's of this row tile and of the next, b's of this quarter and of the next
  asm volatile("s_waitcnt vmcnt(8)" ::: "memory");  // all but the second stage
  __syncthreads();
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    pa[i][0] = piece(lds, ra + i * 2048, 0);
    pb[i][0] = piece(lds, rb + i * 2048, 0);
    vb[0][i] = eight_values(half_of(pb[i][0], 0), scale_of_byte(nb[i], 0));
  }
  va[0] = eight_values(half_of(pa[0][0], 0), scale_of_byte(na[0], 0));
  auto step = [&](auto u, int k, const int (&wa)[4], const int (&wb)[4]) {  // wa, wb: the next step's scales
    constexpr int U = decltype(u)::value, NU = (U + 1) & 3, C = U & 1;
    if (k >= k1) return;
    const uint8_t *s = lds + C * kStage, *n = lds + (1 - C) * kStage;
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const int nq = (q + 1) & 3;
      if (q == 2) {
        landed();  // the next step's operands; and this step's have been read
        stage(C);
      }
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          if ((q & 1) == 0 && j == 0) {  // this step's second pieces, after the barrier the next step's first
            const int c = q == 0 ? 1 : 0;
            pb[i][c] = piece(q == 0 ? s : n, rb + i * 2048, c);
            pa[i][c] = piece(q == 0 ? s : n, ra + i * 2048, c);
          }
          acc[i][j] = product16(vb[q & 1][j], va[i & 1], acc[i][j]);
          vb[nq & 1][i][j] = two_values(half_of(pb[i][nq >> 1], nq), j, q == 3 ? scale_of_byte(wb[i], NU) : scale_of_byte(xb[i], U));
          if (i < 3)
            va[(i + 1) & 1][j] = two_values(half_of(pa[i + 1][q >> 1], q), j, scale_of_byte(xa[i + 1], U));
          else
            va[0][j] = two_values(half_of(pa[0][nq >> 1], nq), j, q == 3 ? scale_of_byte(wa[0], NU) : scale_of_byte(xa[0], U));
          __builtin_amdgcn_sched_barrier(0);
        }
    }
  };
  for (int k = k0; k < k1; k += 4) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      xa[i] = na[i];
      xb[i] = nb[i];
    }
    if (k + 4 < k1) scales(k + 4);
    step(Int<0>(), k, xa, xb);
    step(Int<1>(), k + 1, xa, xb);
    step(Int<2>(), k + 2, xa, xb);
    step(Int<3>(), k + 3, na, nb);
  }
  landed();
  if (p.splits > 1) {
    float* o = p.part + (int64_t)split * p.m * p.n;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int64_t row = i0 + wm * 64 + 16 * i + r;
      if (row >= p.m) continue;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int64_t col = j0 + wn * 64 + 16 * j + 4 * g;
        if (col + 4 <= p.n) {
          __builtin_memcpy(o + row * p.n + col, &acc[i][j], 16);
        } else {
#pragma unroll
          for (int e = 0; e < 4; ++e)
            if (col + e < p.n) o[row * p.n + col + e] = acc[i][j][e];
        }
      }
    }
    return;
  }
  // Each wave's 64 x 64 through its quarter of LDS (rows of 128 + 16 bytes).
  uint8_t* w = lds + wave * (64 * 144);
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int j = 0; j < 4; ++j)
      *(u32x2*)(w + (16 * i + r) * 144 + (16 * j + 4 * g) * 2) =
          u32x2{pack2<F16>(acc[i][j][0], acc[i][j][1]), pack2<F16>(acc[i][j][2], acc[i][j][3])};
  __builtin_amdgcn_wave_barrier();
#pragma unroll
  for (int q = 0; q < 8; ++q) {
    const int rr = q * 8 + (l >> 3), cc = (l & 7) * 8;
    const u32x4 v = *(const u32x4*)(w + rr * 144 + cc * 2);
    const int64_t row = i0 + wm * 64 + rr, col = j0 + wn * 64 + cc;
    if (row < p.m) {
      uint16_t* o = (uint16_t*)p.out + row * p.ldo + col;
      if (col + 8 <= p.n) {
        __builtin_memcpy(o, &v, 16);
      } else {
#pragma unroll
        for (int e = 0; e < 8; ++e)
          if (col + e < p.n) o[e] = (uint16_t)(v[e >> 1] >> (16 * (e & 1)));
      }
    }
  }
}

// Few rows on one side (a token, or up to 32): b here is the long operand (a's
// and b's places exchanged by the caller with `swap`), whose bytes are the
// time.  Four waves share 16 of its rows, each takes every fourth group of four
// blocks (512 bytes of a row), straight into registers, the next group's loads
// in flight; their sums meet in LDS.  1 x 16384 x 4096: 19 to 21 us, 3.4 TB/s.  (Tiles
// for 32 rows: 32 x 4096 x 4096 13.5 against 8.5 us, 32 x 16384 x 4096 22 against 30.)
template <int MT, bool F16>
__global__ __launch_bounds__(256) void k_product_few(ProductArgs p) {
  __shared__ f32x4 sums[4][MT][64];
  const int tid = threadIdx.x, l = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int r = l & 15, g = l >> 4;
  const int split = blockIdx.x / p.tn, tj = blockIdx.x - split * p.tn;
  const int64_t j0 = (int64_t)tj * 16;
  const int k0 = split * p.cps, k1 = min(k0 + p.cps, p.kb);
  const int64_t j = min(j0 + r, p.n - 1);
  const uint8_t* pb = p.b + j * p.pitch + 16 * g;
  const uint8_t* sb = p.bs + (j >> p.b_shift) * p.spitch;
  const uint8_t *pa[MT], *sa[MT];
#pragma unroll
  for (int i = 0; i < MT; ++i) {
    const int64_t row = min((int64_t)16 * i + r, p.m - 1);
    pa[i] = p.a + row * p.pitch + 16 * g;
    sa[i] = p.as + (row >> p.a_shift) * p.spitch;
  }
  f32x4 acc[MT];
#pragma unroll
  for (int i = 0; i < MT; ++i) acc[i] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
  // A group's blocks past the end read the last block (whose products are left out).
  i32x4 x[8];
  int xs = 0;
  auto load = [&](int k) {
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const int64_t o = (int64_t)min(k + u, p.kb - 1) * 128;
      x[2 * u] = *(const i32x4*)(pb + o);
      x[2 * u + 1] = *(const i32x4*)(pb + o + 64);
    }
    xs = *(const int*)(sb + k);
  };
  int k = k0 + 4 * wave;
  if (k < k1) load(k);
  for (; k < k1; k += 16) {
    i32x4 b[8];
#pragma unroll
    for (int u = 0; u < 8; ++u) b[u] = x[u];
    const int bs = xs;
    if (k + 16 < k1) load(k + 16);
    i32x4 a[MT][8];
    int as[MT];
#pragma unroll
    for (int i = 0; i < MT; ++i) {
      as[i] = *(const int*)(sa[i] + k);
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        const int64_t o = (int64_t)min(k + u, p.kb - 1) * 128;
        a[i][2 * u] = *(const i32x4*)(pa[i] + o);
        a[i][2 * u + 1] = *(const i32x4*)(pa[i] + o + 64);
      }
    }
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      if (k + u >= k1) break;
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const i32x4 vb = eight_values(half_of(b[2 * u + (q >> 1)], q), scale_of_byte(bs, u));
#pragma unroll
        for (int i = 0; i < MT; ++i)
          acc[i] = product16(vb, eight_values(half_of(a[i][2 * u + (q >> 1)], q), scale_of_byte(as[i], u)), acc[i]);
      }
    }
  }
#pragma unroll
  for (int i = 0; i < MT; ++i) sums[wave][i][l] = acc[i];
  __syncthreads();
  for (int i = wave; i < MT; i += 4) {
    f32x4 v = sums[0][i][l];
#pragma unroll
    for (int q = 1; q < 4; ++q) {
      const f32x4 w = sums[q][i][l];
#pragma unroll
      for (int e = 0; e < 4; ++e) v[e] += w[e];
    }
    const int64_t row = 16 * i + r, col = j0 + 4 * g;
    if (row >= p.m) continue;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      if (col + e >= p.n) break;
      // the result's row and column: exchanged where the operands are
      const int64_t orow = p.swap ? col + e : row, ocol = p.swap ? row : col + e;
      if (p.splits > 1)
        p.part[(int64_t)split * p.m * p.n + orow * (p.swap ? p.m : p.n) + ocol] = v[e];
      else
        ((uint16_t*)p.out)[orow * p.ldo + ocol] = out_bits<F16>(v[e]);
    }
  }
}

// The splits' partial sums added in order: four columns of a row a thread.
template <bool F16>
__global__ __launch_bounds__(256) void k_product_sum(const float* part, int splits, int64_t m, int64_t n, uint16_t* out,
                                                     int64_t ldo) {
  const int64_t quads = (n + 3) / 4, total = m * quads, mn = m * n;
  for (int64_t e = (int64_t)blockIdx.x * 256 + threadIdx.x; e < total; e += (int64_t)gridDim.x * 256) {
    const int64_t row = e / quads, col = 4 * (e - row * quads);
    const float* p = part + row * n + col;
    uint16_t* o = out + row * ldo + col;
    if (col + 4 <= n) {
      f32x4 v;
      __builtin_memcpy(&v, p, 16);
#pragma unroll 4
      for (int s = 1; s < splits; ++s) {
        f32x4 w;
        __builtin_memcpy(&w, p + s * mn, 16);
#pragma unroll
        for (int q = 0; q < 4; ++q) v[q] += w[q];
      }
      const u32x2 r = {pack2<F16>(v[0], v[1]), pack2<F16>(v[2], v[3])};
      __builtin_memcpy(o, &r, 8);
    } else {
      for (int64_t q = 0; col + q < n; ++q) {
        float v = p[q];
        for (int s = 1; s < splits; ++s) v += p[s * mn + q];
        o[q] = out_bits<F16>(v);
      }
    }
  }
}

// How a product is taken.
struct Plan {
  int kind;  // 0: few rows, 1: 128 x 128, 2: 256 x 256
  int mt;    // few rows: 16-row tiles
  int splits, cps;
};
constexpr int kFewRows = 32;

Plan plan_product(int64_t m, int64_t n, int64_t k) {
  Plan p{};
  const int64_t kb = code_pitch(k) / kBlock, units = (kb + 3) / 4;
  auto split = [&](int64_t want, int64_t least) {
    const int64_t s = std::max<int64_t>(1, std::min(want, units / least));
    p.cps = (int)(4 * ((units + s - 1) / s));
    p.splits = (int)((kb + p.cps - 1) / p.cps);
  };
  const int64_t few = std::min(m, n), many = std::max(m, n);
  if (few <= kFewRows) {
    p.kind = 0;
    p.mt = few <= 16 ? 1 : 2;
    // 512 workgroups, each wave at least two groups of blocks
    split(512 / ((many + 15) / 16), 8);
    return p;
  }
  const int64_t t128 = (m + 127) / 128 * ((n + 127) / 128), t256 = (m + 255) / 256 * ((n + 255) / 256);
  // Rounds of workgroups over 256 CUs (two of the small tiles on each) at the
  // rates that full rounds reach: 1.59 and 1.41 PFLOP/s (2000 x 3000 x 5000, 96
  // large tiles or 384 small ones: 97 against 60 us; 8192^3 691 against 781).  The
  // length of the contraction does not matter (8192 x 8192 x 128: 42.8 against
  // 42.7; 1024 x 150528 x 256 137 against 146).
  const double c256 = (double)((t256 + 255) / 256) * 256 * 65536 / 1.59, c128 = (double)((t128 + 511) / 512) * 512 * 16384 / 1.41;
  p.kind = m >= 256 && n >= 256 && c256 <= c128 ? 2 : 1;
  p.splits = 1;
  p.cps = (int)round_up(kb, 4);
  if (p.kind == 1) split(256 / t128, 2);
  return p;
}

template <bool F16>
int launch_product(hipStream_t s, ProductArgs p, const Plan& pl) {
  const int64_t m = p.m, n = p.n;
  if (pl.kind == 0) {
    if (m > n) {  // the long operand in b's place
      p.swap = 1;
      std::swap(p.a, p.b);
      std::swap(p.as, p.bs);
      std::swap(p.a_shift, p.b_shift);
      std::swap(p.m, p.n);
    }
    p.tn = (int)((p.n + 15) / 16);
    const int64_t grid = (int64_t)p.tn * pl.splits;
    if (grid > kMaxGroups) return invalid("the product has too many tiles");
    if (pl.mt == 1)
      launch(k_product_few<1, F16>, (unsigned)grid, 256, 0, s, p);
    else
      launch(k_product_few<2, F16>, (unsigned)grid, 256, 0, s, p);
  } else {
    const int t = pl.kind == 2 ? 256 : 128;
    const int64_t tm = (m + t - 1) / t, tn = (n + t - 1) / t;
    if (tm * tn * pl.splits > kMaxGroups) return invalid("the product has too many tiles");
    p.tm = (int)tm;
    p.tn = (int)tn;
    const unsigned grid = (unsigned)(tm * tn * pl.splits);
    if (pl.kind == 2) {
      // more LDS than a kernel gets unasked
      const hipError_t e = hipFuncSetAttribute((const void*)k_product_256<F16>, hipFuncAttributeMaxDynamicSharedMemorySize, kBigLds);
      if (e != hipSuccess) {
        set_error(std::string("hieravg_block_product: ") + hipGetErrorString(e));
        return HIERAVG_EHIP;
      }
      launch(k_product_256<F16>, grid, 256, kBigLds, s, p);
    } else {
      launch(k_product_128<F16>, grid, 256, kMidLds, s, p);
    }
  }
  if (pl.splits > 1) {
    const int64_t quads = m * ((n + 3) / 4);
    launch(k_product_sum<F16>, (unsigned)std::min<int64_t>((quads + 255) / 256, 8192), 256, 0, s, (const float*)p.part,
           pl.splits, m, n, (uint16_t*)p.out, p.ldo);
  }
  return HIERAVG_OK;
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
    if (rows < 0 || cols < 1 || rows > kMostRows || cols > kMostRows)
      return invalid("rows must be in [0, 2^31 - 256], cols in [1, 2^31 - 256]");
    if (row_stride < cols || !addressable(rows, row_stride, type_bytes(type)))
      return invalid("row_stride must be at least cols, the rows within 2^56 bytes");
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
    hipStream_t s = (hipStream_t)hip_stream;
    const bool rows_only = codes && !codes_t && !tiles;
    const int64_t quads = a.spitch / 4, step = rows_only ? 4 * kMaxGroups / quads : rows;
    if (!rows_only && a.ctiles * ((rows + 127) / 128) > kMaxGroups) return invalid("the matrix has too many blocks");
    for (int64_t r0 = 0; r0 < rows; r0 += step) {
      QuantArgs b = a;
      b.rows = std::min(rows - r0, step);
      b.x = (const char*)x + r0 * row_stride * type_bytes(type);
      b.codes = codes ? codes + r0 * a.pitch : nullptr;
      b.scales = scales ? scales + r0 * a.spitch : nullptr;
      const int64_t grid = rows_only ? (b.rows * quads + 3) / 4 : a.ctiles * ((rows + 127) / 128);
#define HAV_QUANT(T_)                                                        \
  do {                                                                       \
    if (rows_only)                                                           \
      launch(k_quantize_rows<T_>, (unsigned)grid, 256, 0, s, b);             \
    else if (tiles)                                                          \
      launch(k_quantize_tile<T_, true>, (unsigned)grid, 256, 0, s, b);       \
    else                                                                     \
      launch(k_quantize_tile<T_, false>, (unsigned)grid, 256, 0, s, b);      \
  } while (0)
      if (type == HIERAVG_F32)
        HAV_QUANT(float);
      else if (type == HIERAVG_F16)
        HAV_QUANT(f16_t);
      else
        HAV_QUANT(bf16_t);
    }
#undef HAV_QUANT
    return launched("hieravg_quantize_blocks");
  });
}

size_t hieravg_block_product_scratch(int64_t m, int64_t n, int64_t k) {
  if (m < 1 || n < 1 || k < 1 || m > kMostRows || n > kMostRows || k > kMaxContraction) return 0;
  const Plan p = plan_product(m, n, k);
  return p.splits > 1 ? sizeof(float) * (size_t)p.splits * (size_t)m * (size_t)n : 0;
}

int hieravg_block_product(const uint8_t* a, const uint8_t* a_scales, int32_t a_tiles, const uint8_t* b,
                          const uint8_t* b_scales, int32_t b_tiles, int64_t m, int64_t n, int64_t k, void* out,
                          int32_t out_type, int64_t out_stride, void* scratch, size_t scratch_bytes,
                          void* hip_stream) {
  return guarded([&]() -> int {
    if (out_type != HIERAVG_F16 && out_type != HIERAVG_BF16)
      return invalid("out_type must be HIERAVG_F16 or HIERAVG_BF16");
    if (m < 0 || n < 0 || k < 1 || m > kMostRows || n > kMostRows || k > kMaxContraction)
      return invalid("m and n must be in [0, 2^31 - 256], k in [1, 2^23]");
    if ((a_tiles != 0 && a_tiles != 1) || (b_tiles != 0 && b_tiles != 1)) return invalid("tiles must be 0 or 1");
    if (out_stride < n || !addressable(m, out_stride, 2))
      return invalid("out_stride must be at least n, the rows within 2^56 bytes");
    if (m == 0 || n == 0) return HIERAVG_OK;
    if (!a || !b || !a_scales || !b_scales || !out) return invalid("NULL operand");
    if (!aligned(a, 16) || !aligned(b, 16) || !aligned(a_scales, 4) || !aligned(b_scales, 4) || !aligned(out, 2))
      return invalid("codes must be aligned to 16 bytes, scales to 4, out to its element");
    const Plan pl = plan_product(m, n, k);
    const size_t need = hieravg_block_product_scratch(m, n, k);
    if (need && (!scratch || scratch_bytes < need || !aligned(scratch, 16)))
      return invalid("scratch must hold hieravg_block_product_scratch bytes, 16-byte aligned");
    hipStream_t s = (hipStream_t)hip_stream;
    ProductArgs p{a, a_scales, b, b_scales, a_tiles ? 7 : 0, b_tiles ? 7 : 0, m, n, code_pitch(k), scale_pitch(k),
                  (int)(code_pitch(k) / kBlock), out, out_stride, 0, 0, (float*)scratch, pl.splits, pl.cps, 0};
    const int rc = out_type == HIERAVG_F16 ? launch_product<true>(s, p, pl) : launch_product<false>(s, p, pl);
    if (rc != HIERAVG_OK) return rc;
    return launched("hieravg_block_product");
  });
}

}  // extern "C"
