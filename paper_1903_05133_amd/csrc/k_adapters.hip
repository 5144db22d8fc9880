// Low-rank adapters of many requests beside a shared projection, and their
// gradient (include/hieravg.h, hieravg_adapter_product, hieravg_adapter_grad).
//
// With D [rank][in] and U [rank][out] of a row's adapter, both with the rank
// outermost, the forward is two products, h = x D^T and y = base + s h U, and
// the backward the same two with their sides exchanged, dh = dy U^T and dx =
// base + s dh D, and the sums over rows s dh^T x and s h^T dy.  So there are
// three kernels: one that contracts a long axis to the rank (k_adapter_down),
// one that expands the rank to a long axis (k_adapter_up), and one that
// contracts the rows (k_adapter_outer).  The rows of an adapter are taken
// together, in tiles of 64: a counting sort by adapter finds them
// (k_adapter_plan), for up to 64 rows a ballot.
//
// Products are float32 MFMAs or those of the operands' own type where both are
// 16-bit, sums are float32.  All three are bound by memory: 2 rank flops for each
// element of x or y.  With 16384 rows, 4096 columns on both sides, rank 64 and bf16
// (420 MB of x, base, y) the kernels take 13.9, 50 to 60 and 67 to 72 us; the
// gradient over 8192 rows 144 us, of it k_adapter_outer 52.
#include <algorithm>
#include <cmath>
#include <type_traits>

#include "ops.h"
#include "split.h"

namespace hav {

namespace {

constexpr int kTileRows = 64;    // rows of a tile, in four sixteens
constexpr int kUnitMost = 4096;  // rows that one workgroup contracts at most
constexpr int kOuterRank = 64;   // and ranks
constexpr int kFewRows = 64;     // up to here the rows of an adapter are found by ballots

// Rows of one adapter: `count` places from `first` in the order by adapter.
// Adapter n: rows without one (id < 0), n + 1: with an id that is none.
// slot: of a unit, where its sums wait for those of the adapter's others; -1: it
// has no others, and the sums are results.
struct Tile {
  int adapter, first, count, slot;
};
// An adapter with several units, and its slots.
struct Join {
  int adapter, first, count, pad;
};
struct RowPlan {
  const void* ids;
  int id_bytes, n;
  int64_t rows;
  int32_t* order;  // rows by adapter, or NULL: few rows
  Tile *tiles, *units;
  Join* joins;
  int tile_most, unit_most, join_most, unit_rows;
};

__device__ inline int bin_of(const RowPlan& p, int64_t id) { return id < 0 ? p.n : id >= p.n ? p.n + 1 : (int)id; }

// ------------------------------------------------------------ rows by adapter
// One workgroup: counts of each adapter's rows by waves, each over rows of its
// own, places from the sums of the counts before, then each wave puts its rows
// there.  Equal ids of a wave's 64 rows are found by ballots, a round for each
// id among them, so the runs of requests take one or two rounds; the first lane of
// each id counts for all of them.  The order is the rows' own within an adapter.
// 777 rows 6.5 us, 16384 13.3: one CU's ballots and LDS round trips, a wave's
// sixteen sixty-fours one after the other.
// several: slots, and from bit 16 on joins; at most 8191 (a unit has 4096 of 2^24 rows,
// or fewer where there are 1022 units at most) and 4095.
struct Counts {
  int rows, tiles, units, several;
};
__device__ inline Counts operator+(const Counts& a, const Counts& b) {
  return {a.rows + b.rows, a.tiles + b.tiles, a.units + b.units, a.several + b.several};
}

// I: the ids' type (a branch on it between loads would wait for each).  UNITS: of a
// gradient, whose units and joins are made too (8192 rows 11.4 us).
template <class I, bool UNITS>
__global__ __launch_bounds__(1024) void k_adapter_plan(RowPlan p, int waves) {
  extern __shared__ int counts[];  // [waves][bins]
  __shared__ Counts sums[16];
  constexpr int U = 16;  // sixty-fours of rows under way
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, bins = p.n + 2;
  const int each = (int)((p.rows + waves - 1) / waves + 63) / 64 * 64, rows = (int)p.rows;
  const int r0 = min(wave * each, rows), r1 = wave < waves ? min(r0 + each, rows) : r0;
  int* own = counts + wave * bins;
  for (int i = tid; i < waves * bins; i += 1024) counts[i] = 0;
  if (UNITS)  // those that there are come some barriers later
    for (int i = tid; i < p.join_most; i += 1024) p.joins[i] = {-1, 0, 0, 0};
  // The bins of U sixty-fours, and for each lane those that have its own.
  int bin[U];
  uint64_t alike[U];
  auto take = [&](int from) {
    I id[U];
#pragma unroll
    for (int i = 0; i < U; ++i) id[i] = ((const I*)p.ids)[min(from + i * 64 + lane, r1 - 1)];
#pragma unroll
    for (int i = 0; i < U; ++i) {
      bin[i] = -1;
      alike[i] = 0;
      if (from + i * 64 >= r1) continue;  // none of the wave
      bin[i] = from + i * 64 + lane < r1 ? bin_of(p, (int64_t)id[i]) : -1;
      uint64_t mine = 0, left = __ballot(bin[i] >= 0);
      while (left) {
        const uint64_t with = __ballot(bin[i] == __builtin_amdgcn_readlane(bin[i], __ffsll((unsigned long long)left) - 1));
        if (with >> lane & 1) mine = with;
        left &= ~with;
      }
      alike[i] = mine;
    }
  };
  const uint64_t before = (1ull << lane) - 1;
  __syncthreads();
  for (int from = r0; from < r1; from += U * 64) {
    take(from);
#pragma unroll
    for (int i = 0; i < U; ++i)
      if (alike[i] && !(alike[i] & before)) atomicAdd(&own[bin[i]], (int)__popcll(alike[i]));
  }
  __syncthreads();
  // Places, tiles, units and slots before each bin: a thread has consecutive bins.
  const int per = (bins + 1023) / 1024, b0 = min(tid * per, bins), b1 = min(b0 + per, bins);
  auto counts_of = [&](int b, int (&c)[16]) {
    int all = 0;
#pragma unroll
    for (int w = 0; w < 16; ++w) {
      c[w] = w < waves ? counts[w * bins + b] : 0;
      all += c[w];
    }
    return all;
  };
  auto tiles_of = [&](int b, int c) {
    Counts t{c, (c + kTileRows - 1) / kTileRows, 0, 0};
    if (UNITS && b < p.n) {
      t.units = max(1, (c + p.unit_rows - 1) / p.unit_rows);
      t.several = t.units > 1 ? t.units | 1 << 16 : 0;
    }
    return t;
  };
  Counts mine{0, 0, 0, 0};
  int n[16];
  for (int b = b0; b < b1; ++b) mine = mine + tiles_of(b, counts_of(b, n));
  Counts run = mine;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const Counts up{__shfl_up(run.rows, o, 64), __shfl_up(run.tiles, o, 64), __shfl_up(run.units, o, 64), __shfl_up(run.several, o, 64)};
    if (lane >= o) run = run + up;
  }
  if (lane == 63) sums[wave] = run;
  __syncthreads();
  Counts at{run.rows - mine.rows, run.tiles - mine.tiles, run.units - mine.units, run.several - mine.several}, all{0, 0, 0, 0};
#pragma unroll
  for (int w = 0; w < 16; ++w) {
    const Counts s = sums[w];
    if (w < wave) at = at + s;
    all = all + s;
  }
  // the tiles of one adapter by a wave, which takes its lanes' adapters in turn
  const auto of_lane = [](int v, int l) { return __builtin_amdgcn_readlane(v, l); };
  for (int i = 0; i < per; ++i) {
    const int b = b0 + i;
    const bool in = b < b1;
    const int c = in ? counts_of(b, n) : 0;
    const Counts t = in ? tiles_of(b, c) : Counts{0, 0, 0, 0};
    for (uint64_t left = __ballot(t.tiles + t.units > 0); left; left &= left - 1) {
      const int l = __ffsll((unsigned long long)left) - 1;
      const int bl = of_lane(b, l), cl = of_lane(c, l), tiles = of_lane(t.tiles, l), units = of_lane(t.units, l);
      const int row = of_lane(at.rows, l), tile = of_lane(at.tiles, l), unit = of_lane(at.units, l), several = of_lane(at.several, l);
      for (int j = lane; j < tiles; j += 64)
        p.tiles[tile + j] = {bl, row + j * kTileRows, min(kTileRows, cl - j * kTileRows), -1};
      for (int j = lane; j < units; j += 64)
        p.units[unit + j] = {bl, row + j * p.unit_rows, max(0, min(p.unit_rows, cl - j * p.unit_rows)), units > 1 ? (several & 0xFFFF) + j : -1};
    }
    if (in) {
      if (t.several) p.joins[at.several >> 16] = {b, at.several & 0xFFFF, t.units, 0};
      int place = at.rows;
#pragma unroll
      for (int w = 0; w < 16; ++w)
        if (w < waves) {
          counts[w * bins + b] = place;
          place += n[w];
        }
    }
    at = at + t;
  }
  for (int i = all.tiles + tid; i < p.tile_most; i += 1024) p.tiles[i] = {0, 0, 0, -1};
  if (UNITS)
    for (int i = all.units + tid; i < p.unit_most; i += 1024) p.units[i] = {-1, 0, 0, -1};
  __syncthreads();
  for (int from = r0; from < r1; from += U * 64) {
    if (r1 - r0 > U * 64) take(from);  // else as they are
    int place[U];
    // a wave's additions to one count are made in their order
#pragma unroll
    for (int i = 0; i < U; ++i) {
      place[i] = 0;
      if (from + i * 64 >= r1) continue;
      if (alike[i] && !(alike[i] & before)) place[i] = atomicAdd(&own[bin[i]], (int)__popcll(alike[i]));
    }
#pragma unroll
    for (int i = 0; i < U; ++i) {
      if (from + i * 64 >= r1) continue;
      const int first = __shfl(place[i], alike[i] ? __ffsll((unsigned long long)alike[i]) - 1 : 0, 64);
      if (alike[i]) p.order[first + __popcll(alike[i] & before)] = from + i * 64 + lane;
    }
  }
}

// Tile t and its rows (in LDS; places past the count repeat the first), by the whole workgroup.
__device__ inline Tile find_tile(const RowPlan& p, int t, int (&rows)[kTileRows]) {
  const int tid = threadIdx.x, lane = tid & 63;
  Tile tile{0, 0, 0, -1};
  if (p.order) {
    tile = p.tiles[t];
    if (tid < kTileRows && tile.count > 0) rows[tid] = p.order[tile.first + (tid < tile.count ? tid : 0)];
  } else {
    int bin = -1;
    if (lane < p.rows)
      bin = bin_of(p, p.id_bytes == 8 ? ((const int64_t*)p.ids)[lane] : (int64_t)((const int32_t*)p.ids)[lane]);
    uint64_t left = __ballot(bin >= 0);
    for (; left; --t) {
      const int b = __builtin_amdgcn_readlane(bin, __ffsll((unsigned long long)left) - 1);
      const uint64_t with = __ballot(bin == b);
      if (t == 0) {
        const int first = __ffsll((unsigned long long)with) - 1;
        tile = {b, 0, (int)__popcll(with), -1};
        if (tid < 64) {
          const int rank = __popcll(with & ((1ull << lane) - 1));
          if (with >> lane & 1) rows[rank] = lane;
          if (lane >= tile.count) rows[lane] = first;
        }
        break;
      }
      left &= ~with;
    }
  }
  __syncthreads();
  return tile;
}

// ------------------------------------------------------------ a long axis to the rank
// A workgroup takes a tile's rows over a part of the axis, its waves every
// fourth step of it; 16x16 products of rows and ranks, whose operands a lane
// loads as 16 bytes of a row.  The waves' sums are joined in LDS.  16384 x 4096
// bf16 at rank 64: 50 to 60 us (2.2 to 2.7 TB/s of x, and as much of the weights
// from the L2); x alone takes 49, the weights alone 30.  Measured and not kept:
// three and four steps in flight in registers at one workgroup a CU (54 to 65),
// x past the caches (58).
template <class T>
struct Frag;
template <>
struct Frag<float> {
  static constexpr int E = 4;
  f32x4 v;
};
template <>
struct Frag<f16_t> {
  static constexpr int E = 8;
  f16x8 v;
};
template <>
struct Frag<bf16_t> {
  static constexpr int E = 8;
  bf16x8 v;
};
__device__ inline f32x4 product(const Frag<float>& a, const Frag<float>& b, f32x4 c) {
#pragma unroll
  for (int e = 0; e < 4; ++e) c = __builtin_amdgcn_mfma_f32_16x16x4f32(a.v[e], b.v[e], c, 0, 0, 0);
  return c;
}
__device__ inline f32x4 product(const Frag<f16_t>& a, const Frag<f16_t>& b, f32x4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_f16(a.v, b.v, c, 0, 0, 0);
}
__device__ inline f32x4 product(const Frag<bf16_t>& a, const Frag<bf16_t>& b, f32x4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a.v, b.v, c, 0, 0, 0);
}
// C elements of a row of `len` from n0 on, zeros from its end on, without a branch
// (which would wait for the loads before it): where they do not all lie in the
// row its last C, shifted down.  SMALL: rows shorter than C, one by one.
template <int N>
struct Words {
  uint32_t w[N];
};
template <int N>
__device__ inline void shift_down(Words<N>& v, int bits) {
#pragma unroll
  for (int by = N / 2; by >= 1; by /= 2)
#pragma unroll
    for (int i = 0; i < N; ++i) v.w[i] = bits & (32 * by) ? (i + by < N ? v.w[i + by] : 0) : v.w[i];
  const int rest = bits & 31;
#pragma unroll
  for (int i = 0; i < N; ++i) v.w[i] = __builtin_amdgcn_alignbit(i + 1 < N ? v.w[i + 1] : 0, v.w[i], rest);
#pragma unroll
  for (int i = 0; i < N; ++i) v.w[i] = bits >= 32 * N ? 0 : v.w[i];
}
enum Ends { kWhole, kEnd, kSmall };
template <Ends M, class O, int C>
__device__ inline Pack<O, C> load_row(const O* row, int64_t n0, int64_t len) {
  if (M == kWhole) return load_pack<O, C>(row + n0);
  if (M == kSmall) {
    Pack<O, C> x{};
#pragma unroll
    for (int e = 0; e < C; ++e)
      if (n0 + e < len) x.v[e] = row[n0 + e];
    return x;
  }
  constexpr int N = C * sizeof(O) / 4;
  const int64_t from = min(n0, len - C);
  const Pack<O, C> p = load_pack<O, C>(row + from);
  Words<N> v;
  __builtin_memcpy(&v, &p, sizeof(v));
  shift_down(v, (int)min(int64_t(C), n0 - from) * 8 * (int)sizeof(O));
  Pack<O, C> x;
  __builtin_memcpy(&x, &v, sizeof(v));
  return x;
}
template <Ends M, class T>
__device__ inline Frag<T> load_frag(const T* row, int64_t k, int64_t n) {
  const Pack<T, Frag<T>::E> p = load_row<M, T, Frag<T>::E>(row, k, n);
  Frag<T> f;
  __builtin_memcpy(&f, &p, sizeof(p));
  return f;
}

// Ranks that the kernels are made for, and the length of a row of h in memory.
// Rows too short for one load of a lane are taken by the last kernels alone.
constexpr int kSmallRow = 8;
int padded(const hieravg_adapters& w) {
  if (w.in < kSmallRow || w.out < kSmallRow) return 128;
  return w.rank <= 16 ? 16 : w.rank <= 32 ? 32 : w.rank <= 64 ? 64 : 128;
}

struct DownArgs {
  RowPlan plan;
  const void* x;   // [rows], x_stride apart
  const void* w;   // [n][rank][len]
  float* h;        // [splits][rows][padded], the last rank again behind it
  int64_t x_stride, len;
  int rank, splits;
  int64_t part;    // of the axis, a multiple of a workgroup's step
};

// Steps of a wave whose loads go out together: as many as registers allow.
constexpr int steps_of(int r16) { return r16 <= 16 ? 4 : r16 <= 64 ? 2 : 1; }

// S sixteens of rows.  No branch stands between loads, which would wait for
// those before it: rows past the tile's repeat its first, ranks past the last the
// last, and what is left of the axis after whole steps has a loop of its own.
template <class T, int RT, int S>
__device__ inline void contract(const DownArgs& a, const Tile& tile, const int (&rows)[kTileRows], int split,
                                float (&sums)[4][16][RT * 16]) {
  constexpr int E = Frag<T>::E, U = steps_of(RT * 16), STEP = 4 * E * U, R16 = RT * 16;
  const T* w = (const T*)a.w + (int64_t)tile.adapter * a.rank * a.len;
  const int64_t k0 = split * a.part, k1 = min(k0 + a.part, a.len);
  f32x4 acc[S][RT];
#pragma unroll
  for (int s = 0; s < S; ++s)
#pragma unroll
    for (int r = 0; r < RT; ++r) acc[s][r] = f32x4{0, 0, 0, 0};
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, l16 = lane & 15, g = lane >> 4;
  const T* xr[S];
  const T* wr[RT];
#pragma unroll
  for (int s = 0; s < S; ++s) xr[s] = (const T*)a.x + (int64_t)rows[s * 16 + l16] * a.x_stride;
#pragma unroll
  for (int r = 0; r < RT; ++r) wr[r] = w + (int64_t)min(r * 16 + l16, a.rank - 1) * a.len;
  int64_t k = k0 + wave * STEP;
  for (; k < k1 && k + STEP <= a.len; k += 4 * STEP) {
    Frag<T> wf[U][RT], xf[U][S];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int64_t at = k + u * 4 * E + g * E;
#pragma unroll
      for (int s = 0; s < S; ++s) xf[u][s] = load_frag<kWhole, T>(xr[s], at, 0);
#pragma unroll
      for (int r = 0; r < RT; ++r) wf[u][r] = load_frag<kWhole, T>(wr[r], at, 0);
    }
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int s = 0; s < S; ++s)
#pragma unroll
        for (int r = 0; r < RT; ++r) acc[s][r] = product(xf[u][s], wf[u][r], acc[s][r]);
  }
  auto rest = [&](auto ends) {
    constexpr Ends M = decltype(ends)::value;
    for (int u = 0; u < U && k + u * 4 * E < a.len; ++u) {
      const int64_t at = k + u * 4 * E + g * E;
      Frag<T> wf[RT], xf[S];
#pragma unroll
      for (int s = 0; s < S; ++s) xf[s] = load_frag<M, T>(xr[s], at, a.len);
#pragma unroll
      for (int r = 0; r < RT; ++r) wf[r] = load_frag<M, T>(wr[r], at, a.len);
#pragma unroll
      for (int s = 0; s < S; ++s)
#pragma unroll
        for (int r = 0; r < RT; ++r) acc[s][r] = product(xf[s], wf[r], acc[s][r]);
    }
  };
  if (k < k1) {
    if (RT < 8 || a.len >= E)
      rest(std::integral_constant<Ends, kEnd>{});
    else
      rest(std::integral_constant<Ends, RT < 8 ? kEnd : kSmall>{});
  }
  // the waves' sums, sixteen rows at a time
  float* h = a.h + (int64_t)split * a.plan.rows * R16;
#pragma unroll
  for (int s = 0; s < S; ++s) {
    __syncthreads();  // the sums before have been read
#pragma unroll
    for (int r = 0; r < RT; ++r)
#pragma unroll
      for (int i = 0; i < 4; ++i) sums[wave][g * 4 + i][r * 16 + l16] = acc[s][r][i];
    __syncthreads();
    for (int i = threadIdx.x; i < 16 * R16; i += 256) {
      const int m = i / R16, r = i - m * R16;
      if (s * 16 + m < tile.count)
        h[(int64_t)rows[s * 16 + m] * R16 + r] = (sums[0][m][r] + sums[1][m][r]) + (sums[2][m][r] + sums[3][m][r]);
    }
  }
}

template <class T, int RT>
__global__ __launch_bounds__(256, RT == 8 ? 1 : 2) void k_adapter_down(DownArgs a) {
  __shared__ int rows[kTileRows];
  __shared__ float sums[4][16][RT * 16];
  const int t = blockIdx.x / a.splits, split = blockIdx.x - t * a.splits;
  const Tile tile = find_tile(a.plan, t, rows);
  if (tile.count == 0 || tile.adapter >= a.plan.n) return;
  if (tile.count <= 16)
    contract<T, RT, 1>(a, tile, rows, split, sums);
  else if (tile.count <= 32)
    contract<T, RT, 2>(a, tile, rows, split, sums);
  else
    contract<T, RT, 4>(a, tile, rows, split, sums);
}

// ------------------------------------------------------------ the rank to a long axis
struct UpArgs {
  RowPlan plan;
  const float* h;   // [splits][rows][padded]
  const void* w;    // [n][rank][len]
  const float* scales;
  const void* base;  // or NULL
  void* out;
  float* hidden;     // the joined h, or NULL
  int64_t base_stride, out_stride, len;
  int rank, splits, out_type, chunks;
};

// A wave has 16 lanes' 16 bytes of columns, C consecutive ones a lane: C 16x16
// products for some ranks, whose columns are the lanes' first, second, ..., so
// that a lane ends with C consecutive results of four rows.  The weights of a
// wave's columns stay in registers for all rows of the tile; h is in LDS.
//
// bf16: h as its three bf16 parts, whose products are exact.  f16: each row of h
// scaled by a power of two to [2^14, 2^15), in two f16 parts: off by 2^-23 of
// a value or 2^-40 of the row's largest.  float32: as it is, on float32 products.
//
// No branch stands between loads, which would wait for those before it: ranks
// past the last read the last (h is 0 there), rows past the tile's its first,
// and only workgroups at the end of the columns look at each.
// What is written once and not read again here, past the caches' contents
// (16384 rows of 4096 bf16 columns: 72 us, 79 without).
template <class O, int C>
__device__ inline void store_stream(O* p, const Pack<O, C>& x) {
  typedef uint32_t words __attribute__((ext_vector_type(C * sizeof(O) / 4), aligned(sizeof(O))));
  words w;
  __builtin_memcpy(&w, &x, sizeof(x));
  __builtin_nontemporal_store(w, (words*)p);
}
template <bool WHOLE, class O, int C>
__device__ inline void store_row(O* p, int have, const float (&v)[C]) {
  Pack<O, C> x;
#pragma unroll
  for (int e = 0; e < C; ++e) from_f32(v[e], &x.v[e]);
  if (WHOLE || have >= C) {
    store_stream(p, x);
  } else {
#pragma unroll
    for (int e = 0; e < C; ++e)
      if (e < have) p[e] = x.v[e];
  }
}
template <class T, int R16>
struct UpShared;
template <int R16>
struct UpShared<float, R16> {
  // a lane's ranks one after the other: products i take rank i of each quarter
  float h[kTileRows][R16 + 4];
};
template <int R16>
struct UpShared<bf16_t, R16> {
  uint16_t h[3][kTileRows][R16 + 8];
};
template <int R16>
struct UpShared<f16_t, R16> {
  uint16_t h[2][kTileRows][R16 + 8];
  float unscale[kTileRows];
};

// Four threads have a row of h: its ranks q R16 / 4 .. of it, in v.
template <int N, int R16>
__device__ inline void put_rows(UpShared<float, R16>& sh, int m, int q, const float (&v)[N]) {
#pragma unroll
  for (int i = 0; i < N; ++i) sh.h[m][q * N + i] = v[i];
}
template <int N, int R16>
__device__ inline void put_rows(UpShared<bf16_t, R16>& sh, int m, int q, const float (&v)[N]) {
#pragma unroll
  for (int i = 0; i < N; i += 2) {
    const Split2<3> s = split2<3>(v[i], v[i + 1]);
#pragma unroll
    for (int p = 0; p < 3; ++p) *(uint32_t*)&sh.h[p][m][q * N + i] = s.p[p];
  }
}
template <int N, int R16>
__device__ inline void put_rows(UpShared<f16_t, R16>& sh, int m, int q, const float (&v)[N]) {
  uint32_t most = 0;
#pragma unroll
  for (int i = 0; i < N; ++i) most = max(most, __float_as_uint(v[i]) & 0x7FFFFFFFu);
  most = max(most, dpp_u<0xB1>(most));  // over the four lanes
  most = max(most, dpp_u<0x4E>(most));
  // rows below 2^-86 keep 2^-124; NaN and infinities stay so
  const int e = min(100, split_exp(most));
  const float by = __uint_as_float((uint32_t)(e + 127) << 23);
#pragma unroll
  for (int i = 0; i < N; i += 2) {
    const Split2<2> s = split2<2>(v[i] * by, v[i + 1] * by);
#pragma unroll
    for (int p = 0; p < 2; ++p) *(uint32_t*)&sh.h[p][m][q * N + i] = s.p[p];
  }
  if (q == 0) sh.unscale[m] = __uint_as_float((uint32_t)(127 - e) << 23);
}

// The weights of a lane's C columns: 16-bit ones as operands of 32 ranks each
// (eight ranks of eight columns, turned in registers), float32 ones as they are.
template <class T, int R16, int C>
struct UpWeights {
  static constexpr int CHUNKS = (R16 + 31) / 32;
  uint32_t all[CHUNKS][8][C / 2];
  u32x4 f[CHUNKS][C];
  template <Ends M>
  __device__ inline void load(const T* w, int64_t n0, int64_t len, int rank, int g) {
#pragma unroll
    for (int c = 0; c < CHUNKS; ++c)
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const Pack<T, C> p = load_row<M, T, C>(w + (int64_t)min(c * 32 + g * 8 + i, rank - 1) * len, n0, len);
        __builtin_memcpy(&all[c][i], &p, 2 * C);
      }
  }
  __device__ inline void turn() {
#pragma unroll
    for (int c = 0; c < CHUNKS; ++c) {
      const auto& raw = all[c];
#pragma unroll
      for (int j = 0; j < C; ++j)
#pragma unroll
        for (int q = 0; q < 4; ++q)
          f[c][j][q] = __builtin_amdgcn_perm(raw[2 * q + 1][j / 2], raw[2 * q][j / 2], j & 1 ? 0x07060302u : 0x05040100u);
    }
  }
};
template <int R16, int C>
struct UpWeights<float, R16, C> {
  Pack<float, C> f[R16 / 4];
  template <Ends M>
  __device__ inline void load(const float* w, int64_t n0, int64_t len, int rank, int g) {
#pragma unroll
    for (int i = 0; i < R16 / 4; ++i) f[i] = load_row<M, float, C>(w + (int64_t)min(g * (R16 / 4) + i, rank - 1) * len, n0, len);
  }
  __device__ inline void turn() {}
};
template <int R16, int C>
__device__ inline void expand(const UpShared<float, R16>& sh, const UpWeights<float, R16, C>& w, int m, int g, f32x4 (&acc)[C]) {
#pragma unroll
  for (int i = 0; i < R16 / 4; i += 4) {
    const f32x4 h = *(const f32x4*)&sh.h[m][g * (R16 / 4) + i];
#pragma unroll
    for (int k = 0; k < 4; ++k)
#pragma unroll
      for (int j = 0; j < C; ++j) acc[j] = __builtin_amdgcn_mfma_f32_16x16x4f32(h[k], w.f[i + k].v[j], acc[j], 0, 0, 0);
  }
}
// Eight ranks of a row of 32 from c on, zeros past the sixteenth where there are no more.
template <int R16>
__device__ inline u32x4 ranks_of(const uint16_t* row, int c, int g) {
  u32x4 v = *(const u32x4*)(row + c * 32 + (R16 == 16 ? g & 1 : g) * 8);
  if (R16 == 16 && g > 1) v = u32x4{0, 0, 0, 0};
  return v;
}
template <int R16, int C>
__device__ inline void expand(const UpShared<bf16_t, R16>& sh, const UpWeights<bf16_t, R16, C>& w, int m, int g, f32x4 (&acc)[C]) {
#pragma unroll
  for (int c = 0; c < UpWeights<bf16_t, R16, C>::CHUNKS; ++c)
#pragma unroll
    for (int p = 2; p >= 0; --p) {  // the small parts first
      const bf16x8 h = __builtin_bit_cast(bf16x8, ranks_of<R16>(sh.h[p][m], c, g));
#pragma unroll
      for (int j = 0; j < C; ++j)
        acc[j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(h, __builtin_bit_cast(bf16x8, w.f[c][j]), acc[j], 0, 0, 0);
    }
}
template <int R16, int C>
__device__ inline void expand(const UpShared<f16_t, R16>& sh, const UpWeights<f16_t, R16, C>& w, int m, int g, f32x4 (&acc)[C]) {
#pragma unroll
  for (int c = 0; c < UpWeights<f16_t, R16, C>::CHUNKS; ++c)
#pragma unroll
    for (int p = 1; p >= 0; --p) {
      const f16x8 h = __builtin_bit_cast(f16x8, ranks_of<R16>(sh.h[p][m], c, g));
#pragma unroll
      for (int j = 0; j < C; ++j)
        acc[j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(h, __builtin_bit_cast(f16x8, w.f[c][j]), acc[j], 0, 0, 0);
    }
}
template <class T, int R16>
__device__ inline float unscale(const UpShared<T, R16>&, int) {
  return 1.0f;
}
template <int R16>
__device__ inline float unscale(const UpShared<f16_t, R16>& sh, int m) {
  return sh.unscale[m];
}

// h of a thread's ranks, q N .. of row m: the splits' sum.
template <int N>
__device__ inline void load_hidden(const UpArgs& a, int64_t row, int q, float (&v)[N]) {
  constexpr int U = 32 / N;  // splits under way
  const int64_t split = a.plan.rows * (4 * N);
  const float* p = a.h + row * (4 * N) + q * N;
#pragma unroll
  for (int i = 0; i < N; ++i) v[i] = 0.0f;
#pragma unroll 1
  for (int s0 = 0; s0 < a.splits; s0 += U) {
    Pack<float, N> x[U];
#pragma unroll
    for (int u = 0; u < U; ++u) x[u] = load_pack<float, N>(p + min(s0 + u, a.splits - 1) * split);
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int i = 0; i < N; ++i) v[i] += s0 + u < a.splits ? x[u].v[i] : 0.0f;
  }
#pragma unroll
  for (int i = 0; i < N; ++i)
    if (q * N + i >= a.rank) v[i] = 0.0f;
}

template <class T, class O, int R16, int C, Ends M>
__device__ inline void expand_tile(const UpArgs& a, UpShared<T, R16>& sh, const Tile& tile, const int (&rows)[kTileRows], int64_t n0,
                                   bool keep_hidden) {
  constexpr int N = R16 / 4;
  const int tid = threadIdx.x, lane = tid & 63, l16 = lane & 15, g = lane >> 4;
  const int have = (int)max(int64_t(0), min(int64_t(C), a.len - n0)), subs = (tile.count + 15) / 16;
  // the first loads go out together: the weights, the first rows of base, h
  UpWeights<T, R16, C> w;
  w.template load<M>((const T*)a.w + (int64_t)tile.adapter * a.rank * a.len, n0, a.len, a.rank, g);
  Pack<O, C> base[4] = {}, next[4] = {};
  auto load_base = [&](int s, Pack<O, C> (&to)[4]) {
#pragma unroll
    for (int i = 0; i < 4; ++i)
      to[i] = load_row<M, O, C>((const O*)a.base + (int64_t)rows[s * 16 + g * 4 + i] * a.base_stride, n0, a.len);
  };
  if (a.base) load_base(0, base);
  __builtin_amdgcn_sched_barrier(0);
  {
    const int m = tid >> 2, q = tid & 3;
    float v[N];
    load_hidden<N>(a, rows[m], q, v);
    put_rows(sh, m, q, v);
    if (keep_hidden && m < tile.count)
#pragma unroll
      for (int i = 0; i < N; ++i)
        if (q * N + i < a.rank) a.hidden[(int64_t)rows[m] * a.rank + q * N + i] = v[i];
  }
  const float scale = a.scales ? a.scales[tile.adapter] : 1.0f;
  __builtin_amdgcn_sched_barrier(0);
  w.turn();
  __builtin_amdgcn_sched_barrier(0);
  __syncthreads();
#pragma unroll 1
  for (int s = 0; s < subs; ++s) {
    if (a.base && s + 1 < subs) load_base(s + 1, next);
    f32x4 acc[C];
#pragma unroll
    for (int j = 0; j < C; ++j) acc[j] = f32x4{0, 0, 0, 0};
    expand(sh, w, s * 16 + l16, g, acc);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int m = s * 16 + g * 4 + i;
      const float by = scale * unscale(sh, m);
      float v[C];
#pragma unroll
      for (int j = 0; j < C; ++j) v[j] = fmaf(by, acc[j][i], to_f32(base[i].v[j]));
      if (m < tile.count) store_row<M == kWhole, O, C>((O*)a.out + (int64_t)rows[m] * a.out_stride + n0, have, v);
      base[i] = next[i];
    }
  }
}

// T: of the weights, O: of base and out; ranks up to R16; C columns a lane.
// 16384 x 4096 bf16 at rank 64: 67 to 72 us (3.9 TB/s of base and out; 408 with float32
// products and loads behind branches, 81 with plain stores).  Four columns a lane
// take 90, the rows of base two steps ahead no less.
template <class T, class O, int R16, int C>
__global__ __launch_bounds__(256, 2) void k_adapter_up(UpArgs a) {
  __shared__ int rows[kTileRows];
  __shared__ alignas(16) UpShared<T, R16> sh;
  const int t = blockIdx.x / a.chunks, chunk = blockIdx.x - t * a.chunks;
  const Tile tile = find_tile(a.plan, t, rows);
  if (tile.count == 0) return;
  const int tid = threadIdx.x;
  const int64_t n0 = (int64_t)chunk * (64 * C) + (tid >> 6) * (16 * C) + (tid & 15) * C;
  if (tile.adapter < a.plan.n) {
    if ((int64_t)(chunk + 1) * (64 * C) <= a.len)
      expand_tile<T, O, R16, C, kWhole>(a, sh, tile, rows, n0, a.hidden && chunk == 0);
    else if (R16 < 128 || a.len >= C)
      expand_tile<T, O, R16, C, kEnd>(a, sh, tile, rows, n0, a.hidden && chunk == 0);
    else
      expand_tile<T, O, R16, C, R16 < 128 ? kEnd : kSmall>(a, sh, tile, rows, n0, a.hidden && chunk == 0);
    return;
  }
  // rows without an adapter, and with one that is none
  const bool wrong = tile.adapter > a.plan.n;
  if (a.hidden && chunk == 0)
    for (int i = tid; i < tile.count * a.rank; i += 256)
      a.hidden[(int64_t)rows[i / a.rank] * a.rank + i % a.rank] = wrong ? NAN : 0.0f;
  if (!wrong && a.base == a.out) return;
  const int have = (int)max(int64_t(0), min(int64_t(C), a.len - n0));
  for (int m = (tid & 63) >> 4; m < tile.count; m += 4) {
    float v[C];
    Pack<O, C> b{};
    if (a.base) b = load_row<kSmall, O, C>((const O*)a.base + (int64_t)rows[m] * a.base_stride, n0, a.len);
#pragma unroll
    for (int j = 0; j < C; ++j) v[j] = wrong ? NAN : to_f32(b.v[j]);
    store_row<false, O, C>((O*)a.out + (int64_t)rows[m] * a.out_stride + n0, have, v);
  }
}

// ------------------------------------------------------------ over the rows
// The left side of these products, h or dh, by place in the order instead of by
// row, the splits summed: float32 [places][padded] for float32 operands; for 16-bit
// ones the three bf16 parts, [places / 32][part][padded][32 places], so that a
// lane's operand, eight places of a rank, is one load.
struct PlacesArgs {
  const int32_t* order;
  const float* h;  // [splits][rows], h_stride apart
  void* to;
  int64_t rows, h_stride;
  int rank, splits;
};

template <int R16, bool PARTS>
__device__ inline void place_block(const PlacesArgs& a, int64_t block) {
  __shared__ float v[32][R16 + 1];
  const int64_t p0 = block * 32, split = a.rows * a.h_stride;
  // four ranks of a place
  for (int i = threadIdx.x; i < 32 * R16 / 4; i += 256) {
    const int m = i / (R16 / 4), r = (i - m * (R16 / 4)) * 4;
    const bool in = p0 + m < a.rows;
    const float* p = a.h + (int64_t)a.order[in ? p0 + m : 0] * a.h_stride;
    float s[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll 1
    for (int k0 = 0; k0 < a.splits; k0 += 4) {
      float x[4][4];
#pragma unroll
      for (int k = 0; k < 4; ++k)
#pragma unroll
        for (int e = 0; e < 4; ++e) x[k][e] = p[min(k0 + k, a.splits - 1) * split + min(r + e, a.rank - 1)];
#pragma unroll
      for (int k = 0; k < 4; ++k)
#pragma unroll
        for (int e = 0; e < 4; ++e) s[e] += k0 + k < a.splits ? x[k][e] : 0.0f;
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      if (!in || r + e >= a.rank) s[e] = 0.0f;
      if (PARTS)
        v[m][r + e] = s[e];
      else
        ((float*)a.to)[(p0 + m) * R16 + r + e] = s[e];
    }
  }
  if (!PARTS) return;
  __syncthreads();
  uint32_t* to = (uint32_t*)a.to + block * (3 * R16 * 16);
  for (int i = threadIdx.x; i < R16 * 16; i += 256) {
    const int r = i / 16, m = i % 16 * 2;
    const Split2<3> s = split2<3>(v[m][r], v[m + 1][r]);
#pragma unroll
    for (int p = 0; p < 3; ++p) to[p * R16 * 16 + i] = s.p[p];
  }
}
template <int R16, bool PARTS>
__global__ __launch_bounds__(256) void k_adapter_places(PlacesArgs a, PlacesArgs b, int64_t blocks) {
  if ((int64_t)blockIdx.x < blocks)
    place_block<R16, PARTS>(a, blockIdx.x);
  else
    place_block<R16, PARTS>(b, blockIdx.x - blocks);
}

struct OuterArgs {
  const void* h;   // by place
  const void* x;   // [rows], x_stride apart
  void* out;       // [n][rank][len]
  float* parts;    // [slots][rank][len], of the adapters that have several units
  int64_t x_stride, len;
  int chunks;      // workgroups of a unit's columns and ranks, 0: none
};
struct OuterPair {
  RowPlan plan;
  OuterArgs a, b;  // x's and grad's
  const float* scales;
  int rank, out_type, blocks;  // blocks of 64 ranks
};

// Sums of products over a unit's rows: a wave takes every fourth step of them, for
// 16 C columns (C consecutive ones a lane, as in k_adapter_up) and RT sixteens of
// ranks.  Places before the unit's first and behind its last, where a step has
// some, count as zeros on both sides.
template <Ends M, class T, int RT, int R16, int C>
__device__ inline void over_rows(const RowPlan& plan, const OuterArgs& a, const Tile& unit, int q0, int64_t c0, f32x4 (&acc)[RT][C]) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, l16 = lane & 15, g = lane >> 4;
  const int end = unit.first + unit.count, last = end - 1;
  const T* x = (const T*)a.x;
  if constexpr (sizeof(T) == 4) {
    constexpr int U = 4;  // steps of four rows whose loads go out together
    const float* h = (const float*)a.h + q0 + l16;
    for (int p0 = unit.first + wave * 4 * U; p0 < end; p0 += 16 * U) {
      Pack<T, C> xv[U];
      float hv[U][RT];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int p = min(p0 + u * 4 + g, last);
#pragma unroll
        for (int r = 0; r < RT; ++r) hv[u][r] = h[(int64_t)p * R16 + r * 16];
        xv[u] = load_row<M, T, C>(x + (int64_t)plan.order[p] * a.x_stride, c0, a.len);
      }
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const bool in = p0 + u * 4 + g < end;
#pragma unroll
        for (int j = 0; j < C; ++j) xv[u].v[j] = in ? xv[u].v[j] : 0.0f;
#pragma unroll
        for (int r = 0; r < RT; ++r) {
          const float l = in ? hv[u][r] : 0.0f;
#pragma unroll
          for (int j = 0; j < C; ++j) acc[r][j] = __builtin_amdgcn_mfma_f32_16x16x4f32(l, xv[u].v[j], acc[r][j], 0, 0, 0);
        }
      }
    }
  } else {
    const uint16_t* h = (const uint16_t*)a.h + (q0 + l16) * 32 + g * 8;
    int row[8];  // of the lane's eight places, a step ahead
    auto take_rows = [&](int block) {
#pragma unroll
      for (int i = 0; i < 8; ++i) row[i] = plan.order[min(max(block * 32 + g * 8 + i, unit.first), last)];
    };
    take_rows(unit.first / 32 + wave);
    for (int block = unit.first / 32 + wave; block * 32 < end; block += 4) {
      const int p0 = block * 32 + g * 8;
      uint32_t raw[8][C / 2];
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const Pack<T, C> v = load_row<M, T, C>(x + (int64_t)row[i] * a.x_stride, c0, a.len);
        __builtin_memcpy(&raw[i], &v, 2 * C);
      }
      u32x4 l[3][RT];
#pragma unroll
      for (int p = 0; p < 3; ++p)
#pragma unroll
        for (int r = 0; r < RT; ++r) l[p][r] = *(const u32x4*)(h + ((int64_t)block * 3 + p) * (R16 * 32) + r * 512);
      take_rows(block + 4);
      if (block * 32 < unit.first || block * 32 + 32 > end) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const bool in = p0 + i >= unit.first && p0 + i < end;
#pragma unroll
          for (int e = 0; e < C / 2; ++e) raw[i][e] = in ? raw[i][e] : 0;
          const uint32_t keep = in ? 0xFFFFFFFFu : i & 1 ? 0x0000FFFFu : 0xFFFF0000u;
#pragma unroll
          for (int p = 0; p < 3; ++p)
#pragma unroll
            for (int r = 0; r < RT; ++r) l[p][r][i / 2] &= keep;
        }
      }
#pragma unroll
      for (int j = 0; j < C; ++j) {
        u32x4 f;  // column j of the eight rows
#pragma unroll
        for (int q = 0; q < 4; ++q)
          f[q] = __builtin_amdgcn_perm(raw[2 * q + 1][j / 2], raw[2 * q][j / 2], j & 1 ? 0x07060302u : 0x05040100u);
        if constexpr (__is_same(T, bf16_t)) {
#pragma unroll
          for (int p = 2; p >= 0; --p)
#pragma unroll
            for (int r = 0; r < RT; ++r)
              acc[r][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, l[p][r]), __builtin_bit_cast(bf16x8, f),
                                                                  acc[r][j], 0, 0, 0);
        } else {
          // f16 as two bf16 parts, exactly; of their six products with h's parts
          // the least, 2^-24 of the largest, is left out
          u32x4 hi, lo;
#pragma unroll
          for (int q = 0; q < 4; ++q) {
            const uint32_t u = __float_as_uint(to_f32(f16_t{(uint16_t)f[q]})), v = __float_as_uint(to_f32(f16_t{(uint16_t)(f[q] >> 16)}));
            hi[q] = __builtin_amdgcn_perm(v, u, 0x07060302u);
            lo[q] = __builtin_amdgcn_perm(__float_as_uint(__uint_as_float(v) - __uint_as_float(v & 0xFFFF0000u)),
                                          __float_as_uint(__uint_as_float(u) - __uint_as_float(u & 0xFFFF0000u)), 0x07060302u);
          }
          auto add = [&](const u32x4& y, int p) {
#pragma unroll
            for (int r = 0; r < RT; ++r)
              acc[r][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, l[p][r]), __builtin_bit_cast(bf16x8, y),
                                                                  acc[r][j], 0, 0, 0);
          };
          add(lo, 1);
          add(hi, 2);
          add(lo, 0);
          add(hi, 1);
          add(hi, 0);
        }
      }
    }
  }
}

__device__ inline void store_some(void* p, int type, int64_t i, int have, const float (&v)[4]) {
  if (type == HIERAVG_F32)
    have >= 4 ? store_row<true, float, 4>((float*)p + i, 4, v) : store_row<false, float, 4>((float*)p + i, have, v);
  else if (type == HIERAVG_F16)
    have >= 4 ? store_row<true, f16_t, 4>((f16_t*)p + i, 4, v) : store_row<false, f16_t, 4>((f16_t*)p + i, have, v);
  else
    have >= 4 ? store_row<true, bf16_t, 4>((bf16_t*)p + i, 4, v) : store_row<false, bf16_t, 4>((bf16_t*)p + i, have, v);
}

// A workgroup's columns: 16 lanes of 16 bytes.
template <class T>
constexpr int kOuterCols = 256 / sizeof(T);

// Both products over 8192 rows, 2 x 4096 columns and rank 64 in bf16: 52 us in eight
// units (134 MB of x and grad, 200 MB of h's parts from the L2); with 1024 rows a
// unit 63, with four columns a lane 57 to 71.  512 x 1000 and 300, float32: 4.8.
template <class T, int RT, int R16>
__global__ __launch_bounds__(256, 2) void k_adapter_outer(OuterPair o) {
  constexpr int C = 16 / sizeof(T), COLS = 16 * C;
  __shared__ float sums[RT * 16][COLS];
  const int per = o.a.chunks + o.b.chunks, u = blockIdx.x / per;
  int rest = blockIdx.x - u * per;
  const bool second = rest >= o.a.chunks;
  const OuterArgs& a = second ? o.b : o.a;
  if (second) rest -= o.a.chunks;
  const int block = rest % o.blocks, chunk = rest / o.blocks;
  const Tile unit = o.plan.units[u];
  if (unit.adapter < 0) return;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, l16 = lane & 15, g = lane >> 4;
  const int64_t c0 = (int64_t)chunk * COLS;
  f32x4 acc[RT][C];
#pragma unroll
  for (int r = 0; r < RT; ++r)
#pragma unroll
    for (int j = 0; j < C; ++j) acc[r][j] = f32x4{0, 0, 0, 0};
  const int64_t n0 = c0 + l16 * C;
  if (unit.count == 0)
    ;  // an adapter without rows
  else if (c0 + COLS <= a.len)
    over_rows<kWhole, T, RT, R16, C>(o.plan, a, unit, block * kOuterRank, n0, acc);
  else if (R16 < 128 || a.len >= C)
    over_rows<kEnd, T, RT, R16, C>(o.plan, a, unit, block * kOuterRank, n0, acc);
  else
    over_rows<R16 < 128 ? kEnd : kSmall, T, RT, R16, C>(o.plan, a, unit, block * kOuterRank, n0, acc);
  // the waves' sums, one wave after the other
  for (int w = 0; w < 4; ++w) {
    if (wave == w) {
#pragma unroll
      for (int r = 0; r < RT; ++r)
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
          for (int j = 0; j < C; j += 4) {
            f32x4* s = (f32x4*)&sums[r * 16 + g * 4 + i][l16 * C + j];
            const f32x4 v = {acc[r][j][i], acc[r][j + 1][i], acc[r][j + 2][i], acc[r][j + 3][i]};
            *s = w == 0 ? v : *s + v;
          }
    }
    __syncthreads();
  }
  const bool whole = unit.slot < 0;
  const float scale = whole && o.scales ? o.scales[unit.adapter] : 1.0f;
  for (int i = tid; i < RT * 16 * (COLS / 4); i += 256) {
    const int r = i / (COLS / 4), c = (i - r * (COLS / 4)) * 4, q = block * kOuterRank + r;
    const int n = (int)max(int64_t(0), min(int64_t(4), a.len - c0 - c));
    if (q >= o.rank || n == 0) continue;
    float v[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = unit.count ? sums[r][c + e] * scale : 0.0f;
    if (whole)
      store_some(a.out, o.out_type, ((int64_t)unit.adapter * o.rank + q) * a.len + c0 + c, n, v);
    else
      store_some(a.parts, HIERAVG_F32, ((int64_t)unit.slot * o.rank + q) * a.len + c0 + c, n, v);
  }
}

// The units' sums of the adapters that have several, one after the other.
__global__ __launch_bounds__(256) void k_adapter_join(OuterPair o, int64_t groups_a, int64_t groups_b) {
  const int64_t per = groups_a + groups_b, k = blockIdx.x / per;
  int64_t rest = blockIdx.x - k * per;
  const bool second = rest >= groups_a;
  const OuterArgs& a = second ? o.b : o.a;
  if (second) rest -= groups_a;
  const int64_t i = (rest * 256 + threadIdx.x) * 4, size = (int64_t)o.rank * a.len;
  const Join join = o.plan.joins[k];
  if (join.adapter < 0 || i >= size) return;
  const int n = (int)min(int64_t(4), size - i);
  float s[4] = {0.0f, 0.0f, 0.0f, 0.0f};
  const float* p = a.parts + join.first * size + i;
  if (n == 4) {
#pragma unroll 4
    for (int u = 0; u < join.count; ++u) {
      const Pack<float, 4> v = load_pack<float, 4>(p + u * size);
#pragma unroll
      for (int e = 0; e < 4; ++e) s[e] += v.v[e];
    }
  } else {
    for (int u = 0; u < join.count; ++u)
      for (int e = 0; e < n; ++e) s[e] += p[u * size + e];
  }
  const float scale = o.scales ? o.scales[join.adapter] : 1.0f;
#pragma unroll
  for (int e = 0; e < 4; ++e) s[e] *= scale;
  store_some(a.out, o.out_type, join.adapter * size + i, n, s);
}

// ------------------------------------------------------------ host
constexpr int64_t kMostRows = int64_t(1) << 24, kMostCols = int64_t(1) << 24;

int64_t div_up(int64_t a, int64_t b) { return (a + b - 1) / b; }
// Columns of a workgroup that expands: 16 lanes in each of four waves, 16 bytes
// of weights a lane, or 8 where the ranks' are many.
int64_t up_cols(const hieravg_adapters& w) { return 64 * (16 / type_bytes(w.type)) / (padded(w) > 64 ? 2 : 1); }
int64_t tile_count(int64_t rows, int n, bool few) {
  const int64_t bins = (int64_t)n + 2;
  return few ? std::min(rows, bins) : rows / kTileRows + std::min(rows, bins);
}
int64_t outer_cols(int type) { return type == HIERAVG_F32 ? kOuterCols<float> : kOuterCols<bf16_t>; }
// Rows of a unit: as many as leave some 512 workgroups, 64 at least.
int unit_size(int64_t rows, const hieravg_adapters& w) {
  const int64_t chunks = (div_up(w.in, outer_cols(w.type)) + div_up(w.out, outer_cols(w.type))) * div_up(w.rank, kOuterRank);
  int64_t u = kUnitMost;
  while (u > 64 && (div_up(rows, u) + std::min<int64_t>(w.n, rows) / 2) * chunks < 512) u /= 2;
  return (int)u;
}

// How many parts the long axis is taken in: about 512 workgroups, two a CU.
struct Split {
  int splits;
  int64_t part;
};
Split split_axis(int64_t tiles, int64_t len, int type, int r16) {
  const int64_t step = 256 / type_bytes(type) * steps_of(r16);  // of a workgroup's four waves
  const int64_t most = std::min<int64_t>(div_up(len, step), 16);
  const int64_t splits = std::max<int64_t>(1, std::min(most, (560 + tiles / 2) / std::max<int64_t>(tiles, 1)));
  const int64_t part = round_up(div_up(len, splits), step);
  return {(int)div_up(len, part), part};
}

struct AdapterPlan {
  bool few;
  int unit_rows;
  int64_t tiles, units, slots, joins;
  Split down, down2;  // of the rank's products: x D^T or dy U^T; the backward's x D^T
  size_t order, tile, unit, join, h, h2, places, parts, bytes;
};

// h by place, of one of the two products over the rows.
int64_t place_bytes(int64_t rows, const hieravg_adapters& w) {
  return round_up(rows, 32) * padded(w) * (w.type == HIERAVG_F32 ? 4 : 6);
}

// backward: the gradient; weights: in down and up too; hidden: h is given.
AdapterPlan plan_adapters(int64_t rows, const hieravg_adapters& w, bool backward, bool weights, bool hidden) {
  AdapterPlan p{};
  p.few = !backward && rows <= kFewRows;
  p.tiles = tile_count(rows, w.n, p.few);
  p.unit_rows = unit_size(rows, w);
  p.units = weights ? rows / p.unit_rows + w.n : 0;
  // adapters with several units, c > unit_rows rows, and those units, floor(c /
  // unit_rows) + 1 at most of each
  p.joins = weights ? std::min<int64_t>(rows / (p.unit_rows + 1), w.n) : 0;
  p.slots = p.joins ? rows / p.unit_rows + p.joins : 0;
  // tiles that are there, if every adapter has rows
  const int64_t real = std::min(p.tiles, div_up(rows, kTileRows) + std::min<int64_t>(rows, w.n) / 2);
  p.down = split_axis(real, backward ? w.out : w.in, w.type, padded(w));
  p.down2 = weights && !hidden ? split_axis(real, w.in, w.type, padded(w)) : Split{0, 0};
  size_t at = 0;
  auto take = [&](int64_t n) {
    const size_t o = at;
    at += (size_t)round_up(n, 16);
    return o;
  };
  if (!p.few) {
    p.order = take(4 * rows);
    p.tile = take(p.tiles * sizeof(Tile));
  }
  if (weights) {
    p.unit = take(p.units * sizeof(Tile));
    p.join = take(p.joins * sizeof(Join));
  }
  p.h = take(4 * rows * padded(w) * p.down.splits);
  p.h2 = take(4 * rows * padded(w) * p.down2.splits);
  if (weights) p.places = take(2 * place_bytes(rows, w));
  if (p.slots) p.parts = take(4 * p.slots * w.rank * (w.in + w.out));
  p.bytes = at;
  return p;
}

int check_adapters(const hieravg_adapters* w, int64_t rows) {
  if (!w) return invalid("no adapters");
  if (!known_type(w->type)) return invalid("unknown element type");
  if (rows < 0 || rows > kMostRows) return invalid("rows must be in [0, 2^24]");
  if (w->n < 1 || w->n > HIERAVG_ADAPTERS_MAX) return invalid("n must be in [1, HIERAVG_ADAPTERS_MAX]");
  if (w->rank < 1 || w->rank > HIERAVG_RANK_MAX) return invalid("rank must be in [1, HIERAVG_RANK_MAX]");
  if (w->in < 1 || w->in > kMostCols || w->out < 1 || w->out > kMostCols) return invalid("in and out must be in [1, 2^24]");
  return HIERAVG_OK;
}
// float32 beside any type, 16 bits beside float32 and themselves.
bool result_type(int32_t t, int32_t of) { return t == HIERAVG_F32 || t == of || (known_type(t) && of == HIERAVG_F32); }
int check_weights(const hieravg_adapters* w) {
  if (!w->down || !w->up || !aligned(w->down, type_bytes(w->type)) || !aligned(w->up, type_bytes(w->type)))
    return invalid("down and up must be pointers aligned to their element");
  if (w->scales && !aligned(w->scales, 4)) return invalid("scales must be aligned to their element");
  return HIERAVG_OK;
}
int check_rows(const void* p, int type, int64_t rows, int64_t cols, int64_t stride, const char* what) {
  if (stride < cols || !addressable(rows, stride, type_bytes(type))) return invalid(what);
  if (!p || !aligned(p, type_bytes(type))) return invalid(what);
  return HIERAVG_OK;
}
int check_ids(const void* ids, int32_t id_bytes) {
  if (id_bytes != 4 && id_bytes != 8) return invalid("id_bytes must be 4 or 8");
  if (!ids || !aligned(ids, id_bytes)) return invalid("ids must be a pointer aligned to its element");
  return HIERAVG_OK;
}
Area down_area(const hieravg_adapters& w) { return block_area(w.down, int64_t(w.n) * w.rank * w.in * type_bytes(w.type)); }
Area up_area(const hieravg_adapters& w) { return block_area(w.up, int64_t(w.n) * w.rank * w.out * type_bytes(w.type)); }
Area scales_area(const hieravg_adapters& w) { return block_area(w.scales, int64_t(w.n) * 4); }
bool same_rows(const void* a, int64_t as, const void* b, int64_t bs, int64_t rows) { return a == b && (as == bs || rows == 1); }

RowPlan rows_plan(const AdapterPlan& p, char* scratch, const hieravg_adapters& w, const void* ids, int id_bytes, int64_t rows) {
  RowPlan r{};
  r.ids = ids;
  r.id_bytes = id_bytes;
  r.n = w.n;
  r.rows = rows;
  r.tile_most = (int)p.tiles;
  r.unit_most = (int)p.units;
  r.unit_rows = p.unit_rows;
  if (!p.few) {
    r.order = (int32_t*)(scratch + p.order);
    r.tiles = (Tile*)(scratch + p.tile);
  }
  return r;
}
void launch_plan(hipStream_t s, const RowPlan& r) {
  // counts within 60 KB of LDS
  const int bins = r.n + 2, waves = (int)std::max<int64_t>(1, std::min<int64_t>({16, 15360 / bins, div_up(r.rows, 64)}));
  const uint32_t lds = (uint32_t)(waves * bins * sizeof(int));
  if (r.id_bytes == 8)
    launch(r.units ? k_adapter_plan<int64_t, true> : k_adapter_plan<int64_t, false>, 1, 1024, lds, s, r, waves);
  else
    launch(r.units ? k_adapter_plan<int32_t, true> : k_adapter_plan<int32_t, false>, 1, 1024, lds, s, r, waves);
}

template <class T>
void launch_down(hipStream_t s, const DownArgs& a, int r16, int64_t tiles) {
  const unsigned grid = (unsigned)(tiles * a.splits);
  if (r16 == 16)
    launch(k_adapter_down<T, 1>, grid, 256, 0, s, a);
  else if (r16 == 32)
    launch(k_adapter_down<T, 2>, grid, 256, 0, s, a);
  else if (r16 == 64)
    launch(k_adapter_down<T, 4>, grid, 256, 0, s, a);
  else
    launch(k_adapter_down<T, 8>, grid, 256, 0, s, a);
}
template <class T, class O>
void launch_up(hipStream_t s, const UpArgs& a, int r16, int64_t tiles) {
  constexpr int C = sizeof(T) == 4 ? 4 : 8;
  const unsigned grid = (unsigned)(tiles * a.chunks);
  if (r16 == 16)
    launch(k_adapter_up<T, O, 16, C>, grid, 256, 0, s, a);
  else if (r16 == 32)
    launch(k_adapter_up<T, O, 32, C>, grid, 256, 0, s, a);
  else if (r16 == 64)
    launch(k_adapter_up<T, O, 64, C>, grid, 256, 0, s, a);
  else
    launch(k_adapter_up<T, O, 128, C / 2>, grid, 256, 0, s, a);
}
template <class T>
void launch_up(hipStream_t s, const UpArgs& a, int r16, int64_t tiles) {
  if constexpr (sizeof(T) == 4) {
    if (a.out_type == HIERAVG_F32)
      launch_up<T, float>(s, a, r16, tiles);
    else if (a.out_type == HIERAVG_F16)
      launch_up<T, f16_t>(s, a, r16, tiles);
    else
      launch_up<T, bf16_t>(s, a, r16, tiles);
  } else if (a.out_type == HIERAVG_F32) {
    launch_up<T, float>(s, a, r16, tiles);
  } else {
    launch_up<T, T>(s, a, r16, tiles);
  }
}

template <class T, int RT, int R16>
void launch_outer(hipStream_t s, const OuterPair& o, const PlacesArgs& a, const PlacesArgs& b, int64_t units) {
  const int64_t blocks = div_up(a.rows, 32), na = o.a.chunks ? blocks : 0, nb = o.b.chunks ? blocks : 0;
  launch(k_adapter_places<R16, sizeof(T) == 2>, (unsigned)(na + nb), 256, 0, s, a, b, na);
  launch(k_adapter_outer<T, RT, R16>, (unsigned)(units * (o.a.chunks + o.b.chunks)), 256, 0, s, o);
}
template <class T>
void launch_outer(hipStream_t s, const OuterPair& o, const PlacesArgs& a, const PlacesArgs& b, int r16, int64_t units) {
  if (r16 == 16)
    launch_outer<T, 1, 16>(s, o, a, b, units);
  else if (r16 == 32)
    launch_outer<T, 2, 32>(s, o, a, b, units);
  else if (r16 == 64)
    launch_outer<T, 4, 64>(s, o, a, b, units);
  else
    launch_outer<T, 4, 128>(s, o, a, b, units);
}

template <class T>
void run_product(hipStream_t s, const RowPlan& r, const AdapterPlan& p, DownArgs d, UpArgs u, int r16) {
  if (!p.few) launch_plan(s, r);
  d.plan = u.plan = r;
  launch_down<T>(s, d, r16, p.tiles);
  launch_up<T>(s, u, r16, p.tiles);
}

}  // namespace

}  // namespace hav

using namespace hav;

extern "C" {

size_t hieravg_adapter_product_scratch(int64_t rows, const hieravg_adapters* w) {
  if (check_adapters(w, rows) != HIERAVG_OK || rows == 0) return 0;
  return plan_adapters(rows, *w, false, false, false).bytes;
}

int hieravg_adapter_product(const hieravg_adapters* w, const void* x, int64_t rows, int64_t x_stride, const void* ids,
                            int32_t id_bytes, const void* base, int64_t base_stride, void* out, int32_t out_type,
                            int64_t out_stride, float* hidden, void* scratch, size_t scratch_bytes, void* hip_stream) {
  return guarded([&]() -> int {
    int rc = check_adapters(w, rows);
    if (rc != HIERAVG_OK) return rc;
    if (!result_type(out_type, w->type)) return invalid("unknown element type of out, or 16-bit and not the adapters'");
    if (rows == 0) return HIERAVG_OK;
    if ((rc = check_weights(w)) != HIERAVG_OK || (rc = check_ids(ids, id_bytes)) != HIERAVG_OK) return rc;
    if ((rc = check_rows(x, w->type, rows, w->in, x_stride, "x must be an aligned pointer, x_stride at least in")) != HIERAVG_OK ||
        (rc = check_rows(out, out_type, rows, w->out, out_stride, "out must be an aligned pointer, out_stride at least out")) != HIERAVG_OK ||
        (base && (rc = check_rows(base, out_type, rows, w->out, base_stride,
                                  "base must be an aligned pointer, base_stride at least out")) != HIERAVG_OK))
      return rc;
    if (hidden && !aligned(hidden, 4)) return invalid("hidden must be aligned to its element");
    const Area o = rows_area(out, rows, out_stride, w->out, out_type), xa = rows_area(x, rows, x_stride, w->in, w->type),
               ba = rows_area(base, rows, base_stride, w->out, out_type), ia = block_area(ids, rows * id_bytes);
    if (meet_any(o, xa, ia, down_area(*w), up_area(*w), scales_area(*w)) || (!same_rows(base, base_stride, out, out_stride, rows) && meet(o, ba)))
      return invalid("out must be base (same pointer and row stride) or overlap no rows of base and x and no other operand");
    const AdapterPlan p = plan_adapters(rows, *w, false, false, false);
    if (!scratch || scratch_bytes < p.bytes || !aligned(scratch, 16))
      return invalid("scratch must hold hieravg_adapter_product_scratch bytes, 16-byte aligned");
    if (meet_any(block_area(hidden, rows * w->rank * 4), o, xa, ba, ia, down_area(*w), up_area(*w), scales_area(*w)))
      return invalid("hidden must overlap neither out nor an operand");
    const int64_t chunks = div_up(w->out, up_cols(*w));
    if (p.tiles * std::max<int64_t>(chunks, p.down.splits) > kMaxGroups) return invalid("too many tiles");
    char* mem = (char*)scratch;
    const RowPlan r = rows_plan(p, mem, *w, ids, id_bytes, rows);
    const DownArgs d{{}, x, w->down, (float*)(mem + p.h), x_stride, w->in, w->rank, p.down.splits, p.down.part};
    const UpArgs u{{}, (const float*)(mem + p.h), w->up, w->scales, base, out, hidden, base_stride, out_stride, w->out,
                   w->rank, p.down.splits, out_type, (int)chunks};
    hipStream_t s = (hipStream_t)hip_stream;
    if (w->type == HIERAVG_F32)
      run_product<float>(s, r, p, d, u, padded(*w));
    else if (w->type == HIERAVG_F16)
      run_product<f16_t>(s, r, p, d, u, padded(*w));
    else
      run_product<bf16_t>(s, r, p, d, u, padded(*w));
    return launched("hieravg_adapter_product");
  });
}

size_t hieravg_adapter_grad_scratch(int64_t rows, const hieravg_adapters* w, int32_t hidden) {
  if (check_adapters(w, rows) != HIERAVG_OK || rows == 0) return 0;
  return plan_adapters(rows, *w, true, true, hidden != 0).bytes;
}

size_t hieravg_adapter_dx_scratch(int64_t rows, const hieravg_adapters* w) {
  if (check_adapters(w, rows) != HIERAVG_OK || rows == 0) return 0;
  return plan_adapters(rows, *w, true, false, false).bytes;
}

int hieravg_adapter_grad(const hieravg_adapters* w, const void* grad, int64_t rows, int64_t grad_stride, const void* x,
                         int64_t x_stride, const void* ids, int32_t id_bytes, const float* hidden, const void* base,
                         int64_t base_stride, void* dx, int32_t dx_type, int64_t dx_stride, void* ddown, void* dup,
                         int32_t weight_type, void* scratch, size_t scratch_bytes, void* hip_stream) {
  return guarded([&]() -> int {
    int rc = check_adapters(w, rows);
    if (rc != HIERAVG_OK) return rc;
    if (!result_type(dx_type, w->type) || !known_type(weight_type))
      return invalid("unknown element type of dx, ddown or dup, or a dx that is 16-bit and not of the adapters' type");
    if (!dx && !ddown && !dup) return invalid("dx, ddown and dup are all NULL");
    if ((ddown && !aligned(ddown, type_bytes(weight_type))) || (dup && !aligned(dup, type_bytes(weight_type))))
      return invalid("ddown and dup must be aligned to their element");
    if (rows == 0 && (ddown || dup)) return invalid("a gradient over no rows");
    if (rows == 0) return HIERAVG_OK;
    if ((rc = check_weights(w)) != HIERAVG_OK || (rc = check_ids(ids, id_bytes)) != HIERAVG_OK) return rc;
    if ((rc = check_rows(grad, w->type, rows, w->out, grad_stride, "grad must be an aligned pointer, grad_stride at least out")) != HIERAVG_OK)
      return rc;
    const bool need_x = ddown || (dup && !hidden);
    if (need_x && (rc = check_rows(x, w->type, rows, w->in, x_stride, "x must be an aligned pointer, x_stride at least in")) != HIERAVG_OK)
      return rc;
    if (hidden && !aligned(hidden, 4)) return invalid("hidden must be aligned to its element");
    const Area ga = rows_area(grad, rows, grad_stride, w->out, w->type), xa = rows_area(need_x ? x : nullptr, rows, x_stride, w->in, w->type),
               ia = block_area(ids, rows * id_bytes), ha = block_area(hidden, rows * w->rank * 4);
    Area o{}, ba{};
    if (dx) {
      if ((rc = check_rows(dx, dx_type, rows, w->in, dx_stride, "dx must be an aligned pointer, dx_stride at least in")) != HIERAVG_OK ||
          (base && (rc = check_rows(base, dx_type, rows, w->in, base_stride,
                                    "base must be an aligned pointer, base_stride at least in")) != HIERAVG_OK))
        return rc;
      o = rows_area(dx, rows, dx_stride, w->in, dx_type);
      ba = rows_area(base, rows, base_stride, w->in, dx_type);
      if (meet_any(o, xa, ga, ia, ha, down_area(*w), up_area(*w), scales_area(*w)) || (!same_rows(base, base_stride, dx, dx_stride, rows) && meet(o, ba)))
        return invalid("dx must be base (same pointer and row stride) or overlap no rows of base, x and grad and no other operand");
    }
    const AdapterPlan p = plan_adapters(rows, *w, true, ddown || dup, hidden != nullptr);
    const int64_t up_chunks = div_up(w->in, up_cols(*w)), blocks = div_up(w->rank, kOuterRank);
    const int64_t cols = outer_cols(w->type);
    const int64_t chunks_a = ddown ? div_up(w->in, cols) * blocks : 0, chunks_b = dup ? div_up(w->out, cols) * blocks : 0;
    const int64_t join_a = ddown ? div_up((int64_t)w->rank * w->in, 1024) : 0, join_b = dup ? div_up((int64_t)w->rank * w->out, 1024) : 0;
    if (p.tiles * std::max<int64_t>({up_chunks, p.down.splits, p.down2.splits}) > kMaxGroups ||
        p.units * (chunks_a + chunks_b) > kMaxGroups || (join_a + join_b) * p.joins > kMaxGroups)
      return invalid("too many tiles");
    if (!scratch || scratch_bytes < p.bytes || !aligned(scratch, 16))
      return invalid("scratch must hold hieravg_adapter_grad_scratch (dx alone: hieravg_adapter_dx_scratch) bytes, 16-byte aligned");
    const Area da = block_area(ddown, int64_t(w->n) * w->rank * w->in * type_bytes(weight_type)),
               ua = block_area(dup, int64_t(w->n) * w->rank * w->out * type_bytes(weight_type));
    for (const Area& a : {da, ua})
      if (meet_any(a, xa, ga, ba, ia, ha, o, down_area(*w), up_area(*w), scales_area(*w)))
        return invalid("ddown and dup must overlap neither dx nor an operand");
    if (meet(da, ua)) return invalid("ddown and dup must not overlap");
    char* mem = (char*)scratch;
    RowPlan r = rows_plan(p, mem, *w, ids, id_bytes, rows);
    if (p.units) {
      r.units = (Tile*)(mem + p.unit);
      r.joins = (Join*)(mem + p.join);
      r.join_most = (int)p.joins;
    }
    float *dh = (float*)(mem + p.h), *h = (float*)(mem + p.h2), *parts = (float*)(mem + p.parts);
    char* places = mem + p.places;
    hipStream_t s = (hipStream_t)hip_stream;
    auto run = [&](auto t) {
      using T = decltype(t);
      launch_plan(s, r);
      if (dx || ddown) launch_down<T>(s, DownArgs{r, grad, w->up, dh, grad_stride, w->out, w->rank, p.down.splits, p.down.part}, padded(*w), p.tiles);
      if (dup && !hidden)
        launch_down<T>(s, DownArgs{r, x, w->down, h, x_stride, w->in, w->rank, p.down2.splits, p.down2.part}, padded(*w), p.tiles);
      if (dx)
        launch_up<T>(s, UpArgs{r, dh, w->down, w->scales, base, dx, nullptr, base_stride, dx_stride, w->in, w->rank,
                               p.down.splits, dx_type, (int)up_chunks}, padded(*w), p.tiles);
      if (!ddown && !dup) return;
      const int64_t place = place_bytes(rows, *w);
      const PlacesArgs pa{r.order, dh, places, rows, padded(*w), w->rank, p.down.splits};
      const PlacesArgs pb{r.order, hidden ? hidden : h, places + place, rows, hidden ? w->rank : padded(*w), w->rank,
                          hidden ? 1 : p.down2.splits};
      OuterPair o{r, {places, x, ddown, parts, x_stride, w->in, (int)chunks_a},
                  {places + place, grad, dup, parts + p.slots * w->rank * w->in, grad_stride, w->out, (int)chunks_b},
                  w->scales, w->rank, weight_type, (int)blocks};
      launch_outer<T>(s, o, pa, pb, padded(*w), p.units);
      if (p.joins) launch(k_adapter_join, (unsigned)((join_a + join_b) * p.joins), 256, 0, s, o, join_a, join_b);
    };
    if (w->type == HIERAVG_F32)
      run(float{});
    else if (w->type == HIERAVG_F16)
      run(f16_t{});
    else
      run(bf16_t{});
    return launched("hieravg_adapter_grad");
  });
}

}  // extern "C"
