// 1x1x1 layers in 8 bits: rows and weights of e4m3 values with a scale each.
//
//   out[r, j] = sx[r] sw[j] sum_k x[r, k] w[j, k]
//
// The values become fp16 on their way to the matrix cores, which holds each of them exactly, as do 32 bits each product; sums are held in 32 bits, the scales come behind, one
// rounding to the output's type.  (The matrix cores' products of 8-bit operands line up their terms in fewer bits: 2^-13.5 of the sum of magnitudes off at 128 places
// of values from all binades, 2^-22.8 so.  They would be twice as fast, which bytes leave no use for: 120 k x 256 -> 1024 moves 277 MB for 63 GFLOP.)
// A workgroup holds 256 rows (128 of more than 256 channels) in its waves' registers where their channels fit (up to 512), so x is read once, and walks over the columns in tiles of
// 32, whose weights all four waves read from LDS, where they are halves already; the next tile's bytes and scales are on their way meanwhile.  The weights are the product's left
// operand and a tile's lines are dealt to its 16 x 16 products so that a lane ends up with pieces of 16 bytes of one output row, next to its neighbours': every store of a
// wave fills 64 consecutive bytes of 16 rows.
//
// 120 k x 256 -> 1024 to fp16: 94 us (0.67 PFLOP/s; torch's 8192^3 product reaches 1.15) for 58 of bytes and 55 of products; two waves a SIMD take turns at conversions and products (vector
// unit 53 % of the CUs' cycles; a wave's rows become halves again for each of 32 tiles).  Stores of halves to LDS use every other slot of 16 bytes: 1.9 M conflicts in 1.2 M instructions.  Tiles and rows a wave, us: 32 columns, 64 rows 91; 64, 32 105; 32, 32 102; 64, 64 120 (registers for one wave a SIMD).  All workgroups at the
// same columns at once 128.  Rows' scales and columns' loaded where they are used 99.  60 k x 512 -> 512 47 (rows read again for every tile, 64 a wave: 90).  120 k x 128 -> 512 36 for 29 of bytes, 120 k x 64 -> 256 to fp32 28 for 27.  Rows of
// more than 512 channels are read and made halves again for every 32 columns: 30 k x 1500 -> 512 175 for 40 of products.  Small calls are the host's:
// 6011 x 128 -> 512 9.0 (kernel 6.2), one row 10.4.
#include <algorithm>
#include <type_traits>

#include "rows.h"

namespace spc {
namespace {

constexpr int LIN_COLS = 32, LIN_K = 256, LIN_STEP = 64;  // a tile of weights: columns, bytes of each; places of two products
constexpr int LIN_THREADS = 256;
constexpr int LIN_MAX_C = 65536;

typedef _Float16 half2 __attribute__((ext_vector_type(2)));
typedef _Float16 half8 __attribute__((ext_vector_type(8)));
typedef float floatx4 __attribute__((ext_vector_type(4)));

struct LinearArgs {
  const uint8_t *x, *w;
  const float *sx, *sw;
  void* out;
  int64_t ld_x, ld_w, ld_out, n;
  int c, cout, tiles;  // tiles: column tiles of a workgroup
};

// 16 bytes of a row of c from place k on, zeros behind its end.  WHOLE: c is a multiple of 16.
template <bool WHOLE>
__device__ inline Words4 piece16(const uint8_t* row, int k, int c) {
  typedef int Any __attribute__((ext_vector_type(4), aligned(1), may_alias));
  Words4 v = {0, 0, 0, 0};
  const int left = c - k;
  if (left >= 16) {
    v = *reinterpret_cast<const Any*>(row + k);
  } else if (!WHOLE && left > 0) {
#pragma unroll
    for (int i = 0; i < 15; ++i)
      if (i < left) v[i / 4] |= int(row[k + i]) << (i % 4 * 8);
  }
  return v;
}
__device__ inline void to_halves(Words4 v, half8 (&f)[2]) {
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    const half2 a = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(v[q], 1.f, false), b = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(v[q], 1.f, true);
    f[q / 2][q % 2 * 4] = a[0], f[q / 2][q % 2 * 4 + 1] = a[1], f[q / 2][q % 2 * 4 + 2] = b[0], f[q / 2][q % 2 * 4 + 3] = b[1];
  }
}

// KS: steps of 64 places that a wave's rows are held for (0: they are read again for every tile of columns, 256 places at a time and those ahead).  RT: groups of 16 rows a wave.  Lane l has row (column) l % 16 of every operand and 16 places of a
// step's 64 from 16 (l / 16) on, in two products of 32; of a result column l % 16 and rows 4 (l / 16) + r.
template <typename T, int KS, int RT, bool WHOLE>
__global__ __launch_bounds__(LIN_THREADS) void linear8_kernel(const LinearArgs a) {
  constexpr int STEPS = KS ? KS : LIN_K / LIN_STEP, WIDTH = STEPS * LIN_STEP / 16;  // steps and pieces of 16 bytes of a tile's line
  constexpr int PIECES = LIN_COLS * WIDTH, MINE = (PIECES + LIN_THREADS - 1) / LIN_THREADS, MT = LIN_COLS / 16, TURNS = WIDTH >= 8 ? 16 : 8;  // of which each thread fetches so many
  __shared__ half8 tiles[2][LIN_COLS * WIDTH * 2];
  const int t = threadIdx.x, lane = t % 64, wave = t / 64, i = lane % 16, g = lane / 16;
  const int all = (a.cout + LIN_COLS - 1) / LIN_COLS, splits = (all + a.tiles - 1) / a.tiles, parts = KS ? 1 : (a.c + LIN_K - 1) / LIN_K;
  const int64_t block = blockIdx.x / splits;
  const int first_tile = blockIdx.x % splits * a.tiles, count = min(a.tiles, all - first_tile);
  // (a workgroup starts with a tile of its own: were all at the same columns at once, rows of a power of two would keep few memory channels busy)
  const int turn = static_cast<int>(block % count);
  auto tile_at = [&](int n) { return first_tile + (n + turn < count ? n + turn : n + turn - count); };
  const int64_t row0 = (block * 4 + wave) * (16 * RT) + i;  // of group 0; the lane's row of group q is 16 q further
  // Line 16 m + 4 g + r of a tile is the column that a lane stores of result r of product m: piece 4 m / VEC of its row, lane by lane.  A line's pieces of 8 halves
  // are turned by its number, so that 16 lines' reads of one place lie in different banks.
  constexpr int VEC = 16 / sizeof(T);
  auto column = [](int line) { return line / 16 * 4 / VEC * (4 * VEC) + line % 16 / 4 * VEC + line / 16 * 4 % VEC + line % 4; };
  constexpr int STORES = LIN_COLS / (4 * VEC);
  typedef float Some __attribute__((ext_vector_type(VEC), aligned(4), may_alias));
  typedef T Values __attribute__((ext_vector_type(VEC)));
  Words4 next[MINE];
  Some next_scale[STORES];  // (of the columns that this lane stores)
  auto fetch = [&](int ct, int part) {
#pragma unroll
    for (int p = 0; p < MINE; ++p) {
      const int line = (p * LIN_THREADS + t) / WIDTH % LIN_COLS, k = part * LIN_K + (p * LIN_THREADS + t) % WIDTH * 16;
      const int col = ct * LIN_COLS + column(line);
      next[p] = Words4{0, 0, 0, 0};
      if (col < a.cout) next[p] = piece16<WHOLE>(a.w + int64_t(col) * a.ld_w, k, a.c);
    }
  };
  auto fetch_scale = [&](int ct) {
#pragma unroll
    for (int p = 0; p < STORES; ++p) {
      const int col = ct * LIN_COLS + p * (4 * VEC) + g * VEC;
      if ((ct + 1) * LIN_COLS <= a.cout) {
        next_scale[p] = *reinterpret_cast<const Some*>(a.sw + col);
      } else {
#pragma unroll
        for (int k = 0; k < VEC; ++k) next_scale[p][k] = col + k < a.cout ? a.sw[col + k] : 0.f;
      }
    }
  };
  auto rows = [&](int k, Words4 (&v)[RT]) {
#pragma unroll
    for (int q = 0; q < RT; ++q) {
      v[q] = Words4{0, 0, 0, 0};
      if (row0 + 16 * q < a.n) v[q] = piece16<WHOLE>(a.x + (row0 + 16 * q) * a.ld_x, k + 16 * g, a.c);
    }
  };
  Words4 held[STEPS][RT], ahead[KS ? 1 : STEPS][RT];  // (as bytes: halves of 256 channels would take 128 registers; those of up to 128 would fit, which was not measured)
  fetch(tile_at(0), 0);
  fetch_scale(tile_at(0));
#pragma unroll
  for (int s = 0; s < STEPS; ++s) rows(s * LIN_STEP, KS ? held[s] : ahead[KS ? 0 : s]);
  float sx[RT];
#pragma unroll
  for (int q = 0; q < RT; ++q) sx[q] = row0 + 16 * q < a.n ? a.sx[row0 + 16 * q] : 0.f;
  int buf = 0;
  for (int n = 0; n < count; ++n) {
    const int ct = tile_at(n);
    Some scale[STORES];
#pragma unroll
    for (int p = 0; p < STORES; ++p) scale[p] = next_scale[p];
    if constexpr (KS > 0)
#pragma unroll
      for (int s = 0; s < KS; ++s)
#pragma unroll
        for (int q = 0; q < RT; ++q) asm volatile("" : "+v"(held[s][q]));  // (else they are made halves once for all tiles)
    floatx4 acc[RT][MT];
#pragma unroll
    for (int q = 0; q < RT; ++q)
#pragma unroll
      for (int m = 0; m < MT; ++m) acc[q][m] = floatx4{0.f, 0.f, 0.f, 0.f};
    for (int part = 0; part < parts; ++part, buf ^= 1) {
      half8* tile = tiles[buf];
#pragma unroll
      for (int p = 0; p < MINE; ++p) {
        const int line = (p * LIN_THREADS + t) / WIDTH, at = (p * LIN_THREADS + t) % WIDTH;
        if (PIECES % LIN_THREADS && p * LIN_THREADS + t >= PIECES) continue;
        half8 w[2];
        to_halves(next[p], w);
#pragma unroll
        for (int h = 0; h < 2; ++h) tile[line * (2 * WIDTH) + ((2 * at + h) ^ line % TURNS)] = w[h];
      }
      // (one barrier a tile: whoever stores to a buffer again has passed the barrier behind its last reads, since there are two)
      __syncthreads();
      if (part + 1 < parts) fetch(ct, part + 1);
      else if (n + 1 < count) fetch(tile_at(n + 1), 0), fetch_scale(tile_at(n + 1));
      if constexpr (KS == 0) {
#pragma unroll
        for (int s = 0; s < STEPS; ++s)
#pragma unroll
          for (int q = 0; q < RT; ++q) held[s][q] = ahead[s][q];
        const int k = part + 1 < parts ? (part + 1) * LIN_K : 0;
#pragma unroll
        for (int s = 0; s < STEPS; ++s) rows(k + s * LIN_STEP, ahead[s]);
      }
#pragma unroll
      for (int s = 0; s < STEPS; ++s) {
        half8 f[RT][2];
#pragma unroll
        for (int q = 0; q < RT; ++q) to_halves(held[s][q], f[q]);
#pragma unroll
        for (int m = 0; m < MT; ++m) {
#pragma unroll
          for (int p = 0; p < 2; ++p) {
            const half8 w = tile[(16 * m + i) * (2 * WIDTH) + ((2 * (4 * s + g) + p) ^ i % TURNS)];
#pragma unroll
            for (int q = 0; q < RT; ++q) acc[q][m] = __builtin_amdgcn_mfma_f32_16x16x32_f16(w, f[q][p], acc[q][m], 0, 0, 0);
          }
        }
      }
    }
    const bool full = (ct + 1) * LIN_COLS <= a.cout;
#pragma unroll
    for (int p = 0; p < STORES; ++p) {
      const int col = ct * LIN_COLS + p * (4 * VEC) + g * VEC, left = a.cout - col;
#pragma unroll
      for (int q = 0; q < RT; ++q) {
        if (row0 + 16 * q >= a.n) continue;
        T* to = static_cast<T*>(a.out) + (row0 + 16 * q) * a.ld_out + col;
        Values v;
#pragma unroll
        for (int k = 0; k < VEC; ++k) v[k] = static_cast<T>(acc[q][(p * VEC + k) / 4][k % 4] * sx[q] * scale[p][k]);
        if (full || VEC <= left) {
          *reinterpret_cast<AnyWords4*>(to) = __builtin_bit_cast(Words4, v);
        } else {
#pragma unroll
          for (int k = 0; k < VEC; ++k)
            if (k < left) to[k] = v[k];
        }
      }
    }
  }
}

}  // namespace
}  // namespace spc

extern "C" int spc_linear_f8(const void* x, int64_t ld_x, const float* x_scale, const void* w, int64_t ld_w, const float* w_scale, void* out, int64_t ld_out,
                             int64_t n, int32_t c, int32_t cout, int32_t dtype, void* stream) {
  using namespace spc;
  if (dtype != SPC_DTYPE_F16 && dtype != SPC_DTYPE_BF16 && dtype != SPC_DTYPE_F32) return set_error(SPC_ERR_ARG, "unknown dtype %d", dtype);
  if (n < 0 || c < 1 || cout < 1) return set_error(SPC_ERR_ARG, "n = %lld, c = %d, cout = %d", static_cast<long long>(n), c, cout);
  if (c > LIN_MAX_C || cout > LIN_MAX_C || n > (int64_t(1) << 30))  // (a launch takes less than 2^32 threads, 256 of them to 128 rows)
    return set_error(SPC_ERR_UNSUPPORTED, "%lld rows of %d channels to %d: at most 2^30 and %d", static_cast<long long>(n), c, cout, LIN_MAX_C);
  if (!n) return SPC_OK;
  if (!x || !w || !out || !x_scale || !w_scale) return set_error(SPC_ERR_ARG, "NULL argument");
  if (ld_x < c || ld_w < c || ld_out < cout)
    return set_error(SPC_ERR_ARG, "row pitches %lld, %lld, %lld are below %d, %d, %d", static_cast<long long>(ld_x), static_cast<long long>(ld_w), static_cast<long long>(ld_out),
                     c, c, cout);
  if (reinterpret_cast<uintptr_t>(out) % (dtype == SPC_DTYPE_F32 ? 4 : 2)) return set_error(SPC_ERR_ARG, "out is not aligned to its type");
  LinearArgs a{static_cast<const uint8_t*>(x), static_cast<const uint8_t*>(w), x_scale, w_scale, out, ld_x, ld_w, ld_out, n, c, cout, 1};
  const int all = (cout + LIN_COLS - 1) / LIN_COLS;
  by_dtype(dtype, [&](auto type) {
    auto go = [&](auto ks, auto rt, auto whole) {
      constexpr int RT = decltype(rt)::value, ROWS = 64 * RT;
      const int64_t blocks = (n + ROWS - 1) / ROWS;
      // columns are split between workgroups until there are some 512 of them (120 k x 256 -> 1024, aiming at 512 / 1024 / 2048: 99 / 107 / 124 us)
      const int splits = static_cast<int>(std::min<int64_t>(all, std::max<int64_t>(1, 512 / blocks)));
      a.tiles = (all + splits - 1) / splits;
      hipLaunchKernelGGL((linear8_kernel<decltype(type), decltype(ks)::value, RT, decltype(whole)::value>), dim3(blocks * ((all + a.tiles - 1) / a.tiles)), dim3(LIN_THREADS), 0,
                         static_cast<hipStream_t>(stream), a);
    };
    auto with = [&](auto ks, auto rt) {
      if (c % 16 == 0) go(ks, rt, std::true_type{});
      else go(ks, rt, std::false_type{});
    };
    using std::integral_constant;
    const integral_constant<int, 2> two;
    const integral_constant<int, 4> four;
    if (c <= 64) with(integral_constant<int, 1>{}, four);
    else if (c <= 128) with(integral_constant<int, 2>{}, four);
    else if (c <= 256) with(integral_constant<int, 4>{}, four);
    else if (c <= 512) with(integral_constant<int, 8>{}, two);
    else with(integral_constant<int, 0>{}, two);
  });
  SPC_HIP_CHECK(hipGetLastError());
  return SPC_OK;
}
