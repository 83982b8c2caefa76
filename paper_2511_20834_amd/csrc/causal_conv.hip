// Short causal convolution of every channel along the rows of its scene, with a gate of its own (SiLU).
//
//   p_t = bias + sum_{k < W} w[W-1-k] x_{t-k},   y_t = p_t / (1 + exp(-p_t))  (or p_t itself)
//
// Rows in front of a scene come from a state of W - 1 rows, or are zeros.  Backward, with d_t = dy_t silu'(p_t):
//
//   dx_t = sum_k w[W-1-k] d_{t+k},   dw[W-1-k] = sum_t d_t x_{t-k},   dbias = sum_t d_t
//
// A thread walks down `per` rows of a piece of 16 bytes of channels and keeps the last W - 1 rows (backward: of d as well) in registers, so everything is read once but
// for the W - 1 rows in front (and behind) of its own, which the caches hold.  The bytes bound the forward pass; in the gradients, which make p and its slope again, the vector unit
// issues in 70 % of the CUs' cycles (120 k x 512) and 73 % (70 k x 90), for as many scalar instructions as 29 and 50 % of its own.  Workgroups take segments of scenes; backward they
// walk over several, keep the sums of dw and dbias and store them once; a second launch adds them up in a fixed order.
//
// us a pass (bytes at a copy's 4.76 TB/s): 120 k x 512 bf16, width 4, out of rows of 1024 53 (52); its gradients 122 (75); 70 k x 90 fp16, width 3, gradients 26 (8: a launch of 23, 72 % of the lanes have channels, a thread has 4 rows and loads 8, and one of 4); a row of 2048 streams of
// 512 channels 6.0 in the kernel.
#include <algorithm>
#include <type_traits>

#include "scenes.h"

namespace spc {
namespace {

constexpr int CONV_THREADS = 256;
constexpr int CONV_MAX_W = 4;
constexpr int CONV_MAX_C = 65536;

struct ConvArgs {
  Scenes scenes;
  const void *x, *dy, *past, *dpast;  // past: rows in front of the scenes; dpast: gradient of the rows behind them
  void *y, *past_out;                 // backward: dx and the gradient of past
  const float *weight, *bias;
  float* partial;
  int64_t ld_x, ld_dy, ld_y;
  int c, per, log_tp, col_blocks, ids;
};

// A piece of VEC channels: whole, the row's last ones (moved back to end with the row), or less than a piece.
template <typename T, int VEC_, bool FEW>
struct Channels {
  static constexpr int VEC = VEC_;
  typedef T Values __attribute__((ext_vector_type(VEC)));
  typedef int Words __attribute__((ext_vector_type(VEC * int(sizeof(T)) / 4)));
  typedef int AnyWords __attribute__((ext_vector_type(VEC * int(sizeof(T)) / 4), aligned(2), may_alias));
  typedef float Four __attribute__((ext_vector_type(4), aligned(4), may_alias));
  int at, c;  // first channel
  bool some;  // whether there is a channel
  int own;    // first of the piece's channels that no other piece has
  __device__ Channels(int piece, int channels) : at(FEW ? piece * VEC : min(piece * VEC, channels - VEC)), c(channels), some(piece * VEC < channels), own(piece * VEC - at) {}
  __device__ Values fetch(const void* p, int64_t row, int64_t ld) const {
    const T* from = static_cast<const T*>(p) + row * ld + at;
    Values q{};
    if (FEW) {
#pragma unroll
      for (int k = 0; k < VEC - 1; ++k)
        if (at + k < c) q[k] = from[k];
    } else {
      q = __builtin_bit_cast(Values, static_cast<Words>(*reinterpret_cast<const AnyWords*>(from)));
    }
    return q;
  }
  __device__ static void widen(float (&f)[VEC], Values q) {
#pragma unroll
    for (int k = 0; k < VEC; ++k) f[k] = static_cast<float>(q[k]);
  }
  __device__ void load(float (&f)[VEC], const void* p, int64_t row, int64_t ld) const { widen(f, fetch(p, row, ld)); }
  __device__ void store(const float (&f)[VEC], void* p, int64_t row, int64_t ld) const {
    T* to = static_cast<T*>(p) + row * ld + at;
    Values q;
#pragma unroll
    for (int k = 0; k < VEC; ++k) q[k] = static_cast<T>(f[k]);
    if (FEW) {
#pragma unroll
      for (int k = 0; k < VEC - 1; ++k)
        if (at + k < c) to[k] = q[k];
    } else {
      *reinterpret_cast<AnyWords*>(to) = __builtin_bit_cast(Words, q);
    }
  }
  // Its own channels only: where another piece's thread reads what this one would store, too.
  __device__ void store_own(const float (&f)[VEC], void* p, int64_t row, int64_t ld) const {
    if (own == 0) return store(f, p, row, ld);
    T* to = static_cast<T*>(p) + row * ld + at;
#pragma unroll
    for (int k = 0; k < VEC; ++k)
      if (k >= own) to[k] = static_cast<T>(f[k]);
  }
  // N floats of every channel: they lie one behind the other.
  template <int N>
  __device__ void params(float (&f)[N][VEC], const float* p) const {
    float all[VEC * N];
#pragma unroll
    for (int i = 0; i < VEC * N; ++i) all[i] = 0.f;
    if (p) {
      const float* from = p + int64_t(at) * N;
      if (FEW) {
#pragma unroll
        for (int i = 0; i < VEC * N; ++i)
          if (at + i / N < c) all[i] = from[i];
      } else {
#pragma unroll
        for (int i = 0; i < VEC * N; i += 4) {
          const Four v = *reinterpret_cast<const Four*>(from + i);
#pragma unroll
          for (int k = 0; k < 4; ++k) all[i + k] = v[k];
        }
      }
    }
#pragma unroll
    for (int j = 0; j < N; ++j)
#pragma unroll
      for (int k = 0; k < VEC; ++k) f[j][k] = all[k * N + j];
  }
};
// Channels of a piece: 16 bytes where a row's work is a few operations, four channels in the gradients, which hold some twenty values of each.
template <typename T>
constexpr int WIDE = 16 / int(sizeof(T));
constexpr int NARROW = 4;

// Row `pos` of the scene, which may lie in front of it.
template <typename P, int W>
__device__ inline void row_or_past(const P& piece, float (&f)[P::VEC], const ConvArgs& a, const SceneSegment& s, int pos) {
  if (pos >= 0) {
    piece.load(f, a.x, int64_t(s.lo) + pos, a.ld_x);
  } else if (a.past) {
    piece.load(f, a.past, int64_t(s.scene) * (W - 1) + (W - 1 + pos), a.c);
  } else {
#pragma unroll
    for (int k = 0; k < P::VEC; ++k) f[k] = 0.f;
  }
}

template <typename T, int W, bool FEW, bool SILU>
__global__ __launch_bounds__(CONV_THREADS) void conv_forward_kernel(const ConvArgs a) {
  using P = Channels<T, WIDE<T>, FEW>;
  constexpr int VEC = P::VEC, AHEAD = 4;
  const int tp = 1 << a.log_tp, id = blockIdx.x / a.col_blocks, group = threadIdx.x >> a.log_tp;
  const P piece(blockIdx.x % a.col_blocks * tp + (threadIdx.x & (tp - 1)), a.c);
  SceneSegment s;
  if (!s.find(a.scenes, id) || !piece.some) return;
  if (W > 1 && a.past_out && s.m == s.n - 1 && group == 0)
    for (int i = 0; i < W - 1; ++i) {  // the scene's last rows, as far back as its state reaches
      float f[VEC];
      row_or_past<P, W>(piece, f, a, s, s.hi - s.lo - (W - 1) + i);
      piece.store(f, a.past_out, int64_t(s.scene) * (W - 1) + i, a.c);
    }
  const int t0 = group * a.per, t1 = min(t0 + a.per, s.rows);
  if (t0 >= t1) return;
  typename P::Values next[AHEAD];  // (the next rows are on their way while those at hand are worked on)
  auto fetch = [&](int t) {
#pragma unroll
    for (int q = 0; q < AHEAD; ++q) next[q] = piece.fetch(a.x, int64_t(s.first) + min(t + q, t1 - 1), a.ld_x);
  };
  fetch(t0);
  float w[W][VEC], bias[1][VEC], x[W + AHEAD - 1][VEC];
  piece.params(w, a.weight);
  piece.params(bias, a.bias);
  const int pos = s.first - s.lo + t0;
#pragma unroll
  for (int j = 0; j < W - 1; ++j) row_or_past<P, W>(piece, x[j], a, s, pos - (W - 1) + j);
  for (int t = t0; t < t1; t += AHEAD) {
#pragma unroll
    for (int q = 0; q < AHEAD; ++q) P::widen(x[W - 1 + q], next[q]);
    if (t + AHEAD < t1) fetch(t + AHEAD);
#pragma unroll
    for (int q = 0; q < AHEAD; ++q) {
      if (t + q >= t1) break;
      float y[VEC];
#pragma unroll
      for (int k = 0; k < VEC; ++k) {
        float p = bias[0][k];
#pragma unroll
        for (int j = 0; j < W; ++j) p = fmaf(w[j][k], x[q + j][k], p);
        y[k] = SILU ? p * sigmoid_of<sizeof(T) == 4>(p) : p;
      }
      piece.store(y, a.y, int64_t(s.first) + t + q, a.ld_y);
    }
#pragma unroll
    for (int j = 0; j < W - 1; ++j)
#pragma unroll
      for (int k = 0; k < VEC; ++k) x[j][k] = x[AHEAD + j][k];
  }
}

template <typename T, int W, bool FEW, bool SILU>
__global__ __launch_bounds__(CONV_THREADS) void conv_backward_kernel(const ConvArgs a) {
  using P = Channels<T, NARROW, FEW>;
  constexpr int VEC = P::VEC, AHEAD = 4;
  extern __shared__ float sums[];  // [columns of a workgroup][W + 1] by piece
  const int tp = 1 << a.log_tp, group = threadIdx.x >> a.log_tp, lane_piece = threadIdx.x & (tp - 1);
  const int col_block = blockIdx.x % a.col_blocks, part = blockIdx.x / a.col_blocks, parts = gridDim.x / a.col_blocks;
  const P piece(col_block * tp + lane_piece, a.c);
  float w[W][VEC], bias[1][VEC], dw[W][VEC] = {}, dbias[VEC] = {};
  if (piece.some) {
    piece.params(w, a.weight);
    piece.params(bias, a.bias);
  }
  for (int id = part; id < a.ids; id += parts) {
    SceneSegment s;
    if (!s.find(a.scenes, id) || !piece.some) continue;
    const int len = s.hi - s.lo, base = s.first - s.lo;
    const int t0 = base + group * a.per, t1 = min(t0 + a.per, base + s.rows);  // this thread's rows of the scene
    const bool front = W > 1 && t0 == 0 && a.past_out;
    if (len == 0 && front)
      for (int i = 0; i < W - 1; ++i) {  // (the state goes through as it is)
        float f[VEC] = {};
        if (a.dpast) piece.load(f, a.dpast, int64_t(s.scene) * (W - 1) + i, a.c);
        piece.store(f, a.past_out, int64_t(s.scene) * (W - 1) + i, a.c);
      }
    if (t0 >= t1) continue;
    float x[W + AHEAD - 1][VEC], d[W + AHEAD - 1][VEC] = {};  // d: of the rows t - (W - 1) .. t
#pragma unroll
    for (int j = 0; j < W - 1; ++j) row_or_past<P, W>(piece, x[j], a, s, t0 - (W - 1) + j);
    const int stop = t1 + W - 1;
    typename P::Values next_x[AHEAD], next_d[AHEAD];
    auto fetch = [&](int t) {
#pragma unroll
      for (int q = 0; q < AHEAD; ++q) {
        const int64_t row = int64_t(s.lo) + min(min(t + q, stop - 1), len - 1);
        next_x[q] = piece.fetch(a.x, row, a.ld_x);
        next_d[q] = piece.fetch(a.dy, row, a.ld_dy);
      }
    };
    fetch(t0);
    for (int t = t0; t < stop; t += AHEAD) {
#pragma unroll
      for (int q = 0; q < AHEAD; ++q) P::widen(x[W - 1 + q], next_x[q]), P::widen(d[W - 1 + q], next_d[q]);
      if (t + AHEAD < stop) fetch(t + AHEAD);
#pragma unroll
      for (int q = 0; q < AHEAD; ++q) {
        const int at = t + q;
        if (at >= stop) break;
        const bool there = at < len, own = at < t1;
#pragma unroll
        for (int k = 0; k < VEC; ++k) {
          float slope = 1.f;
          if (SILU) {
            float p = bias[0][k];
#pragma unroll
            for (int j = 0; j < W; ++j) p = fmaf(w[j][k], x[q + j][k], p);
            const float g = sigmoid_of<sizeof(T) == 4>(p);
            slope = fmaf(p * g, 1.f - g, g);
          }
          float& dk = d[W - 1 + q][k];
          dk = there ? dk * slope : 0.f;
          if (own) {
            dbias[k] += dk;
#pragma unroll
            for (int j = 0; j < W; ++j) dw[j][k] = fmaf(dk, x[q + j][k], dw[j][k]);
          }
        }
        const int to = at - (W - 1);  // the row whose gradient is complete
        if (to < t0 && !(front && to < 0)) continue;
        float f[VEC] = {};
        if (W > 1 && a.dpast && to + (W - 1) >= len) piece.load(f, a.dpast, int64_t(s.scene) * (W - 1) + (to + (W - 1) - len), a.c);
#pragma unroll
        for (int k = 0; k < VEC; ++k)
#pragma unroll
          for (int j = 0; j < W; ++j) f[k] = fmaf(w[W - 1 - j][k], d[q + j][k], f[k]);
        if (to >= 0) piece.store(f, a.y, int64_t(s.lo) + to, a.ld_y);
        else piece.store(f, a.past_out, int64_t(s.scene) * (W - 1) + at, a.c);
      }
#pragma unroll
      for (int j = 0; j < W - 1; ++j)
#pragma unroll
        for (int k = 0; k < VEC; ++k) x[j][k] = x[AHEAD + j][k], d[j][k] = d[AHEAD + j][k];
    }
  }
  if (!a.partial) return;
  // a wave's groups of rows, then the waves one after the other: [channel][W] and [channel] as the parameters lie
  for (int o = tp; o < 64; o <<= 1)
#pragma unroll
    for (int k = 0; k < VEC; ++k) {
#pragma unroll
      for (int j = 0; j < W; ++j) dw[j][k] += __shfl_xor(dw[j][k], o, 64);
      dbias[k] += __shfl_xor(dbias[k], o, 64);
    }
  for (int g = 0; g < CONV_THREADS / 64; ++g) {
    if (g == int(threadIdx.x) / 64 && threadIdx.x % 64 < tp && piece.some)
#pragma unroll
      for (int k = 0; k < VEC; ++k) {
        if (k < piece.own || (FEW && piece.at + k >= a.c)) continue;
        float* to = sums + (lane_piece * VEC + k) * (W + 1);
#pragma unroll
        for (int j = 0; j < W; ++j) to[j] = g ? to[j] + dw[j][k] : dw[j][k];
        to[W] = g ? to[W] + dbias[k] : dbias[k];
      }
    __syncthreads();
  }
  float* out = a.partial + int64_t(part) * a.c * (W + 1);
  for (int i = threadIdx.x; i < (tp * VEC) * (W + 1); i += CONV_THREADS) {
    const int local = i / (W + 1), j = i % (W + 1), p = col_block * tp + local / VEC;
    const int channel = (FEW ? p * VEC : min(p * VEC, a.c - VEC)) + local % VEC;
    if (p * VEC >= a.c || channel < p * VEC || channel >= a.c) continue;
    if (j < W) out[int64_t(channel) * W + j] = sums[i];
    else out[int64_t(a.c) * W + channel] = sums[i];
  }
}

// One row more of many streams: a thread has a piece of one stream's channels, its W - 1 rows move up by one.
template <typename T, int W, bool FEW, bool SILU>
__global__ __launch_bounds__(CONV_THREADS) void conv_step_kernel(const ConvArgs a, void* past, int64_t n, int pieces) {
  using P = Channels<T, WIDE<T>, FEW>;
  constexpr int VEC = P::VEC;
  const int64_t i = int64_t(blockIdx.x) * CONV_THREADS + threadIdx.x, row = i / pieces;
  if (row >= n) return;
  const P piece(static_cast<int>(i - row * pieces), a.c);
  float x[W][VEC], p[1][VEC], w[W][VEC];
#pragma unroll
  for (int j = 0; j < W - 1; ++j) piece.load(x[j], past, row * (W - 1) + j, a.c);
  piece.load(x[W - 1], a.x, row, a.ld_x);
  piece.params(p, a.bias);
  piece.params(w, a.weight);
#pragma unroll
  for (int j = 0; j < W; ++j)
#pragma unroll
    for (int k = 0; k < VEC; ++k) p[0][k] = fmaf(w[j][k], x[j][k], p[0][k]);
  if (SILU)
#pragma unroll
    for (int k = 0; k < VEC; ++k) p[0][k] *= sigmoid_of<sizeof(T) == 4>(p[0][k]);
  // (the row's last piece shares channels with the one before it, whose thread may be another wave's and have moved them up already: it leaves them to that)
  piece.store_own(p[0], a.y, row, a.ld_y);
#pragma unroll
  for (int j = 0; j < W - 1; ++j) piece.store_own(x[j + 1], past, row * (W - 1) + j, a.c);
}

// ---------------------------------------------------------------- host
int check_conv(int32_t c, int32_t width, int32_t dtype, const float* weight) {
  if (dtype != SPC_DTYPE_F16 && dtype != SPC_DTYPE_BF16 && dtype != SPC_DTYPE_F32) return set_error(SPC_ERR_ARG, "unknown dtype %d", dtype);
  if (c < 1 || width < 1) return set_error(SPC_ERR_ARG, "%d channels, width %d", c, width);
  if (c > CONV_MAX_C || width > CONV_MAX_W) return set_error(SPC_ERR_UNSUPPORTED, "%d channels, width %d: at most %d and %d", c, width, CONV_MAX_C, CONV_MAX_W);
  if (!weight) return set_error(SPC_ERR_ARG, "weight is NULL");
  return SPC_OK;
}
int check_matrix(const char* what, const void* p, int64_t ld, int32_t c, int32_t dtype) {
  if (!p) return set_error(SPC_ERR_ARG, "%s is NULL", what);
  if (ld < c) return set_error(SPC_ERR_ARG, "row pitch %lld of %s is below %d channels", static_cast<long long>(ld), what, c);
  if (reinterpret_cast<uintptr_t>(p) % (dtype == SPC_DTYPE_F32 ? 4 : 2)) return set_error(SPC_ERR_ARG, "%s is not aligned to its type", what);
  return SPC_OK;
}

// Calls f(type, W, FEW, SILU) for the kernels' variants.
template <typename F>
void conv_variant(int32_t dtype, int c, int width, bool silu, bool narrow, F&& f) {
  using std::integral_constant;
  by_dtype(dtype, [&](auto t) {
    const int VEC = narrow ? NARROW : WIDE<decltype(t)>;
    auto with = [&](auto w) {
      auto fit = [&](auto few) {
        if (silu) f(t, w, few, std::true_type{});
        else f(t, w, few, std::false_type{});
      };
      if (c < VEC) fit(std::true_type{});
      else fit(std::false_type{});
    };
    if (width == 1) with(integral_constant<int, 1>{});
    else if (width == 2) with(integral_constant<int, 2>{});
    else if (width == 3) with(integral_constant<int, 3>{});
    else with(integral_constant<int, 4>{});
  });
}

// How a workgroup's threads are dealt to pieces and rows: up to 64 pieces side by side; rows of a thread so that there are some 2048 workgroups, 4 to 16 (120 k x 512, aiming at
// 1024 / 2048 / 4096: 51 / 52 / 70 us, gradients 121 / 121 / 134; 70 k x 90 25.4 / 26.8 / 26.8).
void conv_grid(ConvArgs& a, int vec, int64_t n_rows) {
  const int pieces = (a.c + vec - 1) / vec;
  a.log_tp = 0;
  while (a.log_tp < 6 && (1 << a.log_tp) < pieces) ++a.log_tp;
  a.col_blocks = (pieces + (1 << a.log_tp) - 1) >> a.log_tp;
  const int groups = CONV_THREADS >> a.log_tp;
  const int64_t fill = n_rows * a.col_blocks / (int64_t(groups) * 2048);
  a.per = static_cast<int>(std::min<int64_t>(16, std::max<int64_t>(4, fill / 4 * 4)));
  a.scenes.seg_rows = groups * a.per;
  a.ids = a.scenes.ids();
}
int check_grid(const ConvArgs& a) {  // (a launch takes less than 2^32 threads)
  if (int64_t(a.ids) * a.col_blocks < (int64_t(1) << 24)) return SPC_OK;
  return set_error(SPC_ERR_UNSUPPORTED, "%d rows of %d channels in %d scenes", a.scenes.n_rows, a.c, a.scenes.n_scenes);
}

}  // namespace
}  // namespace spc

extern "C" int spc_causal_conv_forward(const void* x, int64_t ld_x, const float* weight, const float* bias, int32_t width, int32_t silu, const int32_t* offsets,
                                       int32_t n_scenes, const void* rows_in, void* y, int64_t ld_y, void* rows_out, int64_t n, int32_t c, int32_t dtype, void* stream) {
  using namespace spc;
  SPC_RETURN_IF(check_conv(c, width, dtype, weight));
  SPC_RETURN_IF(check_scenes(offsets, n, n_scenes));
  const int es = dtype == SPC_DTYPE_F32 ? 4 : 2;
  if (n) {
    SPC_RETURN_IF(check_matrix("x", x, ld_x, c, dtype));
    SPC_RETURN_IF(check_matrix("y", y, ld_y, c, dtype));
  }
  for (const void* p : {rows_in, static_cast<const void*>(rows_out)})
    if (reinterpret_cast<uintptr_t>(p) % es) return set_error(SPC_ERR_ARG, "rows in front of the scenes are not aligned to their type");
  if (rows_out && rows_out == rows_in) return set_error(SPC_ERR_ARG, "rows_out is rows_in");
  if (!n && !rows_out) return SPC_OK;
  ConvArgs a{};
  a.scenes = {offsets, static_cast<int>(n), n_scenes, 0};
  a.x = x, a.ld_x = ld_x, a.y = y, a.ld_y = ld_y, a.past = rows_in, a.past_out = rows_out, a.weight = weight, a.bias = bias, a.c = c;
  conv_grid(a, 16 / es, n);
  SPC_RETURN_IF(check_grid(a));
  conv_variant(dtype, c, width, silu != 0, false, [&](auto t, auto w, auto few, auto act) {
    hipLaunchKernelGGL((conv_forward_kernel<decltype(t), decltype(w)::value, decltype(few)::value, decltype(act)::value>), dim3(a.ids * a.col_blocks), dim3(CONV_THREADS), 0,
                       static_cast<hipStream_t>(stream), a);
  });
  SPC_HIP_CHECK(hipGetLastError());
  return SPC_OK;
}

extern "C" int spc_causal_conv_backward(const void* dy, int64_t ld_dy, const void* x, int64_t ld_x, const float* weight, const float* bias, int32_t width, int32_t silu,
                                        const int32_t* offsets, int32_t n_scenes, const void* rows_in, const void* drows_out, void* dx, int64_t ld_dx, float* dweight,
                                        float* dbias, void* drows_in, int64_t n, int32_t c, int32_t dtype, void* stream) {
  using namespace spc;
  SPC_RETURN_IF(check_conv(c, width, dtype, weight));
  SPC_RETURN_IF(check_scenes(offsets, n, n_scenes));
  const int es = dtype == SPC_DTYPE_F32 ? 4 : 2;
  if (n) {
    SPC_RETURN_IF(check_matrix("dy", dy, ld_dy, c, dtype));
    SPC_RETURN_IF(check_matrix("x", x, ld_x, c, dtype));
    SPC_RETURN_IF(check_matrix("dx", dx, ld_dx, c, dtype));
  }
  for (const void* p : {rows_in, drows_out, static_cast<const void*>(drows_in)})
    if (reinterpret_cast<uintptr_t>(p) % es) return set_error(SPC_ERR_ARG, "rows in front of the scenes are not aligned to their type");
  if (drows_in && drows_in == drows_out) return set_error(SPC_ERR_ARG, "drows_in is drows_out");
  const StreamId s(static_cast<hipStream_t>(stream));
  const StreamWorkNote note{s};
  ConvArgs a{};
  a.scenes = {offsets, static_cast<int>(n), n_scenes, 0};
  a.x = x, a.ld_x = ld_x, a.dy = dy, a.ld_dy = ld_dy, a.y = dx, a.ld_y = ld_dx, a.past = rows_in, a.dpast = drows_out, a.past_out = drows_in;
  a.weight = weight, a.bias = bias, a.c = c;
  conv_grid(a, NARROW, n);
  SPC_RETURN_IF(check_grid(a));
  const bool params = dweight || dbias;
  const int parts = std::min(a.ids, std::max(1, 1024 / a.col_blocks));  // (what 256 CUs hold at once; each stores sums)
  if (params) {
    a.partial = static_cast<float*>(pool_alloc(scratch_bytes(size_t(parts) * c * (width + 1) * sizeof(float)), s));
    if (!a.partial) return SPC_ERR_NOMEM;
  }
  conv_variant(dtype, c, width, silu != 0, true, [&](auto t, auto w, auto few, auto act) {
    const size_t lds = (size_t(NARROW) << a.log_tp) * (width + 1) * sizeof(float);
    hipLaunchKernelGGL((conv_backward_kernel<decltype(t), decltype(w)::value, decltype(few)::value, decltype(act)::value>), dim3(parts * a.col_blocks), dim3(CONV_THREADS),
                       lds, s, a);
  });
  if (params) column_sums({{dweight, dbias}, {c * width, c}}, a.partial, parts, s);
  pool_free(a.partial, s);
  SPC_HIP_CHECK(hipGetLastError());
  return SPC_OK;
}

extern "C" int spc_causal_conv_step(const void* x, int64_t ld_x, const float* weight, const float* bias, int32_t width, int32_t silu, void* rows, void* y, int64_t ld_y,
                                    int64_t n, int32_t c, int32_t dtype, void* stream) {
  using namespace spc;
  SPC_RETURN_IF(check_conv(c, width, dtype, weight));
  if (n < 0) return set_error(SPC_ERR_ARG, "n = %lld", static_cast<long long>(n));
  if (!n) return SPC_OK;
  SPC_RETURN_IF(check_matrix("x", x, ld_x, c, dtype));
  SPC_RETURN_IF(check_matrix("y", y, ld_y, c, dtype));
  if (width > 1) SPC_RETURN_IF(check_matrix("rows", rows, c, c, dtype));
  const int pieces = (c * (dtype == SPC_DTYPE_F32 ? 4 : 2) + 15) / 16;
  if (n > (int64_t(1) << 31) / pieces) return set_error(SPC_ERR_UNSUPPORTED, "%lld streams of %d channels", static_cast<long long>(n), c);
  ConvArgs a{};
  a.x = x, a.ld_x = ld_x, a.y = y, a.ld_y = ld_y, a.weight = weight, a.bias = bias, a.c = c;
  conv_variant(dtype, c, width, silu != 0, false, [&](auto t, auto w, auto few, auto act) {
    hipLaunchKernelGGL((conv_step_kernel<decltype(t), decltype(w)::value, decltype(few)::value, decltype(act)::value>), dim3((n * pieces + CONV_THREADS - 1) / CONV_THREADS),
                       dim3(CONV_THREADS), 0, static_cast<hipStream_t>(stream), a, rows, n, pieces);
  });
  SPC_HIP_CHECK(hipGetLastError());
  return SPC_OK;
}
