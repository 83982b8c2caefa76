// Layer norm of feature rows, forward and backward.
//
//   z = x + r,  mu = mean(z),  s = 1/sqrt(mean((z - mu)^2) + eps),  h = (z - mu) s,  y = h gamma + beta
//   w = gamma dy,  dz = s (w - mean(w) - h mean(w h)) + e,  dgamma = sum over rows of dy h,  dbeta = sum over rows of dy
//
// A row stays in the registers of G lanes between its load and its store (NV pieces of VEC channels each), so the variance is the mean
// of squared differences, not a difference of means, and everything is read and written once: the bytes bound both passes.
// Neighbouring lanes hold neighbouring pieces; a wave takes 64/G rows at a time.  The workgroups walk over the rows with a stride of the
// grid, which keeps gamma, and in the backward pass the sums of dgamma and dbeta, in registers.  Every workgroup stores its sums once,
// and a second launch adds them up in a fixed order: no atomics, the same bits every time.
//
// Measured, us a pass among others (with the bytes at the 4.84 TB/s that a copy of 2 GiB reaches, which caches of 256 MB can beat): forward 120 k x 256 fp16 with a residual 42.6
// (50.8), backward 48.3 (50.8); 240 k x 256 bf16 94.6 (101.6), 94.4 (101.6); 70 k x 90 fp16 in rows of 180 backward 18.3 (7.8; 107 with pieces of two
// channels and long shares).  Small calls are the host's: 2118 x 64 fp32 10.7, the gradients of 6011 x 128 bf16 15.3.
#include "rows.h"

namespace spc {
namespace {

constexpr int NORM_MAX_C = 8192;
constexpr int NORM_THREADS = 256;

template <typename T>
struct Piece {
  static constexpr int VEC = 16 / sizeof(T);
  typedef T Values __attribute__((ext_vector_type(VEC)));
};

// Sum over the G lanes of a row (G = 256: of the workgroup), the same bits in all of them.
template <int G>
__device__ inline float row_sum(float v, float* lds) {
#pragma unroll
  for (int d = (G < 64 ? G : 64) / 2; d > 0; d >>= 1) v += __shfl_xor(v, d, 64);
  if constexpr (G > 64) {
    __syncthreads();  // (the sums of the row before have been read)
    if (threadIdx.x % 64 == 0) lds[threadIdx.x / 64] = v;
    __syncthreads();
    v = (lds[0] + lds[1]) + (lds[2] + lds[3]);
  }
  return v;
}

struct NormArgs {
  const void *x, *r, *dy, *e;
  const float *gamma, *beta, *mean_in, *rstd_in;
  void *y, *z;
  float *mean, *rstd, *partial;
  int64_t ld_x, ld_r, ld_dy, ld_e, ld_y, ld_z, n;
  int c;
  float eps;
};

// How a row's channels are dealt to pieces: all pieces whole; the last piece moved back to end with the row, over channels of the one before it; less than one
// piece.
enum Fit { WHOLE, MOVED, FEW };

template <typename T, int NV, int G, Fit FIT>
struct Row {
  static constexpr int VEC = Piece<T>::VEC, E = VEC * NV;
  typedef typename Piece<T>::Values Values;
  int c, first;  // channels, and where this lane's first piece would start
  __device__ Row(int channels) : c(channels), first((threadIdx.x % G) * VEC) {}
  __device__ bool has(int i) const { return first + i * (G * VEC) < c; }
  __device__ int place(int i) const { return FIT == MOVED ? min(first + i * (G * VEC), c - VEC) : first + i * (G * VEC); }
  // whether element k counts in sums: it is a channel of the row, and no other piece's
  __device__ bool counts(int k) const {
    const int at = first + (k / VEC) * (G * VEC);
    return FIT == WHOLE ? at < c : FIT == FEW ? at + k < c : at < c && k % VEC >= at - place(k / VEC);
  }
  __device__ int channel(int k) const { return place(k / VEC) + k % VEC; }
  __device__ void load(float (&f)[E], const void* p, int64_t row, int64_t ld) const {
    const T* at = static_cast<const T*>(p) + row * ld;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      Values q{};
      if (FIT == FEW) {
#pragma unroll
        for (int k = 0; k < VEC - 1; ++k)
          if (first + k < c) q[k] = at[first + k];
      } else if (has(i)) {
        q = __builtin_bit_cast(Values, static_cast<Words4>(*reinterpret_cast<const AnyWords4*>(at + place(i))));
      }
#pragma unroll
      for (int k = 0; k < VEC; ++k) f[i * VEC + k] = static_cast<float>(q[k]);
    }
  }
  // (a moved piece stores the channels it shares with the one before it as that one does: the same values)
  __device__ void store(const float (&f)[E], void* p, int64_t row, int64_t ld) const {
    T* at = static_cast<T*>(p) + row * ld;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      Values q;
#pragma unroll
      for (int k = 0; k < VEC; ++k) q[k] = static_cast<T>(f[i * VEC + k]);
      if (FIT == FEW) {
#pragma unroll
        for (int k = 0; k < VEC - 1; ++k)
          if (first + k < c) at[first + k] = q[k];
      } else if (has(i)) {
        *reinterpret_cast<AnyWords4*>(at + place(i)) = __builtin_bit_cast(Words4, q);
      }
    }
  }
  __device__ void load_param(float (&f)[E], const float* p, float none) const {
#pragma unroll
    for (int k = 0; k < E; ++k) f[k] = p ? 0.f : none;
    if (!p) return;
#pragma unroll
    for (int i = 0; i < NV; ++i)
      if (has(i))
#pragma unroll
        for (int k = 0; k < VEC; ++k)
          if (FIT != FEW || first + k < c) f[i * VEC + k] = p[place(i) + k];
  }
};

template <typename T, int NV, int G, Fit FIT>
__global__ __launch_bounds__(NORM_THREADS) void norm_forward_kernel(const NormArgs a) {
  using R = Row<T, NV, G, FIT>;
  constexpr int ROWS = NORM_THREADS / G;
  __shared__ float lds[4];
  const R me(a.c);
  float gamma[R::E], beta[R::E];
  me.load_param(gamma, a.gamma, 1.f);
  me.load_param(beta, a.beta, 0.f);
  const float c = a.c;
  for (int64_t row = int64_t(blockIdx.x) * ROWS + threadIdx.x / G; row < a.n; row += int64_t(gridDim.x) * ROWS) {
    float z[R::E];
    me.load(z, a.x, row, a.ld_x);
    if (a.r) {
      float r[R::E];
      me.load(r, a.r, row, a.ld_r);
#pragma unroll
      for (int k = 0; k < R::E; ++k) z[k] += r[k];
      if (G > 64 && FIT == MOVED) __syncthreads();  // (z may lie over x or r: another wave's piece is read here too)
      me.store(z, a.z, row, a.ld_z);  // (the norm goes on with the sum as it was before this rounding)
    }
    float s = 0.f;
#pragma unroll
    for (int k = 0; k < R::E; ++k) s += FIT != MOVED || me.counts(k) ? z[k] : 0.f;  // (places behind the last channel hold zeros)
    const float mean = row_sum<G>(s, lds) / c;
    s = 0.f;
#pragma unroll
    for (int k = 0; k < R::E; ++k) {
      z[k] -= mean;
      s += me.counts(k) ? z[k] * z[k] : 0.f;
    }
    const float rstd = 1.f / sqrtf(row_sum<G>(s, lds) / c + a.eps);
#pragma unroll
    for (int k = 0; k < R::E; ++k) z[k] = fmaf(z[k] * rstd, gamma[k], beta[k]);
    me.store(z, a.y, row, a.ld_y);
    if (threadIdx.x % G == 0 && a.mean) {
      a.mean[row] = mean;
      a.rstd[row] = rstd;
    }
  }
}

template <typename T, int NV, int G, Fit FIT>
__global__ __launch_bounds__(NORM_THREADS) void norm_backward_kernel(const NormArgs a) {
  using R = Row<T, NV, G, FIT>;
  constexpr int ROWS = NORM_THREADS / G;
  __shared__ float lds[4];
  extern __shared__ float sums[];  // G <= 64: 2 c floats
  const R me(a.c);
  float gamma[R::E], dgamma[R::E] = {}, dbeta[R::E] = {};
  me.load_param(gamma, a.gamma, 1.f);
  const float c = a.c;
  for (int64_t row = int64_t(blockIdx.x) * ROWS + threadIdx.x / G; row < a.n; row += int64_t(gridDim.x) * ROWS) {
    float h[R::E], dy[R::E];
    me.load(h, a.x, row, a.ld_x);
    me.load(dy, a.dy, row, a.ld_dy);
    const float mean = a.mean_in[row], rstd = a.rstd_in[row];
    float s1 = 0.f, s2 = 0.f;
#pragma unroll
    for (int k = 0; k < R::E; ++k) {
      h[k] = (FIT == FEW ? me.counts(k) : me.has(k / R::VEC)) ? (h[k] - mean) * rstd : 0.f;  // (behind the last channel dy is zero, but this may be infinite)
      dgamma[k] = fmaf(dy[k], h[k], dgamma[k]);
      dbeta[k] += dy[k];
      dy[k] *= gamma[k];
      s1 += FIT != MOVED || me.counts(k) ? dy[k] : 0.f;
      s2 += FIT != MOVED || me.counts(k) ? dy[k] * h[k] : 0.f;
    }
    s1 = row_sum<G>(s1, lds) / c;
    s2 = row_sum<G>(s2, lds) / c;
    if (a.e) {
      float e[R::E];
      me.load(e, a.e, row, a.ld_e);
#pragma unroll
      for (int k = 0; k < R::E; ++k) dy[k] = fmaf(rstd, dy[k] - s1 - h[k] * s2, e[k]);
      if (G > 64 && FIT == MOVED) __syncthreads();  // (dx may lie over e)
    } else {
#pragma unroll
      for (int k = 0; k < R::E; ++k) dy[k] = rstd * (dy[k] - s1 - h[k] * s2);
    }
    me.store(dy, a.y, row, a.ld_y);
  }
  if (!a.partial) return;
  float* out = a.partial + int64_t(blockIdx.x) * (2 * a.c);
  if constexpr (G <= 64) {
    // the rows of a wave, then the waves one after the other
#pragma unroll
    for (int k = 0; k < R::E; ++k)
#pragma unroll
      for (int d = G; d < 64; d <<= 1) {
        dgamma[k] += __shfl_xor(dgamma[k], d, 64);
        dbeta[k] += __shfl_xor(dbeta[k], d, 64);
      }
    for (int w = 0; w < NORM_THREADS / 64; ++w) {
      if (int(threadIdx.x) / 64 == w && threadIdx.x % 64 < G)
#pragma unroll
        for (int k = 0; k < R::E; ++k)
          if (me.counts(k)) {
            const int at = me.channel(k);
            sums[at] = w ? sums[at] + dgamma[k] : dgamma[k];
            sums[a.c + at] = w ? sums[a.c + at] + dbeta[k] : dbeta[k];
          }
      __syncthreads();
    }
    for (int i = threadIdx.x; i < 2 * a.c; i += NORM_THREADS) out[i] = sums[i];
  } else {
#pragma unroll
    for (int k = 0; k < R::E; ++k)
      if (me.counts(k)) {
        const int at = me.channel(k);
        out[at] = dgamma[k];
        out[a.c + at] = dbeta[k];
      }
  }
}

// dgamma and dbeta from the workgroups' sums: 32 columns a workgroup, 32 shares of the rows added up in LDS.
__global__ __launch_bounds__(1024) void norm_params_kernel(const float* __restrict__ partial, int parts, int c, float* dgamma, float* dbeta) {
  __shared__ float lds[32][33];
  const int col = blockIdx.x * 32 + threadIdx.x % 32, share = threadIdx.x / 32;
  float s = 0.f;
  if (col < 2 * c) {
    const float* p = partial + col;
#pragma unroll 8
    for (int q = share; q < parts; q += 32) s += p[int64_t(q) * (2 * c)];
  }
  lds[share][threadIdx.x % 32] = s;
  __syncthreads();
  if (share || col >= 2 * c) return;
  s = 0.f;
#pragma unroll
  for (int q = 0; q < 32; ++q) s += lds[q][threadIdx.x];
  float* to = col < c ? dgamma : dbeta;
  if (to) to[col < c ? col : col - c] = s;
}

int norm_check(int64_t n, int32_t c, int32_t dtype) {
  if (dtype != SPC_DTYPE_F16 && dtype != SPC_DTYPE_BF16 && dtype != SPC_DTYPE_F32) return set_error(SPC_ERR_ARG, "unknown dtype %d", dtype);
  if (n < 0 || c < 1) return set_error(SPC_ERR_ARG, "n = %lld, c = %d", static_cast<long long>(n), c);
  if (c > NORM_MAX_C) return set_error(SPC_ERR_UNSUPPORTED, "rows of %d channels: at most %d", c, NORM_MAX_C);
  return SPC_OK;
}
int norm_check_rows(const char* what, const void* p, int64_t ld, int32_t c, int es, bool optional) {
  if (!p) return optional ? SPC_OK : set_error(SPC_ERR_ARG, "%s is NULL", what);
  if (ld < c) return set_error(SPC_ERR_ARG, "row pitch %lld of %s is below %d channels", static_cast<long long>(ld), what, c);
  if (reinterpret_cast<uintptr_t>(p) % es) return set_error(SPC_ERR_ARG, "%s is not aligned to its type", what);
  return SPC_OK;
}

// Calls f(NV, G, FIT) as integral constants for rows of c channels.  Up to 64 pieces one lane holds one; longer rows are held by whole waves with up to 32
// channels a lane, and beyond by whole workgroups.
template <typename T, typename F>
void norm_shape(int c, F&& f) {
  using std::integral_constant;
  constexpr int VEC = Piece<T>::VEC;
  const int pieces = (c + VEC - 1) / VEC;
  auto with = [&](auto nv, auto g) {
    if (c % VEC == 0) f(nv, g, integral_constant<Fit, WHOLE>{});
    else f(nv, g, integral_constant<Fit, MOVED>{});
  };
  if (c < VEC) return f(integral_constant<int, 1>{}, integral_constant<int, 4>{}, integral_constant<Fit, FEW>{});
#define SPC_NORM_CASE(NV, G) \
  if (NV * VEC <= 32 && pieces <= NV * G) return with(integral_constant<int, NV * VEC <= 32 ? NV : 1>{}, integral_constant<int, G>{})
  SPC_NORM_CASE(1, 4);
  SPC_NORM_CASE(1, 8);
  SPC_NORM_CASE(1, 16);
  SPC_NORM_CASE(1, 32);
  SPC_NORM_CASE(1, 64);
  SPC_NORM_CASE(2, 64);
  SPC_NORM_CASE(4, 64);
  SPC_NORM_CASE(8, 64);
  SPC_NORM_CASE(2, 256);
  SPC_NORM_CASE(4, 256);
  SPC_NORM_CASE(8, 256);
#undef SPC_NORM_CASE
}

// The grid: workgroups that 256 CUs hold at once, and no more than there are rows for.  The forward pass is short of registers nowhere (120 k x 256 fp16: 1024
// workgroups 43.3 us, 2048 42.6; 8000 x 8192 bf16: 51.8, 46.2).  The backward pass holds 8, 16 or 32 channels a lane several times over, and each workgroup stores
// sums: four to a CU, three, two (240 k x 256 bf16: 512 in all 125 us, 1024 97; 30 k x 1024: 512 46, 1024 58), of four turns each at least.
int norm_grid(int32_t dtype, int c, int64_t n, bool backward) {
  int64_t rows = 1, most = 2048;
  by_dtype(dtype, [&](auto t) {
    norm_shape<decltype(t)>(c, [&](auto nv, auto g, auto) {
      rows = NORM_THREADS / decltype(g)::value;
      constexpr int channels = decltype(nv)::value * Piece<decltype(t)>::VEC;
      if (backward) rows *= 4, most = channels <= 8 ? 1024 : channels <= 16 ? 768 : 512;
    });
  });
  return static_cast<int>(std::min(most, (n + rows - 1) / rows));
}
template <typename T>
void norm_forward(const NormArgs& a, int wgs, hipStream_t s) {
  norm_shape<T>(a.c, [&](auto nv, auto g, auto fit) {
    hipLaunchKernelGGL((norm_forward_kernel<T, decltype(nv)::value, decltype(g)::value, decltype(fit)::value>), dim3(wgs), dim3(NORM_THREADS), 0, s, a);
  });
}
template <typename T>
void norm_backward(const NormArgs& a, int wgs, hipStream_t s) {
  norm_shape<T>(a.c, [&](auto nv, auto g, auto fit) {
    constexpr int G = decltype(g)::value;
    hipLaunchKernelGGL((norm_backward_kernel<T, decltype(nv)::value, G, decltype(fit)::value>), dim3(wgs), dim3(NORM_THREADS), G <= 64 ? 8 * a.c : 0, s, a);
  });
}

}  // namespace
}  // namespace spc

extern "C" int spc_layer_norm_forward(const void* x, int64_t ld_x, const void* residual, int64_t ld_r, const float* gamma, const float* beta,
                                      float eps, void* y, int64_t ld_y, void* sum, int64_t ld_s, float* mean, float* rstd, int64_t n, int32_t c,
                                      int32_t dtype, void* stream) {
  using namespace spc;
  SPC_RETURN_IF(norm_check(n, c, dtype));
  const int es = dtype == SPC_DTYPE_F32 ? 4 : 2;
  SPC_RETURN_IF(norm_check_rows("x", x, ld_x, c, es, n == 0));
  SPC_RETURN_IF(norm_check_rows("y", y, ld_y, c, es, n == 0));
  SPC_RETURN_IF(norm_check_rows("residual", residual, ld_r, c, es, true));
  SPC_RETURN_IF(norm_check_rows("sum", sum, ld_s, c, es, true));
  if (!(eps > 0.f && eps < 3.4e38f)) return set_error(SPC_ERR_ARG, "eps must be positive and finite");
  if (n && !residual != !sum) return set_error(SPC_ERR_ARG, "residual and sum come together");
  if (n && !mean != !rstd) return set_error(SPC_ERR_ARG, "mean and rstd come together");
  if (!n) return SPC_OK;
  NormArgs a{};
  a.x = x, a.ld_x = ld_x, a.r = residual, a.ld_r = ld_r, a.gamma = gamma, a.beta = beta, a.eps = eps;
  a.y = y, a.ld_y = ld_y, a.z = sum, a.ld_z = ld_s, a.mean = mean, a.rstd = rstd, a.n = n, a.c = c;
  const int wgs = norm_grid(dtype, c, n, false);
  by_dtype(dtype, [&](auto t) { norm_forward<decltype(t)>(a, wgs, static_cast<hipStream_t>(stream)); });
  SPC_HIP_CHECK(hipGetLastError());
  return SPC_OK;
}

extern "C" int spc_layer_norm_backward(const void* dy, int64_t ld_dy, const void* x, int64_t ld_x, const float* mean, const float* rstd,
                                       const float* gamma, const void* dsum, int64_t ld_ds, void* dx, int64_t ld_dx, float* dgamma, float* dbeta,
                                       int64_t n, int32_t c, int32_t dtype, void* stream) {
  using namespace spc;
  SPC_RETURN_IF(norm_check(n, c, dtype));
  const int es = dtype == SPC_DTYPE_F32 ? 4 : 2;
  SPC_RETURN_IF(norm_check_rows("dy", dy, ld_dy, c, es, n == 0));
  SPC_RETURN_IF(norm_check_rows("x", x, ld_x, c, es, n == 0));
  SPC_RETURN_IF(norm_check_rows("dx", dx, ld_dx, c, es, n == 0));
  SPC_RETURN_IF(norm_check_rows("dsum", dsum, ld_ds, c, es, true));
  if (n && (!mean || !rstd)) return set_error(SPC_ERR_ARG, "mean or rstd is NULL");
  const StreamId s(static_cast<hipStream_t>(stream));
  const StreamWorkNote note{s};
  const bool params = dgamma || dbeta;
  NormArgs a{};
  a.dy = dy, a.ld_dy = ld_dy, a.x = x, a.ld_x = ld_x, a.mean_in = mean, a.rstd_in = rstd, a.gamma = gamma, a.e = dsum, a.ld_e = ld_ds;
  a.y = dx, a.ld_y = ld_dx, a.n = n, a.c = c;
  const int wgs = norm_grid(dtype, c, n, true);
  if (params && n) {
    a.partial = static_cast<float*>(pool_alloc(scratch_bytes(size_t(wgs) * 2 * c * sizeof(float)), s));
    if (!a.partial) return SPC_ERR_NOMEM;
  }
  if (n) by_dtype(dtype, [&](auto t) { norm_backward<decltype(t)>(a, wgs, s); });
  if (params)
    hipLaunchKernelGGL(norm_params_kernel, dim3((2 * c + 31) / 32), dim3(1024), 0, s, a.partial, n ? wgs : 0, c, dgamma, dbeta);
  pool_free(a.partial, s);
  SPC_HIP_CHECK(hipGetLastError());
  return SPC_OK;
}
