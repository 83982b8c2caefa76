// What the kernels over rows of features share: pieces of 16 bytes, and the choice of a kernel by the rows' type.
#pragma once
#include "spc_internal.h"

namespace spc {

// 16 and 8 bytes at any address of a 16-bit type.  (The target's vector loads and stores of global memory need no alignment.)
typedef int Words4 __attribute__((ext_vector_type(4)));
typedef int AnyWords4 __attribute__((ext_vector_type(4), aligned(2), may_alias));
typedef int Words2 __attribute__((ext_vector_type(2)));
typedef int AnyWords2 __attribute__((ext_vector_type(2), aligned(2), may_alias));

// 8 and 4 bytes at any address.
typedef int AnyBytes8 __attribute__((ext_vector_type(2), aligned(1), may_alias));
typedef int AnyBytes4 __attribute__((aligned(1), may_alias));

template <typename F>
void by_dtype(int32_t dtype, F&& f) {
  if (dtype == SPC_DTYPE_F16) f(_Float16{});
  else if (dtype == SPC_DTYPE_BF16) f(__bf16{});
  else f(0.f);
}

// Scratch of about so many bytes: a quarter of a power of two at a time above 1 MiB, so that calls of many sizes share the cache's blocks.
inline size_t scratch_bytes(size_t bytes) {
  size_t step = size_t(1) << 18;
  while (step * 8 <= bytes) step *= 2;
  return bytes <= (size_t(1) << 20) ? bytes : (bytes + step - 1) / step * step;
}

// Sums of the workgroups' parts, column by column in a fixed order: parts x (cols[0] + cols[1] + cols[2]) floats into as many vectors (NULL: left out).
struct ColumnSums {
  float* to[3];
  int cols[3];
};
namespace {
__global__ __launch_bounds__(1024) void column_sums_kernel(ColumnSums out, const float* __restrict__ parts, int n) {
  __shared__ float lds[32][33];  // 32 columns a workgroup, 32 shares of the rows added up in LDS
  int col = blockIdx.x * 32 + threadIdx.x % 32;
  const int share = threadIdx.x / 32, cols = out.cols[0] + out.cols[1] + out.cols[2];
  float s = 0.f;
  if (col < cols) {
    const float* p = parts + col;
#pragma unroll 8
    for (int q = share; q < n; q += 32) s += p[int64_t(q) * cols];
  }
  lds[share][threadIdx.x % 32] = s;
  __syncthreads();
  if (share || col >= cols) return;
  s = 0.f;
#pragma unroll
  for (int q = 0; q < 32; ++q) s += lds[q][threadIdx.x];
  int v = 0;
  while (v < 2 && col >= out.cols[v]) col -= out.cols[v++];
  if (out.to[v]) out.to[v][col] = s;
}
inline void column_sums(const ColumnSums& out, const float* parts, int n, hipStream_t s) {
  const int cols = out.cols[0] + out.cols[1] + out.cols[2];
  hipLaunchKernelGGL(column_sums_kernel, dim3((cols + 31) / 32), dim3(1024), 0, s, out, parts, n);
}
}  // namespace

}  // namespace spc
