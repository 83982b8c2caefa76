// What the kernels over rows of features share: pieces of 16 bytes, and the choice of a kernel by the rows' type.
#pragma once
#include "spc_internal.h"

namespace spc {

// 16 and 8 bytes at any address of a 16-bit type.  (The target's vector loads and stores of global memory need no alignment.)
typedef int Words4 __attribute__((ext_vector_type(4)));
typedef int AnyWords4 __attribute__((ext_vector_type(4), aligned(2), may_alias));
typedef int Words2 __attribute__((ext_vector_type(2)));
typedef int AnyWords2 __attribute__((ext_vector_type(2), aligned(2), may_alias));

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

}  // namespace spc
