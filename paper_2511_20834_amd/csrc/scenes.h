// Scenes of rows that lie one behind the other, cut into segments that different workgroups take at once.
#pragma once
#include "rows.h"

namespace spc {

struct Scenes {
  const int32_t* offsets;  // n_scenes + 1, or NULL: one scene of all rows
  int n_rows, n_scenes, seg_rows;
  int ids() const { return n_rows / seg_rows + n_scenes; }  // more than every segment's number
};

// Segment `id` of all scenes.  Scene b's segments have the numbers lo(b) / seg_rows + b and following: floor(x) + floor(y) <= floor(x + y)
// keeps them apart, so no table is needed.  Offsets are clamped to the rows there are.  An empty scene has one segment of no rows.
struct SceneSegment {
  int scene, lo, hi, m, n, first, rows;  // the scene's rows [lo, hi), number m of n segments, its first row (of all rows) and their count
  __device__ bool find(const Scenes& a, int id) {
    auto start = [&](int b) { return a.offsets ? min(max(a.offsets[b], 0), a.n_rows) : b ? a.n_rows : 0; };
    int low = 0, high = a.n_scenes;  // the last scene whose numbers start at or before id lies in [low, high)
    while (high - low > 1) {
      const int mid = (low + high) / 2;
      if (start(mid) / a.seg_rows + mid <= id) low = mid;
      else high = mid;
    }
    scene = low;
    lo = start(low);
    hi = max(start(low + 1), lo);
    m = id - (lo / a.seg_rows + low);
    n = hi > lo ? (hi - lo - 1) / a.seg_rows + 1 : 1;
    if (m < 0 || m >= n) return false;
    first = lo + m * a.seg_rows;
    rows = min(a.seg_rows, hi - first);
    return true;
  }
  // The same values in scalar registers: every lane has found the same segment.
  __device__ void uniform() {
    for (int* v : {&scene, &lo, &hi, &m, &n, &first, &rows}) *v = __builtin_amdgcn_readfirstlane(*v);
  }
};

// What calls over scenes check of their offsets and counts.
inline int check_scenes(const int32_t* offsets, int64_t n_rows, int32_t n_scenes) {
  if (n_rows < 0 || n_scenes < 1) return set_error(SPC_ERR_ARG, "%lld rows, %d scenes", static_cast<long long>(n_rows), n_scenes);
  if (!offsets && n_scenes != 1) return set_error(SPC_ERR_ARG, "%d scenes without offsets", n_scenes);
  // (numbers of rows and of a segment's more are held in 32 bits)
  if (n_rows > (int64_t(1) << 31) - 65536 || n_scenes > 200000)
    return set_error(SPC_ERR_UNSUPPORTED, "%lld rows in %d scenes: at most 2^31 - 65536 and 200000", static_cast<long long>(n_rows), n_scenes);
  return SPC_OK;
}

// 1 / (1 + e^-x) and friends.  EXACT: for fp32 rows, the exponent's product in two parts (one rounding of it would be |x| 2^-24 of the result).
template <bool EXACT>
__device__ inline float exp_of(float x) {
  constexpr float L = 1.44269504f, REST = 1.92596299e-8f;  // log2(e)
  const float h = x * L;
  if (!EXACT) return __builtin_amdgcn_exp2f(h);
  const float e = __builtin_amdgcn_exp2f(h), l = fmaf(x, REST, fmaf(x, L, -h));
  return fabsf(h) < 128.f ? fmaf(e * l, .69314718f, e) : e;  // (2^l = 1 + l ln 2; infinite powers keep out: times a rest below zero they would give NaN)
}
template <bool EXACT>
__device__ inline float sigmoid_of(float x) {
  return __builtin_amdgcn_rcpf(1.f + exp_of<EXACT>(-x));
}

}  // namespace spc
