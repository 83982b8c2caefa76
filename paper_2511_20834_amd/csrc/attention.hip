// Linear attention with a decay for each head, over the rows of scenes that lie one behind the other.
//
//   S_t = l S_{t-1} + k_t v_t^T,   o_t = a S_t^T q_t,   l = exp(log_decay[head]),  a = scale
//
// The gradients are the same recurrence over other operands, with time running backward for k and v:
//   dq: x = do, y = v, z = k       dv: x = k, y = q, z = do, backward       dk: x = v, y = do, z = q, backward
// so everything below is one scan  S <- l S + y z^T, out = S^T x  of a `Job`, with the factor a on the output where S is the caller's state
// and on the products y z^T where S is a state's gradient.
//
// A scene is cut into segments that different workgroups scan at once: a first launch makes every segment's own sum of y z^T, a second
// turns them into the state in front of every segment, a third scans the segments.  Scenes of one segment take the third alone.
//
// Bytes bound large calls: the sums read k and v (for gradients q and the output's gradient as well), which are read again by the third launch, so a forward
// pass moves 6 tensors for the 4 it cannot do without, a backward pass 11 for 7.  Measured, us a pass among others (in brackets the latter at a copy's
// 4.84 TB/s): 120 k rows, 8 heads of 64, fp16 209 (102), its gradients in bf16 406 (178); 240 k rows, 4 heads of 32, bf16, with states 109 (51).  A row at a time
// through LDS, the first version, took 7033, 13 343 and 3575.  Of the 209 (launches traced alone, the fastest of 12): sums 64 (51 for their bytes), states
// 10, outputs 131 (102).  In the gradients' third launch (285, with 4 tensors read once for its three jobs, 178) the vector unit issues in 55 % of the CUs' busy
// cycles, the matrix cores work in 26 %, LDS in 36 %: three waves to a SIMD wait for each other's fragments and barriers.  Small calls are bound by three launches: 2118 rows, 4 heads of 16, fp32 18.7, of which the kernels take 5.0, 6.0 and 7.6 and an empty one 2.4.
#include <algorithm>
#include <cmath>
#include <type_traits>

#include "rows.h"

namespace spc {
namespace {

constexpr int ATTN_MAX_D = 128;
constexpr int ATTN_MAX_JOBS = 3;
constexpr int64_t ATTN_MAX_SCENE_HEADS = 200000;

struct Rows {
  void* p;
  int64_t row, head;  // pitches
  int group;          // consecutive heads of the scan that share one head of the tensor
  __device__ int64_t at(int64_t r, int h) const { return r * row + int64_t(h / group) * head; }
};
// A matrix of every (index, head): rows of y times columns of z, by pitches.
struct States {
  float* p;
  int64_t each;
  int r, c;
  __device__ float* of(int64_t index, int heads, int h) const { return p + (index * heads + h) * each; }
};
struct Job {
  Rows x, y, z, out;
  States first, last, between;  // of a scene, after it, after every segment but the last
  int dy, dz;
  bool reverse, out_f32;
};
struct ScanArgs {
  Job job[ATTN_MAX_JOBS];
  const float* log_decay;
  const int32_t* offsets;  // n_scenes + 1, or NULL: one scene of all rows
  int n_rows, n_scenes, heads, n_jobs;
  int seg_rows, n_ids;
  int n_cols;  // workgroups that share a head's columns of z
  float scale;
  bool keep;  // whether a state is returned
};

// Segment `id` of all scenes.  Scene b's segments have the numbers lo(b) / seg_rows + b and following: floor(x) + floor(y) <= floor(x + y)
// keeps them apart, so no table is needed, and there are at most n_rows / seg_rows + n_scenes.  Offsets are clamped to the rows there are.
struct Segment {
  int scene, lo, hi, m, n, rows;  // the scene's rows [lo, hi), number m of n segments, its length
  __device__ bool find(const ScanArgs& a, int id) {
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
    n = hi > lo ? (hi - lo - 1) / a.seg_rows + 1 : 1;  // (a scene's rows and a segment's more may pass 32 bits)
    rows = min(a.seg_rows, hi - lo - m * a.seg_rows);
    return m >= 0 && m < n;
  }
  __device__ int64_t row(bool reverse, int i) const { return reverse ? int64_t(hi) - 1 - i : int64_t(lo) + i; }
};

// 2^(g n), n >= 0 (g: the decay's logarithm to base 2, perhaps -infinity)
__device__ inline float decay_power(float g, int n) { return n > 0 ? __builtin_amdgcn_exp2f(g * n) : 1.f; }

__device__ inline float uniform(float v) { return __builtin_bit_cast(float, __builtin_amdgcn_readfirstlane(__builtin_bit_cast(int, v))); }

// l^n for a state that takes it many times: in two parts where l^n is near 1, since its rounding, the same every time, would add up over a long memory.  Both are
// positive: a state that is infinite stays so.  (e^x - 1 by its series: the terms left out are below 2^-28.)
struct Decay {
  float most, rest;
  __device__ explicit Decay(float l) : most(.5f * l), rest(.5f * l) {}
  __device__ Decay(float log_decay, float g, int n) : Decay(decay_power(g, n)) {
    const float x = log_decay * n;
    if (fabsf(x) < .25f) {
      float e = 1.f;
#pragma unroll
      for (int k = 7; k > 1; --k) e = fmaf(e, x * (1.f / k), 1.f);
      e *= x;
      most = __builtin_bit_cast(float, __builtin_bit_cast(int, 1.f + e) - 1);  // the number below
      rest = (1.f - most) + e;
    }
    most = uniform(most), rest = uniform(rest);
  }
  template <typename V>
  __device__ V of(V s, V more) const {
    return s * most + (s * rest + more);
  }
};

// Up to four consecutive channels (`left` of them exist).
template <typename T>
__device__ inline void store4(T* p, float __attribute__((ext_vector_type(4))) v, int left) {
  typedef T Values __attribute__((ext_vector_type(4)));
  const Values q = __builtin_convertvector(v, Values);
  if (left >= 4) {
    if constexpr (sizeof(T) == 2) *reinterpret_cast<AnyWords2*>(p) = __builtin_bit_cast(Words2, q);
    else *reinterpret_cast<AnyWords4*>(p) = __builtin_bit_cast(Words4, q);
    return;
  }
#pragma unroll
  for (int r = 0; r < 3; ++r)
    if (r < left) p[r] = q[r];
}

// ---------------------------------------------------------------- chunks on the matrix cores
typedef _Float16 half8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float floatx8 __attribute__((ext_vector_type(8)));
typedef float floatx4 __attribute__((ext_vector_type(4)));
typedef short shortx4 __attribute__((ext_vector_type(4)));
typedef int intx4 __attribute__((ext_vector_type(4)));

constexpr int CHUNK = 64;  // rows whose products with each other are taken directly

// Tiles in LDS have rows of D channels in pieces of 16 bytes, whose order is another in every row: piece q of row r lies at q ^ turn(r), which spreads lanes that
// read pieces of different rows over the banks without padding.  Chosen by the conflicts counted for the four kinds of access below, of seven such orders (extra cycles a
// wave, D = 64 of 16 bits: rows read along 0, written 4, tile stored 0, columns 0; 32: 0, 4, 0, 0; 128: 0, 4, 0, 2; fp32 64 and 128: none; 32: 4, 0, 0, 0).
template <typename T, int D>
struct Tile {
  static constexpr int VE = 16 / sizeof(T), PIECES = D / VE;
  __device__ static inline int turn(int r) { return PIECES == 4 ? (r >> 1) & 3 : r & (PIECES < 16 ? PIECES - 1 : 15); }  // (of the row modulo 16)
  __device__ static inline int at(int r, int c) { return r * D + ((c / VE ^ turn(r)) * VE + c % VE); }
};

// A fragment holds 32 places of a contraction for 16 rows (A) or columns (B): lane l has row l%16 and the places 16 h + 4 (l/16) + r, h < 2, r < 4,
// as element 4 h + r.  The results of two 16 x 16 products, whose lane l holds column l%16 and rows 4 (l/16) + r, are one as they come: sums of
// products go from one product into the next without passing through LDS.
template <typename T>
struct Ops {
  using V = std::conditional_t<std::is_same_v<T, _Float16>, half8, bf16x8>;
  using LDS4 = __attribute__((address_space(3))) shortx4*;
  __device__ static inline floatx4 mma(V a, V b, floatx4 c) {
    if constexpr (std::is_same_v<T, _Float16>) return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0);
    else return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
  }
  __device__ static inline V both(shortx4 a, shortx4 b) { return __builtin_bit_cast(V, __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7)); }
};
template <>
struct Ops<float> {
  using V = floatx8;
  __device__ static inline floatx4 mma(V a, V b, floatx4 c) {
#pragma unroll
    for (int k = 0; k < 8; ++k) c = __builtin_amdgcn_mfma_f32_16x16x4f32(a[k], b[k], c, 0, 0, 0);
    return c;
  }
};
// Fragments of a tile whose places lie along its rows: row l%16 (of 16 that start at a multiple of 16), 32 places from 32 k on.  Read, a lane holds
// the eight places from 8 (l/16) on: both operands of a product do.  Written as it comes out of a product, it holds those above.  (Channels that are
// multiples of a piece, or two, change other bits of a place than the lane does.)
template <typename T, int D>
struct Along {
  using V = typename Ops<T>::V;
  int at, to;
  __device__ Along(int lane) : at(Tile<T, D>::at(lane % 16, lane / 16 * 8)), to(Tile<T, D>::at(lane % 16, lane / 16 * 4)) {}
  __device__ void renew() { asm volatile("" : "+v"(at), "+v"(to)); }  // (the places made of these before are not to be kept in registers)
  __device__ V get(const T* rows, int k) const {
    if constexpr (sizeof(T) == 2) return *reinterpret_cast<const V*>(rows + (at ^ 32 * k));
    else return __builtin_shufflevector(*reinterpret_cast<const floatx4*>(rows + (at ^ 32 * k)), *reinterpret_cast<const floatx4*>(rows + (at ^ (32 * k + 4))), 0,
                                        1, 2, 3, 4, 5, 6, 7);
  }
  __device__ void put(T* rows, int k, V f) const {
    T *p = rows + (to ^ 32 * k), *q = rows + (to ^ (32 * k + 16));
    if constexpr (sizeof(T) == 2) {
      typedef short shortx8 __attribute__((ext_vector_type(8)));
      const shortx8 v = __builtin_bit_cast(shortx8, f);
      *reinterpret_cast<shortx4*>(p) = __builtin_shufflevector(v, v, 0, 1, 2, 3);
      *reinterpret_cast<shortx4*>(q) = __builtin_shufflevector(v, v, 4, 5, 6, 7);
    } else {
      *reinterpret_cast<floatx4*>(p) = __builtin_shufflevector(f, f, 0, 1, 2, 3);
      *reinterpret_cast<floatx4*>(q) = __builtin_shufflevector(f, f, 4, 5, 6, 7);
    }
  }
};
// Fragments whose places lie down its columns: column l%16 of the 16 from c on, rows from a multiple of 32 on.  (16-bit types: sixteen lanes read
// four rows of sixteen, and each receives a column of them.)
template <typename T, int D>
struct Down {
  using V = typename Ops<T>::V;
  static constexpr int N = sizeof(T) == 2 ? 1 : 4;
  int at[N];
  __device__ Down(int lane) {
    if constexpr (sizeof(T) == 2) at[0] = Tile<T, D>::at(lane / 16 * 4 + lane % 16 / 4, lane % 4 * 4);
    else
#pragma unroll
      for (int r = 0; r < 4; ++r) at[r] = Tile<T, D>::at(lane / 16 * 4 + r, lane % 16);
  }
  __device__ void renew() {
#pragma unroll
    for (int r = 0; r < N; ++r) asm volatile("" : "+v"(at[r]));
  }
  __device__ V get(const T* rows, int c) const {
    if constexpr (sizeof(T) == 2) {
      using P = typename Ops<T>::LDS4;
      const T* p = rows + (at[0] ^ c);
      return Ops<T>::both(__builtin_amdgcn_ds_read_tr16_b64_v4i16((P)(p)), __builtin_amdgcn_ds_read_tr16_b64_v4i16((P)(p + 16 * D)));
    } else {
      V f;
#pragma unroll
      for (int k = 0; k < 8; ++k) f[k] = rows[k / 4 * 16 * D + (at[k % 4] ^ c)];
      return f;
    }
  }
};
// x as a sum of N fragments: each holds what the ones before have left of it, times 2^(SHIFT * its number).
template <typename T, int N, int SHIFT = 0>
__device__ inline void split(floatx8 x, typename Ops<T>::V (&out)[N]) {
  if constexpr (N == 1) {
    out[0] = x;
  } else {
#pragma unroll
    for (int n = 0; n < N; ++n) {
      out[n] = __builtin_convertvector(x, typename Ops<T>::V);
      if (n + 1 == N) break;
      // (what is left is left by the value that the product takes: without this the compiler rounds it twice, once of an unrounded
      // product by a conversion that multiplies, and the two differ now and then)
      intx4 q = __builtin_bit_cast(intx4, out[n]);
      asm("" : "+v"(q));
      out[n] = __builtin_bit_cast(typename Ops<T>::V, q);
      x -= __builtin_convertvector(out[n], floatx8);
      if (SHIFT) x *= float(1 << SHIFT);
    }
  }
}
// fp16's pieces of values of which the largest in this lane is m: times 2^-e for the e returned, e the same in the four lanes of a column (a row of A), the largest of all
// is below 2^15 and no less than half of it.  The second piece goes up by 2^11 more (`split`), so what is lost of a value is 2^-51 of that largest one however small it is
// itself: decays, and features of unlike rows, set values of one row of a product many powers of two apart.
constexpr int HALF_TOP = 15, HALF_SHIFT = 11;
__device__ inline int half_exponent(float m) {
  m = fmaxf(m, __shfl_xor(m, 16, 64));
  m = fmaxf(m, __shfl_xor(m, 32, 64));
  return max(__builtin_amdgcn_frexp_expf(m), -100) - HALF_TOP;
}

// A chunk's rows of one tensor on their way from memory to LDS.  A segment's last chunk, where it is not full, lies in the tile's last rows; the rows in
// front of it, and channels behind the head's last, are zeros.  Heads of whole pieces of 16 bytes, at any address, are in registers while the chunk before is
// worked on; others are read channel by channel when they are due.
template <typename T, int D>
struct TileLoad {
  static constexpr int VE = 16 / sizeof(T), PER_ROW = D / VE, STEP = 256 / PER_ROW, N = CHUNK / STEP;
  static constexpr bool ONCE = STEP % 16 == 0;  // a thread's rows have the same order of pieces
  intx4 q[N];
  const T* origin;  // channel 0 of the columns, row 0 of the next chunk
  int64_t row;      // the next row of the scan
  int width;        // channels of these columns that there are
  bool pieces;
  __device__ void start(const Rows& t, int first_channel, int channels, const Segment& s, bool reverse, int seg_first, int h) {
    width = min(channels - first_channel, D);
    pieces = channels % VE == 0;
    row = reverse ? -t.row : t.row;
    origin = static_cast<const T*>(t.p) + (h / t.group) * t.head + s.row(reverse, seg_first) * t.row + first_channel;
  }
  __device__ void load(int rows) {
    const int i = threadIdx.x / PER_ROW, c = threadIdx.x % PER_ROW * VE, shift = max(CHUNK - rows, 0);
    origin -= shift * row;
    if (!pieces) return;
    const T* at = origin + (i * row + c);
    if (!shift && width == D) {
#pragma unroll
      for (int n = 0; n < N; ++n, at += STEP * row) q[n] = *reinterpret_cast<const AnyWords4*>(at);
      return;
    }
#pragma unroll
    for (int n = 0; n < N; ++n, at += STEP * row) {
      q[n] = intx4{0, 0, 0, 0};
      if (i + n * STEP >= shift && c < width) q[n] = *reinterpret_cast<const AnyWords4*>(at);
    }
  }
  __device__ void store(T* tile, int shift) {
    if (pieces) {
      const int i = threadIdx.x / PER_ROW, c = threadIdx.x % PER_ROW * VE;
      T* to = tile + Tile<T, D>::at(i, c);
#pragma unroll
      for (int n = 0; n < N; ++n) *reinterpret_cast<intx4*>(ONCE ? to + n * STEP * D : tile + Tile<T, D>::at(i + n * STEP, c)) = q[n];
    } else {
      int e = threadIdx.x;
      asm volatile("" : "+v"(e));  // (no places of this loop are kept in registers from chunk to chunk)
#pragma unroll 4
      for (; e < CHUNK * D; e += 256) {
        const int r = e / D, c = e % D;
        tile[Tile<T, D>::at(r, c)] = r >= shift && c < width ? origin[r * row + c] : T(0.f);
      }
    }
    origin += CHUNK * row;
  }
};

template <typename T, int DY, int DZ, bool OUT>
constexpr size_t scan_lds() {
  return sizeof(T) * (CHUNK * (DY + DZ) + (OUT ? CHUNK * DY + (sizeof(T) == 2 ? 2 : 1) * DZ * DY : 0)) + (OUT && std::is_same_v<T, _Float16> ? sizeof(float) * DZ : 0);
}

// Workgroups (a wave on every SIMD) that a CU holds, by registers and LDS.
template <typename T, int DY, int DZ>
constexpr int scan_waves() {
  if (DY == 128) return sizeof(T) == 4 ? 1 : 2;
  return sizeof(T) == 4 && DY == 64 ? 2 : sizeof(T) == 2 && DY == 32 && DZ == 32 ? 4 : 3;
}

// One segment of one head and DZ columns of z: chunk by chunk, with the state in registers.
//   O^T = Z^T P^T + S^T X^T,  P^T = (Y X^T) o l^(i-j),   S <- l^n S + Y^T (w o Z)
// Each of the four waves makes 16 rows of the chunk's output, whose products P^T are the next product's operand as they lie in its registers, and (DZ / 16 of
// them) keeps 16 columns of the state, which all waves read from LDS as the pieces they multiply.
// Operands that are no inputs (P, S, w o Z) go into 16-bit products as two pieces, the weighted values of bf16 as three where the state is returned: 16 bits of every sum that is
// rounded to a 16-bit output in the end, 24 (fp16: 22) of what the state adds up.  fp16's pieces are scaled by powers of two, P by the largest of a row, S and w o Z by
// the largest of a column, since sums leave its range upwards and decays downwards (120 k rows, 8 heads of 64: 204 us, gradients 446; with pieces of P and S that lose what lies
// 2^-25 below the largest, and of w o Z below 2^-36, 200 and 431).  fp32 takes fp32 products.
template <typename T, int DY, int DZ, bool OUT>
__global__ __launch_bounds__(256, (scan_waves<T, DY, DZ>())) void scan_chunks_kernel(const ScanArgs a) {
  using O = Ops<T>;
  using V = typename O::V;
  constexpr bool HALF = std::is_same_v<T, _Float16>, SINGLE = std::is_same_v<T, float>;
  constexpr int NP = SINGLE ? 1 : 2, NU = SINGLE ? 1 : HALF ? 2 : 3;  // pieces of P and S, of the weighted values
  constexpr int SHIFT = HALF ? HALF_SHIFT : 0;
  constexpr int CT = DZ / 16, DT = DY / 16, KT = DY / 32, IT = CHUNK / 16, JT = CHUNK / 32;
  extern __shared__ __align__(16) char lds[];
  T *ys = reinterpret_cast<T*>(lds), *zs = ys + CHUNK * DY, *xs = zs + CHUNK * DZ, *sp = xs + CHUNK * DY;
  float* s_scale = reinterpret_cast<float*>(sp + NP * DZ * DY);  // by column, of the pieces of S

  // workgroups that follow each other go to the eight XCDs in turn: neighbours of one segment share an L2 this way
  const int total = a.n_ids * a.heads * a.n_jobs * a.n_cols, share = (total + 7) / 8, work = blockIdx.x % 8 * share + blockIdx.x / 8;
  if (work >= total) return;
  const Job& j = a.job[work / a.n_cols % a.n_jobs];
  const int h = work / a.n_cols / a.n_jobs % a.heads, id = work / a.n_cols / a.n_jobs / a.heads;
  const int col0 = work % a.n_cols * DZ, dz = j.dz - col0;
  if (dz <= 0) return;
  Segment s;
  if (!s.find(a, id)) return;
  if (!OUT && s.m == s.n - 1) return;  // nobody starts from it
  const int lane = threadIdx.x % 64, lc = lane % 16, lr = lane / 16 * 4, seg_first = s.m * a.seg_rows;
  // (which rows and columns are a wave's changes from workgroup to workgroup: the waves of a SIMD have unlike shares of the work)
  const int it = __builtin_amdgcn_readfirstlane((threadIdx.x / 64 + work) % 4), ct_s = (it + 2) % 4;
  const bool owner = ct_s < CT;
  const bool special = j.reverse && !s.m;  // the gradient of the last state meets the last row undecayed
  const float g = a.log_decay[h] * 1.44269504f;
  const float p_scale = a.scale, upd = j.reverse ? a.scale : 1.f, inter = j.reverse ? 1.f : a.scale;

  TileLoad<T, DY> x, y;
  TileLoad<T, DZ> z;
  if (OUT) x.start(j.x, 0, j.dy, s, j.reverse, seg_first, h);
  y.start(j.y, 0, j.dy, s, j.reverse, seg_first, h);
  z.start(j.z, col0, j.dz, s, j.reverse, seg_first, h);
  auto fetch = [&](int rows) {
    if (OUT) x.load(rows);
    y.load(rows);
    z.load(rows);
  };
  if (s.rows > 0) fetch(s.rows);

  floatx4 S[DT];
  {
    const bool from = OUT && owner && (s.m || j.first.p);
    const States& st = s.m ? j.between : j.first;
    const float* p = from ? st.of(s.m ? id - 1 : s.scene, a.heads, h) : nullptr;
    const int col = 16 * ct_s + lc;
#pragma unroll
    for (int dt = 0; dt < DT; ++dt)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const int row = 16 * dt + lr + r;
        S[dt][r] = from && row < j.dy && col < dz ? p[row * st.r + (col0 + col) * st.c] : 0.f;
        __builtin_amdgcn_sched_barrier(0);  // (few addresses at a time)
      }
  }
  // decays: of P (on the diagonal, and below it as a product of two; its columns are rows 16 it + lc of the chunk), and of a row's product on the way into
  // the state, as a product of two
  float w_same[4], w[4], w_tile[IT - 1], u[4], u_tile[IT];
#pragma unroll
  for (int r = 0; r < 4; ++r) {
    w_same[r] = p_scale * decay_power(g, lc - lr - r);  // (above the diagonal: not used)
    w[r] = p_scale * decay_power(g, 15 + lc - lr - r);
    u[r] = decay_power(g, 15 - lr - r);
    u_tile[r] = uniform((HALF ? 1.f : upd) * decay_power(g, 48 - 16 * r));
    if (r + 1 < IT) w_tile[r] = uniform(decay_power(g, 16 * r + 1));
  }
  const float f_full = inter * decay_power(g, 16 * it + lc + 1);
  const Decay whole_full(a.log_decay[h], g, CHUNK);
  const bool out_f32 = j.out_f32;
  const int es = out_f32 ? 4 : sizeof(T);
  const int64_t out_row = (j.reverse ? -j.out.row : j.out.row) * es;
  char* out = nullptr;  // row 16 it + lc of the chunk, channel lr of these columns
  if (OUT) out = static_cast<char*>(j.out.p) + (j.out.at(s.row(j.reverse, seg_first), h) + col0 + lr) * es + (16 * it + lc) * out_row;
  const bool out_whole = !out_f32 && dz >= DZ;
  const bool keep = a.keep;
  Along<T, DY> along(lane);
  Down<T, DY> down_y(lane);
  Down<T, DZ> down_z(lane);

#pragma unroll 1
  for (int first = 0; first < s.rows; first += CHUNK) {
    const int n = min(CHUNK, s.rows - first), shift = CHUNK - n, e0 = special && !first ? 0 : 1;
    along.renew(), down_y.renew(), down_z.renew();
    int here = lane;
    asm volatile("" : "+v"(here));
    const int lc = here % 16, lr = here / 16 * 4;
    __syncthreads();
    y.store(ys, shift);
    z.store(zs, shift);
    if constexpr (OUT) {
      x.store(xs, shift);
      if (owner) {
        float down = 1.f;
        if constexpr (HALF) {
          float m = 0.f;
#pragma unroll
          for (int dt = 0; dt < DT; ++dt)
#pragma unroll
            for (int r = 0; r < 4; ++r) m = fmaxf(m, fabsf(S[dt][r]));
          const int e = half_exponent(m);
          down = ldexpf(1.f, -e);
          if (lane < 16) s_scale[16 * ct_s + lc] = ldexpf(1.f, e);
        }
#pragma unroll
        for (int k = 0; k < KT; ++k) {
          floatx8 v = __builtin_shufflevector(S[2 * k], S[2 * k + 1], 0, 1, 2, 3, 4, 5, 6, 7);
          if constexpr (HALF) {
#pragma unroll
            for (int q = 0; q < 8; ++q) v[q] *= down;
          }
          V f[NP];
          split<T, NP, SHIFT>(v, f);
#pragma unroll
          for (int q = 0; q < NP; ++q) along.put(sp + (q * DZ + 16 * ct_s) * DY, k, f[q]);
        }
      }
    }
    __syncthreads();
    if (first + CHUNK < s.rows) fetch(s.rows - first - CHUNK);
    if constexpr (OUT) {
      // rows 16 IT_ + lc of the chunk
      auto output = [&](auto rows) {
        constexpr int IT_ = decltype(rows)::value, JN = IT_ / 2 + 1;
        const int i = 16 * IT_ + lc;
        V xf[KT];
#pragma unroll
        for (int k = 0; k < KT; ++k) xf[k] = along.get(xs + 16 * IT_ * DY, k);
        floatx8 P[JN];
        float m = 0.f;
#pragma unroll
        for (int jt = 0; jt < 2 * JN; ++jt) {
          floatx4 p = {0.f, 0.f, 0.f, 0.f};
          if (jt <= IT_) {
#pragma unroll
            for (int k = 0; k < KT; ++k) p = O::mma(along.get(ys + 16 * jt * DY, k), xf[k], p);
#pragma unroll
            for (int r = 0; r < 4; ++r) {
              p[r] *= jt < IT_ ? w[r] * w_tile[IT_ - jt - 1] : w_same[r];
              if (jt == IT_ && lr + r > lc) p[r] = 0.f;
              if constexpr (HALF) m = fmaxf(m, fabsf(p[r]));
            }
          }
#pragma unroll
          for (int r = 0; r < 4; ++r) P[jt / 2][jt % 2 * 4 + r] = p[r];
        }
        float p_up = 1.f;
        if constexpr (HALF) {
          const int e = half_exponent(m);
          const float down = ldexpf(1.f, -e);
          p_up = ldexpf(1.f, e);
#pragma unroll
          for (int t = 0; t < JN; ++t)
#pragma unroll
            for (int k = 0; k < 8; ++k) P[t][k] *= down;
        }
        V pf[JN][NP];
#pragma unroll
        for (int t = 0; t < JN; ++t) split<T, NP, SHIFT>(P[t], pf[t]);
        __builtin_amdgcn_sched_barrier(0);  // (here and below: fragments are read when they are due, few registers have to do)
        const float f = shift || !e0 ? inter * decay_power(g, i - shift + e0) : f_full;
        floatx4 o[CT];
#pragma unroll
        for (int ct = 0; ct < CT; ++ct) {
          o[ct] = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
          for (int q = NP - 1; q >= 0; --q) {
#pragma unroll
            for (int k = 0; k < KT; ++k) o[ct] = O::mma(along.get(sp + (q * DZ + 16 * ct) * DY, k), xf[k], o[ct]);
            if (HALF && q) o[ct] *= 1.f / (1 << SHIFT);
          }
          if constexpr (HALF) o[ct] *= *reinterpret_cast<const floatx4*>(s_scale + 16 * ct + lr);
          o[ct] *= f;
          __builtin_amdgcn_sched_barrier(0);
        }
        bool some = false;  // whether an output is NaN
#pragma unroll
        for (int ct = 0; ct < CT; ++ct) {
          floatx4 v = {0.f, 0.f, 0.f, 0.f};
          if constexpr (!HALF) v = o[ct];
          V zf[JN];
#pragma unroll
          for (int t = 0; t < JN; ++t) zf[t] = down_z.get(zs + 32 * t * DZ, 16 * ct);
#pragma unroll
          for (int q = NP - 1; q >= 0; --q) {
#pragma unroll
            for (int t = 0; t < JN; ++t) v = O::mma(zf[t], pf[t][q], v);
            if (HALF && q) v *= 1.f / (1 << SHIFT);
          }
          if constexpr (HALF) o[ct] += v * p_up;
          else o[ct] = v;
          some |= __builtin_isunordered(o[ct][0], o[ct][1]) | __builtin_isunordered(o[ct][2], o[ct][3]);
        }
        char* at = out - shift * out_row;
        auto put = [&](int ct, floatx4 v) {
          if (i < shift) return;
          if (out_f32) store4(reinterpret_cast<float*>(at) + 16 * ct, v, dz - 16 * ct - lr);
          else store4(reinterpret_cast<T*>(at) + 16 * ct, v, dz - 16 * ct - lr);
        };
        if (out_whole && !shift) {
#pragma unroll
          for (int ct = 0; ct < CT; ++ct) store4(reinterpret_cast<T*>(at) + 16 * ct, o[ct], 4);
        } else {
#pragma unroll
          for (int ct = 0; ct < CT; ++ct) put(ct, o[ct]);
        }
        // Zero times infinity is NaN: where a value is not finite, the zeros of P above the diagonal have brought it to earlier rows.  Outputs that are not numbers are
        // computed once more from their own pairs alone (unless the state has made them so), and replaced.
        if (!__ballot(some)) return;
        unsigned nan = 0;
#pragma unroll
        for (int ct = 0; ct < CT; ++ct)
#pragma unroll
          for (int r = 0; r < 4; ++r) nan |= o[ct][r] != o[ct][r] ? 1u << (4 * ct + r) : 0u;
        if (i < shift) return;
#pragma unroll 1
        for (int b = 0; b < 4 * CT; ++b) {
          const int c = b / 4 * 16 + lr + b % 4;
          if (!(nan >> b & 1) || c >= dz) continue;
          double v = 0;
#pragma unroll 1
          for (int d = 0; d < j.dy; ++d) {
            float st = static_cast<float>(sp[Tile<T, DY>::at(c, d)]);
            if (NP > 1) st += static_cast<float>(sp[DZ * DY + Tile<T, DY>::at(c, d)]) * (1.f / (1 << SHIFT));
            v += double(static_cast<float>(xs[Tile<T, DY>::at(i, d)])) * (HALF ? st * s_scale[c] : st);
          }
          v *= f;
          if (v != v) continue;
#pragma unroll 1
          for (int q = 0; q <= i; ++q) {
            double pq = 0;
#pragma unroll 1
            for (int d = 0; d < j.dy; ++d)
              pq += double(static_cast<float>(xs[Tile<T, DY>::at(i, d)])) * static_cast<float>(ys[Tile<T, DY>::at(q, d)]);
            v += pq * (p_scale * decay_power(g, i - q)) * static_cast<float>(zs[Tile<T, DZ>::at(q, c)]);
          }
          const int place = c - lr;
          if (out_f32) reinterpret_cast<float*>(at)[place] = static_cast<float>(v);
          else reinterpret_cast<T*>(at)[place] = static_cast<T>(static_cast<float>(v));
        }
      };
      if (16 * it + 15 >= shift) {
        if (it == 0) output(std::integral_constant<int, 0>{});
        else if (it == 1) output(std::integral_constant<int, 1>{});
        else if (it == 2) output(std::integral_constant<int, 2>{});
        else output(std::integral_constant<int, 3>{});
      }
      out += CHUNK * out_row;
    }
    if (owner) {
      V uf[JT][NU];
      floatx8 U[JT];
#pragma unroll
      for (int t = 0; t < JT; ++t) {
        U[t] = __builtin_convertvector(down_z.get(zs + 32 * t * DZ, 16 * ct_s), floatx8);
#pragma unroll
        for (int k = 0; k < 8; ++k) U[t][k] *= u[k % 4] * u_tile[2 * t + k / 4];
      }
      float u_up = upd;
      if constexpr (HALF) {
        float m = 0.f;
#pragma unroll
        for (int t = 0; t < JT; ++t)
#pragma unroll
          for (int k = 0; k < 8; ++k) m = fmaxf(m, fabsf(U[t][k]));
        const int e = half_exponent(m);
        const float down = ldexpf(1.f, -e);
        u_up *= ldexpf(1.f, e);
#pragma unroll
        for (int t = 0; t < JT; ++t)
#pragma unroll
          for (int k = 0; k < 8; ++k) U[t][k] *= down;
      }
#pragma unroll
      for (int t = 0; t < JT; ++t) split<T, NU, SHIFT>(U[t], uf[t]);
      const Decay whole = shift || !e0 ? Decay(uniform(decay_power(g, n - 1 + e0))) : whole_full;
      // Products are added up apart and go to the state once a chunk: added to it one by one, each would round it, and a long memory takes many (fp32, 18 k rows a
      // scene, 8 heads of 48: 7.7e-7 of the outputs off, 2.9e-7 so).  A state of bf16 that nobody keeps, rounded to 16 bits a chunk later, takes that, and two pieces:
      // 120 k rows, 8 heads of 64, gradients 399 us for 416.
      auto update = [&](auto exact) {
#pragma unroll
        for (int dt = 0; dt < DT; ++dt) {
          V yf[JT];
#pragma unroll
          for (int t = 0; t < JT; ++t) yf[t] = down_y.get(ys + 32 * t * DY, 16 * dt);
          floatx4 v = {0.f, 0.f, 0.f, 0.f};
          if constexpr (!exact) v = S[dt] * (whole.most + whole.rest);
#pragma unroll
          for (int q = exact ? NU - 1 : 1; q >= 0; --q) {
#pragma unroll
            for (int t = 0; t < JT; ++t) v = O::mma(yf[t], uf[t][q], v);
            if (HALF && q) v *= 1.f / (1 << SHIFT);
          }
          if constexpr (HALF) v *= u_up;
          S[dt] = exact ? whole.of(S[dt], v) : v;
        }
      };
      if constexpr (NU == 3) {
        if (keep) update(std::true_type{});
        else update(std::false_type{});
      } else update(std::true_type{});
    }
  }
  const States& to = OUT ? j.last : j.between;
  if (!owner || (OUT && (s.m != s.n - 1 || !to.p))) return;
  const float f = OUT && j.reverse && s.hi > s.lo ? decay_power(g, 1) : 1.f;  // (what reaches the state before the first row)
  int there = lane;  // (places are not those of the load above, kept over the chunks)
  asm volatile("" : "+v"(there));
  const int col = 16 * ct_s + there % 16;
  float* p = to.of(OUT ? s.scene : id, a.heads, h) + int64_t(col0 + col) * to.c;
#pragma unroll
  for (int dt = 0; dt < DT; ++dt)
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const int row = 16 * dt + there / 16 * 4 + r;
      if (row < j.dy && col < dz) p[row * to.r] = f * S[dt][r];
    }
}

// Sums of segments -> the state behind every segment but the last of its scene, in place.
__global__ __launch_bounds__(256) void scan_states_kernel(const ScanArgs a) {
  const Job& j = a.job[blockIdx.y];
  const int share = (j.dy * j.dz + 255) / 256, sh = blockIdx.x / share, h = sh % a.heads, scene = sh / a.heads;
  const int i = (blockIdx.x - sh * share) * 256 + threadIdx.x;
  if (i >= j.dy * j.dz) return;
  const int lo = a.offsets ? min(max(a.offsets[scene], 0), a.n_rows) : 0;
  const int id = lo / a.seg_rows + scene;
  Segment s;
  if (!s.find(a, id) || s.scene != scene) return;
  const int r = i / j.dz, c = i % j.dz;
  float S = j.first.p ? j.first.of(scene, a.heads, h)[r * j.first.r + c * j.first.c] : 0.f;
  const float g = a.log_decay[h] * 1.44269504f;
  const Decay whole(a.log_decay[h], g, a.seg_rows), first = j.reverse ? Decay(decay_power(g, a.seg_rows - 1)) : whole;
  const int64_t step = a.heads * j.between.each;
  float* p = j.between.of(id, a.heads, h) + r * j.between.r + c * j.between.c;
  constexpr int AHEAD = 32;  // (the loads of a chain's links do not depend on each other)
  for (int m = 0; m + 1 < s.n; m += AHEAD) {
    float v[AHEAD];
#pragma unroll
    for (int q = 0; q < AHEAD; ++q) v[q] = m + q + 1 < s.n ? p[q * step] : 0.f;
#pragma unroll
    for (int q = 0; q < AHEAD; ++q) {
      if (m + q + 1 >= s.n) break;
      S = (m + q ? whole : first).of(S, v[q]);
      p[q * step] = S;
    }
    p += AHEAD * step;
  }
}

// Gradients of keys and values that `group` heads share: sums over the heads, of [row][head][channel] each.  Rows from the first scene's first to the last one's last:
// the scan makes the parts of no others.
struct HeadSums {
  const float* part;
  Rows out;
  int d;
};
template <typename T>
__global__ __launch_bounds__(256) void sum_heads_kernel(HeadSums k, HeadSums v, const int32_t* offsets, int n_scenes, int n_rows, int kv_heads, int group) {
  const int lo = offsets ? min(max(offsets[0], 0), n_rows) : 0, hi = offsets ? min(max(offsets[n_scenes], lo), n_rows) : n_rows;
  const int64_t first = int64_t(lo) * kv_heads, row_heads = int64_t(hi) * kv_heads - first, nk = row_heads * k.d, n = nk + row_heads * v.d;
  for (int64_t at = blockIdx.x * int64_t(256) + threadIdx.x; at < n; at += gridDim.x * int64_t(256)) {
    const bool second = at >= nk;
    const HeadSums a = second ? v : k;
    const int64_t i = second ? at - nk : at, rh = first + i / a.d, row = rh / kv_heads;
    const int c = static_cast<int>(i - (rh - first) * a.d);
    const float* p = a.part + rh * group * a.d + c;
    float s = 0.f;
#pragma unroll 4
    for (int g = 0; g < group; ++g) s += p[int64_t(g) * a.d];
    static_cast<T*>(a.out.p)[row * a.out.row + (rh - row * kv_heads) * a.out.head + c] = static_cast<T>(s);
  }
}

// One row more: a workgroup updates one head's state of one stream, S <- l S + k v^T, and adds up its columns times q on the way.  Every value of the state is read and
// written once, in pieces of VEC columns (4; 1 where the columns are no multiple of it) whose loads are all under way before the first is used; the bytes bound it
// (2048 streams of 8 heads of 64 x 64, fp16: 99 us for 546 MB, 5.5 TB/s; one stream 9.8, the host's call).  Neighbouring lanes have neighbouring pieces of a row, 2^log_q places of which hold one.
template <typename T, int VEC>
__global__ __launch_bounds__(256) void attention_step_kernel(Rows q, Rows k, Rows v, Rows out, float* state, const float* log_decay, int heads, int dk, int dv,
                                                             float scale, int log_q) {
  typedef float Values __attribute__((ext_vector_type(VEC), aligned(4), may_alias));
  constexpr int AHEAD = 8;
  __shared__ float qs[ATTN_MAX_D], ks[ATTN_MAX_D], part[256 * VEC];
  const int h = blockIdx.x % heads, t = threadIdx.x, c = (t & ((1 << log_q) - 1)) * VEC, step = blockDim.x >> log_q;
  const int64_t row = blockIdx.x / heads;
  float* S = state + int64_t(blockIdx.x) * dk * dv + c;
  Values s[AHEAD];
  auto load = [&](int r0) {
#pragma unroll
    for (int a = 0; a < AHEAD; ++a)
      if (r0 + a * step < dk && c < dv) s[a] = *reinterpret_cast<const Values*>(S + (r0 + a * step) * dv);
  };
  load(t >> log_q);
  for (int i = t; i < dk; i += blockDim.x) {
    qs[i] = scale * static_cast<float>(static_cast<const T*>(q.p)[q.at(row, h) + i]);
    ks[i] = static_cast<float>(static_cast<const T*>(k.p)[k.at(row, h) + i]);
  }
  Values vc, o;
#pragma unroll
  for (int e = 0; e < VEC; ++e) {
    vc[e] = c < dv ? static_cast<float>(static_cast<const T*>(v.p)[v.at(row, h) + c + e]) : 0.f;
    o[e] = 0.f;
  }
  const float g = log_decay[h];
  const Decay l(g, g * 1.44269504f, 1);  // (a stream takes it every row: one rounding of it drifts, 20 k rows at a decay of -1/4096 by 1e-4 of the state)
  __syncthreads();
  for (int r0 = t >> log_q; r0 < dk; r0 += AHEAD * step) {
    if (r0 >= AHEAD * step) load(r0);
#pragma unroll
    for (int a = 0; a < AHEAD; ++a) {
      const int r = r0 + a * step;
      if (r < dk && c < dv) {
        const float kr = ks[r], qr = qs[r];
#pragma unroll
        for (int e = 0; e < VEC; ++e) {
          s[a][e] = l.of(s[a][e], kr * vc[e]);
          o[e] = fmaf(qr, s[a][e], o[e]);
        }
        *reinterpret_cast<Values*>(S + r * dv) = s[a];
      }
    }
  }
#pragma unroll
  for (int e = 0; e < VEC; ++e) part[t * VEC + e] = o[e];
  __syncthreads();
  for (int i = t; i < dv; i += blockDim.x) {
    float sum = 0.f;
    for (int g = 0; g < step; ++g) sum += part[(g * VEC << log_q) + i];
    static_cast<T*>(out.p)[out.at(row, h) + i] = static_cast<T>(sum);
  }
}

template <typename KeyT>
__global__ __launch_bounds__(256) void batch_offsets_kernel(const KeyT* __restrict__ keys, int n, int sh_b, int n_batch, int32_t* out) {
  const int b = blockIdx.x * 256 + threadIdx.x;
  if (b > n_batch) return;
  int low = 0, high = n;  // first row of scene b or a later one
  while (low < high) {
    const int mid = low + (high - low) / 2;
    // (a key without batch bits belongs to scene 0; the shift by all bits of a type is undefined)
    const uint64_t scene = sh_b < 64 ? static_cast<uint64_t>(keys[mid]) >> sh_b : 0;
    if (scene < static_cast<uint64_t>(b)) low = mid + 1;
    else high = mid;
  }
  out[b] = low;
}

// ---------------------------------------------------------------- host
int check_desc(const spc_attn_desc* d, bool scenes = true) {  // (without `scenes` their number is not read)
  if (!d) return set_error(SPC_ERR_ARG, "descriptor is NULL");
  if (d->dtype != SPC_DTYPE_F16 && d->dtype != SPC_DTYPE_BF16 && d->dtype != SPC_DTYPE_F32)
    return set_error(SPC_ERR_ARG, "unknown dtype %d", d->dtype);
  if (d->n_rows < 0 || (scenes && d->n_scenes < 1) || d->heads < 1 || d->kv_heads < 1 || d->heads % d->kv_heads || d->dk < 1 || d->dv < 1)
    return set_error(SPC_ERR_ARG, "%lld rows, %d scenes, %d heads over %d, %d and %d channels", static_cast<long long>(d->n_rows), scenes ? d->n_scenes : 1,
                     d->heads, d->kv_heads, d->dk, d->dv);
  if (!(d->scale > -3.4e38f && d->scale < 3.4e38f)) return set_error(SPC_ERR_ARG, "scale is not finite");
  if (d->dk > ATTN_MAX_D || d->dv > ATTN_MAX_D) return set_error(SPC_ERR_UNSUPPORTED, "heads of %d and %d channels: at most %d", d->dk, d->dv, ATTN_MAX_D);
  // (a launch takes less than 2^32 threads, 64 workgroups of 256 of them to a scene and head; a segment's rows grow with all rows)
  if (d->n_rows >= (int64_t(1) << 31) || (scenes && int64_t(d->n_scenes) * d->heads > ATTN_MAX_SCENE_HEADS))
    return set_error(SPC_ERR_UNSUPPORTED, "%lld rows of %d heads in %d scenes", static_cast<long long>(d->n_rows), d->heads, scenes ? d->n_scenes : 1);
  return SPC_OK;
}
// Pitches of an input may be zero (broadcast); places of an output are its own.
int check_rows(const char* what, const spc_attn_rows* t, const spc_attn_desc* d, int heads, int width, bool output) {
  if (!t || !t->data) return set_error(SPC_ERR_ARG, "%s is NULL", what);
  if (reinterpret_cast<uintptr_t>(t->data) % (d->dtype == SPC_DTYPE_F32 ? 4 : 2)) return set_error(SPC_ERR_ARG, "%s is not aligned to its type", what);
  const int64_t row = t->row_pitch, head = t->head_pitch, far = int64_t(1) << 40;
  bool ok = row >= 0 && head >= 0 && row < far && head < far;
  if (output && ok) {
    const bool one_row = d->n_rows <= 1, one_head = heads == 1;
    ok = (one_row || row >= width) && (one_head || head >= width) &&
         (one_row || one_head || row >= (heads - 1) * head + width || head >= (d->n_rows - 1) * row + width);
  }
  return ok ? SPC_OK : set_error(SPC_ERR_ARG, "pitches %lld and %lld of %s do not fit %d heads of %d channels", static_cast<long long>(row),
                                 static_cast<long long>(head), what, heads, width);
}
Rows rows_of(const spc_attn_rows* t, int group) { return {t->data, t->row_pitch, t->head_pitch, group}; }

// Calls f(type, DY, DZ) with the kernels' tile widths for rows of y of dy channels and of z of dz.
template <typename F>
void by_shape(int32_t dtype, int dy, int dz, F&& f) {
  by_dtype(dtype, [&](auto t) {
    auto with = [&](auto w) {
      if (dz <= 32) f(t, w, std::integral_constant<int, 32>{});
      else f(t, w, std::integral_constant<int, 64>{});
    };
    if (dy <= 32) with(std::integral_constant<int, 32>{});
    else if (dy <= 64) with(std::integral_constant<int, 64>{});
    else with(std::integral_constant<int, 128>{});
  });
}

// Rows of a segment, a multiple of 64: as few as give the workgroups that 256 CUs hold at once (twice as many workgroups: 120 k rows, 8 heads of 64, bf16 203 us, not
// 196), but not so few that the chain of a scene's segments takes longer than a segment, which balances at some 64 sqrt(rows / 1200) (us, segments of 64 / 128 / 256
// rows: 2118 rows, 4 heads of 16, fp32 18.0 / 20.6 / 29.2; 6011 rows, 8 heads of 64, bf16 33.4 / 29.5 / 29.0; 12 k rows, 4 heads of 32 27.6 / 23.5 / 24.6).
int segment_rows(const spc_attn_desc* d, int dy, int dz) {
  int64_t at_once = 256;
  by_shape(d->dtype, dy, dz, [&](auto t, auto y, auto z) {
    constexpr int width = decltype(z)::value;
    at_once = 256 * scan_waves<decltype(t), decltype(y)::value, width>() / ((dz + width - 1) / width);
  });
  const int64_t fill = (d->n_rows * d->heads + at_once - 1) / at_once;
  const double chain = std::sqrt(double(d->n_rows) / d->n_scenes / 1200);
  return static_cast<int>(64 * std::max<int64_t>({1, (fill + 63) / 64, std::llround(chain)}));
}

template <typename T, int DY, int DZ>
int launch_scan(ScanArgs& a, int n_sums, hipStream_t s) {
  int dz = 0;
  for (int q = 0; q < a.n_jobs; ++q) dz = std::max(dz, a.job[q].dz);
  a.n_cols = (dz + DZ - 1) / DZ;
  auto grid = [&] { return dim3((a.n_ids * a.heads * a.n_jobs * a.n_cols + 7) / 8 * 8); };
  if (a.n_rows > a.seg_rows) {
    const int jobs = a.n_jobs;
    a.n_jobs = n_sums;
    hipLaunchKernelGGL((scan_chunks_kernel<T, DY, DZ, false>), grid(), dim3(256), (scan_lds<T, DY, DZ, false>()), s, a);
    hipLaunchKernelGGL(scan_states_kernel, dim3((a.job[0].dy * a.job[0].dz + 255) / 256 * a.n_scenes * a.heads, n_sums), dim3(256), 0, s, a);
    a.n_jobs = jobs;
  }
  constexpr size_t lds = scan_lds<T, DY, DZ, true>();
  if constexpr (lds > 64 * 1024) {
    static const hipError_t attr = hipFuncSetAttribute(reinterpret_cast<const void*>(&scan_chunks_kernel<T, DY, DZ, true>),
                                                       hipFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(lds));
    SPC_HIP_CHECK(attr);
  }
  hipLaunchKernelGGL((scan_chunks_kernel<T, DY, DZ, true>), grid(), dim3(256), lds, s, a);
  return SPC_OK;
}

// The states between segments are made for the first n_sums jobs; the jobs behind them share theirs.
int run_scan(ScanArgs& a, int n_sums, int32_t dtype, hipStream_t s) {
  int dy = 0, dz = 0, rc = SPC_OK;
  for (int q = 0; q < a.n_jobs; ++q) dy = std::max(dy, a.job[q].dy), dz = std::max(dz, a.job[q].dz);
  by_shape(dtype, dy, dz, [&](auto t, auto y, auto z) {
    rc = launch_scan<decltype(t), decltype(y)::value, decltype(z)::value>(a, n_sums, s);
  });
  SPC_RETURN_IF(rc);
  SPC_HIP_CHECK(hipGetLastError());
  return SPC_OK;
}

}  // namespace
}  // namespace spc

extern "C" int spc_linear_attention_forward(const spc_attn_desc* d, const spc_attn_rows* q, const spc_attn_rows* k, const spc_attn_rows* v,
                                            const float* log_decay, const int32_t* offsets, const float* state_in, const spc_attn_rows* out,
                                            float* state_out, void* stream) {
  using namespace spc;
  SPC_RETURN_IF(check_desc(d));
  if (!log_decay) return set_error(SPC_ERR_ARG, "log_decay is NULL");
  if (!offsets && d->n_scenes != 1) return set_error(SPC_ERR_ARG, "%d scenes without offsets", d->n_scenes);
  if (d->n_rows) {
    SPC_RETURN_IF(check_rows("q", q, d, d->heads, d->dk, false));
    SPC_RETURN_IF(check_rows("k", k, d, d->kv_heads, d->dk, false));
    SPC_RETURN_IF(check_rows("v", v, d, d->kv_heads, d->dv, false));
    SPC_RETURN_IF(check_rows("out", out, d, d->heads, d->dv, true));
  } else if (!q || !k || !v || !out) {
    return set_error(SPC_ERR_ARG, "NULL argument");
  }
  const StreamId s(static_cast<hipStream_t>(stream));
  const StreamWorkNote note{s};
  const int group = d->heads / d->kv_heads;
  const int64_t e = int64_t(d->dk) * d->dv;
  ScanArgs a{};
  Job& j = a.job[0];
  j.x = rows_of(q, 1), j.y = rows_of(k, group), j.z = rows_of(v, group), j.out = rows_of(out, 1);
  j.dy = d->dk, j.dz = d->dv;
  j.first = {const_cast<float*>(state_in), e, d->dv, 1};
  j.last = {state_out, e, d->dv, 1};
  a.log_decay = log_decay, a.offsets = offsets, a.n_rows = static_cast<int>(d->n_rows), a.n_scenes = d->n_scenes, a.heads = d->heads, a.n_jobs = 1;
  a.scale = d->scale;
  a.keep = state_out != nullptr;
  a.seg_rows = segment_rows(d, d->dk, d->dv);
  a.n_ids = a.n_rows / a.seg_rows + a.n_scenes;
  float* ws = nullptr;
  if (a.n_rows > a.seg_rows) {
    ws = static_cast<float*>(pool_alloc(scratch_bytes(size_t(a.n_ids) * a.heads * e * sizeof(float)), s));
    if (!ws) return SPC_ERR_NOMEM;
  }
  j.between = {ws, e, d->dv, 1};
  const int rc = run_scan(a, 1, d->dtype, s);
  pool_free(ws, s);
  return rc;
}

extern "C" int spc_linear_attention_backward(const spc_attn_desc* d, const spc_attn_rows* dout, const spc_attn_rows* q, const spc_attn_rows* k,
                                             const spc_attn_rows* v, const float* log_decay, const int32_t* offsets, const float* state_in,
                                             const float* dstate_out, const spc_attn_rows* dq, const spc_attn_rows* dk, const spc_attn_rows* dv,
                                             float* dstate_in, void* stream) {
  using namespace spc;
  SPC_RETURN_IF(check_desc(d));
  if (!log_decay) return set_error(SPC_ERR_ARG, "log_decay is NULL");
  if (!offsets && d->n_scenes != 1) return set_error(SPC_ERR_ARG, "%d scenes without offsets", d->n_scenes);
  if (d->n_rows) {
    SPC_RETURN_IF(check_rows("dout", dout, d, d->heads, d->dv, false));
    SPC_RETURN_IF(check_rows("q", q, d, d->heads, d->dk, false));
    SPC_RETURN_IF(check_rows("k", k, d, d->kv_heads, d->dk, false));
    SPC_RETURN_IF(check_rows("v", v, d, d->kv_heads, d->dv, false));
    SPC_RETURN_IF(check_rows("dq", dq, d, d->heads, d->dk, true));
    SPC_RETURN_IF(check_rows("dk", dk, d, d->kv_heads, d->dk, true));
    SPC_RETURN_IF(check_rows("dv", dv, d, d->kv_heads, d->dv, true));
  } else if (!dout || !q || !k || !v || !dq || !dk || !dv) {
    return set_error(SPC_ERR_ARG, "NULL argument");
  }
  const StreamId s(static_cast<hipStream_t>(stream));
  const StreamWorkNote note{s};
  const int group = d->heads / d->kv_heads;
  const int64_t e = int64_t(d->dk) * d->dv;
  ScanArgs a{};
  a.log_decay = log_decay, a.offsets = offsets, a.n_rows = static_cast<int>(d->n_rows), a.n_scenes = d->n_scenes, a.heads = d->heads, a.n_jobs = 3;
  a.scale = d->scale;
  a.keep = dstate_in != nullptr;
  a.seg_rows = segment_rows(d, std::max(d->dk, d->dv), std::max(d->dk, d->dv));
  a.n_ids = a.n_rows / a.seg_rows + a.n_scenes;
  const size_t states = a.n_rows > a.seg_rows ? size_t(a.n_ids) * a.heads * e : 0;
  const size_t parts = group > 1 ? size_t(a.n_rows) * a.heads : 0;  // gradients of shared keys and values, by head
  float* ws = nullptr;
  if (states || parts) {
    ws = static_cast<float*>(pool_alloc(scratch_bytes((2 * states + parts * (d->dk + d->dv)) * sizeof(float)), s));
    if (!ws) return SPC_ERR_NOMEM;
  }
  float *part_k = ws + 2 * states, *part_v = part_k + parts * d->dk;
  auto part = [&](float* p, int w) { return Rows{p, int64_t(a.heads) * w, w, 1}; };
  // the sums of do q^T serve dk as they are and dv transposed
  Job &jq = a.job[0], &jk = a.job[1], &jv = a.job[2];
  jq.x = rows_of(dout, 1), jq.y = rows_of(v, group), jq.z = rows_of(k, group), jq.out = rows_of(dq, 1);
  jq.dy = d->dv, jq.dz = d->dk;
  jq.first = {const_cast<float*>(state_in), e, 1, d->dv};
  jq.between = {ws, e, d->dk, 1};
  jk.x = rows_of(v, group), jk.y = rows_of(dout, 1), jk.z = rows_of(q, 1), jk.out = group > 1 ? part(part_k, d->dk) : rows_of(dk, 1);
  jk.dy = d->dv, jk.dz = d->dk;
  jk.first = {const_cast<float*>(dstate_out), e, 1, d->dv};
  jk.between = {ws + states, e, d->dk, 1};
  jv.x = rows_of(k, group), jv.y = rows_of(q, 1), jv.z = rows_of(dout, 1), jv.out = group > 1 ? part(part_v, d->dv) : rows_of(dv, 1);
  jv.dy = d->dk, jv.dz = d->dv;
  jv.first = {const_cast<float*>(dstate_out), e, d->dv, 1};
  jv.between = {ws + states, e, 1, d->dk};
  jv.last = {dstate_in, e, d->dv, 1};
  jk.reverse = jv.reverse = true;
  jk.out_f32 = jv.out_f32 = group > 1;
  int rc = run_scan(a, 2, d->dtype, s);
  if (rc == SPC_OK && parts) {
    by_dtype(d->dtype, [&](auto t) {
      using T = decltype(t);
      const int64_t n = int64_t(a.n_rows) * d->kv_heads * (d->dk + d->dv);
      hipLaunchKernelGGL(sum_heads_kernel<T>, dim3(std::min<int64_t>((n + 255) / 256, 16384)), dim3(256), 0, s, HeadSums{part_k, rows_of(dk, 1), d->dk},
                         HeadSums{part_v, rows_of(dv, 1), d->dv}, offsets, d->n_scenes, a.n_rows, d->kv_heads, group);
    });
    const hipError_t err = hipGetLastError();
    if (err != hipSuccess) rc = set_error(SPC_ERR_HIP, "launch failed: %s", hipGetErrorString(err));
  }
  pool_free(ws, s);
  return rc;
}

extern "C" int spc_linear_attention_step(const spc_attn_desc* d, const spc_attn_rows* q, const spc_attn_rows* k, const spc_attn_rows* v,
                                         const float* log_decay, float* state, const spc_attn_rows* out, void* stream) {
  using namespace spc;
  SPC_RETURN_IF(check_desc(d, false));
  if (d->n_rows * d->heads >= (int64_t(1) << 24)) return set_error(SPC_ERR_UNSUPPORTED, "%lld streams of %d heads", static_cast<long long>(d->n_rows), d->heads);
  if (!log_decay) return set_error(SPC_ERR_ARG, "log_decay is NULL");
  if (!d->n_rows) return SPC_OK;
  if (!state) return set_error(SPC_ERR_ARG, "state is NULL");
  SPC_RETURN_IF(check_rows("q", q, d, d->heads, d->dk, false));
  SPC_RETURN_IF(check_rows("k", k, d, d->kv_heads, d->dk, false));
  SPC_RETURN_IF(check_rows("v", v, d, d->kv_heads, d->dv, false));
  SPC_RETURN_IF(check_rows("out", out, d, d->heads, d->dv, true));
  const int group = d->heads / d->kv_heads;
  const int vec = d->dv % 4 ? 1 : 4;
  int log_q = 0, threads = 64;
  while ((vec << log_q) < d->dv) ++log_q;
  while (threads < 256 && threads * 4 * vec < d->dk * d->dv) threads *= 2;  // (some four pieces a lane)
  by_dtype(d->dtype, [&](auto t) {
    using T = decltype(t);
    auto go = [&](auto kernel) {
      hipLaunchKernelGGL(kernel, dim3(d->n_rows * d->heads), dim3(std::max(threads, 1 << log_q)), 0, static_cast<hipStream_t>(stream), rows_of(q, 1), rows_of(k, group),
                         rows_of(v, group), rows_of(out, 1), state, log_decay, d->heads, d->dk, d->dv, d->scale, log_q);
    };
    if (vec == 4) go(attention_step_kernel<T, 4>);
    else go(attention_step_kernel<T, 1>);
  });
  SPC_HIP_CHECK(hipGetLastError());
  return SPC_OK;
}

extern "C" int spc_batch_offsets(const void* keys, int64_t n, const spc_pack_desc* d, int32_t n_batch, int32_t* offsets, void* stream) {
  using namespace spc;
  PackInfo pi;
  if (!d || !offsets) return set_error(SPC_ERR_ARG, "NULL argument");
  SPC_RETURN_IF(spc::check_desc(d, &pi));
  if (n < 0 || n >= (int64_t(1) << 31) || n_batch < 1 || n_batch > (1 << 30) || (n && !keys)) return set_error(SPC_ERR_ARG, "%lld keys of %d scenes", static_cast<long long>(n), n_batch);
  const int sh = pi.bits_b ? pi.sh_b : 64;
  const dim3 grid((n_batch + 256) / 256);
  if (pi.key_bits == 32)
    hipLaunchKernelGGL(batch_offsets_kernel<uint32_t>, grid, dim3(256), 0, static_cast<hipStream_t>(stream), static_cast<const uint32_t*>(keys),
                       static_cast<int>(n), sh, n_batch, offsets);
  else
    hipLaunchKernelGGL(batch_offsets_kernel<uint64_t>, grid, dim3(256), 0, static_cast<hipStream_t>(stream), static_cast<const uint64_t*>(keys),
                       static_cast<int>(n), sh, n_batch, offsets);
  SPC_HIP_CHECK(hipGetLastError());
  return SPC_OK;
}
