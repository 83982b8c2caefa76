// Selective state space scan of every channel along the rows of its scene, forward and backward, and one row of many streams.
//
//   d_t = softplus(dt_t + bias),  h_t = exp(d_t A) h_{t-1} + d_t u_t B_t  (N states a channel),  y_t = C_t . h_t + D u_t,  out_t = y_t silu(gate_t)
//
// Backward, with dy = dout silu(gate), q the gradient of a state and a_t = exp(d_t A):
//
//   q_t = C_t dy_t + a_{t+1} q_{t+1},  dC_t = sum over channels of h_t dy_t,  dB_t = sum over channels of q_t d_t u_t,  x_t = sum over states of q_t B_t,
//   du_t = d_t x_t + D dy_t,  p_t = q_t a_t h_{t-1},  dd_t = u_t x_t + sum over states of A p_t,  dA = sum over rows of d_t p_t
//
// A lane has a channel and keeps its states in registers, so that a row is one wide load for 64 channels; B and C are the same for all lanes: a first launch
// writes them as floats, which arrive through scalar loads.  A scene is cut into segments: one launch makes every segment's own state (from zeros) and its sum of d, a
// second chains them (a segment's decay is exp(A sum d)), the last scans the segments from the states in front of them.
//
// The vector unit bounds it: a state and row take an exponential (as long as three products) and three products or sums in the sums, four in the outputs, a row some thirty
// instructions more for step size and gate.  120 k rows of 512 channels of 16 states, bf16, us (share of the CUs' cycles in which the vector unit issues, an instruction counted as four
// cycles): 439, for 105 that the bytes take once at a copy's 4.76 TB/s and 141 for the exponentials and
// products of one pass.  Gradients 1172, bytes 184.  Fastest dispatches under a profiler, which add up to a tenth more
// than a pass without one: B and C 14, sums 190 (98 %), chain 30, outputs 246 (95 %); gradients: B and C 14, sums both ways 309 (92 %), chain 21, the way back 860 (87 %), dB and dC 27,
// parameters 8.
// Small calls wait for launches and memory: 2118 rows of 64 channels, fp32, 28, in launches of some 2.5, 7, 11.3, 7.  First version, a row's loads where they are used: 653 and 2780.
#include <algorithm>
#include <cmath>
#include <type_traits>

#include "scenes.h"

namespace spc {
namespace {

constexpr int SCAN_MAX_N = 64;
constexpr int SCAN_MAX_C = 65536;
constexpr int SCAN_THREADS = 256;  // four waves of segments and blocks of their own (a CU takes no more than 16 workgroups of one wave: four to a SIMD do not fill it)
// Rows whose states are held in registers while the gradient runs back over them, and states of a lane meanwhile: four waves a row of up to 16 states, so that each has fewer of
// the rows' other work; 64 states in eight waves of eight would not fit 16 rows.
constexpr int grad_rows(int np) { return np <= 32 ? 16 : 8; }
constexpr int grad_states(int np) { return np <= 16 ? np / 4 : np <= 32 ? 4 : 8; }
constexpr float LOG2E = 1.44269504f;

struct LowRows {  // B or C: channel j of group g in row r is r * row + g * group + j
  void* p;
  int64_t row, group;
};

struct ScanArgs {
  Scenes scenes;
  const void *u, *dt, *gate, *dout;
  void *out, *ddt, *dgate;  // out: backward du
  int64_t ld_u, ld_dt, ld_gate, ld_dout, ld_out, ld_ddt, ld_dgate;
  LowRows b, c, db, dc;
  const float *A, *skip, *bias;
  const float *state_in, *dstate_out;
  float *state_out, *dstate_in;
  float* low;      // [row][group][16 states at a time][B, C], NP states in all, a row of zeros behind the last one
  float* between;  // [segment][NP][channels]: its state from zeros, then the state behind it
  float* behind;   // the same for the gradient: what reaches the rows in front of a segment, from zeros, then what arrives from behind it
  float* steps;    // [segment][channels]: sum of d
  // [slot][NP + 1][channels]: a segment's state from zeros in front of every grad_rows rows but its first, and the sum of d up to there.  Its slots begin at
  // first row / grad_rows + its number (as segments are numbered in their scenes, so do slots of segments stay apart).
  float* starts;
  float* parts;    // [segment][NP + 2][channels]: dA, dD, dbias
  float* low_parts;  // [block of channels][row][B, C][NP], where several blocks share a group
  int channels, groups, share, N, blocks, ids;  // share: channels of a group; blocks: of 64 channels, of all groups
  bool softplus;
};

typedef const __attribute__((address_space(4))) float* Scalars;  // (read through the scalar cache: nothing writes there while the kernel runs)

// Step sizes.  ln(1 + e) of e = exp(-|raw|): w = 1 + e rounds e off by c, which comes back as c / w (1/w by a line: c is below 2^-24).  Off by 2^-22 at most, measured from
// -16 to 16.
template <typename T>
struct Step {
  float d, slope;  // d and its derivative
  __device__ Step(float raw, bool softplus) {
    const float e = exp_of<sizeof(T) == 4>(-fabsf(raw)), w = 1.f + e, c = e - (w - 1.f), r = __builtin_amdgcn_rcpf(w);
    const float soft = fmaxf(raw, 0.f) + fmaf(__builtin_amdgcn_logf(w), .69314718f, c * fmaf(-.5f, w, 1.5f));  // (NaN where raw is: e is)
    d = softplus ? soft : raw;  // (no branch, which would part the rows of an unrolled loop)
    slope = softplus ? (raw >= 0.f ? r : e * r) : 1.f;
  }
};

// A lane's channel in block `block` of all channels.
struct Lane {
  int channel, group;
  bool some;
  __device__ Lane(const ScanArgs& a, int block, int lane) {
    const int per = a.blocks / a.groups;
    group = block / per;
    const int i = (block - group * per) * 64 + lane;
    some = i < a.share;
    channel = group * a.share + min(i, a.share - 1);
  }
};

// States are taken NB at a time: as many values of B and C as fit the scalar registers twice (8: 497 us, 16: 474).
template <int NP>
constexpr int NB = NP < 16 ? NP : 16;

__device__ inline Scalars low_row(const ScanArgs& a, int64_t row, int group, int np) {
  return (Scalars)(uintptr_t)(a.low + (row * a.groups + group) * (2 * np));
}

// B and C as floats, N of them filled up to NP with zeros.
template <typename T>
__global__ __launch_bounds__(256) void scan_low_kernel(LowRows b, LowRows c, float* low, int n_rows, int groups, int N, int log_np) {
  const int log_nb = min(log_np, 4);
  const int64_t n = (int64_t(n_rows) + 1) * groups << (log_np + 1);
  for (int64_t i = blockIdx.x * int64_t(256) + threadIdx.x; i < n; i += gridDim.x * int64_t(256)) {
    const int at = static_cast<int>(i & ((2 << log_np) - 1)), j = (at >> (log_nb + 1) << log_nb) + (at & ((1 << log_nb) - 1));
    const int64_t rg = i >> (log_np + 1), row = rg / groups, g = rg - row * groups;
    const LowRows& from = at >> log_nb & 1 ? c : b;
    low[i] = row < n_rows && j < N ? static_cast<float>(static_cast<const T*>(from.p)[row * from.row + g * from.group + j]) : 0.f;
  }
}

// Rates of a lane's states first .. first + n of NP, times log2(e).
template <int NP>
__device__ inline void rates(float (&A2)[NP], const ScanArgs& a, int channel, int first) {
#pragma unroll
  for (int n = 0; n < NP; ++n) A2[n] = a.A[int64_t(channel) * a.N + min(first + n, a.N - 1)];  // (all loads under way at once: none hangs on a branch)
#pragma unroll
  for (int n = 0; n < NP; ++n) A2[n] = first + n < a.N ? A2[n] * LOG2E : 0.f;
}
template <int NP>
__device__ inline void load_state(float (&h)[NP], const float* p, const ScanArgs& a, int scene, const Lane& me, int first) {
#pragma unroll
  for (int n = 0; n < NP; ++n) h[n] = 0.f;
  if (!p) return;
#pragma unroll
  for (int n = 0; n < NP; ++n) h[n] = p[(int64_t(scene) * a.channels + me.channel) * a.N + min(first + n, a.N - 1)];
#pragma unroll
  for (int n = 0; n < NP; ++n) h[n] = me.some && first + n < a.N ? h[n] : 0.f;
}
template <int NP>
__device__ inline void store_state(const float (&h)[NP], float* p, const ScanArgs& a, int scene, const Lane& me, int first) {
  if (!p || !me.some) return;
#pragma unroll
  for (int n = 0; n < NP; ++n)
    if (first + n < a.N) p[(int64_t(scene) * a.channels + me.channel) * a.N + first + n] = h[n];
}
template <int NP, int ALL>
__device__ inline void load_between(float (&h)[NP], const float* p, const ScanArgs& a, int id, const Lane& me, int first) {
#pragma unroll
  for (int n = 0; n < NP; ++n) h[n] = me.some ? p[(int64_t(id) * ALL + first + n) * a.channels + me.channel] : 0.f;
}

// 2^w h + v.  GROWS: powers beyond 2^120 are taken by the state first, so that where a run of rows grows beyond 32 bits a state of zero stays zero, and one of little gets to where its rows
// would bring it.  Elsewhere both are the same bits, and waves whose lanes are all there take the shorter one.
constexpr float FAR = 120.f;
template <bool GROWS>
__device__ inline float carried(float w, float h, float v) {
  if (!GROWS) return fmaf(__builtin_amdgcn_exp2f(w), h, v);
  const int k = static_cast<int>(fmaxf(w - FAR, 0.f));
  return fmaf(__builtin_amdgcn_exp2f(w - static_cast<float>(k)), ldexpf(h, k), v);
}

// A lane's place in a row behind a scalar address.  `stays`, in the block of the accesses: widened elsewhere, the compiler adds both up in vector registers.
__device__ inline void stays(unsigned& at) { asm volatile("" : "+v"(at)); }
template <typename T>
__device__ inline SPC_GLOBAL char* row_of(const void* p, int64_t row, int64_t ld) {
  return (SPC_GLOBAL char*)(uintptr_t)p + row * ld * int64_t(sizeof(T));
}
template <typename T>
__device__ inline T load_at(const SPC_GLOBAL char* row, unsigned at) {
  return *reinterpret_cast<SPC_GLOBAL const T*>(row + at);
}
template <typename T>
__device__ inline void store_at(SPC_GLOBAL char* row, unsigned at, T v) {
  *reinterpret_cast<SPC_GLOBAL T*>(row + at) = v;
}
// The rows of a matrix from `first` on, one after the other.
template <typename T>
struct Walk {
  SPC_GLOBAL char* row;
  int64_t pitch;
  __device__ Walk(const void* p, int64_t ld, int64_t first) : row(row_of<T>(p, first, ld)), pitch(ld * int64_t(sizeof(T))) {}
  __device__ T next(unsigned at) {
    const T v = load_at<T>(row, at);
    on();
    return v;
  }
  __device__ void put(unsigned at, T v) {
    store_at<T>(row, at, v);
    on();
  }
  __device__ void on() {
    row += pitch;
    asm("" : "+s"(row));  // (else every row of an unrolled loop has an offset of its own in scalar registers, which then do not suffice)
  }
};

// SUMS: a segment's own state, its sum of d, and (GRAD) what its rows send to those in front of it.  Else: outputs.  Rows are taken U at a time while
// the next ones are on their way, and B and C of the next NB states while those at hand are used.
template <typename T, int NP, bool GATE, bool SUMS, bool GRAD>
__global__ __launch_bounds__(SCAN_THREADS) void scan_kernel(const ScanArgs a) {
  constexpr int U = 4, N1 = NB<NP>, BLOCKS = NP / N1;
  constexpr bool EXACT = sizeof(T) == 4, GATED = GATE && (GRAD || !SUMS), NEEDS_C = GRAD || !SUMS;
  const int unit = blockIdx.x * (SCAN_THREADS / 64) + __builtin_amdgcn_readfirstlane(threadIdx.x / 64), id = unit / a.blocks, block = unit - id * a.blocks;
  SceneSegment s;
  if (!s.find(a.scenes, id) || (SUMS && !GRAD && s.m == s.n - 1)) return;
  s.uniform();
  const Lane me(a, block, threadIdx.x % 64);
  if (!me.some) return;
  const float bias = a.bias ? a.bias[me.channel] : 0.f, skip = a.skip ? a.skip[me.channel] : 0.f;
  float A2[NP], h[NP], sent[GRAD ? NP : 1] = {}, through[GRAD ? NP : 1], steps = 0.f, least = 0.f;
  rates<NP>(A2, a, me.channel, 0);
  if (SUMS) {
#pragma unroll
    for (int n = 0; n < NP; ++n) h[n] = 0.f;
    if (GRAD)
#pragma unroll
      for (int n = 0; n < NP; ++n) through[n] = 1.f;
  } else if (s.m == 0) {
    load_state<NP>(h, a.state_in, a, s.scene, me, 0);
  } else {
    load_between<NP, NP>(h, a.between, a, id - 1, me, 0);
  }
  unsigned at = unsigned(me.channel) * unsigned(sizeof(T));
  Walk<T> in_u(a.u, a.ld_u, s.first), in_dt(a.dt, a.ld_dt, s.first), in_gate(a.gate, a.ld_gate, s.first), in_dout(a.dout, a.ld_dout, s.first), out(a.out, a.ld_out, s.first);
  struct Row {
    T u, dt, gate, dout;
  };
  auto load = [&](Row& r) {
    r.u = in_u.next(at);
    r.dt = in_dt.next(at);
    if (GATED) r.gate = in_gate.next(at);
    if (GRAD) r.dout = in_dout.next(at);
  };
  Scalars low = low_row(a, s.first, me.group, NP);
  const int64_t low_pitch = int64_t(a.groups) * (2 * NP);
  float bc[2 * N1];
  auto fetch = [&](float (&to)[2 * N1], Scalars from) {
#pragma unroll
    for (int n = 0; n < (NEEDS_C ? 2 : 1) * N1; ++n) to[n] = from[n];
  };
  fetch(bc, low);
  auto compute = [&](const Row& r) {
    const float u = static_cast<float>(r.u), d = Step<T>(static_cast<float>(r.dt) + bias, a.softplus).d, x = d * u;
    float dy = 0.f, y = 0.f;
    if constexpr (GRAD) {
      dy = static_cast<float>(r.dout);
      if constexpr (GATED) {
        const float z = static_cast<float>(r.gate);
        dy *= z * sigmoid_of<EXACT>(z);
      }
    }
    if (SUMS) steps += d;
    if (GRAD) least = fminf(least, d);
#pragma unroll
    for (int k = 0; k < BLOCKS; ++k) {
      float ahead[2 * N1];
      const Scalars behind = k + 1 < BLOCKS ? low + 2 * N1 * (k + 1) : low + low_pitch;
      fetch(ahead, behind);  // (behind the last row of all there is one of zeros)
      if (k + 1 == BLOCKS) low = behind;
      __builtin_amdgcn_sched_barrier(0);  // (else the loads are put where their values are used)
#pragma unroll
      for (int n = 0; n < N1; ++n) {
        const int j = k * N1 + n;
        const float e = __builtin_amdgcn_exp2f(d * A2[j]);
        h[j] = fmaf(e, h[j], x * bc[n]);
        if (!SUMS) y = fmaf(bc[N1 + n], h[j], y);
        if constexpr (GRAD) {
          through[j] *= e;
          sent[j] = fmaf(through[j], dy * bc[N1 + n], sent[j]);
        }
      }
#pragma unroll
      for (int n = 0; n < (NEEDS_C ? 2 : 1) * N1; ++n) bc[n] = ahead[n];
    }
    if (!SUMS) {
      y = fmaf(skip, u, y);
      if constexpr (GATED) {
        const float z = static_cast<float>(r.gate);
        y *= z * sigmoid_of<EXACT>(z);
      }
      out.put(at, static_cast<T>(y));
    }
  };
  auto start = [&](int t) {  // in front of row t
    constexpr int L = grad_rows(NP);
    if (!(SUMS && GRAD) || t % L || !t) return;
    float* to = a.starts + (int64_t(s.first) / L + id + t / L) * (NP + 1) * a.channels + me.channel;
#pragma unroll
    for (int n = 0; n < NP; ++n) to[int64_t(n) * a.channels] = h[n];
    to[int64_t(NP) * a.channels] = steps;
  };
  int t = 0;
  if (s.rows >= U) {
    Row now[U], next[U];
#pragma unroll
    for (int q = 0; q < U; ++q) load(now[q]);
    for (; t + 2 * U <= s.rows; t += U) {
      start(t);
      stays(at);
#pragma unroll
      for (int q = 0; q < U; ++q) load(next[q]);
#pragma unroll
      for (int q = 0; q < U; ++q) compute(now[q]);
#pragma unroll
      for (int q = 0; q < U; ++q) now[q] = next[q];
    }
    start(t);
#pragma unroll
    for (int q = 0; q < U; ++q) compute(now[q]);
    t += U;
  }
  for (; t < s.rows; ++t) {
    start(t);
    Row r;
    load(r);
    compute(r);
  }
  if (!SUMS) {
    if (s.m == s.n - 1) store_state<NP>(h, a.state_out, a, s.scene, me, 0);
    return;
  }
  if constexpr (GRAD) {
    // Where decays may be above one, their products from the segment's first row on leave 32 bits (or come back from zero) though what they are multiplied by does not: such lanes take the
    // recurrence from the last row on.
    bool grows = least < 0.f;
#pragma unroll
    for (int n = 0; n < NP; ++n) grows |= A2[n] > 0.f;
    if (__any(grows)) {
      // (the arguments are read again: kept for this, they would push others out of the scalar registers in the loop above)
      auto again = (const __attribute__((address_space(4))) ScanArgs*)__builtin_amdgcn_kernarg_segment_ptr();
      asm volatile("" : "+s"(again));
      const auto& r = *again;
      float back[NP] = {};
      for (int t = s.rows - 1; t >= 0; --t) {
        const int64_t row = int64_t(s.first) + t;
        stays(at);
        const float d = Step<T>(static_cast<float>(load_at<T>(row_of<T>(r.dt, row, r.ld_dt), at)) + bias, r.softplus).d;
        float dy = static_cast<float>(load_at<T>(row_of<T>(r.dout, row, r.ld_dout), at));
        if constexpr (GATED) {
          const float z = static_cast<float>(load_at<T>(row_of<T>(r.gate, row, r.ld_gate), at));
          dy *= z * sigmoid_of<EXACT>(z);
        }
        const Scalars from = (Scalars)(uintptr_t)(r.low + (row * r.groups + me.group) * (2 * NP));
#pragma unroll
        for (int n = 0; n < NP; ++n) back[n] = __builtin_amdgcn_exp2f(d * A2[n]) * fmaf(dy, from[n / N1 * (2 * N1) + N1 + n % N1], back[n]);
      }
#pragma unroll
      for (int n = 0; n < NP; ++n) sent[n] = grows ? back[n] : sent[n];
    }
  }
  a.steps[int64_t(id) * a.channels + me.channel] = steps;
#pragma unroll
  for (int n = 0; n < NP; ++n) {
    const int64_t to = (int64_t(id) * NP + n) * a.channels + me.channel;
    a.between[to] = h[n];
    if (GRAD) a.behind[to] = sent[n];
  }
}

// A scene's segments one after the other: their own states -> the states behind them; with time running backward, what they send forward -> what arrives behind them.
// A wave has 64 (state, channel) pairs and a share of the scene's segments, up to CHAIN_WAVES waves to a scene: each runs over its own from zeros, takes what the ones before
// it come to, and runs over them again.  Loads' latency bounds it, CHAIN_AHEAD of which are under way (500 segments, 512 channels of 16 states, us: one wave and 16 loads 50, eight
// waves 19; with 120 k rows, 64 channels in 1750 segments the whole call 145, with 16 waves and 32 loads 138, 135 now).
// Growing links have code of their own, which costs calls that are launches a percent (6011 rows, gradients 74.0 -> 74.8; one code for all, longer, 74.4, and 120 k rows, 64 channels 134.8 -> 135.3).
constexpr int CHAIN_WAVES = 16, CHAIN_AHEAD = 32;
__global__ __launch_bounds__(64 * CHAIN_WAVES) void scan_chain_kernel(const ScanArgs a, int np) {
  constexpr int AHEAD = CHAIN_AHEAD;
  __shared__ float sums[CHAIN_WAVES][64], powers[CHAIN_WAVES][64];
  const bool back = blockIdx.y;
  const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
  const int64_t each = int64_t(np) * a.channels, groups = (each + 63) / 64;
  const int scene = static_cast<int>(blockIdx.x / groups), at = static_cast<int>(min((blockIdx.x - scene * groups) * 64 + lane, each - 1));
  const bool there = (blockIdx.x - scene * groups) * 64 + lane < each;
  const int n = at / a.channels, channel = at - n * a.channels;
  const int lo = a.scenes.offsets ? min(max(a.scenes.offsets[scene], 0), a.scenes.n_rows) : 0;
  const int id = lo / a.scenes.seg_rows + scene;
  SceneSegment s;
  if (!s.find(a.scenes, id) || s.scene != scene || s.n == 1) return;
  s.uniform();
  const bool is = n < a.N;
  const float A2 = is ? a.A[int64_t(channel) * a.N + n] * LOG2E : 0.f;
  const float* start = back ? a.dstate_out : a.state_in;
  float h = start && is ? start[(int64_t(scene) * a.channels + channel) * a.N + n] : 0.f;
  float* p = (back ? a.behind : a.between) + int64_t(id) * each + at;
  const float* steps = a.steps + int64_t(id) * a.channels + channel;
  const int links = back ? s.n : s.n - 1, waves = blockDim.x / 64;  // (nothing is behind a scene's last segment)
  const int share = max(AHEAD, (links + waves - 1) / waves), first = wave * share, end = min(links, first + share);
  // f(whether powers may leave 32 bits, value, sum of d, link) of the share's links in their order
  auto over = [&](auto&& f) {
    for (int m0 = first; m0 < end; m0 += AHEAD) {
      float v[AHEAD], d[AHEAD], top = 0.f;
#pragma unroll
      for (int q = 0; q < AHEAD; ++q) {
        const int k = min(m0 + q, end - 1), m = back ? s.n - 1 - k : k;
        v[q] = p[m * each];
        d[q] = steps[int64_t(m) * a.channels];
      }
#pragma unroll
      for (int q = 0; q < AHEAD; ++q) top = fmaxf(top, A2 * d[q]);
      auto with = [&](auto grows) {
#pragma unroll
        for (int q = 0; q < AHEAD; ++q)
          if (m0 + q < end) f(grows, v[q], d[q], back ? s.n - 1 - (m0 + q) : m0 + q);
      };
      if (__any(top > FAR)) with(std::true_type{});
      else with(std::false_type{});
    }
  };
  if (links > share) {  // (all waves of the workgroup alike)
    float sum = 0.f, steps_sum = 0.f;
    over([&](auto grows, float v, float d, int) {
      sum = carried<decltype(grows)::value>(A2 * d, sum, v);
      steps_sum += d;
    });
    sums[wave][lane] = sum;
    powers[wave][lane] = A2 * steps_sum;
    __syncthreads();
    for (int w = 0; w < wave; ++w) h = carried<true>(powers[w][lane], h, sums[w][lane]);
  }
  if (!there) return;
  over([&](auto grows, float v, float d, int m) {
    const float after = carried<decltype(grows)::value>(A2 * d, h, v);
    p[m * each] = back ? h : after;  // (back: what arrives behind the segment)
    h = after;
  });
}

// ---------------------------------------------------------------- gradients
template <int CTRL>
__device__ inline float from_lane(float v) {
  return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), CTRL, 0xf, 0xf, true));
}
constexpr int XOR_1 = 0xb1, XOR_2 = 0x4e, XOR_7 = 0x141, XOR_8 = 0x128;  // (of a row's 16 lanes: two orders of four, the half turned round, turned by 8)
template <int CTRL>
__device__ inline float halves(float a, float b, bool upper) {  // a of this lane and its partner where `upper` is false, b where it is true
  return (upper ? b : a) + from_lane<CTRL>(upper ? a : b);
}
template <bool WIDE>
__device__ inline float swapped(float a, float b) {  // the same for lanes 32 (16) apart: a in the lower ones, b in the upper
  const unsigned x = __builtin_bit_cast(unsigned, a), y = __builtin_bit_cast(unsigned, b);
  const auto r = [&] {
    if constexpr (WIDE) return __builtin_amdgcn_permlane32_swap(x, y, false, false);
    else return __builtin_amdgcn_permlane16_swap(x, y, false, false);
  }();
  const unsigned p = r[0], q = r[1];  // (a cast of r[1] itself is one of r[0] to the compiler)
  return __builtin_bit_cast(float, p) + __builtin_bit_cast(float, q);
}
// Sums of V values over the 64 lanes: lane l ends with value l / (64 / V).  Half of the values go with every step, while there are several.
template <int V>
__device__ inline float sums_over_lanes(float (&v)[V], int lane) {
  static_assert(V >= 4 && V <= 32, "two rows of one to eight states");
#pragma unroll
  for (int k = 0; k < V / 2; ++k) v[k] = swapped<true>(v[k], v[k + V / 2]);
#pragma unroll
  for (int k = 0; k < V / 4; ++k) v[k] = swapped<false>(v[k], v[k + V / 4]);
  if constexpr (V >= 8) {
#pragma unroll
    for (int k = 0; k < V / 8; ++k) v[k] = halves<XOR_8>(v[k], v[k + V / 8], lane & 8);
  } else v[0] += from_lane<XOR_8>(v[0]);
  if constexpr (V >= 16) {
#pragma unroll
    for (int k = 0; k < V / 16; ++k) v[k] = halves<XOR_7>(v[k], v[k + V / 16], lane & 4);
  } else v[0] += from_lane<XOR_7>(v[0]);
  if constexpr (V >= 32) v[0] = halves<XOR_2>(v[0], v[1], lane & 2);
  else v[0] += from_lane<XOR_2>(v[0]);
  return v[0] + from_lane<XOR_1>(v[0]);
}

// A workgroup has a segment of 64 channels, each of its LP waves NG of their states.  Chunk by chunk from the segment's last one, the states are made again from that in
// front of the chunk (what the first launch has left, and the decayed state in front of the segment), kept in registers with their decays, and the gradient runs back over
// them.  What rows share (d, d u, dy) is made by one wave a row and read by all from LDS, as are B and C; the sums over states (x, sum of A p, C . h) are parts of the waves,
// which the row's wave adds up.  The next chunk's rows are on their way meanwhile.
constexpr int PART_ROWS = 8;
template <int NP, bool GATE>
struct GradLds {
  static constexpr int VALUES = GATE ? 3 : 2, L = grad_rows(NP), LP = NP / grad_states(NP);
  float stage[3][L][64];
  float low[L][2][NP];
  float part[LP][PART_ROWS][VALUES][64];
};

template <typename T, int NP, bool GATE>
__global__ __launch_bounds__(64 * NP / grad_states(NP), 2) void scan_grad_kernel(const ScanArgs a) {
  constexpr int NG = grad_states(NP), L = grad_rows(NP), LP = NP / NG, RW = L / LP, V = 4 * NG, LOWS = L * 2 * NP, LOW = (LOWS + 64 * LP - 1) / (64 * LP);
  constexpr bool EXACT = sizeof(T) == 4, KEEP = NG <= 4;  // KEEP: decays are kept beside the states (1246 us without, 1179 with; of eight states a lane, there is no room)
  extern __shared__ __attribute__((aligned(16))) char raw[];
  using Lds = GradLds<NP, GATE>;
  Lds& lds = *reinterpret_cast<Lds*>(raw);
  const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), first_n = wave * NG;
  const int id = blockIdx.x / a.blocks, block = blockIdx.x - id * a.blocks;
  const Lane me(a, block, lane);
  float* parts = a.parts + int64_t(id) * (NP + 2) * a.channels + me.channel;
  SceneSegment s;
  if (!s.find(a.scenes, id)) {
    if (me.some) {
#pragma unroll
      for (int n = 0; n < NG; ++n) parts[int64_t(first_n + n) * a.channels] = 0.f;
      if (wave == 0) parts[int64_t(NP) * a.channels] = parts[int64_t(NP + 1) * a.channels] = 0.f;
    }
    return;
  }
  s.uniform();
  const float bias = a.bias ? a.bias[me.channel] : 0.f, skip = a.skip ? a.skip[me.channel] : 0.f;
  float A2[NG], first_h[NG], r[NG], dA[NG] = {};
  rates<NG>(A2, a, me.channel, first_n);
  if (s.m == 0) load_state<NG>(first_h, a.state_in, a, s.scene, me, first_n);
  else load_between<NG, NP>(first_h, a.between, a, id - 1, me, first_n);
  if (s.m == s.n - 1) load_state<NG>(r, a.dstate_out, a, s.scene, me, first_n);
  else load_between<NG, NP>(r, a.behind, a, id, me, first_n);
  const int chunks = (s.rows + L - 1) / L;
  unsigned at = unsigned(me.channel) * unsigned(sizeof(T));
  // what comes of a chunk: this wave's rows of it, t = chunk L + j LP + wave; this thread's values of B and C; the state in front of it
  struct {
    T u[RW], dt[RW], gate[GATE ? RW : 1], dout[RW], low[LOW];
    float h[NG], steps;
  } in;
  auto load = [&](int chunk) {
    stays(at);
    unsigned at4 = unsigned(me.channel) * 4;
    stays(at4);
#pragma unroll
    for (int j = 0; j < RW; ++j) {
      const int64_t row = int64_t(s.first) + min(chunk * L + j * LP + wave, s.rows - 1);
      in.u[j] = load_at<T>(row_of<T>(a.u, row, a.ld_u), at);
      in.dt[j] = load_at<T>(row_of<T>(a.dt, row, a.ld_dt), at);
      in.dout[j] = load_at<T>(row_of<T>(a.dout, row, a.ld_dout), at);
      if (GATE) in.gate[j] = load_at<T>(row_of<T>(a.gate, row, a.ld_gate), at);
    }
#pragma unroll
    for (int j = 0; j < LOW; ++j) {
      const int i = min(j * (64 * LP) + int(threadIdx.x), LOWS - 1), n = min(i % NP, a.N - 1);
      const int64_t row = int64_t(s.first) + min(chunk * L + i / (2 * NP), s.rows - 1);
      const LowRows& from = i / NP % 2 ? a.c : a.b;
      in.low[j] = static_cast<const T*>(from.p)[row * from.row + me.group * from.group + n];
    }
    if (!chunk) return;
    const int64_t p = (int64_t(s.first) / L + id + chunk) * (NP + 1);
#pragma unroll
    for (int n = 0; n < NG; ++n) in.h[n] = load_at<float>(row_of<float>(a.starts, p + first_n + n, a.channels), at4);
    in.steps = load_at<float>(row_of<float>(a.starts, p + NP, a.channels), at4);
  };
  float u[RW], slope[RW], through_gate[GATE ? RW : 1];  // the last: dout silu'(gate)
  float dskip = 0.f, dbias = 0.f;
  if (chunks) load(chunks - 1);
  for (int chunk = chunks - 1; chunk >= 0; --chunk) {
    // (every wave has passed the barrier behind its last reads of what is written here, its own rows aside, which it reads to the end)
#pragma unroll
    for (int j = 0; j < RW; ++j) {
      const int i = j * LP + wave;
      const bool there = me.some && chunk * L + i < s.rows;  // (rows that are not there leave states and gradients as they are)
      const Step<T> step(static_cast<float>(in.dt[j]) + bias, a.softplus);
      const float d = there ? step.d : 0.f;
      float dy = there ? static_cast<float>(in.dout[j]) : 0.f;
      u[j] = there ? static_cast<float>(in.u[j]) : 0.f;
      slope[j] = step.slope;
      if constexpr (GATE) {
        const float z = there ? static_cast<float>(in.gate[j]) : 0.f, g = sigmoid_of<EXACT>(z);
        through_gate[j] = dy * fmaf(z * g, 1.f - g, g);
        dy *= z * g;
      }
      lds.stage[0][i][lane] = d;
      lds.stage[1][i][lane] = d * u[j];
      lds.stage[2][i][lane] = dy;
    }
#pragma unroll
    for (int j = 0; j < LOW; ++j) {
      const int i = j * (64 * LP) + threadIdx.x;
      if (LOWS % (64 * LP) == 0 || i < LOWS) (&lds.low[0][0][0])[i] = i % NP < a.N && chunk * L + i / (2 * NP) < s.rows ? static_cast<float>(in.low[j]) : 0.f;
    }
    float h[NG];
#pragma unroll
    for (int n = 0; n < NG; ++n) h[n] = chunk ? (me.some ? carried<false>(A2[n] * in.steps, first_h[n], in.h[n]) : 0.f) : first_h[n];
    bool far = false;  // (made again where it has to be: a choice between the two takes registers that are not there, 1170 -> 1370 us a pass)
#pragma unroll
    for (int n = 0; n < NG; ++n) far |= A2[n] * in.steps > FAR;
    if (chunk && __any(far)) {
#pragma unroll
      for (int n = 0; n < NG; ++n) h[n] = me.some ? carried<true>(A2[n] * in.steps, first_h[n], in.h[n]) : 0.f;
    }
    __syncthreads();
    if (chunk) load(chunk - 1);
    float hs[L][NG], decay[KEEP ? L : 1][NG];
    // (a row is read while the one before it is worked on; without the barriers all are read at once, which takes more registers than there are)
    struct Row {
      float d, x, dy, B[NG], C[NG];
      __device__ void read(const Lds& lds, int i, int lane, int first_n, bool back) {
        d = lds.stage[0][i][lane], x = lds.stage[1][i][lane];
        if (back) dy = lds.stage[2][i][lane];
#pragma unroll
        for (int n = 0; n < NG; ++n) {
          B[n] = lds.low[i][0][first_n + n];
          if (back) C[n] = lds.low[i][1][first_n + n];
        }
      }
    } now, next;
    now.read(lds, 0, lane, first_n, false);
#pragma unroll
    for (int i = 0; i < L; ++i) {
      if (i + 1 < L) next.read(lds, i + 1, lane, first_n, false);
      else next.read(lds, L - 1, lane, first_n, true);
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int n = 0; n < NG; ++n) {
        const float f = __builtin_amdgcn_exp2f(now.d * A2[n]);
        if (KEEP) decay[KEEP ? i : 0][n] = f;
        hs[i][n] = fmaf(f, i ? hs[i ? i - 1 : 0][n] : h[n], now.x * now.B[n]);
      }
      now = next;
    }
#pragma unroll
    for (int half = L / PART_ROWS - 1; half >= 0; --half) {
      float low_sums[PART_ROWS / 2];
#pragma unroll
      for (int pair = PART_ROWS / 2 - 1; pair >= 0; --pair) {
        float v[V];
#pragma unroll
        for (int e = 1; e >= 0; --e) {
          const int i = half * PART_ROWS + pair * 2 + e;
          if (i) next.read(lds, i - 1, lane, first_n, true);
          __builtin_amdgcn_sched_barrier(0);
          float sx = 0.f, sp = 0.f, sy = 0.f;
#pragma unroll
          for (int n = 0; n < NG; ++n) {
            const float q = fmaf(now.C[n], now.dy, r[n]);
            v[e * 2 * NG + n] = q * now.x;
            v[e * 2 * NG + NG + n] = hs[i][n] * now.dy;
            if (GATE) sy = fmaf(now.C[n], hs[i][n], sy);
            sx = fmaf(q, now.B[n], sx);
            r[n] = q * (KEEP ? decay[KEEP ? i : 0][n] : __builtin_amdgcn_exp2f(now.d * A2[n]));
            const float p = r[n] * (i ? hs[i ? i - 1 : 0][n] : h[n]);
            sp = fmaf(A2[n], p, sp);
            dA[n] = fmaf(now.d, p, dA[n]);
          }
          float(*to)[64] = lds.part[wave][pair * 2 + e];
          to[0][lane] = sx;
          to[1][lane] = sp;
          if (GATE) to[2][lane] = sy;
          if (i) now = next;
        }
        low_sums[pair] = sums_over_lanes<V>(v, lane);
      }
      constexpr int EACH = 64 / V;
      const int k = lane / EACH, n = first_n + k % NG;
      const bool is_c = k / NG % 2;
      if (lane % EACH == 0) {
#pragma unroll
        for (int pair = 0; pair < PART_ROWS / 2; ++pair) {
          const int t = chunk * L + half * PART_ROWS + pair * 2 + k / (2 * NG);
          if (t >= s.rows) continue;
          const int64_t row = int64_t(s.first) + t;
          if (a.low_parts) {
            a.low_parts[((int64_t(block) * a.scenes.n_rows + row) * 2 + is_c) * NP + n] = low_sums[pair];
          } else if (n < a.N) {
            const LowRows& to = is_c ? a.dc : a.db;
            static_cast<T*>(to.p)[row * to.row + me.group * to.group + n] = static_cast<T>(low_sums[pair]);
          }
        }
      }
      __syncthreads();
#pragma unroll
      for (int j = half * PART_ROWS / LP; j < (half + 1) * PART_ROWS / LP; ++j) {
        const int i = j * LP + wave, t = chunk * L + i;
        float sx = 0.f, sp = 0.f, sy = 0.f;
#pragma unroll
        for (int w = 0; w < LP; ++w) {
          sx += lds.part[w][i % PART_ROWS][0][lane];
          sp += lds.part[w][i % PART_ROWS][1][lane];
          if (GATE) sy += lds.part[w][i % PART_ROWS][GATE ? 2 : 0][lane];
        }
        if (!me.some || t >= s.rows) continue;
        const int64_t row = int64_t(s.first) + t;
        stays(at);
        const float ddt = fmaf(u[j], sx, sp * (1.f / LOG2E)) * slope[j], d = lds.stage[0][i][lane], dy = lds.stage[2][i][lane];
        store_at<T>(row_of<T>(a.out, row, a.ld_out), at, static_cast<T>(fmaf(d, sx, skip * dy)));
        store_at<T>(row_of<T>(a.ddt, row, a.ld_ddt), at, static_cast<T>(ddt));
        if constexpr (GATE) store_at<T>(row_of<T>(a.dgate, row, a.ld_dgate), at, static_cast<T>(through_gate[j] * fmaf(skip, u[j], sy)));
        dskip = fmaf(dy, u[j], dskip);
        dbias += ddt;
      }
      if (half) __syncthreads();  // (the parts have been read)
    }
  }
  if (s.m == 0) store_state<NG>(r, a.dstate_in, a, s.scene, me, first_n);
  __syncthreads();
  lds.part[wave][0][0][lane] = dskip;
  lds.part[wave][0][1][lane] = dbias;
  __syncthreads();
  if (!me.some) return;
#pragma unroll
  for (int n = 0; n < NG; ++n) parts[int64_t(first_n + n) * a.channels] = dA[n];
  for (int k = wave; k < 2; k += LP) {
    float sum = 0.f;
#pragma unroll
    for (int w = 0; w < LP; ++w) sum += lds.part[w][0][k][lane];
    parts[int64_t(NP + k) * a.channels] = sum;
  }
}

// Sums of the segments' parts: 32 columns a workgroup, 32 shares of the segments added up in LDS, in a fixed order.
__global__ __launch_bounds__(1024) void scan_params_kernel(const float* __restrict__ parts, int n, int np, int channels, int N, float* dA, float* dskip, float* dbias) {
  __shared__ float lds[32][33];
  const int cols = (np + 2) * channels, col = blockIdx.x * 32 + threadIdx.x % 32, share = threadIdx.x / 32;
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
  const int j = col / channels, channel = col - j * channels;
  if (j < N && dA) dA[int64_t(channel) * N + j] = s;
  if (j == np && dskip) dskip[channel] = s;
  if (j == np + 1 && dbias) dbias[channel] = s;
}

// dB and dC of groups of several blocks of channels.
template <typename T>
__global__ __launch_bounds__(256) void scan_low_grad_kernel(const ScanArgs a, int log_np) {
  const int n_rows = a.scenes.n_rows, per = a.blocks / a.groups;
  const int lo = a.scenes.offsets ? min(max(a.scenes.offsets[0], 0), n_rows) : 0;
  const int hi = a.scenes.offsets ? min(max(a.scenes.offsets[a.scenes.n_scenes], lo), n_rows) : n_rows;
  const int64_t each = int64_t(n_rows) << (log_np + 1), n = int64_t(hi - lo) * a.groups << (log_np + 1);
  for (int64_t i = blockIdx.x * int64_t(256) + threadIdx.x; i < n; i += gridDim.x * int64_t(256)) {
    const int j = static_cast<int>(i & ((1 << log_np) - 1));
    if (j >= a.N) continue;
    const int is_c = i >> log_np & 1;
    const int64_t rg = i >> (log_np + 1), row = lo + rg / a.groups, g = rg % a.groups;
    const float* p = a.low_parts + g * per * each + (row << (log_np + 1)) + (is_c << log_np) + j;
    float s = 0.f;
#pragma unroll 4
    for (int q = 0; q < per; ++q) s += p[q * each];
    const LowRows& to = is_c ? a.dc : a.db;
    static_cast<T*>(to.p)[row * to.row + g * to.group + j] = static_cast<T>(s);
  }
}

// ---------------------------------------------------------------- one row of many streams
// A lane has VEC states of a channel, 2^log_q neighbouring lanes have a channel's; states are read and written once (2048 streams of 512 channels of 16 states, fp16: 36.6 us for
// 142 MB, the vector unit issues in 78 % of the CUs' cycles).  The decay is taken as 1 + (e^w - 1) where it is near 1: rounded to 24 bits every row, a stream's long memory would
// drift (of shorter ones, up to 16 rows, it is off by some 16 x 2^-23).
template <typename T, int VEC, bool GATE>
__global__ __launch_bounds__(256) void scan_step_kernel(const ScanArgs a, float* state, unsigned n, int log_q) {
  typedef float Values __attribute__((ext_vector_type(VEC), aligned(4), may_alias));
  // (fewer than 2^31 lanes have states)
  const unsigned i = (blockIdx.x * 256u + threadIdx.x) >> log_q, first = (threadIdx.x & ((1u << log_q) - 1)) * VEC, channels = a.channels;
  const bool is = i < n * channels && first < unsigned(a.N);
  Values* S = reinterpret_cast<Values*>(state + int64_t(i) * a.N + first);
  Values h;
  if (is) h = *S;
  const int64_t row = i / channels;
  const int channel = static_cast<int>(i - unsigned(row) * channels);
  float y = 0.f, u = 0.f;
  if (is) {
    u = static_cast<float>(static_cast<const T*>(a.u)[row * a.ld_u + channel]);
    const float d = Step<T>(static_cast<float>(static_cast<const T*>(a.dt)[row * a.ld_dt + channel]) + (a.bias ? a.bias[channel] : 0.f), a.softplus).d;
    const int group = a.groups > 1 ? channel / a.share : 0;
    const T* B = static_cast<const T*>(a.b.p) + row * a.b.row + group * a.b.group + first;
    const T* C = static_cast<const T*>(a.c.p) + row * a.c.row + group * a.c.group + first;
    const Values A = *reinterpret_cast<const Values*>(a.A + int64_t(channel) * a.N + first);
#pragma unroll
    for (int k = 0; k < VEC; ++k) {
      const float w = d * A[k], x = d * u * static_cast<float>(B[k]);
      float e = 1.f / 120;  // (e^w - 1) / w by its series; what it leaves out is below 2^-29 for |w| < 1/16
      e = fmaf(e, w, 1.f / 24), e = fmaf(e, w, 1.f / 6), e = fmaf(e, w, .5f), e = fmaf(e, w, 1.f);
      h[k] = fabsf(w) < .0625f ? h[k] + fmaf(h[k], e * w, x) : fmaf(__builtin_amdgcn_exp2f(w * LOG2E), h[k], x);
      y = fmaf(static_cast<float>(C[k]), h[k], y);
    }
    *S = h;
  }
  for (int o = 1; o < (1 << log_q); o <<= 1) y += __shfl_xor(y, o, 64);
  if (!is || first) return;
  y = fmaf(a.skip ? a.skip[channel] : 0.f, u, y);
  if constexpr (GATE) {
    const float z = static_cast<float>(static_cast<const T*>(a.gate)[row * a.ld_gate + channel]);
    y *= z * sigmoid_of<sizeof(T) == 4>(z);
  }
  static_cast<T*>(a.out)[row * a.ld_out + channel] = static_cast<T>(y);
}

// ---------------------------------------------------------------- host
int check_scan(const spc_scan_desc* d, const float* A, bool scenes, const int32_t* offsets) {
  if (!d) return set_error(SPC_ERR_ARG, "descriptor is NULL");
  if (d->dtype != SPC_DTYPE_F16 && d->dtype != SPC_DTYPE_BF16 && d->dtype != SPC_DTYPE_F32) return set_error(SPC_ERR_ARG, "unknown dtype %d", d->dtype);
  if (d->n_rows < 0 || d->channels < 1 || d->groups < 1 || d->channels % d->groups || d->states < 1)
    return set_error(SPC_ERR_ARG, "%lld rows, %d channels in %d groups, %d states", static_cast<long long>(d->n_rows), d->channels, d->groups, d->states);
  if (!A) return set_error(SPC_ERR_ARG, "A is NULL");
  if (d->channels > SCAN_MAX_C || d->states > SCAN_MAX_N)
    return set_error(SPC_ERR_UNSUPPORTED, "%d channels of %d states: at most %d and %d", d->channels, d->states, SCAN_MAX_C, SCAN_MAX_N);
  if (scenes) SPC_RETURN_IF(check_scenes(offsets, d->n_rows, d->n_scenes));
  return SPC_OK;
}
int check_matrix(const char* what, const void* p, int64_t ld, const spc_scan_desc* d) {
  if (!p) return set_error(SPC_ERR_ARG, "%s is NULL", what);
  if (ld < d->channels) return set_error(SPC_ERR_ARG, "row pitch %lld of %s is below %d channels", static_cast<long long>(ld), what, d->channels);
  if (reinterpret_cast<uintptr_t>(p) % (d->dtype == SPC_DTYPE_F32 ? 4 : 2)) return set_error(SPC_ERR_ARG, "%s is not aligned to its type", what);
  return SPC_OK;
}
// Pitches of an input may be zero (broadcast); places of an output are its own.
int check_low(const char* what, const spc_attn_rows* t, const spc_scan_desc* d, bool output) {
  if (!t || !t->data) return set_error(SPC_ERR_ARG, "%s is NULL", what);
  if (reinterpret_cast<uintptr_t>(t->data) % (d->dtype == SPC_DTYPE_F32 ? 4 : 2)) return set_error(SPC_ERR_ARG, "%s is not aligned to its type", what);
  const int64_t row = t->row_pitch, group = t->head_pitch, far = int64_t(1) << 40;
  bool ok = row >= 0 && group >= 0 && row < far && group < far;
  if (output && ok) {
    const bool one_row = d->n_rows <= 1, one_group = d->groups == 1;
    ok = (one_row || row >= d->states) && (one_group || group >= d->states) &&
         (one_row || one_group || row >= (d->groups - 1) * group + d->states || group >= (d->n_rows - 1) * row + d->states);
  }
  return ok ? SPC_OK : set_error(SPC_ERR_ARG, "pitches %lld and %lld of %s do not fit %d groups of %d states", static_cast<long long>(row), static_cast<long long>(group), what,
                                 d->groups, d->states);
}
LowRows low_rows(const spc_attn_rows* t) { return {t->data, t->row_pitch, t->head_pitch}; }

int log_padded(int N) { return N <= 4 ? 2 : N <= 8 ? 3 : N <= 16 ? 4 : N <= 32 ? 5 : 6; }

// Calls f(type, NP, GATE).
template <typename F>
void scan_variant(const spc_scan_desc* d, bool gate, F&& f) {
  using std::integral_constant;
  by_dtype(d->dtype, [&](auto t) {
    auto with = [&](auto np) {
      if (gate) f(t, np, std::true_type{});
      else f(t, np, std::false_type{});
    };
    switch (log_padded(d->states)) {
      case 2: return with(integral_constant<int, 4>{});
      case 3: return with(integral_constant<int, 8>{});
      case 4: return with(integral_constant<int, 16>{});
      case 5: return with(integral_constant<int, 32>{});
      default: return with(integral_constant<int, 64>{});
    }
  });
}

void scan_shape(ScanArgs& a, const spc_scan_desc* d) {
  a.channels = d->channels, a.groups = d->groups, a.share = d->channels / d->groups, a.N = d->states;
  a.blocks = (a.share + 63) / 64 * a.groups;
  a.softplus = d->softplus != 0;
}
// Rows of a segment, a multiple of `unit`: as few as give some `waves` waves, but not so few that the chain of a scene's segments takes longer than a segment, which balances at some
// sqrt(rows) / 4, and, where there is work for every SIMD, about as many as make whole rounds of `round` waves.  us, at sqrt(rows) times 0.1 / 0.2 / 0.3: 30 k rows, 256 channels
// 124 / 104 / 110, in rounds 101 / 98 (0.2, 0.3); 120 k rows, 64 channels 175 / 144 / 162, in rounds 138 / 134.  2118 rows, 64 channels: segments of 8 rows 28, 16 31, 32 39.
int segment_rows(const spc_scan_desc* d, int blocks, int waves, int round, int unit) {
  const double work = double(d->n_rows) * blocks, rows = std::max(work / waves, 0.25 * std::sqrt(double(d->n_rows) / d->n_scenes)), rounds = work / (rows * round);
  const double units = rounds >= .5 ? std::ceil(work / (std::max(1., std::round(rounds)) * round) / unit) : std::round(rows / unit);
  return static_cast<int>(std::min(4096., std::max(1., units) * unit));
}
int check_grid(const ScanArgs& a, int threads) {  // (a launch takes less than 2^32 threads)
  if (int64_t(a.ids) * a.blocks * threads < (int64_t(1) << 32) && (int64_t(a.scenes.n_scenes) * a.channels << log_padded(a.N)) < (int64_t(1) << 29)) return SPC_OK;
  return set_error(SPC_ERR_UNSUPPORTED, "%d rows of %d channels and %d states in %d scenes", a.scenes.n_rows, a.channels, a.N, a.scenes.n_scenes);
}
template <typename T>
void launch_low(const ScanArgs& a, int log_np, hipStream_t s) {
  const int64_t n = (int64_t(a.scenes.n_rows) + 1) * a.groups << (log_np + 1);
  hipLaunchKernelGGL(scan_low_kernel<T>, dim3(std::min<int64_t>((n + 255) / 256, 8192)), dim3(256), 0, s, a.b, a.c, a.low, a.scenes.n_rows, a.groups, a.N, log_np);
}
// Waves that would have no segment, were all rows in one scene, are left out, and those that would take a launch to 2^32 threads.  (check_grid has fewer than 2^29 states and 200 000 scenes
// pass, so that at most 2^23 + 200 000 workgroups have three waves left, both ways.)
void launch_chain(const ScanArgs& a, int np, bool grad, hipStream_t s) {
  const int64_t workgroups = (int64_t(np) * a.channels + 63) / 64 * a.scenes.n_scenes, ways = grad ? 2 : 1;
  const int64_t some = (a.scenes.n_rows / a.scenes.seg_rows + CHAIN_AHEAD) / CHAIN_AHEAD, most = ((int64_t(1) << 32) - 1) / (64 * ways * workgroups);
  const int waves = static_cast<int>(std::min<int64_t>({CHAIN_WAVES, some, most}));
  hipLaunchKernelGGL(scan_chain_kernel, dim3(workgroups, ways), dim3(64 * waves), 0, s, a, np);
}

}  // namespace
}  // namespace spc

extern "C" int spc_selective_scan_forward(const spc_scan_desc* d, const void* u, int64_t ld_u, const void* dt, int64_t ld_dt, const float* A, const spc_attn_rows* B,
                                          const spc_attn_rows* C, const float* skip, const void* gate, int64_t ld_gate, const float* dt_bias, const int32_t* offsets,
                                          const float* state_in, void* out, int64_t ld_out, float* state_out, void* stream) {
  using namespace spc;
  SPC_RETURN_IF(check_scan(d, A, true, offsets));
  if (d->n_rows) {
    SPC_RETURN_IF(check_matrix("u", u, ld_u, d));
    SPC_RETURN_IF(check_matrix("dt", dt, ld_dt, d));
    if (gate) SPC_RETURN_IF(check_matrix("gate", gate, ld_gate, d));
    SPC_RETURN_IF(check_matrix("out", out, ld_out, d));
    SPC_RETURN_IF(check_low("B", B, d, false));
    SPC_RETURN_IF(check_low("C", C, d, false));
  }
  if (state_out && state_out == state_in) return set_error(SPC_ERR_ARG, "state_out is state_in");
  if (!d->n_rows && !state_out) return SPC_OK;
  const StreamId s(static_cast<hipStream_t>(stream));
  const StreamWorkNote note{s};
  const int log_np = log_padded(d->states), np = 1 << log_np;
  ScanArgs a{};
  scan_shape(a, d);
  a.u = u, a.ld_u = ld_u, a.dt = dt, a.ld_dt = ld_dt, a.gate = gate, a.ld_gate = ld_gate, a.out = out, a.ld_out = ld_out;
  if (d->n_rows) a.b = low_rows(B), a.c = low_rows(C);
  a.A = A, a.skip = skip, a.bias = dt_bias, a.state_in = state_in, a.state_out = state_out;
  a.scenes = {offsets, static_cast<int>(d->n_rows), d->n_scenes, segment_rows(d, a.blocks, 8192, 1024, 8)};
  a.ids = a.scenes.ids();
  SPC_RETURN_IF(check_grid(a, 64));
  const bool cut = d->n_rows > a.scenes.seg_rows;
  const size_t low = ((size_t(d->n_rows) + 1) * a.groups * 2) << log_np, states = cut ? size_t(a.ids) * np * a.channels : 0, steps = cut ? size_t(a.ids) * a.channels : 0;
  float* ws = static_cast<float*>(pool_alloc(scratch_bytes((low + states + steps) * sizeof(float)), s));
  if (!ws) return SPC_ERR_NOMEM;
  a.low = ws, a.between = ws + low, a.steps = a.between + states;
  scan_variant(d, gate != nullptr, [&](auto t, auto n, auto g) {
    using T = decltype(t);
    constexpr int NP = decltype(n)::value;
    constexpr bool GATE = decltype(g)::value;
    if (d->n_rows) launch_low<T>(a, log_np, s);
    if (cut) {
      hipLaunchKernelGGL((scan_kernel<T, NP, false, true, false>), dim3((a.ids * a.blocks + 3) / 4), dim3(SCAN_THREADS), 0, s, a);
      launch_chain(a, np, false, s);
    }
    hipLaunchKernelGGL((scan_kernel<T, NP, GATE, false, false>), dim3((a.ids * a.blocks + 3) / 4), dim3(SCAN_THREADS), 0, s, a);
  });
  pool_free(ws, s);
  SPC_HIP_CHECK(hipGetLastError());
  return SPC_OK;
}

extern "C" int spc_selective_scan_backward(const spc_scan_desc* d, const void* dout, int64_t ld_dout, const void* u, int64_t ld_u, const void* dt, int64_t ld_dt, const float* A,
                                           const spc_attn_rows* B, const spc_attn_rows* C, const float* skip, const void* gate, int64_t ld_gate, const float* dt_bias,
                                           const int32_t* offsets, const float* state_in, const float* dstate_out, void* du, int64_t ld_du, void* ddt, int64_t ld_ddt, float* dA,
                                           const spc_attn_rows* dB, const spc_attn_rows* dC, float* dskip, void* dgate, int64_t ld_dgate, float* ddt_bias, float* dstate_in,
                                           void* stream) {
  using namespace spc;
  SPC_RETURN_IF(check_scan(d, A, true, offsets));
  if (d->n_rows) {
    SPC_RETURN_IF(check_matrix("dout", dout, ld_dout, d));
    SPC_RETURN_IF(check_matrix("u", u, ld_u, d));
    SPC_RETURN_IF(check_matrix("dt", dt, ld_dt, d));
    SPC_RETURN_IF(check_matrix("du", du, ld_du, d));
    SPC_RETURN_IF(check_matrix("ddt", ddt, ld_ddt, d));
    if (gate) {
      SPC_RETURN_IF(check_matrix("gate", gate, ld_gate, d));
      SPC_RETURN_IF(check_matrix("dgate", dgate, ld_dgate, d));
    }
    SPC_RETURN_IF(check_low("B", B, d, false));
    SPC_RETURN_IF(check_low("C", C, d, false));
    SPC_RETURN_IF(check_low("dB", dB, d, true));
    SPC_RETURN_IF(check_low("dC", dC, d, true));
  }
  if (dstate_in && dstate_in == dstate_out) return set_error(SPC_ERR_ARG, "dstate_in is dstate_out");
  const StreamId s(static_cast<hipStream_t>(stream));
  const StreamWorkNote note{s};
  const int log_np = log_padded(d->states), np = 1 << log_np, waves = np / grad_states(np);
  ScanArgs a{};
  scan_shape(a, d);
  a.u = u, a.ld_u = ld_u, a.dt = dt, a.ld_dt = ld_dt, a.gate = gate, a.ld_gate = ld_gate, a.dout = dout, a.ld_dout = ld_dout;
  a.out = du, a.ld_out = ld_du, a.ddt = ddt, a.ld_ddt = ld_ddt, a.dgate = dgate, a.ld_dgate = ld_dgate;
  if (d->n_rows) a.b = low_rows(B), a.c = low_rows(C), a.db = low_rows(dB), a.dc = low_rows(dC);
  a.A = A, a.skip = skip, a.bias = dt_bias, a.state_in = state_in, a.dstate_out = dstate_out, a.dstate_in = dstate_in;
  a.scenes = {offsets, static_cast<int>(d->n_rows), d->n_scenes, segment_rows(d, a.blocks, 4096, 512, grad_rows(np))};
  a.ids = a.scenes.ids();
  SPC_RETURN_IF(check_grid(a, 64 * waves));
  const bool shared = a.blocks > a.groups;
  const size_t low = ((size_t(d->n_rows) + 1) * a.groups * 2) << log_np, steps = size_t(a.ids) * a.channels, states = steps * np;
  const size_t starts = (size_t(a.ids) + d->n_rows / grad_rows(np)) * (np + 1) * a.channels;
  const size_t parts = size_t(a.ids) * (np + 2) * a.channels, low_parts = shared ? (size_t(a.blocks) * d->n_rows * 2) << log_np : 0;
  float* ws = static_cast<float*>(pool_alloc(scratch_bytes((low + 2 * states + steps + starts + parts + low_parts) * sizeof(float)), s));
  if (!ws) return SPC_ERR_NOMEM;
  a.low = ws, a.between = ws + low, a.behind = a.between + states, a.steps = a.behind + states, a.starts = a.steps + steps;
  a.parts = a.starts + starts, a.low_parts = shared ? a.parts + parts : nullptr;
  scan_variant(d, gate != nullptr, [&](auto t, auto n, auto g) {
    using T = decltype(t);
    constexpr int NP = decltype(n)::value;
    constexpr bool GATE = decltype(g)::value;
    constexpr size_t lds = sizeof(GradLds<NP, GATE>);
    static_assert(lds <= 64 * 1024, "what a launch may ask for by itself");
    if (d->n_rows) {
      launch_low<T>(a, log_np, s);
      hipLaunchKernelGGL((scan_kernel<T, NP, GATE, true, true>), dim3((a.ids * a.blocks + 3) / 4), dim3(SCAN_THREADS), 0, s, a);
      launch_chain(a, np, true, s);
    }
    hipLaunchKernelGGL((scan_grad_kernel<T, NP, GATE>), dim3(a.ids * a.blocks), dim3(64 * waves), lds, s, a);
    if (shared && d->n_rows) {
      const int64_t m = d->n_rows * a.groups << (log_np + 1);
      hipLaunchKernelGGL(scan_low_grad_kernel<T>, dim3(std::min<int64_t>((m + 255) / 256, 8192)), dim3(256), 0, s, a, log_np);
    }
  });
  if (dA || dskip || ddt_bias)
    hipLaunchKernelGGL(scan_params_kernel, dim3(((np + 2) * a.channels + 31) / 32), dim3(1024), 0, s, a.parts, a.ids, np, a.channels, a.N, dA, dskip, ddt_bias);
  pool_free(ws, s);
  SPC_HIP_CHECK(hipGetLastError());
  return SPC_OK;
}

extern "C" int spc_selective_scan_step(const spc_scan_desc* d, const void* u, int64_t ld_u, const void* dt, int64_t ld_dt, const float* A, const spc_attn_rows* B,
                                       const spc_attn_rows* C, const float* skip, const void* gate, int64_t ld_gate, const float* dt_bias, float* state, void* out, int64_t ld_out,
                                       void* stream) {
  using namespace spc;
  SPC_RETURN_IF(check_scan(d, A, false, nullptr));
  if (!d->n_rows) return SPC_OK;
  SPC_RETURN_IF(check_matrix("u", u, ld_u, d));
  SPC_RETURN_IF(check_matrix("dt", dt, ld_dt, d));
  if (gate) SPC_RETURN_IF(check_matrix("gate", gate, ld_gate, d));
  SPC_RETURN_IF(check_matrix("out", out, ld_out, d));
  SPC_RETURN_IF(check_low("B", B, d, false));
  SPC_RETURN_IF(check_low("C", C, d, false));
  if (!state) return set_error(SPC_ERR_ARG, "state is NULL");
  const int vec = d->states % 4 ? 1 : 4;
  int log_q = 0;
  while ((vec << log_q) < d->states) ++log_q;
  if (d->n_rows > ((int64_t(1) << 31) - 1) / d->channels >> log_q) return set_error(SPC_ERR_UNSUPPORTED, "%lld streams of %d channels and %d states", static_cast<long long>(d->n_rows), d->channels, d->states);
  ScanArgs a{};
  scan_shape(a, d);
  a.u = u, a.ld_u = ld_u, a.dt = dt, a.ld_dt = ld_dt, a.gate = gate, a.ld_gate = ld_gate, a.out = out, a.ld_out = ld_out, a.b = low_rows(B), a.c = low_rows(C);
  a.A = A, a.skip = skip, a.bias = dt_bias;
  by_dtype(d->dtype, [&](auto t) {
    using T = decltype(t);
    const int64_t threads = d->n_rows * d->channels << log_q;
    auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, dim3((threads + 255) / 256), dim3(256), 0, static_cast<hipStream_t>(stream), a, state, static_cast<unsigned>(d->n_rows), log_q); };
    if (vec == 4) gate ? go(scan_step_kernel<T, 4, true>) : go(scan_step_kernel<T, 4, false>);
    else gate ? go(scan_step_kernel<T, 1, true>) : go(scan_step_kernel<T, 1, false>);
  });
  SPC_HIP_CHECK(hipGetLastError());
  return SPC_OK;
}
