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
#include <algorithm>

#include "spc_internal.h"

namespace spc {
namespace {

constexpr int ATTN_MAX_D = 128;
constexpr int ATTN_MAX_JOBS = 3;

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
  float scale;
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
    n = max((hi - lo + a.seg_rows - 1) / a.seg_rows, 1);
    rows = min(a.seg_rows, hi - lo - m * a.seg_rows);
    return m >= 0 && m < n;
  }
  __device__ int64_t row(bool reverse, int i) const { return reverse ? int64_t(hi) - 1 - i : int64_t(lo) + i; }
};

__device__ inline float decay_power(float log_decay, int n) { return n > 0 ? expf(log_decay * n) : 1.f; }

// One token after the other, the state in LDS.
template <typename T, bool OUT>
__global__ __launch_bounds__(256) void scan_rows_kernel(const ScanArgs a) {
  extern __shared__ float lds[];
  const Job& j = a.job[blockIdx.x % a.n_jobs];
  const int h = blockIdx.x / a.n_jobs % a.heads, id = blockIdx.x / a.n_jobs / a.heads;
  Segment s;
  if (!s.find(a, id)) return;
  if (!OUT && s.m == s.n - 1) return;  // nobody starts from it
  const int e = j.dy * j.dz, t = threadIdx.x;
  float *S = lds, *x = S + e, *y = x + ATTN_MAX_D, *z = y + ATTN_MAX_D;
  const float l = expf(a.log_decay[h]), upd = j.reverse ? a.scale : 1.f, of = j.reverse ? 1.f : a.scale;
  for (int i = t; i < e; i += 256) {
    float v = 0.f;
    if (OUT && s.m) v = j.between.of(id - 1, a.heads, h)[(i / j.dz) * j.between.r + (i % j.dz) * j.between.c];
    else if (OUT && j.first.p) v = j.first.of(s.scene, a.heads, h)[(i / j.dz) * j.first.r + (i % j.dz) * j.first.c];
    S[i] = v;
  }
  for (int i = 0; i < s.rows; ++i) {
    const int64_t row = s.row(j.reverse, s.m * a.seg_rows + i);
    __syncthreads();
    if (OUT && t < j.dy) x[t] = static_cast<float>(static_cast<const T*>(j.x.p)[j.x.at(row, h) + t]);
    if (t < j.dy) y[t] = upd * static_cast<float>(static_cast<const T*>(j.y.p)[j.y.at(row, h) + t]);
    if (t < j.dz) z[t] = static_cast<float>(static_cast<const T*>(j.z.p)[j.z.at(row, h) + t]);
    __syncthreads();
    const float f = j.reverse && !s.m && !i ? 1.f : l;  // (the gradient of the last state meets the last token undecayed)
    for (int k = t; k < e; k += 256) S[k] = f * S[k] + y[k / j.dz] * z[k % j.dz];
    __syncthreads();
    if (OUT && t < j.dz) {
      float o = 0.f;
      for (int r = 0; r < j.dy; ++r) o = fmaf(x[r], S[r * j.dz + t], o);
      const int64_t at = j.out.at(row, h) + t;
      if (j.out_f32) static_cast<float*>(j.out.p)[at] = of * o;
      else static_cast<T*>(j.out.p)[at] = static_cast<T>(of * o);
    }
  }
  __syncthreads();
  const States& to = OUT ? j.last : j.between;
  if (OUT && (s.m != s.n - 1 || !to.p)) return;
  const float f = OUT && j.reverse && s.hi > s.lo ? l : 1.f;  // (what reaches the state before the first token)
  float* p = to.of(OUT ? s.scene : id, a.heads, h);
  for (int i = t; i < e; i += 256) p[(i / j.dz) * to.r + (i % j.dz) * to.c] = f * S[i];
}

// Sums of segments -> the state behind every segment but the last of its scene, in place.
__global__ __launch_bounds__(256) void scan_states_kernel(const ScanArgs a) {
  const Job& j = a.job[blockIdx.z];
  const int h = blockIdx.y % a.heads, scene = blockIdx.y / a.heads, i = blockIdx.x * 256 + threadIdx.x;
  if (i >= j.dy * j.dz) return;
  const int lo = a.offsets ? min(max(a.offsets[scene], 0), a.n_rows) : 0;
  const int id = lo / a.seg_rows + scene;
  Segment s;
  if (!s.find(a, id) || s.scene != scene) return;
  const float l = a.log_decay[h];
  const int r = i / j.dz, c = i % j.dz;
  float S = j.first.p ? j.first.of(scene, a.heads, h)[r * j.first.r + c * j.first.c] : 0.f;
  const float whole = decay_power(l, a.seg_rows);
  for (int m = 0; m + 1 < s.n; ++m) {
    float* p = j.between.of(id + m, a.heads, h) + r * j.between.r + c * j.between.c;
    S = (j.reverse && !m ? decay_power(l, a.seg_rows - 1) : whole) * S + *p;
    *p = S;
  }
}

// Gradients of keys and values that `group` heads share.
template <typename T>
__global__ __launch_bounds__(256) void sum_heads_kernel(const float* __restrict__ part, Rows out, int64_t n_rows, int kv_heads, int group, int d) {
  const int64_t i = blockIdx.x * int64_t(256) + threadIdx.x;
  if (i >= n_rows * kv_heads * d) return;
  const int c = static_cast<int>(i % d), h = static_cast<int>(i / d % kv_heads);
  const int64_t row = i / d / kv_heads;
  const float* p = part + ((row * kv_heads + h) * group) * d + c;
  float s = 0.f;
  for (int g = 0; g < group; ++g) s += p[int64_t(g) * d];
  static_cast<T*>(out.p)[row * out.row + h * out.head + c] = static_cast<T>(s);
}

template <typename T>
__global__ __launch_bounds__(256) void attention_step_kernel(Rows q, Rows k, Rows v, Rows out, float* state, const float* log_decay, int heads,
                                                             int dk, int dv, float scale) {
  __shared__ float qs[ATTN_MAX_D], ks[ATTN_MAX_D], part[256];
  const int h = blockIdx.x % heads, t = threadIdx.x;
  const int64_t row = blockIdx.x / heads;
  if (t < dk) {
    qs[t] = scale * static_cast<float>(static_cast<const T*>(q.p)[q.at(row, h) + t]);
    ks[t] = static_cast<float>(static_cast<const T*>(k.p)[k.at(row, h) + t]);
  }
  __syncthreads();
  const float l = expf(log_decay[h]);
  float* S = state + int64_t(blockIdx.x) * dk * dv;
  for (int c0 = 0; c0 < dv; c0 += 32) {
    const int c = c0 + t % 32;
    float o = 0.f;
    if (c < dv) {
      const float vc = static_cast<float>(static_cast<const T*>(v.p)[v.at(row, h) + c]);
      for (int r = t / 32; r < dk; r += 8) {
        const float s = l * S[r * dv + c] + ks[r] * vc;
        S[r * dv + c] = s;
        o = fmaf(qs[r], s, o);
      }
    }
    part[t] = o;
    __syncthreads();
    if (t < 32 && c < dv) {
      for (int g = 1; g < 8; ++g) o += part[t + 32 * g];
      static_cast<T*>(out.p)[out.at(row, h) + c] = static_cast<T>(o);
    }
    __syncthreads();
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
int check_desc(const spc_attn_desc* d) {
  if (!d) return set_error(SPC_ERR_ARG, "descriptor is NULL");
  if (d->dtype != SPC_DTYPE_F16 && d->dtype != SPC_DTYPE_BF16 && d->dtype != SPC_DTYPE_F32)
    return set_error(SPC_ERR_ARG, "unknown dtype %d", d->dtype);
  if (d->n_rows < 0 || d->n_scenes < 1 || d->heads < 1 || d->kv_heads < 1 || d->heads % d->kv_heads || d->dk < 1 || d->dv < 1)
    return set_error(SPC_ERR_ARG, "%lld rows, %d scenes, %d heads over %d, %d and %d channels", static_cast<long long>(d->n_rows), d->n_scenes,
                     d->heads, d->kv_heads, d->dk, d->dv);
  if (!(d->scale > -3.4e38f && d->scale < 3.4e38f)) return set_error(SPC_ERR_ARG, "scale is not finite");
  if (d->dk > ATTN_MAX_D || d->dv > ATTN_MAX_D) return set_error(SPC_ERR_UNSUPPORTED, "heads of %d and %d channels: at most %d", d->dk, d->dv, ATTN_MAX_D);
  if (d->n_rows >= (int64_t(1) << 31) || (d->n_rows / 64 + d->n_scenes) * d->heads * ATTN_MAX_JOBS >= (int64_t(1) << 31))
    return set_error(SPC_ERR_UNSUPPORTED, "%lld rows of %d heads in %d scenes", static_cast<long long>(d->n_rows), d->heads, d->n_scenes);
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

template <typename F>
void by_dtype(int32_t dtype, F&& f) {
  if (dtype == SPC_DTYPE_F16) f(_Float16{});
  else if (dtype == SPC_DTYPE_BF16) f(__bf16{});
  else f(0.f);
}

// Rows of a segment: multiples of 64, as few as give some 1024 workgroups a job.
int segment_rows(const spc_attn_desc* d) {
  const int64_t want = (d->n_rows * d->heads + 1023) / 1024;
  return static_cast<int>(std::max<int64_t>(64, (want + 63) / 64 * 64));
}

// The states between segments of `a`'s first `n_sums` jobs lie in `ws`; the jobs behind them have theirs in place.
int run_scan(ScanArgs& a, int n_sums, int32_t dtype, hipStream_t s) {
  const size_t e = size_t(a.job[0].dy) * a.job[0].dz;
  by_dtype(dtype, [&](auto t) {
    using T = decltype(t);
    const size_t lds = (e + 3 * ATTN_MAX_D) * sizeof(float);
    const int jobs = a.n_jobs;
    if (n_sums && a.n_rows > a.seg_rows) {
      a.n_jobs = n_sums;
      hipLaunchKernelGGL((scan_rows_kernel<T, false>), dim3(a.n_ids * a.heads * n_sums), dim3(256), lds, s, a);
      hipLaunchKernelGGL(scan_states_kernel, dim3((e + 255) / 256, a.n_scenes * a.heads, n_sums), dim3(256), 0, s, a);
      a.n_jobs = jobs;
    }
    hipLaunchKernelGGL((scan_rows_kernel<T, true>), dim3(a.n_ids * a.heads * jobs), dim3(256), lds, s, a);
  });
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
  a.seg_rows = segment_rows(d);
  a.n_ids = a.n_rows / a.seg_rows + a.n_scenes;
  float* ws = nullptr;
  if (a.n_rows > a.seg_rows) {
    ws = static_cast<float*>(pool_alloc(size_t(a.n_ids) * a.heads * e * sizeof(float), s));
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
  a.seg_rows = segment_rows(d);
  a.n_ids = a.n_rows / a.seg_rows + a.n_scenes;
  const size_t states = a.n_rows > a.seg_rows ? size_t(a.n_ids) * a.heads * e : 0;
  const size_t parts = group > 1 ? size_t(a.n_rows) * a.heads : 0;  // gradients of shared keys and values, by head
  float* ws = nullptr;
  if (states || parts) {
    ws = static_cast<float*>(pool_alloc((2 * states + parts * (d->dk + d->dv)) * sizeof(float), s));
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
      const int64_t nk = int64_t(a.n_rows) * d->kv_heads * d->dk, nv = int64_t(a.n_rows) * d->kv_heads * d->dv;
      hipLaunchKernelGGL(sum_heads_kernel<T>, dim3((nk + 255) / 256), dim3(256), 0, s, part_k, rows_of(dk, 1), a.n_rows, d->kv_heads, group, d->dk);
      hipLaunchKernelGGL(sum_heads_kernel<T>, dim3((nv + 255) / 256), dim3(256), 0, s, part_v, rows_of(dv, 1), a.n_rows, d->kv_heads, group, d->dv);
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
  SPC_RETURN_IF(check_desc(d));
  if (d->n_rows * d->heads >= (int64_t(1) << 31)) return set_error(SPC_ERR_UNSUPPORTED, "%lld streams of %d heads", static_cast<long long>(d->n_rows), d->heads);
  if (!log_decay) return set_error(SPC_ERR_ARG, "log_decay is NULL");
  if (!d->n_rows) return SPC_OK;
  if (!state) return set_error(SPC_ERR_ARG, "state is NULL");
  SPC_RETURN_IF(check_rows("q", q, d, d->heads, d->dk, false));
  SPC_RETURN_IF(check_rows("k", k, d, d->kv_heads, d->dk, false));
  SPC_RETURN_IF(check_rows("v", v, d, d->kv_heads, d->dv, false));
  SPC_RETURN_IF(check_rows("out", out, d, d->heads, d->dv, true));
  const int group = d->heads / d->kv_heads;
  by_dtype(d->dtype, [&](auto t) {
    hipLaunchKernelGGL(attention_step_kernel<decltype(t)>, dim3(d->n_rows * d->heads), dim3(256), 0, static_cast<hipStream_t>(stream), rows_of(q, 1),
                       rows_of(k, group), rows_of(v, group), rows_of(out, 1), state, log_decay, d->heads, d->dk, d->dv, d->scale);
  });
  SPC_HIP_CHECK(hipGetLastError());
  return SPC_OK;
}

extern "C" int spc_batch_offsets(const void* keys, int64_t n, const spc_pack_desc* d, int32_t n_batch, int32_t* offsets, void* stream) {
  using namespace spc;
  PackInfo pi;
  if (!d || !offsets) return set_error(SPC_ERR_ARG, "NULL argument");
  SPC_RETURN_IF(spc::check_desc(d, &pi));
  if (n < 0 || n >= (int64_t(1) << 31) || n_batch < 1 || (n && !keys)) return set_error(SPC_ERR_ARG, "%lld keys of %d scenes", static_cast<long long>(n), n_batch);
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
