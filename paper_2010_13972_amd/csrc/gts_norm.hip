// gts_norm_residual and its backward pass: both norms, the gate, the residual scale
// and the residual in one pass over the rows.
//
// A row lives in the registers of the TPR threads that share it, NV 16-byte vectors of
// each stream a thread, so every value is read once and statistics are taken about
// the mean in a second sweep over registers.
#include <algorithm>

#include "gts_nn_common.h"

namespace gts {
namespace nn {
namespace {

// Sums over the TPR threads of a row, up to 4 at once, in a fixed order.  Rows of a wave
// or less need no barrier; wider ones put their waves' sums in one of two LDS slots in
// turn, so that one barrier a sum is enough.
template <int TPR>
struct RowSum {
  static constexpr int kWaves = TPR < 64 ? 1 : TPR / 64;
  float (*lds)[4][kWaves];
  int turn = 0;

  template <int N>
  __device__ __forceinline__ void operator()(float (&v)[N]) {
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = lane_sum<(TPR < 64 ? TPR : 64)>(v[i]);
    if constexpr (kWaves > 1) {
      const int wave = threadIdx.x / 64;
      if (threadIdx.x % 64 == 0)
#pragma unroll
        for (int i = 0; i < N; ++i) lds[turn][i][wave] = v[i];
      __syncthreads();
#pragma unroll
      for (int i = 0; i < N; ++i) {
        v[i] = 0.0f;
#pragma unroll
        for (int w = 0; w < kWaves; ++w) v[i] += lds[turn][i][w];
      }
      turn ^= 1;
    }
  }
};

// Takes the mean off v where the norm is a layer norm (columns past the width stay 0).
template <int NV, int V>
__device__ __forceinline__ void centre(float (&v)[NV][V], float mean, const int64_t (&left)[NV]) {
#pragma unroll
  for (int j = 0; j < NV; ++j)
#pragma unroll
    for (int i = 0; i < V; ++i) v[j][i] = i < left[j] ? v[j][i] - mean : 0.0f;
}

template <int NV, int V>
__device__ __forceinline__ float sum_of(const float (&v)[NV][V]) {
  float s = 0.0f;
#pragma unroll
  for (int j = 0; j < NV; ++j)
#pragma unroll
    for (int i = 0; i < V; ++i) s += v[j][i];
  return s;
}

template <int NV, int V>
__device__ __forceinline__ float dot_of(const float (&a)[NV][V], const float (&b)[NV][V]) {
  float s = 0.0f;
#pragma unroll
  for (int j = 0; j < NV; ++j)
#pragma unroll
    for (int i = 0; i < V; ++i) s += a[j][i] * b[j][i];
  return s;
}

__device__ __forceinline__ float gate_value(float g, int kind) {
  return kind == GTS_GATE_SIGMOID ? sigmoid(g) : g;
}

template <class T, int NV>
__device__ __forceinline__ void load_row(float (&d)[NV][kVec<T>], const T* p, int step,
                                         const int64_t (&left)[NV]) {
#pragma unroll
  for (int j = 0; j < NV; ++j) load_vec<T, kVec<T>>(d[j], p + (int64_t)j * step, left[j]);
}

template <class T, int NV>
__device__ __forceinline__ void store_row(T* p, const float (&d)[NV][kVec<T>], int step,
                                          const int64_t (&left)[NV]) {
#pragma unroll
  for (int j = 0; j < NV; ++j) store_vec<T, kVec<T>>(p + (int64_t)j * step, d[j], left[j]);
}

template <int TPR>
constexpr int kThreads = TPR < 256 ? 256 : TPR;

// TPR threads hold a row in registers, so both norms read it once; narrow rows share a
// workgroup.  Bound by memory: 10000 x 2048 in bf16 takes 42.7 us over inputs that change
// from call to call (4.8 TB/s; a large copy reaches 4.9) and 35 over the same ones, which
// stay in the last-level cache.  4000 x 16384 takes 155 (4.2 TB/s).
template <class T, int TPR, int NV>
__global__ __launch_bounds__(kThreads<TPR>) void norm_kernel(const gts_norm_args a) {
  constexpr int V = kVec<T>, STEP = TPR * V;
  __shared__ float lds[2][4][RowSum<TPR>::kWaves];
  RowSum<TPR> row_sum{lds};
  const int t = threadIdx.x % TPR;
  const int64_t row = group_of_grid() * (kThreads<TPR> / TPR) + threadIdx.x / TPR;
  if (row >= a.rows) return;   // rows of a workgroup share no barrier, or there is one
  const int64_t c = (int64_t)t * V;
  int64_t left[NV];
#pragma unroll
  for (int j = 0; j < NV; ++j) left[j] = a.width - c - (int64_t)j * STEP;
  const float per = 1.0f / (float)a.width;
  const bool layer = a.norm == GTS_NORM_LAYER;
  float x[NV][V], f[NV][V], w[NV][V];
  load_row<T, NV>(f, static_cast<const T*>(a.f) + row * a.ld_f + c, STEP, left);
  load_row<T, NV>(x, static_cast<const T*>(a.x) + row * a.ld_x + c, STEP, left);
  load_row<T, NV>(w, static_cast<const T*>(a.w_post) + c, STEP, left);
  if (layer) {
    float s[1] = {sum_of(f)};
    row_sum(s);
    centre(f, s[0] * per, left);
  }
  float q[1] = {dot_of(f, f)};
  row_sum(q);
  const float rf = rsqrtf(q[0] * per + a.eps);
#pragma unroll
  for (int j = 0; j < NV; ++j)
#pragma unroll
    for (int i = 0; i < V; ++i) f[j][i] *= rf * w[j][i];
  if (a.gate_act != GTS_GATE_NONE) {
    float g[NV][V];
    load_row<T, NV>(g, static_cast<const T*>(a.gate) + row * a.ld_gate + c, STEP, left);
#pragma unroll
    for (int j = 0; j < NV; ++j)
#pragma unroll
      for (int i = 0; i < V; ++i) f[j][i] *= gate_value(g[j][i], a.gate_act);
  }
  if (a.scale != nullptr) {
    load_row<T, NV>(w, static_cast<const T*>(a.scale) + c, STEP, left);
#pragma unroll
    for (int j = 0; j < NV; ++j)
#pragma unroll
      for (int i = 0; i < V; ++i) f[j][i] *= w[j][i];
  }
#pragma unroll
  for (int j = 0; j < NV; ++j)
#pragma unroll
    for (int i = 0; i < V; ++i) x[j][i] += f[j][i];
  store_row<T, NV>(static_cast<T*>(a.u) + row * a.ld_u + c, x, STEP, left);
  load_row<T, NV>(w, static_cast<const T*>(a.w_pre) + c, STEP, left);
  if (layer) {
    float s[1] = {sum_of(x)};
    row_sum(s);
    centre(x, s[0] * per, left);
  }
  q[0] = dot_of(x, x);
  row_sum(q);
  const float ru = rsqrtf(q[0] * per + a.eps);
#pragma unroll
  for (int j = 0; j < NV; ++j)
#pragma unroll
    for (int i = 0; i < V; ++i) x[j][i] *= ru * w[j][i];
  store_row<T, NV>(static_cast<T*>(a.h) + row * a.ld_h + c, x, STEP, left);
}

// Threads of a backward workgroup: several rows of a wave or less, or one row.
template <int TPR>
constexpr int kGradThreads = TPR <= 64 ? 256 : TPR;

// A thread's 16-byte vector of a row as it lies in memory, zeros past the row's end.
template <class T>
using Packed = typename Unaligned<T, kVec<T>>::type;

template <class T, int NV>
__device__ __forceinline__ void load_packed(Packed<T> (&d)[NV], const T* p, int step,
                                            const int (&left)[NV]) {
#pragma unroll
  for (int j = 0; j < NV; ++j) {
    const T* q = p + (int64_t)j * step;
    if (left[j] >= kVec<T>) {
      d[j] = *reinterpret_cast<const Packed<T>*>(q);
    } else {
#pragma unroll
      for (int i = 0; i < kVec<T>; ++i) d[j][i] = i < left[j] ? q[i] : (T)0.0f;
    }
  }
}

// What a row of the backward pass reads.
template <class T, int NV>
struct GradRow {
  Packed<T> u[NV], f[NV], dh[NV], du[NV], gate[NV];

  __device__ __forceinline__ void load(const gts_norm_grad_args& a, int64_t row, int64_t c, int step,
                                       const int (&left)[NV]) {
    load_packed<T, NV>(u, static_cast<const T*>(a.u) + row * a.ld_u + c, step, left);
    load_packed<T, NV>(dh, static_cast<const T*>(a.dh) + row * a.ld_dh + c, step, left);
    load_packed<T, NV>(f, static_cast<const T*>(a.f) + row * a.ld_f + c, step, left);
    if (a.du != nullptr) load_packed<T, NV>(du, static_cast<const T*>(a.du) + row * a.ld_du + c, step, left);
    if (a.gate_act != GTS_GATE_NONE)
      load_packed<T, NV>(gate, static_cast<const T*>(a.gate) + row * a.ld_gate + c, step, left);
  }
};

// A workgroup takes every gridDim-th row (or four rows, a wave each) and keeps its
// threads' columns of the three weight gradients in registers, or with 1024 threads, whose
// registers are few, in LDS as far as it reaches; they go to part[workgroup][3][width] at
// its end, for column_sums_kernel.  Rows and weights stay
// packed as they were read, and with AHEAD the next row is on its way while one is
// worked on.
//
// Both norms' sums of a row meet in one exchange: the gradient along u is linear in u, so
// it needs no 1 / deviation yet.  Through a norm with output n = v / dev, a gradient d
// becomes (d - n mean(d n)) / dev, of a layer norm less its mean.
//
// Bound by memory: 10000 x 2048 in bf16 takes 73 us with column_sums_kernel (4.5 TB/s over
// the same inputs), 10000 x 4096 129 (5.1); 1000 x 785 in fp32 by two rows a workgroup and
// their exchanges, 13 us.  Rows past 8192 columns spill registers, 300 to 470 bytes a lane
// (4000 x 16384 505 us in bf16, 2.1 TB/s; 679 in fp32, 3.1).
template <class T, int TPR, int NV, bool LAYER, bool AHEAD>
__global__ __launch_bounds__(kGradThreads<TPR>) void norm_grad_kernel(const gts_norm_grad_args a,
                                                                      float* part) {
  constexpr int V = kVec<T>, STEP = TPR * V, ROWS = kGradThreads<TPR> / TPR;
  __shared__ float lds[2][4][RowSum<TPR>::kWaves];
  __shared__ float join[ROWS > 1 ? ROWS * STEP * NV : 1];
  constexpr int HELD = TPR < 1024 ? 0 : (3 * NV * STEP * 4 <= 100 * 1024 ? 3 : 2);   // sums in LDS
  __shared__ float held[HELD > 0 ? HELD : 1][HELD > 0 ? NV * STEP : 1];
  RowSum<TPR> row_sum{lds};
  const int t = threadIdx.x % TPR, sub = threadIdx.x / TPR;
  const int64_t c = (int64_t)t * V;
  int left[NV];
#pragma unroll
  for (int j = 0; j < NV; ++j) left[j] = (int)(a.width - c - (int64_t)j * STEP);
  const float per = 1.0f / (float)a.width;
  const bool gated = a.gate_act != GTS_GATE_NONE, scaled = a.scale != nullptr;
  const int64_t stride = (int64_t)gridDim.x * ROWS;
  int64_t row = (int64_t)blockIdx.x * ROWS + sub;
  float sums[HELD < 3 ? 3 - HELD : 1][NV][V] = {};
  if constexpr (HELD > 0)
    for (int k = t; k < HELD * NV * STEP; k += TPR) (&held[0][0])[k] = 0.0f;   // its own places
  // adds to sum k (pre, post, scale) of the thread's element i of vector j
  auto add = [&](auto k, int j, int i, float v) {
    constexpr int K = decltype(k)::value;
    if constexpr (K < HELD)
      held[K][(j * V + i) * TPR + t] += v;
    else
      sums[K - HELD][j][i] += v;
  };
  constexpr std::integral_constant<int, 0> kPre{};
  constexpr std::integral_constant<int, 1> kPost{};
  constexpr std::integral_constant<int, 2> kScale{};
  Packed<T> w_pre[NV], w_post[NV], scale[NV];
  load_packed<T, NV>(w_pre, static_cast<const T*>(a.w_pre) + c, STEP, left);
  load_packed<T, NV>(w_post, static_cast<const T*>(a.w_post) + c, STEP, left);
  if (scaled) load_packed<T, NV>(scale, static_cast<const T*>(a.scale) + c, STEP, left);
  GradRow<T, NV> next;
  if (AHEAD && row < a.rows) next.load(a, row, c, STEP, left);
  for (; row < a.rows; row += stride) {
    GradRow<T, NV> r;
    if constexpr (AHEAD) {
      r = next;
      if (row + stride < a.rows) next.load(a, row + stride, c, STEP, left);
    } else {
      r.load(a, row, c, STEP, left);
    }
    float mean_u = 0.0f, mean_f = 0.0f;
    if constexpr (LAYER) {
      float s[2] = {};
#pragma unroll
      for (int j = 0; j < NV; ++j)
#pragma unroll
        for (int i = 0; i < V; ++i) s[0] += (float)r.u[j][i], s[1] += (float)r.f[j][i];
      row_sum(s);
      mean_u = s[0] * per;
      mean_f = s[1] * per;
    }
    // values about the mean; columns past the width stay zero
    auto at_u = [&](int j, int i) { return LAYER && i >= left[j] ? 0.0f : (float)r.u[j][i] - mean_u; };
    auto at_f = [&](int j, int i) { return LAYER && i >= left[j] ? 0.0f : (float)r.f[j][i] - mean_f; };
    float s[LAYER ? 4 : 3] = {};   // u^2, f^2, d u and, of a layer norm, d; d = dh w_pre
#pragma unroll
    for (int j = 0; j < NV; ++j)
#pragma unroll
      for (int i = 0; i < V; ++i) {
        const float u = at_u(j, i), f = at_f(j, i), d = (float)r.dh[j][i] * (float)w_pre[j][i];
        s[0] += u * u;
        s[1] += f * f;
        s[2] += d * u;
        if constexpr (LAYER) s[3] += d;
      }
    row_sum(s);
    const float ru = rsqrtf(s[0] * per + a.eps), rf = rsqrtf(s[1] * per + a.eps);
    const float along = s[2] * ru * ru * per;
    float mean_d = 0.0f;
    if constexpr (LAYER) mean_d = s[3] * per;
    float e[NV][V], sum[2] = {};   // e = the gradient of N(f); its sums along N(f) and flat
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      float dx[V], dg[V], g[V];
#pragma unroll
      for (int i = 0; i < V; ++i) {
        const float u = at_u(j, i), dh = (float)r.dh[j][i];
        add(kPre, j, i, dh * (u * ru));
        dx[i] = (dh * (float)w_pre[j][i] - mean_d - u * along) * ru;
        g[i] = 1.0f;
      }
      if (a.du != nullptr)
#pragma unroll
        for (int i = 0; i < V; ++i) dx[i] += (float)r.du[j][i];
      store_vec<T, V>(static_cast<T*>(a.dx) + row * a.ld_dx + c + (int64_t)j * STEP, dx, left[j]);
      if (gated)
#pragma unroll
        for (int i = 0; i < V; ++i) g[i] = gate_value((float)r.gate[j][i], a.gate_act);
#pragma unroll
      for (int i = 0; i < V; ++i) {
        const float f = at_f(j, i) * rf, w = (float)w_post[j][i];
        const float to_n = dx[i] * (scaled ? (float)scale[j][i] : 1.0f);   // to gate . N(f) . w_post
        const float dn = to_n * g[i];
        dg[i] = to_n * f * w * (a.gate_act == GTS_GATE_SIGMOID ? g[i] * (1.0f - g[i]) : 1.0f);
        add(kScale, j, i, dx[i] * g[i] * (f * w));
        add(kPost, j, i, dn * f);
        e[j][i] = dn * w;
        sum[0] += e[j][i] * f;
        if constexpr (LAYER) sum[1] += e[j][i];
      }
      if (gated) store_vec<T, V>(static_cast<T*>(a.dgate) + row * a.ld_dgate + c + (int64_t)j * STEP, dg, left[j]);
    }
    row_sum(sum);
    const float along_f = sum[0] * per;
    if constexpr (LAYER) mean_d = sum[1] * per;
#pragma unroll
    for (int j = 0; j < NV; ++j) {
#pragma unroll
      for (int i = 0; i < V; ++i) e[j][i] = (e[j][i] - mean_d - at_f(j, i) * rf * along_f) * rf;
      store_vec<T, V>(static_cast<T*>(a.df) + row * a.ld_df + c + (int64_t)j * STEP, e[j], left[j]);
    }
  }
  float* out = part + (int64_t)blockIdx.x * 3 * a.width;
  auto put = [&](auto k) {
    constexpr int K = decltype(k)::value;
    float s[NV][V];
#pragma unroll
    for (int j = 0; j < NV; ++j)
#pragma unroll
      for (int i = 0; i < V; ++i) {
        if constexpr (K < HELD)
          s[j][i] = held[K][(j * V + i) * TPR + t];
        else
          s[j][i] = sums[K - HELD][j][i];
      }
    if constexpr (ROWS > 1) {
      __syncthreads();
#pragma unroll
      for (int j = 0; j < NV; ++j)
#pragma unroll
        for (int i = 0; i < V; ++i) join[sub * STEP * NV + j * STEP + c + i] = s[j][i];
      __syncthreads();
      for (int w = threadIdx.x; w < a.width; w += kGradThreads<TPR>) {
        float v = 0.0f;
#pragma unroll
        for (int r = 0; r < ROWS; ++r) v += join[r * STEP * NV + w];
        out[w] = v;
      }
    } else {
#pragma unroll
      for (int j = 0; j < NV; ++j) store_vec<float, V>(out + c + (int64_t)j * STEP, s[j], left[j]);
    }
    out += a.width;
  };
  put(kPre);
  put(kPost);
  put(kScale);
}

// The sums over the workgroups' parts.
template <class T>
__global__ __launch_bounds__(1024) void column_sums_kernel(const float* part, int64_t parts,
                                                           int64_t width, T* pre, T* post,
                                                           T* scale) {
  const int64_t c = (int64_t)blockIdx.x * kSumColumns + threadIdx.x % kSumColumns;
  const float sum = column_sum<1024>(part, parts, 3 * width, c);
  if (threadIdx.x >= kSumColumns || c >= 3 * width) return;
  T* out = c < width ? pre : (c < 2 * width ? post : scale);
  if (out != nullptr) out[c % width] = (T)sum;
}

// Calls f with the threads a row takes and the vectors a thread holds.
template <class F>
hipError_t with_shape(int64_t width, int vec, F&& f) {
  using std::integral_constant;
  const int64_t v = ceil_div(width, vec);
  if (v <= 8) return f(integral_constant<int, 8>{}, integral_constant<int, 1>{});
  if (v <= 32) return f(integral_constant<int, 32>{}, integral_constant<int, 1>{});
  if (v <= 64) return f(integral_constant<int, 64>{}, integral_constant<int, 1>{});
  if (v <= 128) return f(integral_constant<int, 64>{}, integral_constant<int, 2>{});
  if (v <= 256) return f(integral_constant<int, 256>{}, integral_constant<int, 1>{});
  if (v <= 512) return f(integral_constant<int, 256>{}, integral_constant<int, 2>{});
  if (v <= 1024) return f(integral_constant<int, 1024>{}, integral_constant<int, 1>{});
  if (v <= 2048) return f(integral_constant<int, 1024>{}, integral_constant<int, 2>{});
  return f(integral_constant<int, 1024>{}, integral_constant<int, 4>{});
}

// The same for the backward pass, whose threads hold a vector of each of eight streams
// and three sums of it: one vector a thread as far as threads go.
template <class F>
hipError_t with_grad_shape(int64_t width, int vec, F&& f) {
  using std::integral_constant;
  const int64_t v = ceil_div(width, vec);
  if (v <= 8) return f(integral_constant<int, 8>{}, integral_constant<int, 1>{});
  if (v <= 32) return f(integral_constant<int, 32>{}, integral_constant<int, 1>{});
  if (v <= 64) return f(integral_constant<int, 64>{}, integral_constant<int, 1>{});
  if (v <= 128) return f(integral_constant<int, 128>{}, integral_constant<int, 1>{});
  if (v <= 256) return f(integral_constant<int, 256>{}, integral_constant<int, 1>{});
  if (v <= 512) return f(integral_constant<int, 512>{}, integral_constant<int, 1>{});
  if (v <= 1024) return f(integral_constant<int, 1024>{}, integral_constant<int, 1>{});
  if (v <= 2048) return f(integral_constant<int, 1024>{}, integral_constant<int, 2>{});
  return f(integral_constant<int, 1024>{}, integral_constant<int, 4>{});
}

// Workgroups of the backward pass: up to 12 waves a compute unit, and few enough rows'
// worth of parts beside the rows themselves.
int64_t grad_groups(int64_t rows, int64_t width, int64_t size) {
  const int64_t v = ceil_div(width * size, 16);
  const int64_t threads = v <= 64 ? 256 : v <= 128 ? 128 : v <= 256 ? 256 : v <= 512 ? 512 : 1024;
  const int64_t at_once = v <= 8 ? 32 : v <= 32 ? 8 : v <= 64 ? 4 : 1;
  const int64_t most = 256 * std::max<int64_t>(1, 768 / threads);
  return std::min(ceil_div(rows, at_once * 2), most);
}

gts_status check_norm(int64_t rows, int64_t width, int32_t dtype, int32_t norm, int32_t gate_act, float eps) {
  if (!known_type(dtype)) return fail(GTS_EINVAL, "dtype %d is not GTS_F32, GTS_BF16 or GTS_F16", dtype);
  if (rows < 0 || rows > INT32_MAX) return fail(GTS_EINVAL, "rows must be >= 0 and below 2^31");
  if (width < 1 || width > GTS_NORM_MAX_WIDTH)
    return fail(GTS_EINVAL, "width must be from 1 to %d", GTS_NORM_MAX_WIDTH);
  if (norm != GTS_NORM_RMS && norm != GTS_NORM_LAYER) return fail(GTS_EINVAL, "unknown norm %d", norm);
  if (gate_act < GTS_GATE_NONE || gate_act > GTS_GATE_SIGMOID)
    return fail(GTS_EINVAL, "unknown gate %d", gate_act);
  if (!(eps >= 0.0f)) return fail(GTS_EINVAL, "eps must be >= 0");
  return GTS_OK;
}

gts_status check_launch(hipError_t e) {
  return e == hipSuccess ? GTS_OK : fail(GTS_EDEVICE, "norm launch failed: %s", hipGetErrorString(e));
}

}  // namespace
}  // namespace nn
}  // namespace gts

extern "C" gts_status gts_norm_residual(const gts_norm_args* a, void* stream) {
  using namespace gts;
  using namespace gts::nn;
  clear_error();
  if (a == nullptr) return fail(GTS_EINVAL, "args must not be NULL");
  gts_status st = check_norm(a->rows, a->width, a->dtype, a->norm, a->gate_act, a->eps);
  if (st != GTS_OK) return st;
  const bool gated = a->gate_act != GTS_GATE_NONE;
  if (!gated && a->gate != nullptr) return fail(GTS_EINVAL, "a gate without a gate_act");
  const Matrix m[] = {{"x", a->x, a->ld_x, a->width, true},
                      {"f", a->f, a->ld_f, a->width, true},
                      {"gate", a->gate, a->ld_gate, a->width, gated},
                      {"u", a->u, a->ld_u, a->width, true},
                      {"h", a->h, a->ld_h, a->width, true},
                      {"scale", a->scale, a->width, a->width, false}};
  if ((st = check_matrices(m, 6, type_size(a->dtype), a->rows == 0)) != GTS_OK) return st;
  const Matrix w[] = {{"w_post", a->w_post, a->width, a->width, true},
                      {"w_pre", a->w_pre, a->width, a->width, true}};
  if ((st = check_matrices(w, 2, type_size(a->dtype), false)) != GTS_OK) return st;
  if (a->rows == 0) return GTS_OK;
  return with_type(a->dtype, [&](auto t) {
    using T = decltype(t);
    return check_launch(with_shape(a->width, kVec<T>, [&](auto tpr, auto nv) {
      constexpr int TPR = decltype(tpr)::value, NV = decltype(nv)::value;
      if constexpr (TPR * NV * kVec<T> < 2 * GTS_NORM_MAX_WIDTH) {
        const dim3 grid = grid_of(ceil_div(a->rows, kThreads<TPR> / TPR));
        norm_kernel<T, TPR, NV><<<grid, kThreads<TPR>, 0, static_cast<hipStream_t>(stream)>>>(*a);
        return hipGetLastError();
      } else {
        return hipErrorInvalidValue;   // wider than any call's row
      }
    }));
  });
}

extern "C" gts_status gts_norm_residual_backward_workspace_bytes(int64_t rows, int64_t width,
                                                                 int64_t* bytes) {
  using namespace gts;
  clear_error();
  if (bytes == nullptr) return fail(GTS_EINVAL, "bytes must not be NULL");
  gts_status st = nn::check_norm(rows, width, GTS_F32, GTS_NORM_RMS, GTS_GATE_NONE, 0.0f);
  if (st != GTS_OK) return st;
  const int64_t groups = std::max(nn::grad_groups(rows, width, 2), nn::grad_groups(rows, width, 4));
  *bytes = nn::ceil_div(groups * 3 * width * 4, 16) * 16;
  return GTS_OK;
}

extern "C" gts_status gts_norm_residual_backward(const gts_norm_grad_args* a, void* d_workspace,
                                                 int64_t workspace_bytes, void* stream) {
  using namespace gts;
  using namespace gts::nn;
  clear_error();
  if (a == nullptr) return fail(GTS_EINVAL, "args must not be NULL");
  gts_status st = check_norm(a->rows, a->width, a->dtype, a->norm, a->gate_act, a->eps);
  if (st != GTS_OK) return st;
  const bool gated = a->gate_act != GTS_GATE_NONE;
  const bool empty = a->rows == 0;
  if (!gated && (a->gate != nullptr || a->dgate != nullptr))
    return fail(GTS_EINVAL, "a gate without a gate_act");
  if ((a->scale != nullptr) != (a->dscale != nullptr))
    return fail(GTS_EINVAL, "dscale must be given exactly if scale is");
  const int64_t es = type_size(a->dtype);
  const Matrix m[] = {{"du", a->du, a->ld_du, a->width, false},
                      {"dh", a->dh, a->ld_dh, a->width, true},
                      {"u", a->u, a->ld_u, a->width, true},
                      {"f", a->f, a->ld_f, a->width, true},
                      {"gate", a->gate, a->ld_gate, a->width, gated},
                      {"dx", a->dx, a->ld_dx, a->width, true},
                      {"df", a->df, a->ld_df, a->width, true},
                      {"dgate", a->dgate, a->ld_dgate, a->width, gated}};
  if ((st = check_matrices(m, 8, es, empty)) != GTS_OK) return st;
  const Matrix w[] = {{"scale", a->scale, a->width, a->width, false},
                      {"dscale", a->dscale, a->width, a->width, false},
                      {"w_post", a->w_post, a->width, a->width, true},
                      {"w_pre", a->w_pre, a->width, a->width, true},
                      {"dw_post", a->dw_post, a->width, a->width, true},
                      {"dw_pre", a->dw_pre, a->width, a->width, true}};
  if ((st = check_matrices(w, 6, es, false)) != GTS_OK) return st;
  int64_t need = 0;
  gts_norm_residual_backward_workspace_bytes(a->rows, a->width, &need);
  if ((st = check_workspace(d_workspace, workspace_bytes, need)) != GTS_OK) return st;
  hipStream_t s = static_cast<hipStream_t>(stream);
  float* part = static_cast<float*>(d_workspace);
  return with_type(a->dtype, [&](auto t) {
    using T = decltype(t);
    int64_t groups = 0;
    hipError_t e = hipSuccess;
    if (!empty)
      e = with_grad_shape(a->width, kVec<T>, [&](auto tpr, auto nv) {
        constexpr int TPR = decltype(tpr)::value, NV = decltype(nv)::value;
        if constexpr (TPR * NV * kVec<T> < 2 * GTS_NORM_MAX_WIDTH) {
          groups = grad_groups(a->rows, a->width, es);
          // 1024 threads have registers for one row only
          if (a->norm == GTS_NORM_LAYER)
            norm_grad_kernel<T, TPR, NV, true, (TPR < 1024)><<<(unsigned)groups, kGradThreads<TPR>, 0, s>>>(*a, part);
          else
            norm_grad_kernel<T, TPR, NV, false, (TPR < 1024)><<<(unsigned)groups, kGradThreads<TPR>, 0, s>>>(*a, part);
          return hipGetLastError();
        } else {
          return hipErrorInvalidValue;
        }
      });
    if (e == hipSuccess) {
      column_sums_kernel<T><<<(unsigned)ceil_div(3 * a->width, kSumColumns), 1024, 0, s>>>(
          part, groups, a->width, static_cast<T*>(a->dw_pre), static_cast<T*>(a->dw_post),
          static_cast<T*>(a->dscale));
      e = hipGetLastError();
    }
    return check_launch(e);
  });
}
