// What the operators of gts_nn.h share: element types, vector loads and stores,
// reductions over lanes, activations.  Not part of the public ABI.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>
#include <type_traits>

#include "gts_internal.h"
#include "gts_nn.h"

namespace gts {
namespace nn {

using bf16 = __bf16;
using f16 = _Float16;

inline bool known_type(int32_t t) { return t == GTS_F32 || t == GTS_BF16 || t == GTS_F16; }
inline int64_t type_size(int32_t t) { return t == GTS_F32 ? 4 : 2; }

// Calls `f` with a value of the element type `t` stands for.
template <class F>
auto with_type(int32_t t, F&& f) {
  if (t == GTS_BF16) return f(bf16{});
  if (t == GTS_F16) return f(f16{});
  return f(float{});
}

inline bool misaligned(const void* p, int64_t to) {
  return (reinterpret_cast<uintptr_t>(p) & (uintptr_t)(to - 1)) != 0;
}

__host__ __device__ inline int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

// The grid of `groups` workgroups (at least 1): work-items along one axis have to stay below
// 2^32, so past 2^20 workgroups they go on along the second, where the last row may be
// longer than what is left.
inline dim3 grid_of(int64_t groups) {
  const int64_t along = groups < (1 << 20) ? groups : 1 << 20;
  return dim3((unsigned)along, (unsigned)ceil_div(groups, along));
}

// The workgroup's number in such a grid.
__device__ __forceinline__ int64_t group_of_grid() { return (int64_t)blockIdx.y * gridDim.x + blockIdx.x; }

// A matrix argument: its row stride must hold its width, both below 2^31.
struct Matrix {
  const char* name;
  const void* p;
  int64_t ld, width;
  bool needed;
};

inline gts_status check_matrices(const Matrix* m, int n, int64_t elem, bool empty) {
  for (int i = 0; i < n; ++i) {
    if (m[i].p == nullptr) {
      // a tensor without elements may have no address
      if (m[i].needed && !empty) return fail(GTS_EINVAL, "%s must not be NULL", m[i].name);
      continue;
    }
    if (misaligned(m[i].p, elem)) return fail(GTS_EINVAL, "%s is not aligned to its element", m[i].name);
    if (m[i].ld < m[i].width || m[i].ld > INT32_MAX)
      return fail(GTS_EINVAL, "the row stride of %s is below its width, or 2^31 or more", m[i].name);
  }
  return GTS_OK;
}

inline gts_status check_workspace(const void* p, int64_t have, int64_t need) {
  if (have < need)
    return fail(GTS_EBUFSIZE, "workspace_bytes %lld < %lld", (long long)have, (long long)need);
  if (need > 0 && (p == nullptr || misaligned(p, 16)))
    return fail(GTS_EINVAL, "d_workspace must not be NULL and be aligned to 16 bytes");
  return GTS_OK;
}

// Elements of a 16-byte access.
template <class T>
constexpr int kVec = 16 / (int)sizeof(T);

template <class T, int N>
struct Unaligned {
  typedef T type __attribute__((ext_vector_type(N), aligned(sizeof(T))));
};

// N consecutive elements from p, of which the first `n` exist (n >= N: all of them);
// the others read as zero.  p has its element's alignment only: the hardware takes
// 16-byte accesses at any element's address, aligned ones faster.
template <class T, int N>
__device__ __forceinline__ void load_vec(float (&d)[N], const T* p, int64_t n) {
  if (n >= N) {
    const auto t = *reinterpret_cast<const typename Unaligned<T, N>::type*>(p);
#pragma unroll
    for (int i = 0; i < N; ++i) d[i] = (float)t[i];
  } else {
#pragma unroll
    for (int i = 0; i < N; ++i) d[i] = i < n ? (float)p[i] : 0.0f;
  }
}

template <class T, int N>
__device__ __forceinline__ void store_vec(T* p, const float (&s)[N], int64_t n) {
  if (n >= N) {
    typename Unaligned<T, N>::type t;
#pragma unroll
    for (int i = 0; i < N; ++i) t[i] = (T)s[i];
    *reinterpret_cast<typename Unaligned<T, N>::type*>(p) = t;
  } else {
#pragma unroll
    for (int i = 0; i < N; ++i)
      if (i < n) p[i] = (T)s[i];
  }
}

constexpr float kLog2e = 1.4426950408889634f;

__device__ __forceinline__ float exp2_of(float x) { return __builtin_amdgcn_exp2f(x); }

// 1 / (1 + 2^x), within a few ulp: 2^x = inf gives 0.
__device__ __forceinline__ float logistic2(float x) { return __builtin_amdgcn_rcpf(1.0f + exp2_of(x)); }

__device__ __forceinline__ float sigmoid(float z) { return logistic2(-kLog2e * z); }

// GELU is z sigmoid(a (z + b z^3)), a = 2 sqrt(2 / pi), since (1 + tanh(t)) / 2 =
// sigmoid(2 t); its sigmoid is 1 / (1 + 2^(z (c + d z^2))).
constexpr float kGeluA = 1.5957691216057308f;
constexpr float kGeluB = 0.044715f;
constexpr float kGeluC = -kLog2e * kGeluA, kGeluD = kGeluC * kGeluB;

// Where a factor can be infinite it is held to a range outside which the sigmoid is 0 or 1 in
// 32 bits, so that the limits at infinity come out; a NaN stays one.
template <int ACT>
__device__ __forceinline__ float act_value(float z) {
  if constexpr (ACT == GTS_ACT_RELU) return z > 0.0f ? z : (z != z ? z : 0.0f);
  if constexpr (ACT == GTS_ACT_SILU) return fmaxf(z, -3e38f) * sigmoid(z);
  if constexpr (ACT == GTS_ACT_GELU) return fmaxf(z, -3e38f) * logistic2(z * (kGeluC + kGeluD * (z * z)));
  return z;
}

template <int ACT>
__device__ __forceinline__ float act_slope(float z) {
  if constexpr (ACT == GTS_ACT_RELU) return z > 0.0f ? 1.0f : (z != z ? z : 0.0f);
  const float zc = fminf(fmaxf(z, -1e4f), 1e4f);
  if constexpr (ACT == GTS_ACT_SILU) {
    const float p = sigmoid(z);
    return p + zc * p * (1.0f - p);
  }
  if constexpr (ACT == GTS_ACT_GELU) {
    const float p = logistic2(z * (kGeluC + kGeluD * (z * z)));
    return p + zc * p * (1.0f - p) * (kGeluA + 3.0f * kGeluA * kGeluB * (zc * zc));
  }
  return 1.0f;
}

// Runs f with the activation as a constant.
template <class F>
__device__ __forceinline__ void with_act(int act, F&& f) {
  if (act == GTS_ACT_RELU) f(std::integral_constant<int, GTS_ACT_RELU>{});
  else if (act == GTS_ACT_SILU) f(std::integral_constant<int, GTS_ACT_SILU>{});
  else if (act == GTS_ACT_GELU) f(std::integral_constant<int, GTS_ACT_GELU>{});
}

// The sum over a group of LANES consecutive lanes (a power of two up to 64), in all
// of them, in a fixed order.
template <int LANES>
__device__ __forceinline__ float lane_sum(float v) {
#pragma unroll
  for (int d = 1; d < LANES; d *= 2) v += __shfl_xor(v, d, 64);
  return v;
}

// The sum over the rows of part[parts][n] of one of 32 columns, by a workgroup of THREADS
// (32 columns side by side, 4 loads a thread on their way), in a fixed order; the result in
// the first 32 threads.
constexpr int kSumColumns = 32;
template <int THREADS>
__device__ __forceinline__ float column_sum(const float* part, int64_t parts, int64_t n, int64_t c) {
  constexpr int DEEP = THREADS / kSumColumns;
  __shared__ float join[THREADS / 64][kSumColumns];
  const int q = threadIdx.x / kSumColumns;
  float acc[4] = {};
  if (c < n)
    for (int64_t p = q; p < parts; p += 4 * DEEP)
#pragma unroll
      for (int i = 0; i < 4; ++i) acc[i] += p + i * DEEP < parts ? part[(p + i * DEEP) * n + c] : 0.0f;
  float sum = (acc[0] + acc[1]) + (acc[2] + acc[3]);
  sum += __shfl_xor(sum, kSumColumns, 64);
  if (threadIdx.x % 64 < kSumColumns) join[threadIdx.x / 64][threadIdx.x % 64] = sum;
  __syncthreads();
  sum = 0.0f;
  if (threadIdx.x < kSumColumns)
    for (int i = 0; i < THREADS / 64; ++i) sum += join[i][threadIdx.x];
  return sum;
}

}  // namespace nn
}  // namespace gts
