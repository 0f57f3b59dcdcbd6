// gts_grad_clip and gts_adamw: the optimizer's step over many tensors at once.
//
// A launch takes up to kTensors tensors, whose addresses travel in its arguments; a
// workgroup finds its tensor by the chunks before it.  Bound by memory: the step moves
// each value once and computes some twenty operations on it.
#include <algorithm>
#include <cmath>

#include "gts_nn_common.h"

namespace gts {
namespace nn {
namespace {

constexpr int kTensors = 80;         // 3856 bytes of arguments
constexpr int kItems = 8;            // consecutive elements a thread takes
constexpr int64_t kChunk = 256 * kItems * 4;
constexpr int64_t kMostChunks = (1 << 24) - 1;   // of a launch
constexpr int kBlockLanes = GTS_STATE_BLOCK / kItems;   // lanes that share a scale

struct Table {
  int64_t first[kTensors + 1];   // chunks before tensor i
  gts_tensor t[kTensors];
  int n;
};
static_assert(sizeof(Table) <= 3900, "the table has to fit a launch's arguments");

__device__ __forceinline__ int find(const Table& tab, int64_t chunk) {
  int lo = 0, hi = tab.n;
  while (hi - lo > 1) {
    const int mid = (lo + hi) / 2;
    if (tab.first[mid] <= chunk)
      lo = mid;
    else
      hi = mid;
  }
  return lo;
}

// The sum of the squares of one chunk of one gradient, in 64 bits: squares of gradients above
// 1.8e19 or below 1e-23 are no 32-bit numbers, though the norm is one.  Bound by
// memory: 127 M values in bf16 take 50 us with clip_kernel (5.1 TB/s) where no pass before
// left the last-level cache full of results yet to be written, and 81 where one did, a fill
// of 0.5 GB as well as the optimizer's step; 4.3 M take 5.1.
template <class G>
__global__ __launch_bounds__(256) void square_kernel(const Table tab, double* part) {
  __shared__ double join[4];
  const int k = find(tab, blockIdx.x);
  const G* g = static_cast<const G*>(tab.t[k].grad);
  const int64_t begin = (blockIdx.x - tab.first[k]) * kChunk, count = tab.t[k].count;
  constexpr int TURNS = kChunk / (256 * kItems);
  float d[TURNS][kItems];   // the whole chunk is on its way at once
#pragma unroll
  for (int j = 0; j < TURNS; ++j) {
    const int64_t at = begin + ((int64_t)j * 256 + threadIdx.x) * kItems;
    load_vec<G, kItems>(d[j], g + at, count - at);
  }
  double acc = 0.0;
#pragma unroll
  for (int j = 0; j < TURNS; ++j)
#pragma unroll
    for (int i = 0; i < kItems; ++i) acc += (double)d[j][i] * (double)d[j][i];
#pragma unroll
  for (int k = 1; k < 64; k *= 2) acc += __shfl_xor(acc, k, 64);
  if (threadIdx.x % 64 == 0) join[threadIdx.x / 64] = acc;
  __syncthreads();
  if (threadIdx.x == 0) part[blockIdx.x] = (join[0] + join[1]) + (join[2] + join[3]);
}

__global__ __launch_bounds__(1024) void clip_kernel(const double* part, int64_t parts,
                                                    float max_norm, float* out) {
  __shared__ double join[1024];
  double acc = 0.0;
  for (int64_t i = threadIdx.x; i < parts; i += 1024) acc += part[i];
  join[threadIdx.x] = acc;
  __syncthreads();
  for (int d = 512; d > 0; d /= 2) {
    if ((int)threadIdx.x < d) join[threadIdx.x] += join[threadIdx.x + d];
    __syncthreads();
  }
  if (threadIdx.x != 0) return;
  const float norm = (float)sqrt(join[0]);
  out[0] = norm;
  out[1] = isfinite(norm) ? fminf(1.0f, max_norm / (norm + 1e-6f)) : __builtin_nanf("");
}

struct Step {
  void* m;
  void* v;
  float* m_scale;
  float* v_scale;
  const float* clip;
  float beta1, beta2, rest1, rest2;   // rest: 1 - beta
  float keep;                         // 1 - lr weight_decay
  float rate;                         // lr / (1 - beta1^step)
  float root;                         // 1 / sqrt(1 - beta2^step)
  float eps;
  int copy_f16;
};

constexpr float kCodeMost = 448.0f;          // the largest e4m3 number
constexpr float kCodeLeast = 0.001953125f;   // the least above zero, 2^-9

// Eight e4m3 codes of a thread: the hardware's conversions, to nearest even.  Finite
// values are within +-448 by the block's scale, up to its rounding, far below the 464
// that would no longer round to 448.
__device__ __forceinline__ uint2 to_codes(const float (&x)[kItems]) {
  int lo = 0, hi = 0;
  lo = __builtin_amdgcn_cvt_pk_fp8_f32(x[0], x[1], lo, false);
  lo = __builtin_amdgcn_cvt_pk_fp8_f32(x[2], x[3], lo, true);
  hi = __builtin_amdgcn_cvt_pk_fp8_f32(x[4], x[5], hi, false);
  hi = __builtin_amdgcn_cvt_pk_fp8_f32(x[6], x[7], hi, true);
  return make_uint2((unsigned)lo, (unsigned)hi);
}

__device__ __forceinline__ void from_codes(float (&x)[kItems], uint2 c) {
  x[0] = __builtin_amdgcn_cvt_f32_fp8((int)c.x, 0);
  x[1] = __builtin_amdgcn_cvt_f32_fp8((int)c.x, 1);
  x[2] = __builtin_amdgcn_cvt_f32_fp8((int)c.x, 2);
  x[3] = __builtin_amdgcn_cvt_f32_fp8((int)c.x, 3);
  x[4] = __builtin_amdgcn_cvt_f32_fp8((int)c.y, 0);
  x[5] = __builtin_amdgcn_cvt_f32_fp8((int)c.y, 1);
  x[6] = __builtin_amdgcn_cvt_f32_fp8((int)c.y, 2);
  x[7] = __builtin_amdgcn_cvt_f32_fp8((int)c.y, 3);
}

// A block's largest magnitude: over the lanes that hold it.
__device__ __forceinline__ float block_scale(const float (&x)[kItems]) {
  float most = 0.0f;
#pragma unroll
  for (int i = 0; i < kItems; ++i) most = fmaxf(most, fabsf(x[i]));
#pragma unroll
  for (int d = 1; d < kBlockLanes; d *= 2) most = fmaxf(most, __shfl_xor(most, d, 64));
  return fmaxf(most * (1.0f / kCodeMost), 0x1p-126f);
}

__device__ __forceinline__ void store_codes(uint8_t* p, uint2 c, int64_t n) {
  if (n >= kItems) {
    *reinterpret_cast<uint2*>(p) = c;   // a block starts at a multiple of 256 bytes
  } else {
#pragma unroll
    for (int i = 0; i < kItems; ++i)
      if (i < n) p[i] = (uint8_t)((i < 4 ? c.x : c.y) >> (8 * (i % 4)));
  }
}

// Bound by memory: with 8-bit states, fp32 weights, a bf16 gradient and copy 16 bytes a
// parameter, 127 M of which take 374 to 380 us (5.4 TB/s); with 32-bit states 28 bytes, 4.3 M of
// which take 23 (5.2 TB/s, partly from the last-level cache).
template <class P, class G, int BITS>
__global__ __launch_bounds__(256) void adamw_kernel(const Table tab, const Step s) {
  const int k = find(tab, blockIdx.x);
  const gts_tensor& t = tab.t[k];
  const int64_t begin = (blockIdx.x - tab.first[k]) * kChunk, count = t.count;
  const float clip = s.clip != nullptr ? s.clip[1] : 1.0f;
  const bool skip = clip != clip;
#pragma unroll 1
  for (int j = 0; j < kChunk / (256 * kItems); ++j) {
    const int64_t at = begin + ((int64_t)j * 256 + threadIdx.x) * kItems, left = count - at;
    // whole waves end here; a block's lanes past the end stay with it, for its scale
    if (at - (int64_t)(threadIdx.x % 64) * kItems >= count) break;
    const int64_t st = t.state_offset + at;
    float p[kItems];
    load_vec<P, kItems>(p, static_cast<const P*>(t.param) + at, left);
    if (!skip) {
      float g[kItems], m[kItems], v[kItems];
      load_vec<G, kItems>(g, static_cast<const G*>(t.grad) + at, left);
      if constexpr (BITS == 32) {
        load_vec<float, kItems>(m, static_cast<const float*>(s.m) + st, left);
        load_vec<float, kItems>(v, static_cast<const float*>(s.v) + st, left);
      } else {
        uint2 cm = make_uint2(0, 0), cv = make_uint2(0, 0);
        float sm = 0.0f, sv = 0.0f;
        if (left > 0) {   // the last block is there in whole
          cm = *reinterpret_cast<const uint2*>(static_cast<const uint8_t*>(s.m) + st);
          cv = *reinterpret_cast<const uint2*>(static_cast<const uint8_t*>(s.v) + st);
          sm = s.m_scale[st / GTS_STATE_BLOCK];
          sv = s.v_scale[st / GTS_STATE_BLOCK];
        }
        from_codes(m, cm);
        from_codes(v, cv);
#pragma unroll
        for (int i = 0; i < kItems; ++i) {
          m[i] = i < left ? m[i] * sm : 0.0f;
          v[i] = i < left ? v[i] * sv : 0.0f;
          v[i] *= v[i];
        }
      }
#pragma unroll
      for (int i = 0; i < kItems; ++i) {
        const float gi = g[i] * clip;
        m[i] = s.beta1 * m[i] + s.rest1 * gi;
        v[i] = s.beta2 * v[i] + s.rest2 * (gi * gi);
        const float r = sqrtf(v[i]);
        // rcp is within an ulp: 1e-7 of a step, not of a parameter
        p[i] = p[i] * s.keep - s.rate * m[i] * __builtin_amdgcn_rcpf(r * s.root + s.eps);
        if constexpr (BITS == 8) v[i] = r;
      }
      if constexpr (BITS == 32) {
        store_vec<float, kItems>(static_cast<float*>(s.m) + st, m, left);
        store_vec<float, kItems>(static_cast<float*>(s.v) + st, v, left);
      } else {
        const float sm = block_scale(m), sv = block_scale(v);
        if (left > 0 && threadIdx.x % kBlockLanes == 0) {
          s.m_scale[st / GTS_STATE_BLOCK] = sm;
          s.v_scale[st / GTS_STATE_BLOCK] = sv;
        }
        const float im = 1.0f / sm, iv = 1.0f / sv;
#pragma unroll
        for (int i = 0; i < kItems; ++i) {
          m[i] *= im;
          v[i] = v[i] > 0.0f ? fmaxf(v[i] * iv, kCodeLeast) : v[i] * iv;
        }
        store_codes(static_cast<uint8_t*>(s.m) + st, to_codes(m), left);
        store_codes(static_cast<uint8_t*>(s.v) + st, to_codes(v), left);
      }
      store_vec<P, kItems>(static_cast<P*>(t.param) + at, p, left);
    }
    if (t.copy != nullptr) {
      if (s.copy_f16)
        store_vec<f16, kItems>(static_cast<f16*>(t.copy) + at, p, left);
      else
        store_vec<bf16, kItems>(static_cast<bf16*>(t.copy) + at, p, left);
    }
  }
}

// Calls run(table, chunks) for each launch's tensors.  Tensors without elements are
// left out.
template <class F>
hipError_t for_tables(const gts_tensor* tensors, int64_t n, F&& run) {
  Table tab;
  tab.n = 0;
  tab.first[0] = 0;
  for (int64_t i = 0; i < n; ++i) {
    const int64_t chunks = ceil_div(tensors[i].count, kChunk);
    // a launch's work-items stay below 2^32
    if (tab.n == kTensors || (tab.n > 0 && tab.first[tab.n] + chunks > kMostChunks)) {
      const hipError_t e = run(tab, tab.first[tab.n]);
      if (e != hipSuccess) return e;
      tab.n = 0;
    }
    if (chunks == 0) continue;
    tab.t[tab.n] = tensors[i];
    tab.first[tab.n + 1] = tab.first[tab.n] + chunks;
    ++tab.n;
  }
  return tab.n > 0 ? run(tab, tab.first[tab.n]) : hipSuccess;
}

gts_status check_tensors(const gts_tensor* t, int64_t n, int64_t grad_size) {
  if (n < 0) return fail(GTS_EINVAL, "num_tensors must be >= 0");
  if (n > 0 && t == nullptr) return fail(GTS_EINVAL, "tensors must not be NULL");
  for (int64_t i = 0; i < n; ++i) {
    if (t[i].count < 0 || t[i].count > kChunk * kMostChunks)
      return fail(GTS_EINVAL, "tensor %lld: count %lld is not possible", (long long)i, (long long)t[i].count);
    if (t[i].count > 0 && (t[i].grad == nullptr || misaligned(t[i].grad, grad_size)))
      return fail(GTS_EINVAL, "tensor %lld: grad is NULL or misaligned", (long long)i);
  }
  return GTS_OK;
}

int64_t all_chunks(const gts_tensor* t, int64_t n) {
  int64_t c = 0;
  for (int64_t i = 0; i < n; ++i) c += ceil_div(t[i].count, kChunk);
  return c;
}

// The chunks' sums.
int64_t clip_bytes(int64_t chunks) { return ceil_div(chunks * (int64_t)sizeof(double), 16) * 16; }

}  // namespace
}  // namespace nn
}  // namespace gts

extern "C" gts_status gts_grad_clip_workspace_bytes(const gts_tensor* tensors, int64_t num_tensors,
                                                    int64_t* bytes) {
  using namespace gts;
  clear_error();
  if (bytes == nullptr) return fail(GTS_EINVAL, "bytes must not be NULL");
  if (num_tensors < 0 || (num_tensors > 0 && tensors == nullptr))
    return fail(GTS_EINVAL, "tensors must not be NULL, num_tensors not negative");
  for (int64_t i = 0; i < num_tensors; ++i)
    if (tensors[i].count < 0) return fail(GTS_EINVAL, "tensor %lld: negative count", (long long)i);
  *bytes = nn::clip_bytes(nn::all_chunks(tensors, num_tensors));
  return GTS_OK;
}

extern "C" gts_status gts_grad_clip(const gts_tensor* tensors, int64_t num_tensors,
                                    int32_t grad_dtype, float max_norm, float* d_out,
                                    void* d_workspace, int64_t workspace_bytes, void* stream) {
  using namespace gts;
  using namespace gts::nn;
  clear_error();
  if (!known_type(grad_dtype))
    return fail(GTS_EINVAL, "dtype %d is not GTS_F32, GTS_BF16 or GTS_F16", grad_dtype);
  gts_status st = check_tensors(tensors, num_tensors, type_size(grad_dtype));
  if (st != GTS_OK) return st;
  if (d_out == nullptr || misaligned(d_out, 4)) return fail(GTS_EINVAL, "d_out is NULL or misaligned");
  if (!(max_norm > 0.0f)) return fail(GTS_EINVAL, "max_norm must be above 0");
  const int64_t chunks = all_chunks(tensors, num_tensors);
  if ((st = check_workspace(d_workspace, workspace_bytes, clip_bytes(chunks))) != GTS_OK) return st;
  hipStream_t s = static_cast<hipStream_t>(stream);
  double* part = static_cast<double*>(d_workspace);
  hipError_t e = for_tables(tensors, num_tensors, [&](const Table& tab, int64_t n) {
    with_type(grad_dtype, [&](auto g) {
      square_kernel<decltype(g)><<<(unsigned)n, 256, 0, s>>>(tab, part);
    });
    part += n;
    return hipGetLastError();
  });
  if (e == hipSuccess) {
    clip_kernel<<<1, 1024, 0, s>>>(static_cast<const double*>(d_workspace), chunks, max_norm, d_out);
    e = hipGetLastError();
  }
  return e == hipSuccess ? GTS_OK : fail(GTS_EDEVICE, "clip launch failed: %s", hipGetErrorString(e));
}

extern "C" gts_status gts_adamw(const gts_adamw_args* a, void* stream) {
  using namespace gts;
  using namespace gts::nn;
  clear_error();
  if (a == nullptr) return fail(GTS_EINVAL, "args must not be NULL");
  if (!known_type(a->param_dtype) || !known_type(a->grad_dtype))
    return fail(GTS_EINVAL, "param_dtype or grad_dtype is not GTS_F32, GTS_BF16 or GTS_F16");
  if (a->state_bits != 8 && a->state_bits != 32) return fail(GTS_EINVAL, "state_bits must be 8 or 32");
  gts_status st = check_tensors(a->tensors, a->num_tensors, type_size(a->grad_dtype));
  if (st != GTS_OK) return st;
  int64_t elements = 0;
  for (int64_t i = 0; i < a->num_tensors; ++i) {
    const gts_tensor& t = a->tensors[i];
    if (t.count == 0) continue;
    elements += t.count;
    if (t.param == nullptr || misaligned(t.param, type_size(a->param_dtype)))
      return fail(GTS_EINVAL, "tensor %lld: param is NULL or misaligned", (long long)i);
    if (t.copy != nullptr && (misaligned(t.copy, 2) || (a->copy_dtype != GTS_BF16 && a->copy_dtype != GTS_F16)))
      return fail(GTS_EINVAL, "tensor %lld: a copy must be aligned and of GTS_BF16 or GTS_F16", (long long)i);
    if (t.state_offset < 0 || t.state_offset % GTS_STATE_BLOCK != 0)
      return fail(GTS_EINVAL, "tensor %lld: state_offset must be a multiple of %d", (long long)i, GTS_STATE_BLOCK);
  }
  if (elements > 0) {
    const int64_t align = a->state_bits == 8 ? 8 : 4;
    if (a->m == nullptr || a->v == nullptr || misaligned(a->m, align) || misaligned(a->v, align))
      return fail(GTS_EINVAL, "m or v is NULL or misaligned");
    if (a->state_bits == 8 && (a->m_scale == nullptr || a->v_scale == nullptr ||
                               misaligned(a->m_scale, 4) || misaligned(a->v_scale, 4)))
      return fail(GTS_EINVAL, "m_scale or v_scale is NULL or misaligned");
    if (misaligned(a->d_clip, 4)) return fail(GTS_EINVAL, "d_clip is misaligned");
  }
  if (a->step < 1) return fail(GTS_EINVAL, "step must be >= 1");
  if (!(a->beta1 >= 0 && a->beta1 < 1 && a->beta2 >= 0 && a->beta2 < 1))
    return fail(GTS_EINVAL, "beta1 and beta2 must be in [0, 1)");
  if (!(a->eps >= 0)) return fail(GTS_EINVAL, "eps must be >= 0");
  Step s;
  s.m = a->m;
  s.v = a->v;
  s.m_scale = a->m_scale;
  s.v_scale = a->v_scale;
  s.clip = a->d_clip;
  s.beta1 = (float)a->beta1;
  s.beta2 = (float)a->beta2;
  s.rest1 = (float)(1.0 - a->beta1);
  s.rest2 = (float)(1.0 - a->beta2);
  s.keep = (float)(1.0 - a->lr * a->weight_decay);
  s.rate = (float)(a->lr / (1.0 - std::pow(a->beta1, (double)a->step)));
  s.root = (float)(1.0 / std::sqrt(1.0 - std::pow(a->beta2, (double)a->step)));
  s.eps = (float)a->eps;
  s.copy_f16 = a->copy_dtype == GTS_F16;
  hipStream_t q = static_cast<hipStream_t>(stream);
  const hipError_t e = for_tables(a->tensors, a->num_tensors, [&](const Table& tab, int64_t n) {
    with_type(a->param_dtype, [&](auto p) {
      with_type(a->grad_dtype, [&](auto g) {
        using P = decltype(p);
        using G = decltype(g);
        if (a->state_bits == 8)
          adamw_kernel<P, G, 8><<<(unsigned)n, 256, 0, q>>>(tab, s);
        else
          adamw_kernel<P, G, 32><<<(unsigned)n, 256, 0, q>>>(tab, s);
      });
    });
    return hipGetLastError();
  });
  return e == hipSuccess ? GTS_OK : fail(GTS_EDEVICE, "adamw launch failed: %s", hipGetErrorString(e));
}
