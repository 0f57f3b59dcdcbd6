// gts_linear and gts_linear_backward: matrix products with their epilogues.
#include <algorithm>

#include "gts_linear_kernel.h"

namespace gts {
namespace nn {
namespace {

// Whether an operand can be copied to LDS 16 bytes a lane: rows that start at multiples
// of 16 bytes, and a tile's offsets within 31 bits.
bool lies(const void* p, int64_t ld, int64_t size) {
  return !misaligned(p, 16) && ld * size % 16 == 0 && ld * size < (int64_t)1 << 22;
}

int64_t padded(int64_t width, int64_t size) { return ceil_div(width * size, 16) * 16 / size; }

constexpr int kUnits = 256;   // compute units of an MI355X
constexpr int kTileM[6] = {256, 192, 128, 64, 64, 128}, kTileN[6] = {256, 256, 128, 64, 32, 128};   // by shape

// The shape, splits and copies of a product of m x n x k.  copied: bytes of the operands
// that do not lie as they have to; below 0 where a copy would not lie either.
//
// Times are in microseconds, fitted to measurements of all shapes on an MI355X: a slice
// (128 bytes of k) takes a compute unit in 16 bits 1.5 for a tile of 256 x 256, 1.15 of
// 192 x 256; of 128 x 128 by two groups of waves 0.6, by one 0.46 where two tiles share the
// unit and 0.8 alone; of 64 x 64 0.19 and 0.36; in 32 bits, where the matrix cores are a
// sixteenth as fast and larger tiles gain nothing, 0.55 of 64 x 64 and 0.29 of 64 x 32;
// the smaller tiles up to a sixth more where operands are transposed on the way; 1.0 on
// operands fetched through registers.  A tile takes 6, 6.5, 2.4, 2, 0.7, 0.7 and 0.5 besides.
// `broken` operands (0 to 2) have rows that do not start at lines of 128 bytes, so that a
// slice's piece of a row lies in two: 64 x 64 tiles in 16 bits then take up to half as much
// again (dw of 3714 x 2552 x 816 62 us, 39 in tiles of 128 x 128), the larger ones, which
// read a row for more columns, little.
// Splits pay for writing and joining their sums: a launch and the traffic.  Up to 32 rows,
// W passes once through registers: 1024 to 4096 in bf16 takes 16 rows 3.9 and 32 rows 4.9 in a
// graph, and 5.8 in tiles, as 33 rows do.  (The same with 64 rows, which is not built, took
// 7.3 against 6.0.)
ProductPlan plan_product(int64_t m, int64_t n, int64_t k, int64_t size, Layout layout, int64_t copied,
                         int broken) {
  struct Cost {
    int shape;
    double slice, alone, tile;   // alone: where a unit has one tile only
    double order[3];             // factors of the slices, by layout
  };
  static const Cost kCosts[2][5] = {{{kLarge, 1.5, 1.5, 6.0, {1, 1, 1}},
                                     {kLower, 1.15, 1.15, 6.5, {1, 1, 1}},
                                     {kMiddle, 0.6, 0.6, 2.4, {1, 1.04, 1.06}},
                                     {kMany, 0.46, 0.8, 2.0, {1, 1.05, 1.05}},
                                     {kSmall, 0.19, 0.36, 0.7, {1, 1, 1.08}}},
                                    {{kSmall, 0.55, 0.55, 0.7, {1, 1.08, 1.16}},
                                     {kNarrow, 0.29, 0.29, 0.5, {1, 1.08, 1.16}}}};
  const int64_t depth = kSliceBytes / size, slices = std::max<int64_t>(1, ceil_div(k, depth));
  if (layout == kForward && m <= 32) return {kFewRows, false, false, 1, slices * depth, 0};
  ProductPlan best{};
  double least = -1;
  auto consider = [&](const Cost& c, bool direct) {
    const int64_t tiles = ceil_div(m, kTileM[c.shape]) * ceil_div(n, kTileN[c.shape]);
    for (int64_t splits = 1; splits <= 32 && (splits == 1 || slices / splits >= 4); splits *= 2) {
      const int64_t chunk = ceil_div(slices, splits), used = ceil_div(slices, chunk);
      const int64_t each = ceil_div(tiles * used, kUnits);
      const double lines = size == 2 && c.shape == kSmall ? 1 + 0.25 * broken : 1.0;
      const double slice = direct ? c.order[layout] * lines * (each == 1 ? c.alone : c.slice) : 1.0;
      double t = (double)each * (slice * (double)chunk + c.tile);
      if (direct && copied > 0) t += 3 + (double)copied / 2.5e6;
      if (used > 1) t += 4 + (double)m * (double)n * (double)(8 * used + size) / 5e6;
      if (least < 0 || t < least) {
        least = t;
        best = {c.shape, direct, direct && copied > 0, (int)used, chunk * depth, used > 1 ? used * m * n * 4 : 0};
      }
    }
  };
  for (const Cost& c : kCosts[size == 4]) {
    if (c.slice == 0) break;
    // the large tiles' loop takes one slice at least
    if (copied >= 0 && (k > 0 || c.shape > kLower)) consider(c, true);
    if (copied != 0 && c.shape == kSmall) consider(c, false);
  }
  return best;
}

hipError_t launch_product(const ProductArgs& p, Layout layout, const ProductPlan& plan,
                          const AlignArgs (&align)[2], hipStream_t s, int32_t dtype) {
  if (dtype == GTS_F32) return launch_product_f32(p, layout, plan, align, s);
  if (dtype == GTS_BF16) return launch_product_bf16(p, layout, plan, align, s);
  return launch_product_f16(p, layout, plan, align, s);
}

// How a product runs: its plan, the operands that are copied first and where.
struct Product {
  ProductPlan plan;
  AlignArgs align[2];
  int64_t bytes;   // of workspace: the copies, then the splits' sums
};

// a_padded: A's rows end in zeros up to a multiple of 16 bytes.
// broken: as for plan_product, or below 0 to take it from the operands' rows.
Product make_product(const ProductArgs& p, Layout layout, bool a_padded, int64_t size, int broken = -1) {
  // A is k-contiguous but for dW; B in the forward pass only
  const bool whole = p.k * size % 16 == 0;
  const bool ok[2] = {lies(p.a, p.lda, size) && (layout == kGradW || whole || a_padded),
                      lies(p.b, p.ldb, size) && (layout != kForward || whole)};
  const int64_t rows[2] = {layout == kGradW ? p.k : p.m, layout == kForward ? p.n : p.k};
  const int64_t width[2] = {layout == kGradW ? p.m : p.k, layout == kForward ? p.k : p.n};
  Product r{};
  int64_t bytes[2] = {}, copied = 0;
  for (int i = 0; i < 2; ++i)
    if (!ok[i]) {
      bytes[i] = rows[i] * padded(width[i], size) * size;
      copied = copied < 0 || padded(width[i], size) * size >= (int64_t)1 << 22 ? -1 : copied + bytes[i];
    }
  // a copy's rows are as wide as the operand's, up to a multiple of 16 bytes
  const int64_t ld[2] = {ok[0] ? p.lda : padded(width[0], size), ok[1] ? p.ldb : padded(width[1], size)};
  if (broken < 0) broken = (ld[0] * size % 128 != 0) + (ld[1] * size % 128 != 0);
  r.plan = plan_product(p.m, p.n, p.k, size, layout, copied, broken);
  for (int i = 0; i < 2; ++i)
    if (!ok[i] && r.plan.align) {
      r.align[i] = {i == 0 ? p.a : p.b, i == 0 ? p.lda : p.ldb, rows[i], width[i],
                    reinterpret_cast<void*>(r.bytes), padded(width[i], size)};
      r.bytes += ceil_div(bytes[i], 16) * 16;
    }
  r.bytes += r.plan.part_bytes;
  return r;
}

// Sets what a product's plan and workspace say about it.
void place(ProductArgs& p, Product& r, char* ws, int32_t dtype) {
  for (AlignArgs& a : r.align)
    if (a.rows > 0) a.dst = ws + reinterpret_cast<intptr_t>(a.dst);
  p.splits = r.plan.splits;
  p.k_chunk = r.plan.k_chunk;
  // a C larger than the L2s (32 MB), in whole lines of 128 bytes, does not pass through
  // them, so that the operands stay there: 8192^3 in bf16 794 against 828 us.  In parts of
  // lines it costs: 10000 x 2048 x 7848 297 against 283.
  const int64_t size = type_size(dtype);
  p.past_l2 = p.m * p.n * size >= (int64_t)32 << 20 && !misaligned(p.c, 128) && p.ld_c * size % 128 == 0;
  p.part = p.splits > 1 ? reinterpret_cast<float*>(ws + r.bytes - r.plan.part_bytes) : nullptr;
}

// Runs the product that `p` describes (its splits and tiles are set here).
hipError_t run_product(ProductArgs p, Product r, Layout layout, char* ws, int32_t dtype,
                       hipStream_t s) {
  place(p, r, ws, dtype);
  return launch_product(p, layout, r.plan, r.align, s, dtype);
}

// Whether both gradients' products run in one launch: in small tiles (in 32 bits in the
// narrower, if they differ), up to 4 a compute unit.  4096 x 512 x 2048 in bf16 38 against
// 47 us with the bias' sums, 256 x 512 x 512 7.7 against 13; more tiles fill the device by
// themselves (2500 x 784 x 1000 in fp32 106 against 102).
bool make_pair(const ProductArgs& px, Product& x, const ProductArgs& pw, Product& w) {
  const auto small = [](const Product& r) {
    return r.plan.direct && (r.plan.shape == kSmall || r.plan.shape == kNarrow);
  };
  if (!small(x) || !small(w)) return false;
  const int shape = x.plan.shape == w.plan.shape ? x.plan.shape : kNarrow;
  const auto tiles = [&](const ProductArgs& p, const Product& r) {
    return ceil_div(p.m, kTileM[shape]) * ceil_div(p.n, kTileN[shape]) * r.plan.splits;
  };
  if (tiles(px, x) + tiles(pw, w) > 4 * kUnits) return false;
  x.plan.shape = w.plan.shape = shape;
  return true;
}

hipError_t run_pair(ProductArgs x, Product rx, char* ws_x, ProductArgs w, Product rw, char* ws_w,
                    const ColumnSums& sums, int32_t dtype, hipStream_t s) {
  place(x, rx, ws_x, dtype);
  place(w, rw, ws_w, dtype);
  const auto launch = dtype == GTS_F32 ? launch_pair_f32 : dtype == GTS_BF16 ? launch_pair_bf16 : launch_pair_f16;
  return launch(x, w, rx.plan.shape, rx.align[1], rw.align[1], sums, s);
}

// A product of these extents whose operands A and B lie or not.
Product product_of(int64_t m, int64_t n, int64_t k, Layout layout, int64_t size, bool off_a, bool off_b,
                   bool a_padded, int broken = -1) {
  ProductArgs p{};
  p.m = m;
  p.n = n;
  p.k = k;
  p.a = reinterpret_cast<void*>((uintptr_t)(off_a ? size : 16));
  p.b = reinterpret_cast<void*>((uintptr_t)(off_b ? size : 16));
  p.lda = padded(layout == kGradW ? m : k, size);
  p.ldb = padded(layout == kForward ? k : n, size);
  return make_product(p, layout, a_padded, size, broken);
}

// The workspace of a product of these extents, of operands that lie as they have to or,
// if not `aligned`, of any.
int64_t product_bytes(int64_t m, int64_t n, int64_t k, Layout layout, int64_t size, bool aligned) {
  // whichever operands are copied and whatever their row strides, the copies and the splits
  // are no more than the most of these
  int64_t most = 0;
  for (int which = 0; which < (aligned ? 2 : 8); ++which)
    for (int broken = 0; broken <= 2; ++broken)
      most = std::max(most, product_of(m, n, k, layout, size, (which & 2) != 0, (which & 4) != 0, (which & 1) != 0,
                                       broken).bytes);
  return ceil_div(most, 16) * 16;
}

// dz = dy act'(z), and the column sums of dz over one chunk of rows into
// sums[chunk][n].  LPR lanes take a row, each kVec consecutive columns; a wave's 64 / LPR
// rows and the workgroup's 4 waves walk the chunk together and their sums are joined at
// its end.  dz or sums may be null; rows of dz are ld_dz apart, a multiple of kVec, and
// end in zeros.  Bound by memory: 10000 x 4096 in bf16 with GELU 50 us under a profiler
// (246 MB, 4.9 TB/s).
//
// In 16 bits dz is rounded to the type, since the matrix cores take no more: the gradients of
// 10000 x 1024 x 4096 in bf16 are 2.3e-3 off 64 bits, where their own rounding alone makes
// 1.7e-3.  What the rounding leaves could go in as a second operand, but would take both
// products once more, some 200 us beside the 253 of the call.  The sums are of dz unrounded.
template <class T, int LPR>
__global__ __launch_bounds__(256) void dz_kernel(const T* dy, int64_t ld_dy, const T* pre,
                                                 int64_t ld_pre, int64_t rows, int64_t n,
                                                 int64_t chunk, int act, T* dz, int64_t ld_dz, float* sums) {
  constexpr int V = kVec<T>, RPW = 64 / LPR;
  __shared__ float part[4][64 * V];
  const int lane = threadIdx.x % 64, wave = threadIdx.x / 64;
  const int64_t col = ((int64_t)blockIdx.x * LPR + lane % LPR) * V, left = n - col;
  const int64_t end = min(rows, ((int64_t)blockIdx.y + 1) * chunk);
  float acc[V] = {};
  if (left > 0)
    for (int64_t r = blockIdx.y * chunk + wave * RPW + lane / LPR; r < end; r += 4 * RPW) {
      float d[V];
      load_vec<T, V>(d, dy + r * ld_dy + col, left);
      if (act != GTS_ACT_NONE) {
        float z[V];
        load_vec<T, V>(z, pre + r * ld_pre + col, left);
        with_act(act, [&](auto a) {
#pragma unroll
          for (int i = 0; i < V; ++i) d[i] *= act_slope<decltype(a)::value>(z[i]);
        });
      }
      if (dz) store_vec<T, V>(dz + r * ld_dz + col, d, V);
#pragma unroll
      for (int i = 0; i < V; ++i) acc[i] += d[i];
    }
  if (sums == nullptr) return;
#pragma unroll
  for (int i = 0; i < V; ++i) {
#pragma unroll
    for (int d = LPR; d < 64; d *= 2) acc[i] += __shfl_xor(acc[i], d, 64);
    part[wave][lane * V + i] = acc[i];
  }
  __syncthreads();
  for (int c = threadIdx.x; c < LPR * V; c += 256) {
    const int64_t at = (int64_t)blockIdx.x * LPR * V + c;
    if (at < n) sums[blockIdx.y * n + at] = (part[0][c] + part[1][c]) + (part[2][c] + part[3][c]);
  }
}

// out[c] = the sum over the chunks of sums[chunk][c].
template <class T>
__global__ __launch_bounds__(1024) void column_sum_kernel(const float* sums, int64_t chunks,
                                                          int64_t n, T* out) {
  const int64_t c = group_of_grid() * kSumColumns + threadIdx.x % kSumColumns;
  const float sum = column_sum<1024>(sums, chunks, n, c);
  if (threadIdx.x < kSumColumns && c < n) out[c] = (T)sum;
}

struct DzPlan {
  int lpr;             // lanes a row
  int64_t spans;       // workgroups across the columns
  int64_t chunk, chunks;
};

DzPlan plan_dz(int64_t rows, int64_t n, int64_t elem) {
  DzPlan d;
  const int64_t vec = 16 / elem;
  d.lpr = 1;
  while (d.lpr < 64 && d.lpr * vec < n) d.lpr *= 2;
  d.spans = ceil_div(n, d.lpr * vec);
  const int64_t step = 4 * (64 / d.lpr);   // rows a workgroup takes at once
  // about 1024 workgroups, at least 4 steps each
  d.chunk = step * std::max<int64_t>(4, ceil_div(rows * d.spans, 1024 * step));
  d.chunks = ceil_div(rows, d.chunk);
  return d;
}

template <class T>
hipError_t launch_dz(const gts_linear_grad_args& a, const DzPlan& d, T* dz, int64_t ld_dz,
                     float* sums, hipStream_t s) {
  const dim3 grid((unsigned)d.spans, (unsigned)d.chunks);
  auto run = [&](auto lpr) {
    dz_kernel<T, decltype(lpr)::value><<<grid, 256, 0, s>>>(
        static_cast<const T*>(a.dy), a.ld_dy, static_cast<const T*>(a.pre), a.ld_pre, a.rows,
        a.outputs, d.chunk, a.act, dz, ld_dz, sums);
    return hipGetLastError();
  };
  switch (d.lpr) {
    case 1: return run(std::integral_constant<int, 1>{});
    case 2: return run(std::integral_constant<int, 2>{});
    case 4: return run(std::integral_constant<int, 4>{});
    case 8: return run(std::integral_constant<int, 8>{});
    case 16: return run(std::integral_constant<int, 16>{});
    case 32: return run(std::integral_constant<int, 32>{});
    default: return run(std::integral_constant<int, 64>{});
  }
}

gts_status check_extents(int64_t rows, int64_t inputs, int64_t outputs, int32_t dtype) {
  if (!known_type(dtype)) return fail(GTS_EINVAL, "dtype %d is not GTS_F32, GTS_BF16 or GTS_F16", dtype);
  if (rows < 0) return fail(GTS_EINVAL, "rows must be >= 0");
  if (inputs < 1 || outputs < 1) return fail(GTS_EINVAL, "inputs and outputs must be >= 1");
  if (rows > INT32_MAX || inputs > INT32_MAX || outputs > INT32_MAX)
    return fail(GTS_EINVAL, "rows, inputs and outputs must be below 2^31");
  return GTS_OK;
}

gts_status check_launch(hipError_t e) {
  return e == hipSuccess ? GTS_OK : fail(GTS_EDEVICE, "linear launch failed: %s", hipGetErrorString(e));
}

// The workspace of the backward pass: dz, its column sums by chunk, a product's own.
struct BackwardLayout {
  DzPlan dz;
  int64_t ld_dz;
  int64_t sums, product, bytes;
};

BackwardLayout dz_layout(int64_t rows, int64_t outputs, int64_t size) {
  BackwardLayout l;
  l.dz = plan_dz(rows, outputs, size);
  l.ld_dz = padded(outputs, size);
  l.sums = rows * l.ld_dz * size;
  l.bytes = l.product = l.sums + ceil_div(l.dz.chunks * outputs * 4, 16) * 16;
  return l;
}

BackwardLayout backward_layout(int64_t rows, int64_t inputs, int64_t outputs, int32_t dtype,
                               bool aligned) {
  const int64_t size = type_size(dtype);
  BackwardLayout l = dz_layout(rows, outputs, size);
  l.bytes = l.product + product_bytes(rows, inputs, outputs, kGradX, size, aligned) +
            product_bytes(outputs, inputs, rows, kGradW, size, aligned);
  return l;
}

}  // namespace
}  // namespace nn
}  // namespace gts

extern "C" gts_status gts_linear_workspace_bytes(int64_t rows, int64_t inputs, int64_t outputs,
                                                 int32_t dtype, int32_t aligned,
                                                 int64_t* bytes) {
  using namespace gts;
  clear_error();
  if (bytes == nullptr) return fail(GTS_EINVAL, "bytes must not be NULL");
  gts_status st = nn::check_extents(rows, inputs, outputs, dtype);
  if (st != GTS_OK) return st;
  *bytes = nn::product_bytes(rows, outputs, inputs, nn::kForward, nn::type_size(dtype), aligned != 0);
  return GTS_OK;
}

extern "C" gts_status gts_linear_config(int64_t rows, int64_t inputs, int64_t outputs, int32_t dtype,
                                        int32_t aligned, int32_t product, gts_linear_launch* out) {
  using namespace gts;
  using namespace gts::nn;
  clear_error();
  if (out == nullptr) return fail(GTS_EINVAL, "out must not be NULL");
  gts_status st = check_extents(rows, inputs, outputs, dtype);
  if (st != GTS_OK) return st;
  if (product < kForward || product > kGradW) return fail(GTS_EINVAL, "unknown product %d", product);
  const int64_t m = product == kGradW ? outputs : rows, n = product == kForward ? outputs : inputs;
  const int64_t k = product == kForward ? inputs : product == kGradX ? outputs : rows;
  // dz, A of the gradients, is made to lie, its rows padded, where dy does not
  const bool off = aligned == 0;
  const ProductPlan plan = product_of(m, n, k, (Layout)product, type_size(dtype), off && product == kForward, off,
                                      product == kGradX).plan;
  const bool few = plan.shape == kFewRows;
  *out = {few ? (m <= 16 ? 16 : 32) : kTileM[plan.shape], few ? 16 : kTileN[plan.shape], plan.splits, plan.align,
          plan.direct};
  return GTS_OK;
}

extern "C" gts_status gts_linear(const gts_linear_args* a, void* d_workspace,
                                 int64_t workspace_bytes, void* stream) {
  using namespace gts;
  using namespace gts::nn;
  clear_error();
  if (a == nullptr) return fail(GTS_EINVAL, "args must not be NULL");
  gts_status st = check_extents(a->rows, a->inputs, a->outputs, a->dtype);
  if (st != GTS_OK) return st;
  if (a->act < GTS_ACT_NONE || a->act > GTS_ACT_GELU) return fail(GTS_EINVAL, "unknown activation %d", a->act);
  const int64_t es = type_size(a->dtype);
  Matrix m[] = {{"x", a->x, a->ld_x, a->inputs, true},
                {"w", a->w, a->ld_w, a->inputs, true},
                {"bias", a->bias, a->outputs, a->outputs, false},
                {"residual", a->residual, a->ld_r, a->outputs, false},
                {"y", a->y, a->ld_y, a->outputs, true},
                {"pre", a->pre, a->ld_pre, a->outputs, false}};
  if ((st = check_matrices(m, 6, es, a->rows == 0)) != GTS_OK) return st;
  ProductArgs p{};
  p.a = a->x;
  p.lda = a->ld_x;
  p.b = a->w;
  p.ldb = a->ld_w;
  p.m = a->rows;
  p.n = a->outputs;
  p.k = a->inputs;
  p.act = a->act;
  p.bias = a->bias;
  p.residual = a->residual;
  p.ld_r = a->ld_r;
  p.c = a->y;
  p.ld_c = a->ld_y;
  p.pre = a->pre;
  p.ld_pre = a->ld_pre;
  const Product r = make_product(p, kForward, false, es);
  if ((st = check_workspace(d_workspace, workspace_bytes, r.bytes)) != GTS_OK) return st;
  if (a->rows == 0) return GTS_OK;
  return check_launch(run_product(p, r, kForward, static_cast<char*>(d_workspace), a->dtype,
                                  static_cast<hipStream_t>(stream)));
}

extern "C" gts_status gts_linear_backward_workspace_bytes(int64_t rows, int64_t inputs,
                                                          int64_t outputs, int32_t dtype,
                                                          int32_t aligned, int64_t* bytes) {
  using namespace gts;
  clear_error();
  if (bytes == nullptr) return fail(GTS_EINVAL, "bytes must not be NULL");
  gts_status st = nn::check_extents(rows, inputs, outputs, dtype);
  if (st != GTS_OK) return st;
  *bytes = nn::backward_layout(rows, inputs, outputs, dtype, aligned != 0).bytes;
  return GTS_OK;
}

extern "C" gts_status gts_linear_backward(const gts_linear_grad_args* a, void* d_workspace,
                                          int64_t workspace_bytes, void* stream) {
  using namespace gts;
  using namespace gts::nn;
  clear_error();
  if (a == nullptr) return fail(GTS_EINVAL, "args must not be NULL");
  gts_status st = check_extents(a->rows, a->inputs, a->outputs, a->dtype);
  if (st != GTS_OK) return st;
  if (a->act < GTS_ACT_NONE || a->act > GTS_ACT_GELU) return fail(GTS_EINVAL, "unknown activation %d", a->act);
  const int64_t es = type_size(a->dtype);
  Matrix m[] = {{"dy", a->dy, a->ld_dy, a->outputs, true},
                {"pre", a->act != GTS_ACT_NONE ? a->pre : nullptr, a->ld_pre, a->outputs, a->act != GTS_ACT_NONE},
                {"x", a->dw ? a->x : nullptr, a->ld_x, a->inputs, a->dw != nullptr},
                {"w", a->dx ? a->w : nullptr, a->ld_w, a->inputs, a->dx != nullptr},
                {"dx", a->dx, a->ld_dx, a->inputs, false},
                {"dw", a->dw, a->ld_dw, a->inputs, false},
                {"db", a->db, a->outputs, a->outputs, false}};
  if ((st = check_matrices(m, 7, es, a->rows == 0)) != GTS_OK) return st;
  BackwardLayout l = dz_layout(a->rows, a->outputs, es);
  // dz is made where there is an activation, and where dy's rows cannot be copied as they lie
  const bool products = a->dx != nullptr || a->dw != nullptr;
  const bool direct = lies(a->dy, a->ld_dy, es) && (a->dx == nullptr || a->outputs * es % 16 == 0);
  const bool make = products && (a->act != GTS_ACT_NONE || !direct);
  // the products read dz where it lies: a bad address is refused before it is planned with
  if (make && (st = check_workspace(d_workspace, workspace_bytes, l.product)) != GTS_OK) return st;
  ProductArgs px{}, pw{};
  px.a = make ? d_workspace : a->dy;
  px.lda = make ? l.ld_dz : a->ld_dy;
  px.b = a->w;
  px.ldb = a->ld_w;
  px.m = a->rows;
  px.n = a->inputs;
  px.k = a->outputs;
  px.c = a->dx;
  px.ld_c = a->ld_dx;
  pw.a = px.a;
  pw.lda = px.lda;
  pw.b = a->x;
  pw.ldb = a->ld_x;
  pw.m = a->outputs;
  pw.n = a->inputs;
  pw.k = a->rows;
  pw.c = a->dw;
  pw.ld_c = a->ld_dw;
  Product rx{}, rw{};
  if (a->dx) rx = make_product(px, kGradX, make, es);
  if (a->dw) rw = make_product(pw, kGradW, false, es);
  const int64_t second = l.product + ceil_div(rx.bytes, 16) * 16;
  l.bytes = second + rw.bytes;
  if ((st = check_workspace(d_workspace, workspace_bytes, l.bytes)) != GTS_OK) return st;
  hipStream_t s = static_cast<hipStream_t>(stream);
  return with_type(a->dtype, [&](auto t) {
    using T = decltype(t);
    char* ws = static_cast<char*>(d_workspace);
    float* sums = a->db ? reinterpret_cast<float*>(ws + l.sums) : nullptr;
    T* made = make ? reinterpret_cast<T*>(ws) : nullptr;
    hipError_t e = hipSuccess;
    if (a->rows > 0 && (made || sums)) e = launch_dz<T>(*a, l.dz, made, l.ld_dz, sums, s);
    if (e == hipSuccess && a->dx && a->dw && a->rows > 0 && make_pair(px, rx, pw, rw)) {
      e = run_pair(px, rx, ws + l.product, pw, rw, ws + second, {sums, l.dz.chunks, a->outputs, a->db}, a->dtype, s);
      return check_launch(e);
    }
    if (e == hipSuccess && a->db) {
      column_sum_kernel<T><<<grid_of(ceil_div(a->outputs, kSumColumns)), 1024, 0, s>>>(
          sums, l.dz.chunks, a->outputs, static_cast<T*>(a->db));
      e = hipGetLastError();
    }
    if (e == hipSuccess && a->dx && a->rows > 0) e = run_product(px, rx, kGradX, ws + l.product, a->dtype, s);
    if (e == hipSuccess && a->dw) e = run_product(pw, rw, kGradW, ws + second, a->dtype, s);
    return check_launch(e);
  });
}
