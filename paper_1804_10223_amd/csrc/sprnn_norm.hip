// Root-mean-square norm of rows after the addition of a residual stream, with its output in the stream's type or in e4m3
// with a scale per 128 elements, and its backward pass.
//
//   r = x + residual,   rs = 1 / sqrt(mean r^2 + eps),   y = r rs w
//   dr = rs (dy w - n mean(dy w n)) + d_residual  with n = r rs,   dw = sum over rows of dy n
//
// Bound by bytes: a row is read once, kept in registers while its sum is formed, and written once.  A workgroup takes one
// row at a time, eight consecutive elements a lane and pass, with as many wavefronts as one pass needs (rows of up to 8192;
// wider ones take two passes), so that no lane is idle in any but the last wavefront and a block of 128 elements is
// a DPP row of 16 lanes.  It fetches its next row before it sums the present one.  Rows wider than 16384 are read twice.
#include "sprnn_sums.h"

namespace sprnn {
namespace {

constexpr int kV = 8;                  // elements of a lane in one pass
constexpr int kMaxWaves = 16;
constexpr float kLargestE4m3 = 448.0f;
constexpr float kSmallestAmax = 0x1p-100f;

template <typename E>
__device__ __forceinline__ void widen(const Pack<E, kV>& p, float (&f)[kV]) {
#pragma unroll
  for (int i = 0; i < kV; ++i) f[i] = (float)p.v[i];
}
template <typename E>
__device__ __forceinline__ Pack<E, kV> narrow(const float (&f)[kV]) {
  Pack<E, kV> p;
#pragma unroll
  for (int i = 0; i < kV; ++i) p.v[i] = (E)f[i];
  return p;
}
template <typename E>
__device__ __forceinline__ Pack<E, kV> load_row(const E* row, int at, int width) {
  if (at + kV <= width) return load_pack<kV>(row + at);
  return load_part<kV>(row + at, width - at);
}
template <typename E>
__device__ __forceinline__ void store_row(E* row, int at, int width, const Pack<E, kV>& p) {
  if (at + kV <= width) store_pack(row + at, p);
  else store_part(row + at, p, width - at);
}

// Sum over the workgroup; `slots` alternates between calls, so that one barrier a call is enough.
__device__ __forceinline__ float sum_workgroup(float v, float* slots) {
  const int waves = blockDim.x >> 6;
  v = sum_lanes<64>(v);
  if (waves == 1) return v;
  if ((threadIdx.x & 63) == 0) slots[threadIdx.x >> 6] = v;
  __syncthreads();
  float total = slots[0];
  for (int w = 1; w < waves; ++w) total += slots[w];
  return total;
}

struct NormArgs {
  int64_t rows;
  int batch, width;
  float eps, inv_width;
  const float* weight;
  float* scales;
};

// The 8 elements of a lane as e4m3 with the scale of its block of 128 (16 lanes).
__device__ __forceinline__ void store_e4m3(const float (&y)[kV], uint8_t* row, int at, int width, float* scale_at) {
  uint32_t top = 0;
#pragma unroll
  for (int i = 0; i < kV; ++i) top = max(top, __builtin_bit_cast(uint32_t, y[i]) & 0x7fffffffu);   // as numbers, infinity, NaN in this order
  top = max_lanes16(top);
  const float amax = __builtin_bit_cast(float, max(top, __builtin_bit_cast(uint32_t, kSmallestAmax)));
  const float scale = amax / kLargestE4m3, inverse = 1.0f / scale;
  if (at >= width) return;
  Pack<uint32_t, 2> q;
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    int packed = __builtin_amdgcn_cvt_pk_fp8_f32(y[4 * i] * inverse, y[4 * i + 1] * inverse, 0, false);
    packed = __builtin_amdgcn_cvt_pk_fp8_f32(y[4 * i + 2] * inverse, y[4 * i + 3] * inverse, packed, true);
    q.v[i] = (uint32_t)packed;
  }
  if (at + kV <= width) __builtin_memcpy(row + at, &q, sizeof(q));
  else {
#pragma unroll
    for (int i = 0; i < kV; ++i)
      if (at + i < width) row[at + i] = (uint8_t)(q.v[i >> 2] >> (8 * (i & 3)));
  }
  if ((threadIdx.x & 15) == 0) scale_at[at >> 7] = scale;
}

template <int TYPE, int RTYPE, int P, bool E4M3>
__global__ __launch_bounds__(1024) void norm_kernel(NormArgs a, View<const Element<TYPE>> x, View<const Element<RTYPE>> res,
                                                    View<Element<RTYPE>> res_out, View<uint8_t> y8, View<Element<TYPE>> y) {
  typedef Element<TYPE> E;
  typedef Element<RTYPE> R;
  __shared__ float slots[2][kMaxWaves];
  const int threads = blockDim.x, first = threadIdx.x * kV, stride = threads * kV;
  const int blocks = (a.width + 127) >> 7;
  float w[P][kV];
#pragma unroll
  for (int p = 0; p < P; ++p) {
    const int at = first + p * stride;
#pragma unroll
    for (int i = 0; i < kV; ++i) w[p][i] = a.weight && at + i < a.width ? a.weight[at + i] : 1.0f;
  }
  Pack<E, kV> xs[P];
  Pack<R, kV> rs[P];
  auto fetch = [&](int64_t row) {
    const int64_t t = row / a.batch, b = row - t * a.batch;
#pragma unroll
    for (int p = 0; p < P; ++p) {
      const int at = first + p * stride;
      if (at < a.width) {
        xs[p] = load_row(x.row(t, b), at, a.width);
        if (res.data) rs[p] = load_row(res.row(t, b), at, a.width);
      }
    }
  };
  int64_t row = blockIdx.x;
  if (row < a.rows) fetch(row);
  for (int turn = 0; row < a.rows; row += gridDim.x, turn ^= 1) {
    const int64_t t = row / a.batch, b = row - t * a.batch;
    float r[P][kV], sum = 0.0f;
#pragma unroll
    for (int p = 0; p < P; ++p) {
      const int at = first + p * stride;
#pragma unroll
      for (int i = 0; i < kV; ++i) r[p][i] = 0.0f;
      if (at >= a.width) continue;
      widen(xs[p], r[p]);
      if (res.data) {
        float f[kV];
        widen(rs[p], f);
#pragma unroll
        for (int i = 0; i < kV; ++i) r[p][i] += f[i];
      }
      const Pack<R, kV> kept = narrow<R>(r[p]);      // the stream that goes on is what is normed
      if (res_out.data) store_row(res_out.row(t, b), at, a.width, kept);
      if (RTYPE != SPRNN_TYPE_F32 && res.data) widen(kept, r[p]);
#pragma unroll
      for (int i = 0; i < kV; ++i) sum += r[p][i] * r[p][i];
    }
    if (row + gridDim.x < a.rows) fetch(row + gridDim.x);
    const float scale = 1.0f / sqrtf(sum_workgroup(sum, slots[turn]) * a.inv_width + a.eps);
#pragma unroll
    for (int p = 0; p < P; ++p) {
      const int at = first + p * stride;
      if (!E4M3 && at >= a.width) continue;
#pragma unroll
      for (int i = 0; i < kV; ++i) r[p][i] = r[p][i] * scale * w[p][i];
      if (E4M3) store_e4m3(r[p], y8.row(t, b), at, a.width, a.scales + row * blocks);
      else store_row(y.row(t, b), at, a.width, narrow<E>(r[p]));
    }
  }
}

// Rows wider than a workgroup's registers: summed in one pass, read again in a second.
template <int TYPE, int RTYPE, bool E4M3>
__global__ __launch_bounds__(1024) void norm_wide_kernel(NormArgs a, View<const Element<TYPE>> x, View<const Element<RTYPE>> res,
                                                         View<Element<RTYPE>> res_out, View<uint8_t> y8, View<Element<TYPE>> y) {
  typedef Element<TYPE> E;
  typedef Element<RTYPE> R;
  __shared__ float slots[2][kMaxWaves];
  const int stride = blockDim.x * kV;
  const int blocks = (a.width + 127) >> 7;
  int turn = 0;
  for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x, turn ^= 1) {
    const int64_t t = row / a.batch, b = row - t * a.batch;
    auto stream = [&](int at, float (&r)[kV]) {      // the row's elements as they are normed
      widen(load_row(x.row(t, b), at, a.width), r);
      Pack<R, kV> kept;
      if (res.data) {
        float f[kV];
        widen(load_row(res.row(t, b), at, a.width), f);
#pragma unroll
        for (int i = 0; i < kV; ++i) r[i] += f[i];
        kept = narrow<R>(r);
        widen(kept, r);
      } else {
        kept = narrow<R>(r);
      }
      return kept;
    };
    float sum = 0.0f;
    for (int at = threadIdx.x * kV; at < a.width; at += stride) {
      float r[kV];
      stream(at, r);
#pragma unroll
      for (int i = 0; i < kV; ++i) sum += r[i] * r[i];
    }
    const float scale = 1.0f / sqrtf(sum_workgroup(sum, slots[turn]) * a.inv_width + a.eps);
    for (int base = 0; base < a.width; base += stride) {
      const int at = base + threadIdx.x * kV;
      float r[kV] = {};
      if (at < a.width) {
        const Pack<R, kV> kept = stream(at, r);
        if (res_out.data) store_row(res_out.row(t, b), at, a.width, kept);
#pragma unroll
        for (int i = 0; i < kV; ++i) r[i] = r[i] * scale * (a.weight && at + i < a.width ? a.weight[at + i] : 1.0f);
      }
      if (E4M3) store_e4m3(r, y8.row(t, b), at, a.width, a.scales + row * blocks);
      else if (at < a.width) store_row(y.row(t, b), at, a.width, narrow<E>(r));
    }
  }
}

// Backward pass of rows that fit a workgroup's registers; the weight's gradient is summed over a workgroup's rows in
// registers and left in `partial` [workgroup][width].
template <int TYPE, int RTYPE>
__global__ __launch_bounds__(1024) void norm_backward_kernel(NormArgs a, View<const Element<TYPE>> dy, View<const Element<RTYPE>> r,
                                                             View<const Element<RTYPE>> d_res, View<Element<RTYPE>> dr,
                                                             float* partial) {
  typedef Element<TYPE> E;
  typedef Element<RTYPE> R;
  __shared__ float slots[2][2][kMaxWaves];
  const int first = threadIdx.x * kV;
  auto weight = [&](int at, int i) { return a.weight && at + i < a.width ? a.weight[at + i] : 1.0f; };
  float* const mine = partial ? partial + (int64_t)blockIdx.x * a.width : nullptr;
  float w[kV], dw[kV];
#pragma unroll
  for (int i = 0; i < kV; ++i) { w[i] = weight(first, i); dw[i] = 0.0f; }
  Pack<R, kV> rs_, ds;
  Pack<E, kV> gs;
  auto fetch = [&](int64_t row) {
    const int64_t t = row / a.batch, b = row - t * a.batch;
    if (first < a.width) {
      rs_ = load_row(r.row(t, b), first, a.width);
      gs = load_row(dy.row(t, b), first, a.width);
      if (d_res.data) ds = load_row(d_res.row(t, b), first, a.width);
    }
  };
  int64_t row = blockIdx.x;
  if (row < a.rows) fetch(row);
  for (int turn = 0; row < a.rows; row += gridDim.x, turn ^= 1) {
    const int64_t t = row / a.batch, b = row - t * a.batch;
    float f[kV] = {}, g[kV] = {}, o[kV] = {}, square = 0.0f, dot = 0.0f;
    if (first < a.width) {
      widen(rs_, f);
      widen(gs, g);
      if (d_res.data) widen(ds, o);
#pragma unroll
      for (int i = 0; i < kV; ++i) { square += f[i] * f[i]; dot += f[i] * (g[i] * w[i]); }
    }
    if (row + gridDim.x < a.rows) fetch(row + gridDim.x);
    const float rs = 1.0f / sqrtf(sum_workgroup(square, slots[turn][0]) * a.inv_width + a.eps);
    const float along = sum_workgroup(dot, slots[turn][1]) * a.inv_width * rs * rs;   // mean(dy w n) rs: n = f rs takes one more
    if (first >= a.width) continue;
#pragma unroll
    for (int i = 0; i < kV; ++i) {
      dw[i] += g[i] * (f[i] * rs);
      o[i] += rs * (g[i] * w[i] - f[i] * along);
    }
    store_row(dr.row(t, b), first, a.width, narrow<R>(o));
  }
  if (mine && first < a.width) {
    Pack<float, kV> out;
#pragma unroll
    for (int i = 0; i < kV; ++i) out.v[i] = dw[i];
    store_row(mine, first, a.width, out);
  }
}

// ... of wider rows: read twice, P passes of a workgroup each time (0: as many as it takes).  The weight's gradient stays in
// registers where P says how many there are, and is otherwise summed in memory by the one lane that owns the element.
template <int TYPE, int RTYPE, int P>
__global__ __launch_bounds__(1024) void norm_backward_wide_kernel(NormArgs a, View<const Element<TYPE>> dy,
                                                                  View<const Element<RTYPE>> r, View<const Element<RTYPE>> d_res,
                                                                  View<Element<RTYPE>> dr, float* partial) {
  typedef Element<RTYPE> R;
  __shared__ float slots[2][2][kMaxWaves];
  const int first = threadIdx.x * kV, stride = blockDim.x * kV;
  auto weight = [&](int at, int i) { return a.weight && at + i < a.width ? a.weight[at + i] : 1.0f; };
  float* const mine = partial ? partial + (int64_t)blockIdx.x * a.width : nullptr;
  const int passes = P ? P : (a.width + stride - 1) / stride;
  constexpr int kKept = P ? P : 1;
  float dw[kKept][kV];
#pragma unroll
  for (int p = 0; p < kKept; ++p)
#pragma unroll
    for (int i = 0; i < kV; ++i) dw[p][i] = 0.0f;
  int turn = 0;
  bool begun = false;
  for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x, turn ^= 1) {
    const int64_t t = row / a.batch, b = row - t * a.batch;
    float square = 0.0f, dot = 0.0f;
    auto sum = [&](int at) {
      float f[kV], g[kV];
      widen(load_row(r.row(t, b), at, a.width), f);
      widen(load_row(dy.row(t, b), at, a.width), g);
#pragma unroll
      for (int i = 0; i < kV; ++i) { square += f[i] * f[i]; dot += f[i] * (g[i] * weight(at, i)); }
    };
#pragma unroll kKept
    for (int p = 0; p < passes; ++p)
      if (first + p * stride < a.width) sum(first + p * stride);
    const float rs = 1.0f / sqrtf(sum_workgroup(square, slots[turn][0]) * a.inv_width + a.eps);
    const float along = sum_workgroup(dot, slots[turn][1]) * a.inv_width * rs * rs;
    auto finish = [&](int at, float (&d)[kV], bool in_memory) {
      float f[kV], g[kV], o[kV] = {};
      widen(load_row(r.row(t, b), at, a.width), f);
      widen(load_row(dy.row(t, b), at, a.width), g);
      if (d_res.data) widen(load_row(d_res.row(t, b), at, a.width), o);
#pragma unroll
      for (int i = 0; i < kV; ++i) {
        const float term = g[i] * (f[i] * rs);
        if (!in_memory) d[i] += term;
        else if (mine && at + i < a.width) mine[at + i] = (begun ? mine[at + i] : 0.0f) + term;
        o[i] += rs * (g[i] * weight(at, i) - f[i] * along);
      }
      store_row(dr.row(t, b), at, a.width, narrow<R>(o));
    };
#pragma unroll kKept
    for (int p = 0; p < passes; ++p)
      if (first + p * stride < a.width) finish(first + p * stride, dw[P ? p : 0], P == 0);
    begun = true;
  }
  if (P && mine) {
#pragma unroll
    for (int p = 0; p < P; ++p) {
      const int at = first + p * stride;
      Pack<float, kV> out;
#pragma unroll
      for (int i = 0; i < kV; ++i) out.v[i] = dw[p][i];
      if (at < a.width) store_row(mine, at, a.width, out);
    }
  }
}

struct PutWeight {
  float* out;
  __device__ void operator()(int64_t i, float sum) const { out[i] = sum; }
};

struct Shape {
  int waves, passes;   // passes 0: the row does not fit in registers
};
Shape shape_of(int width) {
  const int once = 64 * kV;
  for (int passes = 1; passes <= 2; ++passes) {
    const int waves = (width + once * passes - 1) / (once * passes);
    if (waves <= kMaxWaves) return {waves, passes};
  }
  return {kMaxWaves, 0};
}
// Workgroups of the backward pass: enough wavefronts to keep the memory busy, few enough that the partial sums are small
// beside the rows.
int backward_groups(int64_t rows, int width) {
  const int waves = shape_of(width).waves;
  const int64_t most = waves <= 2 ? 2048 : waves <= 4 ? 1024 : 512;
  return (int)(rows < most ? rows : most);
}

template <int TYPE, int RTYPE, bool E4M3>
hipError_t run_norm(const NormArgs& a, const sprnn_seq_t& x, const sprnn_seq_t& res, const sprnn_seq_t& res_out,
                    const sprnn_seq_t& y, hipStream_t stream) {
  const Shape s = shape_of(a.width);
  const int64_t most = (int64_t)256 * (s.waves <= 2 ? 16 : s.waves <= 8 ? 6 : 2);
  const dim3 grid((unsigned)(a.rows < most ? a.rows : most)), block((unsigned)s.waves * 64);
  auto kernel = s.passes == 1 ? norm_kernel<TYPE, RTYPE, 1, E4M3> : s.passes == 2 ? norm_kernel<TYPE, RTYPE, 2, E4M3>
              : norm_wide_kernel<TYPE, RTYPE, E4M3>;
  return launch(kernel, grid, block, 0, stream, a, view<const Element<TYPE>>(x), view<const Element<RTYPE>>(res),
                view<Element<RTYPE>>(res_out), view<uint8_t>(y), view<Element<TYPE>>(y));
}

template <int TYPE, int RTYPE>
hipError_t run_backward(const NormArgs& a, const sprnn_seq_t& dy, const sprnn_seq_t& r, const sprnn_seq_t& d_res,
                        const sprnn_seq_t& dr, float* d_weight, float* partial, hipStream_t stream) {
  const Shape s = shape_of(a.width);
  const int groups = backward_groups(a.rows, a.width);
  if (groups > 0) {
    auto kernel = s.passes == 1 ? norm_backward_kernel<TYPE, RTYPE> : s.passes == 2 ? norm_backward_wide_kernel<TYPE, RTYPE, 2>
                                : norm_backward_wide_kernel<TYPE, RTYPE, 0>;
    const hipError_t e = launch(kernel, dim3((unsigned)groups), dim3((unsigned)s.waves * 64), 0, stream, a, view<const Element<TYPE>>(dy),
                                view<const Element<RTYPE>>(r), view<const Element<RTYPE>>(d_res), view<Element<RTYPE>>(dr),
                                d_weight ? partial : nullptr);
    if (e != hipSuccess) return e;
  }
  if (!d_weight) return hipSuccess;
  return launch_sum_partials(partial, groups, (int64_t)a.width, PutWeight{d_weight}, stream);
}

bool good_norm(const sprnn_norm_t* n) {
  return n && good_sizes(n->steps, n->batch, n->width) && activation_type(n->type) &&
         (n->residual_type == n->type || n->residual_type == SPRNN_TYPE_F32) && n->eps >= 0.0f && aligned_to(n->weight, 4);
}
NormArgs arguments(const sprnn_norm_t* n, float* scales) {
  return NormArgs{(int64_t)n->steps * n->batch, n->batch, n->width, n->eps, 1.0f / (float)n->width, n->weight, scales};
}

}  // namespace

}  // namespace sprnn

using namespace sprnn;

extern "C" {

int sprnn_rms_norm(int device_id, const sprnn_norm_t* norm, sprnn_seq_t x, sprnn_seq_t residual, sprnn_seq_t residual_out,
                   int y_type, sprnn_seq_t y, float* scales, void* stream) {
  if (device_id < 0 || !good_norm(norm)) return SPRNN_ERR_INVALID;
  const int T = norm->steps, B = norm->batch, W = norm->width, type = norm->type, rtype = norm->residual_type;
  const bool quantized = y_type == SPRNN_TYPE_E4M3;
  if (!quantized && y_type != type) return SPRNN_ERR_INVALID;
  if (T == 0 || B == 0) return SPRNN_OK;
  if (!good_view(x, type) || (residual.data && !good_view(residual, rtype)) ||
      (residual_out.data && !good_output(residual_out, rtype, T, B, W)) || !good_output(y, y_type, T, B, W))
    return SPRNN_ERR_INVALID;
  if (quantized ? !scales || !aligned_to(scales, 4) : scales != nullptr) return SPRNN_ERR_INVALID;
  DeviceGuard guard(device_id);
  if (!guard.ok) return SPRNN_ERR_HIP;
  const NormArgs a = arguments(norm, scales);
  const hipStream_t s = static_cast<hipStream_t>(stream);
  hipError_t e = hipErrorInvalidValue;
#define CASE(TYPE, RTYPE)                                                                         \
  if (type == TYPE && rtype == RTYPE)                                                             \
    e = quantized ? run_norm<TYPE, RTYPE, true>(a, x, residual, residual_out, y, s)               \
                  : run_norm<TYPE, RTYPE, false>(a, x, residual, residual_out, y, s);
  CASE(SPRNN_TYPE_F32, SPRNN_TYPE_F32)
  CASE(SPRNN_TYPE_F16, SPRNN_TYPE_F16)
  CASE(SPRNN_TYPE_F16, SPRNN_TYPE_F32)
  CASE(SPRNN_TYPE_BF16, SPRNN_TYPE_BF16)
  CASE(SPRNN_TYPE_BF16, SPRNN_TYPE_F32)
#undef CASE
  return SPRNN_HIP(e) ? SPRNN_OK : SPRNN_ERR_HIP;
}

int sprnn_rms_norm_sizes(const sprnn_norm_t* norm, int64_t* backward_workspace) {
  if (!norm || !good_sizes(norm->steps, norm->batch, norm->width)) return SPRNN_ERR_INVALID;
  if (backward_workspace) *backward_workspace = (int64_t)backward_groups((int64_t)norm->steps * norm->batch, norm->width) * norm->width * 4;
  return SPRNN_OK;
}

int sprnn_rms_norm_backward(int device_id, const sprnn_norm_t* norm, sprnn_seq_t dy, sprnn_seq_t r, sprnn_seq_t d_residual,
                            sprnn_seq_t dr, float* d_weight, void* workspace, int64_t workspace_bytes, void* stream) {
  if (device_id < 0 || !good_norm(norm) || !aligned_to(d_weight, 4)) return SPRNN_ERR_INVALID;
  const int T = norm->steps, B = norm->batch, W = norm->width, type = norm->type, rtype = norm->residual_type;
  int64_t need = 0;
  (void)sprnn_rms_norm_sizes(norm, &need);
  if (d_weight && need > 0 && (!workspace || !aligned_to(workspace, 16) || workspace_bytes < need)) return SPRNN_ERR_INVALID;
  if (T > 0 && B > 0 &&
      (!good_view(dy, type) || !good_view(r, rtype) || (d_residual.data && !good_view(d_residual, rtype)) || !good_output(dr, rtype, T, B, W)))
    return SPRNN_ERR_INVALID;
  if ((T == 0 || B == 0) && !d_weight) return SPRNN_OK;
  DeviceGuard guard(device_id);
  if (!guard.ok) return SPRNN_ERR_HIP;
  const NormArgs a = arguments(norm, nullptr);
  const hipStream_t s = static_cast<hipStream_t>(stream);
  float* const partial = static_cast<float*>(workspace);
  hipError_t e = hipErrorInvalidValue;
#define CASE(TYPE, RTYPE) \
  if (type == TYPE && rtype == RTYPE) e = run_backward<TYPE, RTYPE>(a, dy, r, d_residual, dr, d_weight, partial, s);
  CASE(SPRNN_TYPE_F32, SPRNN_TYPE_F32)
  CASE(SPRNN_TYPE_F16, SPRNN_TYPE_F16)
  CASE(SPRNN_TYPE_F16, SPRNN_TYPE_F32)
  CASE(SPRNN_TYPE_BF16, SPRNN_TYPE_BF16)
  CASE(SPRNN_TYPE_BF16, SPRNN_TYPE_F32)
#undef CASE
  return SPRNN_HIP(e) ? SPRNN_OK : SPRNN_ERR_HIP;
}

}  // extern "C"
