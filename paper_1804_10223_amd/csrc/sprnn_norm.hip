// Root-mean-square norm of rows after the addition of a residual stream, with its output in the stream's type or in e4m3
// with a scale per 128 elements, and its backward pass.
//
//   r = x + residual,   rs = 1 / sqrt(mean r^2 + eps),   y = r rs w
//   dr = rs (dy w - n mean(dy w n)) + d_residual  with n = r rs,   dw = sum over rows of dy n
//
// Bound by bytes: a row is read once, kept in registers while its sum is formed, and written once.  A workgroup takes one
// row at a time, eight consecutive elements a lane and pass, with as many wavefronts as one pass needs (rows of up to 8192;
// wider ones take two passes), so that no lane is idle in any but the last wavefront and a block of 128 elements is
// a DPP row of 16 lanes.  It loads its next row before it sums the present one; 16 wavefronts a compute unit then keep enough
// bytes in flight, and later workgroups would only begin with nothing in flight.  Rows wider than 16384, and two-pass rows that
// are not whole (below), are read twice.  Measured, bfloat16 with a float32 residual stream: 8192 x 2304 to e4m3 35 us
// (5.9 TB/s; 108 -> 82 us where nothing is in a cache when the loads waited in front of the sums), backward 4096 x 2560
// 30 us (4.9 TB/s).
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
template <bool WHOLE = false, typename E>
__device__ __forceinline__ void store_row(E* row, int at, int width, const Pack<E, kV>& p) {
  if (WHOLE || at + kV <= width) store_pack(row + at, p);
  else store_part(row + at, p, width - at);
}

// Eight elements of the row at `row`, zeros behind its end and of a row that is not there (`there`; a tensor that is not there
// has no address).  WHOLE: rows are 16-byte aligned and a multiple of eight elements long; they are read through a buffer, whose
// own check of the range takes the branches' place.  A branch around a load ends with a wait for it: with branches nothing is
// in flight while a row is worked on.
template <bool WHOLE, typename E>
__device__ __forceinline__ Pack<E, kV> fetch_row(const E* row, int at, int width, bool there) {
  if constexpr (WHOLE) {
    const uint64_t base = reinterpret_cast<uint64_t>(row);
    const uint64_t lo = (uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)base), hi = (uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)(base >> 32));
    const auto buffer = __builtin_amdgcn_make_buffer_rsrc(reinterpret_cast<void*>(lo | hi << 32), 0, there ? width * (int)sizeof(E) : 0, 0x00020000);
    typedef uint32_t words __attribute__((ext_vector_type(4)));
    words v[sizeof(E) / 2];
#pragma unroll
    for (int i = 0; i < (int)sizeof(E) / 2; ++i) v[i] = __builtin_amdgcn_raw_buffer_load_b128(buffer, at * (int)sizeof(E) + 16 * i, 0, 0);
    Pack<E, kV> p;
    __builtin_memcpy(&p, v, sizeof(p));
    return p;
  } else {
    if (!there || at >= width) return Pack<E, kV>{};
    return load_row(row, at, width);
  }
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

// ... of two numbers.
__device__ __forceinline__ float2 sum_workgroup(float2 v, float2* slots) {
  const int waves = blockDim.x >> 6;
  v.x = sum_lanes<64>(v.x);
  v.y = sum_lanes<64>(v.y);
  if (waves == 1) return v;
  if ((threadIdx.x & 63) == 0) slots[threadIdx.x >> 6] = v;
  __syncthreads();
  float2 total = slots[0];
  for (int w = 1; w < waves; ++w) { total.x += slots[w].x; total.y += slots[w].y; }
  return total;
}

// A lane's weights; 1 without any.
__device__ __forceinline__ void load_weight(const float* weight, int at, int width, float (&w)[kV]) {
#pragma unroll
  for (int i = 0; i < kV; ++i) w[i] = 1.0f;
  if (weight && at < width) widen(load_row(weight, at, width), w);
}

// The rows of a workgroup: every gridDim.x-th, found without a division after the first.
struct RowCursor {
  uint32_t row, rows, batch, t, b, by_t, by_b;
  __device__ __forceinline__ RowCursor(uint32_t rows, uint32_t batch)
      : row(blockIdx.x), rows(rows), batch(batch), t(row / batch), b(row - t * batch), by_t(gridDim.x / batch), by_b(gridDim.x - by_t * batch) {}
  __device__ __forceinline__ bool there() const { return row < rows; }
  __device__ __forceinline__ void forth() {
    row += gridDim.x;
    t += by_t;
    b += by_b;
    if (b >= batch) { b -= batch; ++t; }
  }
};

struct NormArgs {
  uint32_t rows;
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

template <int TYPE, int RTYPE, int P, bool E4M3, bool WHOLE>
__global__ __launch_bounds__(1024) void norm_kernel(NormArgs a, View<const Element<TYPE>> x, View<const Element<RTYPE>> res,
                                                    View<Element<RTYPE>> res_out, View<uint8_t> y8, View<Element<TYPE>> y) {
  typedef Element<TYPE> E;
  typedef Element<RTYPE> R;
  __shared__ float slots[2][kMaxWaves];
  const int threads = blockDim.x, first = threadIdx.x * kV, stride = threads * kV;
  const int blocks = (a.width + 127) >> 7;
  float w[P][kV];
#pragma unroll
  for (int p = 0; p < P; ++p) load_weight(a.weight, first + p * stride, a.width, w[p]);
  struct Fetched {
    Pack<E, kV> x[P];
    Pack<R, kV> res[P];
  };
  auto fetch = [&](Fetched& to, const RowCursor& from) {
#pragma unroll
    for (int p = 0; p < P; ++p) {
      const int at = first + p * stride;
      to.x[p] = fetch_row<WHOLE>(x.row(from.t, from.b), at, a.width, from.there());
      to.res[p] = fetch_row<WHOLE>(res.row(from.t, from.b), at, a.width, from.there() && res.data);
    }
  };
  RowCursor now(a.rows, a.batch);
  auto work = [&](const Fetched& own, Fetched& next, int turn) {
    float r[P][kV], sum = 0.0f;
#pragma unroll
    for (int p = 0; p < P; ++p) {
      const int at = first + p * stride;
      float f[kV];
      widen(own.x[p], r[p]);
      widen(own.res[p], f);
#pragma unroll
      for (int i = 0; i < kV; ++i) r[p][i] += f[i];
      const Pack<R, kV> kept = narrow<R>(r[p]);      // the stream that goes on is what is normed
      if (res_out.data && at < a.width) store_row<WHOLE>(res_out.row(now.t, now.b), at, a.width, kept);
      if (RTYPE != SPRNN_TYPE_F32) widen(kept, r[p]);
#pragma unroll
      for (int i = 0; i < kV; ++i) sum += r[p][i] * r[p][i];
    }
    RowCursor ahead = now;
    ahead.forth();
    fetch(next, ahead);
    const float scale = 1.0f / sqrtf(sum_workgroup(sum, slots[turn]) * a.inv_width + a.eps);
#pragma unroll
    for (int p = 0; p < P; ++p) {
      const int at = first + p * stride;
      if (!E4M3 && at >= a.width) continue;
#pragma unroll
      for (int i = 0; i < kV; ++i) r[p][i] = r[p][i] * scale * w[p][i];
      if (E4M3) store_e4m3(r[p], y8.row(now.t, now.b), at, a.width, a.scales + (int64_t)now.row * blocks);
      else store_row<WHOLE>(y.row(now.t, now.b), at, a.width, narrow<E>(r[p]));
    }
    now = ahead;
  };
  Fetched one, two;                                  // in turn: a copy of what is in flight would wait for it
  fetch(one, now);
  while (now.there()) {
    work(one, two, 0);
    if (!now.there()) break;
    work(two, one, 1);
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
template <int TYPE, int RTYPE, bool WHOLE>
__global__ __launch_bounds__(1024) void norm_backward_kernel(NormArgs a, View<const Element<TYPE>> dy, View<const Element<RTYPE>> r,
                                                             View<const Element<RTYPE>> d_res, View<Element<RTYPE>> dr,
                                                             float* partial) {
  typedef Element<TYPE> E;
  typedef Element<RTYPE> R;
  __shared__ float2 slots[2][kMaxWaves];
  const int first = threadIdx.x * kV;
  float* const mine = partial ? partial + (int64_t)blockIdx.x * a.width : nullptr;
  float w[kV], dw[kV] = {};
  load_weight(a.weight, first, a.width, w);
  struct Fetched {
    Pack<R, kV> r, d;
    Pack<E, kV> g;
  };
  auto fetch = [&](Fetched& to, const RowCursor& from) {
    to.r = fetch_row<WHOLE>(r.row(from.t, from.b), first, a.width, from.there());
    to.g = fetch_row<WHOLE>(dy.row(from.t, from.b), first, a.width, from.there());
    to.d = fetch_row<WHOLE>(d_res.row(from.t, from.b), first, a.width, from.there() && d_res.data);
  };
  RowCursor now(a.rows, a.batch);
  auto work = [&](const Fetched& own, Fetched& next, int turn) {
    float f[kV], g[kV], o[kV], square = 0.0f, dot = 0.0f;
    widen(own.r, f);
    widen(own.g, g);
#pragma unroll
    for (int i = 0; i < kV; ++i) { square += f[i] * f[i]; dot += f[i] * (g[i] * w[i]); }
    RowCursor ahead = now;
    ahead.forth();
    fetch(next, ahead);
    const float2 sums = sum_workgroup(make_float2(square, dot), slots[turn]);
    const float rs = 1.0f / sqrtf(sums.x * a.inv_width + a.eps);
    const float along = sums.y * a.inv_width * rs * rs;   // mean(dy w n) rs: n = f rs takes one more
    widen(own.d, o);
#pragma unroll
    for (int i = 0; i < kV; ++i) {
      dw[i] += g[i] * (f[i] * rs);
      o[i] += rs * (g[i] * w[i] - f[i] * along);
    }
    if (first < a.width) store_row<WHOLE>(dr.row(now.t, now.b), first, a.width, narrow<R>(o));
    now = ahead;
  };
  Fetched one, two;                                  // in turn: a copy of what is in flight would wait for it
  fetch(one, now);
  while (now.there()) {
    work(one, two, 0);
    if (!now.there()) break;
    work(two, one, 1);
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
  __shared__ float2 slots[2][kMaxWaves];
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
    const float2 sums = sum_workgroup(make_float2(square, dot), slots[turn]);
    const float rs = 1.0f / sqrtf(sums.x * a.inv_width + a.eps);
    const float along = sums.y * a.inv_width * rs * rs;
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
// Every row of the view is 16-byte aligned and a whole number of lanes' elements.
bool whole_rows(const sprnn_seq_t& s, int type, int width) {
  const int64_t per_16 = 16 / type_bytes(type);
  return width % kV == 0 && aligned_to(s.data, 16) && s.step % per_16 == 0 && s.sample % per_16 == 0;
}
// Workgroups of the backward pass: ten wavefronts a compute unit keep the memory busy; more only leave more partial sums
// of the weight's gradient (4096 x 2560 as above, 16 wavefronts 35.5 us, 10 30.0; 16384 x 1024 53 and 50).
int backward_groups(int64_t rows, int width) {
  const int waves = shape_of(width).waves;
  const int64_t most = (int64_t)256 * (waves < 10 ? 10 / waves : 1);
  return (int)(rows < most ? rows : most);
}

template <int TYPE, int RTYPE, bool E4M3>
hipError_t run_norm(const NormArgs& a, const sprnn_seq_t& x, const sprnn_seq_t& res, const sprnn_seq_t& res_out,
                    const sprnn_seq_t& y, hipStream_t stream) {
  const Shape s = shape_of(a.width);
  const int64_t most = (int64_t)256 * (s.waves < 16 ? 16 / s.waves : 1);
  const dim3 grid((unsigned)((int64_t)a.rows < most ? a.rows : most)), block((unsigned)s.waves * 64);
  const bool whole = whole_rows(x, TYPE, a.width) && (!res.data || whole_rows(res, RTYPE, a.width));
  auto kernel = s.passes == 1 ? whole ? norm_kernel<TYPE, RTYPE, 1, E4M3, true> : norm_kernel<TYPE, RTYPE, 1, E4M3, false>
              : s.passes == 2 && whole ? norm_kernel<TYPE, RTYPE, 2, E4M3, true> : norm_wide_kernel<TYPE, RTYPE, E4M3>;
  return launch(kernel, grid, block, 0, stream, a, view<const Element<TYPE>>(x), view<const Element<RTYPE>>(res),
                view<Element<RTYPE>>(res_out), view<uint8_t>(y), view<Element<TYPE>>(y));
}

template <int TYPE, int RTYPE>
hipError_t run_backward(const NormArgs& a, const sprnn_seq_t& dy, const sprnn_seq_t& r, const sprnn_seq_t& d_res,
                        const sprnn_seq_t& dr, float* d_weight, float* partial, hipStream_t stream) {
  const Shape s = shape_of(a.width);
  const int groups = backward_groups((int64_t)a.rows, a.width);
  if (groups > 0) {
    const bool whole = whole_rows(dy, TYPE, a.width) && whole_rows(r, RTYPE, a.width) && (!d_res.data || whole_rows(d_res, RTYPE, a.width));
    auto kernel = s.passes == 1 ? whole ? norm_backward_kernel<TYPE, RTYPE, true> : norm_backward_kernel<TYPE, RTYPE, false>
                                : s.passes == 2 ? norm_backward_wide_kernel<TYPE, RTYPE, 2>
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
  return NormArgs{(uint32_t)((int64_t)n->steps * n->batch), n->batch, n->width, n->eps, 1.0f / (float)n->width, n->weight, scales};
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
