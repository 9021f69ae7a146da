// Causal depthwise convolution over a channel's last K inputs, with SiLU, and its backward pass.
//
//   p_t[c] = bias[c] + sum_k w[c][k] x_{t-K+1+k}[c],   y_t = p_t sigmoid(p_t)
//   g_t = dy_t y'(p_t),   dx_s = sum_k w[k] g_{s+K-1-k},   dw[k] = sum_t g_t x_{t-K+1+k},   dbias = sum_t g_t
//
// Bound by bytes: x is read and y written once.  A lane owns V neighbouring channels (8 bytes of them, at any alignment) and
// walks a stretch of time with the last K - 1 inputs in registers, four rows in flight while four are worked on.  8 x 2048 x
// 4608 in bfloat16: 61 us, 4.9 TB/s; with 16 bytes a lane three wavefronts a SIMD are left (101 us against 70 at the time), and
// eight rows fetched and then worked on took 95.  Backward 8 x 1024 x 2048: 32 us and 4 for the parameters' sums, 21 by its
// bytes: the vector units work on 35 numbers a step and channel (p again, the sigmoid, both gradients), and on K - 1 steps more
// for every stretch of 32 (stretches of 64, 40 us: half as many wavefronts).  The state of the K - 1 inputs before the call is
// read and written by the lanes of the first stretch alone: it may be updated in place.
#include "sprnn_sums.h"

namespace sprnn {
namespace {

constexpr int kWaves = 4;              // a workgroup: side by side in the forward pass, stretches of the backward pass
constexpr int kStretch = 32;           // steps of a stretch
constexpr int kStretchBack = 32;       // ... of the backward pass, which reads K - 1 steps more on both sides

struct ConvArgs {
  int T, B, C, silu;
  const float* weight;
  const float* bias;
  const int32_t* lengths;
};

// WHOLE: the channels are a multiple of V, so that no load stands under a branch, which would be waited for where it ends.
template <typename E, int V, bool WHOLE = false>
__device__ __forceinline__ Pack<E, V> load_channels(const E* row, int c, int C) {
  if (WHOLE || c + V <= C) return load_pack<V>(row + c);
  return load_part<V>(row + c, C - c);
}
template <typename E, int V, bool WHOLE = false>
__device__ __forceinline__ void store_channels(E* row, int c, int C, const float (&f)[V]) {
  Pack<E, V> p;
#pragma unroll
  for (int i = 0; i < V; ++i) p.v[i] = (E)f[i];
  if (WHOLE || c + V <= C) store_pack(row + c, p);
  else store_part(row + c, p, C - c);
}

// The parameters of a lane's channels.
template <int K, int V>
struct Filter {
  float w[K][V], bias[V];
  __device__ __forceinline__ void read(const ConvArgs& a, int c) {
#pragma unroll
    for (int i = 0; i < V; ++i) {
      const int own = min(c + i, a.C - 1);       // (no branch that a load would be waited for; a lane's channels behind C go nowhere)
      bias[i] = 0.0f;
#pragma unroll
      for (int k = 0; k < K; ++k) w[k][i] = a.weight[(int64_t)own * K + k];
    }
    if (a.bias) {
#pragma unroll
      for (int i = 0; i < V; ++i) bias[i] = a.bias[min(c + i, a.C - 1)];
    }
  }
};

// The K - 1 inputs before step t0, oldest first: from the state before step 0, zeros without one.
template <typename E, int K, int V>
__device__ __forceinline__ void read_history(float (&past)[K][V], const ConvArgs& a, View<const E> x, const E* state, int t0, int end,
                                             int b, int c) {
#pragma unroll
  for (int j = 0; j + 1 < K; ++j) {
    const int t = t0 - (K - 1) + j;
    Pack<E, V> p = {};
    if (t >= 0) {
      if (t < end) p = load_channels<E, V>(x.row(t, b), c, a.C);
    } else if (state) {
      p = load_channels<E, V>(state + ((int64_t)(K - 1 + t) * a.B + b) * a.C, c, a.C);
    }
#pragma unroll
    for (int i = 0; i < V; ++i) past[j][i] = (float)p.v[i];
  }
}

template <int TYPE, int K, int V, bool WHOLE>
__global__ __launch_bounds__(64 * kWaves) void conv_kernel(ConvArgs a, View<const Element<TYPE>> x, const Element<TYPE>* state,
                                                           View<Element<TYPE>> y, Element<TYPE>* state_out) {
  typedef Element<TYPE> E;
  const int columns = (a.C + 64 * kWaves * V - 1) / (64 * kWaves * V);
  const int stretch = blockIdx.x / columns, b = blockIdx.y;
  const int c = ((blockIdx.x - stretch * columns) * 64 * kWaves + threadIdx.x) * V;
  if (c >= a.C) return;
  const int t0 = stretch * kStretch, t1 = min(t0 + kStretch, a.T), end = sample_end(a.lengths, b, a.T);
  Filter<K, V> f;
  f.read(a, c);
  float past[K][V];                              // the newest input joins as the last
  read_history<E, K, V>(past, a, x, state, t0, end, b, c);
  if (stretch == 0 && state_out && K > 1) {
    // the inputs end - (K - 1) .. end - 1, all of them read before one is written
    Pack<E, V> last[K];
#pragma unroll
    for (int j = 0; j + 1 < K; ++j) {
      const int t = end - (K - 1) + j;
      last[j] = Pack<E, V>{};
      if (t >= 0) last[j] = load_channels<E, V>(x.row(t, b), c, a.C);
      else if (state) last[j] = load_channels<E, V>(state + ((int64_t)(K - 1 + t) * a.B + b) * a.C, c, a.C);
    }
#pragma unroll
    for (int j = 0; j + 1 < K; ++j) {
      E* const row = state_out + ((int64_t)j * a.B + b) * a.C;
      if (c + V <= a.C) store_pack(row + c, last[j]);
      else store_part(row + c, last[j], a.C - c);
    }
  }
  constexpr int kAhead = 4;                      // rows in flight while as many are worked on
  const int live = min(t1, end);
  Pack<E, V> in[2][kAhead];
  auto fetch = [&](Pack<E, V> (&to)[kAhead], int t) {
#pragma unroll
    for (int q = 0; q < kAhead; ++q) to[q] = load_channels<E, V, WHOLE>(x.row(min(t + q, live - 1), b), c, a.C);   // (no branch around a load)
  };
  auto work = [&](const Pack<E, V> (&from)[kAhead], int t) {
#pragma unroll
    for (int q = 0; q < kAhead; ++q) {
      float out[V];
#pragma unroll
      for (int i = 0; i < V; ++i) {
        past[K - 1][i] = (float)from[q].v[i];
        float p = f.bias[i];
#pragma unroll
        for (int k = 0; k < K; ++k) p += f.w[k][i] * past[k][i];
        out[i] = a.silu ? p * sigmoid(p) : p;
#pragma unroll
        for (int k = 0; k + 1 < K; ++k) past[k][i] = past[k + 1][i];
      }
      if (t + q < live) store_channels<E, V, WHOLE>(y.row(t + q, b), c, a.C, out);
    }
  };
  if (t0 < live) {
    fetch(in[0], t0);
    for (int t = t0; t < live; t += 2 * kAhead) {
      fetch(in[1], t + kAhead);
      work(in[0], t);
      fetch(in[0], t + 2 * kAhead);
      work(in[1], t + kAhead);
    }
  }
  const float zeros[V] = {};
  for (int t = max(t0, end); t < t1; ++t) store_channels<E, V>(y.row(t, b), c, a.C, zeros);
}

// A stretch [t0, t1) owns dx there and the parameters' sums over its g; it forms g for K - 1 steps more, which dx needs.
// The first one also owns the state's gradient, the steps -(K - 1) .. -1.
template <int TYPE, int K, int V, bool WHOLE>
__global__ __launch_bounds__(64 * kWaves) void conv_backward_kernel(ConvArgs a, View<const Element<TYPE>> x, const Element<TYPE>* state,
                                                                    View<const Element<TYPE>> dy, const Element<TYPE>* d_state_out,
                                                                    View<Element<TYPE>> dx, Element<TYPE>* d_state, float* partial,
                                                                    int stretches) {
  typedef Element<TYPE> E;
  __shared__ float sums[kWaves][64 * V];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, stretch = blockIdx.y * kWaves + wave;
  const int c = (blockIdx.x * 64 + lane) * V, b = blockIdx.z;
  float dw[K][V], db[V];
#pragma unroll
  for (int i = 0; i < V; ++i) {
    db[i] = 0.0f;
#pragma unroll
    for (int k = 0; k < K; ++k) dw[k][i] = 0.0f;
  }
  if (stretch < stretches && c < a.C) {
    const int t0 = stretch * kStretchBack, t1 = min(t0 + kStretchBack, a.T), end = sample_end(a.lengths, b, a.T);
    const int from = stretch == 0 ? -(K - 1) : t0;
    Filter<K, V> f;
    f.read(a, c);
    float past[K][V], g[K][V];                   // inputs and g of the last K steps, the newest last
    read_history<E, K, V>(past, a, x, state, t0, end, b, c);
#pragma unroll
    for (int k = 0; k < K; ++k)
#pragma unroll
      for (int i = 0; i < V; ++i) g[k][i] = 0.0f;
    constexpr int kAhead = 4;
    const int last = min(t1 + K - 1, end) - 1;   // of the steps that are read
    Pack<E, V> in[2][kAhead] = {}, up[2][kAhead] = {};
    auto fetch = [&](int set, int t) {
#pragma unroll
      for (int q = 0; q < kAhead; ++q) {
        const int at = min(t + q, max(last, t0));
        in[set][q] = load_channels<E, V, WHOLE>(x.row(at, b), c, a.C);
        up[set][q] = load_channels<E, V, WHOLE>(dy.row(at, b), c, a.C);
      }
    };
    auto work = [&](int set, int t) {
#pragma unroll
      for (int q = 0; q < kAhead; ++q) {
        if (t + q >= t1 + K - 1) break;
        const bool live = t + q < end, mine = live && t + q < t1;
        float out[V];
#pragma unroll
        for (int i = 0; i < V; ++i) {
          past[K - 1][i] = (float)in[set][q].v[i];
          float slope = 1.0f;
          if (a.silu) {
            float p = f.bias[i];
#pragma unroll
            for (int k = 0; k < K; ++k) p += f.w[k][i] * past[k][i];
            const float s = sigmoid(p);
            slope = s * (1.0f + p * (1.0f - s));
          }
          g[K - 1][i] = live ? (float)up[set][q].v[i] * slope : 0.0f;
          if (mine) {
            db[i] += g[K - 1][i];
#pragma unroll
            for (int k = 0; k < K; ++k) dw[k][i] += g[K - 1][i] * past[k][i];
          }
          float d = 0.0f;
#pragma unroll
          for (int k = 0; k < K; ++k) d += f.w[k][i] * g[K - 1 - k][i];
          out[i] = d;
#pragma unroll
          for (int k = 0; k + 1 < K; ++k) { past[k][i] = past[k + 1][i]; g[k][i] = g[k + 1][i]; }
        }
        const int s = t + q - (K - 1);           // the step whose gradient is complete
        if (s < from || s >= t1) continue;
        if (d_state_out && s >= end - (K - 1) && s < end) {
          const Pack<E, V> add = load_channels<E, V>(d_state_out + ((int64_t)(s - end + K - 1) * a.B + b) * a.C, c, a.C);
#pragma unroll
          for (int i = 0; i < V; ++i) out[i] += (float)add.v[i];
        }
        if (s >= 0) {
          if (dx.data) store_channels<E, V, WHOLE>(dx.row(s, b), c, a.C, out);
        } else if (d_state) {
          store_channels<E, V>(d_state + ((int64_t)(s + K - 1) * a.B + b) * a.C, c, a.C, out);
        }
      }
    };
    const bool any = WHOLE || last >= t0;          // (where there is a step at all, step t0 can be read)
    if (any) fetch(0, t0);
    for (int t = t0; t < t1 + K - 1; t += 2 * kAhead) {
      if (any) fetch(1, t + kAhead);
      work(0, t);
      if (any) fetch(0, t + 2 * kAhead);
      work(1, t + kAhead);
    }
  }
  if (!partial) return;
  // the workgroup's sums, [K + 1][C] a workgroup: the wavefronts meet in LDS in their order
  float* const mine = partial + ((int64_t)blockIdx.z * gridDim.y + blockIdx.y) * (K + 1) * a.C;
#pragma unroll
  for (int k = 0; k <= K; ++k) {
    __syncthreads();
#pragma unroll
    for (int i = 0; i < V; ++i) sums[wave][i * 64 + lane] = k < K ? dw[k < K ? k : 0][i] : db[i];
    __syncthreads();
    for (int i = wave; i < V; i += kWaves) {
      const float sum = (sums[0][i * 64 + lane] + sums[1][i * 64 + lane]) + (sums[2][i * 64 + lane] + sums[3][i * 64 + lane]);
      if (c + i < a.C) mine[(int64_t)k * a.C + c + i] = sum;
    }
  }
}

// Sums [K + 1][C] to d_weight [C][K] and d_bias [C].
struct PutParameters {
  float* d_weight;
  float* d_bias;
  int C, K;
  __device__ void operator()(int64_t i, float sum) const {
    const int k = (int)(i / C), c = (int)(i - (int64_t)k * C);
    if (k < K && d_weight) d_weight[(int64_t)c * K + k] = sum;
    if (k == K && d_bias) d_bias[c] = sum;
  }
};

int stretches_of(int T, int length) { return T > length ? (T + length - 1) / length : 1; }
int groups_of(int stretches) { return (stretches + kWaves - 1) / kWaves; }

template <int TYPE, int K>
hipError_t run_forward(const ConvArgs& a, const sprnn_conv_t* p, const sprnn_seq_t& y, void* state_out, hipStream_t stream) {
  typedef Element<TYPE> E;
  constexpr int V = 8 / (int)sizeof(E);
  const int stretches = stretches_of(a.T, kStretch);
  const int64_t groups = (int64_t)((a.C + 64 * kWaves * V - 1) / (64 * kWaves * V)) * stretches;
  if (groups > 0x7fffffffLL) return hipErrorInvalidValue;
  return launch(a.C % V == 0 ? conv_kernel<TYPE, K, V, true> : conv_kernel<TYPE, K, V, false>, dim3((unsigned)groups, (unsigned)a.B), dim3(64 * kWaves), 0, stream, a, view<const E>(p->x), static_cast<const E*>(p->state),
                view<E>(y), static_cast<E*>(state_out));
}

template <int TYPE, int K>
hipError_t run_backward(const ConvArgs& a, const sprnn_conv_t* p, const sprnn_seq_t& dy, const void* d_state_out, const sprnn_seq_t& dx,
                        float* d_weight, float* d_bias, void* d_state, float* workspace, hipStream_t stream) {
  typedef Element<TYPE> E;
  constexpr int V = 2;                           // the window of g and the parameters' sums are in registers, too
  const int stretches = stretches_of(a.T, kStretchBack), groups = groups_of(stretches);
  const bool summed = d_weight || d_bias;
  float* const partial = summed ? workspace : nullptr;         // (none without a sample: sums of nothing are zeros)
  if (a.B > 0) {
    const dim3 grid((unsigned)((a.C + 64 * V - 1) / (64 * V)), (unsigned)groups, (unsigned)a.B);
    const hipError_t e = launch(a.C % V == 0 && a.T > 0 ? conv_backward_kernel<TYPE, K, V, true> : conv_backward_kernel<TYPE, K, V, false>, grid, dim3(64 * kWaves), 0, stream, a, view<const E>(p->x),
                                static_cast<const E*>(p->state), view<const E>(dy), static_cast<const E*>(d_state_out), view<E>(dx),
                                static_cast<E*>(d_state), partial, stretches);
    if (e != hipSuccess) return e;
  }
  if (!summed) return hipSuccess;
  return launch_sum_partials(partial, groups * a.B, (int64_t)(K + 1) * a.C, PutParameters{d_weight, d_bias, a.C, K}, stream);
}

bool good_conv(const sprnn_conv_t* p) {
  return p && good_sizes(p->steps, p->batch, p->channels) && p->width >= 1 && p->width <= 8 && activation_type(p->type) &&
         (p->silu == 0 || p->silu == 1) && p->weight && aligned_to(p->weight, 4) && aligned_to(p->bias, 4) &&
         aligned_to(p->state, type_bytes(p->type)) && aligned_to(p->lengths, 4);
}
ConvArgs arguments(const sprnn_conv_t* p) { return ConvArgs{p->steps, p->batch, p->channels, p->silu, p->weight, p->bias, p->lengths}; }

}  // namespace
}  // namespace sprnn

using namespace sprnn;

#define EVERY_WIDTH(TYPE) CASE(TYPE, 1) CASE(TYPE, 2) CASE(TYPE, 3) CASE(TYPE, 4) CASE(TYPE, 5) CASE(TYPE, 6) CASE(TYPE, 7) CASE(TYPE, 8)

extern "C" {

int sprnn_conv_forward(int device_id, const sprnn_conv_t* conv, sprnn_seq_t y, void* state_out, void* stream) {
  if (device_id < 0 || !good_conv(conv)) return SPRNN_ERR_INVALID;
  const int T = conv->steps, B = conv->batch, type = conv->type;
  if (!aligned_to(state_out, type_bytes(type))) return SPRNN_ERR_INVALID;
  if (B == 0 || (T == 0 && (!state_out || conv->width == 1))) return SPRNN_OK;
  if (T > 0 && (!good_view(conv->x, type) || !good_output(y, type, T, B, conv->channels))) return SPRNN_ERR_INVALID;
  DeviceGuard guard(device_id);
  if (!guard.ok) return SPRNN_ERR_HIP;
  const ConvArgs a = arguments(conv);
  const hipStream_t s = static_cast<hipStream_t>(stream);
  hipError_t e = hipErrorInvalidValue;
#define CASE(TYPE, K) \
  if (type == TYPE && conv->width == K) e = run_forward<TYPE, K>(a, conv, y, state_out, s);
  EVERY_WIDTH(SPRNN_TYPE_F32)
  EVERY_WIDTH(SPRNN_TYPE_F16)
  EVERY_WIDTH(SPRNN_TYPE_BF16)
#undef CASE
  if (e == hipErrorInvalidValue) return SPRNN_ERR_INVALID;   // more workgroups than a launch can have
  return SPRNN_HIP(e) ? SPRNN_OK : SPRNN_ERR_HIP;
}

int sprnn_conv_sizes(const sprnn_conv_t* conv, int64_t* backward_workspace) {
  if (!conv || !good_sizes(conv->steps, conv->batch, conv->channels) || conv->width < 1 || conv->width > 8) return SPRNN_ERR_INVALID;
  const int64_t groups = groups_of(stretches_of(conv->steps, kStretchBack));
  if (backward_workspace) *backward_workspace = groups * conv->batch * (conv->width + 1) * conv->channels * 4;
  return SPRNN_OK;
}

int sprnn_conv_backward(int device_id, const sprnn_conv_t* conv, sprnn_seq_t dy, const void* d_state_out, sprnn_seq_t dx,
                        float* d_weight, float* d_bias, void* d_state, void* workspace, int64_t workspace_bytes, void* stream) {
  if (device_id < 0 || !good_conv(conv)) return SPRNN_ERR_INVALID;
  const int T = conv->steps, B = conv->batch, type = conv->type;
  if (!aligned_to(d_state_out, type_bytes(type)) || !aligned_to(d_state, type_bytes(type)) || !aligned_to(d_weight, 4) || !aligned_to(d_bias, 4))
    return SPRNN_ERR_INVALID;
  if (T > 0 && B > 0 &&
      (!good_view(conv->x, type) || !good_view(dy, type) || (dx.data && !good_output(dx, type, T, B, conv->channels))))
    return SPRNN_ERR_INVALID;
  int64_t need = 0;
  (void)sprnn_conv_sizes(conv, &need);
  if ((d_weight || d_bias) && need > 0 && (!workspace || !aligned_to(workspace, 16) || workspace_bytes < need)) return SPRNN_ERR_INVALID;
  DeviceGuard guard(device_id);
  if (!guard.ok) return SPRNN_ERR_HIP;
  const ConvArgs a = arguments(conv);
  const hipStream_t s = static_cast<hipStream_t>(stream);
  hipError_t e = hipErrorInvalidValue;
#define CASE(TYPE, K)                   \
  if (type == TYPE && conv->width == K) \
    e = run_backward<TYPE, K>(a, conv, dy, d_state_out, dx, d_weight, d_bias, d_state, static_cast<float*>(workspace), s);
  EVERY_WIDTH(SPRNN_TYPE_F32)
  EVERY_WIDTH(SPRNN_TYPE_F16)
  EVERY_WIDTH(SPRNN_TYPE_BF16)
#undef CASE
  return SPRNN_HIP(e) ? SPRNN_OK : SPRNN_ERR_HIP;
}

}  // extern "C"
