// Forward pass of the selective scan (see sprnn_scan.h for the mathematics) and its C entry points.
#include "sprnn_scan.h"

namespace sprnn {
namespace {

// Prompts.  A wavefront owns 64 / S channels of one sample (and group) and a segment of time; a lane holds NS states of a
// channel, S lanes share one.  B and C of a tile of steps are the same for all its channels: they are brought into LDS in
// binary32 once a tile, and u, dt and z of the next tile are in flight while a tile is worked through.
// LOCAL: a segment's effect only (H[segment + 1] from a zero state, sums[segment] = sum of d).
template <int TYPE, int NS, int S, bool LOCAL>
__global__ __launch_bounds__(64) void scan_kernel(ScanArgs a, View<const Element<TYPE>> us, View<const Element<TYPE>> dts,
                                                  View<const Element<TYPE>> zs, View<const Element<TYPE>> Bs,
                                                  View<const Element<TYPE>> Cs, const float* state_in, View<Element<TYPE>> ys,
                                                  float* state_out, float* kept, float* H, float* sums) {
  typedef Element<TYPE> E;
  constexpr int kN = NS * S, kOwn = kTile * kN / 64;   // of B; as many of C
  static_assert(kTile * kN % 64 == 0, "the tile's states are dealt out evenly");
  __shared__ __attribute__((aligned(16))) float low[2][LOCAL ? 1 : 2][kTile][kN];
  const int lane = threadIdx.x, sub = lane % S;
  const int group = blockIdx.x / a.blocks, block = blockIdx.x - group * a.blocks;
  const int b = blockIdx.y, seg = blockIdx.z;
  const int in_group = block * (64 / S) + lane / S;
  const bool mine = in_group < a.per_group;
  const int c = group * a.per_group + min(in_group, a.per_group - 1);
  const int t0 = seg * a.segment, t1 = min(t0 + a.segment, a.T), end = sample_end(a.lengths, b, a.T);
  const int live = min(t1, end);

  float A[NS], h[NS];
#pragma unroll
  for (int i = 0; i < NS; ++i) {
    const int n = sub * NS + i;
    A[i] = n < a.N ? a.A[(int64_t)c * a.N + n] * kLog2e : 0.0f;
    h[i] = 0.0f;
  }
  if (!LOCAL) {
    if (H) {
      const States from(H, seg, b, a.B, a.quads, a.C);
#pragma unroll
      for (int q = 0; q < NS / 4; ++q) {
        const floatx4_t p = from.load(sub * (NS / 4) + q, c);
#pragma unroll
        for (int i = 0; i < 4; ++i) h[4 * q + i] = p[i];
      }
    } else if (state_in) {
#pragma unroll
      for (int i = 0; i < NS; ++i) {
        const int n = sub * NS + i;
        if (n < a.N) h[i] = state_in[((int64_t)b * a.C + c) * a.N + n];
      }
    }
  }
  auto put_states = [&](float* base, int64_t copy) {
    const States to(base, copy, b, a.B, a.quads, a.C);
#pragma unroll
    for (int q = 0; q < NS / 4; ++q) to.store(sub * (NS / 4) + q, c, floatx4_t{h[4 * q], h[4 * q + 1], h[4 * q + 2], h[4 * q + 3]});
  };
  const float D = !LOCAL && a.D ? a.D[c] : 0.0f, bias = a.dt_bias ? a.dt_bias[c] : 0.0f;

  E u[kTile], dt[kTile], z[kTile];
  E own_B[kOwn], own_C[kOwn];
  Cursor<const E> u_at(us, t0, b), dt_at(dts, t0, b), z_at(zs, t0, b);
  Cursor<const E> B_at(Bs, t0, b, group * a.N), C_at(Cs, t0, b, group * a.N);
  Cursor<E> y_at(ys, t0, b);
  const bool gated = zs.data != nullptr;
  auto fetch = [&](int rows) {
    const Tile<const E> u_rows = u_at.tile(rows, a.C), dt_rows = dt_at.tile(rows, a.C), z_rows = z_at.tile(rows, gated ? a.C : 0);
    const Tile<const E> B_rows = B_at.tile(rows, a.N), C_rows = C_at.tile(rows, a.N);
    u_at.forth(); dt_at.forth(); z_at.forth(); B_at.forth(); C_at.forth();
#pragma unroll
    for (int q = 0; q < kTile; ++q) {
      u[q] = u_rows.load(q, c);
      dt[q] = dt_rows.load(q, c);
      if (!LOCAL) z[q] = z_rows.load(q, c);
    }
#pragma unroll
    for (int i = 0; i < kOwn; ++i) {
      const int at = i * 64 + lane;
      own_B[i] = B_rows.load(at / kN, at % kN);
      if (!LOCAL) own_C[i] = C_rows.load(at / kN, at % kN);
    }
  };
  float total = 0.0f;
  fetch(live - t0);
  int buffer = 0;
  for (int t = t0; t < live; t += kTile, buffer ^= 1) {
#pragma unroll
    for (int i = 0; i < kOwn; ++i) {
      const int at = i * 64 + lane;
      const bool in = at % kN < a.N && t + at / kN < live;   // neither the next group's states nor what lies behind the end
      (&low[buffer][0][0][0])[at] = in ? (float)own_B[i] : 0.0f;
      if (!LOCAL) (&low[buffer][LOCAL ? 0 : 1][0][0])[at] = in ? (float)own_C[i] : 0.0f;
    }
    if (kept && mine) put_states(kept, t / kTile);
    float d[kTile], x[kTile], gate[kTile], skip[kTile];
#pragma unroll
    for (int q = 0; q < kTile; ++q) {
      const float v = (float)dt[q] + bias;
      const bool in = t + q < live;
      const float uq = in ? (float)u[q] : 0.0f;
      d[q] = in ? a.softplus ? softplus(v) : v : 0.0f;
      x[q] = d[q] * uq;
      skip[q] = D * uq;
      const float g = (float)z[q];
      gate[q] = gated ? g * sigmoid(g) : 1.0f;
    }
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
    fetch(live - t - kTile);
    const Tile<E> y_rows = y_at.tile(live - t, a.C);
    y_at.forth();
#pragma unroll
    for (int q = 0; q < kTile; ++q) {
      const float* const Bq = &low[buffer][0][q][sub * NS];
      const float* const Cq = &low[buffer][LOCAL ? 0 : 1][q][sub * NS];
      float y = 0.0f;
#pragma unroll
      for (int i = 0; i < NS; ++i) {
        h[i] = exp2_fast(d[q] * A[i]) * h[i] + x[q] * Bq[i];
        if (!LOCAL) y += Cq[i] * h[i];
      }
      if (LOCAL) {
        total += d[q];
      } else {
        y = (sum_lanes<S>(y) + skip[q]) * gate[q];
        if (S == 1 && mine) y_rows.store(q, c, y);
        else if (sub == q % S && mine) y_rows.store(q, c, y);
      }
    }
  }
  if (!mine) return;
  if (LOCAL) {
    put_states(H, seg + 1);
    if (sub == 0) sums[((int64_t)seg * a.B + b) * a.C + c] = total;
    return;
  }
  if (sub == 0)
    for (int t = max(t0, end); t < t1; ++t) ys.row(t, b)[c] = (E)0.0f;
  // the segment that holds the sample's last step has its last state
  if (state_out && (end > t0 || t0 == 0) && end <= t1) {
#pragma unroll
    for (int i = 0; i < NS; ++i) {
      const int n = sub * NS + i;
      if (n < a.N) state_out[((int64_t)b * a.C + c) * a.N + n] = h[i];
    }
  }
}

// One lane per (sample, channel, quad of states).
__global__ __launch_bounds__(256) void chain_kernel(ScanArgs a, int segments, const float* first, float* H, const float* sums) {
  const int64_t at = (int64_t)blockIdx.x * 256 + threadIdx.x;
  const int64_t lanes = (int64_t)a.B * a.quads * a.C;
  if (at >= lanes) return;
  const int c = (int)(at % a.C), quad = (int)(at / a.C % a.quads), b = (int)(at / ((int64_t)a.C * a.quads));
  float A[4], h[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int n = quad * 4 + i;
    A[i] = n < a.N ? a.A[(int64_t)c * a.N + n] * kLog2e : 0.0f;
    h[i] = first && n < a.N ? first[((int64_t)b * a.C + c) * a.N + n] : 0.0f;
  }
  for (int s = 0; s < segments; ++s) {
    float* const slot = H + ((int64_t)s * lanes + at) * 4;
    Pack<float, 4> p;
    if (s > 0) {
      p = load_pack<4>(slot);
      const float total = sums[((int64_t)(s - 1) * a.B + b) * a.C + c];
#pragma unroll
      for (int i = 0; i < 4; ++i) h[i] = exp2_fast(A[i] * total) * h[i] + p.v[i];
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) p.v[i] = h[i];
    store_pack(slot, p);
  }
}

// Single tokens: the state is read and written once and bounds the call.  S lanes of four states a channel, so that a
// wavefront's states are consecutive 16 bytes in memory; a lane reads its own part of everything.
template <int TYPE, int S>
__global__ __launch_bounds__(64) void scan_token_kernel(ScanArgs a, View<const Element<TYPE>> us, View<const Element<TYPE>> dts,
                                                        View<const Element<TYPE>> zs, View<const Element<TYPE>> Bs,
                                                        View<const Element<TYPE>> Cs, const float* state_in,
                                                        View<Element<TYPE>> ys, float* state_out) {
  typedef Element<TYPE> E;
  const int lane = threadIdx.x, sub = lane % S, b = blockIdx.y;
  const int own = blockIdx.x * (64 / S) + lane / S, c = min(own, a.C - 1);
  const int n0 = sub * 4, count = min(4, a.N - n0);        // may be 0 or less: a lane without states
  const bool live = sample_end(a.lengths, b, 1) > 0;
  const int64_t group = c / a.per_group, at = ((int64_t)b * a.C + c) * a.N + n0;
  Pack<float, 4> h = {}, A = {};
  Pack<E, 4> Bn = {}, Cn = {};
  const float* const A_row = a.A + (int64_t)c * a.N + n0;
  if (count == 4) {
    if (state_in) h = load_pack<4>(state_in + at);
    A = load_pack<4>(A_row);
    if (live) {
      Bn = load_pack<4>(Bs.row(0, b) + group * a.N + n0);
      Cn = load_pack<4>(Cs.row(0, b) + group * a.N + n0);
    }
  } else if (count > 0) {
    if (state_in) h = load_part<4>(state_in + at, count);
    A = load_part<4>(A_row, count);
    if (live) {
      Bn = load_part<4>(Bs.row(0, b) + group * a.N + n0, count);
      Cn = load_part<4>(Cs.row(0, b) + group * a.N + n0, count);
    }
  }
  float y = 0.0f;
  if (live) {
    const float u = (float)us.row(0, b)[c], v = (float)dts.row(0, b)[c] + (a.dt_bias ? a.dt_bias[c] : 0.0f);
    const float z = zs.data ? (float)zs.row(0, b)[c] : 0.0f, D = a.D ? a.D[c] : 0.0f;
    const float d = a.softplus ? softplus(v) : v, x = d * u;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      h.v[i] = exp2_fast(d * (A.v[i] * kLog2e)) * h.v[i] + x * (float)Bn.v[i];
      y += (float)Cn.v[i] * h.v[i];
    }
    y = sum_lanes<S>(y) + D * u;
    if (zs.data) y *= z * sigmoid(z);
  }
  if (own >= a.C) return;
  if (sub == 0) ys.row(0, b)[c] = (E)y;
  if (!state_out) return;
  if (count == 4) store_pack(state_out + at, h);
  else if (count > 0) store_part(state_out + at, h, count);
}

template <int TYPE, int NS, int S>
hipError_t run_prompt(ScanArgs a, const ScanShape& s, const sprnn_scan_t* p, const float* state_in, const sprnn_seq_t& y, float* state_out,
                      float* kept, float* H, float* sums, hipStream_t stream) {
  typedef Element<TYPE> E;
  a.blocks = (s.per_group + 64 / S - 1) / (64 / S);
  const View<const E> u = view<const E>(p->u), dt = view<const E>(p->dt), z = view<const E>(p->z), B = view<const E>(p->B), C = view<const E>(p->C);
  const dim3 block(64);
  if (s.segments > 1) {
    hipError_t e = launch(scan_kernel<TYPE, NS, S, true>, dim3((unsigned)(a.blocks * s.G), (unsigned)s.B, (unsigned)s.segments - 1), block, 0, stream,
                          a, u, dt, z, B, C, (const float*)nullptr, view<E>(y), (float*)nullptr, (float*)nullptr, H, sums);
    if (e != hipSuccess) return e;
    e = launch_chain(a, s.segments, state_in, H, sums, stream);
    if (e != hipSuccess) return e;
  } else {
    H = nullptr;
  }
  return launch(scan_kernel<TYPE, NS, S, false>, dim3((unsigned)(a.blocks * s.G), (unsigned)s.B, (unsigned)s.segments), block, 0, stream, a, u,
                dt, z, B, C, state_in, view<E>(y), state_out, kept, H, sums);
}

template <int TYPE>
hipError_t run_scan(const ScanShape& s, const sprnn_scan_t* p, const float* state_in, const sprnn_seq_t& y, float* state_out, float* kept,
                    float* workspace, hipStream_t stream) {
  typedef Element<TYPE> E;
  const ScanArgs a = scan_arguments(p, s);
  if (s.T == 1 && !kept) {
    auto run = [&](auto lanes) {
      constexpr int S = decltype(lanes)::value;
      return launch(scan_token_kernel<TYPE, S>, dim3((unsigned)((s.C + 64 / S - 1) / (64 / S)), (unsigned)s.B), dim3(64), 0, stream, a,
                    view<const E>(p->u), view<const E>(p->dt), view<const E>(p->z), view<const E>(p->B), view<const E>(p->C), state_in,
                    view<E>(y), state_out);
    };
    return s.quads <= 1 ? run(std::integral_constant<int, 1>()) : s.quads <= 2 ? run(std::integral_constant<int, 2>())
         : s.quads <= 4 ? run(std::integral_constant<int, 4>()) : s.quads <= 8 ? run(std::integral_constant<int, 8>())
         : s.quads <= 16 ? run(std::integral_constant<int, 16>()) : run(std::integral_constant<int, 32>());
  }
  float* const H = workspace;
  float* const sums = workspace + s.segments * s.state_floats();
  return s.N <= 8 ? run_prompt<TYPE, 8, 1>(a, s, p, state_in, y, state_out, kept, H, sums, stream)
       : s.N <= 16 ? run_prompt<TYPE, 16, 1>(a, s, p, state_in, y, state_out, kept, H, sums, stream)
       : s.N <= 32 ? run_prompt<TYPE, 16, 2>(a, s, p, state_in, y, state_out, kept, H, sums, stream)
       : s.N <= 64 ? run_prompt<TYPE, 16, 4>(a, s, p, state_in, y, state_out, kept, H, sums, stream)
                   : run_prompt<TYPE, 16, 8>(a, s, p, state_in, y, state_out, kept, H, sums, stream);
}

int round_up(int n, int to) { return (n + to - 1) / to * to; }

}  // namespace

hipError_t launch_chain(const ScanArgs& a, int segments, const float* first, float* H, const float* sums, hipStream_t stream) {
  const int64_t lanes = (int64_t)a.B * a.quads * a.C;
  return launch(chain_kernel, dim3((unsigned)((lanes + 255) / 256)), dim3(256), 0, stream, a, segments, first, H, sums);
}

// A wavefront per 64 states' lanes and sample runs at its best rate with one or two wavefronts a SIMD; below half a
// wavefront a SIMD two runs over divided time (1.9 times the work) win.
ScanShape scan_shape(const sprnn_scan_t* p) {
  ScanShape s{};
  s.T = p->steps; s.B = p->batch; s.C = p->channels; s.N = p->states; s.G = p->groups;
  s.per_group = s.C / s.G;
  s.quads = (s.N + 3) / 4;
  auto divide = [&](int64_t waves, int* segments, int* segment) {
    int64_t n = waves > 0 ? 2 * kSimds / waves : 1;
    n = n < s.T / 64 ? n : s.T / 64;
    if (n < 4) n = 1;
    *segment = round_up(s.T > 0 ? (int)((s.T + n - 1) / n) : 1, kTile);
    *segments = s.T > 0 ? (s.T + *segment - 1) / *segment : 1;
  };
  const int lanes = s.N <= 16 ? 1 : s.N <= 32 ? 2 : s.N <= 64 ? 4 : 8;
  const int64_t waves = (int64_t)s.G * ((s.per_group + 64 / lanes - 1) / (64 / lanes)) * s.B;
  divide(waves, &s.segments, &s.segment);
  divide(waves, &s.back_segments, &s.back_segment);
  return s;
}

bool good_scan(const sprnn_scan_t* p) {
  return p && good_sizes(p->steps, p->batch, p->channels) && p->channels <= kChannelsMost && p->states >= 1 && p->states <= kStatesMost && p->groups >= 1 &&
         p->channels % p->groups == 0;
}

// Bytes of what the passes need besides their arguments.
static void scan_sizes(const ScanShape& s, int64_t* forward, int64_t* backward, int64_t* kept) {
  *forward = s.segments > 1 ? (s.segments * s.state_floats() + (int64_t)s.segments * s.B * s.C) * 4 : 0;
  *kept = (int64_t)((s.T + kTile - 1) / kTile) * s.state_floats() * 4;
  *backward = scan_backward_bytes(s);
}

static bool good_rows(const sprnn_seq_t& s, int type) { return good_view(s, type) && s.step <= kStepMost; }
static bool good_rows(const sprnn_seq_t& s, int type, int T, int B, int width) { return good_output(s, type, T, B, width) && s.step <= kStepMost; }

static bool good_arguments(const sprnn_scan_t* p) {
  if (!good_scan(p) || !activation_type(p->type) || (p->softplus != 0 && p->softplus != 1)) return false;
  if (!p->A || !aligned_to(p->A, 4) || !aligned_to(p->D, 4) || !aligned_to(p->dt_bias, 4) || !aligned_to(p->lengths, 4)) return false;
  if (p->steps == 0 || p->batch == 0) return true;
  const int type = p->type;
  return good_rows(p->u, type) && good_rows(p->dt, type) && (!p->z.data || good_rows(p->z, type)) && good_rows(p->B, type) && good_rows(p->C, type);
}

}  // namespace sprnn

using namespace sprnn;

extern "C" {

int sprnn_scan_sizes(const sprnn_scan_t* scan, int64_t* forward_workspace, int64_t* backward_workspace, int64_t* kept) {
  if (!good_scan(scan)) return SPRNN_ERR_INVALID;
  int64_t f, b, k;
  scan_sizes(scan_shape(scan), &f, &b, &k);
  if (forward_workspace) *forward_workspace = f;
  if (backward_workspace) *backward_workspace = b;
  if (kept) *kept = k;
  return SPRNN_OK;
}

int sprnn_scan_forward(int device_id, const sprnn_scan_t* scan, const float* state_in, sprnn_seq_t y, float* state_out,
                       void* kept, void* workspace, int64_t workspace_bytes, void* stream) {
  if (device_id < 0 || !good_arguments(scan)) return SPRNN_ERR_INVALID;
  if (!aligned_to(state_in, 4) || !aligned_to(state_out, 4) || !aligned_to(kept, 16)) return SPRNN_ERR_INVALID;
  const ScanShape s = scan_shape(scan);
  if (s.B == 0) return SPRNN_OK;
  if (s.T > 0 && !good_rows(y, scan->type, s.T, s.B, s.C)) return SPRNN_ERR_INVALID;
  int64_t need, back, keep;
  scan_sizes(s, &need, &back, &keep);
  if (need > 0 && (!workspace || !aligned_to(workspace, 16) || workspace_bytes < need)) return SPRNN_ERR_INVALID;
  DeviceGuard guard(device_id);
  if (!guard.ok) return SPRNN_ERR_HIP;
  const hipStream_t stream_ = static_cast<hipStream_t>(stream);
  float* const kept_ = static_cast<float*>(kept);
  float* const workspace_ = static_cast<float*>(workspace);
  const hipError_t e = scan->type == SPRNN_TYPE_F32 ? run_scan<SPRNN_TYPE_F32>(s, scan, state_in, y, state_out, kept_, workspace_, stream_)
                     : scan->type == SPRNN_TYPE_F16 ? run_scan<SPRNN_TYPE_F16>(s, scan, state_in, y, state_out, kept_, workspace_, stream_)
                                                    : run_scan<SPRNN_TYPE_BF16>(s, scan, state_in, y, state_out, kept_, workspace_, stream_);
  return SPRNN_HIP(e) ? SPRNN_OK : SPRNN_ERR_HIP;
}

int sprnn_scan_backward(int device_id, const sprnn_scan_t* scan, sprnn_seq_t dy, const float* d_state_out, const void* kept,
                        const sprnn_scan_gradients_t* gradients, void* workspace, int64_t workspace_bytes, void* stream) {
  if (device_id < 0 || !good_arguments(scan) || !gradients) return SPRNN_ERR_INVALID;
  const ScanShape s = scan_shape(scan);
  const sprnn_scan_gradients_t& g = *gradients;
  if (!aligned_to(d_state_out, 4) || !aligned_to(kept, 16) || !aligned_to(g.A, 4) || !aligned_to(g.D, 4) || !aligned_to(g.dt_bias, 4) ||
      !aligned_to(g.state, 4))
    return SPRNN_ERR_INVALID;
  if (s.T > 0 && s.B > 0) {
    auto good = [&](const sprnn_seq_t& o, int width) { return !o.data || good_rows(o, scan->type, s.T, s.B, width); };
    if (!kept || !good_rows(dy, scan->type) || !good(g.u, s.C) || !good(g.dt, s.C) || !good(g.z, s.C) || !good(g.B, s.G * s.N) || !good(g.C, s.G * s.N))
      return SPRNN_ERR_INVALID;
    if (g.z.data && !scan->z.data) return SPRNN_ERR_INVALID;
  }
  if (!workspace || !aligned_to(workspace, 16) || workspace_bytes < scan_backward_bytes(s)) return SPRNN_ERR_INVALID;
  DeviceGuard guard(device_id);
  if (!guard.ok) return SPRNN_ERR_HIP;
  return SPRNN_HIP(launch_scan_backward(s, scan, dy, d_state_out, static_cast<const float*>(kept), gradients, static_cast<float*>(workspace),
                                        static_cast<hipStream_t>(stream)))
             ? SPRNN_OK
             : SPRNN_ERR_HIP;
}

}  // extern "C"
