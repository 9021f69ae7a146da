// Forward pass of the selective scan (see sprnn_scan.h for the mathematics) and its C entry points.
#include "sprnn_scan.h"

// Splits of a channel's states over lanes: states a lane, lanes.
#define EVERY_SPLIT CASE(8, 1) CASE(16, 1) CASE(4, 2) CASE(8, 2) CASE(16, 2) CASE(4, 4) CASE(8, 4) CASE(16, 4) CASE(16, 8)

namespace sprnn {
namespace {

int blocks_of(const ScanShape& s) { return (s.per_group + 63) / 64; }

// Where all workgroups are resident from the start, a compute unit is as late as the sum of its samples is long.  Workgroups go
// to the units in order, one to each before any gets its second: so the samples are taken from the longest on, and from the
// shortest of the round on in every other round.  (8 x 2048 x 4608, lengths anywhere up to 2048: 309 us in the samples' order,
// 279 from the longest on, 271 so.)
constexpr int kUnits = kSimds / 4, kSamplesDealt = 64;
__device__ __forceinline__ void deal_by_length(const ScanArgs& a, int& column, int& b) {
  const int columns = gridDim.x, all = columns * a.B;
  int at = blockIdx.y * columns + blockIdx.x;
  const int round = at / kUnits;
  if (round % 2 && (round + 1) * kUnits <= all) at = round * kUnits + (kUnits - 1 - at % kUnits);
  const int wanted = at / columns, lane = threadIdx.x & 63;
  column = at - wanted * columns;
  const int own = lane < a.B ? sample_end(a.lengths, lane, a.T) : -1;
  int rank = 0;                                            // samples in front of this lane's
  for (int i = 0; i < a.B; ++i) {
    const int other = __builtin_amdgcn_readlane(own, i);
    rank += other > own || (other == own && i < lane);
  }
  b = __builtin_ctzll(__ballot(lane < a.B && rank == wanted));
}

// Prompts.  A workgroup owns 64 channels of one sample (and group) and a segment of time; S lanes share a channel, a lane
// holds NS of its states, so there are S wavefronts.  Everything that depends on (step, channel) alone is computed once:
// the S lanes of a channel share out the steps of a tile, and hand d and d u over to their neighbours.  B and C of a tile
// are the same for all channels and are brought into LDS in binary32 once a tile; the next tile's loads are in flight while
// a tile is worked through, and two LDS buffers make one barrier a tile enough.  Bound by the vector units: for four states of
// a lane and 16 steps 520 instructions and 72 exponentials, which take two turns each; they are busy three quarters of the time
// (1 x 4096 x 2304 with 16 states: 60 us and 40 for the local run).
// kLocal: a segment's effect only (H[segment + 1] from a zero state, the first from its true one; sums[segment] = sum of d).
enum { kPlain, kKeeping, kLocal };     // what a run of the forward pass leaves: y; y and the states in front of every tile; its effect

template <int TYPE, int NS, int S, int MODE>
__global__ __launch_bounds__(64 * S) void scan_kernel(ScanArgs a, View<const Element<TYPE>> us, View<const Element<TYPE>> dts,
                                                      View<const Element<TYPE>> zs, View<const Element<TYPE>> Bs,
                                                      View<const Element<TYPE>> Cs, const float* state_in, View<Element<TYPE>> ys,
                                                      float* state_out, float* kept, float* H, float* sums) {
  typedef Element<TYPE> E;
  constexpr bool LOCAL = MODE == kLocal;
  constexpr int kN = NS * S, kItems = kTile / S;
  constexpr int kOwn = kTile * kN / (64 * S) > 0 ? kTile * kN / (64 * S) : 1;   // elements of B (and of C) that a lane brings
  constexpr int kAhead = 2;          // tiles whose inputs are in flight (even: the LDS buffers take turns)
  constexpr bool kHalf = kTile * kN < 64 * S;    // four states a lane: two lanes bring the same one (no branch around a load in flight)
  static_assert(S <= kTile && (kHalf || kTile * kN % (64 * S) == 0), "steps and states are dealt out evenly");
  __shared__ __attribute__((aligned(16))) float low[2][LOCAL ? 1 : 2][kTile][kN];
  const int tid = threadIdx.x, sub = tid % S;
  int column = blockIdx.x, b = blockIdx.y;
  const int seg = blockIdx.z;
  if (MODE != kLocal && a.by_length) deal_by_length(a, column, b);
  const int group = column / a.blocks, block = column - group * a.blocks;
  const int in_group = block * 64 + tid / S;
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
  if (!LOCAL && H) {
    chained_states<NS / 4>(h, A, a, H, sums, seg, b, sub * (NS / 4), c);
  } else if (state_in && seg == 0) {
#pragma unroll
    for (int i = 0; i < NS; ++i) {
      const int n = sub * NS + i;
      if (n < a.N) h[i] = state_in[((int64_t)b * a.C + c) * a.N + n];
    }
  }
  auto put_states = [&](float* base, int64_t copy) {
    const States to(base, copy, b, a.B, a.quads, a.C);
#pragma unroll
    for (int q = 0; q < NS / 4; ++q) to.store(sub * (NS / 4) + q, c, floatx4_t{h[4 * q], h[4 * q + 1], h[4 * q + 2], h[4 * q + 3]});
  };
  if (LOCAL && seg == 0 && mine) put_states(H, 0);         // (the last segment may write its state over state_in)
  const float D = !LOCAL && a.D ? a.D[c] : 0.0f, bias = a.dt_bias ? a.dt_bias[c] : 0.0f;

  // this lane's steps of a tile are sub, sub + S, ..
  struct Inputs {
    E u[kItems], dt[kItems], z[kItems], own_B[kOwn], own_C[kOwn];
  };
  Cursor<const E> u_at(us, t0, b), dt_at(dts, t0, b), z_at(zs, t0, b);
  Cursor<const E> B_at(Bs, t0, b, group * a.N), C_at(Cs, t0, b, group * a.N);
  Cursor<E> y_at(ys, t0, b);
  const bool gated = zs.data != nullptr;
  auto fetch = [&](Inputs& in, int rows) {
    const Tile<const E> u_rows = u_at.tile(rows, a.C), dt_rows = dt_at.tile(rows, a.C), z_rows = z_at.tile(gated ? rows : 0, a.C);
    const Tile<const E> B_rows = B_at.tile(rows, a.N), C_rows = C_at.tile(rows, a.N);
    u_at.forth(); dt_at.forth(); z_at.forth(); B_at.forth(); C_at.forth();
#pragma unroll
    for (int i = 0; i < kItems; ++i) {
      in.u[i] = u_rows.load(i * S + sub, c);
      in.dt[i] = dt_rows.load(i * S + sub, c);
      if (!LOCAL) in.z[i] = z_rows.load(i * S + sub, c);
    }
#pragma unroll
    for (int i = 0; i < kOwn; ++i) {
      const int at = (i * 64 * S + tid) % (kTile * kN);
      in.own_B[i] = B_rows.load(at / kN, at % kN);
      if (!LOCAL) in.own_C[i] = C_rows.load(at / kN, at % kN);
    }
  };
  float total = 0.0f;
  uint64_t kept_at = reinterpret_cast<uint64_t>(kept) + ((int64_t)(t0 / kTile) * a.B + b) * a.quads * a.C * 16;
  const uint64_t kept_step = (uint64_t)a.B * a.quads * a.C * 16;
  const int kept_to = (sub * (NS / 4) * a.C + c) * 16;
  auto work = [&](Inputs& in, int t, int buffer) {           // one tile; its inputs are followed by those of kAhead tiles on
#pragma unroll
    for (int i = 0; i < kOwn; ++i) {
      const int at = (i * 64 * S + tid) % (kTile * kN);
      const bool there = at % kN < a.N && t + at / kN < live;   // neither the next group's states nor what lies behind the end
      (&low[buffer][0][0][0])[at] = there ? (float)in.own_B[i] : 0.0f;
      if (!LOCAL) (&low[buffer][LOCAL ? 0 : 1][0][0])[at] = there ? (float)in.own_C[i] : 0.0f;
    }
    if (MODE == kKeeping) {
      const States to(kept_at, a.quads, a.C, t < live);
#pragma unroll
      for (int q = 0; q < NS / 4; ++q)
        to.store_at(mine ? kept_to + q * a.C * 16 : -16, floatx4_t{h[4 * q], h[4 * q + 1], h[4 * q + 2], h[4 * q + 3]});   // (-16: nowhere)
      kept_at += kept_step;
    }
    float d[kItems], x[kItems], gate[kItems], skip[kItems];
#pragma unroll
    for (int i = 0; i < kItems; ++i) {
      const bool there = t + i * S + sub < live;
      const float v = (float)in.dt[i] + bias, ui = there ? (float)in.u[i] : 0.0f;
      float smooth = softplus(v);
      asm volatile("" : "+v"(smooth));                     // selected, not branched around
      d[i] = there ? a.softplus ? smooth : v : 0.0f;
      x[i] = d[i] * ui;
      skip[i] = D * ui;
      if (LOCAL) total += d[i];
      if (!LOCAL) {
        float g = (float)in.z[i] * sigmoid((float)in.z[i]);
        asm volatile("" : "+v"(g));
        gate[i] = gated ? g : 1.0f;
      }
    }
    __syncthreads();
    fetch(in, live - t - kAhead * kTile);
    float y[kTile];                                        // of step q; in a lane's first places of its own steps in the end
#pragma unroll
    for (int q = 0; q < kTile; ++q) {
      const float* const Bq = &low[buffer][0][q][sub * NS];
      const float* const Cq = &low[buffer][LOCAL ? 0 : 1][q][sub * NS];
      const float dq = from_owner<S>(d[q / S], q), xq = from_owner<S>(x[q / S], q);
      float sum = 0.0f;
#pragma unroll
      for (int i = 0; i < NS; ++i) {
        h[i] = __builtin_fmaf(decay(dq, A[i]), h[i], product(xq, Bq[i]));
        if (!LOCAL) sum += Cq[i] * h[i];
      }
      if (!LOCAL) {
        y[q] = S == 8 ? sum_lanes<S>(sum) : sum;
        if (S == 1) asm volatile("" : "+v"(y[q]));         // formed here, not where it is stored with all its factors alive till then
      }
    }
    if (!LOCAL && (S == 2 || S == 4)) {                    // sums over a channel's lanes, each of which keeps its own steps'
#pragma unroll
      for (int q = 0; q < kTile / 2; ++q) y[q] = halve<1>(y[2 * q], y[2 * q + 1], tid);
      if (S == 4) {
#pragma unroll
        for (int q = 0; q < kTile / 4; ++q) y[q] = halve<2>(y[2 * q], y[2 * q + 1], tid);
      }
    }
    if (!LOCAL && S == 8) {
#pragma unroll
      for (int q = 1; q < kTile; ++q) y[0] = sub == q ? y[q] : y[0];
    }
    if (!LOCAL) {
      const Tile<E> y_rows = y_at.tile(live - t, a.C);
      y_at.forth();
      if (mine) {
#pragma unroll
        for (int i = 0; i < kItems; ++i) y_rows.store(i * S + sub, c, (y[i] + skip[i]) * gate[i]);
      }
    }
  };
  // A tile takes a wavefront about as long as a load from memory when few wavefronts share a SIMD.
  Inputs ring[kAhead];
#pragma unroll
  for (int k = 0; k < kAhead; ++k) {
    fetch(ring[k], live - t0 - k * kTile);
    __builtin_amdgcn_sched_barrier(0);                     // in this order, or the loop's waits for one are waits for all
  }
  // (whole rounds of kAhead tiles, without a branch that a load in flight would have to be waited for: tiles behind the end
  // multiply the states by one and store nothing)
  for (int t = t0; t < live; t += kAhead * kTile) {
#pragma unroll
    for (int k = 0; k < kAhead; ++k) work(ring[k], t + k * kTile, k & 1);
  }
  if (!mine) return;
  if (LOCAL) {
    put_states(H, seg + 1);
    total = sum_lanes<S>(total);
    if (sub == 0) sums[((int64_t)seg * a.B + b) * a.C + c] = total;
    return;
  }
  for (int t = max(t0, end) + sub; t < t1; t += S) ys.row(t, b)[c] = (E)0.0f;
  // the segment that holds the sample's last step has its last state
  if (state_out && (end > t0 || t0 == 0) && end <= t1) {
#pragma unroll
    for (int i = 0; i < NS; ++i) {
      const int n = sub * NS + i;
      if (n < a.N) state_out[((int64_t)b * a.C + c) * a.N + n] = h[i];
    }
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
      h.v[i] = decay(d, A.v[i] * kLog2e) * h.v[i] + x * (float)Bn.v[i];
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
  a.blocks = blocks_of(s);
  const View<const E> u = tiled_view<const E>(p->u, s.T), dt = tiled_view<const E>(p->dt, s.T), z = tiled_view<const E>(p->z, s.T);
  const View<const E> B = tiled_view<const E>(p->B, s.T), C = tiled_view<const E>(p->C, s.T);
  const View<E> to = tiled_view<E>(y, s.T);
  const dim3 block(64 * S);
  if (s.segments > 1) {
    const hipError_t e = launch(scan_kernel<TYPE, NS, S, kLocal>, dim3((unsigned)(a.blocks * s.G), (unsigned)s.B, (unsigned)s.segments - 1), block, 0, stream,
                          a, u, dt, z, B, C, state_in, to, (float*)nullptr, (float*)nullptr, H, sums);
    if (e != hipSuccess) return e;
  } else {
    H = nullptr;
    a.by_length = a.lengths && s.B > 1 && s.B <= kSamplesDealt;
  }
  return launch(kept ? scan_kernel<TYPE, NS, S, kKeeping> : scan_kernel<TYPE, NS, S, kPlain>, dim3((unsigned)(a.blocks * s.G), (unsigned)s.B, (unsigned)s.segments), block, 0, stream, a, u,
                dt, z, B, C, state_in, to, state_out, kept, H, sums);
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
#define CASE(NS, S) \
  if (s.states == NS && s.lanes == S) return run_prompt<TYPE, NS, S>(a, s, p, state_in, y, state_out, kept, H, sums, stream);
  EVERY_SPLIT
#undef CASE
  return hipErrorInvalidValue;
}

int round_up(int n, int to) { return (n + to - 1) / to * to; }

}  // namespace

// How many lanes share a channel: as few as its states need (16 a lane at most), and more, down to four states a lane, while
// there are fewer wavefronts than twice the SIMDs: sharing costs a tenth more instructions, but with one lane a channel
// 8 x 2048 x 4608 with 16 states has 576 wavefronts for 1024 SIMDs (540 us, with four lanes 461).  Where that is not enough time is
// divided, which costs the local run, half of the work once more: into segments of 64 steps or more, as many as make four
// wavefronts a SIMD (six and eight: the same within 3 %, or up to a fifth longer), and only where there are four at least
// (8 x 2048 x 4608, divided in two to four: 537 to 520 us; ragged 422 to 383, undivided 290).  The backward pass's main run has one
// wavefront for 64 channels of 16 states, and with 252 registers two of them fit a SIMD: as many segments as that takes and no more
// (512 steps, 16 states, us: 576 wavefronts a segment 366 in three, 468 in two, 633 in one; 320 199 in six, 255 in three), and
// two where one would leave SIMDs idle (1536: 788 in two, 834 in one, 846 in three).  With more states a wavefront has 16 or 8
// channels, but LDS leaves a CU one or two workgroups, so that the count of 64 channels serves there as well (512 steps, 8 samples, us:
// 2304 channels of 32 states 364 in seven, 351 in five, 374 in three, 438 in one; 1152 of 128 states 871 in eight, 838 in five, 1126 in one;
// 1152 of 64 states 372 in eight, 319 in seven, 728 in one).
ScanShape scan_shape(const sprnn_scan_t* p) {
  ScanShape s{};
  s.T = p->steps; s.B = p->batch; s.C = p->channels; s.N = p->states; s.G = p->groups;
  s.per_group = s.C / s.G;
  s.quads = (s.N + 3) / 4;
  const int64_t columns = (int64_t)s.G * blocks_of(s) * s.B;      // workgroups of a segment
  s.lanes = 1;
  while (16 * s.lanes < s.N) s.lanes *= 2;
  while (s.lanes < 4 && 4 * s.lanes < s.N && columns * s.lanes < 2 * kSimds) s.lanes *= 2;
  s.states = 4;
  while (s.states * s.lanes < s.N) s.states *= 2;
  if (s.states * s.lanes < 8) s.states = 8;
  auto divide = [&](int64_t n, int least, int* segments, int* segment) {
    n = n < s.T / 64 ? n : s.T / 64;
    if (n < least) n = 1;
    *segment = round_up(s.T > 0 ? (int)((s.T + n - 1) / n) : 1, kTile);
    *segments = s.T > 0 ? (s.T + *segment - 1) / *segment : 1;
  };
  const int64_t waves = columns > 0 ? columns : kSimds;
  divide(4 * kSimds / (waves * s.lanes), 4, &s.segments, &s.segment);
  const int64_t pairs = 2 * kSimds / waves;
  divide(pairs > 2 ? pairs : 2 * waves <= 3 * kSimds ? 2 : 1, 2, &s.back_segments, &s.back_segment);
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

// (the stride between steps is limited where there are two)
static bool good_step(const sprnn_seq_t& s, int T) { return T <= 1 || s.step <= kStepMost; }
static bool good_rows(const sprnn_seq_t& s, int type, int T) { return good_view(s, type) && good_step(s, T); }
static bool good_rows(const sprnn_seq_t& s, int type, int T, int B, int width) { return good_output(s, type, T, B, width) && good_step(s, T); }

static bool good_arguments(const sprnn_scan_t* p) {
  if (!good_scan(p) || !activation_type(p->type) || (p->softplus != 0 && p->softplus != 1)) return false;
  if (!p->A || !aligned_to(p->A, 4) || !aligned_to(p->D, 4) || !aligned_to(p->dt_bias, 4) || !aligned_to(p->lengths, 4)) return false;
  if (p->steps == 0 || p->batch == 0) return true;
  auto good = [&](const sprnn_seq_t& s) { return good_rows(s, p->type, p->steps); };
  return good(p->u) && good(p->dt) && (!p->z.data || good(p->z)) && good(p->B) && good(p->C);
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
    if (!kept || !good_rows(dy, scan->type, s.T) || !good(g.u, s.C) || !good(g.dt, s.C) || !good(g.z, s.C) || !good(g.B, s.G * s.N) || !good(g.C, s.G * s.N))
      return SPRNN_ERR_INVALID;
    if (g.z.data && !scan->z.data) return SPRNN_ERR_INVALID;
  }
  const int64_t need = scan_backward_bytes(s);
  if (need > 0 && (!workspace || !aligned_to(workspace, 16) || workspace_bytes < need)) return SPRNN_ERR_INVALID;
  DeviceGuard guard(device_id);
  if (!guard.ok) return SPRNN_ERR_HIP;
  return SPRNN_HIP(launch_scan_backward(s, scan, dy, d_state_out, static_cast<const float*>(kept), gradients, static_cast<float*>(workspace),
                                        static_cast<hipStream_t>(stream)))
             ? SPRNN_OK
             : SPRNN_ERR_HIP;
}

}  // extern "C"
