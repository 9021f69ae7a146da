// Backward pass of the selective scan.  With e_t = dy_t silu(z_t) and everything behind the last step d_state_out:
//
//   g_t = a_{t+1} g_{t+1} + C_t e_t                      the adjoint of h_t: the same recurrence from the end
//   dB_t = sum_c g_t d_t u_t,   dC_t = sum_c e_t h_t      over the channels of a group
//   du_t = d_t sum_n g_t B_t + D e_t,   dd_t = u_t sum_n g_t B_t + sum_n g_t a_t h_{t-1} A,   ddt_t = dd_t softplus'(v_t)
//   dA = sum_t g_t a_t h_{t-1} d_t,   dD = sum_t e_t u_t,   dz_t = dy_t y_t silu'(z_t)
//
// h is not kept for every step: the forward pass left the states in front of every tile of kTile steps, and a tile is run
// forward again with its states and factors in registers before it is run backward.
//
// Two kinds of sums meet here, over the states of a channel and over the channels of a step.  A lane holds four states of
// R channels, S lanes share a channel: the sums over states are in the lane but for S neighbours, and the sums over channels
// are in the lane for R channels before they cross lanes.  What crosses lanes, 64 numbers a tile, is halved at every lane bit
// it crosses (each half of the lanes keeps half of the numbers), so that a lane ends with S of them, and the wavefronts of
// a workgroup meet in LDS.  Everything that depends on (step, channel) alone is done once, with one lane a channel, before
// and after the states' work, and handed over through LDS.
//
// Bound by the vector units: a state costs 13 instructions and an exponential a step, and the sums and what is done once a step
// and channel half as much again.  8 x 1024 x 2048 with 16 states in bfloat16: 240 us, the vector units busy 80 % of them with
// two wavefronts a SIMD (252 registers: 64 sums, 64 states and factors of a tile, 48 of the channels); the local run 58.
#include "sprnn_scan.h"
#include "sprnn_sums.h"

namespace sprnn {
namespace {

// A segment's effect on the adjoint, from zero behind it: like the forward pass's, from the end.  S lanes a channel share out the
// steps of a tile; the next two tiles' loads are in flight while a tile is worked through.  The S wavefronts of a workgroup have 64
// neighbouring channels, a row's 128 bytes, and nothing else in common: as workgroups, on several XCDs, they fetched twice
// the bytes.
template <int TYPE, int NS, int S>
__global__ __launch_bounds__(64 * S) void scan_adjoint_kernel(ScanArgs a, int segments, View<const Element<TYPE>> dys,
                                                          View<const Element<TYPE>> dts, View<const Element<TYPE>> zs,
                                                          View<const Element<TYPE>> Cs, const float* d_state_out, float* H, float* sums) {
  typedef Element<TYPE> E;
  constexpr int kRow = NS * S, kOwn = kTile * kRow / 64, kItems = kTile / S;
  static_assert(kTile * kRow % 64 == 0 && kTile % S == 0, "the tile's states and steps are dealt out evenly");
  __shared__ __attribute__((aligned(16))) float every_low[S][2][kTile][kRow];
  const int lane = threadIdx.x & 63, sub = lane % S;
  float (&low)[2][kTile][kRow] = every_low[threadIdx.x >> 6];
  const int group = blockIdx.x / a.blocks, block = blockIdx.x - group * a.blocks;
  const int b = blockIdx.y, seg = blockIdx.z + 1, slot = segments - 1 - seg;         // nothing asks for the effect of the first one
  const int in_group = block * 64 + (int)threadIdx.x / S;
  const bool mine = in_group < a.per_group;
  const int c = group * a.per_group + min(in_group, a.per_group - 1);
  const int t0 = seg * a.segment, t1 = min(t0 + a.segment, a.T), live = min(t1, sample_end(a.lengths, b, a.T));
  float A[NS], g[NS];
#pragma unroll
  for (int i = 0; i < NS; ++i) {
    const int n = sub * NS + i;
    A[i] = n < a.N ? a.A[(int64_t)c * a.N + n] * kLog2e : 0.0f;
    g[i] = slot == 0 && d_state_out && n < a.N ? d_state_out[((int64_t)b * a.C + c) * a.N + n] : 0.0f;
  }
  auto put_states = [&](int copy) {
    const States to(H, copy, b, a.B, a.quads, a.C);
#pragma unroll
    for (int q = 0; q < NS / 4; ++q) to.store(sub * (NS / 4) + q, c, floatx4_t{g[4 * q], g[4 * q + 1], g[4 * q + 2], g[4 * q + 3]});
  };
  if (slot == 0 && mine) put_states(0);
  const float bias = a.dt_bias ? a.dt_bias[c] : 0.0f;
  struct Inputs {
    E dy[kItems], dt[kItems], z[kItems], own[kOwn];
  };
  const int last = t0 + (live > t0 ? (live - t0 - 1) / kTile * kTile : 0);
  Cursor<const E> dy_at(dys, last, b), dt_at(dts, last, b), z_at(zs, last, b), C_at(Cs, last, b, group * a.N);
  const bool gated = zs.data != nullptr;
  auto fetch = [&](Inputs& in, int rows) {
    const Tile<const E> dy_rows = dy_at.tile(rows, a.C), dt_rows = dt_at.tile(rows, a.C), z_rows = z_at.tile(gated ? rows : 0, a.C), C_rows = C_at.tile(rows, a.N);
    dy_at.back(); dt_at.back(); z_at.back(); C_at.back();
#pragma unroll
    for (int i = 0; i < kItems; ++i) {
      in.dy[i] = dy_rows.load(i * S + sub, c);
      in.dt[i] = dt_rows.load(i * S + sub, c);
      in.z[i] = z_rows.load(i * S + sub, c);
    }
#pragma unroll
    for (int i = 0; i < kOwn; ++i) in.own[i] = C_rows.load((i * 64 + lane) / kRow, (i * 64 + lane) % kRow);
  };
  float total = 0.0f, behind = 0.0f;                       // g_t = a_{t+1} g_{t+1} + C_t e_t takes its factor from the step behind
  auto work = [&](Inputs& in, int t, int buffer) {
#pragma unroll
    for (int i = 0; i < kOwn; ++i) {
      const int at = i * 64 + lane;
      (&low[buffer][0][0])[at] = at % kRow < a.N && t + at / kRow < live ? (float)in.own[i] : 0.0f;
    }
    float d[kItems], e[kItems];
#pragma unroll
    for (int i = 0; i < kItems; ++i) {
      const bool there = t >= t0 && t + i * S + sub < live;
      const float v = (float)in.dt[i] + bias, z = (float)in.z[i];
      float smooth = softplus(v), gate = z * sigmoid(z);
      asm volatile("" : "+v"(smooth), "+v"(gate));         // selected, not branched around
      d[i] = there ? a.softplus ? smooth : v : 0.0f;
      e[i] = there ? (float)in.dy[i] * (gated ? gate : 1.0f) : 0.0f;
      total += d[i];
    }
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
    fetch(in, t - 2 * kTile >= t0 ? kTile : 0);
#pragma unroll
    for (int q = kTile - 1; q >= 0; --q) {
      const float dq = from_owner<S>(d[q / S], q), eq = from_owner<S>(e[q / S], q);
#pragma unroll
      for (int i = 0; i < NS; ++i) g[i] = __builtin_fmaf(decay(behind, A[i]), g[i], product(eq, low[buffer][q][sub * NS + i]));
      behind = dq;
    }
  };
  Inputs even, odd;                                        // in turn; a tile in front of the segment multiplies by one
  fetch(even, live - last);
  __builtin_amdgcn_sched_barrier(0);                       // in this order, or the loop's waits for one are waits for both
  fetch(odd, last > t0 ? kTile : 0);
  for (int t = last; t >= t0 && live > t0; t -= 2 * kTile) {
    work(even, t, 0);
    work(odd, t - kTile, 1);
  }
#pragma unroll
  for (int i = 0; i < NS; ++i) g[i] *= decay(behind, A[i]);
  total = sum_lanes<S>(total);
  if (!mine) return;
  put_states(slot + 1);
  if (sub == 0) sums[((int64_t)slot * a.B + b) * a.C + c] = total;
}

constexpr int kSums = kTile * 8;       // numbers of a tile and quad: [step][dB, dC][state]

// v[0 .. kSums) of every lane summed over the lanes that have the same lane % S; lane l is left with the numbers from
// l / S * S on, in v[0 .. S).
template <int S>
__device__ __forceinline__ void sum_channels(float (&v)[kSums], int lane) {
  static_assert(kSums == 64, "one number per lane at S = 1");
#pragma unroll
  for (int i = 0; i < 32; ++i) v[i] = halve<32>(v[i], v[i + 32], lane);
  if (S <= 16) {
#pragma unroll
    for (int i = 0; i < 16; ++i) v[i] = halve<16>(v[i], v[i + 16], lane);
  }
  if (S <= 8) {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = halve<8>(v[i], v[i + 8], lane);
  }
  if (S <= 4) {
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = halve<4>(v[i], v[i + 4], lane);
  }
  if (S <= 2) {
#pragma unroll
    for (int i = 0; i < 2; ++i) v[i] = halve<2>(v[i], v[i + 2], lane);
  }
  if (S <= 1) v[0] = halve<1>(v[0], v[1], lane);
}

constexpr int waves_of(int S) { return S <= 4 ? 4 : 8; }
constexpr int lane_channels(int S) { return S < 4 ? S : S == 8 ? 2 : 4; }    // R; four at S = 8 are four registers too many
constexpr int wave_channels(int S) { return 64 / S * lane_channels(S); }

// A lane's elements of one channel: steps lane / CW, lane / CW + 64 / CW, ...
template <int CW, int COUNT, typename E>
__device__ __forceinline__ void load_items(E (&v)[COUNT], const Tile<const E>& rows, int lane, int c) {
  uint32_t at = rows.offset(lane / CW, c);
#pragma unroll
  for (int i = 0; i < COUNT; ++i, at += 64 / CW * rows.step) v[i] = rows.load_at(at);
}

template <int TYPE>
struct BackViews {
  View<const Element<TYPE>> u, dt, z, B, C, dy;
  View<Element<TYPE>> du, ddt, dz;
};

// partial: [block of channels][T][B][groups][2][4 S] sums of dB and dC; totals: [segment][B][quads * C * 4 of dA, C of dD, C of d dt_bias].
template <int TYPE, int S>
__global__ __launch_bounds__(64 * waves_of(S), 2) void scan_backward_kernel(ScanArgs a, int segments, BackViews<TYPE> io, const float* kept,
                                                                            const float* carry, const float* carry_sums, const float* d_state_out, float* partial,
                                                                            float* totals, float* d_state) {
  typedef Element<TYPE> E;
  constexpr int W = waves_of(S), R = lane_channels(S), CW = wave_channels(S), CL = 64 / S;
  constexpr int kItems = kTile * CW / 64;      // (step, channel) pairs of a lane
  constexpr int kRow = 4 * S;
  constexpr bool kStartAhead = S < 32;         // a channel's first states are loaded a channel ahead; at S = 32 they are three registers too many
  // [d, later sum g B][d u, later sum through A][e, later y] of every (step, channel); B and C of the tile; sums over channels
  __shared__ float hand[W][3][kTile][CW];
  __shared__ __attribute__((aligned(16))) float low[2][kTile][2][kRow];
  __shared__ __attribute__((aligned(16))) float sums[2][W][kSums * S];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, sub = lane % S;
  const int group = blockIdx.x / a.blocks, block = blockIdx.x - group * a.blocks;
  const int b = blockIdx.y, seg = blockIdx.z;
  const int first = (block * W + wave) * CW;                 // of this wavefront, in its group
  const int t0 = seg * a.segment, t1 = min(t0 + a.segment, a.T), end = sample_end(a.lengths, b, a.T), live = min(t1, end);
  auto channel = [&](int i) { return group * a.per_group + min(first + i, a.per_group - 1); };
  auto owned = [&](int i) { return first + i < a.per_group; };

  float A[R][4], g[R][4], dA[R][4];
#pragma unroll
  for (int r = 0; r < R; ++r) {
    const int c = channel(r * CL + lane / S);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int n = sub * 4 + i;
      A[r][i] = n < a.N ? a.A[(int64_t)c * a.N + n] * kLog2e : 0.0f;
      g[r][i] = !carry && d_state_out && n < a.N ? d_state_out[((int64_t)b * a.C + c) * a.N + n] : 0.0f;
      dA[r][i] = 0.0f;
    }
    if (carry) chained_states<1>(g[r], A[r], a, carry, carry_sums, segments - 1 - seg, b, sub, c);
  }
  float dD = 0.0f, dbias = 0.0f;                             // of this lane's items, all of one channel
  const int item_channel = lane % CW, c_item = channel(item_channel);
  const float D = a.D ? a.D[c_item] : 0.0f, bias = a.dt_bias ? a.dt_bias[c_item] : 0.0f;
  auto item_step = [&](int i) { return i * (64 / CW) + lane / CW; };

  const int last = t0 + (live > t0 ? (live - t0 - 1) / kTile * kTile : 0);
  Cursor<const E> u_at(io.u, last, b), dt_at(io.dt, last, b), z_at(io.z, last, b), dy_at(io.dy, last, b);
  Cursor<E> du_at(io.du, last, b), ddt_at(io.ddt, last, b), dz_at(io.dz, last, b);
  Cursor<const E> B_at(io.B, last, b, group * a.N), C_at(io.C, last, b, group * a.N);
  const bool gated = io.z.data != nullptr;
  // Items and rows of B and C are loaded a tile ahead, behind the states' work (whose registers they take), and this tile's
  // items again at the same place: their latency passes under the sums.  No load stands under a branch: it would be waited for.
  struct Items {
    E u[kItems], dt[kItems], z[kItems], dy[kItems];
  };
  auto fetch_items = [&](Items& to, int rows) {
    load_items<CW>(to.u, u_at.template tile<true>(rows, a.C), lane, c_item);
    load_items<CW>(to.dt, dt_at.template tile<true>(rows, a.C), lane, c_item);
    load_items<CW>(to.z, z_at.template tile<true>(gated ? rows : 0, a.C), lane, c_item);
    load_items<CW>(to.dy, dy_at.template tile<true>(rows, a.C), lane, c_item);
  };
  constexpr int kLow = (kTile * kRow + 64 * W - 1) / (64 * W);
  E B_next[kLow], C_next[kLow];
  auto low_item = [&](int i) { return min((int)threadIdx.x + i * 64 * W, kTile * kRow - 1); };   // (several lanes may have the last)
  auto fetch_low = [&](int rows) {
    const Tile<const E> B_rows = B_at.template tile<true>(rows, a.N), C_rows = C_at.template tile<true>(rows, a.N);
    B_at.back(); C_at.back();
#pragma unroll
    for (int i = 0; i < kLow; ++i) {
      B_next[i] = B_rows.load(low_item(i) / kRow, low_item(i) % kRow);
      C_next[i] = C_rows.load(low_item(i) / kRow, low_item(i) % kRow);
    }
  };
  Items next;
  fetch_items(next, live - last);
  fetch_low(live - last);
  int buffer = 0;
  for (int t = last; t >= t0 && live > t0; t -= kTile, buffer ^= 1) {
    // what depends on (step, channel) alone
    {
      int rows = live - t;                                   // (asked anew for every item: eight kept answers are 16 scalar registers)
#pragma unroll
      for (int i = 0; i < kItems; ++i) {
        const int q = item_step(i);
        asm volatile("" : "+v"(rows));
        const bool in = q < rows, counts = in && owned(item_channel);   // else a copy of the group's last channel
        const float v = (float)next.dt[i] + bias, z = (float)next.z[i];
        float smooth = softplus(v), gate = z * sigmoid(z);
        asm volatile("" : "+v"(smooth), "+v"(gate));         // selected below, not branched around
        const float d = in ? a.softplus ? smooth : v : 0.0f;
        hand[wave][0][q][item_channel] = d;
        hand[wave][1][q][item_channel] = counts ? d * (float)next.u[i] : 0.0f;
        hand[wave][2][q][item_channel] = counts ? (float)next.dy[i] * (gated ? gate : 1.0f) : 0.0f;
      }
#pragma unroll
      for (int i = 0; i < kLow; ++i) {
        const int n = low_item(i) % kRow, q = low_item(i) / kRow;
        const bool in = n < a.N && t + q < live;
        low[buffer][q][0][n] = in ? (float)B_next[i] : 0.0f;
        low[buffer][q][1][n] = in ? (float)C_next[i] : 0.0f;
      }
    }
    const States in_front(kept, t / kTile, b, a.B, a.quads, a.C);
    floatx4_t starts[2];
    starts[0] = in_front.load(sub, channel(lane / S));
    __syncthreads();

    float acc[kSums];
#pragma unroll
    for (int i = 0; i < kSums; ++i) acc[i] = 0.0f;
#pragma unroll
    for (int r = 0; r < R; ++r) {
      __builtin_amdgcn_sched_barrier(0);                     // channels one after the other: their registers are the same
      const int own = r * CL + lane / S;
      if (!kStartAhead && r > 0) starts[r % 2] = in_front.load(sub, channel(own));
      const floatx4_t start = starts[r % 2];
      if (kStartAhead && r + 1 < R) starts[(r + 1) % 2] = in_front.load(sub, channel(own + CL));
      float h[kTile][4], f[kTile][4];
      // What is in LDS is read again for every channel and direction (through offsets that the compiler knows nothing
      // about): kept in registers for the whole tile it is 80 too many.
      int at = sub * 4, back = own;
      asm volatile("" : "+v"(at), "+v"(back));
#pragma unroll
      for (int q = 0; q < kTile; ++q) {
        const float d = hand[wave][0][q][own], x = hand[wave][1][q][own];
        const floatx4_t Bq = *reinterpret_cast<const floatx4_t*>(&low[buffer][q][0][at]);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          f[q][i] = decay(d, A[r][i]);
          h[q][i] = f[q][i] * (q ? h[q ? q - 1 : 0][i] : start[i]) + x * Bq[i];
        }
      }
#pragma unroll
      for (int q = kTile - 1; q >= 0; --q) {
        if (q % 2) {
          __builtin_amdgcn_sched_barrier(0);
          asm volatile("" : "+v"(at));
        }
        const float e = hand[wave][2][q][back], dq = hand[wave][0][q][back], xq = hand[wave][1][q][back];
        const floatx4_t Bq = *reinterpret_cast<const floatx4_t*>(&low[buffer][q][0][at]);
        const floatx4_t Cq = *reinterpret_cast<const floatx4_t*>(&low[buffer][q][1][at]);
        float gB = 0.0f, through = 0.0f, y = 0.0f;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          g[r][i] += Cq[i] * e;
          acc[q * 8 + i] += g[r][i] * xq;
          acc[q * 8 + 4 + i] += h[q][i] * e;
          gB += g[r][i] * Bq[i];
          y += Cq[i] * h[q][i];
          g[r][i] *= f[q][i];
          const float p = g[r][i] * (q ? h[q ? q - 1 : 0][i] : start[i]);
          through += p * A[r][i];
          dA[r][i] += p * dq;
        }
        // The sums are formed here: left to the end of the tile, where they are used, they keep all their factors alive.
#pragma unroll
        for (int i = 0; i < 8; ++i) asm volatile("" : "+v"(acc[q * 8 + i]));
#pragma unroll
        for (int i = 0; i < 4; ++i) asm volatile("" : "+v"(dA[r][i]));
        gB = sum_lanes<S>(gB);
        through = sum_lanes<S>(through);
        y = sum_lanes<S>(y);
        hand[wave][0][q][own] = gB;                          // by all S lanes, which hold the same
        hand[wave][1][q][own] = through;
        hand[wave][2][q][own] = y;
      }
    }
    __builtin_amdgcn_sched_barrier(0);
    Items own;
    fetch_items(own, live - t);
    u_at.back(); dt_at.back(); z_at.back(); dy_at.back();
    fetch_items(next, t > t0 ? kTile : 0);
    fetch_low(t > t0 ? kTile : 0);
    __builtin_amdgcn_sched_barrier(0);
    sum_channels<S>(acc, lane);
#pragma unroll
    for (int i = 0; i < S; ++i) {
      const int v = lane / S * S + i;                        // [step][dB, dC][state of the quad]
      sums[buffer][wave][(v >> 2) * kRow + sub * 4 + (v & 3)] = acc[i];
    }
    __syncthreads();
    for (int i = threadIdx.x; i < kTile * 2 * kRow; i += 64 * W) {
      float sum = sums[buffer][0][i];
#pragma unroll
      for (int w = 1; w < W; ++w) sum += sums[buffer][w][i];
      const int q = i / (2 * kRow);
      if (t + q < live) partial[((((int64_t)block * a.T + t + q) * a.B + b) * a.G + group) * (2 * kRow) + i % (2 * kRow)] = sum;
    }
    // gradients of what depends on (step, channel) alone
    const Tile<E> du_rows = du_at.template tile<true>(io.du.data ? live - t : 0, a.C), ddt_rows = ddt_at.template tile<true>(io.ddt.data ? live - t : 0, a.C), dz_rows = dz_at.template tile<true>(io.dz.data ? live - t : 0, a.C);
    du_at.back(); ddt_at.back(); dz_at.back();
    if (owned(item_channel)) {
      int rows = live - t;
      uint32_t du_to = du_rows.offset(lane / CW, c_item), ddt_to = ddt_rows.offset(lane / CW, c_item), dz_to = dz_rows.offset(lane / CW, c_item);
#pragma unroll
      for (int i = 0; i < kItems; ++i, du_to += 64 / CW * du_rows.step, ddt_to += 64 / CW * ddt_rows.step, dz_to += 64 / CW * dz_rows.step) {
        const int q = item_step(i);
        asm volatile("" : "+v"(rows));
        const float gB = hand[wave][0][q][item_channel], through = hand[wave][1][q][item_channel] * kLn2, sum = hand[wave][2][q][item_channel];
        const bool in = q < rows;
        const float u = in ? (float)own.u[i] : 0.0f, v = (float)own.dt[i] + bias;
        float smooth = softplus(v), slope = sigmoid(v);
        const float z = (float)own.z[i], s = sigmoid(z), dy = in ? (float)own.dy[i] : 0.0f;
        asm volatile("" : "+v"(smooth), "+v"(slope));        // selected, not branched around
        const float d = a.softplus ? smooth : v;
        dz_rows.store_at(dz_to, dy * (sum + D * u) * (s * (1.0f + z * (1.0f - s))));
        const float e = !gated ? dy : in ? dy * (z * s) : 0.0f;
        du_rows.store_at(du_to, d * gB + D * e);
        const float dv = (u * gB + through) * (a.softplus ? slope : 1.0f);
        ddt_rows.store_at(ddt_to, dv);
        dD += e * u;
        dbias += in ? dv : 0.0f;
      }
    }
  }
  // behind a sample's end
  for (int t = max(t0, end) + lane / CW; t < t1; t += 64 / CW) {
    if (!owned(item_channel)) break;
    if (io.du.data) io.du.row(t, b)[c_item] = (E)0.0f;
    if (io.ddt.data) io.ddt.row(t, b)[c_item] = (E)0.0f;
    if (io.dz.data) io.dz.row(t, b)[c_item] = (E)0.0f;
  }
  const int64_t width = (int64_t)a.quads * a.C * 4 + 2 * (int64_t)a.C;
  float* const mine = totals + ((int64_t)seg * a.B + b) * width;
#pragma unroll
  for (int r = 0; r < R; ++r) {
    const int own = r * CL + lane / S, c = channel(own);
    if (!owned(own) || sub >= a.quads) continue;
    Pack<float, 4> p;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      p.v[i] = dA[r][i];
      if (d_state && seg == 0 && sub * 4 + i < a.N) d_state[((int64_t)b * a.C + c) * a.N + sub * 4 + i] = g[r][i];
    }
    store_pack(mine + ((int64_t)sub * a.C + c) * 4, p);
  }
#pragma unroll
  for (int bit = CW; bit < 64; bit *= 2) {
    dD += __shfl_xor(dD, bit);
    dbias += __shfl_xor(dbias, bit);
  }
  if (lane < CW && owned(item_channel)) {
    mine[(int64_t)a.quads * a.C * 4 + c_item] = dD;
    mine[(int64_t)a.quads * a.C * 4 + a.C + c_item] = dbias;
  }
}

// dB and dC from the sums of the blocks of channels: one lane per (step, sample, group, dB or dC, state) at a time (a launch has
// fewer than 2^32 lanes).
constexpr int64_t kLowGroups = 1 << 20;
template <int TYPE>
__global__ __launch_bounds__(256) void scan_low_gradients_kernel(ScanArgs a, int row, const float* partial, View<Element<TYPE>> dB,
                                                                 View<Element<TYPE>> dC) {
  const int64_t width = (int64_t)a.G * 2 * row, all = (int64_t)a.T * a.B * width;
  for (int64_t at = (int64_t)blockIdx.x * 256 + threadIdx.x; at < all; at += (int64_t)gridDim.x * 256) {
    const int n = (int)(at % row), which = (int)(at / row % 2), group = (int)(at / (2 * row) % a.G);
    const int64_t vector = at / width;
    const int t = (int)(vector / a.B), b = (int)(vector % a.B);
    const View<Element<TYPE>> out = which ? dC : dB;
    if (n >= a.N || !out.data) continue;
    float sum = 0.0f;
    if (t < sample_end(a.lengths, b, a.T))
      for (int k = 0; k < a.blocks; ++k) sum += partial[k * all + at];
    out.row(t, b)[(int64_t)group * a.N + n] = (Element<TYPE>)sum;
  }
}

// Sums [quads][C][4], [C], [C] to dA [C][N], dD and d dt_bias [C].
struct PutParameters {
  float* dA;
  float* dD;
  float* dbias;
  int C, N;
  int64_t states;                      // quads * C * 4
  __device__ void operator()(int64_t i, float sum) const {
    if (i < states) {
      const int c = (int)(i / 4 % C), n = (int)(i / 4 / C) * 4 + (int)(i & 3);
      if (dA && n < N) dA[(int64_t)c * N + n] = sum;
    } else if (i < states + C) {
      if (dD) dD[i - states] = sum;
    } else if (dbias) {
      dbias[i - states - C] = sum;
    }
  }
};

int lanes_of(int quads) {
  int S = 1;
  while (S < quads) S *= 2;
  return S;
}
int blocks_of(const ScanShape& s, int S) {
  const int channels = waves_of(S) * wave_channels(S);
  return (s.per_group + channels - 1) / channels;
}

struct Workspace {   // in floats
  int64_t carry, sums, partial, totals, all;
};
Workspace layout(const ScanShape& s) {
  const int S = lanes_of(s.quads);
  Workspace w{};
  int64_t at = 0;
  auto take = [&](int64_t floats) { const int64_t from = at; at += (floats + 3) / 4 * 4; return from; };
  const int64_t width = (int64_t)s.quads * s.C * 4 + 2 * (int64_t)s.C;
  w.carry = take(s.back_segments > 1 ? s.back_segments * s.state_floats() : 0);
  w.sums = take(s.back_segments > 1 ? (int64_t)s.back_segments * s.B * s.C : 0);
  w.partial = take((int64_t)blocks_of(s, S) * s.T * s.B * s.G * 8 * S);
  w.totals = take(s.back_segments * s.B * width);
  w.all = at;
  return w;
}

template <int TYPE, int NS, int SA, int S>
hipError_t run(const ScanShape& s, const sprnn_scan_t* p, const sprnn_seq_t& dy, const float* d_state_out, const float* kept,
               const sprnn_scan_gradients_t* out, float* workspace, hipStream_t stream) {
  typedef Element<TYPE> E;
  const Workspace w = layout(s);
  const int64_t width = (int64_t)s.quads * s.C * 4 + 2 * (int64_t)s.C;
  ScanArgs a = scan_arguments(p, s);
  a.segment = s.back_segment;
  auto in = [&](const sprnn_seq_t& v) { return tiled_view<const E>(v, s.T); };
  auto to = [&](const sprnn_seq_t& v) { return tiled_view<E>(v, s.T); };
  BackViews<TYPE> io{in(p->u), in(p->dt), in(p->z), in(p->B), in(p->C), in(dy), to(out->u), to(out->dt), to(out->z)};
  const float* carry = nullptr;
  hipError_t e = hipSuccess;
  if (s.B > 0) {
    if (s.back_segments > 1) {
      a.blocks = (s.per_group + 63) / 64;
      e = launch(scan_adjoint_kernel<TYPE, NS, SA>, dim3((unsigned)(a.blocks * s.G), (unsigned)s.B, (unsigned)s.back_segments - 1), dim3(64 * SA), 0, stream, a,
                 s.back_segments, io.dy, io.dt, io.z, io.C, d_state_out, workspace + w.carry, workspace + w.sums);
      if (e != hipSuccess) return e;
      carry = workspace + w.carry;
    }
    a.blocks = blocks_of(s, S);
    e = launch(scan_backward_kernel<TYPE, S>, dim3((unsigned)(a.blocks * s.G), (unsigned)s.B, (unsigned)s.back_segments), dim3(64 * waves_of(S)), 0, stream, a,
               s.back_segments, io, kept, carry, (const float*)(workspace + w.sums), d_state_out, workspace + w.partial, workspace + w.totals, out->state);
    if (e != hipSuccess) return e;
    const int64_t lows = (int64_t)s.T * s.B * s.G * 8 * S;
    if (lows > 0 && (out->B.data || out->C.data)) {
      e = launch(scan_low_gradients_kernel<TYPE>, dim3((unsigned)(lows < 256 * kLowGroups ? (lows + 255) / 256 : kLowGroups)), dim3(256), 0, stream, a, 4 * S,
                 (const float*)(workspace + w.partial), view<E>(out->B), view<E>(out->C));
      if (e != hipSuccess) return e;
    }
  }
  if (!out->A && !out->D && !out->dt_bias) return hipSuccess;
  return launch_sum_partials(workspace + w.totals, s.back_segments * s.B, width,
                             PutParameters{out->A, out->D, out->dt_bias, s.C, s.N, (int64_t)s.quads * s.C * 4}, stream);
}

template <int TYPE>
hipError_t run_backward(const ScanShape& s, const sprnn_scan_t* p, const sprnn_seq_t& dy, const float* d_state_out, const float* kept,
                        const sprnn_scan_gradients_t* out, float* workspace, hipStream_t stream) {
  return s.N <= 4 ? run<TYPE, 4, 2, 1>(s, p, dy, d_state_out, kept, out, workspace, stream)
       : s.N <= 8 ? run<TYPE, 4, 2, 2>(s, p, dy, d_state_out, kept, out, workspace, stream)
       : s.N <= 16 ? run<TYPE, 4, 4, 4>(s, p, dy, d_state_out, kept, out, workspace, stream)
       : s.N <= 32 ? run<TYPE, 8, 4, 8>(s, p, dy, d_state_out, kept, out, workspace, stream)
       : s.N <= 64 ? run<TYPE, 16, 4, 16>(s, p, dy, d_state_out, kept, out, workspace, stream)
                   : run<TYPE, 16, 8, 32>(s, p, dy, d_state_out, kept, out, workspace, stream);
}

}  // namespace

int64_t scan_backward_bytes(const ScanShape& s) { return layout(s).all * 4; }

hipError_t launch_scan_backward(const ScanShape& s, const sprnn_scan_t* p, const sprnn_seq_t& dy, const float* d_state_out, const float* kept,
                                const sprnn_scan_gradients_t* out, float* workspace, hipStream_t stream) {
  return p->type == SPRNN_TYPE_F32 ? run_backward<SPRNN_TYPE_F32>(s, p, dy, d_state_out, kept, out, workspace, stream)
       : p->type == SPRNN_TYPE_F16 ? run_backward<SPRNN_TYPE_F16>(s, p, dy, d_state_out, kept, out, workspace, stream)
                                   : run_backward<SPRNN_TYPE_BF16>(s, p, dy, d_state_out, kept, out, workspace, stream);
}

}  // namespace sprnn
