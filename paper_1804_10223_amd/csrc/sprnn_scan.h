// Selective scan: what its forward and backward kernels share.
//
//   d_t = softplus(dt_t + dt_bias),  a_t = exp(d_t A),  h_t = a_t h_{t-1} + d_t u_t B_t,  y_t = (C_t h_t + D u_t) silu(z_t)
//
// A state costs one exponential and four multiply-adds a step, and the vector units set the pace: 8 cycles of a SIMD for
// the exponential of a wavefront, 4 for each of the others, 24 where memory would allow 6 (16 states, 16 bits).  So states live in registers, everything that depends on (step,
// channel) alone is done once for all states of a channel, and steps are independent only through the state: where the
// samples and channels are too few to fill the chip, time is divided into segments.  Segments but the last are run once from
// a zero state for their effect (end state, sum of d: the product of all a of a state is exp(A sum d)), and a second run chains
// these and starts every segment from its true state.
#ifndef SPRNN_SCAN_H_
#define SPRNN_SCAN_H_

#include "sprnn_seq.h"

namespace sprnn {

typedef float floatx4_t __attribute__((ext_vector_type(4)));

constexpr int kTile = 8;               // steps fetched together; the backward pass reads the state in front of every tile
constexpr int kStatesMost = 128;
constexpr int kSimds = 1024;           // of the chip: 256 CUs of four

// How a scan is laid out: `quads` groups of four states (the last may be partial), states in memory of this library's own
// [..][quad][C][4], so that neighbouring channels are neighbouring 16 bytes.
struct ScanShape {
  int T, B, C, N, G;
  int per_group;                       // channels that share B and C
  int quads;
  int states, lanes;                   // of the forward pass: states that a lane holds, lanes that share a channel
  int segments, segment;               // segments of time and their steps (a multiple of kTile)
  int back_segments, back_segment;     // ... of the backward pass
  int64_t state_floats() const { return (int64_t)B * quads * C * 4; }
};
ScanShape scan_shape(const sprnn_scan_t* p);

struct ScanArgs {
  int T, B, C, N, G, per_group, blocks, quads, softplus;   // blocks: wavefronts per group of channels
  int by_length;                       // workgroups are dealt out by their samples' lengths
  int segment;
  const float* A;
  const float* D;
  const float* dt_bias;
  const int32_t* lengths;
};
inline ScanArgs scan_arguments(const sprnn_scan_t* p, const ScanShape& s) {
  return ScanArgs{s.T, s.B, s.C, s.N, s.G, s.per_group, 0, s.quads, p->softplus, 0, s.segment, p->A, p->D, p->dt_bias, p->lengths};
}
bool good_scan(const sprnn_scan_t* p);

// The rows t .. t + kTile - 1 of one sample as a buffer: an element is found by a 32-bit offset, loads of rows that are not
// there give zeros and stores to them nothing, both without a branch.  (Rows of an input may lie closer than they are long;
// then what is read of a row that is not there is some element of another: callers do not use it.)
constexpr int64_t kStepMost = (int64_t)1 << 25;   // elements between two steps: eight rows stay below 2^31 bytes
// A sequence of one step may have any stride between steps: in the tiles' kernels it has the longest one, which keeps the rows
// that are not there out of the range of the one that is.
template <typename E>
inline View<E> tiled_view(const sprnn_seq_t& s, int T) { return View<E>{static_cast<E*>(s.data), T > 1 ? s.step : kStepMost, s.sample}; }
template <typename E>
struct Tile {
  __amdgpu_buffer_rsrc_t buffer;
  uint32_t step;                       // bytes between rows
  typedef typename std::remove_const<E>::type V;
  __device__ __forceinline__ uint32_t offset(uint32_t row, uint32_t i) const { return row * step + i * (uint32_t)sizeof(E); }
  __device__ __forceinline__ V load(uint32_t row, uint32_t i) const { return load_at(offset(row, i)); }
  __device__ __forceinline__ void store(uint32_t row, uint32_t i, float f) const { store_at(offset(row, i), f); }
  __device__ __forceinline__ V load_at(uint32_t byte) const {
    const int at = (int)byte;
    if constexpr (sizeof(E) == 4) return __builtin_bit_cast(V, __builtin_amdgcn_raw_buffer_load_b32(buffer, at, 0, 0));
    else return __builtin_bit_cast(V, (uint16_t)__builtin_amdgcn_raw_buffer_load_b16(buffer, at, 0, 0));
  }
  __device__ __forceinline__ void store_at(uint32_t byte, float f) const {
    const int at = (int)byte;
    const V v = (V)f;
    if constexpr (sizeof(E) == 4) __builtin_amdgcn_raw_buffer_store_b32(__builtin_bit_cast(uint32_t, v), buffer, at, 0, 0);
    else __builtin_amdgcn_raw_buffer_store_b16(__builtin_bit_cast(uint16_t, v), buffer, at, 0, 0);
  }
};
// One sample's rows, tile by tile: all that a tile needs is an address, a stride and how many rows there are.
template <typename E>
struct Cursor {
  uint64_t base;
  uint32_t step;                       // bytes between rows
  __device__ __forceinline__ Cursor(const View<E>& v, int t, int b, int offset = 0)
      : base(reinterpret_cast<uint64_t>(v.data + ((int64_t)t * v.step + (int64_t)b * v.sample + offset))), step((uint32_t)v.step * (uint32_t)sizeof(E)) {}
  // (rows: 0 where there is no tensor.  FRESH: the compiler is to form offsets where they are used; kept for eight rows of
  // seven tensors they fill the registers that the states of the backward pass are in.)
  template <bool FRESH = false>
  __device__ __forceinline__ Tile<E> tile(int rows, int width) const {
    rows = min(rows, kTile);
    uint32_t own_step = step;
    if (FRESH) asm volatile("" : "+s"(own_step));
    const uint32_t bytes = rows > 0 ? (uint32_t)(rows - 1) * own_step + (uint32_t)width * (uint32_t)sizeof(E) : 0u;
    const uint64_t lo = (uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)base), hi = (uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)(base >> 32));
    return Tile<E>{__builtin_amdgcn_make_buffer_rsrc(reinterpret_cast<void*>(lo | hi << 32), 0, __builtin_amdgcn_readfirstlane((int)bytes), 0x00020000), own_step};
  }
  __device__ __forceinline__ void forth() { base += (uint32_t)kTile * step; }    // (below 2^30)
  __device__ __forceinline__ void back() { base -= (uint32_t)kTile * step; }
};
// One sample's states in this library's own layout, [quad][C][4]: an element's offset stays below 2^31 bytes.
constexpr int kChannelsMost = 1 << 20;
struct States {
  __amdgpu_buffer_rsrc_t buffer;
  int channels;
  __device__ __forceinline__ States(const float* base, int64_t copy, int b, int batch, int quads, int channels) : channels(channels) {
    const uint64_t at = reinterpret_cast<uint64_t>(base + (copy * batch + b) * quads * channels * 4);
    const uint64_t lo = (uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)at), hi = (uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)(at >> 32));
    buffer = __builtin_amdgcn_make_buffer_rsrc(reinterpret_cast<void*>(lo | hi << 32), 0, base ? quads * channels * 16 : 0, 0x00020000);
  }
  // the copy at an address, or none
  __device__ __forceinline__ States(uint64_t at, int quads, int channels, bool there) : channels(channels) {
    const uint64_t lo = (uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)at), hi = (uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)(at >> 32));
    buffer = __builtin_amdgcn_make_buffer_rsrc(reinterpret_cast<void*>(lo | hi << 32), 0, there ? quads * channels * 16 : 0, 0x00020000);
  }
  __device__ __forceinline__ floatx4_t load(int quad, int c) const {          // zeros behind the last quad
    return __builtin_bit_cast(floatx4_t, __builtin_amdgcn_raw_buffer_load_b128(buffer, (quad * channels + c) * 16, 0, 0));
  }
  __device__ __forceinline__ void store(int quad, int c, const floatx4_t& v) const { store_at((quad * channels + c) * 16, v); }
  __device__ __forceinline__ void store_at(int byte, const floatx4_t& v) const {
    typedef uint32_t words __attribute__((ext_vector_type(4)));
    __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(words, v), buffer, byte, 0, 0);
  }
};

// d from v = dt + dt_bias: max(v, 0) + log1p(exp(-|v|)).  exp's argument v log2(e) and the sum 1 + e are rounded, which would
// cost small steps (v far below 0) their last digits; what the roundings took is added to the results again (to log1p
// undivided by 1 + e: off by less than e 2^-24).  exp(-128) is 0 in binary32, so |v| is bounded there: beyond 2.36e38 v log2(e)
// would be infinite and the correction NaN, where a step that is masked by the type's lowest value or -infinity has d = 0.
// (A maximum that hands NaN on: d of NaN is NaN.)
__device__ __forceinline__ float softplus(float v) {
  const float m = __builtin_elementwise_maximum(-__builtin_fabsf(v), -128.0f);
  const float hi = m * kLog2e, lo = __builtin_fmaf(m, kLog2e, -hi);
  float e = exp2_fast(hi);
  e = __builtin_fmaf(e, lo * kLn2, e);
  const float s = 1.0f + e;
  return fmaxf(v, 0.0f) + __builtin_fmaf(__builtin_amdgcn_logf(s), kLn2, e - (s - 1.0f));
}

// a = exp(d A), with A times log2(e) at hand.  v_exp_f32 is 0.11 x 2^-24 low on average for results just below 1 (measured
// over arguments from -1e-2 on; 0.31 x 2^-24 in the root mean square), and a slow state multiplies by a thousand such results
// in a row: 7e-6 of its value.  The argument is raised by as much, which costs nothing in a multiply-add, leaves exp(0) at 1
// and is below half a step of arguments that matter less.
constexpr float kRaise = 1.0e-8f;
__device__ __forceinline__ float decay(float d, float A) { return exp2_fast(__builtin_fmaf(d, A, kRaise)); }

// x y rounded: a product of its own can take x from another lane's register, a multiply-add can not.
__device__ __forceinline__ float product(float x, float y) {
#pragma clang fp contract(off)
  return x * y;
}

// Step q's value out of S neighbouring lanes, of which lane q % S holds it.
template <int S>
__device__ __forceinline__ float from_owner(float v, int q) {
  const int bits = __builtin_bit_cast(int, v);
  if constexpr (S == 1) return v;
  else if constexpr (S == 2)
    return __builtin_bit_cast(float, q % 2 ? __builtin_amdgcn_mov_dpp(bits, 0xf5, 0xf, 0xf, true) : __builtin_amdgcn_mov_dpp(bits, 0xa0, 0xf, 0xf, true));
  else if constexpr (S == 4)
    return __builtin_bit_cast(float, q % 4 == 0   ? __builtin_amdgcn_mov_dpp(bits, 0x00, 0xf, 0xf, true)
                                     : q % 4 == 1 ? __builtin_amdgcn_mov_dpp(bits, 0x55, 0xf, 0xf, true)
                                     : q % 4 == 2 ? __builtin_amdgcn_mov_dpp(bits, 0xaa, 0xf, 0xf, true)
                                                  : __builtin_amdgcn_mov_dpp(bits, 0xff, 0xf, 0xf, true));
  else return __shfl(v, ((threadIdx.x & 63) & ~(S - 1)) | (q % S));
}

// (p, q): lanes without `BIT` get the sum of p over the two lanes that differ in BIT, the others that of q.
template <int BIT>
__device__ __forceinline__ float halve(float p, float q, int lane) {
  if (BIT == 32 || BIT == 16) {
    const uint32_t up = __builtin_bit_cast(uint32_t, p), uq = __builtin_bit_cast(uint32_t, q);
    const auto r = BIT == 32 ? __builtin_amdgcn_permlane32_swap(up, uq, false, false) : __builtin_amdgcn_permlane16_swap(up, uq, false, false);
    const uint32_t r0 = r[0], r1 = r[1];
    return __builtin_bit_cast(float, r0) + __builtin_bit_cast(float, r1);
  }
  const bool upper = lane & BIT;
  const float keep = upper ? q : p, give = upper ? p : q;
  const int bits = __builtin_bit_cast(int, give);
  if (BIT == 4) {   // from four lanes up in the lower halves of eight lanes, from four lanes down in the upper ones
    const float up = __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, bits, 0x104, 0xf, 0x5, false));
    const float down = __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, bits, 0x114, 0xf, 0xa, false));
    return (keep + up) + down;
  }
  constexpr int kCtrl = BIT == 8 ? 0x128 : BIT == 2 ? 0x4e : 0xb1;   // row_ror 8, quad_perm 2 3 0 1, quad_perm 1 0 3 2
  return keep + __builtin_bit_cast(float, __builtin_amdgcn_mov_dpp(bits, kCtrl, 0xf, 0xf, true));
}

// The state in front of segment `seg` (of the adjoint: of the seg-th from the end).  The local runs left in H[0] the state in
// front of the first segment, in H[1] the one behind it, and behind every other segment k what it makes of zero, H[k + 1], with
// the sum of its d, sums[k]: h = exp(A sums[k]) h + H[k + 1] from there on.  Every workgroup of the second run does this for
// itself, with four segments in flight: a launch in between took 8 us at 27 segments (1 x 4096 x 2304, 16 states).
template <int Q>
__device__ __forceinline__ void chained_states(float (&h)[4 * Q], const float (&A)[4 * Q], const ScanArgs& a, const float* H, const float* sums,
                                               int seg, int b, int quad, int c) {
  constexpr int kAhead = 4;
  const States front(H, min(seg, 1), b, a.B, a.quads, a.C);
#pragma unroll
  for (int q = 0; q < Q; ++q) {
    const floatx4_t p = front.load(quad + q, c);
#pragma unroll
    for (int i = 0; i < 4; ++i) h[4 * q + i] = p[i];
  }
  for (int s = 1; s < seg; s += kAhead) {
    floatx4_t p[kAhead][Q];
    float total[kAhead];
#pragma unroll
    for (int k = 0; k < kAhead; ++k) {
      const int from = min(s + k, seg - 1);
      const States behind(H, from + 1, b, a.B, a.quads, a.C);
#pragma unroll
      for (int q = 0; q < Q; ++q) p[k][q] = behind.load(quad + q, c);
      total[k] = sums[((int64_t)from * a.B + b) * a.C + c];
    }
#pragma unroll
    for (int k = 0; k < kAhead; ++k) {
      if (s + k >= seg) break;
#pragma unroll
      for (int i = 0; i < 4 * Q; ++i) h[i] = __builtin_fmaf(exp2_fast(A[i] * total[k]), h[i], p[k][i / 4][i % 4]);
    }
  }
}

int64_t scan_backward_bytes(const ScanShape& s);
hipError_t launch_scan_backward(const ScanShape& s, const sprnn_scan_t* p, const sprnn_seq_t& dy, const float* d_state_out, const float* kept,
                                const sprnn_scan_gradients_t* out, float* workspace, hipStream_t stream);

}  // namespace sprnn
#endif
