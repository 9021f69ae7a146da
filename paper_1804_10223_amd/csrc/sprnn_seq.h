// Shared by the operators on sequences [T][B][H] that need no handle (scan, convolution, norm, 8-bit projection): views,
// element types, lane exchanges, and the checks that their C entry points make.
#ifndef SPRNN_SEQ_H_
#define SPRNN_SEQ_H_

#include <hip/hip_runtime.h>

#include <cstdint>
#include <type_traits>

#include "sprnn.h"
#include "sprnn_guard.h"

namespace sprnn {

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;

// ---- element types.  v_cvt_pk_bf16_f32 and v_cvt_f16_f32 round to nearest even.
template <int TYPE> struct ElementOf;
template <> struct ElementOf<SPRNN_TYPE_F32> { typedef float type; };
template <> struct ElementOf<SPRNN_TYPE_F16> { typedef _Float16 type; };
template <> struct ElementOf<SPRNN_TYPE_BF16> { typedef __bf16 type; };
template <int TYPE> using Element = typename ElementOf<TYPE>::type;

// V elements from an address that is aligned to an element only (the memory pipeline takes any).
template <typename E, int V>
struct Pack {
  E v[V];
};
template <int V, typename E>
__device__ __forceinline__ Pack<E, V> load_pack(const E* at) {
  Pack<E, V> p;
  __builtin_memcpy(&p, at, sizeof(p));
  return p;
}
// the first `n` of V elements, zeros behind them
template <int V, typename E>
__device__ __forceinline__ Pack<E, V> load_part(const E* at, int n) {
  Pack<E, V> p;
#pragma unroll
  for (int i = 0; i < V; ++i) p.v[i] = i < n ? at[i] : (E)0.0f;
  return p;
}
template <int V, typename E>
__device__ __forceinline__ void store_pack(E* at, const Pack<E, V>& p) { __builtin_memcpy(at, &p, sizeof(p)); }
template <int V, typename E>
__device__ __forceinline__ void store_part(E* at, const Pack<E, V>& p, int n) {
#pragma unroll
  for (int i = 0; i < V; ++i)
    if (i < n) at[i] = p.v[i];
}

// A view's row (t, b).
template <typename E>
struct View {
  E* data;
  int64_t step, sample;
  __device__ __forceinline__ E* row(int64_t t, int64_t b) const { return data + t * step + b * sample; }
};
template <typename E>
inline View<E> view(const sprnn_seq_t& s) { return View<E>{static_cast<E*>(s.data), s.step, s.sample}; }

__device__ __forceinline__ float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }     // 1 unit in the last place
// Both ends are exact: exp2 gives infinity or 0 there, and 1 / infinity is 0.
__device__ __forceinline__ float sigmoid(float x) { return __builtin_amdgcn_rcpf(1.0f + exp2_fast(-kLog2e * x)); }

__device__ __forceinline__ int sample_end(const int32_t* lengths, int b, int T) {
  if (!lengths) return T;
  const int n = lengths[b];
  return n < 0 ? 0 : n < T ? n : T;
}

// ---- sums over neighbouring lanes (every lane of 2^k neighbours gets their sum)
template <int CTRL>
__device__ __forceinline__ float dpp(float v) {
  return __builtin_bit_cast(float, __builtin_amdgcn_mov_dpp(__builtin_bit_cast(int, v), CTRL, 0xf, 0xf, true));
}
template <int LANES>
__device__ __forceinline__ float sum_lanes(float v) {
  if (LANES >= 2) v += dpp<0xb1>(v);        // quad_perm 1 0 3 2
  if (LANES >= 4) v += dpp<0x4e>(v);        // quad_perm 2 3 0 1
  if (LANES >= 8) v += dpp<0x141>(v);       // row_half_mirror
  if (LANES >= 16) v += dpp<0x140>(v);      // row_mirror
  if (LANES >= 32) v += __shfl_xor(v, 16);
  if (LANES >= 64) v += __shfl_xor(v, 32);
  return v;
}

__device__ __forceinline__ uint32_t max_lanes16(uint32_t v) {   // of 16 neighbours
  auto other = [&](auto ctrl) { return (uint32_t)__builtin_amdgcn_mov_dpp((int)v, decltype(ctrl)::value, 0xf, 0xf, true); };
  v = max(v, other(std::integral_constant<int, 0xb1>()));
  v = max(v, other(std::integral_constant<int, 0x4e>()));
  v = max(v, other(std::integral_constant<int, 0x141>()));
  return max(v, other(std::integral_constant<int, 0x140>()));
}

// ---- checks of the C entry points
inline bool aligned_to(const void* p, int bytes) { return (reinterpret_cast<uintptr_t>(p) & (uintptr_t)(bytes - 1)) == 0; }
inline int type_bytes(int type) { return type == SPRNN_TYPE_F32 ? 4 : type == SPRNN_TYPE_E4M3 ? 1 : 2; }
inline bool activation_type(int type) { return type == SPRNN_TYPE_F32 || type == SPRNN_TYPE_F16 || type == SPRNN_TYPE_BF16; }
// data, strides and alignment of a view whose rows are read
inline bool good_view(const sprnn_seq_t& s, int type) {
  return s.data && s.step >= 0 && s.sample >= 0 && aligned_to(s.data, type_bytes(type));
}
// ... of one whose rows are written: T x B rows of `width` that do not overlap
inline bool good_output(const sprnn_seq_t& s, int type, int T, int B, int width) {
  if (!good_view(s, type)) return false;
  const bool times = T > 1, samples = B > 1;
  if (times && s.step < width) return false;
  if (samples && s.sample < width) return false;
  if (times && samples) {   // one of the two strides spans all rows of the other
    const __int128 by_step = (__int128)s.step * (T - 1) + width, by_sample = (__int128)s.sample * (B - 1) + width;
    if (s.sample < by_step && s.step < by_sample) return false;
  }
  return true;
}
inline bool good_sizes(int T, int B, int width) {
  return T >= 0 && T <= (1 << 22) && B >= 0 && B <= 65535 && width >= 1 && width <= (1 << 24) && (long long)T * B <= 0x7fffffffLL;
}

// One launch, its own status (an error that the caller left behind is not reported as this launch's).
template <typename... P, typename... A>
inline hipError_t launch(void (*kernel)(P...), dim3 grid, dim3 block, int lds, hipStream_t stream, A... a) {
  static_assert(sizeof...(P) == sizeof...(A), "arguments of the kernel");
  struct Holder { static void run(void** at, P&... p) { int i = 0; ((at[i++] = (void*)&p), ...); } };
  return [&](P... p) {
    void* args[sizeof...(P)];
    Holder::run(args, p...);
    return hipLaunchKernel((const void*)kernel, grid, block, args, (size_t)lds, stream);
  }(a...);
}

}  // namespace sprnn
#endif
