// Input projection with operands of 8 bits: out[m][r] = sum_k (x[m][k] sx[m][k / 128]) (w[r][k] sw[r / 128][k / 128]) + bias[r].
//
// A block of 128 inputs is multiplied by the matrix cores, its result scaled by sx sw and added to the running sum: four
// multiply-adds of a lane for 16 x 16 outputs.  The weights are the first operand and the rows of x the second, so that a
// lane's four results belong to one row of x: one scale for the four, and four neighbouring outputs.
//
// The instructions on e4m3 itself (v_mfma_f32_16x16x128_f8f6f4, 32 cycles a block; the older one for 32 inputs no less)
// add the products of eight neighbours at the scale of the largest one, to about 13 bits: over random blocks the sums are
// 1.4e-5 of their norm off, where binary32 sums are 2e-7 off.  Outputs of 16 bits, rounded by 2e-3 or 2e-4 at the end, take
// them.  For float32 outputs the operands are widened to binary16 (exact) on their way from LDS and multiplied by
// v_mfma_f32_16x16x32_f16, whose sums are binary32: half the rate (4 x 16 cycles), 7e-8 off.
#include "sprnn_seq.h"

namespace sprnn {
namespace {

typedef int intx8 __attribute__((ext_vector_type(8)));
typedef float floatx4 __attribute__((ext_vector_type(4)));
typedef _Float16 half2_t __attribute__((ext_vector_type(2)));
typedef _Float16 half8_t __attribute__((ext_vector_type(8)));

constexpr int kSlab = 128;             // inputs of one step: a block of scales
constexpr int kTileM = 128, kTileR = 128, kThreads = 256;

struct ProductArgs {
  int64_t vectors;                     // T * B rows of x
  int batch, rows, inputs, blocks;     // blocks of 128 inputs
  int64_t x_step, x_sample, out_step, out_sample;
  const uint8_t* x;
  const float* x_scales;
  const uint8_t* w;
  const float* w_scales;
  const float* bias;
  int tiles_m;
};

// 16 bytes of a row from k on, zeros behind its end.
__device__ __forceinline__ uint4 load_piece(const uint8_t* row, int k, int inputs) {
  uint4 v = make_uint4(0, 0, 0, 0);
  if (k + 16 <= inputs) {
    __builtin_memcpy(&v, row + k, 16);
  } else if (k < inputs) {
    uint32_t word[4] = {0, 0, 0, 0};
#pragma unroll
    for (int i = 0; i < 16; ++i)
      if (k + i < inputs) word[i >> 2] |= (uint32_t)row[k + i] << (8 * (i & 3));
    v = make_uint4(word[0], word[1], word[2], word[3]);
  }
  return v;
}

// Rows of 128 bytes repeat their banks every other row: piece q (16 bytes) of a row changes places with the row's upper
// bits, so that the sixteen rows that an LDS cycle serves are in sixteen different groups of banks.
__device__ __forceinline__ int piece_at(int row, int q) { return row * kSlab + ((q ^ ((row >> 1) & 7)) << 4); }

template <typename E>
__device__ __forceinline__ void store_four(E* row, int r, int rows, const floatx4& v, const float* bias) {
  Pack<E, 4> p;
#pragma unroll
  for (int i = 0; i < 4; ++i) p.v[i] = (E)(v[i] + (bias && r + i < rows ? bias[r + i] : 0.0f));
  if (r + 4 <= rows) store_pack(row + r, p);
  else store_part(row + r, p, rows - r);
}

// A lane's 32 inputs of one row of a block, and the product of 16 x 16 of them.
template <bool WIDE> struct Fragment;
template <> struct Fragment<false> {
  intx8 v;
  __device__ __forceinline__ Fragment(const uint4& lo, const uint4& hi)
      : v{(int)lo.x, (int)lo.y, (int)lo.z, (int)lo.w, (int)hi.x, (int)hi.y, (int)hi.z, (int)hi.w} {}
};
template <> struct Fragment<true> {
  half8_t v[4];
  static __device__ __forceinline__ half8_t widen(uint32_t a, uint32_t b) {
    const half2_t p = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8((int)a, 1.0f, false), q = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8((int)a, 1.0f, true);
    const half2_t r = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8((int)b, 1.0f, false), s = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8((int)b, 1.0f, true);
    return half8_t{p[0], p[1], q[0], q[1], r[0], r[1], s[0], s[1]};
  }
  __device__ __forceinline__ Fragment(const uint4& lo, const uint4& hi) : v{widen(lo.x, lo.y), widen(lo.z, lo.w), widen(hi.x, hi.y), widen(hi.z, hi.w)} {}
};
__device__ __forceinline__ floatx4 multiply(const Fragment<false>& w, const Fragment<false>& x) {
  return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(w.v, x.v, floatx4{0.0f, 0.0f, 0.0f, 0.0f}, 0, 0, 0, 0, 0, 0);   // scales of one
}
__device__ __forceinline__ floatx4 multiply(const Fragment<true>& w, const Fragment<true>& x) {
  floatx4 c = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
  for (int i = 0; i < 4; ++i) c = __builtin_amdgcn_mfma_f32_16x16x32_f16(w.v[i], x.v[i], c, 0, 0, 0);
  return c;
}

template <int TYPE>
__global__ __launch_bounds__(kThreads) void product_kernel(ProductArgs a, Element<TYPE>* out) {
  constexpr bool kWide = TYPE == SPRNN_TYPE_F32;
  __shared__ __attribute__((aligned(16))) uint8_t ws[2][kTileR * kSlab];
  __shared__ __attribute__((aligned(16))) uint8_t xs[2][kTileM * kSlab];
  __shared__ float scales[2][kTileM];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int64_t m0 = (int64_t)(blockIdx.x % a.tiles_m) * kTileM;
  const int r0 = (int)(blockIdx.x / a.tiles_m) * kTileR;
  const int wm = (wave & 1) * 64, wr = (wave >> 1) * 64;
  const uint8_t* x_row[4];
  const uint8_t* w_row[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int64_t m = min(m0 + (tid >> 3) + 32 * i, a.vectors - 1);
    x_row[i] = a.x + (m / a.batch) * a.x_step + (m % a.batch) * a.x_sample;
    w_row[i] = a.w + (int64_t)min(r0 + (tid >> 3) + 32 * i, a.rows - 1) * a.inputs;
  }
  const float* const scale_row = a.x_scales + min(m0 + (tid & (kTileM - 1)), a.vectors - 1) * a.blocks;
  const float* const w_scale = a.w_scales + (int64_t)(r0 / 128) * a.blocks;
  uint4 xv[4], wv[4];
  float sv;
  auto fetch = [&](int slab) {
    const int k = slab * kSlab + (tid & 7) * 16;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      xv[i] = load_piece(x_row[i], k, a.inputs);
      wv[i] = load_piece(w_row[i], k, a.inputs);
    }
    sv = scale_row[slab] * w_scale[slab];
  };
  auto stage = [&](int at) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      *reinterpret_cast<uint4*>(xs[at] + piece_at((tid >> 3) + 32 * i, tid & 7)) = xv[i];
      *reinterpret_cast<uint4*>(ws[at] + piece_at((tid >> 3) + 32 * i, tid & 7)) = wv[i];
    }
    if (tid < kTileM) scales[at][tid] = sv;
  };
  floatx4 acc[4][4];                   // [16 rows of w][16 rows of x]
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int j = 0; j < 4; ++j) acc[i][j] = floatx4{0.0f, 0.0f, 0.0f, 0.0f};
  const int fr = lane & 15, fq = lane >> 4;
  auto fragment = [&](const uint8_t* tile, int row) {
    return Fragment<kWide>(*reinterpret_cast<const uint4*>(tile + piece_at(row, fq)), *reinterpret_cast<const uint4*>(tile + piece_at(row, fq + 4)));
  };
  fetch(0);
  for (int slab = 0; slab < a.blocks; ++slab) {
    const int at = slab & 1;
    stage(at);
    if (slab + 1 < a.blocks) fetch(slab + 1);
    __syncthreads();
    float s[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) s[j] = scales[at][wm + j * 16 + fr];
    const Fragment<kWide> xf[4] = {fragment(xs[at], wm + fr), fragment(xs[at], wm + 16 + fr), fragment(xs[at], wm + 32 + fr), fragment(xs[at], wm + 48 + fr)};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const Fragment<kWide> wf = fragment(ws[at], wr + i * 16 + fr);
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const floatx4 block = multiply(wf, xf[j]);
#pragma unroll
        for (int v = 0; v < 4; ++v) acc[i][j][v] += block[v] * s[j];
      }
    }
  }
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const int64_t m = m0 + wm + j * 16 + fr;
    if (m >= a.vectors) continue;
    Element<TYPE>* const row = out + (m / a.batch) * a.out_step + (m % a.batch) * a.out_sample;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int r = r0 + wr + i * 16 + fq * 4;
      if (r < a.rows) store_four(row, r, a.rows, acc[i][j], a.bias);
    }
  }
}

template <int TYPE>
hipError_t run_product(ProductArgs a, const sprnn_seq_t& out, hipStream_t stream) {
  a.tiles_m = (int)((a.vectors + kTileM - 1) / kTileM);
  const int64_t tiles = (int64_t)a.tiles_m * ((a.rows + kTileR - 1) / kTileR);
  if (tiles > 0x7fffffffLL) return hipErrorInvalidValue;
  return launch(product_kernel<TYPE>, dim3((unsigned)tiles), dim3(kThreads), 0, stream, a, static_cast<Element<TYPE>*>(out.data));
}

}  // namespace
}  // namespace sprnn

using namespace sprnn;

extern "C" int sprnn_project_quantized(int device_id, const sprnn_product_t* p, int out_type, sprnn_seq_t out, void* stream) {
  if (device_id < 0 || !p || !good_sizes(p->steps, p->batch, p->rows) || !good_sizes(p->steps, p->batch, p->inputs) || !activation_type(out_type))
    return SPRNN_ERR_INVALID;
  if (p->steps == 0 || p->batch == 0) return SPRNN_OK;
  if (!good_view(p->x, SPRNN_TYPE_E4M3) || !p->x_scales || !aligned_to(p->x_scales, 4) || !p->w || !p->w_scales || !aligned_to(p->w_scales, 4) ||
      !aligned_to(p->bias, 4) || !good_output(out, out_type, p->steps, p->batch, p->rows))
    return SPRNN_ERR_INVALID;
  DeviceGuard guard(device_id);
  if (!guard.ok) return SPRNN_ERR_HIP;
  const ProductArgs a{(int64_t)p->steps * p->batch, p->batch, p->rows, p->inputs, (p->inputs + 127) / 128, p->x.step, p->x.sample, out.step, out.sample,
                      static_cast<const uint8_t*>(p->x.data), p->x_scales, static_cast<const uint8_t*>(p->w), p->w_scales, p->bias, 0};
  const hipStream_t s = static_cast<hipStream_t>(stream);
  const hipError_t e = out_type == SPRNN_TYPE_F32 ? run_product<SPRNN_TYPE_F32>(a, out, s) : out_type == SPRNN_TYPE_F16 ? run_product<SPRNN_TYPE_F16>(a, out, s)
                                                                                          : run_product<SPRNN_TYPE_BF16>(a, out, s);
  if (e == hipErrorInvalidValue) return SPRNN_ERR_INVALID;
  return SPRNN_HIP(e) ? SPRNN_OK : SPRNN_ERR_HIP;
}
