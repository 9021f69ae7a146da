// Input projection with operands of 8 bits: out[m][r] = sum_k (x[m][k] sx[m][k / 128]) (w[r][k] sw[r / 128][k / 128]) + bias[r].
//
// A block of 128 inputs is multiplied by the matrix cores, its result scaled by sx sw and added to the running sum: four
// multiply-adds of a lane for 16 x 16 outputs.  The weights are the first operand and the rows of x the second, so that a
// lane's four results belong to one row of x: one scale for the four, and four neighbouring outputs.
//
// The instructions on e4m3 itself (v_mfma_f32_16x16x128_f8f6f4, 32 cycles a block; the older one for 32 inputs no less)
// add the products of eight neighbours at the scale of the largest one, to about 13 bits: a sum that cancels loses digits
// that even an output of 16 bits has.  So the operands are widened to binary16 (exact) on their way from LDS or memory and
// multiplied by v_mfma_f32_16x16x32_f16, whose sums are binary32, for every type of output: half the rate (4 x 16 cycles).
#include "sprnn_seq.h"

namespace sprnn {
namespace {

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
  bool x_even, out_even;               // row m of the view is m times its sample stride away
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

__device__ __attribute__((aligned(16))) const uint8_t nothing[16] = {};   // what whole pieces behind a row's end are read from
// The same for rows that are whole pieces long: no branch around a load in flight.
__device__ __forceinline__ uint4 load_whole_piece(const uint8_t* row, int k, int inputs) {
  uint4 v;
  __builtin_memcpy(&v, k < inputs ? row + k : nothing, 16);
  return v;
}

// Rows of 128 bytes repeat their banks every other row: piece q (16 bytes) of a row changes places with the row's upper
// bits, so that the sixteen rows that an LDS cycle serves are in sixteen different groups of banks.
__device__ __forceinline__ int piece_at(int row, int q) { return row * kSlab + ((q ^ ((row >> 1) & 7)) << 4); }

// Rows of a [T][B] view by their number t B + b: where the strides allow it (even), one multiplication.
__device__ __forceinline__ int64_t row_offset(int64_t m, int batch, int64_t step, int64_t sample, bool even) {
  if (even) return m * sample;
  const uint32_t t = (uint32_t)m / (uint32_t)batch, b = (uint32_t)m - t * (uint32_t)batch;   // T B is below 2^31
  return (int64_t)t * step + (int64_t)b * sample;
}
__device__ __forceinline__ const uint8_t* x_row_at(const ProductArgs& a, int64_t m) { return a.x + row_offset(m, a.batch, a.x_step, a.x_sample, a.x_even); }

// Four neighbouring outputs of a row; their biases, zeros without any.
__device__ __forceinline__ floatx4 bias_of(const float* bias, int r, int rows) {
  floatx4 v = {0.0f, 0.0f, 0.0f, 0.0f};
  if (!bias) return v;
  if (r + 4 <= rows) {
    const Pack<float, 4> p = load_pack<4>(bias + r);
    v = floatx4{p.v[0], p.v[1], p.v[2], p.v[3]};
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (r + i < rows) v[i] = bias[r + i];
  }
  return v;
}
template <typename E>
__device__ __forceinline__ void store_four(E* row, int r, int rows, const floatx4& v) {
  Pack<E, 4> p;
#pragma unroll
  for (int i = 0; i < 4; ++i) p.v[i] = (E)v[i];
  if (r + 4 <= rows) store_pack(row + r, p);
  else store_part(row + r, p, rows - r);
}

__device__ __forceinline__ half8_t widen(uint32_t a, uint32_t b) {
  const half2_t p = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8((int)a, 1.0f, false), q = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8((int)a, 1.0f, true);
  const half2_t r = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8((int)b, 1.0f, false), s = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8((int)b, 1.0f, true);
  return half8_t{p[0], p[1], q[0], q[1], r[0], r[1], s[0], s[1]};
}
// A lane's 32 inputs of one row of a block, and the product of 16 x 16 of them.
struct Fragment {
  half8_t v[4];
  __device__ __forceinline__ Fragment(const uint4& lo, const uint4& hi) : v{widen(lo.x, lo.y), widen(lo.z, lo.w), widen(hi.x, hi.y), widen(hi.z, hi.w)} {}
};
__device__ __forceinline__ floatx4 multiply(const Fragment& w, const Fragment& x) {
  floatx4 c = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
  for (int i = 0; i < 4; ++i) c = __builtin_amdgcn_mfma_f32_16x16x32_f16(w.v[i], x.v[i], c, 0, 0, 0);
  return c;
}

template <int TYPE>
__global__ __launch_bounds__(kThreads) void product_kernel(ProductArgs a, Element<TYPE>* out) {
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
    x_row[i] = x_row_at(a, m);
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
    return Fragment(*reinterpret_cast<const uint4*>(tile + piece_at(row, fq)), *reinterpret_cast<const uint4*>(tile + piece_at(row, fq + 4)));
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
    const Fragment xf[4] = {fragment(xs[at], wm + fr), fragment(xs[at], wm + 16 + fr), fragment(xs[at], wm + 32 + fr), fragment(xs[at], wm + 48 + fr)};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const Fragment wf = fragment(ws[at], wr + i * 16 + fr);
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const floatx4 block = multiply(wf, xf[j]);
#pragma unroll
        for (int v = 0; v < 4; ++v) acc[i][j][v] += block[v] * s[j];
      }
    }
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int r = r0 + wr + i * 16 + fq * 4;
    if (r >= a.rows) break;
    const floatx4 bias = bias_of(a.bias, r, a.rows);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int64_t m = m0 + wm + j * 16 + fr;
      if (m < a.vectors) store_four(out + row_offset(m, a.batch, a.out_step, a.out_sample, a.out_even), r, a.rows, acc[i][j] + bias);
    }
  }
}

// Few rows of x: the weights are read once and bound the call.  A workgroup owns 16 RT rows of w and up to 16 MT rows of x,
// its eight wavefronts share out the blocks of 128 inputs and fetch their fragments straight from memory, two blocks ahead;
// the eight sums meet in LDS.  (8 x 2304 x 9216 on 128 x 128 tiles: 28 us, 72 workgroups; here 9.  RT = 2 halves how often
// many rows of x are fetched.)
constexpr int kFewWaves = 8;
template <int TYPE, int MT, int RT, bool WHOLE>
__global__ __launch_bounds__(64 * kFewWaves) void product_few_kernel(ProductArgs a, Element<TYPE>* out) {
  __shared__ floatx4 sums[kFewWaves][RT * MT][64];
  const int lane = threadIdx.x & 63, fr = lane & 15, fq = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int tiles_r = (a.rows + 16 * RT - 1) / (16 * RT);
  const int r0 = (int)(blockIdx.x % tiles_r) * (16 * RT);
  const int64_t m0 = (int64_t)(blockIdx.x / tiles_r) * (16 * MT);
  const uint8_t* w_row[RT];
#pragma unroll
  for (int i = 0; i < RT; ++i) w_row[i] = a.w + (int64_t)min(r0 + i * 16 + fr, a.rows - 1) * a.inputs;
  const float* const w_scale = a.w_scales + (int64_t)(r0 / 128) * a.blocks;
  const uint8_t* x_row[MT];
  const float* scale_row[MT];
#pragma unroll
  for (int j = 0; j < MT; ++j) {
    const int64_t m = min(m0 + j * 16 + fr, a.vectors - 1);
    x_row[j] = x_row_at(a, m);
    scale_row[j] = a.x_scales + m * a.blocks;
  }
  struct Block {
    uint4 w[RT][2], x[MT][2];
    float s[MT], ws;
  };
  auto load = [&](const uint8_t* row, int k) { return WHOLE ? load_whole_piece(row, k, a.inputs) : load_piece(row, k, a.inputs); };
  auto fetch = [&](Block& f, int block) {
    const int at = min(block, a.blocks - 1), k = at * kSlab + fq * 16;
#pragma unroll
    for (int i = 0; i < RT; ++i)
#pragma unroll
      for (int h = 0; h < 2; ++h) f.w[i][h] = load(w_row[i], k + 64 * h);
    f.ws = w_scale[at];
#pragma unroll
    for (int j = 0; j < MT; ++j) {
#pragma unroll
      for (int h = 0; h < 2; ++h) f.x[j][h] = load(x_row[j], k + 64 * h);
      f.s[j] = scale_row[j][at];
    }
  };
  floatx4 acc[RT][MT];
#pragma unroll
  for (int i = 0; i < RT; ++i)
#pragma unroll
    for (int j = 0; j < MT; ++j) acc[i][j] = floatx4{0.0f, 0.0f, 0.0f, 0.0f};
  auto work = [&](const Block& f) {
#pragma unroll
    for (int j = 0; j < MT; ++j) {
      const Fragment xf(f.x[j][0], f.x[j][1]);
      const float s = f.s[j] * f.ws;
#pragma unroll
      for (int i = 0; i < RT; ++i) {
        const floatx4 block = multiply(Fragment(f.w[i][0], f.w[i][1]), xf);
#pragma unroll
        for (int v = 0; v < 4; ++v) acc[i][j][v] += block[v] * s;
      }
    }
  };
  for (int block = wave; block < a.blocks; block += 2 * kFewWaves) {
    Block f[2];
    fetch(f[0], block);
    fetch(f[1], block + kFewWaves);
    work(f[0]);
    if (block + kFewWaves < a.blocks) work(f[1]);
  }
#pragma unroll
  for (int i = 0; i < RT; ++i)
#pragma unroll
    for (int j = 0; j < MT; ++j) sums[wave][i * MT + j][lane] = acc[i][j];
  __syncthreads();
  for (int tile = wave; tile < RT * MT; tile += kFewWaves) {
    floatx4 sum = sums[0][tile][lane];
#pragma unroll
    for (int w = 1; w < kFewWaves; ++w) sum += sums[w][tile][lane];
    const int r = r0 + tile / MT * 16 + fq * 4;
    const int64_t m = m0 + tile % MT * 16 + fr;
    if (m >= a.vectors || r >= a.rows) continue;
    store_four(out + row_offset(m, a.batch, a.out_step, a.out_sample, a.out_even), r, a.rows, sum + bias_of(a.bias, r, a.rows));
  }
}

// Many rows: a wavefront multiplies 64 rows of x with 64 rows of w, two by two of them are a workgroup.  Rows go from
// memory into LDS without registers between (16 bytes a lane), a slab ahead of the one that is multiplied; the swizzle of
// piece_at is in the addresses that the lanes fetch.  Instructions of 32 x 32 take half the issue slots of 16 x 16, and the
// vector unit needs them: 64 x 64 outputs of a slab are 1024 cycles of matrix instructions next to 128 conversions (5 cycles)
// and 64 scaled sums; the widened fragments and the running sums fill the registers (128 rows of w a wavefront are 27 too many).
// Where a CU has one workgroup, one wavefront a SIMD would go through loads from LDS, products and sums one after the other:
// KS = 2 gives a workgroup a second set of wavefronts and stages for every other slab, and the two sums meet in the end.
// Measured on 8192 x 2304 x 9216: 365 to 385 us, by the card, for outputs of any type (matrix instructions 139 us of it at 2.4 GHz; the
// chip runs at 1.7 to 1.9 here, and a profiler's single runs take up to 460).  Others came out within 5 % (eight wavefronts and three stages, half slabs in five stages), and widening once a
// workgroup, on the way into LDS, a sixth slower: twice the bytes through LDS.
constexpr int kWR = 2, kWM = 2, kIR = 2;           // wavefronts of a workgroup (and part) along w and x, 32 rows of w of each
constexpr int kManyR = kWR * kIR * 32, kManyM = kWM * 64, kManyThreads = kWR * kWM * 64;
constexpr int kManyRows = (kManyR + kManyM) * kSlab;                  // bytes of a slab's rows
constexpr int kManyStage = kManyRows + kManyThreads * 8;              // ... and its scales
typedef float floatx16 __attribute__((ext_vector_type(16)));

// 32 rows of a slab: this lane's four pieces, every other one of its row.
struct Strip {
  half8_t v[8];
  __device__ __forceinline__ void set(int i, const uint4& p) {
    v[2 * i] = widen(p.x, p.y);
    v[2 * i + 1] = widen(p.z, p.w);
  }
};
__device__ __forceinline__ floatx16 multiply(const Strip& w, const Strip& x) {
  floatx16 c = {};
#pragma unroll
  for (int i = 0; i < 8; ++i) c = __builtin_amdgcn_mfma_f32_32x32x16_f16(w.v[i], x.v[i], c, 0, 0, 0);
  return c;
}

template <int TYPE, int KS>
__global__ __launch_bounds__(kManyThreads * KS, 2) void product_many_kernel(ProductArgs a, Element<TYPE>* out) {
  constexpr int kM = kManyM, kR = kManyR, kWaves = kManyThreads / 64, kCopiesM = kM / (kWaves * 8), kCopiesR = kR / (kWaves * 8);
  static_assert(kWaves * 8 % 16 == 0, "a lane fetches the same piece of all its rows");
  extern __shared__ __attribute__((aligned(16))) uint8_t lds[];
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6) % kWaves, part = __builtin_amdgcn_readfirstlane(tid >> 6) / kWaves;
  uint8_t* const own_lds = lds + part * 2 * kManyStage;
  // Workgroups go to the eight XCDs in turn: each gets a run of tiles, eight along m by a few along r at a time, whose rows
  // its L2 holds.
  const int nb = gridDim.x, bid = blockIdx.x;
  const int tiles_r = (a.rows + kR - 1) / kR;
  const int id = nb % 8 == 0 ? (bid % 8) * (nb / 8) + bid / 8 : bid;
  const int group = id / (8 * tiles_r), in_group = id - group * 8 * tiles_r, deep = min(8, a.tiles_m - group * 8);
  const int64_t m0 = (int64_t)(group * 8 + in_group % deep) * kM;
  const int r0 = in_group / deep * kR;

  // this lane's part of the copies: rows (i * kWaves + wave) * 8 + lane / 8 of x and w, 16 bytes
  const int own_row = wave * 8 + (lane >> 3), piece = ((lane & 7) ^ ((own_row >> 1) & 7)) * 16;
  const uint8_t* x_at[kCopiesM];
  const uint8_t* w_at[kCopiesR];
#pragma unroll
  for (int i = 0; i < kCopiesM; ++i) {
    const int64_t m = min(m0 + i * kWaves * 8 + own_row, a.vectors - 1);
    x_at[i] = x_row_at(a, m) + piece;
  }
#pragma unroll
  for (int i = 0; i < kCopiesR; ++i) w_at[i] = a.w + (int64_t)min(r0 + i * kWaves * 8 + own_row, a.rows - 1) * a.inputs + piece;
  typedef const __attribute__((address_space(1))) void* Global;
  typedef __attribute__((address_space(3))) void* Local;
  auto bring = [&](const uint8_t* from, uint8_t* to) {
    asm volatile("" : "+v"(from));               // one copy whatever the address, no branch
    __builtin_amdgcn_global_load_lds((Global)from, (Local)to, 16, 0, 0);
  };
  const int wr = wave % kWR * (kIR * 32), wm = wave / kWR * 64;
  const float* const x_scale = a.x_scales + min(m0 + wm + lane, a.vectors - 1) * a.blocks;
  const float* const w_scale = a.w_scales + (int64_t)min((r0 + wr) / 128, (a.rows - 1) / 128) * a.blocks;
  auto copy = [&](int slab, int at) {
    uint8_t* const stage = own_lds + at * kManyStage;
    uint8_t* const to = stage + wave * 8 * kSlab;
    const int64_t k = (int64_t)slab * kSlab;
    const bool there = k + piece < a.inputs;     // pieces are whole: the rows' length is a multiple of 16
#pragma unroll
    for (int i = 0; i < kCopiesM; ++i) bring(there ? x_at[i] + k : nothing, to + i * kWaves * 8 * kSlab);
#pragma unroll
    for (int i = 0; i < kCopiesR; ++i) bring(there ? w_at[i] + k : nothing, to + (kM + i * kWaves * 8) * kSlab);
    // the scales of this wavefront's 64 rows of x, and 64 times that of its rows of w
    uint8_t* const scales = stage + kManyRows + wave * 512;
    const int from = min(slab, a.blocks - 1);
    __builtin_amdgcn_global_load_lds((Global)(x_scale + from), (Local)scales, 4, 0, 0);
    __builtin_amdgcn_global_load_lds((Global)(w_scale + from), (Local)(scales + 256), 4, 0, 0);
  };
  // The copies have no registers that the compiler would wait for: every wavefront waits for its own, and for its reads of
  // the slab that the next copies replace.
  auto next_slab = [&] {
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_waitcnt(0x0070);          // vmcnt(0) lgkmcnt(0)
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
  };

  const int fr = lane & 31, half = lane >> 5;
  floatx16 acc[kIR][2];
#pragma unroll
  for (int i = 0; i < kIR; ++i)
#pragma unroll
    for (int j = 0; j < 2; ++j) acc[i][j] = floatx16{};

  auto strip = [&](Strip& f, const uint8_t* tile, int row) {
#pragma unroll
    for (int i = 0; i < 4; ++i) f.set(i, *reinterpret_cast<const uint4*>(tile + piece_at(row, 2 * i + half)));
  };
  copy(part, 0);
  next_slab();
  for (int first = 0, at = 0; first < a.blocks; first += KS, at ^= 1) {
    const int slab = first + part;
    const uint8_t* const xs = own_lds + at * kManyStage;
    const uint8_t* const ws = xs + kM * kSlab;
    copy(slab + KS, at ^ 1);                     // (zeros behind the last one)
    if (KS > 1 && slab >= a.blocks) {
      next_slab();
      continue;
    }
    const float* const scales = reinterpret_cast<const float*>(xs + kManyRows + wave * 512);
    const float s[2] = {scales[fr] * scales[64], scales[32 + fr] * scales[64]};
    Strip xf[2];
#pragma unroll
    for (int j = 0; j < 2; ++j) strip(xf[j], xs, wm + j * 32 + fr);
#pragma unroll
    for (int i = 0; i < kIR; ++i) {
      Strip wf;
      strip(wf, ws, wr + i * 32 + fr);
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        const floatx16 block = multiply(wf, xf[j]);
#pragma unroll
        for (int v = 0; v < 16; ++v) acc[i][j][v] += block[v] * s[j];
      }
    }
    next_slab();
  }
  uint8_t* free_lds = lds;
  if (KS > 1) {                                  // the parts of the slabs meet
    floatx4* const meet = reinterpret_cast<floatx4*>(lds) + wave * 64 + lane;
    constexpr int kMeet = kWaves * 64;
    static_assert(KS == 1 || (KS == 2 && kIR * 2 * 4 * kMeet * 16 + kWaves * 32 * 68 * 4 <= 4 * kManyStage), "the other part's sums and the turns fit");
    if (part == 1) {
#pragma unroll
      for (int i = 0; i < kIR * 2 * 4; ++i) {
        const floatx16& t = acc[i / 8][i / 4 % 2];
        meet[i * kMeet] = floatx4{t[4 * (i % 4)], t[4 * (i % 4) + 1], t[4 * (i % 4) + 2], t[4 * (i % 4) + 3]};
      }
    }
    __syncthreads();
    if (part == 1) return;
#pragma unroll
    for (int i = 0; i < kIR * 2 * 4; ++i) {
      const floatx4 other = meet[i * kMeet];
#pragma unroll
      for (int v = 0; v < 4; ++v) acc[i / 8][i / 4 % 2][4 * (i % 4) + v] += other[v];
    }
    free_lds += kIR * 2 * 4 * kMeet * 16;
  }
  // Sums leave through LDS: a lane has four neighbouring outputs of a row, 32 bytes of it a store with its neighbour.  A
  // wavefront turns its own tiles, 32 rows of x by 64 of w at a time, and stores rows of 64 outputs.
  constexpr int kPitch = 64 + 4;                 // floats; four more keep the rows of a turn off each other's banks
  static_assert(kWaves * 32 * kPitch * 4 <= 2 * kManyStage, "a turn of every wavefront fits");
  float* const turn = reinterpret_cast<float*>(free_lds) + wave * 32 * kPitch;
  auto in_order = [] {                           // LDS serves a wavefront in order; the compiler is to keep it
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
  };
#pragma unroll
  for (int pair = 0; pair < kIR / 2; ++pair) {
    const int r = r0 + wr + pair * 64 + (lane & 15) * 4;
    const floatx4 bias = r < a.rows ? bias_of(a.bias, r, a.rows) : floatx4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      // element v of lane (fr, half) of a 32 x 32 tile: row 8 (v / 4) + 4 half + v % 4 of w, row fr of x
#pragma unroll
      for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int v = 0; v < 4; ++v) {
          const floatx16& t = acc[2 * pair + i][j];
          *reinterpret_cast<floatx4*>(turn + fr * kPitch + i * 32 + v * 8 + half * 4) = floatx4{t[4 * v], t[4 * v + 1], t[4 * v + 2], t[4 * v + 3]};
        }
      in_order();
#pragma unroll
      for (int q = 0; q < 32; q += 4) {
        const int row = q + (lane >> 4);
        const int64_t m = m0 + wm + j * 32 + row;
        const floatx4 sum = *reinterpret_cast<const floatx4*>(turn + row * kPitch + (lane & 15) * 4);
        if (m < a.vectors && r < a.rows)
          store_four(out + row_offset(m, a.batch, a.out_step, a.out_sample, a.out_even), r, a.rows, sum + bias);
      }
      in_order();
    }
  }
}

template <int TYPE>
hipError_t run_product(ProductArgs a, const sprnn_seq_t& out, hipStream_t stream) {
  Element<TYPE>* const to = static_cast<Element<TYPE>*>(out.data);
  auto groups = [&](int m, int r) { return (a.vectors + m - 1) / m * ((a.rows + r - 1) / r); };
  // Few rows, or outputs of fewer 128 x 128 tiles than a quarter of the CUs (tiles at 128 x 2304 x 9216, 72 of them: 22 us,
  // the few rows' kernel 26; at 768 x 5120 x 2560, 120, 42 and 78; at 256 x 5120 x 2560, 40, both 40; at 256 x 4096 x 1024, 16,
  // 32 and 16).
  if (a.vectors <= 64 || groups(kTileM, kTileR) < 64) {
    const int rows = a.vectors <= 16 ? 16 : a.vectors <= 32 ? 32 : 64;
    // 16 rows of w a workgroup while each has a CU for itself, else 32 (64 rows of x, K x R: 5120 x 2560, 160 workgroups of 16, 19.0 us
    // and 21.2; 1024 x 4096, 256, 5.9 and 6.5; 4096 x 6144, 384, 28 and 18).
    const bool whole = a.inputs % 16 == 0, wide = rows > 16 && groups(rows, 16) > 256;
    auto kernel = rows == 16   ? whole ? product_few_kernel<TYPE, 1, 1, true> : product_few_kernel<TYPE, 1, 1, false>
                  : rows == 32 ? wide ? whole ? product_few_kernel<TYPE, 2, 2, true> : product_few_kernel<TYPE, 2, 2, false>
                                      : whole ? product_few_kernel<TYPE, 2, 1, true> : product_few_kernel<TYPE, 2, 1, false>
                  : wide ? whole ? product_few_kernel<TYPE, 4, 2, true> : product_few_kernel<TYPE, 4, 2, false>
                         : whole ? product_few_kernel<TYPE, 4, 1, true> : product_few_kernel<TYPE, 4, 1, false>;
    return launch(kernel, dim3((unsigned)groups(rows, wide ? 32 : 16)), dim3(64 * kFewWaves), 0, stream, a, to);
  }
  // Copies of 16 bytes need rows that begin and end at multiples of them.
  if (a.inputs % 16 == 0 && aligned_to(a.x, 16) && aligned_to(a.w, 16) && a.x_step % 16 == 0 && a.x_sample % 16 == 0) {
    a.tiles_m = (int)((a.vectors + kManyM - 1) / kManyM);
    const int64_t n = groups(kManyM, kManyR);
    if (n > 0x7fffffffLL) return hipErrorInvalidValue;
    auto run = [&](auto kernel, int parts) {
      const int lds = parts * 2 * kManyStage;
      const hipError_t e = hipFuncSetAttribute((const void*)kernel, hipFuncAttributeMaxDynamicSharedMemorySize, lds);
      if (e != hipSuccess) return e;
      return launch(kernel, dim3((unsigned)n), dim3((unsigned)(parts * kManyThreads)), lds, stream, a, to);
    };
    // One workgroup to a CU or less: two halves of the slabs side by side (256 x 2304 x 9216, 144 tiles: 23 us,
    // one 27; at 512, 288 of them, 44 and 38).
    return n <= 256 ? run(product_many_kernel<TYPE, 2>, 2) : run(product_many_kernel<TYPE, 1>, 1);
  }
  a.tiles_m = (int)((a.vectors + kTileM - 1) / kTileM);
  const int64_t tiles = groups(kTileM, kTileR);
  if (tiles > 0x7fffffffLL) return hipErrorInvalidValue;
  return launch(product_kernel<TYPE>, dim3((unsigned)tiles), dim3(kThreads), 0, stream, a, to);
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
                      static_cast<const uint8_t*>(p->x.data), p->x_scales, static_cast<const uint8_t*>(p->w), p->w_scales, p->bias, p->steps == 1 || p->x.step == p->batch * p->x.sample, p->steps == 1 || out.step == p->batch * out.sample, 0};
  const hipStream_t s = static_cast<hipStream_t>(stream);
  const hipError_t e = out_type == SPRNN_TYPE_F32 ? run_product<SPRNN_TYPE_F32>(a, out, s) : out_type == SPRNN_TYPE_F16 ? run_product<SPRNN_TYPE_F16>(a, out, s)
                                                                                          : run_product<SPRNN_TYPE_BF16>(a, out, s);
  if (e == hipErrorInvalidValue) return SPRNN_ERR_INVALID;
  return SPRNN_HIP(e) ? SPRNN_OK : SPRNN_ERR_HIP;
}
