// Rows that leave in 8 bits (argument contracts in include/aeris_fp8.h): quantised bf16 or fp32 rows and
// their transpose, gated residual + RMSNorm + modulation, SwiGLU gate, and the way back to bf16.
//
// All of them are bound by memory traffic: every input is read once, results leave once, with fp32
// arithmetic in between.  A block of 128 columns lies in 16 lanes, eight columns each, so its largest
// magnitude is three instructions per lane pair and four rotations inside a row of lanes, without the LDS.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "aeris_fp8.h"
#include "aeris_layer_ops.h"
#include "aeris_winattn.h"
#include "fp8_common.hpp"
#include "fp8_rows.hpp"
#include "winattn_launch.hpp"

namespace aeris {
namespace {

constexpr int kThreads256 = 256;
constexpr int kGroups = kThreads256 / kBlockLanes;   // blocks a workgroup works on side by side
constexpr unsigned kMostBlocks = 1u << 22;           // workgroups of a launch over blocks

// Blocks the 16 groups of lanes of workgroup `index` of `count` walk over: all blocks of its rows, 16 apart.
struct BlockWalk {
  long long row, end;
  int block, blocks;
  int row_step, block_step;
  __device__ __forceinline__ void init(long long n_rows, int cols, unsigned index, unsigned count) {
    blocks = (cols + AERIS_FP8_BLOCK - 1) / AERIS_FP8_BLOCK;
    const int group = threadIdx.x / kBlockLanes;
    const long long r0 = n_rows * index / count;
    end = n_rows * (index + 1) / count;
    row = r0 + group / blocks;
    block = group % blocks;
    row_step = kGroups / blocks;
    block_step = kGroups % blocks;
  }
  __device__ __forceinline__ bool valid() const { return row < end; }
  __device__ __forceinline__ void step() {
    row += row_step;
    block += block_step;
    if (block >= blocks) {
      block -= blocks;
      row += 1;
    }
  }
};
// Workgroups for such a walk: whole rows each, about `each` blocks per group of lanes.  Many short workgroups are faster
// than few long ones (quantised rows, 172,800 x 2048: 187 us, 5.7 TB/s; 8192 workgroups 211, 2048 218).
unsigned walk_grid(long long n_rows, int cols, int each) {
  const long long blocks = (cols + AERIS_FP8_BLOCK - 1) / AERIS_FP8_BLOCK;
  const long long rows_each = (each * kGroups + blocks - 1) / blocks;
  const long long want = (n_rows + rows_each - 1) / rows_each;
  return (unsigned)(want < (long long)kMostBlocks ? want : (long long)kMostBlocks);
}

// ---- rows of bf16 or fp32, by rows -----------------------------------------------------------------
template <typename T>
__device__ __forceinline__ void quantize_rows(const T* __restrict__ x, long long n_rows, int cols,
                                              unsigned char* __restrict__ x8, unsigned char* __restrict__ xs,
                                              unsigned index, unsigned count) {
  const int lane = threadIdx.x & (kBlockLanes - 1), pitch = scale_pitch(cols);
  BlockWalk at;
  at.init(n_rows, cols, index, count);
  // every lane of a wave takes part in the rotations, so all leave together
  for (; __any(at.valid()); at.step()) {
    const int c = at.block * AERIS_FP8_BLOCK + lane * 8;
    const bool in = at.valid() && c < cols;
    float v[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    if (in) {
      Raw8<T> raw;
      raw.load(x + at.row * cols + c);
      raw.values(v);
    }
    u32x2 q;
    const uint32_t byte = quantize_block(v, q);
    if (in) *reinterpret_cast<u32x2*>(x8 + at.row * cols + c) = q;
    if (at.valid()) store_scale(xs + at.row * pitch, at.block, at.blocks, pitch, byte, lane);
  }
}
template <typename T>
__global__ __launch_bounds__(kThreads256) void fp8_quantize_rows_kernel(const T* __restrict__ x, long long n_rows,
                                                                        int cols, unsigned char* __restrict__ x8,
                                                                        unsigned char* __restrict__ xs) {
  quantize_rows(x, n_rows, cols, x8, xs, blockIdx.x, gridDim.x);
}

// ---- the transpose, and by rows from the same read ---------------------------------------------------
// A workgroup takes 128 rows x 128 columns: thread t holds rows 8 (t / 16) ... + 7 of columns 8 (t % 16) ... + 7, as
// they lie in memory.  Block8 holds them and gives the largest magnitudes of its rows and columns, as their fp32 bits,
// and its rows and columns as e4m3.  Vector instructions bound it unless
// bf16 stays packed: maxima of two values per instruction, conversions that divide by the scale themselves.
// 11,008 x 2048, both layouts: 16.4 us from bf16 (5.5 TB/s; unpacked to fp32 25.1), 23.7 from fp32 (5.7 TB/s).
template <typename T>
struct Block8;

template <>
struct Block8<bf16_t> {
  typedef unsigned short u16x2 __attribute__((ext_vector_type(2)));
  u32x4 r[8];                       // two columns per register
  uint32_t column[4];               // largest magnitudes of two columns
  static __device__ __forceinline__ uint32_t larger(uint32_t a, uint32_t b) {
    return __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(u16x2, a), __builtin_bit_cast(u16x2, b)));
  }
  __device__ __forceinline__ void load(int i, const bf16_t* src) { r[i] = *reinterpret_cast<const u32x4*>(src); }
  __device__ __forceinline__ void clear(int i) { r[i] = u32x4{0, 0, 0, 0}; }
  template <bool kFinite>
  __device__ __forceinline__ uint32_t magnitudes(int i, int w) const {
    uint32_t m = r[i][w] & 0x7fff7fffu;
    if (kFinite) {
      if ((m & 0xffffu) >= 0x7f80u) m &= 0xffff0000u;
      if (m >= 0x7f800000u) m &= 0xffffu;
    }
    return m;
  }
  template <bool kFinite>
  __device__ __forceinline__ void most(uint32_t (&row)[8]) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      uint32_t m[4];
#pragma unroll
      for (int w = 0; w < 4; ++w) {
        m[w] = magnitudes<kFinite>(i, w);
        column[w] = i == 0 ? m[w] : larger(column[w], m[w]);
      }
      const uint32_t all = larger(larger(m[0], m[1]), larger(m[2], m[3])), lo = all << 16, hi = all & 0xffff0000u;
      row[i] = lo > hi ? lo : hi;
    }
  }
  __device__ __forceinline__ uint32_t column_most(int e) const {
    return e & 1 ? column[e >> 1] & 0xffff0000u : column[e >> 1] << 16;
  }
  __device__ __forceinline__ u32x2 row(int i, float scale) const {
    return u32x2{pack4_e4m3(r[i][0], r[i][1], scale), pack4_e4m3(r[i][2], r[i][3], scale)};
  }
  __device__ __forceinline__ u32x2 column_of(int e, float scale) const {
    const uint32_t pick = e & 1 ? 0x07060302u : 0x05040100u;          // one half of each of two registers
    u32x2 q;
#pragma unroll
    for (int h = 0; h < 2; ++h)
      q[h] = pack4_e4m3(__builtin_amdgcn_perm(r[4 * h + 1][e >> 1], r[4 * h][e >> 1], pick),
                        __builtin_amdgcn_perm(r[4 * h + 3][e >> 1], r[4 * h + 2][e >> 1], pick), scale);
    return q;
  }
};

template <>
struct Block8<float> {
  float v[8][8];
  uint32_t column[8];
  __device__ __forceinline__ void load(int i, const float* src) {
    const f32x4 a = *reinterpret_cast<const f32x4*>(src), b = *reinterpret_cast<const f32x4*>(src + 4);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      v[i][e] = a[e];
      v[i][4 + e] = b[e];
    }
  }
  __device__ __forceinline__ void clear(int i) {
#pragma unroll
    for (int e = 0; e < 8; ++e) v[i][e] = 0.f;
  }
  template <bool kFinite>
  __device__ __forceinline__ void most(uint32_t (&row)[8]) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        uint32_t m = __float_as_uint(v[i][e]) & 0x7fffffffu;
        if (kFinite && m >= kNotFinite) m = 0;
        column[e] = i == 0 || m > column[e] ? m : column[e];
        row[i] = e == 0 || m > row[i] ? m : row[i];
      }
    }
  }
  __device__ __forceinline__ uint32_t column_most(int e) const { return column[e]; }
  __device__ __forceinline__ u32x2 row(int i, float scale) const {
    return u32x2{pack4_e4m3(v[i][0], v[i][1], v[i][2], v[i][3], scale),
                 pack4_e4m3(v[i][4], v[i][5], v[i][6], v[i][7], scale)};
  }
  __device__ __forceinline__ u32x2 column_of(int e, float scale) const {
    return u32x2{pack4_e4m3(v[0][e], v[1][e], v[2][e], v[3][e], scale),
                 pack4_e4m3(v[4][e], v[5][e], v[6][e], v[7][e], scale)};
  }
};

// Columns' maxima: over a thread's rows, over the four threads of a wave that share columns, over the waves through the
// LDS.  The transposed bytes pass through the LDS: a row of 128 bytes per column, eight-byte chunks XORed with the
// column's thread, so that neither side meets many bank conflicts.
template <typename T>
__global__ __launch_bounds__(kThreads256) void fp8_quantize_transposed_kernel(
    const T* __restrict__ x, int n_rows, int cols, unsigned char* __restrict__ x8, unsigned char* __restrict__ xs,
    unsigned char* __restrict__ xt8, unsigned char* __restrict__ xts) {
  __shared__ __align__(16) uint32_t most_of[kThreads256 / 64][AERIS_FP8_BLOCK];
  __shared__ __align__(16) unsigned char turned[AERIS_FP8_BLOCK * AERIS_FP8_BLOCK];
  const int lane = threadIdx.x & 15, strip = threadIdx.x >> 4, wave = threadIdx.x >> 6;
  const int blocks = (cols + AERIS_FP8_BLOCK - 1) / AERIS_FP8_BLOCK;
  const int row_blocks = (n_rows + AERIS_FP8_BLOCK - 1) / AERIS_FP8_BLOCK;
  const int block = blockIdx.x % blocks, row_block = blockIdx.x / blocks;
  const int c = block * AERIS_FP8_BLOCK + lane * 8, r0 = row_block * AERIS_FP8_BLOCK + strip * 8;
  const int pitch = scale_pitch(cols), t_pitch = scale_pitch(n_rows);
  const bool in = c < cols && r0 < n_rows;         // n_rows % 64 == 0: all eight rows or none

  Block8<T> v;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    if (in) v.load(i, x + (long long)(r0 + i) * cols + c);
    else v.clear(i);
  }
  // only finite values count; that is worked out where a wave meets one that is not
  uint32_t most[8];
  v.template most<false>(most);
  uint32_t all = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) all = most[i] > all ? most[i] : all;
  if (__builtin_expect(__any(all >= kNotFinite), 0)) v.template most<true>(most);
  if (x8 != nullptr) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const uint32_t byte = scale_byte(block_max(most[i]));
      const long long row = r0 + i;
      if (in) *reinterpret_cast<u32x2*>(x8 + row * cols + c) = v.row(i, scale_value(byte));
      if (r0 < n_rows) store_scale(xs + row * pitch, block, blocks, pitch, byte, lane);
    }
  }

  uint32_t column[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    column[e] = v.column_most(e);
#pragma unroll
    for (int d = 16; d < 64; d <<= 1) {
      const uint32_t o = (uint32_t)__shfl_xor((int)column[e], d, 64);
      column[e] = column[e] > o ? column[e] : o;
    }
  }
  if ((threadIdx.x & 63) < kBlockLanes) {
#pragma unroll
    for (int e = 0; e < 8; ++e) most_of[wave][lane * 8 + e] = column[e];
  }
  __syncthreads();
  uint32_t byte[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    uint32_t m = most_of[0][lane * 8 + e];
#pragma unroll
    for (int w = 1; w < kThreads256 / 64; ++w) m = m > most_of[w][lane * 8 + e] ? m : most_of[w][lane * 8 + e];
    byte[e] = scale_byte(m);
  }
#pragma unroll
  for (int e = 0; e < 8; ++e)
    *reinterpret_cast<u32x2*>(turned + (lane * 8 + e) * 128 + ((strip ^ ((lane << 1) & 15)) << 3)) =
        v.column_of(e, scale_value(byte[e]));
  __syncthreads();
  // 16 bytes per thread and pass: 8 threads per column
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int col = i * 32 + (threadIdx.x >> 3), piece = threadIdx.x & 7;      // bytes 16 piece ... + 15
    const int turn = ((col >> 3) << 1) & 15;
    const u32x4 q = *reinterpret_cast<const u32x4*>(turned + col * 128 + (((2 * piece) ^ turn) << 3));
    const int gc = block * AERIS_FP8_BLOCK + col, gr = row_block * AERIS_FP8_BLOCK + piece * 16;
    if (gc < cols && gr < n_rows) *reinterpret_cast<u32x4*>(xt8 + (long long)gc * n_rows + gr) = q;
  }
  // the column scales: threads 0 ... 15 hold those of all 128 columns
  if (threadIdx.x < kBlockLanes && c < cols) {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      unsigned char* row = xts + (long long)(c + e) * t_pitch;
      row[row_block] = (unsigned char)byte[e];
      if (row_block == row_blocks - 1)
        for (int b = row_blocks; b < t_pitch; ++b) row[b] = kScaleOne;
    }
  }
}

// ---- back to bf16, exact (172,800 x 5504: 514 us, 5.55 TB/s) ------------------------------------------
__device__ __forceinline__ void dequantize_rows(const unsigned char* __restrict__ x8, const unsigned char* __restrict__ xs,
                                                long long n_rows, int cols, bf16_t* __restrict__ x, unsigned index,
                                                unsigned count) {
  const int lane = threadIdx.x & (kBlockLanes - 1), pitch = scale_pitch(cols);
  BlockWalk at;
  at.init(n_rows, cols, index, count);
  for (; at.valid(); at.step()) {
    const int c = at.block * AERIS_FP8_BLOCK + lane * 8;
    if (c >= cols) continue;
    const u32x2 q = *reinterpret_cast<const u32x2*>(x8 + at.row * cols + c);
    const float scale = __uint_as_float((uint32_t)xs[at.row * pitch + at.block] << 23);
    u32x4 o;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const f32x2 lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)q[h], false);
      const f32x2 hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)q[h], true);
      o[2 * h] = pack_bf16(lo[0] * scale, lo[1] * scale);
      o[2 * h + 1] = pack_bf16(hi[0] * scale, hi[1] * scale);
    }
    *reinterpret_cast<u32x4*>(x + at.row * cols + c) = o;
  }
}
__global__ __launch_bounds__(kThreads256) void fp8_dequantize_kernel(const unsigned char* __restrict__ x8,
                                                                     const unsigned char* __restrict__ xs,
                                                                     long long n_rows, int cols,
                                                                     bf16_t* __restrict__ x) {
  dequantize_rows(x8, xs, n_rows, cols, x, blockIdx.x, gridDim.x);
}

// What both gradients of a projection need, dy quantised (the first `first` workgroups) and x in bf16 (the others),
// side by side in one launch (172,800 rows, 2048 and 5504: 678 us, 5.8 TB/s; one after the other 690).
__global__ __launch_bounds__(kThreads256) void fp8_backward_operands_kernel(
    const bf16_t* __restrict__ dy, int features, unsigned char* __restrict__ dy8, unsigned char* __restrict__ dys,
    unsigned first, const unsigned char* __restrict__ x8, const unsigned char* __restrict__ xs, int channels,
    bf16_t* __restrict__ x, long long n_rows) {
  if (blockIdx.x < first) quantize_rows(dy, n_rows, features, dy8, dys, blockIdx.x, first);
  else dequantize_rows(x8, xs, n_rows, channels, x, blockIdx.x - first, gridDim.x - first);
}

// ---- gated residual + RMSNorm + modulation --------------------------------------------------------------
// A wave per row at a time, K vectors of eight channels per lane, a workgroup on a contiguous chunk of the
// rows of one sample, whose modulation it keeps in the LDS: w (1 + gamma), beta, alpha.  The row stays in
// registers between its sum of squares and its result.  The expressions are those of
// aeris_gate_residual_fwd and aeris_rmsnorm_adaln_fwd, so that s and r have their bits.
constexpr int kRowWaves = 4;

struct NormParams {
  const bf16_t* x;
  const bf16_t* y;          // null: nothing to add
  const float *alpha, *w, *gamma, *beta;
  float eps;
  long long rows_per_sample;
  int chunks;               // workgroups per sample
  int C;
  bf16_t* s;
  float* r;
  unsigned char *h8, *hs;
};

__device__ __forceinline__ void unpack8(const u32x4& raw, float (&f)[8]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    f[2 * i] = __uint_as_float(raw[i] << 16);
    f[2 * i + 1] = __uint_as_float(raw[i] & 0xffff0000u);
  }
}

// Rows of up to 128 or 256 channels take 16 or 32 lanes (L), so that a wave has several (172,800 rows x 128: 53 -> 28 us).
template <int K, int L, bool kResidual>
__global__ __launch_bounds__(kThreads256) void residual_norm_fp8_kernel(NormParams p) {
  extern __shared__ __align__(16) float lds_f[];
  const int C = p.C;
  float *s_lds = lds_f, *b_lds = lds_f + C, *a_lds = lds_f + 2 * C;
  const int sample = blockIdx.x / p.chunks, chunk = blockIdx.x - sample * p.chunks;
  const long long base = sample * p.rows_per_sample;
  const long long r0 = base + p.rows_per_sample * chunk / p.chunks;
  const long long r1 = base + p.rows_per_sample * (chunk + 1) / p.chunks;
  for (int c = threadIdx.x; c < C; c += kThreads256) {
    s_lds[c] = p.w[c] * (1.f + p.gamma[(long long)sample * C + c]);
    b_lds[c] = p.beta[(long long)sample * C + c];
    if (kResidual) a_lds[c] = p.alpha[(long long)sample * C + c];
  }
  __syncthreads();
  constexpr int kRows = 64 / L;                          // of a wave
  const int lane = threadIdx.x & (L - 1), wave = threadIdx.x >> 6;
  const float inv_c = 1.f / (float)C;
  const int blocks = (C + AERIS_FP8_BLOCK - 1) / AERIS_FP8_BLOCK, pitch = scale_pitch(C);
  // every lane of a wave takes part in the sums and rotations
  for (long long first = r0 + wave * kRows; first < r1; first += kRowWaves * kRows) {
    const long long row = first + (L == 64 ? 0 : (threadIdx.x & 63) / L);
    const bool valid = L == 64 || row < r1;
    const u32x4* src = reinterpret_cast<const u32x4*>(p.x + row * C);
    const u32x4* add = kResidual ? reinterpret_cast<const u32x4*>(p.y + row * C) : nullptr;
    u32x4 raw[K], more[K];
#pragma unroll
    for (int k = 0; k < K; ++k) {
      const int v = k * 64 + lane;
      const bool in = valid && v * 8 < C;
      raw[k] = in ? __builtin_nontemporal_load(&src[v]) : u32x4{0, 0, 0, 0};
      if (kResidual) more[k] = in ? __builtin_nontemporal_load(&add[v]) : u32x4{0, 0, 0, 0};
    }
    if (kResidual) {
      u32x4* dst = reinterpret_cast<u32x4*>(p.s + row * C);
#pragma unroll
      for (int k = 0; k < K; ++k) {
        const int v = k * 64 + lane;
        if (valid && v * 8 < C) {
          float f[8], g[8];
          unpack8(raw[k], f);
          unpack8(more[k], g);
          const f32x4 a0 = *reinterpret_cast<const f32x4*>(a_lds + v * 8);
          const f32x4 a1 = *reinterpret_cast<const f32x4*>(a_lds + v * 8 + 4);
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const float lo = __builtin_fmaf((i < 2 ? a0 : a1)[2 * i & 3], g[2 * i], f[2 * i]);
            const float hi = __builtin_fmaf((i < 2 ? a0 : a1)[(2 * i + 1) & 3], g[2 * i + 1], f[2 * i + 1]);
            raw[k][i] = pack_bf16(lo, hi);
          }
          __builtin_nontemporal_store(raw[k], &dst[v]);
        }
      }
    }
    float ss = 0.f;
#pragma unroll
    for (int k = 0; k < K; ++k) {
      float f[8];
      unpack8(raw[k], f);
#pragma unroll
      for (int i = 0; i < 8; ++i) ss = __builtin_fmaf(f[i], f[i], ss);
    }
#pragma unroll
    for (int m = L / 2; m >= 1; m >>= 1) ss += __shfl_xor(ss, m, 64);
    const float r = 1.f / __builtin_sqrtf(ss * inv_c + p.eps);
    if (p.r != nullptr && lane == 0 && valid) p.r[row] = r;
#pragma unroll
    for (int k = 0; k < K; ++k) {
      const int v = k * 64 + lane;
      const bool in = valid && v * 8 < C;
      float o[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
      if (in) {
        float f[8];
        unpack8(raw[k], f);
        const f32x4 s0 = *reinterpret_cast<const f32x4*>(s_lds + v * 8);
        const f32x4 s1 = *reinterpret_cast<const f32x4*>(s_lds + v * 8 + 4);
        const f32x4 b0 = *reinterpret_cast<const f32x4*>(b_lds + v * 8);
        const f32x4 b1 = *reinterpret_cast<const f32x4*>(b_lds + v * 8 + 4);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          o[i] = __builtin_fmaf(f[i] * r, s0[i], b0[i]);
          o[4 + i] = __builtin_fmaf(f[4 + i] * r, s1[i], b1[i]);
        }
      }
      u32x2 q;
      const uint32_t byte = quantize_block(o, q);
      if (in) __builtin_nontemporal_store(q, reinterpret_cast<u32x2*>(p.h8 + row * C) + v);
      const int block = v / kBlockLanes;
      if (valid && block < blocks) store_scale(p.hs + row * pitch, block, blocks, pitch, byte, lane);
    }
  }
}

// ---- SwiGLU gate ------------------------------------------------------------------------------------
// u sigma(u) v = u v / (1 + e^-u), whose e^-u passes fp32 below u = -88.7 and whose reciprocal the hardware takes for
// zero from -87.4 on.  g is a number that a block can hold far beyond: down to u = -190 if v is large.
constexpr float kGateFar = -87.f;
// Below kGateFar: 1 + e^u is 1 in fp32, so g = u e^u v, with e^u = 2^(n + f), |f| <= 1/2, and 2^n applied in two parts,
// of which the first goes to v: neither passes the range where g does not.  u log2 e in two parts too: rounded to 24 bits
// it would carry 5e-6 into g.
__device__ __forceinline__ float gate_far(float u, float v) {
  constexpr float kLog2eRest = 1.9259629911e-8f;       // log2 e - kLog2e
  const float held = u > -400.f ? u : -400.f;          // g is zero from -300 on
  const float t = held * kLog2e, n = __builtin_rintf(t);
  const float rest = __builtin_fmaf(held, kLog2eRest, __builtin_fmaf(held, kLog2e, -t));
  const int e = (int)n, half = e >> 1;
  const float factor = __builtin_fmaf(0.f, u, held);   // held, but NaN where u is infinite, as nearer to zero
  return __builtin_ldexpf(__builtin_ldexpf(v, half) * (factor * __builtin_amdgcn_exp2f((t - n) + rest)), e - half);
}

// Two blocks per group of lanes, read before either is worked on, and no more per workgroup: 172,800 rows x 5504 837 us,
// 5.7 TB/s (one block at a time in 8192 workgroups 991; results that pass the caches like the rest 981).
constexpr int kGateAhead = 2;
__global__ __launch_bounds__(kThreads256) void swiglu_fp8_kernel(const bf16_t* __restrict__ uv, long long n_rows,
                                                                 int hidden, unsigned char* __restrict__ g8,
                                                                 unsigned char* __restrict__ gs) {
  const int lane = threadIdx.x & (kBlockLanes - 1), pitch = scale_pitch(hidden);
  BlockWalk at;
  at.init(n_rows, hidden, blockIdx.x, gridDim.x);
  constexpr int U = kGateAhead;
  while (__any(at.valid())) {
    u32x4 u[U], v[U];
    long long row[U];
    int block[U];
#pragma unroll
    for (int i = 0; i < U; ++i) {
      row[i] = at.row;
      block[i] = at.block;
      const int c = block[i] * AERIS_FP8_BLOCK + lane * 8;
      u[i] = v[i] = u32x4{0, 0, 0, 0};
      if (row[i] < at.end && c < hidden) {
        const bf16_t* src = uv + row[i] * 2 * hidden + c;
        u[i] = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(src));
        v[i] = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(src + hidden));
      }
      at.step();
    }
#pragma unroll
    for (int i = 0; i < U; ++i) {
      const int c = block[i] * AERIS_FP8_BLOCK + lane * 8;
      const bool in = row[i] < at.end && c < hidden;
      float uf[8], vf[8], o[8];
      unpack8(u[i], uf);
      unpack8(v[i], vf);
#pragma unroll
      for (int e = 0; e < 8; ++e)
        o[e] = uf[e] * __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(-uf[e] * kLog2e)) * vf[e];
      // the most negative u has the largest bits
      uint32_t lowest = 0;
#pragma unroll
      for (int e = 0; e < 8; ++e) lowest = __float_as_uint(uf[e]) > lowest ? __float_as_uint(uf[e]) : lowest;
      if (__builtin_expect(__any(lowest > __float_as_uint(kGateFar)), 0)) {
#pragma unroll
        for (int e = 0; e < 8; ++e) o[e] = uf[e] < kGateFar ? gate_far(uf[e], vf[e]) : o[e];
      }
      u32x2 q;
      const uint32_t byte = quantize_block(o, q);
      if (in) __builtin_nontemporal_store(q, reinterpret_cast<u32x2*>(g8 + row[i] * hidden + c));
      if (row[i] < at.end) store_scale(gs + row[i] * pitch, block[i], at.blocks, pitch, byte, lane);
    }
  }
}

// Workgroups per sample, of two rows per wave and place (at most kMostBlocks in all, and one per sample).  172,800 rows
// x 2048 with residual 417 us, 5.95 TB/s, in 2048 workgroups 499, 8192 478, one row each 407; but 3 x 5477 rows x 1600
// 20.7 in rows of two, 22.3 of one.
int64_t chunks_per_sample(int64_t n_samples, int64_t rows_per_sample, int channels) {
  const int64_t rows = 2 * kRowWaves * (channels <= 128 ? 4 : channels <= 256 ? 2 : 1);
  const int64_t chunks = (rows_per_sample + rows - 1) / rows, most = (kMostBlocks + n_samples - 1) / n_samples;
  return chunks < most ? chunks : most;
}

int status(int launch_rc) { return launch_rc == 0 ? AERIS_OK : AERIS_ERR_HIP_LAUNCH; }

// Calls f(Const<K>, Const<L>): vectors of eight channels per lane that hold a row, lanes of a row.
template <typename F>
void with_row_shape(int channels, F&& f) {
  const int v = (channels / 8 + 63) / 64;
  if (channels <= 128) f(Const<1>{}, Const<16>{});
  else if (channels <= 256) f(Const<1>{}, Const<32>{});
  else if (v <= 1) f(Const<1>{}, Const<64>{});
  else if (v <= 2) f(Const<2>{}, Const<64>{});
  else if (v <= 4) f(Const<4>{}, Const<64>{});
  else f(Const<8>{}, Const<64>{});
}

}  // namespace

int fp8_check(int64_t n_rows, int64_t cols) {
  if (n_rows <= 0 || cols < 64 || cols > AERIS_MAX_FP8_COLUMNS) return AERIS_ERR_INVALID_SHAPE;
  if (cols % 64 != 0) return AERIS_ERR_NOT_DIVISIBLE;
  // 64-bit products of a row and a workgroup number, byte offsets of rows
  if (n_rows >= (1LL << 40)) return AERIS_ERR_INVALID_SHAPE;
  return AERIS_OK;
}

int launch_fp8_quantize_rows(const void* x, bool f32, long long n_rows, int cols, unsigned char* x8,
                             unsigned char* xs, hipStream_t stream) {
  const dim3 grid(walk_grid(n_rows, cols, 4));
  return f32 ? launch_kernel(fp8_quantize_rows_kernel<float>, grid, dim3(kThreads256), 0, stream,
                             static_cast<const float*>(x), n_rows, cols, x8, xs)
             : launch_kernel(fp8_quantize_rows_kernel<bf16_t>, grid, dim3(kThreads256), 0, stream,
                             static_cast<const bf16_t*>(x), n_rows, cols, x8, xs);
}

int launch_fp8_dequantize(const unsigned char* x8, const unsigned char* xs, long long n_rows, int cols, bf16_t* x,
                          hipStream_t stream) {
  return launch_kernel(fp8_dequantize_kernel, dim3(walk_grid(n_rows, cols, 4)), dim3(kThreads256), 0, stream, x8, xs,
                       n_rows, cols, x);
}

int launch_fp8_backward_operands(const bf16_t* dy, int features, unsigned char* dy8, unsigned char* dys,
                                 const unsigned char* x8, const unsigned char* xs, int channels, bf16_t* x,
                                 long long n_rows, hipStream_t stream) {
  const unsigned first = walk_grid(n_rows, features, 4);
  return launch_kernel(fp8_backward_operands_kernel, dim3(first + walk_grid(n_rows, channels, 4)), dim3(kThreads256), 0,
                       stream, dy, features, dy8, dys, first, x8, xs, channels, x, n_rows);
}

}  // namespace aeris

using namespace aeris;

extern "C" int32_t aeris_fp8_scale_pitch(int32_t cols) {
  return fp8_check(1, cols) == AERIS_OK ? scale_pitch(cols) : 0;
}

extern "C" int aeris_fp8_quantize(const void* x, int32_t x_dtype, int64_t n_rows, int32_t channels, void* x8,
                                  void* xs, void* xt8, void* xts, void* hip_stream) {
  if (!x || (!x8 && !xt8) || !x8 != !xs || !xt8 != !xts) return AERIS_ERR_NULL_POINTER;
  if (x_dtype != AERIS_DT_BF16 && x_dtype != AERIS_DT_F32) return AERIS_ERR_BAD_DTYPE;
  if (const int rc = fp8_check(n_rows, channels)) return rc;
  if (xt8)
    if (const int rc = fp8_check(channels, n_rows)) return rc;
  if (bad16(x) || bad16(x8) || bad16(xs) || bad16(xt8) || bad16(xts)) return AERIS_ERR_MISALIGNED;
  const hipStream_t st = static_cast<hipStream_t>(hip_stream);
  unsigned char *q = static_cast<unsigned char*>(x8), *qs = static_cast<unsigned char*>(xs);
  if (!xt8) return status(launch_fp8_quantize_rows(x, x_dtype == AERIS_DT_F32, n_rows, channels, q, qs, st));
  const dim3 grid((unsigned)((channels + AERIS_FP8_BLOCK - 1) / AERIS_FP8_BLOCK) *
                  (unsigned)((n_rows + AERIS_FP8_BLOCK - 1) / AERIS_FP8_BLOCK));
  unsigned char *t = static_cast<unsigned char*>(xt8), *ts = static_cast<unsigned char*>(xts);
  return status(x_dtype == AERIS_DT_F32
                    ? launch_kernel(fp8_quantize_transposed_kernel<float>, grid, dim3(kThreads256), 0, st,
                                    static_cast<const float*>(x), (int)n_rows, channels, q, qs, t, ts)
                    : launch_kernel(fp8_quantize_transposed_kernel<bf16_t>, grid, dim3(kThreads256), 0, st,
                                    static_cast<const bf16_t*>(x), (int)n_rows, channels, q, qs, t, ts));
}

extern "C" int aeris_residual_norm_fp8_fwd(const void* x, const void* y, const float* alpha, const float* w,
                                           const float* gamma, const float* beta, float eps, int64_t n_rows,
                                           int64_t rows_per_sample, int32_t channels, void* s, float* r, void* h8,
                                           void* hs, void* hip_stream) {
  if (!x || !w || !gamma || !beta || !h8 || !hs || (y && (!alpha || !s))) return AERIS_ERR_NULL_POINTER;
  if (const int rc = fp8_check(n_rows, channels)) return rc;
  if (channels > AERIS_MAX_CHANNELS || rows_per_sample <= 0 || !(eps >= 0.f)) return AERIS_ERR_INVALID_SHAPE;
  if (n_rows % rows_per_sample != 0) return AERIS_ERR_NOT_DIVISIBLE;
  const int64_t n_samples = n_rows / rows_per_sample;
  if (n_samples > (1 << 20)) return AERIS_ERR_INVALID_SHAPE;
  if (bad16(x) || bad16(w) || bad16(gamma) || bad16(beta) || bad16(h8) || bad16(hs) ||
      (y && (bad16(y) || bad16(alpha) || bad16(s))) || (reinterpret_cast<uintptr_t>(r) & 3))
    return AERIS_ERR_MISALIGNED;
  const int64_t chunks = chunks_per_sample(n_samples, rows_per_sample, channels);
  const NormParams p{static_cast<const bf16_t*>(x), static_cast<const bf16_t*>(y), alpha, w, gamma, beta, eps,
                     (long long)rows_per_sample, (int)chunks, channels, static_cast<bf16_t*>(s), r,
                     static_cast<unsigned char*>(h8), static_cast<unsigned char*>(hs)};
  const dim3 grid((unsigned)(n_samples * chunks));
  const size_t smem = (y ? 3 : 2) * sizeof(float) * channels;
  const hipStream_t st = static_cast<hipStream_t>(hip_stream);
  int rc = -1;
  with_row_shape(channels, [&](auto k, auto lanes) {
    constexpr int K = decltype(k)::value, L = decltype(lanes)::value;
    rc = y ? launch_kernel(residual_norm_fp8_kernel<K, L, true>, grid, dim3(kThreads256), smem, st, p)
           : launch_kernel(residual_norm_fp8_kernel<K, L, false>, grid, dim3(kThreads256), smem, st, p);
  });
  return status(rc);
}

extern "C" int aeris_swiglu_fp8_fwd(const void* uv, int64_t n_rows, int32_t hidden, void* g8, void* gs,
                                    void* hip_stream) {
  if (!uv || !g8 || !gs) return AERIS_ERR_NULL_POINTER;
  if (const int rc = fp8_check(n_rows, hidden)) return rc;
  if (bad16(uv) || bad16(g8) || bad16(gs)) return AERIS_ERR_MISALIGNED;
  return status(launch_kernel(swiglu_fp8_kernel, dim3(walk_grid(n_rows, hidden, kGateAhead)), dim3(kThreads256), 0,
                              static_cast<hipStream_t>(hip_stream), static_cast<const bf16_t*>(uv),
                              (long long)n_rows, hidden, static_cast<unsigned char*>(g8),
                              static_cast<unsigned char*>(gs)));
}
