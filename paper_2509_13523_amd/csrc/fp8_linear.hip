// Projections of quantised operands and their gradients (argument contracts in include/aeris_fp8.h).
//
//     y_if = sum over blocks k of 2^(a_ik + b_fk) sum_c x_ikc w_fkc
// is a product of two matrices that are contiguous along the contraction, of which 128 channels are 128 bytes
// of a row: the workgroup tiles, copies and operand reads are those of the bf16 projections with 64 channels
// per step (norm_linear.hip).  v_mfma_scale_f32_32x32x64_f8f6f4 multiplies 64 channels at twice the bf16 rate
// and applies one scale per lane, that is per row of an operand: a step of 128 channels is one block, so both
// products of a step take the same two scales.
//
// Which channels a lane holds does not matter as long as both operands agree and all of them share a scale:
// a lane of half g reads the 16-byte chunks g and g + 2 of its row for the first product of a step, g + 4 and
// g + 6 for the second, which are the first and the last 64 channels of the block.
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

typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef int i32x8 __attribute__((ext_vector_type(8)));

constexpr int kStep = AERIS_FP8_BLOCK;   // channels, and bytes of a row, per step
using Sub = Tile<64, 8>;                 // chunk swizzle of rows of 128 bytes

struct LinearParams {
  const unsigned char *x, *xs;   // [n_rows, K] and scales
  const unsigned char *w, *ws;   // [F, K] and scales
  bf16_t* y;                     // [n_rows, F]
  long long n_rows;
  int K, F, pitch;
  int m_tiles, n_tiles;
};

// A workgroup tile of WM x WN wavefronts, each NB * 32 token rows x 64 features, and kStages stages in the
// LDS: weight rows, token rows, and four bytes of scales (of four steps) for each of them.
template <int WM_, int WN_, int NB_, int STAGES_>
struct LinearShape {
  static constexpr int WM = WM_, WN = WN_, NB = NB_, kStages = STAGES_;
  static constexpr int kWaves = WM * WN;
  static constexpr int kBM = WM * NB * 32, kBN = WN * 64;
  static constexpr int kPartBytes = kBN * kStep;
  static constexpr int kScaleAt = kPartBytes + kBM * kStep;
  static constexpr int kStageBytes = kScaleAt + (kBM + kBN) * 4;
  static constexpr int kSmem = kStages * kStageBytes;
  static constexpr int kStoreBytes = NB * 32 * 128;             // results of a wave, staged
  static_assert(kWaves * kStoreBytes <= kSmem, "results are staged in the operand stages");
  // every wave copies 32 weight rows, 32 token rows and the scales of 64 rows of one operand
  static_assert(kBN == 32 * kWaves && kBM == 32 * kWaves && kWaves % 2 == 0);
};
using LinearMedium = LinearShape<2, 2, 2, 2>;   // 128 x 128, two workgroups per CU
using LinearSmall = LinearShape<2, 1, 1, 4>;    // 64 x 64, two workgroups per CU, three stages in flight

// Workgroup -> tile.  Each XCD takes a contiguous piece of the list, in groups of eight token tiles, feature
// tile by feature tile, so that every operand tile that reaches its L2 serves several workgroups.
__device__ __forceinline__ void linear_tile(const LinearParams& p, int id, int& mt, int& nt) {
  const int slot = xcd_contiguous(id, p.m_tiles * p.n_tiles);
  const int per_group = 8 * p.n_tiles, group = slot / per_group, rem = slot - group * per_group;
  const int left = p.m_tiles - group * 8, gm = left < 8 ? left : 8;
  nt = rem / gm;
  mt = group * 8 + (rem - nt * gm);
}

__device__ __forceinline__ f32x16 mfma_e4m3(i32x8 a, i32x8 b, f32x16 c, int scale_a, int scale_b) {
  return __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(a, b, c, 0, 0, 0, scale_a, 0, scale_b);
}

__device__ __forceinline__ i32x8 read_pair(uint32_t lo, uint32_t hi) {
  const i32x4 a = *reinterpret_cast<const AERIS_LDS i32x4*>(lo);
  const i32x4 b = *reinterpret_cast<const AERIS_LDS i32x4*>(hi);
  return __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7);
}

// Four bytes per lane, global -> LDS; executed only if `enable` (wave-uniform) is non-zero.
__device__ __forceinline__ void async_copy4_off(uint32_t offset, unsigned long long base, uint32_t lds_base,
                                                uint32_t enable) {
  asm volatile(
      "s_cmp_eq_u32 %3, 0\n\t"
      "s_cbranch_scc1 1f\n\t"
      "s_mov_b32 m0, %2\n\t"
      "s_nop 0\n\t"
      "global_load_lds_dword %0, %1\n"
      "1:"
      :
      : "v"(offset), "s"(base), "s"(__builtin_amdgcn_readfirstlane(lds_base)),
        "s"(__builtin_amdgcn_readfirstlane(enable))
      : "memory", "scc");
}

// Results of a wave, NB * 32 token rows x 64 features, through its own region at `stage` of the LDS (128-byte
// rows, 16-byte chunks XORed with the row), out in 16-byte pieces, eight lanes per row.
template <int NB>
__device__ __forceinline__ void linear_store(const LinearParams& p, f32x16 (&acc)[2][NB], uint32_t stage,
                                             long long row0, int valid_rows, int feature0, int lane) {
  const int li = lane & 31, g = lane >> 5;
  auto position = [](int row, int chunk) __attribute__((always_inline)) {
    return (uint32_t)(row * 128 + ((chunk ^ ((row >> 1) & 7)) << 4));
  };
#pragma unroll
  for (int b = 0; b < NB; ++b)
#pragma unroll
    for (int a = 0; a < 2; ++a)
#pragma unroll
      for (int v = 0; v < 4; ++v) {
        const int col = a * 32 + 8 * v + 4 * g;
        const f32x16& c = acc[a][b];
        const u32x2 o = {pack_bf16(c[4 * v], c[4 * v + 1]), pack_bf16(c[4 * v + 2], c[4 * v + 3])};
        *reinterpret_cast<AERIS_LDS u32x2*>(stage + position(b * 32 + li, col >> 3) + (col & 4) * 2) = o;
      }
  const int r_in = lane >> 3, chunk = lane & 7, col = feature0 + 8 * chunk;
#pragma unroll 4
  for (int i = 0; i < NB * 4; ++i) {
    const int row = i * 8 + r_in;
    const u32x4 v = *reinterpret_cast<const AERIS_LDS u32x4*>(stage + position(row, chunk));
    if (row < valid_rows && col < p.F) *reinterpret_cast<u32x4*>(p.y + (row0 + row) * p.F + col) = v;
  }
}

// One workgroup per tile.  Rows past the end repeat the last valid row (never stored); where the channels end
// in the middle of the last block, the copies of its second half repeat the first and are not multiplied.
template <class Sh>
__global__ __launch_bounds__(Sh::kWaves * 64, 2) void fp8_linear_kernel(LinearParams p) {
  constexpr int kBN = Sh::kBN, kBM = Sh::kBM, NB = Sh::NB, W = Sh::kWaves, kStages = Sh::kStages;
  constexpr int kStageBytes = Sh::kStageBytes;
  extern __shared__ __align__(16) unsigned char smem[];
  int mt, nt;
  linear_tile(p, blockIdx.x, mt, nt);
  const int tid = threadIdx.x;
  const int lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wm = wave / Sh::WN, wn = wave % Sh::WN;
  const int li = lane & 31, g = lane >> 5;
  const long long row0 = (long long)mt * kBM;
  const int f0 = nt * kBN;
  const int rows = p.n_rows - row0 < kBM ? (int)(p.n_rows - row0) : kBM;
  const int features = p.F - f0 < kBN ? p.F - f0 : kBN;

  // ---- copies: instruction j moves rows 8j..8j+7 of the weight rows, then of the token rows; wave w
  // issues j = w + W i.  Lane: row j*8 + lane/8, LDS chunk position lane%8.
  const unsigned long long wbase = reinterpret_cast<unsigned long long>(p.w + (long long)f0 * p.K);
  const unsigned long long xbase = reinterpret_cast<unsigned long long>(p.x + row0 * p.K);
  const int r_in = lane >> 3, chunk = (lane & 7) ^ Sub::swz(((wave & 1) << 3) | r_in);
  const bool half = (p.K & 64) != 0;                   // the last block has 64 channels
  const uint32_t back = half && chunk >= 4 ? 64 : 0;
  uint32_t voff[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int R = ((wave + W * (i & 3)) << 3) + r_in, limit = i < 4 ? features : rows;
    voff[i] = (uint32_t)((R < limit ? R : limit - 1) * p.K + chunk * 16);
  }
  // scales: wave w copies those of rows 64 w ... of both operands' rows in a line
  const bool of_w = wave < kBN / 64;
  const int R = (of_w ? wave * 64 : wave * 64 - kBN) + lane, limit = of_w ? features : rows;
  const uint32_t soff = (uint32_t)((R < limit ? R : limit - 1) * p.pitch);
  const unsigned long long sbase = reinterpret_cast<unsigned long long>(
      of_w ? p.ws + (long long)f0 * p.pitch : p.xs + row0 * p.pitch);

  const uint32_t lds0 = lds_address(smem);
  const int k_steps = (p.K + kStep - 1) / kStep;
  auto copy_step = [&](uint32_t stage, int step) __attribute__((always_inline)) {
    const uint32_t enable = step < k_steps, less = step == k_steps - 1 ? back : 0;
#pragma unroll
    for (int i = 0; i < 8; ++i)
      async_copy16_off(voff[i] - less, (i < 4 ? wbase : xbase) + (unsigned long long)step * kStep,
                       stage + (uint32_t)((wave + W * i) << 10), enable);
    async_copy4_off(soff, sbase + (unsigned long long)(step >> 2) * 4, stage + Sh::kScaleAt + wave * 256, enable);
  };

  uint32_t va[4], vb[4];
#pragma unroll
  for (int kk = 0; kk < 4; ++kk) {
    const uint32_t off = li * 128 + (((2 * kk + g) ^ Sub::swz(li)) << 4);
    va[kk] = lds0 + wn * 8192 + off;
    vb[kk] = lds0 + Sh::kPartBytes + wm * (NB * 4096) + off;
  }
  const uint32_t sa = lds0 + Sh::kScaleAt + (wn * 64 + li) * 4;
  const uint32_t sb = lds0 + Sh::kScaleAt + (kBN + wm * (NB * 32) + li) * 4;

  f32x16 acc[2][NB];
#pragma unroll
  for (int a = 0; a < 2; ++a)
#pragma unroll
    for (int b = 0; b < NB; ++b)
#pragma unroll
      for (int i = 0; i < 16; ++i) acc[a][b][i] = 0.f;

#pragma unroll
  for (int st = 0; st < kStages - 1; ++st) copy_step(lds0 + st * kStageBytes, st);
  uint32_t here = 0;
  for (int ks = 0; ks < k_steps; ++ks) {
    // this wave's copies of this stage have landed; those of later stages, nine each, may be on their way
    const int later = k_steps - 1 - ks;
    if (kStages >= 4 && later >= 2) asm volatile("s_waitcnt vmcnt(18)" ::: "memory");
    else if (kStages >= 4 && later >= 1) asm volatile("s_waitcnt vmcnt(9)" ::: "memory");
    else wait_async_loads();
    __syncthreads();               // this stage has landed; every reader of the stage before is done
    const uint32_t next = here == 0 ? (kStages - 1) * kStageBytes : here - kStageBytes;
    copy_step(lds0 + next, ks + kStages - 1);
    int scale_w[2], scale_x[NB];
#pragma unroll
    for (int a = 0; a < 2; ++a)
      scale_w[a] = *reinterpret_cast<const AERIS_LDS unsigned char*>(sa + here + a * 128 + (ks & 3));
#pragma unroll
    for (int b = 0; b < NB; ++b)
      scale_x[b] = *reinterpret_cast<const AERIS_LDS unsigned char*>(sb + here + b * 128 + (ks & 3));
#pragma unroll
    for (int m = 0; m < 2; ++m) {
      if (m == 1 && half && later == 0) break;
      i32x8 w[2], x[NB];
#pragma unroll
      for (int a = 0; a < 2; ++a)
        w[a] = read_pair(va[2 * m] + here + a * 4096, va[2 * m + 1] + here + a * 4096);
#pragma unroll
      for (int b = 0; b < NB; ++b)
        x[b] = read_pair(vb[2 * m] + here + b * 4096, vb[2 * m + 1] + here + b * 4096);
#pragma unroll
      for (int a = 0; a < 2; ++a)
#pragma unroll
        for (int b = 0; b < NB; ++b) acc[a][b] = mfma_e4m3(w[a], x[b], acc[a][b], scale_w[a], scale_x[b]);
    }
    here = here + kStageBytes == (uint32_t)Sh::kSmem ? 0 : here + kStageBytes;
  }
  __syncthreads();                 // every wave is done with the operand stages
  linear_store<NB>(p, acc, lds0 + wave * Sh::kStoreBytes, row0 + wm * (NB * 32), rows - wm * (NB * 32),
                   f0 + wn * 64, lane);
}

template <class Sh>
int launch_linear_shape(LinearParams p, hipStream_t stream) {
  const long long m_tiles = (p.n_rows + Sh::kBM - 1) / Sh::kBM;
  p.n_tiles = (p.F + Sh::kBN - 1) / Sh::kBN;
  p.m_tiles = (int)m_tiles;
  if (!allow_full_lds<fp8_linear_kernel<Sh>>()) return -1;
  return launch_kernel(fp8_linear_kernel<Sh>, dim3((unsigned)(m_tiles * p.n_tiles)), dim3(Sh::kWaves * 64),
                       (size_t)Sh::kSmem, stream, p);
}

int launch_linear(const LinearParams& p, hipStream_t stream) {
  const long long medium = ((p.n_rows + 127) / 128) * ((p.F + 127) / 128);
  return medium < 256 ? launch_linear_shape<LinearSmall>(p, stream) : launch_linear_shape<LinearMedium>(p, stream);
}

int check_linear(int64_t n_rows, int32_t channels, int32_t features) {
  if (const int rc = fp8_check(n_rows, channels)) return rc;
  if (const int rc = fp8_check(n_rows, features)) return rc;
  // a launch holds less than 2^32 threads, 256 per 128 x 128 tile
  return (n_rows + 127) / 128 * ((features + 127) / 128) < (1LL << 24) ? AERIS_OK : AERIS_ERR_INVALID_SHAPE;
}

bool bad16(const void* ptr) { return (reinterpret_cast<uintptr_t>(ptr) & 15) != 0; }
size_t round256(size_t n) { return (n + 255) & ~(size_t)255; }

// The workspace of the gradients: dy quantised for dx; then, in the same place, x in bf16 for dW and what
// the product of dW needs.
struct Backward {
  size_t dys;             // offset of dy's scales
  size_t wgrad;           // offset of the workspace of the product of dW
  size_t bytes;
};
Backward backward_layout(int64_t n_rows, int32_t channels, int32_t features) {
  Backward b;
  b.dys = round256((size_t)n_rows * features);
  b.wgrad = round256((size_t)n_rows * channels * 2);
  const size_t for_dx = b.dys + round256((size_t)n_rows * scale_pitch(features));
  const size_t for_dw = b.wgrad + aeris_linear_bwd_workspace_bytes(n_rows, channels, features);
  b.bytes = for_dx > for_dw ? for_dx : for_dw;
  return b;
}

// The limits of both products of the backward pass.
int check_linear_bwd(int64_t n_rows, int32_t channels, int32_t features) {
  if (const int rc = check_linear(n_rows, features, channels)) return rc;
  if ((long long)channels * features >= (1LL << 31)) return AERIS_ERR_INVALID_SHAPE;
  return aeris_linear_bwd_workspace_bytes(n_rows, channels, features) == 0 ? AERIS_ERR_INVALID_SHAPE : AERIS_OK;
}

}  // namespace
}  // namespace aeris

using namespace aeris;

extern "C" int aeris_linear_fp8_fwd(const void* x8, const void* xs, const void* w8, const void* ws, int64_t n_rows,
                                    int32_t channels, int32_t out_features, void* y, void* hip_stream) {
  if (!x8 || !xs || !w8 || !ws || !y) return AERIS_ERR_NULL_POINTER;
  if (const int rc = check_linear(n_rows, channels, out_features)) return rc;
  if (bad16(x8) || bad16(xs) || bad16(w8) || bad16(ws) || bad16(y)) return AERIS_ERR_MISALIGNED;
  LinearParams p{};
  p.x = static_cast<const unsigned char*>(x8);
  p.xs = static_cast<const unsigned char*>(xs);
  p.w = static_cast<const unsigned char*>(w8);
  p.ws = static_cast<const unsigned char*>(ws);
  p.y = static_cast<bf16_t*>(y);
  p.n_rows = n_rows;
  p.K = channels;
  p.F = out_features;
  p.pitch = scale_pitch(channels);
  return launch_linear(p, static_cast<hipStream_t>(hip_stream)) == 0 ? AERIS_OK : AERIS_ERR_HIP_LAUNCH;
}

extern "C" size_t aeris_linear_fp8_bwd_workspace_bytes(int64_t n_rows, int32_t channels, int32_t out_features) {
  if (check_linear_bwd(n_rows, channels, out_features) != AERIS_OK) return 0;
  return backward_layout(n_rows, channels, out_features).bytes;
}

extern "C" int aeris_linear_fp8_bwd(const void* x8, const void* xs, const void* wt8, const void* wts, const void* dy,
                                    int64_t n_rows, int32_t channels, int32_t out_features, void* dx, float* dweight,
                                    void* workspace, size_t workspace_bytes, void* hip_stream) {
  if (!dy || !workspace || (!dx && !dweight) || (dx && (!wt8 || !wts)) || (dweight && (!x8 || !xs)))
    return AERIS_ERR_NULL_POINTER;
  if (const int rc = check_linear_bwd(n_rows, channels, out_features)) return rc;
  if (bad16(x8) || bad16(xs) || bad16(wt8) || bad16(wts) || bad16(dy) || bad16(dx) || bad16(dweight) ||
      bad16(workspace))
    return AERIS_ERR_MISALIGNED;
  const Backward at = backward_layout(n_rows, channels, out_features);
  if (workspace_bytes < at.bytes) return AERIS_ERR_WORKSPACE_TOO_SMALL;
  const hipStream_t st = static_cast<hipStream_t>(hip_stream);
  unsigned char* space = static_cast<unsigned char*>(workspace);
  if (dx) {
    if (launch_fp8_quantize_rows(dy, false, n_rows, out_features, space, space + at.dys, st) != 0)
      return AERIS_ERR_HIP_LAUNCH;
    if (const int rc = aeris_linear_fp8_fwd(space, space + at.dys, wt8, wts, n_rows, out_features, channels, dx,
                                            hip_stream))
      return rc;
  }
  if (dweight) {
    if (launch_fp8_dequantize(static_cast<const unsigned char*>(x8), static_cast<const unsigned char*>(xs), n_rows,
                              channels, reinterpret_cast<bf16_t*>(space), st) != 0)
      return AERIS_ERR_HIP_LAUNCH;
    return aeris_linear_bwd(space, nullptr, dy, n_rows, channels, out_features, nullptr, dweight, space + at.wgrad,
                            workspace_bytes - at.wgrad, hip_stream);
  }
  return AERIS_OK;
}
