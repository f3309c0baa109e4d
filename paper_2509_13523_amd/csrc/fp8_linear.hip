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
#include "aeris_probe.h"
#include "aeris_winattn.h"
#include "fp8_common.hpp"
#include "fp8_rows.hpp"
#include "winattn_launch.hpp"

namespace aeris {
namespace {

#define AERIS_GLOBAL __attribute__((address_space(1)))
typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef int i32x8 __attribute__((ext_vector_type(8)));

constexpr unsigned kCus = 256;           // of the chip
constexpr int kStep = AERIS_FP8_BLOCK;   // channels, and bytes of a row, per step
using Sub = Tile<64, 8>;                 // chunk swizzle of rows of 128 bytes

struct LinearParams {
  const unsigned char *x, *xs;   // [n_rows, K] and scales
  const unsigned char *w, *ws;   // [F, K] and scales
  bf16_t* y;                     // [n_rows, F]
  long long n_rows;
  int K, F, pitch;
  int m_tiles, n_tiles;
  int interleave;                // 256 x 256 tiles: how token tiles are dealt to the XCDs
};

// A workgroup tile of WM x WN wavefronts, each NB * 32 token rows x NA * 32 features, and kStages stages in the
// LDS: weight rows, token rows, and four bytes of scales (of four steps) for each of them.
template <int WM_, int WN_, int NB_, int NA_, int STAGES_>
struct LinearShape {
  static constexpr int WM = WM_, WN = WN_, NB = NB_, NA = NA_, kStages = STAGES_;
  static constexpr int kWaves = WM * WN;
  static constexpr int kBM = WM * NB * 32, kBN = WN * NA * 32;
  static constexpr int kPartBytes = kBN * kStep;
  static constexpr int kScaleAt = kPartBytes + kBM * kStep;
  static constexpr int kStageBytes = kScaleAt + (kBM + kBN) * 4;
  static constexpr int kSmem = kStages * kStageBytes;
};
using LinearMedium = LinearShape<2, 2, 2, 2, 2>;   // 128 x 128, two workgroups per CU
using LinearSmall = LinearShape<2, 1, 1, 2, 4>;    // 64 x 64, two workgroups per CU, three stages in flight
// one workgroup per CU: groups of waves share the channels
using LinearShared = LinearShape<2, 1, 1, 2, 2>;   // 64 x 64
constexpr int kSmallGroups = 4, kMediumGroups = 2;

// Where a workgroup's tile lies: two scalar registers, from which the rest is worked out where it is needed.
template <class Sh>
struct LinearTileAt {
  int mt, nt;
  __device__ __forceinline__ long long row0() const { return (long long)mt * Sh::kBM; }
  __device__ __forceinline__ int f0() const { return nt * Sh::kBN; }
  // rows and features of the tile that exist
  __device__ __forceinline__ int rows(const LinearParams& p) const {
    const long long left = p.n_rows - row0();
    return left < Sh::kBM ? (int)left : Sh::kBM;
  }
  __device__ __forceinline__ int features(const LinearParams& p) const {
    return p.F - f0() < Sh::kBN ? p.F - f0() : Sh::kBN;
  }
};
// Workgroup -> tile.  Tiles are walked in groups of eight token tiles, feature tile by feature tile, and each XCD
// takes a contiguous piece of the list, so that every operand tile that reaches its L2 serves several workgroups.
template <class Sh>
__device__ __forceinline__ void linear_tile(const LinearParams& p, int id, LinearTileAt<Sh>& t) {
  const int slot = xcd_contiguous(id, p.m_tiles * p.n_tiles);
  const int per_group = 8 * p.n_tiles, group = slot / per_group, rem = slot - group * per_group;
  const int left = p.m_tiles - group * 8, gm = left < 8 ? left : 8;
  t.nt = rem / gm;
  t.mt = group * 8 + (rem - t.nt * gm);
}

__device__ __forceinline__ f32x16 mfma_e4m3(i32x8 a, i32x8 b, f32x16 c, int scale_a, int scale_b) {
  return __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(a, b, c, 0, 0, 0, scale_a, 0, scale_b);
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

// A wave-uniform address that the compiler would keep in vector registers.
__device__ __forceinline__ unsigned long long uniform(const void* ptr) {
  const unsigned long long a = reinterpret_cast<unsigned long long>(ptr);
  return (unsigned long long)(uint32_t)__builtin_amdgcn_readfirstlane((int)(a >> 32)) << 32 |
         (uint32_t)__builtin_amdgcn_readfirstlane((int)a);
}

// 32 bytes of an operand row, its chunks at `lo` and `hi`, and a scale; a constant distance behind the addresses goes
// into the instructions.
__device__ __forceinline__ i32x8 read_tile(uint32_t lo, uint32_t hi, int behind = 0) {
  const i32x4 a = *reinterpret_cast<const AERIS_LDS i32x4*>(reinterpret_cast<const AERIS_LDS char*>(lo) + behind);
  const i32x4 b = *reinterpret_cast<const AERIS_LDS i32x4*>(reinterpret_cast<const AERIS_LDS char*>(hi) + behind);
  return __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7);
}
__device__ __forceinline__ int read_scale(uint32_t lds, int behind = 0) {
  return *(reinterpret_cast<const AERIS_LDS unsigned char*>(lds) + behind);
}

// Results of the wave (wm, wn), NB * 32 token rows x 64 features, through its own region at `stage` of the LDS
// (128-byte rows, 16-byte chunks XORed with the row), two blocks of rows at a time, out in 16-byte pieces,
// eight lanes per row.
template <class Sh>
__device__ __forceinline__ void linear_store(const LinearParams& p, const LinearTileAt<Sh>& t, f32x16 (&acc)[2][Sh::NB],
                                             uint32_t stage, int wm, int wn, int lane) {
  constexpr int NB = Sh::NB, SB = NB < 2 ? NB : 2;
  settle(lane);   // addresses are worked out here, not kept through the caller's loop over tiles
  const int li = lane & 31, g = lane >> 5;
  auto position = [](int row, int chunk) __attribute__((always_inline)) {
    return (uint32_t)(row * 128 + ((chunk ^ ((row >> 1) & 7)) << 4));
  };
  const int r_in = lane >> 3, chunk = lane & 7, col = wn * 64 + 8 * chunk;
  const int rows = t.rows(p);
  const bool exists = col < t.features(p);
  bf16_t* const y = p.y + t.row0() * p.F + t.f0() + col;
#pragma unroll
  for (int b0 = 0; b0 < NB; b0 += SB) {
#pragma unroll
    for (int b = 0; b < SB; ++b)
#pragma unroll
      for (int a = 0; a < 2; ++a)
#pragma unroll
        for (int v = 0; v < 4; ++v) {
          const int at = a * 32 + 8 * v + 4 * g;
          const f32x16& c = acc[a][b0 + b];
          const u32x2 o = {pack_bf16(c[4 * v], c[4 * v + 1]), pack_bf16(c[4 * v + 2], c[4 * v + 3])};
          *reinterpret_cast<AERIS_LDS u32x2*>(stage + position(b * 32 + li, at >> 3) + (at & 4) * 2) = o;
        }
#pragma unroll 4
    for (int i = 0; i < SB * 4; ++i) {
      const int staged = i * 8 + r_in, row = wm * (NB * 32) + b0 * 32 + staged;
      const u32x4 v = *reinterpret_cast<const AERIS_LDS u32x4*>(stage + position(staged, chunk));
      if (row < rows && exists) *reinterpret_cast<u32x4*>(y + (long long)row * p.F) = v;
    }
  }
}

template <int NB>
__device__ __forceinline__ void linear_clear(f32x16 (&acc)[2][NB]) {
#pragma unroll
  for (int a = 0; a < 2; ++a)
#pragma unroll
    for (int b = 0; b < NB; ++b)
#pragma unroll
      for (int i = 0; i < 16; ++i) acc[a][b][i] = 0.f;
}

// One workgroup per tile.  Rows past the end repeat the last valid row (never stored); where the channels end
// in the middle of the last block, the copies of its second half repeat the first and are not multiplied.
// Bound by the LDS for long sums (a wave's 64 x 64 results need 127 of the 128 bytes a cycle that it gives), by the
// latency of the first and last steps for short ones.  128 x 128 / 64 x 64 tiles, us: 172,800 x 2048 -> 11008 4030 / 8140,
// 4096 x 2048 -> 2048 21 / 39, 1024 x 768 -> 2304 7.2 / 10.2, 512 x 768 -> 2304 6.9 / 6.8.
// G groups of Sh::kWaves waves share the channels of the tile: each takes a contiguous part of the steps, with stages
// of its own, and the first adds the others' sums to its own in their order.  For no more tiles than CUs, where a step
// is its instructions and latencies (64 x 64: 0.5 us) and nothing else runs beside it.  us, calls on two sets of operands
// in turn: 64 x 64, four groups: 128 rows x 5504 -> 2048 21.2 -> 14.8 (on one set, which stays in the L2s, 21.0 -> 12.4),
// x 2048 -> 2048 10.1 -> 7.2, x 768 -> 2304 6.1 -> 5.6 (two groups with four stages each 14.9, 7.9, 5.5; three with three
// 14.4, 7.9, 5.5); 128 x 128, two groups: 2048 rows x 5504 -> 2048 35.3 -> 31.3, x 2048 -> 2048 15.5 -> 14.4.
template <class Sh, int G>
__global__ __launch_bounds__(Sh::kWaves * G * 64, 2) void fp8_linear_kernel(LinearParams p) {
  constexpr int kBN = Sh::kBN, NB = Sh::NB, W = Sh::kWaves, kStages = Sh::kStages;
  constexpr int kStageBytes = Sh::kStageBytes;
  // every wave copies 32 weight rows, 32 token rows and the scales of 64 rows of one operand
  static_assert(Sh::NA == 2 && kBN == 32 * W && Sh::kBM == 32 * W && W % 2 == 0);
  static_assert(W * NB * 4096 <= kStages * kStageBytes, "results are staged in the operand stages");
  extern __shared__ __align__(16) unsigned char smem[];
  LinearTileAt<Sh> at;
  linear_tile(p, blockIdx.x, at);
  const int tid = threadIdx.x;
  const int lane = tid & 63, group = __builtin_amdgcn_readfirstlane((tid >> 6) / W);
  const int wave = __builtin_amdgcn_readfirstlane((tid >> 6) % W);
  const int wm = wave / Sh::WN, wn = wave % Sh::WN;
  const int li = lane & 31, g = lane >> 5;
  // ---- copies: instruction j moves rows 8j..8j+7 of the weight rows, then of the token rows; wave w
  // issues j = w + W i.  Lane: row j*8 + lane/8, LDS chunk position lane%8.
  const unsigned long long wbase = reinterpret_cast<unsigned long long>(p.w + (long long)at.f0() * p.K);
  const unsigned long long xbase = reinterpret_cast<unsigned long long>(p.x + at.row0() * p.K);
  const int r_in = lane >> 3, chunk = (lane & 7) ^ Sub::swz(((wave & 1) << 3) | r_in);
  const bool half = (p.K & 64) != 0;                   // the last block has 64 channels
  const uint32_t back = half && chunk >= 4 ? 64 : 0;
  uint32_t voff[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int R = ((wave + W * (i & 3)) << 3) + r_in, limit = i < 4 ? at.features(p) : at.rows(p);
    voff[i] = (uint32_t)((R < limit ? R : limit - 1) * p.K + chunk * 16);
  }
  // scales: wave w copies those of rows 64 w ... of both operands' rows in a line
  const bool of_w = wave < kBN / 64;
  const int R = (of_w ? wave * 64 : wave * 64 - kBN) + lane, limit = of_w ? at.features(p) : at.rows(p);
  const uint32_t soff = (uint32_t)((R < limit ? R : limit - 1) * p.pitch);
  const unsigned long long sbase = reinterpret_cast<unsigned long long>(
      of_w ? p.ws + (long long)at.f0() * p.pitch : p.xs + at.row0() * p.pitch);

  const uint32_t lds0 = lds_address(smem) + (uint32_t)(group * Sh::kSmem);
  const int k_steps = (p.K + kStep - 1) / kStep;
  const int begin = k_steps * group / G, end = k_steps * (group + 1) / G;
  auto copy_step = [&](uint32_t stage, int step) __attribute__((always_inline)) {
    const uint32_t enable = step < end, less = step == k_steps - 1 ? back : 0;
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
  linear_clear(acc);

#pragma unroll
  for (int st = 0; st < kStages - 1; ++st) copy_step(lds0 + st * kStageBytes, begin + st);
  uint32_t here = 0;
  const int most = (k_steps + G - 1) / G;              // steps of the longest part: all waves meet as often
  for (int i = 0, ks = begin; i < most; ++i, ++ks) {
    // this wave's copies of this stage have landed; those of later stages, nine each, may be on their way
    const int later = end - 1 - ks;
    if (kStages >= 4 && later >= 2) asm volatile("s_waitcnt vmcnt(18)" ::: "memory");
    else if (kStages >= 3 && later >= 1) asm volatile("s_waitcnt vmcnt(9)" ::: "memory");
    else wait_async_loads();
    __syncthreads();               // this stage has landed; every reader of the stage before is done
    const uint32_t next = here == 0 ? (kStages - 1) * kStageBytes : here - kStageBytes;
    copy_step(lds0 + next, ks + kStages - 1);
    if (G > 1 && later < 0) break;                     // only ever in the last of all
    int scale_w[2], scale_x[NB];
#pragma unroll
    for (int a = 0; a < 2; ++a) scale_w[a] = read_scale(sa + here + a * 128 + (ks & 3));
#pragma unroll
    for (int b = 0; b < NB; ++b) scale_x[b] = read_scale(sb + here + b * 128 + (ks & 3));
#pragma unroll
    for (int m = 0; m < 2; ++m) {
      if (m == 1 && half && ks == k_steps - 1) break;
      i32x8 w[2], x[NB];
#pragma unroll
      for (int a = 0; a < 2; ++a)
        w[a] = read_tile(va[2 * m] + here + a * 4096, va[2 * m + 1] + here + a * 4096);
#pragma unroll
      for (int b = 0; b < NB; ++b)
        x[b] = read_tile(vb[2 * m] + here + b * 4096, vb[2 * m + 1] + here + b * 4096);
#pragma unroll
      for (int a = 0; a < 2; ++a)
#pragma unroll
        for (int b = 0; b < NB; ++b) acc[a][b] = mfma_e4m3(w[a], x[b], acc[a][b], scale_w[a], scale_x[b]);
    }
    here = here + kStageBytes == (uint32_t)Sh::kSmem ? 0 : here + kStageBytes;
  }
  __syncthreads();                 // every wave is done with the operand stages
  if constexpr (G > 1) {
    // the sums of the other groups, in their stages
    const uint32_t part = lds_address(smem) + (uint32_t)(wave * (NB * 8192) + lane * 16);
    auto each = [&](auto&& f) __attribute__((always_inline)) {
#pragma unroll
      for (int a = 0; a < 2; ++a)
#pragma unroll
        for (int b = 0; b < NB; ++b)
#pragma unroll
          for (int q = 0; q < 4; ++q) f(acc[a][b], q, (uint32_t)(((a * NB + b) * 4 + q) << 10));
    };
    if (group > 0)
      each([&](const f32x16& c, int q, uint32_t off) __attribute__((always_inline)) {
        *reinterpret_cast<AERIS_LDS f32x4*>(part + (uint32_t)(group * Sh::kSmem) + off) =
            f32x4{c[4 * q], c[4 * q + 1], c[4 * q + 2], c[4 * q + 3]};
      });
    __syncthreads();
    if (group > 0) return;
#pragma unroll
    for (int j = 1; j < G; ++j)
      each([&](f32x16& c, int q, uint32_t off) __attribute__((always_inline)) {
        const f32x4 v = *reinterpret_cast<const AERIS_LDS f32x4*>(part + (uint32_t)(j * Sh::kSmem) + off);
#pragma unroll
        for (int e = 0; e < 4; ++e) c[4 * q + e] += v[e];
      });
  }
  linear_store<Sh>(p, at, acc, lds0 + wave * (NB * 4096), wm, wn, lane);
}

// The 256 x 256 shape: one workgroup of four wavefronts per CU, which walks over its tiles; a wave has 128 token
// rows x 128 features, so that an operand read from the LDS serves eight products of 16 x 16 x 128.  (With eight
// waves of 128 x 64 the LDS, 192 KB read and 64 KB written per step, takes as long as the products.)
//
// A step of 128 channels is two phases of 32 products, on the first and on the last 64 of the wave's token rows,
// weight rows by weight rows.  While they run, operands are read into the registers that are free: in phase 0 the
// token rows of phase 1 and the last 32 weight rows, in phase 1 the token rows of the next step's phase 0 and, each
// as soon as its last product is issued, the other weight rows of the next step.  Rows that every wave has read are
// copied over with those of the step after the next: what phase 1 read from the start of the next phase 0 on, what
// phase 0 read from the phase 1 behind it on; copies have two phases to land.  Phases end in a barrier, at which
// copies are counted.  The walk over steps goes on from tile to tile: the last steps of a tile copy and read the
// first of the next one.
//
// There is one wave per SIMD, so nothing but its own products covers what it does in between.  Tiles at the end of
// the rows or features are moved back to end with them, whatever they share with their neighbours is computed and
// stored twice, to the same bits: neither copies nor stores test anything.  Past its last tile a workgroup copies
// (and never uses) that one again, so the counts of copies in flight hold to the end.
//
// Scales: four bytes per row are those of four steps, so a group of four steps has one copy of 512 dwords, into one
// of two buffers behind the operand stages.
//
// Bound by the board's power cap and by the results.  172,800 x 2048 -> 11008 runs at 1.7 to 2.0 GHz with the matrix
// pipe busy 59 % of a tile's 55,600 cycles: 16 steps take 2900 each (2048 of them products), 8000 go into moving 256
// accumulators of a lane to the vector registers, rounding and storing them.  Moved among the products of the next
// phase instead they cost the same (they wait for the matrix pipe); stores that pass the caches, or accumulators
// cleared by the matrix pipe, gained nothing either.  Few channels are bound by the burst of results that all CUs
// store at a time: 20,011 x 768 -> 2304 44 us (stores among products 47, past the caches 48), at 2.4 GHz.  Per call,
// us, eight waves of two SIMD mates in turns (the scheme of the bf16 projections) / this: 172,800 x 2048 -> 11008
// 3320 / 3200, 172,800 x 5504 -> 2048 1545 / 1480, 8192 x 8192 -> 8192 413 / 400; the vendor's product with one scale
// 3030, 1383, 341 (one board; this takes 3200 to 3360, 1480 to 1535, 400 from board to board).
constexpr int kLargeSide = 256;
constexpr int kLargeStage = 2 * kLargeSide * kStep;                  // bytes of a stage; XORed into LDS addresses
constexpr int kLargeScales = 2 * kLargeStage, kLargeScaleBytes = 2 * kLargeSide * 4;
constexpr int kLargeSmem = kLargeScales + 2 * kLargeScaleBytes;

// The tiles of a workgroup: every 32nd of its XCD's list, which is in the order of linear_tile().  The list has a
// contiguous piece of all tiles, or every eighth token tile (interleave).
struct LargeWalk {
  int m_tiles, group, rem, left;       // token tiles of the list; place in it; tiles after this one
  int row0, f0, xcd;
  __device__ __forceinline__ void locate(const LinearParams& p) {
    int gm;
    for (;;) {
      gm = m_tiles - group * 8;
      gm = gm < 8 ? gm : 8;
      if (rem < gm * p.n_tiles) break;
      rem -= gm * p.n_tiles;
      ++group;
    }
    int nt, m;
    if (gm == 8) {
      nt = rem >> 3;
      m = rem & 7;
    } else {
      nt = rem / gm;
      m = rem - nt * gm;
    }
    m += group * 8;
    if (p.interleave) m = m * 8 + xcd;
    // moved back to end with the rows and features
    const long long last = p.n_rows - kLargeSide, row = (long long)m * kLargeSide;
    row0 = (int)(row < last ? row : last);
    f0 = nt * kLargeSide < p.F - kLargeSide ? nt * kLargeSide : p.F - kLargeSide;
  }
  __device__ __forceinline__ bool begin(const LinearParams& p) {
    const int slot = blockIdx.x >> 3;
    xcd = blockIdx.x & 7;
    int first = 0, size;
    if (p.interleave) {
      m_tiles = (p.m_tiles + 7 - xcd) >> 3;
      size = m_tiles * p.n_tiles;
    } else {
      const int total = p.m_tiles * p.n_tiles, share = total >> 3, extra = total & 7;
      m_tiles = p.m_tiles;
      first = xcd * share + (xcd < extra ? xcd : extra);
      size = share + (xcd < extra);
    }
    if (slot >= size) return false;
    left = (size - 1 - slot) / (int)(kCus / 8);
    group = (first + slot) / (8 * p.n_tiles);
    rem = first + slot - group * 8 * p.n_tiles;
    locate(p);
    return true;
  }
  __device__ __forceinline__ void advance(const LinearParams& p) {
    if (left == 0) return;             // stays where it is
    --left;
    rem += kCus / 8;
    locate(p);
  }
};

// kHalf: the channels end in the middle of the last block.
template <bool kHalf>
__global__ __launch_bounds__(256, 1) void fp8_linear_large_kernel(LinearParams p) {
  extern __shared__ __align__(16) unsigned char smem[];
  const int tid = threadIdx.x;
  const int lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wm = wave >> 1, wn = wave & 1;
  const int li = lane & 15, g = lane >> 4;
  const uint32_t lds0 = lds_address(smem);
  const int k_steps = (p.K + kStep - 1) / kStep;       // 2 or more

  // ---- copies run two steps ahead of the products, at step `ahead` of the tile that `from` is at.  Copy i of a wave
  // moves rows 32 i + 8 wave ... + 7 of the weight rows, i >= 8: of the token rows; lane: row lane / 8, LDS chunk
  // position lane % 8.
  LargeWalk from;
  if (!from.begin(p)) return;
  int tiles = from.left + 1, ahead = 0;
  unsigned long long wbase, xbase, wscales, xscales;
  unsigned long long y_done, y_now, y_next;            // results of the tile done, of this and of the copies'
  auto sources = [&]() __attribute__((always_inline)) {
    wbase = uniform(p.w + (long long)from.f0 * p.K);
    xbase = uniform(p.x + (long long)from.row0 * p.K);
    wscales = uniform(p.ws + (long long)from.f0 * p.pitch);
    xscales = uniform(p.xs + (long long)from.row0 * p.pitch);
    y_next = uniform(p.y + (long long)from.row0 * p.F + from.f0);
  };
  const int chunk = (lane & 7) ^ Sub::swz(((wave & 1) << 3) | (lane >> 3));
  const uint32_t back = kHalf && chunk >= 4 ? 64 : 0;
  uint32_t voff[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) voff[i] = (uint32_t)((32 * i + 8 * wave + (lane >> 3)) * p.K + chunk * 16);
  const uint32_t soff = (uint32_t)((wave * 64 + lane) * p.pitch);
  uint32_t here = 0;                                   // stage of the products' step: 0 or kLargeStage
  auto copy = [&](int i, uint32_t stage) __attribute__((always_inline)) {
    uint32_t off = voff[i & 7];
    if (kHalf) off -= ahead == k_steps - 1 ? back : 0;
    async_copy16_at(off, i < 8 ? wbase : xbase, lds0 + stage + (uint32_t)((wave + 4 * i) << 10));
  };
  uint32_t copied_scales = 0;                          // buffer that the next copied group goes to
  auto copy_scales = [&]() __attribute__((always_inline)) {
    const uint32_t enable = (ahead & 3) == 0;
    const uint32_t to = lds0 + kLargeScales + copied_scales + wave * 256;
    async_copy4_off(soff, wscales, to, enable);
    async_copy4_off(soff, xscales, to + kLargeSide * 4, enable);
    wscales += enable * 4;
    xscales += enable * 4;
    copied_scales ^= enable * kLargeScaleBytes;
  };
  auto advance_copies = [&]() __attribute__((always_inline)) {
    ++ahead;
    wbase += kStep;
    xbase += kStep;
    if (ahead == k_steps) {
      ahead = 0;
      from.advance(p);
      sources();
    }
  };

  // ---- operand reads: per lane two 16-byte chunks of a row, g' and g' + 4 with g' = 0, 3, 1, 2.  An LDS access takes
  // the lanes 0 ... 3, 12 ... 15 and 20 ... 27 of a half together (rows 0 ... 3, 12 ... 15 at one g, 4 ... 11 at the
  // next): with g' = g half of each collided, 15 % of a long product's cycles, though under the power cap not its time.
  uint32_t va[2], vb[2];
#pragma unroll
  for (int j = 0; j < 2; ++j) {
    const uint32_t off = li * 128 + ((((g >> 1) ^ (g & 1 ? 3 : 0)) + 4 * j) ^ Sub::swz(li)) * 16;
    va[j] = lds0 + wn * 16384 + off;
    vb[j] = lds0 + kLargeSide * kStep + wm * 16384 + off;
  }
  const uint32_t sa = lds0 + kLargeScales + (wn * 128 + li) * 4;
  const uint32_t sb = lds0 + kLargeScales + (kLargeSide + wm * 128 + li) * 4;
  i32x8 w[8], x[2][4];
  int scale_w[8], scale_x[2][4];
  uint32_t scales = 0;                                 // buffer of the step's group
  struct At {                                          // where a step's operands and scales lie, per lane
    uint32_t w[2], x[2], sw, sx;
  };
  auto at_step = [&](uint32_t stage, uint32_t scales_at) __attribute__((always_inline)) {
    At at = {{va[0] ^ stage, va[1] ^ stage}, {vb[0] ^ stage, vb[1] ^ stage}, sa + scales_at, sb + scales_at};
    settle(at.w[0]); settle(at.w[1]); settle(at.x[0]); settle(at.x[1]); settle(at.sw); settle(at.sx);
    return at;
  };
  auto read_w = [&](int a, const At& at) __attribute__((always_inline)) {
    w[a] = read_tile(at.w[0], at.w[1], a * 2048);
    scale_w[a] = read_scale(at.sw, a * 64);
  };
  auto read_x = [&](int h, int b, const At& at) __attribute__((always_inline)) {
    x[h][b] = read_tile(at.x[0], at.x[1], (4 * h + b) * 2048);
    scale_x[h][b] = read_scale(at.sx, (4 * h + b) * 64);
  };

  f32x4 acc[8][8];                                     // [16 features][16 token rows]
  // product q of phase h, weight rows by weight rows
  auto product = [&](int h, int q) __attribute__((always_inline)) {
    const int a = q >> 2, b = q & 3;
    acc[a][4 * h + b] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(w[a], x[h][b], acc[a][4 * h + b], 0, 0, 0,
                                                                         scale_w[a], 0, scale_x[h][b]);
    asm volatile("" : "+a"(acc[a][4 * h + b]));        // issued here, not behind a branch
  };
  auto clear = [&](int a, int b) __attribute__((always_inline)) {
    acc[a][b] = f32x4{0.f, 0.f, 0.f, 0.f};
    asm volatile("" : "+a"(acc[a][b]));
  };
  // The reads of this wave are complete, and its copies but for the newest `behind`, among which, behind the stores of
  // a tile (stored != 0), those 32 count too; and so are the other waves'.
  auto meet = [&](auto behind, int stored) __attribute__((always_inline)) {
    sched_fence();
    asm volatile(
        "s_cmp_eq_u32 %0, 0\n\t"
        "s_cbranch_scc1 1f\n\t"
        "s_waitcnt vmcnt(%2)\n\t"
        "s_branch 2f\n"
        "1:\n\t"
        "s_waitcnt vmcnt(%1)\n"
        "2:\n\t"
        "s_waitcnt lgkmcnt(0)\n\t"
        "s_barrier"
        :
        : "s"(__builtin_amdgcn_readfirstlane(stored)), "n"(decltype(behind)::value), "n"(decltype(behind)::value + 32)
        : "memory", "scc");
    sched_fence();
  };
  // Results of 16 token rows x 128 features, which leaves the accumulators zero.  A lane has four features of a row,
  // its neighbour 16 lanes on the next four: they swap, so that each stores eight, 16 bytes.
  const uint32_t y_lane = (uint32_t)((wm * 128 + li) * p.F + wn * 128 + 16 * (g & 1) + 8 * (g >> 1)) * 2;
  auto store = [&](int b) __attribute__((always_inline)) {
#pragma unroll
    for (int a = 0; a < 8; ++a) asm volatile("" : "+a"(acc[a][b]));
    uint32_t off = y_lane;
    settle(off);                                       // worked out here, not kept for every row
    AERIS_GLOBAL char* row = reinterpret_cast<AERIS_GLOBAL char*>(y_done) + (off + (uint32_t)(b * 32) * (uint32_t)p.F);
    uint32_t lo[8], hi[8];
#pragma unroll
    for (int a = 0; a < 8; ++a) {
      lo[a] = pack_bf16(acc[a][b][0], acc[a][b][1]);
      hi[a] = pack_bf16(acc[a][b][2], acc[a][b][3]);
    }
#pragma unroll
    for (int a = 0; a < 8; a += 2) {
      const auto l = __builtin_amdgcn_permlane16_swap(lo[a], lo[a + 1], false, false);
      const auto h = __builtin_amdgcn_permlane16_swap(hi[a], hi[a + 1], false, false);
      *reinterpret_cast<AERIS_GLOBAL u32x4*>(row + a * 32) = u32x4{l[0], h[0], l[1], h[1]};
    }
#pragma unroll
    for (int a = 0; a < 8; ++a) clear(a, b);
  };

  // The copies of a step, in the order they are issued: ten of rows that phase 1 reads for the next step (weight rows
  // but for the last 32 of each wave's, token rows of phase 0), then six that phase 0 reads.
  constexpr int kOrder[16] = {0, 1, 2, 4, 5, 6, 8, 9, 12, 13, 3, 7, 10, 11, 14, 15};
  sources();
  y_now = y_next;
#pragma unroll
  for (int st = 0; st < 2; ++st) {
    copy_scales();
#pragma unroll
    for (int i = 0; i < 16; ++i) copy(kOrder[i], st * kLargeStage);
    advance_copies();
  }
  meet(Const<0>{}, 0);
  At now = at_step(0, 0), next;
#pragma unroll
  for (int a = 0; a < 6; ++a) read_w(a, now);
#pragma unroll
  for (int b = 0; b < 4; ++b) read_x(0, b, now);
  meet(Const<0>{}, 0);
#pragma unroll
  for (int a = 0; a < 8; ++a)
#pragma unroll
    for (int b = 0; b < 8; ++b) clear(a, b);
  int stored = 0;                                      // results were stored before this step
  for (int t = 0;;) {
    const int last = __builtin_amdgcn_readfirstlane(t == k_steps - 1);
    const int t_next = last ? 0 : t + 1;
#pragma unroll
    for (int q = 0; q < 32; ++q) {
      // in a last step of 64 channels the copies of the second half repeated the first: weights of zero for it
      if (kHalf && (q & 3) == 0) {
#pragma unroll
        for (int i = 4; i < 8; ++i) w[q >> 2][i] &= last - 1;
      }
      product(0, q);
      if (q == 1 || q == 6) read_w(6 + q / 6, now);
      if (q == 11 || q == 15 || q == 19 || q == 23) read_x(1, (q - 11) / 4, now);
      if ((q & 3) == 0) copy(kOrder[q >> 2], here);
      if (q == 13) {                                   // what the next step needs, worked out among the products
        if ((t & 3) == 3 || last) scales ^= kLargeScaleBytes;
        next = at_step(here ^ kLargeStage, scales + (uint32_t)(t_next & 3));
      }
      sched_fence();
    }
    // newer than the last copy that phase 1 needs: six of the phase before this one, this one's eight
    meet(Const<14>{}, stored);
#pragma unroll
    for (int i = 0; i < 4; ++i) settle(scale_x[1][i]);
    settle(scale_w[6]);
    settle(scale_w[7]);
#pragma unroll
    for (int q = 0; q < 32; ++q) {
      product(1, q);
      constexpr int kX[4] = {1, 3, 9, 13}, kW[6] = {5, 11, 15, 18, 22, 25};
#pragma unroll
      for (int i = 0; i < 4; ++i) if (q == kX[i]) read_x(0, i, next);
#pragma unroll
      for (int i = 0; i < 6; ++i) if (q == kW[i]) read_w(i, next);
      if (q == 2) copy_scales();                       // the buffer's last reads were in phase 0
      if ((q & 3) == 0) copy(kOrder[8 + (q >> 2)], here);
      if (q == 31) {
        if (last) {
          y_done = y_now;
          y_now = y_next;
        }
        advance_copies();
        here ^= kLargeStage;
      }
      sched_fence();
    }
    // newer than the last copy that the next phase 0 needs: this step's sixteen
    meet(Const<16>{}, stored);
#pragma unroll
    for (int i = 0; i < 4; ++i) settle(scale_x[0][i]);
#pragma unroll
    for (int i = 0; i < 6; ++i) settle(scale_w[i]);
    now = next;
    stored = last;
    if (last) {
#pragma unroll
      for (int b = 0; b < 8; ++b) store(b);
      if (--tiles == 0) break;
    }
    t = t_next;
  }
}

// Up to 64 token rows: bound by reading the weight once.  A workgroup has 16 features; its eight waves share the steps,
// read both operands straight into registers (16 x 16 x 128 products, token rows in MB blocks of 16) and join their
// sums through the LDS, in the order of the waves.  One row, 2048 -> 12288: 6.6 us, 3.8 TB/s of weights from the
// last-level cache (four waves 6.5, but 7.1 instead of 5.7 for 5504 -> 2048).
constexpr int kRowsWaves = 8;
template <int MB>
__global__ __launch_bounds__(kRowsWaves * 64) void fp8_linear_rows_kernel(LinearParams p) {
  constexpr int W = kRowsWaves;
  __shared__ f32x4 part[W][MB][64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int li = lane & 15, g = lane >> 4;
  const int f0 = blockIdx.x * 16, rows = (int)p.n_rows;
  const int k_steps = (p.K + kStep - 1) / kStep;
  const bool half = (p.K & 64) != 0;
  const unsigned char* w = p.w + (long long)(f0 + li) * p.K + g * 16;
  const unsigned char* ws = p.ws + (long long)(f0 + li) * p.pitch;
  const unsigned char *x[MB], *xs[MB];
  f32x4 acc[MB];
#pragma unroll
  for (int b = 0; b < MB; ++b) {
    const int row = b * 16 + li < rows ? b * 16 + li : rows - 1;       // rows past the end: never stored
    x[b] = p.x + (long long)row * p.K + g * 16;
    xs[b] = p.xs + (long long)row * p.pitch;
    acc[b] = f32x4{0.f, 0.f, 0.f, 0.f};
  }
  const int end = k_steps * (wave + 1) / W;
  for (int t = k_steps * wave / W; t < end; ++t) {
    // a last step of 64 channels: its second half repeats the first, with weights of zero
    const bool whole = !half || t != k_steps - 1;
    const int at = t * kStep, second = at + (whole ? 64 : 0);
    const i32x4 w0 = *reinterpret_cast<const i32x4*>(w + at);
    i32x4 w1 = *reinterpret_cast<const i32x4*>(w + second);
    if (!whole) w1 = i32x4{0, 0, 0, 0};
    const int scale_w = ws[t];
#pragma unroll
    for (int b = 0; b < MB; ++b) {
      const i32x4 x0 = *reinterpret_cast<const i32x4*>(x[b] + at);
      const i32x4 x1 = *reinterpret_cast<const i32x4*>(x[b] + second);
      acc[b] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(
          __builtin_shufflevector(w0, w1, 0, 1, 2, 3, 4, 5, 6, 7), __builtin_shufflevector(x0, x1, 0, 1, 2, 3, 4, 5, 6, 7),
          acc[b], 0, 0, 0, scale_w, 0, (int)xs[b][t]);
    }
  }
#pragma unroll
  for (int b = 0; b < MB; ++b) part[wave][b][lane] = acc[b];
  __syncthreads();
  const int b = wave;                                  // MB <= W
  const int row = b * 16 + li;
  if (b >= MB || row >= rows) return;
  f32x4 sum = part[0][b][lane];
#pragma unroll
  for (int i = 1; i < W; ++i) sum += part[i][b][lane];
  const u32x2 o = {pack_bf16(sum[0], sum[1]), pack_bf16(sum[2], sum[3])};
  *reinterpret_cast<u32x2*>(p.y + (long long)row * p.F + f0 + 4 * g) = o;
}

int launch_linear_rows(const LinearParams& p, hipStream_t stream) {
  const dim3 grid((unsigned)(p.F / 16)), block(kRowsWaves * 64);
  return p.n_rows <= 16   ? launch_kernel(fp8_linear_rows_kernel<1>, grid, block, 0, stream, p)
         : p.n_rows <= 32 ? launch_kernel(fp8_linear_rows_kernel<2>, grid, block, 0, stream, p)
                          : launch_kernel(fp8_linear_rows_kernel<4>, grid, block, 0, stream, p);
}

template <class Sh, int G = 1>
int launch_linear_shape(LinearParams p, hipStream_t stream) {
  p.n_tiles = (p.F + Sh::kBN - 1) / Sh::kBN;
  p.m_tiles = (int)((p.n_rows + Sh::kBM - 1) / Sh::kBM);
  const dim3 grid((unsigned)p.m_tiles * (unsigned)p.n_tiles), block(Sh::kWaves * G * 64);
  if (!allow_full_lds<fp8_linear_kernel<Sh, G>>()) return -1;
  return launch_kernel(fp8_linear_kernel<Sh, G>, grid, block, (size_t)(G * Sh::kSmem), stream, p);
}

int launch_linear_large(LinearParams p, hipStream_t stream) {
  p.n_tiles = (p.F + kLargeSide - 1) / kLargeSide;
  p.m_tiles = (int)((p.n_rows + kLargeSide - 1) / kLargeSide);
  // one workgroup per CU, which walks its tiles; an XCD may have more than its eighth of them
  const unsigned tiles = (unsigned)(p.interleave ? (p.m_tiles + 7) / 8 * 8 : p.m_tiles) * (unsigned)p.n_tiles;
  auto launch = [&](auto half) {
    constexpr auto kernel = fp8_linear_large_kernel<decltype(half)::value>;
    if (!allow_full_lds<kernel>()) return -1;
    return launch_kernel(kernel, dim3(tiles > kCus ? kCus : tiles), dim3(256), (size_t)kLargeSmem, stream, p);
  };
  return p.K % kStep != 0 ? launch(std::true_type{}) : launch(std::false_type{});
}

// Microseconds a shape takes: rounds of `slots` workgroups, each a fixed part and a part per step, a last round that
// leaves slots empty less; at least what the bytes take.  Fitted to 3386 sizes of 65 ... 200,000 rows, 64 ... 5504
// channels and 64 ... 11,008 features (mean deviation 4 to 6 %).  What is taken by all of choose_linear(), against the
// best of the six forms (drawn sizes, channels and features as above): 6000 ... 200,000 rows 0.5 % slower on average, 8 %
// or more at 2.1 % of 10,521 sizes, 31 % at worst (184,904 x 640 -> 256: 65 us, 256 x 256 tiles 50); 65 ... 6000 rows 0.3 %,
// 8 % at 0.4 % of 28,427, 23 % at worst; 1 ... 64 rows 0.2 %, 8 % at 1.1 % of 18,201, 51 % at worst (35 x 2816 -> 4224: 14.2
// us, shared 64 x 64 tiles 9.4).
struct ShapeTime {
  double round, round_step;             // of a full round
  double last, last_step, last_filled;  // of the last: per step, and by how full it is
  double bytes;                         // microseconds per 5 MB
};
constexpr ShapeTime kSmallTime = {1.95, 0.528, 3.47, 0.356, 0.294, 1.24};
constexpr ShapeTime kMediumTime = {2.61, 1.14, 3.48, 0.537, 0.78, 1.14};
constexpr ShapeTime kLargeTime = {5.06, 1.545, 8.54, 1.17, 1.12, 1.22};
double shape_time(const ShapeTime& t, long long n_rows, int K, int F, int side, int slots) {
  const long long tiles = (n_rows + side - 1) / side * ((F + side - 1) / side);
  const double steps = (K + kStep - 1) / kStep, rest = (double)(tiles % slots) / slots;
  const double rounds = (double)(tiles / slots) * (t.round + t.round_step * steps) +
                        (rest > 0.0 ? t.last + steps * (t.last_step + t.last_filled * (side == 256 ? rest * rest : rest))
                                    : 0.0);
  const double bytes = 2.0 + t.bytes / 5e6 * ((double)n_rows * K + (double)F * K + 2.0 * (double)n_rows * F);
  return rounds > bytes ? rounds : bytes;
}

// The same of workgroups whose groups of waves share the channels, one per CU: for one round of tiles.  A part of the
// steps is longer the more CUs work.
double shared_time(double fixed, double step, double step_filled, long long n_rows, int K, int F, int side, int groups) {
  const long long tiles = (n_rows + side - 1) / side * ((F + side - 1) / side);
  if (tiles > kCus) return 1e30;
  const int part = ((K + kStep - 1) / kStep + groups - 1) / groups;
  return fixed + part * (step + step_filled / kCus * (double)tiles);
}

enum class LinearTile { kLarge, kMedium, kMediumShared, kSmall, kSmallShared, kRows };
LinearTile choose_linear(long long n_rows, int K, int F) {
  auto faster = [](LinearTile a, double time_a, LinearTile b, double time_b, double& time) {
    time = time_a <= time_b ? time_a : time_b;
    return time_a <= time_b ? a : b;
  };
  double small, medium;
  const LinearTile of_64 = faster(LinearTile::kSmall, shape_time(kSmallTime, n_rows, K, F, 64, 512),
                                  LinearTile::kSmallShared, shared_time(4.15, 0.66, 0.4, n_rows, K, F, 64, kSmallGroups),
                                  small);
  // A few rows: every workgroup of 16 features reads them and its part of the weight, from the L2s, in steps that wait
  // for each other (us, 64 x 64 tiles / this: 1 x 2048 -> 12288 8.5 / 7.1, 1 x 5504 -> 2048 11.6 / 6.1, 17 x 5504 ->
  // 2048 11.8 / 8.9, 64 x 5504 -> 2048 13.3 / 16.5, 17 x 2048 -> 11008 9.1 / 10.7, 64 x 768 -> 2304 5.5 / 4.7).
  if (n_rows <= 64) {
    const double filled = 0.15 + 0.026 * (F / 16), rate = filled < 7.0 ? filled : 7.0;       // TB/s
    const double bytes = (double)(F / 16) * (double)(n_rows + 16) * K / (1e6 * rate);
    const int blocks = n_rows <= 16 ? 1 : n_rows <= 32 ? 2 : 4, wave_steps = (K + kRowsWaves * kStep - 1) / (kRowsWaves * kStep);
    const double waits = 0.25 * blocks + (wave_steps - 1) * (0.25 + 0.44 * blocks);
    if (2.3 + (bytes > waits ? bytes : waits) < small) return LinearTile::kRows;
  }
  const LinearTile of_128 = faster(LinearTile::kMedium, shape_time(kMediumTime, n_rows, K, F, 128, 512),
                                   LinearTile::kMediumShared,
                                   shared_time(6.0, 1.05, 0.1, n_rows, K, F, 128, kMediumGroups), medium);
  // 256 x 256 tiles are moved back from the ends, and look a step ahead
  const double large = n_rows >= kLargeSide && F >= kLargeSide && K > kStep
                           ? shape_time(kLargeTime, n_rows, K, F, 256, (int)kCus) : 1e30;
  if (large <= medium && large <= small) return LinearTile::kLarge;
  return small <= medium ? of_64 : of_128;
}

// Whether the XCDs take the token tiles of 256 rows in turn, or each a contiguous piece of all tiles.  In turn is the
// faster way with fewer than 4096 features (time over that of pieces 0.97 to 1.0 in the mean, 1.02 to 1.06 with
// more), but where an XCD's whole token tiles make one round more (up to 1.35).
bool interleave_large(long long n_rows, int F) {
  const long long m = (n_rows + kLargeSide - 1) / kLargeSide, n = (F + kLargeSide - 1) / kLargeSide;
  auto rounds = [](long long tiles_of_an_xcd) { return (tiles_of_an_xcd + kCus / 8 - 1) / (kCus / 8); };
  return F < 4096 && rounds((m + 7) / 8 * n) == rounds((m * n + 7) / 8);
}

int launch_linear(LinearParams p, hipStream_t stream) {
  switch (choose_linear(p.n_rows, p.K, p.F)) {
    case LinearTile::kRows: return launch_linear_rows(p, stream);
    case LinearTile::kSmall: return launch_linear_shape<LinearSmall>(p, stream);
    case LinearTile::kSmallShared: return launch_linear_shape<LinearShared, kSmallGroups>(p, stream);
    case LinearTile::kMediumShared: return launch_linear_shape<LinearMedium, kMediumGroups>(p, stream);
    case LinearTile::kMedium: return launch_linear_shape<LinearMedium>(p, stream);
    default:
      p.interleave = interleave_large(p.n_rows, p.F);
      return launch_linear_large(p, stream);
  }
}

int check_linear(int64_t n_rows, int32_t channels, int32_t features) {
  if (const int rc = fp8_check(n_rows, channels)) return rc;
  if (const int rc = fp8_check(n_rows, features)) return rc;
  // a launch holds less than 2^32 threads, 128 per 64 x 64 tile
  return (n_rows + 63) / 64 * (features / 64) < (1LL << 25) ? AERIS_OK : AERIS_ERR_INVALID_SHAPE;
}

size_t round256(size_t n) { return (n + 255) & ~(size_t)255; }

// The workspace of the gradients.  For dW: x in bf16 and, behind it, what its product needs.  For dx: dy quantised.  For
// both dy comes first, in the place of what dW's product needs where that is large enough, else of all of it.
struct Backward {
  size_t wgrad;           // offset of the workspace of the product of dW
  size_t dy, dys;         // offsets of dy's values and scales
  size_t bytes;
};
// AERIS_OK if both products of the backward pass accept the size, else an AERIS_ERR_ code.
int backward_layout(int64_t n_rows, int32_t channels, int32_t features, bool want_dx, bool want_dw, Backward& b) {
  if (const int rc = check_linear(n_rows, features, channels)) return rc;
  if ((long long)channels * features >= (1LL << 31)) return AERIS_ERR_INVALID_SHAPE;
  const size_t product = aeris_linear_bwd_workspace_bytes(n_rows, channels, features);
  if (product == 0) return AERIS_ERR_INVALID_SHAPE;
  b.wgrad = round256((size_t)n_rows * channels * 2);
  const size_t values = round256((size_t)n_rows * features);
  const size_t for_dx = want_dx ? values + round256((size_t)n_rows * scale_pitch(features)) : 0;
  const size_t for_dw = want_dw ? b.wgrad + product : 0;
  b.dy = want_dw && for_dx <= product ? b.wgrad : 0;
  b.dys = b.dy + values;
  b.bytes = for_dw > for_dx ? for_dw : for_dx;
  return AERIS_OK;
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

extern "C" int aeris_linear_fp8_plan(int64_t n_rows, int32_t channels, int32_t out_features, int32_t* tile,
                                     int32_t* in_turn) {
  if (!tile || !in_turn) return AERIS_ERR_NULL_POINTER;
  if (const int rc = check_linear(n_rows, channels, out_features)) return rc;
  const LinearTile t = choose_linear(n_rows, channels, out_features);
  *tile = t == LinearTile::kLarge ? 256
          : t == LinearTile::kMedium || t == LinearTile::kMediumShared ? 128
          : t == LinearTile::kRows ? 16 : 64;
  *in_turn = t == LinearTile::kLarge && interleave_large(n_rows, out_features);
  return AERIS_OK;
}

extern "C" int aeris_linear_fp8_parts(int64_t n_rows, int32_t channels, int32_t out_features, int32_t* parts) {
  if (!parts) return AERIS_ERR_NULL_POINTER;
  if (const int rc = check_linear(n_rows, channels, out_features)) return rc;
  const LinearTile t = choose_linear(n_rows, channels, out_features);
  *parts = t == LinearTile::kRows ? kRowsWaves
           : t == LinearTile::kSmallShared ? kSmallGroups
           : t == LinearTile::kMediumShared ? kMediumGroups : 1;
  return AERIS_OK;
}

extern "C" size_t aeris_linear_fp8_bwd_workspace_bytes_for(int64_t n_rows, int32_t channels, int32_t out_features,
                                                           int32_t want_dx, int32_t want_dweight) {
  Backward at;
  if (backward_layout(n_rows, channels, out_features, want_dx != 0, want_dweight != 0, at) != AERIS_OK) return 0;
  return at.bytes;
}

extern "C" size_t aeris_linear_fp8_bwd_workspace_bytes(int64_t n_rows, int32_t channels, int32_t out_features) {
  return aeris_linear_fp8_bwd_workspace_bytes_for(n_rows, channels, out_features, 1, 1);
}

extern "C" int aeris_linear_fp8_bwd(const void* x8, const void* xs, const void* wt8, const void* wts, const void* dy,
                                    int64_t n_rows, int32_t channels, int32_t out_features, void* dx, float* dweight,
                                    void* workspace, size_t workspace_bytes, void* hip_stream) {
  if (!dy || !workspace || (!dx && !dweight) || (dx && (!wt8 || !wts)) || (dweight && (!x8 || !xs)))
    return AERIS_ERR_NULL_POINTER;
  Backward at;
  if (const int rc = backward_layout(n_rows, channels, out_features, dx != nullptr, dweight != nullptr, at))
    return rc;
  if (bad16(x8) || bad16(xs) || bad16(wt8) || bad16(wts) || bad16(dy) || bad16(dx) || bad16(dweight) ||
      bad16(workspace))
    return AERIS_ERR_MISALIGNED;
  if (workspace_bytes < at.bytes) return AERIS_ERR_WORKSPACE_TOO_SMALL;
  const hipStream_t st = static_cast<hipStream_t>(hip_stream);
  unsigned char* space = static_cast<unsigned char*>(workspace);
  const unsigned char *q = static_cast<const unsigned char*>(x8), *qs = static_cast<const unsigned char*>(xs);
  bf16_t* const x = reinterpret_cast<bf16_t*>(space);
  // one launch for the operands of both products where they do not share memory: 2 us less on the host
  const bool together = dx && dweight && at.dy != 0;
  if (together && launch_fp8_backward_operands(static_cast<const bf16_t*>(dy), out_features, space + at.dy,
                                               space + at.dys, q, qs, channels, x, n_rows, st) != 0)
    return AERIS_ERR_HIP_LAUNCH;
  if (dx) {
    if (!together && launch_fp8_quantize_rows(dy, false, n_rows, out_features, space + at.dy, space + at.dys, st) != 0)
      return AERIS_ERR_HIP_LAUNCH;
    if (const int rc = aeris_linear_fp8_fwd(space + at.dy, space + at.dys, wt8, wts, n_rows, out_features, channels, dx,
                                            hip_stream))
      return rc;
  }
  if (dweight) {
    if (!together && launch_fp8_dequantize(q, qs, n_rows, channels, x, st) != 0) return AERIS_ERR_HIP_LAUNCH;
    return aeris_linear_bwd(x, nullptr, dy, n_rows, channels, out_features, nullptr, dweight, space + at.wgrad,
                            workspace_bytes - at.wgrad, hip_stream);
  }
  return AERIS_OK;
}
