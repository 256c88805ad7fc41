// Arguments and launchers of the stand-alone operators (rotary tables, head
// norms with the rotation, 8-bit products), which the encoder calls too.
#pragma once

#include "common.hpp"
#include "incvit.h"

namespace incvit {

// Refusals of entry points without a handle: sets incvit_last_error(NULL).
incvit_status op_fail(incvit_status st, const char* msg);

// ------------------------------------------------------- rotary positions --

constexpr int kMaxPairs = 128;   // pairs of one head: head dims up to 256
constexpr int kGridsPerLaunch = 32;

struct RopeGrid {
  double per_frame, per_band;  // 1 / (h w), 1 / (merge w)
  int h, w, t0, y0, x0;
  int first;  // first token of the grid within the launch
};

struct RopeArgs {
  double freq[kMaxPairs];   // turns per position unit of each pair
  uint8_t axis[kMaxPairs];  // the axis of each pair
  int pairs, axes;
  int tokens;               // of this launch
  int n_grids, merge;       // n_grids == 0: positions from `pos`
  double per_window, per_side, per_token;  // 1 / merge^2, 1 / merge, 1 / threads of a token
  const int* pos;           // axis ax, token k: pos[ax * axis_stride + k * token_stride]
  long axis_stride, token_stride;
  float* table;             // [tokens][pairs][2]
  RopeGrid grid[kGridsPerLaunch];
};
static_assert(sizeof(RopeArgs) <= 4096, "kernel arguments");

// Fills freq, axis, pairs and axes; false for a description out of range.
bool rope_pairs(const incvit_rope& r, RopeArgs& a);
// The i-th grid of a launch, whose tokens follow those before it.
void rope_grid(RopeArgs& a, int i, const incvit_grid& g);
hipError_t launch_rope(const RopeArgs& a, hipStream_t s);

// ------------------------------------------- head norms with the rotation --

struct QkSide {
  const void* in;
  void* out;
  const void* gamma;  // [head_dim] storage type, or null: ones
  const void* beta;   // likewise, or null: zeros
  long in_row, in_head, out_row, out_head;  // strides in elements
  int heads;
};

struct QkArgs {
  QkSide q, k;
  int dtype, head_dim, rot_pairs, adjacent, norm;
  float eps;
  long rows;           // all of the call's
  long row0;           // the launch's first
  const float* table;  // [table_rows][rot_pairs][2]
  long table_rows;
  const int* index;    // [rows] table row of a row, or null: r % table_rows
  const int* k_rows;   // [rows] row of k.out, or null: r
  long k_out_rows;
};

// One layer of an encode call: the compact query rows in place, the keys of
// the same rows in place in their caches (operand order).
struct QkLayerArgs {
  const RowInfo* rows;
  const Meta* meta;
  Shape sh;
  CacheLayout cl;
  int layer;
  void* q;             // [Mpad][D]
  const float* q_gamma;  // [d_h], null without a norm
  const float* q_beta;
  const float* k_gamma;
  const float* k_beta;
  const float* table;    // [N][d_h / 2][2], null without rotation
  int adjacent, norm;
  float eps;
};

// ----------------------------------------------------------- 8-bit products --

// Operands of the 8-bit matrix instruction (16 x 16 x 64): 16 rows (or weight
// columns) by 64 values of K are one kilobyte, in which lane 16 g + n holds the
// 16 values k = 16 g .. 16 g + 15 of row n.  kc: chunks of 64 along K.
__host__ __device__ __forceinline__ size_t q_off(int r, int k, int kc) {
  return ((size_t)(r >> 4) * kc + (k >> 6)) * 1024 + ((k >> 4) & 3) * 256 + (r & 15) * 16 + (k & 15);
}

__host__ __device__ constexpr size_t q_align(size_t x) { return (x + 255) / 256 * 256; }

// Quantised rows: the operand kilobytes of ceil(rows / 16) row tiles, then the
// rows' scales.
struct QRowsLayout {
  int kc;
  size_t scale, total;
  __host__ __device__ QRowsLayout(long rows, int K) : kc((K + 63) / 64) {
    const size_t tiles = (size_t)(rows + 15) / 16;
    scale = q_align(tiles * kc * 1024);
    total = scale + q_align(tiles * 64);
  }
};
// Packed weights: the operand kilobytes of ceil(N / 16) column blocks, then the
// columns' scales and biases (fp32, zero past N).
struct QWeightsLayout {
  int kc, blocks;
  size_t scale, bias, total;
  __host__ __device__ QWeightsLayout(int K, int N) : kc((K + 63) / 64), blocks((N + 15) / 16) {
    scale = q_align((size_t)blocks * kc * 1024);
    bias = scale + q_align((size_t)blocks * 64);
    total = bias + q_align((size_t)blocks * 64);
  }
};

struct QPackArgs {
  const void* w;        // value (k, n) at k * wk + n * wn
  long wk, wn;
  const float* scales;  // given scales (int8 weights), else null
  const void* bias;     // [N], or null
  char* dst;            // QWeightsLayout
  int K, N, dtype;      // dtype 2: int8 weights, fp32 bias
};

struct QRowsArgs {
  const void* x;        // [rows][ld], or with `frag` 16 x 32 operand order (frag_off) of `ld` columns
  long ld;
  const void* gamma;    // LayerNorm before the quantisation: of the rows' type, or null;
  const void* beta;     // with `frag` fp32, 16-byte aligned and both there
  float eps;
  char* dst;            // QRowsLayout's kilobytes
  float* scale;
  const Meta* meta;     // rows on the device, or null
  long rows;
  int K, dtype, frag;
};

hipError_t launch_q_pack(const QPackArgs& a, hipStream_t s);
hipError_t launch_q_rows(const QRowsArgs& a, hipStream_t s);
// out = act(rows x weights) (+ resid): `expected` rows to tune for, at most `rows`
hipError_t launch_q_gemm(const GemmArgs& a, int out_f32, int expected, int rows, hipStream_t s);
// A few rows quantised and multiplied in one launch (a.A = the rows): for which
// sizes, and the launch.
bool q_token_fits(int64_t rows, int K);
hipError_t launch_q_token(const GemmArgs& a, int f32, hipStream_t s);
// the encoder's down projection: out = S(resid + S(rows x weights + bias)), both in
// operand order, also written to the cache's X^{layer + 1}
hipError_t launch_q_down(const GemmArgs& a, int out_f32, int expected, int rows, hipStream_t s);

hipError_t launch_qk(const QkArgs& a, hipStream_t s);
hipError_t launch_qk_layer(const QkLayerArgs& a, int rows, hipStream_t s);

}  // namespace incvit

#if defined(__HIPCC__)
namespace incvit {

template <int CTRL>
__device__ __forceinline__ uint32_t dpp(uint32_t x) {
  return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, CTRL, 0xf, 0xf, false);
}

// op over the GL lanes (a power of two from 4 on, aligned) that share a value's
// work; every lane gets the result, the same bits.  Neighbours and quads by
// quad permutes, then mirrors of 8 and 16 lanes (whose halves hold one value
// each by then), then gfx950's swaps of 16 and of 32: no trip through LDS.
template <int GL, class Op>
__device__ __forceinline__ uint32_t lanes_join(uint32_t x, Op op) {
  x = op(x, dpp<0xb1>(x));
  x = op(x, dpp<0x4e>(x));
  if constexpr (GL >= 8) x = op(x, dpp<0x141>(x));
  if constexpr (GL >= 16) x = op(x, dpp<0x140>(x));
  if constexpr (GL >= 32) {
    const auto p = __builtin_amdgcn_permlane16_swap(x, x, false, false);
    x = op(p[0], p[1]);
  }
  if constexpr (GL >= 64) {
    const auto p = __builtin_amdgcn_permlane32_swap(x, x, false, false);
    x = op(p[0], p[1]);
  }
  return x;
}
template <int GL>
__device__ __forceinline__ float lanes_sum(float x) {
  return __uint_as_float(lanes_join<GL>(__float_as_uint(x), [](uint32_t a, uint32_t b) {
    return __float_as_uint(__uint_as_float(a) + __uint_as_float(b));
  }));
}
template <int GL>
__device__ __forceinline__ uint32_t lanes_max(uint32_t x) {
  return lanes_join<GL>(x, [](uint32_t a, uint32_t b) { return a > b ? a : b; });
}

}  // namespace incvit
#endif
