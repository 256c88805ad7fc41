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
  int t, h, w, t0, y0, x0;
  int first;  // first token of the grid within the launch
};

struct RopeArgs {
  double freq[kMaxPairs];   // turns per position unit of each pair
  uint8_t axis[kMaxPairs];  // the axis of each pair
  int pairs, axes;
  int tokens;               // of this launch
  int n_grids, merge;       // n_grids == 0: positions from `pos`
  const int* pos;           // axis ax, token k: pos[ax * axis_stride + k * token_stride]
  long axis_stride, token_stride;
  float* table;             // [tokens][pairs][2]
  RopeGrid grid[kGridsPerLaunch];
};
static_assert(sizeof(RopeArgs) <= 4096, "kernel arguments");

// Fills freq, axis, pairs and axes; false for a description out of range.
bool rope_pairs(const incvit_rope& r, RopeArgs& a);
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
  long rows;
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

hipError_t launch_qk(const QkArgs& a, hipStream_t s);
hipError_t launch_qk_layer(const QkLayerArgs& a, int rows, hipStream_t s);

}  // namespace incvit
