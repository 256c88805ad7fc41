// Cosines and sines of rotary positions with one to three axes.
//
// A pair's angle is position * f.  In turns (f / 2 pi) it is formed in fp64,
// where the product of an int32 position has 21 bits to spare over fp32, and
// reduced exactly to a quarter turn q and a rest in [-1/8, 1/8] of a turn; the
// rest's sine and cosine are Taylor polynomials in fp32 (|x| <= pi/4: the first
// dropped terms are 1.8e-9 and 1.2e-10), swapped and signed by q.
//
// Bound: the table's bytes (8 per token and pair), and for a single frame the
// launch.  A thread forms one pair; a wave's 64 pairs are 512 consecutive bytes.
#include <cmath>

#include "ops.hpp"

namespace incvit {

__device__ __forceinline__ float2 cos_sin_turns(double turns) {
  const double k = rint(4.0 * turns);
  const float x = (float)((turns - 0.25 * k) * 6.283185307179586);
  const int quarter = (int)(long)k & 3;
  const float x2 = x * x;
  float s = fmaf(x2, 2.7557319e-6f, -1.9841270e-4f);
  s = fmaf(x2, s, 8.3333333e-3f);
  s = fmaf(x2, s, -1.6666667e-1f);
  s = fmaf(x * x2, s, x);
  float c = fmaf(x2, -2.7557319e-7f, 2.4801587e-5f);
  c = fmaf(x2, c, -1.3888889e-3f);
  c = fmaf(x2, c, 4.1666667e-2f);
  c = fmaf(x2, c, -0.5f);
  c = fmaf(x2, c, 1.0f);
  const bool swap = quarter & 1;
  const float cs = swap ? s : c, sn = swap ? c : s;
  return make_float2(quarter == 1 || quarter == 2 ? -cs : cs, quarter >= 2 ? -sn : sn);
}

// The position of token `tok` of the launch on axis `ax`.
__device__ __forceinline__ double grid_position(const RopeArgs& a, int tok, int ax) {
  int g = 0;
  for (int i = 1; i < a.n_grids; ++i) g = tok >= a.grid[i].first ? i : g;
  const RopeGrid& r = a.grid[g];
  const int m = a.merge, hw = r.h * r.w;
  const int local = tok - r.first, f = local / hw, in = local - f * hw;
  // window row, window, row and column inside it
  const int band = in / (m * r.w), b = in - band * m * r.w;
  const int win = b / (m * m), c = b - win * m * m;
  const int y = band * m + c / m, x = win * m + c % m;
  if (a.axes == 1) return (double)r.t0 + (double)f * hw + (double)y * r.w + x;
  const int which = ax + 3 - a.axes;
  return which == 0 ? (double)r.t0 + f : which == 1 ? (double)r.y0 + y : (double)r.x0 + x;
}

__global__ __launch_bounds__(256) void rope_kernel(RopeArgs a) {
  const int total = a.tokens * a.pairs;
  for (long e = (long)blockIdx.x * 256 + threadIdx.x; e < total; e += (long)gridDim.x * 256) {
    const int tok = (int)e / a.pairs, p = (int)e - tok * a.pairs;
    const int ax = a.axis[p];
    const double pos = a.n_grids ? grid_position(a, tok, ax) : (double)a.pos[ax * a.axis_stride + tok * a.token_stride];
    reinterpret_cast<float2*>(a.table)[e] = cos_sin_turns(pos * a.freq[p]);
  }
}

hipError_t launch_rope(const RopeArgs& a, hipStream_t s) {
  const long blocks = ((long)a.tokens * a.pairs + 255) / 256;
  return launch_k(rope_kernel, dim3((unsigned)std::min<long>(blocks, 4096)), dim3(256), 0, s, a);
}

bool rope_pairs(const incvit_rope& r, RopeArgs& a) {
  if (r.axes < 1 || r.axes > 3) return false;
  if ((r.ladder != INCVIT_LADDER_AXIS && r.ladder != INCVIT_LADDER_HEAD) ||
      (r.layout != INCVIT_LAYOUT_BLOCKS && r.layout != INCVIT_LAYOUT_CYCLE))
    return false;
  if (!(r.theta >= 1.0 && r.theta <= 1e12)) return false;
  int n = 0;
  for (int x = 0; x < r.axes; ++x) {
    if (r.pairs[x] < 1 || r.pairs[x] > kMaxPairs) return false;
    if (!(std::fabs(r.scale[x]) <= 1048576.0) || r.scale[x] == 0.0) return false;
    n += r.pairs[x];
  }
  if (n > kMaxPairs) return false;
  a.axes = r.axes;
  a.pairs = n;
  int taken[3] = {0, 0, 0}, ax = 0;
  for (int i = 0; i < n; ++i) {
    while (taken[ax] == r.pairs[ax]) ax = (ax + 1) % r.axes;
    const double e = r.ladder == INCVIT_LADDER_AXIS ? (double)taken[ax] / r.pairs[ax] : (double)i / n;
    a.axis[i] = (uint8_t)ax;
    a.freq[i] = r.scale[ax] * std::pow(r.theta, -e) / 6.283185307179586476925;
    ++taken[ax];
    if (r.layout == INCVIT_LAYOUT_CYCLE) ax = (ax + 1) % r.axes;
  }
  return true;
}

}  // namespace incvit
