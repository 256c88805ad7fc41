// Cosines and sines of rotary positions with one to three axes.
//
// A pair's angle is position * f.  In turns (f / 2 pi) it is formed in fp64,
// where the product of an int32 position has 21 bits to spare over fp32, and
// reduced exactly to a quarter turn q and a rest in [-1/8, 1/8] of a turn; the
// rest's sine and cosine are Taylor polynomials in fp32 (|x| <= pi/4: the first
// dropped terms are 1.8e-9 and 1.2e-10), swapped and signed by q.
//
// Bound: for a few thousand tokens the launch (256 tokens of 36 pairs 3.4 us in
// a trace); then the tokens' places and the table's bytes (8 per token and
// pair).  A 6.7 MB table of video grids takes 4.7 us in a graph: 1.0 of it for the
// places (3.75 without), 0.3 for sines and cosines (4.4 without), while a fill of
// the bytes takes 2.7.  A thread forms two pairs of one token, 16 bytes, and finds
// the token's place in its grid by products with reciprocals in fp64.
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

// n / d for 0 <= n < 2^31 and per = 1 / d in fp64: (n + 1/2) / d is at least
// 1 / 2d from a whole number, 2^20 times the product's error.
__device__ __forceinline__ int divided(int n, double per) { return (int)(((double)n + 0.5) * per); }

// The positions of token `tok` of the launch, in the last `axes` of x.
__device__ __forceinline__ void grid_position(const RopeArgs& a, int tok, double (&x)[3]) {
  int g = 0;
  for (int i = 1; i < a.n_grids; ++i) g = tok >= a.grid[i].first ? i : g;
  const RopeGrid r = a.grid[g];
  const int m = a.merge, hw = r.h * r.w;
  const int local = tok - r.first, f = divided(local, r.per_frame), in = local - f * hw;
  // window row, window, row and column inside it
  const int band = divided(in, r.per_band), b = in - band * m * r.w;
  const int win = divided(b, a.per_window), c = b - win * m * m, cy = divided(c, a.per_side);
  const int row = band * m + cy, col = win * m + c - cy * m;
  x[0] = (double)r.t0 + f;
  x[1] = (double)r.y0 + row;
  x[2] = a.axes == 1 ? (double)r.t0 + (double)f * hw + (double)row * r.w + col : (double)r.x0 + col;
}

// VEC: pairs are even and the table 16-byte aligned.
template <bool VEC>
__global__ __launch_bounds__(256) void rope_kernel(RopeArgs a) {
  const int per = (a.pairs + 1) / 2;  // threads of a token
  const uint32_t total = (uint32_t)a.tokens * per;
  for (uint32_t e = blockIdx.x * 256 + threadIdx.x; e < total; e += gridDim.x * 256) {
    const int tok = divided((int)e, a.per_token), p0 = 2 * ((int)e - tok * per);
    double x[3] = {0.0, 0.0, 0.0};
    if (a.n_grids) {  // uniform
      grid_position(a, tok, x);
    } else {
#pragma unroll
      for (int i = 0; i < 3; ++i) {
        const int ax = i - 3 + a.axes;
        if (ax >= 0) x[i] = (double)a.pos[ax * a.axis_stride + tok * a.token_stride];  // uniform
      }
    }
    float2 t[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int p = min(p0 + i, a.pairs - 1), ax = a.axis[p] + 3 - a.axes;
      t[i] = cos_sin_turns((ax == 0 ? x[0] : ax == 1 ? x[1] : x[2]) * a.freq[p]);
    }
    float2* out = reinterpret_cast<float2*>(a.table) + (size_t)tok * a.pairs + p0;
#pragma unroll
    for (int i = 0; i < 2; i += 2) {
      if (VEC) {
        if (p0 + i < a.pairs) *reinterpret_cast<float4*>(out + i) = make_float4(t[i].x, t[i].y, t[i + 1].x, t[i + 1].y);
      } else {
        if (p0 + i < a.pairs) out[i] = t[i];
        if (p0 + i + 1 < a.pairs) out[i + 1] = t[i + 1];
      }
    }
  }
}

void rope_grid(RopeArgs& a, int i, const incvit_grid& g) {
  const int first = i == 0 ? 0 : a.tokens;
  a.grid[i] = RopeGrid{1.0 / ((double)g.h * g.w), 1.0 / ((double)a.merge * g.w), g.h, g.w, g.t0, g.y0, g.x0, first};
  a.n_grids = i + 1;
  a.tokens = first + g.t * g.h * g.w;
}

hipError_t launch_rope(const RopeArgs& a0, hipStream_t s) {
  RopeArgs a = a0;
  a.per_token = 1.0 / ((a.pairs + 1) / 2);
  if (a.n_grids) {
    a.per_side = 1.0 / a.merge;
    a.per_window = 1.0 / ((double)a.merge * a.merge);
  }
  const long blocks = ((long)a.tokens * ((a.pairs + 1) / 2) + 255) / 256;
  const dim3 grid((unsigned)std::min<long>(blocks, 8192));
  if (a.pairs % 2 == 0 && (uintptr_t)a.table % 16 == 0) return launch_k(rope_kernel<true>, grid, dim3(256), 0, s, a);
  return launch_k(rope_kernel<false>, grid, dim3(256), 0, s, a);
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
