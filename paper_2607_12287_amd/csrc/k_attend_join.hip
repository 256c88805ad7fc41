// Partial results of a row's shares of keys joined into the output:
//   m = max m_s,  l = sum 2^(m_s - m) l_s,  out = sum 2^(m_s - m) O_s / l.
// A workgroup has a row: its threads take the shares' weights together, then 4 dims
// each of every (1024 / DS)-th share, and add those through LDS, in a fixed order.
// Row tiles whose keys were one workgroup's are there already.  Where row tiles are
// large, and their shares few, a thread has 4 dims of a row and all of its shares.
//
// 5.0 us behind 32 decoding sequences in 416 shares, 8.5 behind 1024 rows in 4 (34 MB of parts:
// 4.0 TB/s).  All shares in one thread for decoding rows too:
// one sequence of 131072 keys 113 us instead of 32.
#include "attend.hpp"

namespace incvit {

namespace {

template <class T, int DS>
__global__ __launch_bounds__(256) void attend_join_kernel(AttendArgs a) {
  constexpr int Q = DS / 4, PARTS = 256 / Q;  // threads of a part, and parts (192 dims: 5 of 48, the rest idle)
  __shared__ float s_e[kMostShares], s_m[4], s_l[4];
  __shared__ f32x4_t s_o[PARTS][Q];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int h = blockIdx.x % a.hk, f = blockIdx.x / a.hk, r = blockIdx.y;
  RowTile w;
  Share sh;
  if (!shares_of(a, f, w, sh) || sh.n < 2 || w.first + r >= w.q_len * a.group) return;
  const int shares = sh.n;
  const size_t step = (size_t)(DS + 2) << a.row_log;
  const float* part = a.parts + (size_t)(sh.slot * a.hk + h) * step;
  float m = -INFINITY, l = 0.0f;
  if (tid < shares) {
    const u32x2_t ml = *(const INCVIT_GLOBAL u32x2_t*)(part + tid * a.hk * step + 2 * r);
    m = __uint_as_float(ml[0]);
    l = __uint_as_float(ml[1]);
  }
  const float top = wave_max(m);
  if (lane == 0) s_m[wave] = top;
  __syncthreads();
  const float mm = fmaxf(fmaxf(s_m[0], s_m[1]), fmaxf(s_m[2], s_m[3]));
  const float e = m == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(m - mm);
  s_e[tid] = e;
  const float sum = wave_sum(e * l);
  if (lane == 0) s_l[wave] = sum;
  __syncthreads();
  const int p = tid / Q, d = (tid - p * Q) * 4;
  f32x4_t o = {0.0f, 0.0f, 0.0f, 0.0f};
  if (p < PARTS) {
    const float* at = part + ((size_t)2 << a.row_log) + (size_t)r * DS + d;
#pragma unroll 8
    for (int s = p; s < shares; s += PARTS) o += *(const INCVIT_GLOBAL f32x4_t*)(at + s * a.hk * step) * s_e[s];
    s_o[p][d / 4] = o;
  }
  __syncthreads();
  if (p != 0 || d >= a.d) return;
#pragma unroll
  for (int k = 1; k < PARTS; ++k) o += s_o[k][d / 4];
  const float inv = 1.0f / (s_l[0] + s_l[1] + s_l[2] + s_l[3]);
  const int row = w.first + r, tok = row / a.group, head = h * a.group + row - tok * a.group;
  float y[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) y[j] = mm == -INFINITY ? 0.0f : o[j] * inv;
  store_out4<T>(static_cast<T*>(const_cast<void*>(a.out.p)) + (w.q0 + tok) * a.out.row + (long)head * a.out.head + d, y);
}

template <class T, int DS>
__global__ __launch_bounds__(256) void attend_join_rows_kernel(AttendArgs a) {
  constexpr int Q = DS / 4, ROWS = 256 / Q;  // rows of a workgroup
  const int h = blockIdx.x % a.hk, f = blockIdx.x / a.hk;
  const int at = threadIdx.x / Q, r = blockIdx.y * ROWS + at, d = (threadIdx.x - at * Q) * 4;
  RowTile w;
  Share sh;
  if (!shares_of(a, f, w, sh) || sh.n < 2) return;
  if (at >= ROWS || d >= a.d || r >= min(1 << a.row_log, w.q_len * a.group - w.first)) return;
  const size_t step = ((size_t)(DS + 2) << a.row_log) * a.hk;
  const float* part = a.parts + ((size_t)(sh.slot * a.hk + h) << a.row_log) * (DS + 2);
  const float* row = part + ((size_t)2 << a.row_log) + (size_t)r * DS + d;
  float m = -INFINITY, l = 0.0f;
#pragma unroll 4
  for (int s = 0; s < sh.n; ++s) m = fmaxf(m, gbl(part)[s * step + 2 * r]);
  f32x4_t o = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll 4
  for (int s = 0; s < sh.n; ++s) {
    const u32x2_t ml = *(const INCVIT_GLOBAL u32x2_t*)(part + s * step + 2 * r);
    const f32x4_t x = *(const INCVIT_GLOBAL f32x4_t*)(row + s * step);
    const float ms = __uint_as_float(ml[0]), e = ms == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(ms - m);
    l += e * __uint_as_float(ml[1]);
    o += x * e;
  }
  const float inv = 1.0f / l;
  const int n = w.first + r, tok = n / a.group, head = h * a.group + n - tok * a.group;
  float y[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) y[j] = m == -INFINITY ? 0.0f : o[j] * inv;
  store_out4<T>(static_cast<T*>(const_cast<void*>(a.out.p)) + (w.q0 + tok) * a.out.row + (long)head * a.out.head + d, y);
}

template <class T, int DS>
hipError_t launch_ds(const AttendArgs& a, hipStream_t s) {
  const int rows = std::min(1 << a.row_log, a.most_rows);
  if (a.row_log > 5) {
    constexpr int each = 256 / (DS / 4);
    return launch_k(attend_join_rows_kernel<T, DS>, dim3((unsigned)((long)a.tiles * a.hk), (rows + each - 1) / each), dim3(256), 0, s, a);
  }
  const dim3 grid((unsigned)((long)a.tiles * a.hk), rows);
  return launch_k(attend_join_kernel<T, DS>, grid, dim3(256), 0, s, a);
}

template <class T>
hipError_t launch_t(const AttendArgs& a, hipStream_t s) {
  switch (kv_dims(a.d)) {
    case 32: return launch_ds<T, 32>(a, s);
    case 64: return launch_ds<T, 64>(a, s);
    case 80: return launch_ds<T, 80>(a, s);
    case 96: return launch_ds<T, 96>(a, s);
    case 128: return launch_ds<T, 128>(a, s);
    case 192: return launch_ds<T, 192>(a, s);
    default: return launch_ds<T, 256>(a, s);
  }
}

}  // namespace

hipError_t launch_attend_join(const AttendArgs& a, int dtype, hipStream_t s) {
  if (a.splits < 2 && !a.even) return hipSuccess;
  return dtype == INCVIT_BF16 ? launch_t<uint16_t>(a, s) : launch_t<float>(a, s);
}

}  // namespace incvit
