// Partial results of a row tile's shares of keys joined into rows of the output:
//   m = max m_s,  l = sum 2^(m_s - m) l_s,  out = sum 2^(m_s - m) O_s / l
// in the order of the shares.  A thread has 4 dims of a row.  Row tiles whose keys
// were one workgroup's are there already.
#include "attend.hpp"

namespace incvit {

namespace {

// cached: whether key tiles are those of the cache (lens) or of given keys
template <class T, int DS, bool CACHED>
__global__ __launch_bounds__(256) void attend_join_kernel(AttendArgs a) {
  const int TR = 1 << a.row_log;
  const int h = blockIdx.x % a.hk, f = blockIdx.x / a.hk;
  RowTile w;
  if (!row_tile(a, f, w)) return;
  w.len = CACHED ? cached_len(a, w.seq) : plain_len(a, w);
  const int shares = key_shares(a, key_tiles(a, w).nt);
  if (shares < 2) return;
  const int rows = min(TR, w.q_len * a.group - w.first);
  const float* part = a.parts + (size_t)((long)f * a.hk + h) * a.splits * TR * (DS + 2);
  const int i = blockIdx.y * 256 + threadIdx.x;
  const int r = i / (DS / 4), d = (i - r * (DS / 4)) * 4;
  if (r >= rows || d >= a.d) return;
  float m = -INFINITY;
  for (int s = 0; s < shares; ++s) m = fmaxf(m, gbl(part)[(size_t)s * TR * (DS + 2) + 2 * r]);
  float l = 0.0f;
  f32x4_t o = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll 4
  for (int s = 0; s < shares; ++s) {
    const float* p = part + (size_t)s * TR * (DS + 2);
    const u32x2_t ml = *(const INCVIT_GLOBAL u32x2_t*)(p + 2 * r);
    const f32x4_t v = *(const INCVIT_GLOBAL f32x4_t*)(p + 2 * TR + r * DS + d);
    const float ms = __uint_as_float(ml[0]), e = ms == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(ms - m);
    l += e * __uint_as_float(ml[1]);
    o += v * e;
  }
  const int row = w.first + r, tok = row / a.group, head = h * a.group + row - tok * a.group;
  const float inv = 1.0f / l;
  float y[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) y[j] = m == -INFINITY ? 0.0f : o[j] * inv;
  store_out4<T>(static_cast<T*>(const_cast<void*>(a.out.p)) + (w.q0 + tok) * a.out.row + (long)head * a.out.head + d, y);
}

template <class T, int DS>
hipError_t launch_ds(const AttendArgs& a, hipStream_t s) {
  const dim3 grid((unsigned)((long)a.tiles * a.hk), (std::min(1 << a.row_log, a.most_rows) * (DS / 4) + 255) / 256);
  return a.lens ? launch_k(attend_join_kernel<T, DS, true>, grid, dim3(256), 0, s, a)
                : launch_k(attend_join_kernel<T, DS, false>, grid, dim3(256), 0, s, a);
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
  if (a.splits < 2) return hipSuccess;
  return dtype == INCVIT_BF16 ? launch_t<uint16_t>(a, s) : launch_t<float>(a, s);
}

}  // namespace incvit
