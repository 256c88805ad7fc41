// 8-bit products with a scale for each row (token) and each column (channel):
//   out = act(sum_k q_mk w_kn * (s_m s_n) + b_n) + resid
// with q = round(x / s), s = max |x| / 127 over a row's K values, and likewise
// for the columns of W.  Sums of 8-bit products are exact in int32 (K <= 65536).
//
// The kernels (us of a launch within a graph on an MI355X, bf16):
//   * q_rows_kernel: one or four waves per row find its largest magnitude and
//     write the row's integers in the matrix instruction's operand order (with a
//     LayerNorm before it, whose statistics are two passes over registers).
//     8192 x 1024 7.2 us (3.5 TB/s; fp32 9.1 and 4.6, a copy 5.1), behind a LayerNorm
//     9.8; 8192 x 4096 27 and 39; 1024 x 4304 5.3 and 8.2; 23 x 1152 2.5 and 3.9 (latency).
//     Counters give each byte read and written once;
//   * q_tile_kernel: the same for the encoder's rows in operand order;
//   * q_gemm_kernel, few rows: weights stream past them once.  A workgroup owns
//     16 columns; its waves take the K chunks in turn, so every wave has loads of
//     its own in flight, and add their int32 partial tiles through LDS (in any
//     order: integer sums are exact).  Bound by the weights' bytes and the
//     latency of the loads: 64 x 1152 -> 4304 3.8 us;
//   * q_token_kernel: up to 8 rows, which every workgroup quantises for itself;
//   * the large-row GEMM (gemm_tiled.hpp) otherwise.
#include "gemm_tiled.hpp"
#include "ops.hpp"

namespace incvit {

namespace {

// ------------------------------------------------------------- quantisation --

// scale of a largest magnitude given as fp32 bits; NaN where it is not finite
__device__ __forceinline__ float q_scale(uint32_t top) {
  const float s = __fdiv_rn(__uint_as_float(top), 127.0f);
  return top >= 0x7f800000u ? __uint_as_float(0x7fc00000u) : s;
}
// x / s, rounded to fp32, then to the nearest integer (ties to even); 0 for a
// row of zeros, and for one whose scale is NaN
__device__ __forceinline__ int q_value(float x, float s) {
  const float r = rintf(__fdiv_rn(x, s));
  return s > 0.0f ? (int)fminf(fmaxf(r, -127.0f), 127.0f) : 0;
}
// The same in the low byte of the result, without a division, for scales whose
// reciprocal and quotients stay normal (q_plain).  inv = 1 / s, correctly
// rounded: x * inv is within 2 ulp of the quotient, one residual step makes it
// faithful and the second correctly rounded (Markstein's theorem: a faithful
// quotient, its exact residual and the correctly rounded reciprocal).  With x
// and the row's largest magnitude bf16 numbers (BF), one step gives the same
// integer, which a test shows for every pair of their significands.  Adding
// 1.5 * 2^23 rounds to an integer, ties to even, in the low bits; |x / s| is
// below 127.5, so no clamp.
__device__ __forceinline__ bool q_plain(float s) { return s > 0x1p-90f && s < 0x1p90f; }
template <bool BF>
__device__ __forceinline__ uint32_t q_byte(float x, float s, float inv) {
  float q = x * inv;
  q = fmaf(fmaf(-q, s, x), inv, q);
  if (!BF) q = fmaf(fmaf(-q, s, x), inv, q);
  return __float_as_uint(q + 12582912.0f);
}
// low bytes of four words in one
__device__ __forceinline__ uint32_t low_bytes(uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
  return __builtin_amdgcn_perm(__builtin_amdgcn_perm(d, c, 0x0c0c0400u), __builtin_amdgcn_perm(b, a, 0x0c0c0400u), 0x05040100u);
}
__device__ __forceinline__ uint32_t mag(float x) { return __float_as_uint(x) & 0x7fffffffu; }

// 8 values from p on, or zeros: the load runs either way (p is readable), so that
// a lane's loads go out together.
template <class T>
__device__ __forceinline__ void load8(const T* p, bool any, float* v) {
  if constexpr (std::is_same<T, float>::value) {
    const f32x4_t a = *(const INCVIT_GLOBAL f32x4_t*)p, b = *(const INCVIT_GLOBAL f32x4_t*)(p + 4);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      v[i] = any ? a[i] : 0.0f;
      v[4 + i] = any ? b[i] : 0.0f;
    }
  } else {
    const u32x4_t u = *(const INCVIT_GLOBAL u32x4_t*)p;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint32_t w = any ? u[i] : 0u;
      v[2 * i] = __uint_as_float(w << 16);
      v[2 * i + 1] = __uint_as_float(w & 0xffff0000u);
    }
  }
}
// 8 values of a row of K from k on, zeros past K.  VEC: K % 8 == 0, 16-byte aligned.
template <class T, bool VEC>
__device__ __forceinline__ void row8(const T* row, int k, int K, float* v) {
  if constexpr (VEC) {
    load8<T>(row + min(k, K - 8), k < K, v);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const T x = *gbl(row + min(k + i, K - 1));
      v[i] = k + i < K ? Elem<T>::f(x) : 0.0f;
    }
  }
}

// Four rows to a workgroup, WPR waves to a row.  A lane holds 8 values of every
// 512 WPR in registers, CH times (K <= 512 WPR CH); longer rows (CH = 0) are
// read again for each pass.  The four rows' 16-byte pieces of a chunk are 64
// consecutive bytes.
template <class T, int CH, int WPR, bool VEC>
__global__ __launch_bounds__(256 * WPR) void q_rows_kernel(QRowsArgs a) {
  __shared__ float s_sum[4][WPR], s_sq[4][WPR];
  __shared__ uint32_t s_top[4][WPR];
  const int lane = threadIdx.x & 63;
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), wr = w / WPR, wk = w % WPR;
  const long r = (long)blockIdx.x * 4 + wr;
  const long rows = a.meta ? a.meta->m : a.rows;
  if ((long)blockIdx.x * 4 >= rows) return;  // uniform
  const bool live = r < rows;                // uniform per wave
  const int K = a.K, kc = (K + 63) / 64;
  const T* x = static_cast<const T*>(a.x);
  const T* row = x + (size_t)min(r, rows - 1) * a.ld;
  auto fetch = [&](int i, float* v) { row8<T, VEC>(row, 8 * (lane + 64 * (wk + WPR * i)), K, v); };  // the lane's i-th run of 8
  constexpr int NH = CH > 0 ? CH : 1;
  const int runs = CH > 0 ? CH : (kc * 8 + 64 * WPR - 1) / (64 * WPR);
  float held[NH][8];
  if constexpr (CH > 0) {
#pragma unroll
    for (int i = 0; i < CH; ++i) fetch(i, held[i]);
  }
  // f(its first k, its 8 values) for every run of the lane
  auto each = [&](auto f) {
    if constexpr (CH > 0) {
#pragma unroll
      for (int i = 0; i < CH; ++i) f(8 * (lane + 64 * (wk + WPR * i)), held[i]);
    } else {
      for (int i = 0; i < runs; ++i) {
        fetch(i, held[0]);
        f(8 * (lane + 64 * (wk + WPR * i)), held[0]);
      }
    }
  };
  // sums over the row's waves, in wave order
  auto row_sum = [&](float v, float (&sh)[4][WPR]) {
    v = lanes_sum<64>(v);
    if constexpr (WPR > 1) {
      if (lane == 0) sh[wr][wk] = v;
      __syncthreads();
      v = sh[wr][0];
#pragma unroll
      for (int i = 1; i < WPR; ++i) v += sh[wr][i];
    }
    return v;
  };
  float mean = 0.0f, rstd = 1.0f;
  const bool ln = a.gamma != nullptr;
  if (ln) {  // uniform
    float s = 0.0f, q = 0.0f;
    each([&](int, float* v) {
#pragma unroll
      for (int j = 0; j < 8; ++j) s += v[j];  // zeros past K
    });
    mean = row_sum(s, s_sum) / (float)K;
    each([&](int k, float* v) {
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const float d = v[j] - mean;
        q += k + j < K ? d * d : 0.0f;
      }
    });
    rstd = 1.0f / sqrtf(row_sum(q, s_sq) / (float)K + a.eps);
  }
  auto normed = [&](int k, float* v) {
    if (!ln) return;
    float gm[8], bt[8];
    row8<T, VEC>(static_cast<const T*>(a.gamma), k, K, gm);
#pragma unroll
    for (int j = 0; j < 8; ++j) bt[j] = 0.0f;
    if (a.beta) row8<T, VEC>(static_cast<const T*>(a.beta), k, K, bt);
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = k + j < K ? fmaf((v[j] - mean) * rstd, gm[j], bt[j]) : 0.0f;
  };
  uint32_t top = 0;
  each([&](int k, float* v) {
    normed(k, v);
#pragma unroll
    for (int j = 0; j < 8; ++j) top = max(top, mag(v[j]));
  });
  top = lanes_max<64>(top);
  if constexpr (WPR > 1) {
    if (lane == 0) s_top[wr][wk] = top;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < WPR; ++i) top = max(top, s_top[wr][i]);
  }
  if (!live) return;
  const float s = q_scale(top), inv = __fdiv_rn(1.0f, s);
  if (lane == 0 && wk == 0) a.scale[r] = s;
  auto write = [&](auto byte) {
    each([&](int k, float* v) {
      if constexpr (CH == 0) normed(k, v);
      if (k >= 64 * kc) return;
      uint32_t b[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) b[j] = byte(v[j]);
      *reinterpret_cast<uint2*>(a.dst + q_off((int)r, k, kc)) =
          make_uint2(low_bytes(b[0], b[1], b[2], b[3]), low_bytes(b[4], b[5], b[6], b[7]));
    });
  };
  // uniform per wave
  if (!q_plain(s)) write([&](float v) { return (uint32_t)q_value(v, s); });
  else if (sizeof(T) == 2 && !ln) write([&](float v) { return q_byte<true>(v, s, inv); });
  else write([&](float v) { return q_byte<false>(v, s, inv); });
}


// Rows in operand order (the encoder's H: 16 rows x 32 columns to a kilobyte of
// bf16, frag_off) behind their LayerNorm: a tile of 16 rows to a workgroup of NW waves.  Lane 16 g + n
// works on row n as the product will hold it, values 64 c + 16 g .. + 15 of the
// CI chunks c = w, w + NW, ... (K <= 64 NW CI), so a wave reads and writes whole
// runs of 256 bytes; a wave per row, as above, would use 16 bytes of every line
// that it touches (8192 rows of 1024: 33 us against 10).
template <class T, int NW, int CI>
__global__ __launch_bounds__(64 * NW) void q_tile_kernel(QRowsArgs a) {
  __shared__ uint32_t s_row[3][16][NW];
  __shared__ float4 s_gain[kMaxDim / 4], s_shift[kMaxDim / 4];
  const int lane = threadIdx.x & 63, g = lane >> 4, n = lane & 15;
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int K = a.K, kc = (K + 63) / 64;
  const long r = (long)blockIdx.x * 16 + n;
  // the first rows, the likely ones, load before the row count is read (the
  // compact rows are padded past every launched one); the LayerNorm's gains and
  // shifts (fp32) go to LDS beside them
  const bool ahead = blockIdx.x < 8;  // uniform
  if (!ahead && (long)blockIdx.x * 16 >= a.meta->m) return;
  float held[CI][16];
#pragma unroll
  for (int i = 0; i < CI; ++i)
#pragma unroll
    for (int h = 0; h < 2; ++h) {  // K % 32 == 0: a run of 8 is inside or outside as a whole
      const int k = 64 * (w + NW * i) + 16 * g + 8 * h;
      load8<T>(static_cast<const T*>(a.x) + frag_off((int)r, min(k, K - 8), (int)a.ld / 32), k < K, held[i] + 8 * h);
    }
  if ((int)threadIdx.x < K / 4) {
    s_gain[threadIdx.x] = static_cast<const float4*>(a.gamma)[threadIdx.x];
    s_shift[threadIdx.x] = static_cast<const float4*>(a.beta)[threadIdx.x];
  }
  const long rows = a.meta->m;
  if ((long)blockIdx.x * 16 >= rows) return;  // uniform
  const bool live = r < rows;
  // f(i, first k, the 16 values) for every chunk w + NW i of the wave
  auto each = [&](auto f) {
#pragma unroll
    for (int i = 0; i < CI; ++i) f(i, 64 * (w + NW * i) + 16 * g, held[i]);
  };
  // op over the values that the lanes of row n hold, in every wave, in a fixed order
  auto over_row = [&](uint32_t v, int slot, auto op) {
    const auto p = __builtin_amdgcn_permlane16_swap(v, v, false, false);
    v = op(p[0], p[1]);
    const auto q = __builtin_amdgcn_permlane32_swap(v, v, false, false);
    v = op(q[0], q[1]);
    if (g == 0) s_row[slot][n][w] = v;
    __syncthreads();
    v = s_row[slot][n][0];
#pragma unroll
    for (int i = 1; i < NW; ++i) v = op(v, s_row[slot][n][i]);
    return v;
  };
  auto add = [](uint32_t x, uint32_t y) { return __float_as_uint(__uint_as_float(x) + __uint_as_float(y)); };
  float s = 0.0f, q = 0.0f;
  each([&](int, int, float* v) {
#pragma unroll
    for (int j = 0; j < 16; ++j) s += v[j];  // zeros past K
  });
  const float mean = __uint_as_float(over_row(__float_as_uint(s), 0, add)) / (float)K;
  each([&](int, int k, float* v) {
#pragma unroll
    for (int j = 0; j < 16; ++j) {
      const float d = v[j] - mean;
      q += k < K ? d * d : 0.0f;  // K % 32 == 0
    }
  });
  const float rstd = 1.0f / sqrtf(__uint_as_float(over_row(__float_as_uint(q), 1, add)) / (float)K + a.eps);
  uint32_t top = 0;
  each([&](int, int k, float* v) {
    if (k >= K) return;  // zeros
#pragma unroll
    for (int m = 0; m < 4; ++m) {
      const float4 gm = s_gain[k / 4 + m], bm = s_shift[k / 4 + m];
      const float gv[4] = {gm.x, gm.y, gm.z, gm.w}, bv[4] = {bm.x, bm.y, bm.z, bm.w};
#pragma unroll
      for (int j = 0; j < 4; ++j) v[4 * m + j] = fmaf((v[4 * m + j] - mean) * rstd, gv[j], bv[j]);
    }
#pragma unroll
    for (int j = 0; j < 16; ++j) top = max(top, mag(v[j]));
  });
  top = over_row(top, 2, [](uint32_t x, uint32_t y) { return x > y ? x : y; });
  const float sc = q_scale(top), inv = __fdiv_rn(1.0f, sc);
  if (live && threadIdx.x < 16) a.scale[r] = sc;
  const bool plain = __all(q_plain(sc) || !live);
  auto write = [&](auto byte) {
    each([&](int i, int, float* v) {
      const int c = w + NW * i;
      if (c >= kc) return;  // uniform
      uint32_t b[16];
#pragma unroll
      for (int j = 0; j < 16; ++j) b[j] = byte(v[j]);
      uint4 o;
      o.x = low_bytes(b[0], b[1], b[2], b[3]);
      o.y = low_bytes(b[4], b[5], b[6], b[7]);
      o.z = low_bytes(b[8], b[9], b[10], b[11]);
      o.w = low_bytes(b[12], b[13], b[14], b[15]);
      if (live) reinterpret_cast<uint4*>(a.dst)[((size_t)blockIdx.x * kc + c) * 64 + lane] = o;
    });
  };
  // uniform per wave
  if (!plain) write([&](float v) { return (uint32_t)q_value(v, sc); });
  else write([&](float v) { return q_byte<false>(v, sc, inv); });
}

template <class T>
hipError_t launch_tile_t(const QRowsArgs& a, hipStream_t s) {
  const dim3 grid((unsigned)((a.rows + 15) / 16));
  if (a.K <= 512) return launch_k(q_tile_kernel<T, 8, 1>, grid, dim3(512), 0, s, a);
  if (a.K <= 1024) return launch_k(q_tile_kernel<T, 16, 1>, grid, dim3(1024), 0, s, a);
  if (a.K <= 2048) return launch_k(q_tile_kernel<T, 16, 2>, grid, dim3(1024), 0, s, a);
  return hipErrorInvalidValue;  // the widest model (kMaxDim)
}

template <class T, bool VEC>
hipError_t launch_rows_t(const QRowsArgs& a, hipStream_t s) {
  const dim3 grid((unsigned)((a.rows + 3) / 4));
  if (a.K <= 1024) return launch_k(q_rows_kernel<T, 2, 1, VEC>, grid, dim3(256), 0, s, a);
  if (a.K <= 2048) return launch_k(q_rows_kernel<T, 1, 4, VEC>, grid, dim3(1024), 0, s, a);
  if (a.K <= 6144) return launch_k(q_rows_kernel<T, 3, 4, VEC>, grid, dim3(1024), 0, s, a);
  return launch_k(q_rows_kernel<T, 0, 4, VEC>, grid, dim3(1024), 0, s, a);
}

// ------------------------------------------------------------------ weights --

template <class T>
__device__ __forceinline__ float w_value(T x) { return Elem<T>::f(x); }
template <>
__device__ __forceinline__ float w_value<int8_t>(int8_t x) { return (float)x; }

// Scales and biases of 64 columns by 16 shares of K; columns past N: zeros.
template <class T>
__global__ __launch_bounds__(1024) void q_scale_kernel(QPackArgs a) {
  __shared__ uint32_t s_top[16][64];
  const QWeightsLayout l(a.K, a.N);
  const int c = threadIdx.x & 63, part = threadIdx.x >> 6, n = blockIdx.x * 64 + c;
  const T* w = static_cast<const T*>(a.w);
  uint32_t top = 0;
  if (n < a.N && !a.scales) {
#pragma unroll 8
    for (int k = part; k < a.K; k += 16) top = max(top, mag(w_value<T>(w[k * a.wk + n * a.wn])));
  }
  s_top[part][c] = top;
  __syncthreads();
  if (part || n >= l.blocks * 16) return;
  for (int i = 1; i < 16; ++i) top = max(top, s_top[i][c]);
  float s = 0.0f, b = 0.0f;
  if (n < a.N) {
    s = a.scales ? a.scales[n] : q_scale(top);
    if (a.bias) b = a.dtype == INCVIT_BF16 ? bf2f(static_cast<const uint16_t*>(a.bias)[n]) : static_cast<const float*>(a.bias)[n];
  }
  reinterpret_cast<float*>(a.dst + l.scale)[n] = s;
  reinterpret_cast<float*>(a.dst + l.bias)[n] = b;
}

// One 16-byte lane of an operand kilobyte per thread.
template <class T>
__global__ __launch_bounds__(256) void q_pack_kernel(QPackArgs a) {
  const QWeightsLayout l(a.K, a.N);
  const T* w = static_cast<const T*>(a.w);
  const float* scale = reinterpret_cast<const float*>(a.dst + l.scale);
  const size_t total = (size_t)l.blocks * l.kc * 64;
  for (size_t e = (size_t)blockIdx.x * 256 + threadIdx.x; e < total; e += (size_t)gridDim.x * 256) {
    const int lane = (int)(e & 63);
    const size_t ch = e >> 6;
    const int c = (int)(ch % l.kc), n = (int)(ch / l.kc) * 16 + (lane & 15), k0 = 64 * c + 16 * (lane >> 4);
    uint32_t v[4] = {0, 0, 0, 0};
    if (n < a.N) {
      const float s = scale[n];
#pragma unroll
      for (int j = 0; j < 16; ++j) {
        if (k0 + j >= a.K) continue;
        const T x = w[(k0 + j) * a.wk + n * a.wn];
        int q;
        if constexpr (std::is_same<T, int8_t>::value) q = x;
        else q = q_value(w_value<T>(x), s);
        v[j >> 2] |= (uint32_t)(q & 0xff) << (8 * (j & 3));
      }
    }
    reinterpret_cast<uint4*>(a.dst)[e] = make_uint4(v[0], v[1], v[2], v[3]);
  }
}

template <class T>
hipError_t launch_pack_t(const QPackArgs& a, hipStream_t s) {
  const QWeightsLayout l(a.K, a.N);
  hipError_t e = launch_k(q_scale_kernel<T>, dim3((l.blocks * 16 + 63) / 64), dim3(1024), 0, s, a);
  if (e != hipSuccess) return e;
  const long blocks = ((long)l.blocks * l.kc * 64 + 255) / 256;
  return launch_k(q_pack_kernel<T>, dim3((unsigned)std::min<long>(blocks, 4096)), dim3(256), 0, s, a);
}

// ----------------------------------------------------------------- few rows --

constexpr int kQWaves = 8;

// One block of 16 columns by RT tiles of 16 rows; with more rows than the launch
// was sized for, also those `rgroups` groups further on.  Wave w multiplies
// chunks w, w + 8, ...; U of them are in flight together.
template <int EPI, int RT, int U>
__global__ __launch_bounds__(kQWaves * 64) void q_gemm_kernel(GemmArgs a) {
  using T = q8_out<EPI>;
  __shared__ i32x4_t part[kQWaves][RT][64];
  const int lane = threadIdx.x & 63, g = lane >> 4, n = lane & 15;
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int M = a.meta ? a.meta->m : a.m_host;
  // column blocks are dealt to the XCDs in runs, the row groups of one block
  // together: its weights are fetched by one XCD (128 x 1152 -> 4304: 6.2 -> 5.0 us)
  const int nz = a.rgroups, total = gridDim.x, lin = blockIdx.x;
  const int xcd = lin % 8, pos = xcd * (total / 8) + min(xcd, total % 8) + lin / 8;
  const int cblk = pos / nz, kc = a.kchunks, tiles = (M + 15) / 16;
  const uint4* W = reinterpret_cast<const uint4*>(a.W) + (size_t)cblk * kc * 64 + lane;
  const uint4* A = reinterpret_cast<const uint4*>(a.A) + lane;
  for (int m0 = pos % nz * RT * 16; m0 < M; m0 += nz * RT * 16) {  // uniform
    i32x4_t acc[RT];
    const uint4* At[RT];
#pragma unroll
    for (int r = 0; r < RT; ++r) {
      acc[r] = i32x4_t{0, 0, 0, 0};
      At[r] = A + (size_t)min(m0 / 16 + r, tiles - 1) * kc * 64;
    }
    for (int c0 = w; c0 < kc; c0 += kQWaves * U) {
      uint4 wf[U], af[U][RT];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int c = min(c0 + kQWaves * u, kc - 1);
        wf[u] = W[(size_t)c * 64];
#pragma unroll
        for (int r = 0; r < RT; ++r) af[u][r] = At[r][(size_t)c * 64];
      }
#pragma unroll
      for (int u = 0; u < U; ++u) {
        if (c0 + kQWaves * u < kc) {  // uniform
#pragma unroll
          for (int r = 0; r < RT; ++r)
            mma_q8(acc[r], __builtin_bit_cast(u32x4_t, wf[u]), __builtin_bit_cast(u32x4_t, af[u][r]));
        }
      }
    }
#pragma unroll
    for (int r = 0; r < RT; ++r) part[w][r][lane] = acc[r];
    __syncthreads();
    const int row = m0 + 16 * w + n, col = cblk * 16 + 4 * g;
    if (w < RT && row < M && col < a.n) {
      i32x4_t sum = part[0][w][lane];
#pragma unroll
      for (int i = 1; i < kQWaves; ++i) sum += part[i][w][lane];
      const float4 cs = *reinterpret_cast<const float4*>(a.col_scale + col), bi = *reinterpret_cast<const float4*>(a.bias + col);
      ResRun<T, 4> res;
      if constexpr (q8_resid<EPI>()) res.load(q8_res<T, 4>(a, q8_down<EPI>(), row, col));
      if constexpr (q8_down<EPI>()) q8_down_store<T, 4>(a, row, col, true, &sum, a.row_scale[row], &cs, &bi, res, a.rows[row]);
      else q8_store<T, 4, q8_wide<EPI>(), q8_resid<EPI>()>(a, row, col, true, &sum, a.row_scale[row], &cs, &bi, res);
    }
    __syncthreads();  // `part` is written again
  }
}

// Up to 8 rows quantised by every workgroup for itself, a wave per row: one launch
// for a few tokens.  A = x, rows on the host; the integers take rows * (64 kc +
// 16) bytes of LDS (the 16 keep a fragment's rows on different banks).  The first
// weights are on their way meanwhile.  HELD: a wave's row stays in registers
// (bf16, 16-byte runs, K <= 2048), else it is read twice.
template <int EPI, bool VEC, bool HELD>
__global__ __launch_bounds__(kQWaves * 64) void q_token_kernel(GemmArgs a) {
  using T = q8_out<EPI>;
  constexpr int U = 3;
  __shared__ i32x4_t part[kQWaves][64];
  __shared__ float s_scale[kQWaves];
  extern __shared__ __align__(16) char s_q[];
  const int lane = threadIdx.x & 63, g = lane >> 4, n = lane & 15;
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int M = a.m_host, K = a.k, kc = a.kchunks, cblk = blockIdx.x, pitch = 64 * kc + 16;
  const u32x4_t* W = reinterpret_cast<const u32x4_t*>(a.W) + (size_t)cblk * kc * 64 + lane;
  u32x4_t wf[U];
#pragma unroll
  for (int u = 0; u < U; ++u) wf[u] = W[(size_t)min(w + kQWaves * u, kc - 1) * 64];
  if (w < M) {  // uniform
    const T* row = static_cast<const T*>(a.A) + (size_t)w * a.x_ld;
    auto write = [&](int k, const float* v, float s, float inv, bool plain) {
      uint32_t b[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) b[j] = plain ? q_byte<sizeof(T) == 2>(v[j], s, inv) : (uint32_t)q_value(v[j], s);
      *reinterpret_cast<uint2*>(s_q + w * pitch + k) = make_uint2(low_bytes(b[0], b[1], b[2], b[3]), low_bytes(b[4], b[5], b[6], b[7]));
    };
    uint32_t top = 0;
    constexpr int RUNS = HELD ? 4 : 1;
    float held[RUNS][8];
    if constexpr (HELD) {
#pragma unroll
      for (int j = 0; j < RUNS; ++j) row8<T, VEC>(row, 8 * lane + 512 * j, K, held[j]);
#pragma unroll
      for (int j = 0; j < RUNS; ++j)
#pragma unroll
        for (int e = 0; e < 8; ++e) top = max(top, mag(held[j][e]));
    } else {
      for (int k = 8 * lane; k < K; k += 512) {
        row8<T, VEC>(row, k, K, held[0]);
#pragma unroll
        for (int e = 0; e < 8; ++e) top = max(top, mag(held[0][e]));
      }
    }
    const float s = q_scale(lanes_max<64>(top)), inv = __fdiv_rn(1.0f, s);
    if (lane == 0) s_scale[w] = s;
    const bool plain = q_plain(s);  // uniform
    if constexpr (HELD) {
#pragma unroll
      for (int j = 0; j < RUNS; ++j)
        if (8 * lane + 512 * j < 64 * kc) write(8 * lane + 512 * j, held[j], s, inv, plain);
    } else {
      for (int k = 8 * lane; k < 64 * kc; k += 512) {
        row8<T, VEC>(row, k, K, held[0]);  // from the L1
        write(k, held[0], s, inv, plain);
      }
    }
  }
  __syncthreads();
  i32x4_t acc = i32x4_t{0, 0, 0, 0};
  const char* Ar = s_q + min(n, M - 1) * pitch + 16 * g;
  for (int c0 = w; c0 < kc; c0 += kQWaves * U) {
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (c0 + kQWaves * u < kc) mma_q8(acc, wf[u], *reinterpret_cast<const u32x4_t*>(Ar + 64 * (c0 + kQWaves * u)));  // uniform
    if (c0 + kQWaves * U < kc) {
#pragma unroll
      for (int u = 0; u < U; ++u) wf[u] = W[(size_t)min(c0 + kQWaves * (U + u), kc - 1) * 64];
    }
  }
  part[w][lane] = acc;
  __syncthreads();
  const int col = cblk * 16 + 4 * g;
  if (w > 0 || n >= M || col >= a.n) return;
  i32x4_t sum = part[0][lane];
#pragma unroll
  for (int i = 1; i < kQWaves; ++i) sum += part[i][lane];
  const float4 cs = *reinterpret_cast<const float4*>(a.col_scale + col), bi = *reinterpret_cast<const float4*>(a.bias + col);
  ResRun<T, 4> res;
  if constexpr (q8_resid<EPI>()) res.load(q8_res<T, 4>(a, false, n, col));
  q8_store<T, 4, q8_wide<EPI>(), q8_resid<EPI>()>(a, n, col, true, &sum, s_scale[n], &cs, &bi, res);
}

template <int EPI, int RT, int U>
hipError_t launch_few(const GemmArgs& a0, int expected, hipStream_t s) {
  GemmArgs a = a0;
  a.rgroups = (expected + 16 * RT - 1) / (16 * RT);
  return launch_k(q_gemm_kernel<EPI, RT, U>, dim3((unsigned)(a.Nout / 16) * a.rgroups), dim3(kQWaves * 64), 0, s, a);
}

// Few rows or the large-row GEMM.  us per launch: the former takes about 2.3 +
// (1.6 + 0.2 chunks) per 10^6 outputs (chunks of 64 along K), the latter 3.9 +
// 0.105 per chunk while it has one round of tiles (its workgroup's chunks follow
// one another); they meet at the outputs below.  Measured, few rows against
// large-row: 128 x 1152 -> 4304 5.0 against 5.6, 192 rows 6.2 against 5.7;
// 448 x 4304 -> 1152 10.1 against 11.2, 512 rows 13.3 (the former's workgroups
// pass two to a CU) against 11.2; 512 x 4096 -> 1024 8.9 against 10.6, 576 rows
// 11.9 against 10.8; 1024 x 192 -> 768 3.9 against 4.4, 2048 rows 5.6 against 4.8.
// Outputs that end off 16 bytes cost both forms more and meet at the same place
// (fp32): 546 x 1000 -> 1013 5.9 against 6.6, 1024 rows 8.6 against 7.9; 128 x 1152
// -> 4305 6.5 against 6.8, 192 rows 7.9 against 7.7; 448 x 4304 -> 1153 11.5 against
// 12.2, 512 rows 15.3 against 12.4; but 700 x 1000 -> 1013 6.5 against 6.9.
//
// Few rows: as many row tiles to a workgroup (each W fragment read once for all)
// as still leave three workgroups to four CUs, four only beyond 128 rows: 64 x
// 1152 -> 4304 2 tiles 3.8, 1 tile 4.6, 4 tiles 4.2; 192 x 1024 -> 4096 4 tiles
// 5.2, 2 tiles 5.6; 48 x 4304 -> 1152 2 tiles 4.0, 1 tile 3.5.  Chunks in flight
// per wave: 2 where its share is at most 4 (more would load some twice), else 4:
// 23 x 1152 -> 4304 3.3 against 3.7, 64 x 4304 -> 1152 4.0 against 4.4.
template <int EPI>
hipError_t launch_gemm_e(const GemmArgs& a, int expected, int rows, hipStream_t s) {
  const double outputs = (double)expected * a.n, kc = a.kchunks;
  if (outputs * (1.6 + 0.2 * kc) > 1e6 * (1.6 + 0.105 * kc)) return launch_tiled_epi<EPI>(a, expected, rows, s);
  const int blocks = a.Nout / 16;
  auto fills = [&](int rt) { return blocks * ((expected + 16 * rt - 1) / (16 * rt)) >= 192; };
  const int rt = expected > 128 && fills(4) ? 4 : expected > 16 && fills(2) ? 2 : 1;
  if ((a.kchunks + kQWaves - 1) / kQWaves <= 4) {
    if (rt == 4) return launch_few<EPI, 4, 2>(a, expected, s);
    return rt == 2 ? launch_few<EPI, 2, 2>(a, expected, s) : launch_few<EPI, 1, 2>(a, expected, s);
  }
  if (rt == 4) return launch_few<EPI, 4, 4>(a, expected, s);
  return rt == 2 ? launch_few<EPI, 2, 4>(a, expected, s) : launch_few<EPI, 1, 4>(a, expected, s);
}

template <int EPI>
hipError_t launch_token_e(const GemmArgs& a, hipStream_t s) {
  constexpr bool F32 = std::is_same<q8_out<EPI>, float>::value;
  const size_t lds = (size_t)a.m_host * (64 * a.kchunks + 16);
  const dim3 grid(a.Nout / 16), block(kQWaves * 64);
  const bool vec = a.k % 8 == 0 && ((uintptr_t)a.x_ld * (F32 ? 4 : 2) | (uintptr_t)a.A) % 16 == 0;
  if constexpr (!F32) {
    if (vec && a.k <= 2048) return launch_k(q_token_kernel<EPI, true, true>, grid, block, lds, s, a);
  }
  if (vec) return launch_k(q_token_kernel<EPI, true, false>, grid, block, lds, s, a);
  return launch_k(q_token_kernel<EPI, false, false>, grid, block, lds, s, a);
}

// whether out (and the residual) take 16 bytes at once
bool q_wide(const GemmArgs& a, int out_f32) {
  const uintptr_t eb = out_f32 ? 4 : 2;
  uintptr_t bits = (uintptr_t)a.out | (uintptr_t)a.resid | (uintptr_t)a.n * eb | (uintptr_t)a.out_ld * eb;
  if (a.resid) bits |= (uintptr_t)a.res_ld * eb;
  return bits % 16 == 0;
}

}  // namespace

// Us per call, one launch against two: 1 x 1152 -> 4304 3.7 against 5.2, 8 rows 4.7
// against 5.7 (16 rows, two to a wave: 6.5 against 5.8); 1 x 4304 -> 1152 6.8
// against 7.1; and a launch of 3.5 us of the host's less.
bool q_token_fits(int64_t rows, int K) { return rows <= 8 && rows * ((K + 63) / 64 * 64 + 16) <= 49152; }

hipError_t launch_q_token(const GemmArgs& a, int f32, hipStream_t s) {
  if (!q_wide(a, f32)) return f32 ? launch_token_e<EPI_QF32_ANY>(a, s) : launch_token_e<EPI_QBF_ANY>(a, s);
  if (a.resid) return f32 ? launch_token_e<EPI_QRES_F32>(a, s) : launch_token_e<EPI_QRES_BF>(a, s);
  return f32 ? launch_token_e<EPI_QF32>(a, s) : launch_token_e<EPI_QBF>(a, s);
}

hipError_t launch_q_rows(const QRowsArgs& a, hipStream_t s) {
  if (a.frag) return a.dtype ? launch_tile_t<uint16_t>(a, s) : launch_tile_t<float>(a, s);
  const bool vec = a.K % 8 == 0 && ((uintptr_t)a.ld * (a.dtype ? 2 : 4) | (uintptr_t)a.x | (uintptr_t)a.gamma | (uintptr_t)a.beta) % 16 == 0;
  if (a.dtype) return vec ? launch_rows_t<uint16_t, true>(a, s) : launch_rows_t<uint16_t, false>(a, s);
  return vec ? launch_rows_t<float, true>(a, s) : launch_rows_t<float, false>(a, s);
}

hipError_t launch_q_pack(const QPackArgs& a, hipStream_t s) {
  if (a.dtype == 2) return launch_pack_t<int8_t>(a, s);
  return a.dtype ? launch_pack_t<uint16_t>(a, s) : launch_pack_t<float>(a, s);
}

hipError_t launch_q_down(const GemmArgs& a, int out_f32, int expected, int rows, hipStream_t s) {
  return out_f32 ? launch_gemm_e<EPI_QDOWN_F32>(a, expected, rows, s) : launch_gemm_e<EPI_QDOWN_BF>(a, expected, rows, s);
}

hipError_t launch_q_gemm(const GemmArgs& a, int out_f32, int expected, int rows, hipStream_t s) {
  auto go = [&](auto e) { return launch_gemm_e<decltype(e)::value>(a, expected, rows, s); };
  using std::integral_constant;
  if (!q_wide(a, out_f32)) return out_f32 ? go(integral_constant<int, EPI_QF32_ANY>{}) : go(integral_constant<int, EPI_QBF_ANY>{});
  if (a.resid) return out_f32 ? go(integral_constant<int, EPI_QRES_F32>{}) : go(integral_constant<int, EPI_QRES_BF>{});
  return out_f32 ? go(integral_constant<int, EPI_QF32>{}) : go(integral_constant<int, EPI_QBF>{});
}

}  // namespace incvit
