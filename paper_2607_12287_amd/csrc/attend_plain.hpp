// Operands of the attention over given keys and values: values through LDS, and
// infinities and NaN among them.
//
// A value that a row does not see must not reach its sum, where 0 * NaN is NaN.  Rows
// past the sequence are zeros in LDS, and so are infinities and NaN in a tile that is
// partly masked; where a wave found any, it adds them behind its last tile for the
// rows that see them (add_special).
#pragma once

#include "attend.hpp"

namespace incvit {

typedef short i16x4_t __attribute__((ext_vector_type(4)));

// Bytes of a row in LDS, which spread over the banks what lanes read at once: of keys
// 16 bytes of 8 rows each (an odd number of 16 bytes more than 128); of values, which
// bf16 reads transposed, 32 bytes of 4 rows (an odd number of 32 more).
template <class T, int DS>
constexpr int row_bytes() {
  return DS * (int)sizeof(T) + 16;
}
template <class T, int DS>
constexpr int value_bytes() {
  return sizeof(T) == 4 ? row_bytes<T, DS>() : 2 * DS + (2 * DS % 64 == 0 ? 32 : 0);
}

template <class T>
__device__ __forceinline__ bool special(const V8<T>& x) {
  bool any = false;
  if constexpr (sizeof(T) == 2) {
    const uint32_t w[4] = {x.v.x, x.v.y, x.v.z, x.v.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) any |= (w[i] & 0x7f800000u) == 0x7f800000u || (w[i] & 0x7f80u) == 0x7f80u;
  } else {
    float y[8];
    floats_of(x, y);
#pragma unroll
    for (int i = 0; i < 8; ++i) any |= (__float_as_uint(y[i]) & 0x7f800000u) == 0x7f800000u;
  }
  return any;
}
// infinities and NaN as zeros
__device__ __forceinline__ void drop_special(V8<uint16_t>& x) {
  uint32_t w[4] = {x.v.x, x.v.y, x.v.z, x.v.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const bool hi = (w[i] & 0x7f800000u) == 0x7f800000u, lo = (w[i] & 0x7f80u) == 0x7f80u;
    w[i] &= (hi ? 0u : 0xffff0000u) | (lo ? 0u : 0xffffu);
  }
  x.v = make_uint4(w[0], w[1], w[2], w[3]);
}
__device__ __forceinline__ void drop_special(V8<float>& x) {
  float y[8];
  floats_of(x, y);
#pragma unroll
  for (int i = 0; i < 8; ++i) y[i] = (__float_as_uint(y[i]) & 0x7f800000u) == 0x7f800000u ? 0.0f : y[i];
  x.a = make_float4(y[0], y[1], y[2], y[3]);
  x.b = make_float4(y[4], y[5], y[6], y[7]);
}

// The transposed operand of 32 keys: lane (g, n) has dim `dim0` + n of keys 4 g ..
// + 3 and 16 + 4 g .. + 3, which is the order of its P.
template <class T, int RB>
__device__ __forceinline__ V8<T> value_op(const char* v, int dim0, int lane) {
  const int g = lane >> 4, n = lane & 15;
  V8<T> x;
  if constexpr (sizeof(T) == 2) {
    // 16 lanes give the places of 4 rows of 16 dims, 4 dims each, and get a dim of the 4 rows
    typedef __attribute__((address_space(3))) i16x4_t* Lds;
    char* at = const_cast<char*>(v) + (4 * g + (n >> 2)) * RB + (dim0 + 4 * (n & 3)) * 2;
    const u32x2_t a = __builtin_bit_cast(u32x2_t, __builtin_amdgcn_ds_read_tr16_b64_v4i16((Lds)at));
    const u32x2_t b = __builtin_bit_cast(u32x2_t, __builtin_amdgcn_ds_read_tr16_b64_v4i16((Lds)(at + 16 * RB)));
    x.v = make_uint4(a[0], a[1], b[0], b[1]);
  } else {
    const char* at = v + 4 * g * RB + (dim0 + n) * 4;
    float y[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) y[j] = *reinterpret_cast<const float*>(at + (16 * (j >> 2) + (j & 3)) * RB);
    x.a = make_float4(y[0], y[1], y[2], y[3]);
    x.b = make_float4(y[4], y[5], y[6], y[7]);
  }
  return x;
}

__device__ __forceinline__ void p_op(V8<uint16_t>& out, const float* p) { split8<1>(p, &out.v); }
__device__ __forceinline__ void p_op(V8<float>& out, const float* p) {
  out.a = make_float4(p[0], p[1], p[2], p[3]);
  out.b = make_float4(p[4], p[5], p[6], p[7]);
}

// Dim i of the 4 that lane group g has of piece k, in a row of d; 0 for dims past the head
// (heads of 8: groups 2 and 3), whose value is not used.
__host__ __device__ constexpr int special_dim(int k, int g, int i, int d) { return 16 * k + 4 * g < d ? 16 * k + 4 * g + i : 0; }

// The infinities and NaN of the values of keys j0 to j1, for the rows that see them:
// a weight is above 0, so each makes its sum what it is itself.
template <class T, int NP, int NT>
__device__ __forceinline__ void add_special(f32x4_t (&o)[NT][NP], const Sight (&eye)[NT], const char* values, long v_row, int d, int j0,
                                            int j1, int lane) {
  const int g = lane >> 4;
#pragma unroll 1
  for (int key = j0; key <= j1; ++key) {
    const T* src = reinterpret_cast<const T*>(values + key * v_row);
#pragma unroll
    for (int k = 0; k < NP; ++k) {
      __builtin_amdgcn_sched_barrier(0);  // a rare path: few registers
      float x[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) x[i] = Elem<T>::f(gbl(src)[special_dim(k, g, i, d)]);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const bool odd = !__builtin_isfinite(x[i]) & (16 * k + 4 * g < d);
#pragma unroll
        for (int t = 0; t < NT; ++t) o[t][k][i] += odd & eye[t].sees(key) ? x[i] : 0.0f;
      }
    }
  }
}

}  // namespace incvit
