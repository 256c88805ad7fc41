// Norm of the queries and keys over each head and their rotation, in one pass
// over the rows (and the scatter of new keys into a cache).
//
// A head is cut into chunks of V pairs of values.  A chunk that is rotated in
// halves takes V values from each half, so both members of every pair are in
// one lane and the rotation needs no exchange; every other chunk is 2 V values
// that follow one another.  GL lanes (a power of two) share a head, C chunks to
// a lane; its sums are combined across them by a butterfly in a fixed order.
//   RMS: one sum of squares; LayerNorm: the mean, then the squared deviations
// from it (two passes over registers, no cancellation), all in fp32; the result
// is rounded once, when it is stored.
//
// Bound: memory (each value is read and written once), and for few rows the
// launch.  Every load of a lane (its values, gains, cosines and sines) is
// issued before the first one is used.
#include "ops.hpp"

namespace incvit {

namespace {

// V consecutive values as floats
template <class T, int V> struct Run;
template <> struct Run<uint16_t, 8> {
  uint4 v;
  __device__ void load(const uint16_t* p) { v = *reinterpret_cast<const uint4*>(p); }
  __device__ float get(int i) const {
    const uint32_t w = i < 2 ? v.x : i < 4 ? v.y : i < 6 ? v.z : v.w;
    return __uint_as_float(i & 1 ? w & 0xffff0000u : w << 16);
  }
  __device__ static void store(uint16_t* p, const float* f) {
    *reinterpret_cast<uint4*>(p) = make_uint4(f2bf2(f[0], f[1]), f2bf2(f[2], f[3]), f2bf2(f[4], f[5]), f2bf2(f[6], f[7]));
  }
};
template <> struct Run<uint16_t, 4> {
  uint2 v;
  __device__ void load(const uint16_t* p) { v = *reinterpret_cast<const uint2*>(p); }
  __device__ float get(int i) const {
    const uint32_t w = i < 2 ? v.x : v.y;
    return __uint_as_float(i & 1 ? w & 0xffff0000u : w << 16);
  }
  __device__ static void store(uint16_t* p, const float* f) {
    *reinterpret_cast<uint2*>(p) = make_uint2(f2bf2(f[0], f[1]), f2bf2(f[2], f[3]));
  }
};
template <> struct Run<float, 4> {
  float4 v;
  __device__ void load(const float* p) { v = *reinterpret_cast<const float4*>(p); }
  __device__ float get(int i) const { return i == 0 ? v.x : i == 1 ? v.y : i == 2 ? v.z : v.w; }
  __device__ static void store(float* p, const float* f) { *reinterpret_cast<float4*>(p) = make_float4(f[0], f[1], f[2], f[3]); }
};
template <class T> struct Run<T, 1> {
  T v;
  __device__ void load(const T* p) { v = *p; }
  __device__ float get(int) const { return Elem<T>::f(v); }
  __device__ static void store(T* p, const float* f) { *p = Elem<T>::cv(f[0]); }
};
// V pairs of (cos, sin): 2 V floats
template <int V>
struct Turns {
  float4 v[V / 2];
  __device__ void load(const float* p) {
#pragma unroll
    for (int i = 0; i < V / 2; ++i) v[i] = reinterpret_cast<const float4*>(p)[i];
  }
  __device__ float cos(int i) const { return i & 1 ? v[i / 2].z : v[i / 2].x; }
  __device__ float sin(int i) const { return i & 1 ? v[i / 2].w : v[i / 2].y; }
};
template <>
struct Turns<1> {
  float2 v;
  __device__ void load(const float* p) { v = *reinterpret_cast<const float2*>(p); }
  __device__ float cos(int) const { return v.x; }
  __device__ float sin(int) const { return v.y; }
};

template <int GL>
__device__ __forceinline__ float lanes_sum(float x) {
#pragma unroll
  for (int off = GL / 2; off >= 1; off >>= 1) x += __shfl_xor(x, off, 64);
  return x;
}

struct HeadSpec {
  int pairs, rot_pairs, adjacent, norm;
  float eps, inv_dim;
};

// One head of one row by GL lanes.  in, out: pointers to value d of the head by
// d; gamma, beta: null where there is none; turns: the row's cosines and sines.
template <class T, class G, int V, int GL, int C, class In, class Out>
__device__ __forceinline__ void one_head(const HeadSpec& h, int lane, const G* gamma, const G* beta, const float* turns, In in,
                                         Out out) {
  Run<T, V> xa[C], xb[C];
  Run<G, V> ga[C], gb[C], ba[C], bb[C];
  Turns<V> cs[C];
  int da[C], db[C];
  bool any[C], rot[C];
  const bool normed = h.norm != INCVIT_NORM_NONE;
#pragma unroll
  for (int c = 0; c < C; ++c) {
    const int p = (lane + GL * c) * V;
    any[c] = p < h.pairs;
    rot[c] = p < h.rot_pairs;
    const bool halves = rot[c] && !h.adjacent;
    da[c] = any[c] ? (halves ? p : 2 * p) : 0;
    db[c] = any[c] ? (halves ? p + h.rot_pairs : 2 * p + V) : V;
    xa[c].load(in(da[c]));
    xb[c].load(in(db[c]));
    if (normed && gamma) {
      ga[c].load(gamma + da[c]);
      gb[c].load(gamma + db[c]);
    }
    if (normed && beta) {
      ba[c].load(beta + da[c]);
      bb[c].load(beta + db[c]);
    }
    if (h.rot_pairs) cs[c].load(turns + 2 * (rot[c] ? p : 0));
  }
  float a[C][V], b[C][V];
#pragma unroll
  for (int c = 0; c < C; ++c)
#pragma unroll
    for (int i = 0; i < V; ++i) {
      a[c][i] = xa[c].get(i);
      b[c][i] = xb[c].get(i);
    }
  if (normed) {
    float mean = 0.0f;
    if (h.norm == INCVIT_NORM_LAYER) {
      float s = 0.0f;
#pragma unroll
      for (int c = 0; c < C; ++c)
#pragma unroll
        for (int i = 0; i < V; ++i) s += any[c] ? a[c][i] + b[c][i] : 0.0f;
      mean = lanes_sum<GL>(s) * h.inv_dim;
    }
    float q = 0.0f;
#pragma unroll
    for (int c = 0; c < C; ++c)
#pragma unroll
      for (int i = 0; i < V; ++i) {
        a[c][i] -= mean;
        b[c][i] -= mean;
        q += any[c] ? a[c][i] * a[c][i] + b[c][i] * b[c][i] : 0.0f;
      }
    const float r = 1.0f / sqrtf(lanes_sum<GL>(q) * h.inv_dim + h.eps);
#pragma unroll
    for (int c = 0; c < C; ++c)
#pragma unroll
      for (int i = 0; i < V; ++i) {
        a[c][i] *= r;
        b[c][i] *= r;
        if (gamma) {
          a[c][i] *= ga[c].get(i);
          b[c][i] *= gb[c].get(i);
        }
        if (beta) {
          a[c][i] += ba[c].get(i);
          b[c][i] += bb[c].get(i);
        }
      }
  }
#pragma unroll
  for (int c = 0; c < C; ++c) {
    if (rot[c]) {
      const bool pairs_split = !h.adjacent;
      float ya[V], yb[V];
#pragma unroll
      for (int i = 0; i < V; ++i) {
        if (pairs_split) {  // pair i: (a_i, b_i)
          ya[i] = a[c][i] * cs[c].cos(i) - b[c][i] * cs[c].sin(i);
          yb[i] = b[c][i] * cs[c].cos(i) + a[c][i] * cs[c].sin(i);
        }
      }
      if (!pairs_split) {  // the 2 V values one after another: pair i is values 2 i and 2 i + 1
        float z[2 * V];
#pragma unroll
        for (int i = 0; i < V; ++i) {
          z[i] = a[c][i];
          z[V + i] = b[c][i];
        }
#pragma unroll
        for (int i = 0; i < V; ++i) {
          const float u = z[2 * i] * cs[c].cos(i) - z[2 * i + 1] * cs[c].sin(i);
          z[2 * i + 1] = z[2 * i + 1] * cs[c].cos(i) + z[2 * i] * cs[c].sin(i);
          z[2 * i] = u;
        }
#pragma unroll
        for (int i = 0; i < V; ++i) {
          ya[i] = z[i];
          yb[i] = z[V + i];
        }
      }
#pragma unroll
      for (int i = 0; i < V; ++i) {
        a[c][i] = ya[i];
        b[c][i] = yb[i];
      }
    }
    if (any[c]) {
      Run<T, V>::store(out(da[c]), a[c]);
      Run<T, V>::store(out(db[c]), b[c]);
    }
  }
}

template <class T, int V, int GL, int C>
__global__ __launch_bounds__(256) void qk_kernel(QkArgs a) {
  const int heads = a.q.heads + a.k.heads;
  const long item = (long)blockIdx.x * (256 / GL) + threadIdx.x / GL;
  const int lane = threadIdx.x % GL;
  if (item >= a.rows * heads) return;  // whole groups of lanes
  const long r = item / heads;
  const int hh = (int)(item - r * heads);
  const bool isk = hh >= a.q.heads;
  const QkSide& s = isk ? a.k : a.q;
  const int h = isk ? hh - a.q.heads : hh;
  long t = r, dst = r;
  if (a.rot_pairs) {
    t = a.index ? (long)a.index[r] : r % a.table_rows;
    if (t < 0 || t >= a.table_rows) return;
  }
  if (isk && a.k_rows) {
    dst = a.k_rows[r];
    if (dst < 0 || dst >= a.k_out_rows) return;
  }
  const HeadSpec spec{a.head_dim / 2, a.rot_pairs, a.adjacent, a.norm, a.eps, 1.0f / (float)a.head_dim};
  const T* in = static_cast<const T*>(s.in) + r * s.in_row + h * s.in_head;
  T* out = static_cast<T*>(s.out) + dst * s.out_row + h * s.out_head;
  one_head<T, T, V, GL, C>(spec, lane, static_cast<const T*>(s.gamma), static_cast<const T*>(s.beta),
                           a.table + t * 2 * a.rot_pairs, [&](int d) { return in + d; }, [&](int d) { return out + d; });
}

// The encoder's rows: queries in the compact buffer, keys where the QKV
// projection left them in the cache.  A chunk's 4 values lie inside one run of 8
// of the cache's operand order (k_elem), so they are consecutive there too.
template <class T, int GL, int C>
__global__ __launch_bounds__(256) void qk_layer_kernel(QkLayerArgs a) {
  const int H = a.sh.H, dh = a.sh.dh;
  const int item = blockIdx.x * (256 / GL) + threadIdx.x / GL;
  const int lane = threadIdx.x % GL;
  const int r = item / (2 * H), hh = item - r * 2 * H;
  if (r >= a.meta->m) return;
  const RowInfo ri = a.rows[r];
  const bool isk = hh >= H;
  const int h = isk ? hh - H : hh;
  T* q = static_cast<T*>(a.q) + (size_t)r * a.sh.D + h * dh;
  T* k = reinterpret_cast<T*>(ri.cache + a.cl.k + (size_t)a.layer * a.cl.kv_layer);
  const HeadSpec spec{dh / 2, a.table ? dh / 2 : 0, a.adjacent, a.norm, a.eps, 1.0f / (float)dh};
  auto at = [&](int d) { return isk ? k + k_elem(a.sh, h, ri.tok, d) : q + d; };
  one_head<T, float, 4, GL, C>(spec, lane, isk ? a.k_gamma : a.q_gamma, isk ? a.k_beta : a.q_beta,
                               a.table + (size_t)ri.tok * dh, at, at);
}

template <class T, int V, int GL, int C>
hipError_t launch_v(const QkArgs& a, hipStream_t s) {
  const long items = a.rows * (a.q.heads + a.k.heads);
  return launch_k(qk_kernel<T, V, GL, C>, dim3((unsigned)((items + 256 / GL - 1) / (256 / GL))), dim3(256), 0, s, a);
}

// lanes of a head: the power of two that covers its chunks
template <class T, int V>
hipError_t launch_lanes(const QkArgs& a, hipStream_t s) {
  const int chunks = a.head_dim / 2 / V;
  if (chunks <= 4) return launch_v<T, V, 4, 1>(a, s);
  if (chunks <= 8) return launch_v<T, V, 8, 1>(a, s);
  if (chunks <= 16) return launch_v<T, V, 16, 1>(a, s);
  return launch_v<T, V, 32, 1>(a, s);
}

// whether every chunk of v values that a call touches is aligned to itself
bool chunks_aligned(const QkArgs& a, int v) {
  const int eb = a.dtype ? 2 : 4;
  if (a.head_dim % (2 * v) || a.rot_pairs % v) return false;
  uintptr_t bits = 0;
  for (const QkSide* s : {&a.q, &a.k}) {
    if (s->heads == 0) continue;
    bits |= (uintptr_t)s->in | (uintptr_t)s->out | (uintptr_t)s->gamma | (uintptr_t)s->beta;
    for (long st : {s->in_row, s->in_head, s->out_row, s->out_head}) bits |= (uintptr_t)st * eb;
  }
  return bits % (v * eb) == 0 && (a.rot_pairs == 0 || (uintptr_t)a.table % 16 == 0);
}

}  // namespace

hipError_t launch_qk(const QkArgs& a, hipStream_t s) {
  if (a.dtype) {
    if (chunks_aligned(a, 8)) return launch_lanes<uint16_t, 8>(a, s);
    if (chunks_aligned(a, 4)) return launch_lanes<uint16_t, 4>(a, s);
    return launch_v<uint16_t, 1, 64, 2>(a, s);
  }
  if (chunks_aligned(a, 4)) return launch_lanes<float, 4>(a, s);
  return launch_v<float, 1, 64, 2>(a, s);
}

hipError_t launch_qk_layer(const QkLayerArgs& a, int rows, hipStream_t s) {
  const int chunks = a.sh.dh / 8;
  const int gl = chunks <= 4 ? 4 : chunks <= 8 ? 8 : 16;
  const dim3 grid((unsigned)(((long)rows * 2 * a.sh.H + 256 / gl - 1) / (256 / gl)));
  auto go = [&](auto t) {
    using T = decltype(t);
    if (gl == 4) return launch_k(qk_layer_kernel<T, 4, 1>, grid, dim3(256), 0, s, a);
    if (gl == 8) return launch_k(qk_layer_kernel<T, 8, 1>, grid, dim3(256), 0, s, a);
    return launch_k(qk_layer_kernel<T, 16, 1>, grid, dim3(256), 0, s, a);
  };
  return a.sh.dtype ? go(uint16_t{}) : go(float{});
}

}  // namespace incvit
