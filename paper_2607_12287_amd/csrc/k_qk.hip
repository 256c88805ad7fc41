// Norm of the queries and keys over each head and their rotation, in one pass
// over the rows (and the scatter of new keys into a cache).
//
// A head is cut into chunks of V pairs of values.  A chunk that is rotated in
// halves takes V values from each half, so both members of every pair are in
// one lane and the rotation needs no exchange; every other chunk is 2 V values
// that follow one another.  GL lanes (a power of two) share a head, C chunks to
// a lane, and with many rows two heads; sums are combined across the lanes in
// a fixed order.
//   RMS: one sum of squares; LayerNorm: the mean, then the squared deviations
// from it (two passes over registers, no cancellation), all in fp32; the result
// is rounded once, when it is stored.
//
// Bound: memory (each value is read and written once), and for few rows the
// launch.  8192 rows of 32 heads of 64 (67 MB read and written): 15.1 us, a
// plain copy of the same bytes 14.1; a single row 2.7.  Every load of a lane (its
// values, gains, cosines and sines) is issued before the first one is used.  Heads
// whose chunks are no power of two leave lanes idle: 1024 rows of 32 heads of 72
// (9 chunks on 16 lanes) 6.4 us, where the bytes and a launch take 4.4.
#include <type_traits>

#include "ops.hpp"

namespace incvit {

namespace {

typedef float f32x2_t __attribute__((ext_vector_type(2)));

// V consecutive values as floats (global memory: a cache's address comes from
// memory, and would be taken for any address space)
template <class T, int V> struct Run;
template <int V> struct Run<uint16_t, V> {
  uint32_t w[V / 2];
  __device__ void load(const uint16_t* p) {
    if constexpr (V == 8) *reinterpret_cast<u32x4_t*>(w) = *(const INCVIT_GLOBAL u32x4_t*)p;
    else if constexpr (V == 4) *reinterpret_cast<u32x2_t*>(w) = *(const INCVIT_GLOBAL u32x2_t*)p;
    else w[0] = *(const INCVIT_GLOBAL uint32_t*)p;
  }
  __device__ float get(int i) const { return __uint_as_float(i & 1 ? w[i / 2] & 0xffff0000u : w[i / 2] << 16); }
  __device__ static void store(uint16_t* p, const float* f) {
    if constexpr (V == 8) *(INCVIT_GLOBAL u32x4_t*)p = u32x4_t{f2bf2(f[0], f[1]), f2bf2(f[2], f[3]), f2bf2(f[4], f[5]), f2bf2(f[6], f[7])};
    else if constexpr (V == 4) *(INCVIT_GLOBAL u32x2_t*)p = u32x2_t{f2bf2(f[0], f[1]), f2bf2(f[2], f[3])};
    else *(INCVIT_GLOBAL uint32_t*)p = f2bf2(f[0], f[1]);
  }
};
template <int V> struct Run<float, V> {
  float v[V];
  __device__ void load(const float* p) {
    if constexpr (V == 8) {
      *reinterpret_cast<f32x4_t*>(v) = ((const INCVIT_GLOBAL f32x4_t*)p)[0];
      *reinterpret_cast<f32x4_t*>(v + 4) = ((const INCVIT_GLOBAL f32x4_t*)p)[1];
    } else if constexpr (V == 4) {
      *reinterpret_cast<f32x4_t*>(v) = *(const INCVIT_GLOBAL f32x4_t*)p;
    } else {
      *reinterpret_cast<f32x2_t*>(v) = *(const INCVIT_GLOBAL f32x2_t*)p;
    }
  }
  __device__ float get(int i) const { return v[i]; }
  __device__ static void store(float* p, const float* f) {
    static_assert(V <= 4, "runs of 8 are bf16 values, whose gains alone are fp32");
    if constexpr (V == 4) *(INCVIT_GLOBAL f32x4_t*)p = f32x4_t{f[0], f[1], f[2], f[3]};
    else *(INCVIT_GLOBAL f32x2_t*)p = f32x2_t{f[0], f[1]};
  }
};
template <class T> struct Run1 {
  T v;
  __device__ void load(const T* p) { v = *gbl(p); }
  __device__ float get(int) const { return Elem<T>::f(v); }
  __device__ static void store(T* p, const float* f) { *gbl(p) = Elem<T>::cv(f[0]); }
};
template <> struct Run<uint16_t, 1> : Run1<uint16_t> {};
template <> struct Run<float, 1> : Run1<float> {};
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

struct HeadSpec {
  int pairs, rot_pairs, adjacent, norm;
  float eps, inv_dim;
};

// HP heads of one row by GL lanes, which share their gains, cosines and sines.
// in, out: value d of head i by (i, d), for i below `heads`; gamma, beta: null
// where there is none; turns: the row's cosines and sines.
template <class T, class G, int V, int GL, int C, int HP, class In, class Out>
__device__ __forceinline__ void some_heads(const HeadSpec& h, int lane, int heads, const G* gamma, const G* beta,
                                           const float* turns, In in, Out out) {
  Run<T, V> xa[HP][C], xb[HP][C];
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
#pragma unroll
    for (int i = 0; i < HP; ++i) {
      const int j = min(i, heads - 1);
      xa[i][c].load(in(j, da[c]));
      xb[i][c].load(in(j, db[c]));
    }
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
#pragma unroll
  for (int i = 0; i < HP; ++i) {
    if (i >= heads) break;  // uniform over the lanes of a head
    float a[C][V], b[C][V];
#pragma unroll
    for (int c = 0; c < C; ++c)
#pragma unroll
      for (int v = 0; v < V; ++v) {
        a[c][v] = any[c] ? xa[i][c].get(v) : 0.0f;
        b[c][v] = any[c] ? xb[i][c].get(v) : 0.0f;
      }
    if (normed) {
      float mean = 0.0f;
      if (h.norm == INCVIT_NORM_LAYER) {
        float s = 0.0f;
#pragma unroll
        for (int c = 0; c < C; ++c)
#pragma unroll
          for (int v = 0; v < V; ++v) s += a[c][v] + b[c][v];
        mean = lanes_sum<GL>(s) * h.inv_dim;
      }
      float q = 0.0f;
#pragma unroll
      for (int c = 0; c < C; ++c)
#pragma unroll
        for (int v = 0; v < V; ++v) {
          a[c][v] -= mean;
          b[c][v] -= mean;
          const float e = a[c][v] * a[c][v] + b[c][v] * b[c][v];
          q += any[c] ? e : 0.0f;
        }
      const float r = 1.0f / sqrtf(lanes_sum<GL>(q) * h.inv_dim + h.eps);
#pragma unroll
      for (int c = 0; c < C; ++c)
#pragma unroll
        for (int v = 0; v < V; ++v) {
          a[c][v] *= r;
          b[c][v] *= r;
          if (gamma) {
            a[c][v] *= ga[c].get(v);
            b[c][v] *= gb[c].get(v);
          }
          if (beta) {
            a[c][v] += ba[c].get(v);
            b[c][v] += bb[c].get(v);
          }
        }
    }
#pragma unroll
    for (int c = 0; c < C; ++c) {
      // pair v is (a_v, b_v), or values 2 v and 2 v + 1 of the 2 V in a row; the
      // values past the rotated ones stay
      if (rot[c]) {
        if (!h.adjacent) {
#pragma unroll
          for (int v = 0; v < V; ++v) {
            const float u = a[c][v] * cs[c].cos(v) - b[c][v] * cs[c].sin(v);
            b[c][v] = b[c][v] * cs[c].cos(v) + a[c][v] * cs[c].sin(v);
            a[c][v] = u;
          }
        } else {
          float z[2 * V];
#pragma unroll
          for (int v = 0; v < V; ++v) {
            z[v] = a[c][v];
            z[V + v] = b[c][v];
          }
#pragma unroll
          for (int v = 0; v < V; ++v) {
            const float u = z[2 * v] * cs[c].cos(v) - z[2 * v + 1] * cs[c].sin(v);
            z[2 * v + 1] = z[2 * v + 1] * cs[c].cos(v) + z[2 * v] * cs[c].sin(v);
            z[2 * v] = u;
          }
#pragma unroll
          for (int v = 0; v < V; ++v) {
            a[c][v] = z[v];
            b[c][v] = z[V + v];
          }
        }
      }
      if (any[c]) {
        Run<T, V>::store(out(i, da[c]), a[c]);
        Run<T, V>::store(out(i, db[c]), b[c]);
      }
    }
  }
}

// Which heads of which row a group of lanes works on: units of up to HP heads of
// the queries, then of the keys; a workgroup takes `rpb` whole rows, or a share
// (blockIdx.y) of one row's units where they are more than its groups.
struct Units {
  int uq, per_row, rpb, upb;  // units of the queries, of a row; rows, units of a row per workgroup
};
template <int GL>
Units units_of(int hq, int hk, int hp) {
  Units u;
  u.uq = (hq + hp - 1) / hp;
  u.per_row = u.uq + (hk + hp - 1) / hp;
  u.upb = std::min(u.per_row, 256 / GL);
  u.rpb = 256 / GL / u.upb;
  return u;
}
template <int GL>
__device__ __forceinline__ bool unit_of(const Units& u, int bx, int by, uint32_t& row, int& unit) {
  const int g = threadIdx.x / GL;
  const int rl = (int)(((float)g + 0.5f) * __builtin_amdgcn_rcpf((float)u.upb));  // g / upb: both below 256
  row = bx * (uint32_t)u.rpb + rl;
  unit = by * u.upb + g - rl * u.upb;
  return rl < u.rpb && unit < u.per_row;
}

struct QkLaunch {
  QkArgs a;
  Units u;
};

template <class T, int V, int GL, int C, int HP>
__global__ __launch_bounds__(256) void qk_kernel(QkLaunch l) {
  const QkArgs& a = l.a;
  uint32_t r;
  int unit;
  const bool mine = unit_of<GL>(l.u, blockIdx.x, blockIdx.y, r, unit);
  r += (uint32_t)a.row0;
  if (!mine || r >= a.rows) return;  // whole groups of lanes
  const bool isk = unit >= l.u.uq;
  const QkSide s = isk ? a.k : a.q;
  const int h0 = (isk ? unit - l.u.uq : unit) * HP;
  long t = r, dst = r;
  if (a.rot_pairs) {
    if (a.index) t = a.index[r];  // uniform
    else if (a.table_rows < a.rows) t = r % (uint32_t)a.table_rows;
    if (t < 0 || t >= a.table_rows) return;
  }
  if (isk && a.k_rows) {
    dst = a.k_rows[r];
    if (dst < 0 || dst >= a.k_out_rows) return;
  }
  const HeadSpec spec{a.head_dim / 2, a.rot_pairs, a.adjacent, a.norm, a.eps, 1.0f / (float)a.head_dim};
  const T* in = static_cast<const T*>(s.in) + (long)r * s.in_row + h0 * s.in_head;
  T* out = static_cast<T*>(s.out) + dst * s.out_row + h0 * s.out_head;
  some_heads<T, T, V, GL, C, HP>(spec, threadIdx.x % GL, s.heads - h0, static_cast<const T*>(s.gamma),
                                 static_cast<const T*>(s.beta), a.table + t * 2 * a.rot_pairs,
                                 [&](int i, int d) { return in + i * s.in_head + d; },
                                 [&](int i, int d) { return out + i * s.out_head + d; });
}

// The encoder's rows: queries in the compact buffer, keys where the QKV
// projection left them in the cache.  A chunk's V values (4 or 8) lie inside one
// run of 8 of the cache's operand order (k_elem), so they are consecutive there
// too.  The first `qblocks` workgroups take the queries, rows of heads after one
// another; the others the keys, 16 rows of a few heads, since the same run of 4
// tokens is 64 consecutive bytes there (8192 rows of 16 heads of 64: 28 -> 17.6 us).
struct QkLayerLaunch {
  QkLayerArgs a;
  Units u;       // of the queries
  int qblocks;
};

template <class T, int V, int GL, int HP>
__global__ __launch_bounds__(256) void qk_layer_kernel(QkLayerLaunch l) {
  const QkLayerArgs& a = l.a;
  const int dh = a.sh.dh, H = a.sh.H;
  const uint32_t m = (uint32_t)a.meta->m;
  const HeadSpec spec{dh / 2, a.table ? dh / 2 : 0, a.adjacent, a.norm, a.eps, 1.0f / (float)dh};
  const int lane = threadIdx.x % GL;
  if ((int)blockIdx.x < l.qblocks) {  // uniform
    uint32_t r;
    int unit;
    const int ny = (l.u.per_row + l.u.upb - 1) / l.u.upb;
    if (!unit_of<GL>(l.u, (int)blockIdx.x / ny, (int)blockIdx.x % ny, r, unit) || r >= m) return;
    T* q = static_cast<T*>(a.q) + (size_t)r * a.sh.D + unit * HP * dh;
    auto at = [&](int i, int d) { return q + i * dh + d; };
    some_heads<T, float, V, GL, 1, HP>(spec, lane, H - unit * HP, a.q_gamma, a.q_beta, a.table + (size_t)a.rows[r].tok * dh, at, at);
    return;
  }
  constexpr int G = 256 / GL, HB = (G + 15) / 16;  // heads per workgroup
  const int kb = blockIdx.x - l.qblocks, hb = (H + HB - 1) / HB, g = threadIdx.x / GL;
  const uint32_t r = (uint32_t)(kb / hb) * 16 + g % 16;
  const int h = kb % hb * HB + g / 16;
  if (r >= m || h >= H) return;
  const RowInfo ri = a.rows[r];
  T* k = reinterpret_cast<T*>(ri.cache + a.cl.k + (size_t)a.layer * a.cl.kv_layer);
  auto at = [&](int, int d) { return k + k_elem(a.sh, h, ri.tok, d); };
  some_heads<T, float, V, GL, 1, 1>(spec, lane, 1, a.k_gamma, a.k_beta, a.table + (size_t)ri.tok * dh, at, at);
}

// Two heads of a row to a group of lanes where that still leaves every SIMD two
// waves, else one (few rows: latency).  1024 rows of 32 heads of 72: 6.5 us
// against 6.9 with one and 6.6 with four; 8192 rows of 32 of 64: 15.2, 16.0, 15.3.
inline bool many_heads(long rows, int hq, int hk, int gl) { return hq % 2 == 0 && hk % 2 == 0 && rows * (hq + hk) * gl >= 1 << 18; }

template <class T, int V, int GL, int C, int HP>
hipError_t launch_h(const QkArgs& a, hipStream_t s) {
  QkLaunch l{a, units_of<GL>(a.q.heads, a.k.heads, HP)};
  constexpr long kBlocks = 1 << 22;  // of a launch: threads are counted in 32 bits
  for (l.a.row0 = 0; l.a.row0 < a.rows; l.a.row0 += kBlocks * l.u.rpb) {
    const long blocks = (a.rows - l.a.row0 + l.u.rpb - 1) / l.u.rpb;
    const dim3 grid((unsigned)std::min(blocks, kBlocks), (l.u.per_row + l.u.upb - 1) / l.u.upb);
    const hipError_t e = launch_k(qk_kernel<T, V, GL, C, HP>, grid, dim3(256), 0, s, l);
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}
template <class T, int V, int GL, int C>
hipError_t launch_v(const QkArgs& a, hipStream_t s) {
  if constexpr (GL <= 16 && V > 1) {
    if (many_heads(a.rows, a.q.heads, a.k.heads, GL)) return launch_h<T, V, GL, C, 2>(a, s);
  }
  return launch_h<T, V, GL, C, 1>(a, s);
}

// lanes of a head: the power of two that covers its chunks, of which kMaxPairs / V at most
template <class T, int V>
hipError_t launch_lanes(const QkArgs& a, hipStream_t s) {
  const int chunks = a.head_dim / 2 / V;
  if (chunks <= 4) return launch_v<T, V, 4, 1>(a, s);
  if (chunks <= 8) return launch_v<T, V, 8, 1>(a, s);
  if constexpr (kMaxPairs / V > 16) {
    if (chunks > 32) {
      if constexpr (kMaxPairs / V > 32) return launch_v<T, V, 64, 1>(a, s);
    }
    if (chunks > 16) return launch_v<T, V, 32, 1>(a, s);
  }
  return launch_v<T, V, 16, 1>(a, s);
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
    if (chunks_aligned(a, 2)) return launch_lanes<uint16_t, 2>(a, s);
    return launch_v<uint16_t, 1, 64, 2>(a, s);
  }
  if (chunks_aligned(a, 4)) return launch_lanes<float, 4>(a, s);
  if (chunks_aligned(a, 2)) return launch_lanes<float, 2>(a, s);
  return launch_v<float, 1, 64, 2>(a, s);
}

hipError_t launch_qk_layer(const QkLayerArgs& a, int rows, hipStream_t s) {
  const int H = a.sh.H;
  auto go = [&](auto t, auto v, auto gl, auto hp) {
    using T = decltype(t);
    constexpr int V = decltype(v)::value, GL = decltype(gl)::value, HP = decltype(hp)::value, HB = (256 / GL + 15) / 16;
    QkLayerLaunch l{a, units_of<GL>(H, 0, HP), 0};
    l.qblocks = (rows + l.u.rpb - 1) / l.u.rpb * ((l.u.per_row + l.u.upb - 1) / l.u.upb);
    const unsigned kblocks = (unsigned)(rows + 15) / 16 * ((H + HB - 1) / HB);
    return launch_k(qk_layer_kernel<T, V, GL, HP>, dim3(l.qblocks + kblocks), dim3(256), 0, s, l);
  };
  auto heads = [&](auto t, auto v, auto gl) {
    if (many_heads(rows, H, H, decltype(gl)::value)) return go(t, v, gl, std::integral_constant<int, 2>{});
    return go(t, v, gl, std::integral_constant<int, 1>{});
  };
  auto lanes = [&](auto t, auto v) {
    const int chunks = a.sh.dh / 2 / decltype(v)::value;
    if (chunks <= 4) return heads(t, v, std::integral_constant<int, 4>{});
    if constexpr (kMaxHeadDim / 2 / decltype(v)::value > 8) {
      if (chunks > 8) return heads(t, v, std::integral_constant<int, 16>{});
    }
    return heads(t, v, std::integral_constant<int, 8>{});
  };
  if (!a.sh.dtype) return lanes(float{}, std::integral_constant<int, 4>{});
  if (a.sh.dh % 16 == 0) return lanes(uint16_t{}, std::integral_constant<int, 8>{});
  return lanes(uint16_t{}, std::integral_constant<int, 4>{});
}

}  // namespace incvit
