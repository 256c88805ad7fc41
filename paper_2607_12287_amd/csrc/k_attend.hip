// Attention over keys and values in their own type, packed sequences.
//
// As over the cache (the same row tiles, shares of keys, softmax and joins), with
// other operands: a wave has 32 keys at once, S^T = K Q^T with the keys' rows as
// loaded, O^T = V^T P^T with values that go through LDS rows, from which bf16 is
// read transposed.  fp32 multiplies in fp32.  bf16: the sum is of the weights as
// rounded, so that a key that carries a row alone leaves no rounding there.
//
// Bound by the keys' and values' bytes for few rows: 8 sequences of 8192 keys, one
// row each, 16 + 4 heads of 128, bf16: 34 us with the join, 3.9 TB/s; fp32 62.5 us, 4.3
// TB/s.  The next tile's keys, and its values where registers hold them, are on the
// way while one is worked on.
#include "attend_plain.hpp"

namespace incvit {

namespace {

template <class T, int DS>
__global__ __launch_bounds__(64 * kKeyWaves) void attend_kernel(AttendArgs a) {
  constexpr int NT = 1;  // 16-row tiles of a workgroup (attend_plan)
  constexpr int NP = DS / 16, NC = DS / 32 + (DS % 32 != 0), TR = 16 * NT, RB = value_bytes<T, DS>();
  constexpr int PER = DS / 8, NV = (kKeyTile * PER + 63) / 64;  // 8-dim pieces of a row of values, of a lane
  constexpr bool AHEAD = DS * sizeof(T) <= 384;  // whether registers hold the next tile's values as well
  extern __shared__ __align__(16) char lds[];
  const int lane = threadIdx.x & 63, g = lane >> 4, n = lane & 15;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int h = blockIdx.x % a.hk;
  RowTile w;
  KeyTiles kt;
  Share sh;
  if (!my_share(a, blockIdx.x / a.hk, w, kt, sh)) return;
  const int i1 = min(kt.nt, (sh.share + 1) * sh.per);
  const int first = sh.share * sh.per + wave;
  int i = first;

  const T* keys = static_cast<const T*>(a.k.p) + w.k0 * a.k.row + (long)h * a.k.head;
  const T* values = static_cast<const T*>(a.v.p) + w.k0 * a.v.row + (long)h * a.v.head;
  char* vbuf = lds + wave * kKeyTile * RB;

  V8<T> kraw[2][NC], vraw[NV];
  auto load_keys = [&](int tile) {
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      const T* src = keys + (long)min(tile * kKeyTile + 16 * u + n, w.len - 1) * a.k.row;
#pragma unroll
      for (int c = 0; c < NC; ++c) {
        const int d = 32 * c + 8 * g;
        kraw[u][c].load(src + (d < a.d ? d : 0));
        if (d >= a.d) kraw[u][c].zero();
      }
    }
  };
  auto load_values = [&](int tile) {
#pragma unroll
    for (int k = 0; k < NV; ++k) {
      const int e = k * 64 + lane, r = e / PER, d = (e - r * PER) * 8, key = tile * kKeyTile + r;
      const bool in = r < kKeyTile && key < w.len && d < a.d;
      vraw[k].load(values + (long)min(key, w.len - 1) * a.v.row + (d < a.d ? d : 0));
      if (!in) vraw[k].zero();
    }
  };
  auto put_values = [&]() {
#pragma unroll
    for (int k = 0; k < NV; ++k) {
      const int e = k * 64 + lane, r = e / PER, d = (e - r * PER) * 8;
      if (r < kKeyTile) *reinterpret_cast<V8<T>*>(vbuf + r * RB + d * sizeof(T)) = vraw[k];
    }
  };

  V8<T> q[NT][NC];
  Sight eye[NT];
#pragma unroll
  for (int t = 0; t < NT; ++t) {
    const int row = min(w.first + 16 * t + n, w.q_len * a.group - 1), tok = row / a.group;
    eye[t] = sight(a, w.len, w.len - w.q_len + tok);
    const T* src = static_cast<const T*>(a.q.p) + (w.q0 + tok) * a.q.row + (long)(h * a.group + row - tok * a.group) * a.q.head;
#pragma unroll
    for (int c = 0; c < NC; ++c) {
      const int d = 32 * c + 8 * g;
      q[t][c].load(src + (d < a.d ? d : 0));
      if (d >= a.d) q[t][c].zero();
    }
  }

  float m[NT], l[NT];
  bool seen[NT];
  f32x4_t o[NT][NP];
#pragma unroll
  for (int t = 0; t < NT; ++t) {
    m[t] = -INFINITY;
    l[t] = 0.0f;
    seen[t] = false;
#pragma unroll
    for (int p = 0; p < NP; ++p) o[t][p] = f32x4_t{0.0f, 0.0f, 0.0f, 0.0f};
  }

  bool odd = false;
  auto work = [&](int tile, int next) {
    const int j0 = tile * kKeyTile, j1 = j0 + kKeyTile - 1;
    const bool whole = all_seen(a, w.len, kt.p0, kt.p1, j0, j1);
    auto stage = [&]() {
      if (!whole) {
        bool any = false;
#pragma unroll
        for (int k = 0; k < NV; ++k) any |= special(vraw[k]);
        if (__any(any)) {
          odd = true;
#pragma unroll
          for (int k = 0; k < NV; ++k) drop_special(vraw[k]);
        }
      }
      put_values();
    };
    if constexpr (AHEAD) {
      stage();
      load_values(next);
    }
    f32x4_t s[NT][2];
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        s[t][u] = f32x4_t{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int c = 0; c < NC; ++c) mma(s[t][u], kraw[u][c], q[t][c]);
      }
    if constexpr (!AHEAD) {
      load_values(tile);
      stage();
    }
    load_keys(next);
    V8<T> pop[NT];
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      float y[8], p[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) y[j] = s[t][j >> 2][j & 3] * a.scale_log2;
      uint32_t see = 0xff;
      if (!whole) {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const bool v = eye[t].sees(j0 + 16 * (j >> 2) + 4 * g + (j & 3));
          see &= v ? ~0u : ~(1u << j);
          y[j] = v ? y[j] : -INFINITY;
        }
      }
      seen[t] |= see != 0;
      const float alpha = soft_step(y, m[t], l[t], p);
      if (__any(alpha != 1.0f)) {
#pragma unroll
        for (int k = 0; k < NP; ++k) o[t][k] *= alpha;
      }
      if (!whole) {
#pragma unroll
        for (int j = 0; j < 8; ++j) p[j] = see >> j & 1 ? p[j] : 0.0f;  // also where the row's scores are NaN
      }
      p_op(pop[t], p);
      if constexpr (sizeof(T) == 2) {
        float r[8];
        floats_of(pop[t], r);
#pragma unroll
        for (int j = 0; j < 8; ++j) l[t] += r[j] - p[j];
      }
    }
    // the wave's own values: its LDS operations are in order
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
#pragma unroll
    for (int k = 0; k < NP; ++k) {
      const V8<T> vop = value_op<T, RB>(vbuf, 16 * k, lane);
#pragma unroll
      for (int t = 0; t < NT; ++t) mma(o[t][k], vop, pop[t]);
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  };

  if (i < i1) {
    load_keys(kt.at(i));
    if constexpr (AHEAD) load_values(kt.at(i));
    for (; i < i1; i += kKeyWaves) work(kt.at(i), kt.at(min(i + kKeyWaves, i1 - 1)));
  }
  if (odd) {
#pragma unroll 1
    for (int e = first; e < i1; e += kKeyWaves) {
      const int j0 = kt.at(e) * kKeyTile, j1 = j0 + kKeyTile - 1;
      if (!all_seen(a, w.len, kt.p0, kt.p1, j0, j1))
        add_special<T, NP, NT>(o, eye, reinterpret_cast<const char*>(values), a.v.row * (long)sizeof(T), a.d, j0, min(j1, w.len - 1), lane);
    }
  }

  __syncthreads();  // the exchange takes the values' place
  float* s_m = reinterpret_cast<float*>(lds);
  float* s_l = s_m + kKeyWaves * TR;
  float* s_o = s_l + kKeyWaves * TR;
#pragma unroll
  for (int t = 0; t < NT; ++t) {
    const float sum = group4_sum(l[t]);
    const bool any = group4_max(seen[t] ? 1.0f : 0.0f) > 0.0f;
    const int r = wave * TR + 16 * t + n;
    if (g == 0) {
      s_m[r] = m[t] == -INFINITY && any ? kNoMax : m[t];
      s_l[r] = sum;
    }
#pragma unroll
    for (int k = 0; k < NP; ++k) *reinterpret_cast<f32x4_t*>(s_o + (size_t)r * (DS + 4) + 16 * k + 4 * g) = o[t][k];
  }
  __syncthreads();
  join_waves<T, DS, NT>(a, w, sh, lds, h, threadIdx.x);
}

template <class T, int DS>
hipError_t launch_one(const AttendArgs& a, hipStream_t s) {
  constexpr int bytes = std::max(exchange_bytes<DS, 1>(), kKeyWaves * kKeyTile * value_bytes<T, DS>());
  static_assert(bytes <= 160 * 1024, "LDS");
  const hipError_t e = with_lds<attend_kernel<T, DS>>(bytes);
  if (e != hipSuccess) return e;
  return launch_k(attend_kernel<T, DS>, dim3((unsigned)(a.shares * a.hk)), dim3(64 * kKeyWaves), (size_t)bytes, s, a);
}

template <class T>
hipError_t launch_t(const AttendArgs& a, hipStream_t s) {
  switch (kv_dims(a.d)) {
    case 32: return launch_one<T, 32>(a, s);
    case 64: return launch_one<T, 64>(a, s);
    case 80: return launch_one<T, 80>(a, s);
    case 96: return launch_one<T, 96>(a, s);
    case 128: return launch_one<T, 128>(a, s);
    case 192: return launch_one<T, 192>(a, s);
    default: return launch_one<T, 256>(a, s);
  }
}

}  // namespace

hipError_t launch_attend(const AttendArgs& a, int dtype, hipStream_t s) {
  return dtype == INCVIT_BF16 ? launch_t<uint16_t>(a, s) : launch_t<float>(a, s);
}

}  // namespace incvit
