// Attention over keys and values in their own type, for sequences of many rows.
//
// A workgroup has 64 NT rows of one key head, each of its four waves 16 NT of them,
// and takes the key tiles that any of its rows sees one after another: a tile's
// keys and values go from memory into registers while the tile before is worked
// on, then into one of two places in LDS, from which all waves read their operands.
// S^T, softmax and O^T are those of k_attend.hip, but a row stays with its wave, so
// nothing is exchanged at the end.  A wave leaves out tiles that none of its rows
// sees.
//
// Bound by the three things that a tile needs in turn, products, LDS operands and
// softmax, which two workgroups to a CU overlap in part.  A causal prompt of 8192, 16 +
// 4 heads of 128: 293 us, 939 TFLOP/s (a large library product here: 1300); matrix
// cores busy 40% of the cycles, vector instructions 55%, LDS reads 41% and their
// conflicts 10%.  Taken out of a variant of 326 us one at a time: operand reads 267,
// staging and barriers 254, softmax 293, all three 150.  32 rows of a wave: 16 took
// 437 us, since every row tile reads all operands, 64 453, with one wave to a SIMD.
// Workgroups of eight waves whose halves take turns at products and softmax 356 (308
// without), and operands read a group ahead gained nothing.  fp32, 2048 rows: 184 us,
// 93 TFLOP/s of 154.
#include "attend_plain.hpp"

namespace incvit {

namespace {

template <class T, int DS, int NT>
__global__ __launch_bounds__(64 * kKeyWaves) void attend_rows_kernel(AttendArgs a) {
  constexpr int NP = DS / 16, NC = DS / 32 + (DS % 32 != 0), RB = row_bytes<T, DS>(), VB = value_bytes<T, DS>(), EB = sizeof(T);
  constexpr int KL = rows_key_log(EB == 2, DS), KT = 1 << KL, KU = KT / 16, KS = KT / 32;
  constexpr int PER = DS / 8, NV = (KT * PER + 255) / 256;  // 8-dim pieces of a row, of a thread
  constexpr uint32_t kNowhere = 0xc0000000u;                // past every buffer's end
  extern __shared__ __align__(16) char lds[];
  __shared__ int s_special[2][kKeyWaves];
  const int tid = threadIdx.x, lane = tid & 63, g = lane >> 4, n = lane & 15;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int h = blockIdx.x % a.hk;
  RowTile w;
  KeyTiles kt;
  Share sh;
  if (!my_share(a, blockIdx.x / a.hk, w, kt, sh)) return;
  const int i0 = sh.share * sh.per, i1 = min(kt.nt, i0 + sh.per);

  const int all = w.q_len * a.group, first = w.first + wave * 16 * NT;
  const int p0 = w.len - w.q_len + min(first, all - 1) / a.group, p1 = w.len - w.q_len + (min(first + 16 * NT, all) - 1) / a.group;

  const char* keys = reinterpret_cast<const char*>(static_cast<const T*>(a.k.p) + w.k0 * a.k.row + (long)h * a.k.head);
  const char* values = reinterpret_cast<const char*>(static_cast<const T*>(a.v.p) + w.k0 * a.v.row + (long)h * a.v.head);
  const long k_row = a.k.row * EB, v_row = a.v.row * EB;
  uint32_t k_off[NV], v_off[NV];
#pragma unroll
  for (int k = 0; k < NV; ++k) {
    const int e = k * 256 + tid, r = e / PER, d = (e - r * PER) * 8;
    const bool in = r < KT && d < a.d;
    k_off[k] = in ? (uint32_t)(r * (int)k_row + d * EB) : kNowhere;
    v_off[k] = in ? (uint32_t)(r * (int)v_row + d * EB) : kNowhere;
  }
  V8<T> kraw[NV], vraw[NV];
  // rows past the sequence and dims past the head read as zeros
  auto load_tile = [&](int tile) {
    const long j0 = (long)tile * KT, left = w.len - j0 - 1;
    const Rsrc kr = make_rsrc(keys + j0 * k_row, (uint32_t)min(left * k_row + a.d * EB, 0x80000000L));
    const Rsrc vr = make_rsrc(values + j0 * v_row, (uint32_t)min(left * v_row + a.d * EB, 0x80000000L));
#pragma unroll
    for (int k = 0; k < NV; ++k) kraw[k].bload(kr, k_off[k], 0);
#pragma unroll
    for (int k = 0; k < NV; ++k) vraw[k].bload(vr, v_off[k], 0);
  };
  auto put = [&](char* buf, const V8<T>* x, int rb) {
#pragma unroll
    for (int k = 0; k < NV; ++k) {
      const int e = k * 256 + tid, r = e / PER, d = (e - r * PER) * 8;
      if (KT * PER % 256 == 0 || r < KT) *reinterpret_cast<V8<T>*>(buf + r * rb + d * EB) = x[k];
    }
  };

  V8<T> q[NT][NC];
  Sight eye[NT];
#pragma unroll
  for (int t = 0; t < NT; ++t) {
    const int row = min(first + 16 * t + n, all - 1), tok = row / a.group;
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

  auto work = [&](const char* kbuf, const char* vbuf, int tile) {
    const int j0 = tile * KT, j1 = j0 + KT - 1;
    const bool none = (first >= all) | ((a.causal != 0) & (j0 > p1)) |
                      ((a.window != 0) & (j0 >= a.sinks) & ((p0 - j1 >= a.window) | (j0 - p1 >= a.window)));
    if (none) return;
    const bool whole = all_seen(a, w.len, p0, p1, j0, j1);
    f32x4_t s[NT][KU];
    __builtin_amdgcn_s_setprio(1);  // products before the other waves' softmax
#pragma unroll
    for (int u = 0; u < KU; ++u) {
#pragma unroll
      for (int t = 0; t < NT; ++t) s[t][u] = f32x4_t{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
      for (int c = 0; c < NC; ++c) {
        V8<T> x = *reinterpret_cast<const V8<T>*>(kbuf + (16 * u + n) * RB + min(32 * c + 8 * g, DS - 8) * EB);
        if (DS % 32 != 0 && c == NC - 1 && 32 * c + 8 * g >= DS) x.zero();
#pragma unroll
        for (int t = 0; t < NT; ++t) mma(s[t][u], x, q[t][c]);
      }
    }
    __builtin_amdgcn_s_setprio(0);
    V8<T> pop[NT][KS];
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      __builtin_amdgcn_sched_barrier(0);
      uint32_t see = (1u << (4 * KU)) - 1;
      if (!whole) {
        see = 0;
#pragma unroll
        for (int j = 0; j < 4 * KU; ++j) {
          const bool v = eye[t].sees(j0 + 16 * (j >> 2) + 4 * g + (j & 3));
          see |= v ? 1u << j : 0u;
          s[t][j >> 2][j & 3] = v ? s[t][j >> 2][j & 3] : -INFINITY;
        }
      }
      seen[t] |= see != 0;
      float top = -INFINITY;
#pragma unroll
      for (int j = 0; j < 4 * KU; ++j) top = fmaxf(top, s[t][j >> 2][j & 3]);
      top = group4_max(top) * a.scale_log2;
      if (__any(top > m[t] + kSlack)) {
        const float m_new = top > m[t] + kSlack ? top : m[t];
        const float alpha = m_new == m[t] ? 1.0f : __builtin_amdgcn_exp2f(m[t] - m_new);
        l[t] *= alpha;
#pragma unroll
        for (int k = 0; k < NP; ++k) o[t][k] *= alpha;
        m[t] = m_new;
      }
      const float sub = m[t] == -INFINITY ? 0.0f : m[t];
      float p[4 * KU];
#pragma unroll
      for (int j = 0; j < 4 * KU; ++j) {
        p[j] = __builtin_amdgcn_exp2f(fmaf(s[t][j >> 2][j & 3], a.scale_log2, -sub));
        l[t] += p[j];
      }
      if (!whole) {
#pragma unroll
        for (int j = 0; j < 4 * KU; ++j) p[j] = see >> j & 1 ? p[j] : 0.0f;  // also where the row's scores are NaN
      }
#pragma unroll
      for (int b = 0; b < KS; ++b) p_op(pop[t][b], p + 8 * b);
    }
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int k = 0; k < NP; ++k)
#pragma unroll
      for (int b = 0; b < KS; ++b) {
        const V8<T> vop = value_op<T, VB>(vbuf + 32 * b * VB, 16 * k, lane);
#pragma unroll
        for (int t = 0; t < NT; ++t) mma(o[t][k], vop, pop[t][b]);
      }
  };

  bool odd = false;
  if (i0 < i1) load_tile(kt.at(i0));
  for (int i = i0; i < i1; ++i) {
    char* kbuf = lds + (i & 1) * KT * (RB + VB);
    char* vbuf = kbuf + KT * RB;
    const int tile = kt.at(i), j0 = tile * KT, j1 = j0 + KT - 1;
    __builtin_amdgcn_s_setprio(2);  // what a whole workgroup waits for goes first
    put(kbuf, kraw, RB);
    put(vbuf, vraw, VB);
    // whether every row of the workgroup sees all of the tile
    const bool whole = all_seen(a, w.len, kt.p0, kt.p1, j0, j1);
    if (!whole) {
      bool any = false;
#pragma unroll
      for (int k = 0; k < NV; ++k) any |= special(vraw[k]);
      any = __any(any);
      if (lane == 0) s_special[i & 1][wave] = any;
    }
    if (i + 1 < i1) load_tile(kt.at(i + 1));
    __builtin_amdgcn_s_setprio(0);
    __syncthreads();
    if (!whole) {
      bool here = false;
#pragma unroll
      for (int k = 0; k < kKeyWaves; ++k) here |= s_special[i & 1][k] != 0;
      if (__builtin_amdgcn_readfirstlane(here)) {
        odd = true;
#pragma unroll 1
        for (int e = tid; e < KT * PER; e += 256) {
          V8<T>* at = reinterpret_cast<V8<T>*>(vbuf + e / PER * VB + e % PER * 8 * EB);
          V8<T> x = *at;
          drop_special(x);
          *at = x;
        }
        __syncthreads();
      }
    }
    work(kbuf, vbuf, tile);
  }
  if (odd) {
#pragma unroll 1
    for (int i = i0; i < i1; ++i) {
      const int j0 = kt.at(i) * KT, j1 = j0 + KT - 1;
      if (!all_seen(a, w.len, kt.p0, kt.p1, j0, j1))
        add_special<T, NP, NT>(o, eye, values, v_row, a.d, j0, min(j1, w.len - 1), lane);
    }
  }

  // a lane has dims 16 k + 4 g .. + 3 of its rows
  if (sh.n == 1) __syncthreads();  // the rows take the tiles' place
  char* rows = lds + wave * 16 * RB;
#pragma unroll
  for (int t = 0; t < NT; ++t) {
    const float sum = group4_sum(l[t]);
    const bool any = group4_max(seen[t] ? 1.0f : 0.0f) > 0.0f;
    const int row0 = first + 16 * t;
    if (row0 >= all) break;
    if (sh.n > 1) {
      const int r = row0 - w.first + n;
      if (row0 + n < all) {
        float* part = a.parts + ((size_t)(sh.slot * a.hk + h) << a.row_log) * (DS + 2);
        if (g == 0)
          *(INCVIT_GLOBAL u32x2_t*)(part + 2 * r) =
              u32x2_t{__float_as_uint(m[t] == -INFINITY && any ? kNoMax : m[t]), __float_as_uint(sum)};
        part += ((size_t)2 << a.row_log) + (size_t)r * DS + 4 * g;
#pragma unroll
        for (int k = 0; k < NP; ++k) *(INCVIT_GLOBAL f32x4_t*)(part + 16 * k) = o[t][k];
      }
      continue;
    }
    const float inv = any ? 1.0f / sum : 0.0f;
#pragma unroll
    for (int k = 0; k < NP; ++k) {
      const f32x4_t y = any ? o[t][k] * inv : f32x4_t{0.0f, 0.0f, 0.0f, 0.0f};
      char* at = rows + n * RB + (16 * k + 4 * g) * EB;
      if constexpr (EB == 2) *reinterpret_cast<uint2*>(at) = make_uint2(f2bf2(y[0], y[1]), f2bf2(y[2], y[3]));
      else *reinterpret_cast<f32x4_t*>(at) = y;
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
#pragma unroll
    for (int k = 0; k < (16 * PER + 63) / 64; ++k) {
      const int e = k * 64 + lane, r = e / PER, d = (e - r * PER) * 8;
      if (r < 16 && row0 + r < all && d < a.d) {
        const int tok = (row0 + r) / a.group, head = h * a.group + row0 + r - tok * a.group;
        const V8<T> y = *reinterpret_cast<const V8<T>*>(rows + r * RB + d * EB);
        T* dst = static_cast<T*>(const_cast<void*>(a.out.p)) + (w.q0 + tok) * a.out.row + (long)head * a.out.head + d;
        if constexpr (EB == 2) {
          *(INCVIT_GLOBAL u32x4_t*)dst = __builtin_bit_cast(u32x4_t, y.v);
        } else {
          *(INCVIT_GLOBAL u32x4_t*)dst = __builtin_bit_cast(u32x4_t, y.a);
          *(INCVIT_GLOBAL u32x4_t*)(dst + 4) = __builtin_bit_cast(u32x4_t, y.b);
        }
      }
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  }
}

template <class T, int DS, int NT>
hipError_t launch_one(const AttendArgs& a, hipStream_t s) {
  constexpr int bytes = (2 << rows_key_log(sizeof(T) == 2, DS)) * (row_bytes<T, DS>() + value_bytes<T, DS>());
  static_assert(bytes <= 156 * 1024, "LDS");
  const hipError_t e = with_lds<attend_rows_kernel<T, DS, NT>>(bytes);
  if (e != hipSuccess) return e;
  return launch_k(attend_rows_kernel<T, DS, NT>, dim3((unsigned)(a.shares * a.hk)), dim3(64 * kKeyWaves), (size_t)bytes, s, a);
}

template <class T, int DS>
hipError_t launch_ds(const AttendArgs& a, int nt, hipStream_t s) {
  constexpr int most = most_wave_tiles(sizeof(T) == 2, DS);
  if constexpr (most >= 2) {
    if (nt == 2) return launch_one<T, DS, 2>(a, s);
  }
  return launch_one<T, DS, 1>(a, s);
}

template <class T>
hipError_t launch_t(const AttendArgs& a, int nt, hipStream_t s) {
  switch (kv_dims(a.d)) {
    case 32: return launch_ds<T, 32>(a, nt, s);
    case 64: return launch_ds<T, 64>(a, nt, s);
    case 80: return launch_ds<T, 80>(a, nt, s);
    case 96: return launch_ds<T, 96>(a, nt, s);
    case 128: return launch_ds<T, 128>(a, nt, s);
    case 192: return launch_ds<T, 192>(a, nt, s);
    default: return launch_ds<T, 256>(a, nt, s);
  }
}

}  // namespace

hipError_t launch_attend_rows(const AttendArgs& a, const AttendPlan& p, int dtype, hipStream_t s) {
  return dtype == INCVIT_BF16 ? launch_t<uint16_t>(a, p.nt, s) : launch_t<float>(a, p.nt, s);
}

}  // namespace incvit
