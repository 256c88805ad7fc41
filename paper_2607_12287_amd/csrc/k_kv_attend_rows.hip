// Attention over the cache in 8 bits, bf16, for sequences of many rows.
//
// As k_attend_rows.hip: a workgroup has 64 NT rows of one key head, each wave 16 NT
// of them, and the key tiles go through one of two places in LDS.  A tile is 64 keys;
// each wave takes a group of 16 from the cache while the tile before is worked on,
// turns its integers into bf16 (exact) and puts them into LDS in operand order, so
// they are turned once for all rows and read back without conflicts.  With the
// group's scales go c = ks * scale * log2(e) for its scores, log2(vs), which joins the
// exponent of the weights for the values, and 1 / vs, which takes it from their sum;
// a vs that is not near 1 (2^-60 to 2^60) multiplies the weights instead.
//
// 1024 rows over 8192 keys, 16 + 4 heads of 128: 106 us with the join, 610 TFLOP/s
// (by waves that share keys 64 more).  Of 120 us in a variant 34 are the same
// for one key tile as for sixteen: queries, partial results and the join.  What bounds
// the rest is as in k_attend_rows.hip.
#include "attend.hpp"

namespace incvit {

namespace {

template <int DS, int NT>
__global__ __launch_bounds__(64 * kKeyWaves) void kv_attend_rows_kernel(AttendArgs a) {
  constexpr int NP = DS / 16, NC = (NP + 3) / 4, TAIL = NP % 4, KT = 64, KU = 4, KS = 2;
  constexpr int KB = KU * 2 * NC * 1024, VB = KS * NP * 1024, RB = DS * 2 + 16;  // bytes of a tile's keys, values; of a row of the output
  extern __shared__ __align__(16) char lds[];  // [2][keys, values]
  __shared__ float4 s_scale[2][KU];            // c, log2(vs), 1 / vs, 1; with other scales c, vs, 1, 2; without a block 0 at the end
  const int lane = threadIdx.x & 63, g = lane >> 4, n = lane & 15;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int h = blockIdx.x % a.hk;
  RowTile w;
  KeyTiles kt;
  Share sh;
  if (!my_share(a, blockIdx.x / a.hk, w, kt, sh)) return;
  const int i0 = sh.share * sh.per, i1 = min(kt.nt, i0 + sh.per);

  const int all = w.q_len * a.group, first = w.first + wave * 16 * NT;
  const int p0 = w.len - w.q_len + min(first, all - 1) / a.group, p1 = w.len - w.q_len + (min(first + 16 * NT, all) - 1) / a.group;

  const int* table = a.table + (long)w.seq * a.table_stride;
  const int mask = (1 << a.lb) - 1;
  const size_t half = (size_t)(16 << a.lb) * DS;  // bytes of a block's keys
  const char* data = a.cache + a.data + (size_t)h * 2 * half;

  // the wave's group of a tile: group `wave`
  uint4 kraw[NC];
  uint32_t vraw[NP];
  float ks, vs;
  int there;
  GroupInfo info;  // of tile number (64 * whole) + lane
  auto load_group = [&](int i) {
    const int e = (i - i0) & 63, tile = kt.at(i);
    if (e == 0) info.load(a, table, h, KU * kt.at(min(i + lane, i1 - 1)) + wave);
    const int blk = __builtin_amdgcn_readlane(info.blk, e);
    there = blk >= 0;
    ks = lane_float(info.ks, e);
    vs = lane_float(info.vs, e);
    const char* p = data + (size_t)max(blk, 0) * a.hk * 2 * half + (size_t)((KU * tile + wave) & mask) * (16 * DS);
#pragma unroll
    for (int c = 0; c < NC; ++c) {
      const bool in = TAIL == 0 || c < NC - 1 || g < TAIL;
      const u32x4_t x = *(const INCVIT_GLOBAL u32x4_t*)(p + c * 1024 + (in ? lane : n) * 16);
      kraw[c] = in ? make_uint4(x[0], x[1], x[2], x[3]) : make_uint4(0, 0, 0, 0);
    }
#pragma unroll
    for (int c = 0; c < NC; ++c) {
      const int P = TAIL == 0 || c < NC - 1 ? 4 : TAIL;
      const char* at = p + half + c * 1024 + lane * 4 * P;
      if (P == 4) {
        const u32x4_t x = *(const INCVIT_GLOBAL u32x4_t*)at;
#pragma unroll
        for (int i = 0; i < 4; ++i) vraw[4 * c + i] = x[i];
      } else if (P == 2) {
        const u32x2_t x = *(const INCVIT_GLOBAL u32x2_t*)at;
        vraw[4 * c] = x[0];
        vraw[4 * c + (P > 1)] = x[1];
      } else {
        vraw[4 * c] = *(const INCVIT_GLOBAL uint32_t*)at;
      }
    }
  };
  auto put_group = [&](char* kbuf, char* vbuf, int at) {
#pragma unroll
    for (int c = 0; c < NC; ++c) {
      uint4* dst = reinterpret_cast<uint4*>(kbuf + (wave * 2 * NC + 2 * c) * 1024) + lane;
      dst[0] = bf_of_i8x8(kraw[c].x, kraw[c].y);
      dst[64] = bf_of_i8x8(kraw[c].z, kraw[c].w);
    }
    char* dst = vbuf + (wave >> 1) * NP * 1024 + lane * 16 + (wave & 1) * 8;
#pragma unroll
    for (int k = 0; k < NP; ++k) *reinterpret_cast<uint2*>(dst + k * 1024) = bf_of_i8(vraw[k]);
    if (lane == 0) {
      const float v = vs == 0.0f ? 1.0f : vs;  // zeros under any scale
      const bool near = v > 0x1p-60f && v < 0x1p60f;
      s_scale[at][wave] = make_float4(ks * a.scale_log2, near ? __builtin_amdgcn_logf(v) : v, near ? 1.0f / v : 1.0f,
                                      !there ? 0.0f : near ? 1.0f : 2.0f);
    }
  };

  // queries: lane (g, n) has dims 64 c + 16 g .. + 15 of row n
  uint4 q[NT][2 * NC];
  Sight eye[NT];
#pragma unroll
  for (int t = 0; t < NT; ++t) {
    const int row = min(first + 16 * t + n, all - 1), tok = row / a.group;
    eye[t] = sight(a, w.len, w.len - w.q_len + tok);
    const uint16_t* src = static_cast<const uint16_t*>(a.q.p) + (w.q0 + tok) * a.q.row + (long)(h * a.group + row - tok * a.group) * a.q.head;
#pragma unroll
    for (int c = 0; c < 2 * NC; ++c) {
      const int d = 64 * (c >> 1) + 16 * g + 8 * (c & 1);
      V8<uint16_t> x;
      x.load(src + (d < a.d ? d : 0));
      if (d >= a.d) x.zero();
      q[t][c] = x.v;
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

  auto work = [&](const char* kbuf, const char* vbuf, int tile, int at) {
    const int j0 = tile * KT, j1 = j0 + KT - 1;
    const bool none = (first >= all) | ((a.causal != 0) & (j0 > p1)) |
                      ((a.window != 0) & (j0 >= a.sinks) & ((p0 - j1 >= a.window) | (j0 - p1 >= a.window)));
    if (none) return;
    float4 z[KU];
    bool whole = all_seen(a, w.len, p0, p1, j0, j1), near = true;
#pragma unroll
    for (int u = 0; u < KU; ++u) {
      z[u] = s_scale[at][u];
      whole = whole & (z[u].w != 0.0f);
      near = near & (z[u].w != 2.0f);
    }
    whole = __builtin_amdgcn_readfirstlane(whole);
    near = __builtin_amdgcn_readfirstlane(near);
    float vs_far[KU];
    if (!near) {
#pragma unroll
      for (int u = 0; u < KU; ++u) {
        vs_far[u] = z[u].w == 2.0f ? z[u].y : 1.0f;
        z[u].y = z[u].w == 2.0f ? 0.0f : z[u].y;
      }
    }
    f32x4_t s[NT][KU];
    __builtin_amdgcn_s_setprio(1);  // products before the other waves' softmax
#pragma unroll
    for (int u = 0; u < KU; ++u) {
#pragma unroll
      for (int t = 0; t < NT; ++t) s[t][u] = f32x4_t{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
      for (int c = 0; c < 2 * NC; ++c) {
        const uint4 x = reinterpret_cast<const uint4*>(kbuf + (u * 2 * NC + c) * 1024)[lane];
#pragma unroll
        for (int t = 0; t < NT; ++t) s[t][u] = mma16(x, q[t][c], s[t][u]);
      }
    }
    __builtin_amdgcn_s_setprio(0);
    uint4 pop[NT][KS];
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      __builtin_amdgcn_sched_barrier(0);
      uint32_t see = (1u << (4 * KU)) - 1;
      if (!whole) {
        see = 0;
#pragma unroll
        for (int j = 0; j < 4 * KU; ++j) {
          const bool v = eye[t].sees(j0 + 16 * (j >> 2) + 4 * g + (j & 3)) & (z[j >> 2].w != 0.0f);
          see |= v ? 1u << j : 0u;
          s[t][j >> 2][j & 3] = v ? s[t][j >> 2][j & 3] : -INFINITY;
        }
      }
      seen[t] |= see != 0;
      // c is not below 0; a NaN (c is one, or 0 and nothing of the group is seen) does not count
      float top = -INFINITY;
#pragma unroll
      for (int u = 0; u < KU; ++u)
        top = fmaxf(top, fmaxf(fmaxf(s[t][u][0], s[t][u][1]), fmaxf(s[t][u][2], s[t][u][3])) * z[u].x);
      top = group4_max(top);
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
      for (int j = 0; j < 4 * KU; ++j) p[j] = __builtin_amdgcn_exp2f(fmaf(s[t][j >> 2][j & 3], z[j >> 2].x, z[j >> 2].y - sub));
      if (!whole) {
#pragma unroll
        for (int j = 0; j < 4 * KU; ++j) p[j] = see >> j & 1 ? p[j] : 0.0f;  // whatever the scales are
      }
#pragma unroll
      for (int u = 0; u < KU; ++u) {
        const float sum = (p[4 * u] + p[4 * u + 1]) + (p[4 * u + 2] + p[4 * u + 3]);
        l[t] = fmaf(sum, z[u].z, l[t]);
      }
      if (!near) {
#pragma unroll
        for (int j = 0; j < 4 * KU; ++j) p[j] = whole | ((see >> j & 1) != 0) ? p[j] * vs_far[j >> 2] : 0.0f;
      }
#pragma unroll
      for (int b = 0; b < KS; ++b) split8<1>(p + 8 * b, &pop[t][b]);
    }
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int k = 0; k < NP; ++k)
#pragma unroll
      for (int b = 0; b < KS; ++b) {
        const uint4 vop = reinterpret_cast<const uint4*>(vbuf + (b * NP + k) * 1024)[lane];
#pragma unroll
        for (int t = 0; t < NT; ++t) o[t][k] = mma16(vop, pop[t][b], o[t][k]);
      }
  };

  // the next tile's group is loaded while a tile is worked on
  if (i0 < i1) load_group(i0);
  for (int i = i0; i < i1; ++i) {
    char* kbuf = lds + (i & 1) * (KB + VB);
    __builtin_amdgcn_s_setprio(2);  // what a whole workgroup waits for goes first
    put_group(kbuf, kbuf + KB, i & 1);
    if (i + 1 < i1) load_group(i + 1);
    __builtin_amdgcn_s_setprio(0);
    __syncthreads();
    work(kbuf, kbuf + KB, kt.at(i), i & 1);
  }

  if (sh.n == 1) __syncthreads();  // the rows take the tiles' place
  char* rows = lds + wave * 16 * RB;
#pragma unroll
  for (int t = 0; t < NT; ++t) {
    const float sum = group4_sum(l[t]);
    const bool any = group4_max(seen[t] ? 1.0f : 0.0f) > 0.0f;
    const int row0 = first + 16 * t;
    if (row0 >= all) break;
    float* part = nullptr;
    if (sh.n > 1) {
      part = a.parts + ((size_t)(sh.slot * a.hk + h) << a.row_log) * (DS + 2);
      const int r = row0 - w.first + n;
      if (row0 + n < all && g == 0)
        *(INCVIT_GLOBAL u32x2_t*)(part + 2 * r) = u32x2_t{__float_as_uint(m[t] == -INFINITY && any ? kNoMax : m[t]), __float_as_uint(sum)};
      part += ((size_t)2 << a.row_log) + (size_t)r * DS;
    }
    const float inv = any ? 1.0f / sum : 0.0f;
    // register j of piece k is row 4 g + j of the piece, dim P (4 g + j) + p of its
    // chunk: 4 P dims of a lane's row follow one another
#pragma unroll
    for (int c = 0; c < NC; ++c) {
      constexpr int kLast = TAIL == 0 ? 4 : TAIL;
      const int P = c < NC - 1 ? 4 : kLast, d = 64 * c + 4 * P * g;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        if (i >= P) continue;
        f32x4_t x;  // dims d + 4 i ..
#pragma unroll
        for (int e = 0; e < 4; ++e) x[e] = o[t][min(4 * c + (4 * i + e) % P, NP - 1)][(4 * i + e) / P];
        if (sh.n > 1) {
          if (row0 + n < all) *(INCVIT_GLOBAL f32x4_t*)(part + d + 4 * i) = x;
        } else {
          x = any ? x * inv : f32x4_t{0.0f, 0.0f, 0.0f, 0.0f};
          *reinterpret_cast<uint2*>(rows + n * RB + (d + 4 * i) * 2) = make_uint2(f2bf2(x[0], x[1]), f2bf2(x[2], x[3]));
        }
      }
    }
    if (sh.n > 1) continue;
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
#pragma unroll
    for (int k = 0; k < (16 * DS / 8 + 63) / 64; ++k) {
      const int e = k * 64 + lane, r = e / (DS / 8), d = (e - r * (DS / 8)) * 8;
      if (r < 16 && row0 + r < all && d < a.d) {
        const int tok = (row0 + r) / a.group, head = h * a.group + row0 + r - tok * a.group;
        const u32x4_t y = *reinterpret_cast<const u32x4_t*>(rows + r * RB + d * 2);
        uint16_t* dst = static_cast<uint16_t*>(const_cast<void*>(a.out.p)) + (w.q0 + tok) * a.out.row + (long)head * a.out.head + d;
        *(INCVIT_GLOBAL u32x4_t*)dst = y;
      }
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  }
}

template <int DS>
hipError_t launch_one(const AttendArgs& a, hipStream_t s) {
  constexpr int NT = cached_wave_tiles(DS), NP = DS / 16, NC = (NP + 3) / 4, bytes = 2 * (8 * NC + 2 * NP) * 1024;
  static_assert(bytes <= 156 * 1024 && bytes >= 64 * (DS * 2 + 16), "LDS");
  const hipError_t e = with_lds<kv_attend_rows_kernel<DS, NT>>(bytes);
  if (e != hipSuccess) return e;
  return launch_k(kv_attend_rows_kernel<DS, NT>, dim3((unsigned)(a.shares * a.hk)), dim3(64 * kKeyWaves), (size_t)bytes, s, a);
}

}  // namespace

hipError_t launch_kv_attend_rows(const AttendArgs& a, hipStream_t s) {
  switch (kv_dims(a.d)) {
    case 32: return launch_one<32>(a, s);
    case 64: return launch_one<64>(a, s);
    case 80: return launch_one<80>(a, s);
    case 96: return launch_one<96>(a, s);
    case 128: return launch_one<128>(a, s);
    case 192: return launch_one<192>(a, s);
    default: return launch_one<256>(a, s);
  }
}

}  // namespace incvit
