// Attention over the cache of keys and values in 8 bits.
//
// A workgroup has 16 NT rows of one key head (the tokens of a sequence with the
// query heads of the group) and a share of the key tiles that they see; its four
// waves take the tiles of 32 keys in turn, each for all rows, and join their
// results at the end.  Per tile a wave forms S^T = K Q^T, so that a lane keeps one
// query and four keys of each group of 16; updates that query's softmax; and
// accumulates O^T = V^T P^T, for which the lane's P is the operand as it stands.
// Keys and values come from the cache in operand order, one load per lane and
// 64 dims, without LDS; integers are exact in bf16.  Scales go on the scores and
// on P.  fp32: queries and P as sums of three bf16 numbers, which is exact.  bf16: P as
// two, within 2^-15, since few keys may carry a row (rounded to one, a row of one key was
// off by two roundings); the loads hide the second product.
//
// fp32 has no form by rows and takes this one for any: 64 rows over 8192 keys, 16 + 4
// heads of 128, 35 us; 1024 249 us, 259 TFLOP/s (what fp32 products reach here: 154).
//
// A few rows are bound by the cache's bytes, so waves have keys and not rows: every
// byte is loaded once for all heads of a group, 16 NT queries to a load.  32 sequences
// over 152 k keys, 16 + 4 heads of 128 (156 MB): 35 us with the join, 4.4 TB/s, each
// byte once by the counters; 256
// sequences of 1000 keys 46 us, 5.7 TB/s; one of 777 keys 11.3 us, a workgroup's chain
// of table, scales, keys and values seven times over.  Two tiles of loads ahead in
// registers let three workgroups share a CU; looking up blocks and scales a lane at a
// time gained nothing and left registers in memory.
#include "attend.hpp"

namespace incvit {

namespace {

template <int P>
__device__ __forceinline__ void load_dwords(const char* p, uint32_t* w) {
  if constexpr (P == 4) {
    const u32x4_t v = *(const INCVIT_GLOBAL u32x4_t*)p;
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = v[i];
  } else if constexpr (P == 2) {
    const u32x2_t v = *(const INCVIT_GLOBAL u32x2_t*)p;
    w[0] = v[0];
    w[1] = v[1];
  } else {
    w[0] = *(const INCVIT_GLOBAL uint32_t*)p;
  }
}

// The raw operands of a tile of 32 keys: two groups of 16.
template <int NP>
struct RawTile {
  static constexpr int NC = (NP + 3) / 4;
  uint4 k[2][NC];
  uint32_t v[2][NP];
  float ks[2], vs[2];
  int ok;  // bit u: group u lies in a block of the pool
};

// Three workgroups to a CU where the registers allow it without spills.
template <class T, int DS, int NT>
constexpr int kPerCu = NT == 1 && DS <= (sizeof(T) == 2 ? 128 : 64) ? 3 : 1;

template <class T, int DS, int NT>
__global__ __launch_bounds__(64 * kKeyWaves, (kPerCu<T, DS, NT>)) void kv_attend_kernel(AttendArgs a) {
  constexpr int NP = DS / 16, NC = (NP + 3) / 4, TAIL = NP % 4, TR = 16 * NT, PARTS = sizeof(T) == 4 ? 3 : 1, WP = sizeof(T) == 4 ? 3 : 2;
  extern __shared__ __align__(16) char lds[];
  const int lane = threadIdx.x & 63, g = lane >> 4, n = lane & 15;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  // heads first: a head's workgroups share an XCD's L2 where heads are a multiple of 8
  const int h = blockIdx.x % a.hk;
  RowTile w;
  KeyTiles kt;
  Share sh;
  if (!my_share(a, blockIdx.x / a.hk, w, kt, sh)) return;
  const int i1 = min(kt.nt, (sh.share + 1) * sh.per);
  int i = sh.share * sh.per + wave;

  const int* table = a.table + (long)w.seq * a.table_stride;
  const int mask = (1 << a.lb) - 1;
  const size_t half = (size_t)(16 << a.lb) * DS;  // bytes of a block's keys
  const char* data = a.cache + a.data + (size_t)h * 2 * half;
  const float* scales = reinterpret_cast<const float*>(a.cache) + 2 * h;

  auto block_of = [&](int tile, int u) {
    const int e = (2 * tile + u) >> a.lb;
    return e < a.width ? gbl(table)[e] : -1;
  };
  auto load_tile = [&](RawTile<NP>& t, int tile, const int* blk) {
    t.ok = 0;
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      const bool in = blk[u] >= 0 && blk[u] < a.blocks;
      const int b = in ? blk[u] : 0;
      t.ok |= (in ? 1 : 0) << u;
      const char* p = data + (size_t)b * a.hk * 2 * half + (size_t)((2 * tile + u) & mask) * (16 * DS);
      const float* s = scales + (size_t)b * a.hk * 2;
      t.ks[u] = gbl(s)[0];
      t.vs[u] = gbl(s)[1];
#pragma unroll
      for (int c = 0; c < NC; ++c) {
        const bool there = TAIL == 0 || c < NC - 1 || g < TAIL;
        const u32x4_t x = *(const INCVIT_GLOBAL u32x4_t*)(p + c * 1024 + (there ? lane : n) * 16);
        t.k[u][c] = there ? make_uint4(x[0], x[1], x[2], x[3]) : make_uint4(0, 0, 0, 0);
      }
#pragma unroll
      for (int c = 0; c < NC; ++c) {
        if (TAIL == 0 || c < NC - 1) load_dwords<4>(p + half + c * 1024 + lane * 16, &t.v[u][4 * c]);
        else load_dwords<TAIL == 0 ? 4 : TAIL>(p + half + c * 1024 + lane * 4 * TAIL, &t.v[u][4 * c]);
      }
    }
  };

  // queries: lane (g, n) has dims 64 c + 16 g .. + 15 of row n
  uint4 q[NT][2 * NC][PARTS];
  Sight eye[NT];
#pragma unroll
  for (int t = 0; t < NT; ++t) {
    const int row = min(w.first + 16 * t + n, w.q_len * a.group - 1), tok = row / a.group;
    eye[t] = sight(a, w.len, w.len - w.q_len + tok);
    const T* src = static_cast<const T*>(a.q.p) + (w.q0 + tok) * a.q.row + (long)(h * a.group + row - tok * a.group) * a.q.head;
#pragma unroll
    for (int c = 0; c < 2 * NC; ++c) {
      const int d = 64 * (c >> 1) + 16 * g + 8 * (c & 1);
      const bool there = d < a.d;
      V8<T> x;
      x.load(src + (there ? d : 0));
      if (!there) x.zero();
      if constexpr (PARTS == 1) {
        q[t][c][0] = x.v;
      } else {
        float y[8];
        floats_of(x, y);
        split8<PARTS>(y, q[t][c]);
      }
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

  auto work = [&](const RawTile<NP>& x, int tile) {
    f32x4_t s[NT][2];
#pragma unroll
    for (int t = 0; t < NT; ++t) s[t][0] = s[t][1] = f32x4_t{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int u = 0; u < 2; ++u)
#pragma unroll
      for (int c = 0; c < 2 * NC; ++c) {
        const uint4 kw = x.k[u][c >> 1];
        const uint4 kop = c & 1 ? bf_of_i8x8(kw.z, kw.w) : bf_of_i8x8(kw.x, kw.y);
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
          for (int k = 0; k < PARTS; ++k) s[t][u] = mma16(kop, q[t][c][k], s[t][u]);
      }
    const int j0 = tile * kKeyTile, j1 = j0 + kKeyTile - 1;
    const bool whole = (x.ok == 3) & all_seen(a, w.len, kt.p0, kt.p1, j0, j1);
    const float c0 = x.ks[0] * a.scale_log2, c1 = x.ks[1] * a.scale_log2;
    uint4 pop[NT][WP];
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      float y[8], p[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) y[j] = s[t][j >> 2][j & 3] * (j < 4 ? c0 : c1);
      uint32_t see = 0xff;
      if (!whole) {  // the same for the wave
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const bool v = eye[t].sees(j0 + 16 * (j >> 2) + 4 * g + (j & 3)) & ((x.ok >> (j >> 2) & 1) != 0);
          see &= v ? ~0u : ~(1u << j);
          y[j] = v ? y[j] : -INFINITY;
        }
      }
      seen[t] |= see != 0;
      const float alpha = soft_step(y, m[t], l[t], p);
#pragma unroll
      for (int j = 0; j < 8; ++j) p[j] *= j < 4 ? x.vs[0] : x.vs[1];
      if (!whole) {
#pragma unroll
        for (int j = 0; j < 8; ++j) p[j] = see >> j & 1 ? p[j] : 0.0f;  // whatever the scale of a value that is not seen
      }
      split8<WP>(p, pop[t]);
      if (__any(alpha != 1.0f)) {
#pragma unroll
        for (int k = 0; k < NP; ++k) o[t][k] *= alpha;
      }
    }
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int k = 0; k < NP; ++k) {
      const uint4 vop = bf_of_i8x8(x.v[0][k], x.v[1][k]);
#pragma unroll
      for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int r = 0; r < WP; ++r) o[t][k] = mma16(vop, pop[t][r], o[t][k]);
    }
  };

  // the next tile's operands are loaded, and the one after's blocks looked up,
  // while a tile is worked on
  if (i < i1) {
    RawTile<NP> x[2];
    int blk[2];
    auto look = [&](int j) {
      const int tile = kt.at(min(j, i1 - 1));
      blk[0] = block_of(tile, 0);
      blk[1] = block_of(tile, 1);
    };
    look(i);
    load_tile(x[0], kt.at(i), blk);
    look(i + kKeyWaves);
    while (true) {
      load_tile(x[1], kt.at(min(i + kKeyWaves, i1 - 1)), blk);
      look(i + 2 * kKeyWaves);
      work(x[0], kt.at(i));
      if ((i += kKeyWaves) >= i1) break;
      load_tile(x[0], kt.at(min(i + kKeyWaves, i1 - 1)), blk);
      look(i + 2 * kKeyWaves);
      work(x[1], kt.at(i));
      if ((i += kKeyWaves) >= i1) break;
    }
  }

  const int at = lane_now();
  float* s_m = reinterpret_cast<float*>(lds);
  float* s_l = s_m + kKeyWaves * TR;
  float* s_o = s_l + kKeyWaves * TR;
#pragma unroll
  for (int t = 0; t < NT; ++t) {
    const float sum = group4_sum(l[t]);
    const bool any = group4_max(seen[t] ? 1.0f : 0.0f) > 0.0f;
    const int r = wave * TR + 16 * t + (at & 15);
    if (at < 16) {
      s_m[r] = m[t] == -INFINITY && any ? kNoMax : m[t];
      s_l[r] = sum;
    }
    // O^T: register i of piece p is row 4 g + i of the piece, dim P (4 g + i) + p of its chunk
#pragma unroll
    for (int k = 0; k < NP; ++k) {
      const int c = k >> 2, P = TAIL != 0 && c == NC - 1 ? TAIL : 4;
#pragma unroll
      for (int j = 0; j < 4; ++j) s_o[(size_t)r * (DS + 4) + 64 * c + P * (4 * (at >> 4) + j) + (k & 3)] = o[t][k][j];
    }
  }
  __syncthreads();
  join_waves<T, DS, NT>(a, w, sh, lds, h, wave * 64 + at);
}

template <class T, int DS, int NT>
hipError_t launch_one(const AttendArgs& a, hipStream_t s) {
  constexpr int bytes = exchange_bytes<DS, NT>();
  static_assert(bytes <= 160 * 1024, "LDS");
  const hipError_t e = with_lds<kv_attend_kernel<T, DS, NT>>(bytes);
  if (e != hipSuccess) return e;
  return launch_k(kv_attend_kernel<T, DS, NT>, dim3((unsigned)(a.shares * a.hk)), dim3(64 * kKeyWaves), (size_t)bytes, s, a);
}

template <class T, int DS>
hipError_t launch_ds(const AttendArgs& a, int nt, hipStream_t s) {
  constexpr int most = most_row_tiles(sizeof(T) == 2, DS);
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

hipError_t launch_kv_attend(const AttendArgs& a, const AttendPlan& p, int dtype, hipStream_t s) {
  return dtype == INCVIT_BF16 ? launch_t<uint16_t>(a, p.nt, s) : launch_t<float>(a, p.nt, s);
}

}  // namespace incvit
