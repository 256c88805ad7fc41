// The cache of keys and values in 8 bits and the attention operators: layouts,
// arguments, launchers, and what both attention kernels share.
#pragma once

#include <atomic>

#include "ops.hpp"

namespace incvit {

// ------------------------------------------------------------------ cache --

// Head dims are stored padded to one of these.
__host__ __device__ constexpr int kv_dims(int d) {
  return d <= 32 ? 32 : d <= 64 ? 64 : d <= 80 ? 80 : d <= 96 ? 96 : d <= 128 ? 128 : d <= 192 ? 192 : 256;
}

// Scales [blocks][heads] (key, value), then the integers [blocks][heads]: a block
// of a head is its keys (block * ds bytes), then its values.  Both lie in groups
// of 16 tokens (16 * ds bytes), in the operand order of the attention's matrix
// instructions, so that one load per lane is one operand:
//   keys:   [dims / 16][token][16 dims];
//   values: chunks of 64 dims (the last of the 16 P that are left, P = 1, 2 or 4);
//           a chunk is [token / 4][16 P dims][token % 4].
struct KvLayout {
  int block, heads, ds, lb;  // lb: log2 of a block's groups
  size_t head_bytes;         // of one block and head: keys and values
  size_t data, total;
  __host__ __device__ KvLayout(int blocks, int block_, int heads_, int d) : block(block_), heads(heads_), ds(kv_dims(d)) {
    lb = block == 16 ? 0 : block == 32 ? 1 : block == 64 ? 2 : 3;
    head_bytes = (size_t)2 * block * ds;
    data = q_align((size_t)blocks * heads * 8);
    total = data + q_align((size_t)blocks * heads * head_bytes);
  }
};

struct KvSide {
  const void* p;
  long row, head;
};

struct KvWriteArgs {
  KvSide x[2];  // keys, values
  const int* slots;
  char* cache;
  size_t data;
  long rows;
  int blocks, block, heads, d, begin, dtype;
  int each;  // rows of a wave
};

struct KvReadArgs {
  KvSide x[2];  // written
  const int* slots;
  const char* cache;
  size_t data;
  long rows;
  int blocks, block, heads, d, dtype, fill;
  uint32_t per_inv;  // 2^32 / (d / 8), rounded up
};

hipError_t launch_kv_write(const KvWriteArgs& a, hipStream_t s);
hipError_t launch_kv_read(const KvReadArgs& a, hipStream_t s);

// -------------------------------------------------------------- attention --

constexpr int kKeyTile = 32;   // keys that a wave takes at once where the waves of a workgroup share its keys
constexpr int kKeyWaves = 4;   // waves of a workgroup
constexpr int kMostShares = 256;  // of a row tile's keys
constexpr int kMostKeys = 1 << 30;  // of a sequence that are looked at: no position overflows
constexpr int kEvenTiles = 64;    // sequences whose shares are made even: the lanes of a wave (a batch of 32, 200 to 16384 keys: 35 us, without 48)

struct AttendArgs {
  const int* q_start;  // null: q_len rows for each sequence
  const int* k_start;  // plain: null: k_len keys for each
  const int* lens;     // cached
  const int* table;
  const char* cache;
  size_t data;         // of the cache's integers
  KvSide q, k, v, out;
  long table_stride;
  float* parts;        // workspace
  long rows, key_rows;
  int n, q_len, k_len, width, blocks, lb;
  int hk, group, d;
  int causal, window, sinks;
  int fill;            // with q_start: rows behind the last sequence as those of one without keys
  float scale_log2;    // scale * log2(e)
  long shares;         // workgroups of a head
  int most_rows;       // rows * group of a sequence at most
  int row_log, key_log;  // rows of a row tile and keys of a key tile: powers of two
  int tiles;           // row tiles of the call
  int tiles_each;      // of each sequence (q_start null)
  // workgroups that share a row tile's keys: at most `splits` for each, of at least
  // `chunk` key tiles; or (even > 0) as many as give `even` to a head in all, each of
  // about as many key tiles, at least `chunk`
  int splits, chunk, even;
};

// 16-row tiles of a workgroup over the cache, at most: as many as the registers hold.
constexpr int most_row_tiles(bool bf16, int ds) { return ds <= (bf16 ? 192 : 128) ? 2 : 1; }

// 16-row tiles of a wave of its own rows, at most (fp32 with two takes all registers
// of a SIMD for one wave: a prompt of 2048 and heads of 128 295 us against 226); keys
// of a tile there: 64, or 32 in fp32 where two workgroups then fit a CU's LDS (8192
// keys, window 500, heads of 64: 181 us with 64, 160 with 32; heads of 128: 182, 227)
constexpr int most_wave_tiles(bool bf16, int ds) { return bf16 ? 2 : 1; }
constexpr int cached_wave_tiles(int ds) { return ds <= 128 ? 2 : 1; }
constexpr int rows_key_log(bool bf16, int ds) { return bf16 || ds == 128 ? 6 : 5; }

struct AttendPlan {
  int by_rows;         // the waves have rows of their own (else keys)
  int nt;              // 16-row tiles of a workgroup, or of a wave of its own rows
  int row_log, key_log;
  long tiles;          // row tiles
  int tiles_each, splits, chunk, even;
  long shares;         // of a head at most
  size_t bytes;        // workspace
};
AttendPlan attend_plan(const incvit_attention& a, bool cached, long n, long rows, bool ragged, long max_len);

hipError_t launch_kv_attend(const AttendArgs& a, const AttendPlan& p, int dtype, hipStream_t s);
hipError_t launch_attend(const AttendArgs& a, int dtype, hipStream_t s);
hipError_t launch_kv_attend_rows(const AttendArgs& a, hipStream_t s);
hipError_t launch_attend_rows(const AttendArgs& a, const AttendPlan& p, int dtype, hipStream_t s);
hipError_t launch_attend_join(const AttendArgs& a, int dtype, hipStream_t s);

}  // namespace incvit

#if defined(__HIPCC__)
namespace incvit {

// Where a row tile is: rows [first, first + rows) of a sequence's q_len * group
// rows (token by token, the heads of a group together), whose token 0 is row q0
// of the call; its keys: k0 (plain) and len.
struct RowTile {
  int seq, first, q_len, len;
  long q0, k0;
};

// The tile number f of the launch.  Ragged: sequence i's tiles count from
// floor(q_start[i] * group / rows of a tile) + i on, which leaves each enough numbers,
// and a wave counts the starts up to f by a search over 64 of them at a time.
// Whatever the starts hold, the rows are within the call's.
__device__ __forceinline__ bool row_tile(const AttendArgs& a, int f, RowTile& w) {
  const int log = a.row_log;
  if (!a.q_start) {
    w.seq = f / a.tiles_each;
    w.first = (f - w.seq * a.tiles_each) << log;
    w.q_len = a.q_len;
    w.q0 = (long)w.seq * a.q_len;
  } else {
    const int lane = threadIdx.x & 63;
    int count = 0;  // starts up to f: `left` ones from `count` on are open
    for (int left = a.n + a.fill; left > 0;) {
      const int step = (left + 63) / 64, j = count + lane * step;
      const long at = min(max((long)gbl(a.q_start)[min(j, a.n)], 0L), a.rows);
      const int up = __popcll(__ballot((lane * step < left) & (((at * a.group) >> log) + j <= f)));
      if (up == 0) break;
      count += (up - 1) * step + 1;
      left = min(step - 1, left - (up - 1) * step - 1);
    }
    if (count == 0) return false;
    w.seq = __builtin_amdgcn_readfirstlane(count - 1);
    const long q0 = min(max((long)gbl(a.q_start)[w.seq], 0L), a.rows);
    const long q1 = w.seq < a.n ? min(max((long)gbl(a.q_start)[w.seq + 1], q0), a.rows) : a.rows;
    w.first = (int)(f - ((q0 * a.group) >> log) - w.seq) * (1 << log);
    w.q_len = (int)(q1 - q0);
    w.q0 = q0;
  }
  return w.first >= 0 && w.first < w.q_len * a.group;  // below 0: starts that do not ascend
}

__device__ __forceinline__ int cached_len(const AttendArgs& a, int seq) {
  if (seq >= a.n) return 0;
  return max(min(gbl(a.lens)[seq], (int)min((long)a.width * (16 << a.lb), (long)kMostKeys)), 0);
}
// (and the first one's row, k0)
__device__ __forceinline__ int plain_len(const AttendArgs& a, RowTile& w) {
  w.k0 = (long)w.seq * a.k_len;
  if (w.seq >= a.n) return 0;
  if (!a.k_start) return a.k_len;
  const long k0 = min(max((long)gbl(a.k_start)[w.seq], 0L), a.key_rows), k1 = min(max((long)gbl(a.k_start)[w.seq + 1], k0), a.key_rows);
  w.k0 = k0;
  return (int)(k1 - k0);
}

// Key tiles that some row of a row tile sees: n0 from key 0 on (the sinks, where
// they are apart from the window), then those from `t1` on; nt in all.  p0, p1:
// the first and the last row's position.
struct KeyTiles {
  int n0, t1, nt;
  int p0, p1;
  __device__ __forceinline__ int at(int i) const { return i < n0 ? i : i - n0 + t1; }
};
__device__ __forceinline__ KeyTiles key_tiles(const AttendArgs& a, int len, int p0, int p1) {
  const int log = a.key_log, up = (1 << log) - 1;
  KeyTiles k;
  k.p0 = p0;
  k.p1 = p1;
  const int top = max(0, a.causal ? min(len, p1 + 1) : len);
  int lo = 0, hi = top;
  k.n0 = 0;
  if (a.window) {
    lo = max(0, p0 - a.window + 1);
    if (!a.causal) hi = max(0, min(top, p1 + a.window));  // both at most 2^30
  }
  k.t1 = lo >> log;
  int t2 = lo < hi ? (hi + up) >> log : k.t1;
  if (a.window && a.sinks) {
    const int s = (min(a.sinks, top) + up) >> log;
    if (s >= k.t1) {
      k.t1 = 0;
      t2 = max(t2, s);
    } else {
      k.n0 = s;
    }
  }
  k.nt = k.n0 + t2 - k.t1;
  return k;
}
__device__ __forceinline__ KeyTiles key_tiles(const AttendArgs& a, const RowTile& w) {
  const int last = min(w.first + (1 << a.row_log), w.q_len * a.group) - 1, at = w.len - w.q_len;
  return key_tiles(a, w.len, at + w.first / a.group, at + last / a.group);
}

// A workgroup's share of a row tile's keys: tiles [share * per, + per) of nt, the
// n-th part; its partial result is number `slot` (of the call's, for a head).
struct Share {
  int f, share, n, per;
  long slot;
};

__device__ __forceinline__ int seq_len(const AttendArgs& a, RowTile& w) { return a.lens ? cached_len(a, w.seq) : plain_len(a, w); }

// Sums over the lanes up to each.
__device__ __forceinline__ int lanes_scan(int x) {
  x += __builtin_amdgcn_update_dpp(0, x, 0x111, 0xf, 0xf, true);  // within rows of 16: from 1, 2, 4, 8 lanes before
  x += __builtin_amdgcn_update_dpp(0, x, 0x112, 0xf, 0xf, true);
  x += __builtin_amdgcn_update_dpp(0, x, 0x114, 0xf, 0xf, true);
  x += __builtin_amdgcn_update_dpp(0, x, 0x118, 0xf, 0xf, true);
  x += __builtin_amdgcn_update_dpp(0, x, 0x142, 0xa, 0xf, false);  // row 0's sum to row 1, row 2's to row 3
  x += __builtin_amdgcn_update_dpp(0, x, 0x143, 0xc, 0xf, false);  // the first two rows' sum to the others
  return x;
}

// Even shares: key tiles that one has, of `total` and at least `least`, and how many
// a sequence of nt key tiles gets.  `even` and one for each sequence are enough for
// all of them if the total counts what even_count does: kEvenMost at most, so that
// 64 of them add up within 32 bits.
constexpr int kEvenMost = 1 << 24;
__host__ __device__ constexpr int even_chunk(int total, int least, int even) {
  const int chunk = (total + even - 1) / even;
  return chunk > least ? chunk : least;
}
__host__ __device__ constexpr int even_count(int nt, int chunk) {
  const int n = ((nt < kEvenMost ? nt : kEvenMost) + chunk - 1) / chunk;
  return n < 1 ? 1 : n < kMostShares ? n : kMostShares;
}

// Even shares, for up to 64 sequences of one row tile each: every wave has their key
// tiles in its lanes, which gives the size of a share, and from the shares before
// each sequence its own.  want: share number (of a head), or with TILE the sequence
// whose shares are asked for.
template <bool TILE>
__device__ __forceinline__ bool even_share(const AttendArgs& a, int want, Share& s) {
  const int lane = threadIdx.x & 63;
  const bool in = lane < a.tiles;
  RowTile w;
  w.seq = min(lane, a.tiles - 1);
  const int len = seq_len(a, w), nt = in ? key_tiles(a, len, len - a.q_len, len - 1).nt : 0;
  const int total = __builtin_amdgcn_readlane(lanes_scan(min(nt, kEvenMost)), 63), chunk = even_chunk(total, a.chunk, a.even);
  const int n = in ? even_count(nt, chunk) : 0, upto = lanes_scan(n);
  const uint64_t there = __ballot(TILE ? lane == want : in & (upto > want));
  if (!there) return false;
  s.f = __builtin_ctzll(there);
  s.n = __builtin_amdgcn_readlane(n, s.f);
  s.per = (__builtin_amdgcn_readlane(nt, s.f) + s.n - 1) / s.n;
  const int first = __builtin_amdgcn_readlane(upto, s.f) - s.n;
  s.share = TILE ? 0 : want - first;
  s.slot = first + s.share;
  return true;
}

// The share of workgroup number b (of a head), its row tile and key tiles; false for
// one that has none.
__device__ __forceinline__ bool my_share(const AttendArgs& a, int b, RowTile& w, KeyTiles& k, Share& s) {
  if (a.even) {
    if (!even_share<false>(a, b, s) || !row_tile(a, s.f, w)) return false;
    w.len = seq_len(a, w);
    k = key_tiles(a, w);
    return true;
  }
  // of the row tiles the last, which see the most keys, start first
  s.share = b / a.tiles;
  s.f = a.tiles - 1 - (b - s.share * a.tiles);
  if (!row_tile(a, s.f, w)) return false;
  w.len = seq_len(a, w);
  k = key_tiles(a, w);
  s.n = max(1, min(a.splits, (k.nt + a.chunk - 1) / a.chunk));
  s.per = (k.nt + s.n - 1) / s.n;
  s.slot = (long)s.f * a.splits + s.share;
  return s.share < s.n;
}
// The shares of row tile f, to join them.
__device__ __forceinline__ bool shares_of(const AttendArgs& a, int f, RowTile& w, Share& s) {
  if (!row_tile(a, f, w)) return false;
  if (a.even) return even_share<true>(a, f, s);
  w.len = seq_len(a, w);
  s.n = max(1, min(a.splits, (key_tiles(a, w).nt + a.chunk - 1) / a.chunk));
  s.slot = (long)f * a.splits;
  return true;
}

// The keys that a row at position `pos` sees: `n` from lo on, and those below
// `sinks`.  Two comparisons without a branch (a chain of && over a lane's keys
// came out as branches, slower, and in one kernel with scores that the mask had
// taken put back).
struct Sight {
  int lo, sinks;
  uint32_t n;
  __device__ __forceinline__ bool sees(int key) const { return ((uint32_t)(key - lo) < n) | (key < sinks); }
};
__device__ __forceinline__ Sight sight(const AttendArgs& a, int len, int pos) {
  const int top = a.causal ? min(len, pos + 1) : len;
  const int hi = a.window && !a.causal ? min(top, pos + a.window) : top;
  Sight s;
  s.lo = a.window ? max(0, pos - a.window + 1) : 0;
  s.sinks = a.window ? min(a.sinks, top) : 0;
  s.n = (uint32_t)max(0, hi - s.lo);
  return s;
}

// Whether rows at positions p0 to p1 see all of the keys j0 to j1.
__device__ __forceinline__ bool all_seen(const AttendArgs& a, int len, int p0, int p1, int j0, int j1) {
  const bool window = !a.window | ((p1 - j0 < a.window) & ((a.causal != 0) | (j1 - p0 < a.window))) | (j1 < a.sinks);
  return (j1 < len) & (!a.causal | (j1 <= p0)) & window;
}

// A row's partial result: m, the largest score in units of log2; l, the sum of
// 2^(x - m); O.  m = -inf: no key was seen.  kNoMax: keys were seen, none above -inf.
constexpr float kNoMax = -3.0e38f;

// Blocks and scales of groups of 16 tokens, one in each lane: read by vector loads
// for many tiles at once.  (One by one they became scalar loads, each of which a
// wave waits for alone.)  blk: -1 where the group lies in no block of the pool.
struct GroupInfo {
  int blk;
  float ks, vs;
  __device__ __forceinline__ void load(const AttendArgs& a, const int* table, int h, int group) {
    const int e = min(group >> a.lb, a.width - 1);
    const int b = gbl(table)[e];
    const bool in = (group >> a.lb < a.width) & (b >= 0) & (b < a.blocks);
    blk = in ? b : -1;
    const u32x2_t s = *(const INCVIT_GLOBAL u32x2_t*)(a.cache + ((size_t)(in ? b : 0) * a.hk + h) * 8);
    ks = __uint_as_float(s[0]);
    vs = __uint_as_float(s[1]);
  }
};
__device__ __forceinline__ float lane_float(float x, int lane) {
  return __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(x), lane));
}

// max, sum and "any" over the four lane groups (lanes n, n + 16, n + 32, n + 48)
__device__ __forceinline__ float group4_max(float x) {
  const uint32_t u = __float_as_uint(x);
  const auto p = __builtin_amdgcn_permlane16_swap(u, u, false, false);
  const float y = fmaxf(__uint_as_float(p[0]), __uint_as_float(p[1]));
  const auto q = __builtin_amdgcn_permlane32_swap(__float_as_uint(y), __float_as_uint(y), false, false);
  return fmaxf(__uint_as_float(q[0]), __uint_as_float(q[1]));
}
__device__ __forceinline__ float group4_sum(float x) {
  const uint32_t u = __float_as_uint(x);
  const auto p = __builtin_amdgcn_permlane16_swap(u, u, false, false);
  const float y = __uint_as_float(p[0]) + __uint_as_float(p[1]);
  const auto q = __builtin_amdgcn_permlane32_swap(__float_as_uint(y), __float_as_uint(y), false, false);
  return __uint_as_float(q[0]) + __uint_as_float(q[1]);
}

// four 8-bit integers as bf16, which is exact
__device__ __forceinline__ uint2 bf_of_i8(uint32_t w) {
  const float a = (float)(int8_t)w, b = (float)(int8_t)(w >> 8), c = (float)(int8_t)(w >> 16), d = (float)(int8_t)(w >> 24);
  return make_uint2(f2bf2(a, b), f2bf2(c, d));
}
__device__ __forceinline__ uint4 bf_of_i8x8(uint32_t w0, uint32_t w1) {
  const uint2 a = bf_of_i8(w0), b = bf_of_i8(w1);
  return make_uint4(a.x, a.y, b.x, b.y);
}

// fp32 values as sums of bf16 numbers, without a rounding: the leading 8 bits of
// the significand, the next 8 and the last 8.
__device__ __forceinline__ uint32_t top_halves(float lo, float hi) {
  return __builtin_amdgcn_perm(__float_as_uint(hi), __float_as_uint(lo), 0x07060302u);
}
__device__ __forceinline__ float without_top(float x) { return x - __uint_as_float(__float_as_uint(x) & 0xffff0000u); }

__device__ __forceinline__ void floats_of(const V8<float>& x, float* y) {
  y[0] = x.a.x, y[1] = x.a.y, y[2] = x.a.z, y[3] = x.a.w, y[4] = x.b.x, y[5] = x.b.y, y[6] = x.b.z, y[7] = x.b.w;
}
__device__ __forceinline__ void floats_of(const V8<uint16_t>& x, float* y) {
  const uint32_t w[4] = {x.v.x, x.v.y, x.v.z, x.v.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    y[2 * i] = __uint_as_float(w[i] << 16);
    y[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
  }
}

// PARTS = 1: x rounded to bf16; 2: x within 2^-15; 3: x exactly
template <int PARTS>
__device__ __forceinline__ void split8(const float* x, uint4* out) {
  if constexpr (PARTS == 1) {
    out[0] = make_uint4(f2bf2(x[0], x[1]), f2bf2(x[2], x[3]), f2bf2(x[4], x[5]), f2bf2(x[6], x[7]));
  } else {
    float r[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) r[i] = x[i];
#pragma unroll
    for (int k = 0; k < PARTS; ++k) {
      out[k] = make_uint4(top_halves(r[0], r[1]), top_halves(r[2], r[3]), top_halves(r[4], r[5]), top_halves(r[6], r[7]));
#pragma unroll
      for (int i = 0; i < 8; ++i) r[i] = without_top(r[i]);
    }
  }
}

__device__ __forceinline__ f32x4_t mma16(const uint4& a, const uint4& b, f32x4_t c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, a), __builtin_bit_cast(bf16x8_t, b), c, 0, 0, 0);
}

// The running maximum follows the scores only where they leave it by more than
// this (in units of log2): weights stay below 2^8, and sums are rescaled rarely.
constexpr float kSlack = 8.0f;

// One step of the online softmax for a lane's 8 scores x (in units of log2, -inf
// where masked) of one query: p = 2^(x - m), and the factor for what was summed.
__device__ __forceinline__ float soft_step(const float* x, float& m, float& l, float* p) {
  float top = fmaxf(fmaxf(fmaxf(x[0], x[1]), fmaxf(x[2], x[3])), fmaxf(fmaxf(x[4], x[5]), fmaxf(x[6], x[7])));
  top = group4_max(top);
  const float m_new = top > m + kSlack ? top : m;
  const float sub = m_new == -INFINITY ? 0.0f : m_new;  // nothing yet: every p is 0
  const float alpha = m_new == m ? 1.0f : __builtin_amdgcn_exp2f(m - sub);
  float sum = 0.0f;
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    p[j] = __builtin_amdgcn_exp2f(x[j] - sub);
    sum += p[j];
  }
  l = fmaf(l, alpha, sum);
  m = m_new;
  return alpha;
}

// `bytes` of dynamic LDS for kernel F on the current device: where they may be more
// than 64 KB with what the kernel has itself, they are asked for once on each.
template <auto F>
hipError_t with_lds(int bytes) {
  static std::atomic<bool> done[kMaxDevices];
  if (bytes <= 60 * 1024) return hipSuccess;
  int dev = 0;
  hipError_t e = hipGetDevice(&dev);
  if (e != hipSuccess || (dev >= 0 && dev < kMaxDevices && done[dev])) return e;
  e = hipFuncSetAttribute(reinterpret_cast<const void*>(F), hipFuncAttributeMaxDynamicSharedMemorySize, bytes);
  if (e == hipSuccess && dev >= 0 && dev < kMaxDevices) done[dev] = true;
  return e;
}

template <class T>
__device__ __forceinline__ void store_out4(T* dst, const float* v) {
  if constexpr (sizeof(T) == 2) *(INCVIT_GLOBAL u32x2_t*)dst = u32x2_t{f2bf2(v[0], v[1]), f2bf2(v[2], v[3])};
  else *(INCVIT_GLOBAL f32x4_t*)dst = f32x4_t{v[0], v[1], v[2], v[3]};
}

// The lane, counted anew: nothing that holds it has to live through a loop.
__device__ __forceinline__ int lane_now() { return (int)__builtin_amdgcn_mbcnt_hi(~0u, __builtin_amdgcn_mbcnt_lo(~0u, 0u)); }

// LDS of the exchange between a workgroup's waves: m, l, then O
template <int DS, int NT>
constexpr int exchange_bytes() {
  return kKeyWaves * NT * 16 * (8 + 4 * (DS + 4));
}

// Joins the waves' partial results, which they have put into LDS (m, l
// [wave][row], O [wave][row][DS + 4]), and stores rows below `rows`: the result
// where the tile's keys are one workgroup's, else the partial result.
template <class T, int DS, int NT>
__device__ __forceinline__ void join_waves(const AttendArgs& a, const RowTile& w, const Share& sh, const char* lds, int h, int tid) {
  constexpr int TR = 16 * NT;
  const float* s_m = reinterpret_cast<const float*>(lds);
  const float* s_l = s_m + kKeyWaves * TR;
  const float* s_o = s_l + kKeyWaves * TR;
  const int rows = min(TR, w.q_len * a.group - w.first);
  float* part = a.parts + (size_t)(sh.slot * a.hk + h) * TR * (DS + 2);
  for (int i = tid; i < rows * (DS / 4); i += 64 * kKeyWaves) {
    const int r = i / (DS / 4), d = (i - r * (DS / 4)) * 4;
    float m = -INFINITY;
#pragma unroll
    for (int k = 0; k < kKeyWaves; ++k) m = fmaxf(m, s_m[k * TR + r]);
    float l = 0.0f;
    f32x4_t o = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int k = 0; k < kKeyWaves; ++k) {
      const float mk = s_m[k * TR + r];
      const float e = mk == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(mk - m);
      l += e * s_l[k * TR + r];
      o += *reinterpret_cast<const f32x4_t*>(s_o + (size_t)(k * TR + r) * (DS + 4) + d) * e;
    }
    if (sh.n > 1) {
      if (d == 0) *(INCVIT_GLOBAL u32x2_t*)(part + 2 * r) = u32x2_t{__float_as_uint(m), __float_as_uint(l)};
      *(INCVIT_GLOBAL f32x4_t*)(part + 2 * TR + r * DS + d) = o;
    } else if (d < a.d) {
      const int row = w.first + r, tok = row / a.group, head = h * a.group + row - tok * a.group;
      const float inv = 1.0f / l;
      float y[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) y[j] = m == -INFINITY ? 0.0f : o[j] * inv;
      store_out4<T>(static_cast<T*>(const_cast<void*>(a.out.p)) + (w.q0 + tok) * a.out.row + (long)head * a.out.head + d, y);
    }
  }
}

}  // namespace incvit
#endif
