// Keys and values written into a cache in 8 bits, and read back.
//
// Write: a wave for each group of 16 tokens of a block, one head, keys or values,
// takes the rows of the block that follow one another, padding aside.  They are put at
// their places (a map in LDS; of rows of one slot the last), loaded into registers
// together with what the group keeps, and the waves of a block join their largest
// magnitudes; then new rows are quantised, kept integers rounded anew where the scale
// has grown, and only what changes is written.  The launch has a block's waves for every row (those
// whose row goes on with a block end at once) or, from kFewItems and kManyItems on,
// for every 4 and 16 (32) rows, and they take the blocks that begin there in turn.
//
// Read: a wave has a row, a lane pieces of 8 dims of a head: 8 bytes of the keys and 32
// of the values (4 tokens together, of which it takes a byte of each dim).
//
// Both are bound by memory where rows are many: 8192 rows of 16 heads of 64 in bf16,
// written 15.6 us for 33.6 MB in and 16.8 MB out (counters: 33.7 and 16.5; 3.2 TB/s of
// a copy's 5.1), read 11.3 us for the same the other way (4.5 TB/s; 25.2 MB in, since
// 8 tokens' keys share a line and workgroups on two XCDs read it).  Few rows are a chain of
// latencies: slots, rows and what the block keeps, then the waves' exchange (one row
// of 4 heads of 128: 5.2 us in a graph, read 3.4).  A wave for 2, 4 or 8 rows of a
// read gained nothing, nor did 8 or 16 waves to a workgroup.
#include "attend.hpp"

namespace incvit {

namespace {

// rows * heads * 2.  A wave that finds nothing to do costs, and so does taking blocks
// in turn; measured, us, for 1, 4 and 16 (32) rows: 256 sequences' tokens (4096 items)
// 6.5, 12.1, 39.6; 1024 of 16 heads (32768) 37.7, 32.3, 50.0; 2728 scattered rows
// (87392) 22.5, 16.1, 14.1; a prompt of 8192 (262144) 61.2, 40.5, 14.6, in blocks of 32
// 16.7, of 64 18.5, of 128 186, 66.0, 25.6: of the workgroups there, which look for
// starts among 32 rows, three of four find none.  fp32, 8 heads of 128: 16.8 in blocks
// of 16 (84 MB), 27 of 64.
constexpr int64_t kFewItems = 8192, kManyItems = 32768;

__device__ __forceinline__ float kv_scale(float top) {
  return __builtin_isfinite(top) ? __fdiv_rn(top, 127.0f) : __uint_as_float(0x7fc00000u);
}

// x / s rounded to fp32, then to the nearest integer (ties to even), within 127, in
// the low byte.  For scales whose reciprocal and quotients stay normal without a
// division: inv = 1 / s correctly rounded, x * inv within 2 ulp of the quotient, a
// residual step makes it faithful, a second one correctly rounded (Markstein); the
// largest quotient rounds to 127.  Adding 1.5 * 2^23 leaves the integer in the low
// bits.  Otherwise a division, and 0 for a scale of 0 or NaN.
struct Quantiser {
  float s, inv;
  bool plain;
  __device__ __forceinline__ explicit Quantiser(float s_) : s(s_), inv(__fdiv_rn(1.0f, s_)), plain(s_ > 0x1p-90f && s_ < 0x1p90f) {}
  __device__ __forceinline__ uint32_t fast(float x) const {
    float q = x * inv;
    q = fmaf(fmaf(-q, s, x), inv, q);
    q = fmaf(fmaf(-q, s, x), inv, q);
    return __float_as_uint(q + 12582912.0f);
  }
  __device__ __forceinline__ uint32_t slow(float x) const {
    const float r = rintf(__fdiv_rn(x, s));
    return s > 0.0f ? (uint32_t)(int)fminf(fmaxf(r, -127.0f), 127.0f) : 0u;
  }
};
__device__ __forceinline__ uint32_t low_bytes(uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
  return __builtin_amdgcn_perm(__builtin_amdgcn_perm(d, c, 0x0c0c0400u), __builtin_amdgcn_perm(b, a, 0x0c0c0400u), 0x05040100u);
}
// four kept integers under a larger scale
__device__ __forceinline__ uint32_t kept_again(uint32_t w, float r) {
  uint32_t q[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) q[i] = (uint32_t)(int)rintf(__fmul_rn((float)(int8_t)(w >> (8 * i)), r));
  return low_bytes(q[0], q[1], q[2], q[3]);
}

// P consecutive values
template <class T, int P>
__device__ __forceinline__ void load_dims(const T* p, float* x) {
  if constexpr (P == 1) {
    x[0] = Elem<T>::f(*gbl(p));
  } else if constexpr (sizeof(T) == 4 && P == 4) {
    const f32x4_t v = *(const INCVIT_GLOBAL f32x4_t*)p;
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = v[i];
  } else if constexpr (sizeof(T) == 4) {
    const u32x2_t v = *(const INCVIT_GLOBAL u32x2_t*)p;
    x[0] = __uint_as_float(v[0]);
    x[1] = __uint_as_float(v[1]);
  } else if constexpr (P == 4) {
    const u32x2_t v = *(const INCVIT_GLOBAL u32x2_t*)p;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      x[2 * i] = __uint_as_float(v[i] << 16);
      x[2 * i + 1] = __uint_as_float(v[i] & 0xffff0000u);
    }
  } else {
    const uint32_t v = *(const INCVIT_GLOBAL uint32_t*)p;
    x[0] = __uint_as_float(v << 16);
    x[1] = __uint_as_float(v & 0xffff0000u);
  }
}

// A lane's part of a group of 16 tokens, in up to NPC pieces.  Keys: piece c is the
// 16 dims 16 (4 c + g) .. of token n.  Values: 4 tokens 4 g .. of P dims from 64 c + P
// n on, token by token (4 places each).
template <int NPC>
struct Group {
  float x[NPC][16];
  uint32_t old[NPC][4];
  int named;  // keys: whether token n is new; values: a bit for each of the 4 tokens
};

template <class T, int NPC>
__device__ __forceinline__ void load_group(Group<NPC>& q, const KvWriteArgs& a, const KvSide& x, const int* map, int grp, int h, int side,
                                           int np, int lane) {
  const int g = lane >> 4, n = lane & 15;
  const T* base = static_cast<const T*>(x.p) + (long)h * x.head;
  if (!side) {
    const int row = map[16 * grp + n];
    q.named = row >= 0;
    const T* src = base + (long)max(row, 0) * x.row;
#pragma unroll
    for (int c = 0; c < NPC; ++c)
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const int d = 16 * (4 * c + g) + 8 * e;
        const bool in = row >= 0 && d < a.d;
        V8<T> y;
        y.zero();
        if (in) y.load(src + d);
        floats_of(y, &q.x[c][8 * e]);
      }
    return;
  }
  int rows[4];
  q.named = 0;
#pragma unroll
  for (int t = 0; t < 4; ++t) {
    rows[t] = map[16 * grp + 4 * g + t];
    q.named |= rows[t] >= 0 ? 1 << t : 0;
  }
#pragma unroll
  for (int c = 0; c < NPC; ++c) {
    const int P = min(4, np - 4 * c);  // the same for the wave
    const int d = 64 * c + P * n;
#pragma unroll
    for (int t = 0; t < 4; ++t) {
      float* y = &q.x[c][4 * t];
      y[0] = y[1] = y[2] = y[3] = 0.0f;
      if (rows[t] < 0 || P < 1 || d >= a.d) continue;
      const T* src = base + (long)rows[t] * x.row + d;
      if (P == 4) load_dims<T, 4>(src, y);
      else if (P == 2) load_dims<T, 2>(src, y);
      else load_dims<T, 1>(src, y);
    }
  }
}

// What the block holds at the group's places.
template <int NPC>
__device__ __forceinline__ void load_old(Group<NPC>& q, const char* dst, int side, int np, int lane) {
  const int g = lane >> 4, n = lane & 15;
#pragma unroll
  for (int c = 0; c < NPC; ++c) {
    q.old[c][0] = q.old[c][1] = q.old[c][2] = q.old[c][3] = 0;
    const int P = min(4, np - 4 * c);
    if (!side ? 4 * c + g < np : P == 4) {
      const u32x4_t w = *(const INCVIT_GLOBAL u32x4_t*)(dst + 1024 * c + (side ? lane * 16 : g * 256 + n * 16));
#pragma unroll
      for (int i = 0; i < 4; ++i) q.old[c][i] = w[i];
    } else if (side && P == 2) {
      const u32x2_t w = *(const INCVIT_GLOBAL u32x2_t*)(dst + 1024 * c + lane * 8);
      q.old[c][0] = w[0];
      q.old[c][1] = w[1];
    } else if (side && P == 1) {
      q.old[c][0] = *(const INCVIT_GLOBAL uint32_t*)(dst + 1024 * c + lane * 4);
    }
  }
}

// anew: nothing is kept; r: what kept integers are multiplied by (1: they stay)
template <int NPC>
__device__ __forceinline__ void store_group(const Group<NPC>& q, const Quantiser& z, bool anew, float r, char* dst, int side, int np,
                                            int lane) {
  const int g = lane >> 4, n = lane & 15;
  if (!q.named && !anew && r == 1.0f) return;
#pragma unroll
  for (int c = 0; c < NPC; ++c) {
    uint32_t b[16], out[4];
    if (z.plain) {
#pragma unroll
      for (int i = 0; i < 16; ++i) b[i] = z.fast(q.x[c][i]);
    } else {
#pragma unroll
      for (int i = 0; i < 16; ++i) b[i] = z.slow(q.x[c][i]);
    }
    const int P = min(4, np - 4 * c);
    if (!side) {
      if (4 * c + g >= np) continue;
#pragma unroll
      for (int i = 0; i < 4; ++i) out[i] = low_bytes(b[4 * i], b[4 * i + 1], b[4 * i + 2], b[4 * i + 3]);
      if (!q.named) {
#pragma unroll
        for (int i = 0; i < 4; ++i) out[i] = anew ? 0u : kept_again(q.old[c][i], r);
      }
      *(INCVIT_GLOBAL u32x4_t*)(dst + 1024 * c + g * 256 + n * 16) = u32x4_t{out[0], out[1], out[2], out[3]};
      continue;
    }
    uint32_t take = 0;  // bytes of new tokens
#pragma unroll
    for (int t = 0; t < 4; ++t) take |= q.named >> t & 1 ? 0xffu << (8 * t) : 0u;
#pragma unroll
    for (int p = 0; p < 4; ++p) {
      const uint32_t fresh = low_bytes(b[p], b[4 + p], b[8 + p], b[12 + p]);
      const uint32_t kept = anew ? 0u : r == 1.0f ? q.old[c][p] : kept_again(q.old[c][p], r);
      out[p] = (fresh & take) | (kept & ~take);
    }
    if (P == 4) *(INCVIT_GLOBAL u32x4_t*)(dst + 1024 * c + lane * 16) = u32x4_t{out[0], out[1], out[2], out[3]};
    else if (P == 2) *(INCVIT_GLOBAL u32x2_t*)(dst + 1024 * c + lane * 8) = u32x2_t{out[0], out[1]};
    else if (P == 1) *(INCVIT_GLOBAL uint32_t*)(dst + 1024 * c + lane * 4) = out[0];
  }
}

// W waves, one for each group of the block: `wave` is the group.
template <int W>
__device__ __forceinline__ void block_sync() {
  if constexpr (W > 1) __syncthreads();
  else __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
}

// Slots of the 64 rows from `base` on; -1 past the call's.  (Rows have 24 bits.)
__device__ __forceinline__ int slots_of(const KvWriteArgs& a, int base, int lane) {
  const int r = base + lane, rows = (int)a.rows, s = gbl(a.slots)[(uint32_t)min(max(r, 0), rows - 1)];
  return (uint32_t)r < (uint32_t)rows ? s : -1;
}
__device__ __forceinline__ bool in_pool(const KvWriteArgs& a, int slot) { return (uint32_t)slot < (uint32_t)(a.blocks * a.block); }

// Padding is passed over 256 rows at a time, whose slots are on the way together:
// the slots of the next 64 rows (from base + 64 on) or those before (from base - 64)
// that are not padding alone, and `base` is where they are; false if none.
template <int STEP>
__device__ __forceinline__ bool pass_padding(const KvWriteArgs& a, int& base, int& slot, int lane) {
  constexpr int N = 4;
  while (true) {
    int s[N];
#pragma unroll
    for (int k = 0; k < N; ++k) s[k] = slots_of(a, base + STEP * (k + 1), lane);
#pragma unroll
    for (int k = 0; k < N; ++k) {
      base += STEP;
      slot = s[k];
      if (__ballot(in_pool(a, slot))) return true;
      if (STEP > 0 ? base >= (int)a.rows : base <= 0) return false;
    }
  }
}

// The block of a slot; -1 for padding.
template <int W>
__device__ __forceinline__ int block_of(const KvWriteArgs& a, int slot) {
  return in_pool(a, slot) ? slot / (16 * W) : -1;
}

// The run that begins with row base + first, up to the next row of another block
// (padding does not end it); the lanes have the slots of the rows from base on.
template <class T, int NPC, int W>
__device__ __forceinline__ void write_block(const KvWriteArgs& a, int* map, uint32_t* tops, int base, int first, int slot, int blk, int h,
                                            int side, int lane, int wave) {
  constexpr int B = 16 * W;
  if (lane < 16) map[16 * wave + lane] = -1;
  block_sync<W>();
  if (wave == 0) {
    while (true) {
      const int mine = block_of<W>(a, slot);
      const uint64_t other = __ballot(mine >= 0 && mine != blk) & (~0ull << first);
      const int end = other ? __builtin_ctzll(other) : 64;
      if (mine == blk && lane >= first && lane < end) atomicMax(&map[slot % B], base + lane);
      if (other || base + 64 >= (int)a.rows || !pass_padding<64>(a, base, slot, lane)) break;
      first = 0;
    }
  }
  block_sync<W>();
  int named = 0;
#pragma unroll
  for (int t = 0; t < B; t += 64) named += __popcll(__ballot(t + lane < B && map[min(t + lane, B - 1)] >= 0));
  const bool anew = named == B || (a.begin && map[0] >= 0);

  const KvLayout lay(a.blocks, B, a.heads, a.d);
  const KvSide x = side ? a.x[1] : a.x[0];
  const int np = lay.ds / 16;
  float* scale = reinterpret_cast<float*>(a.cache) + ((long)blk * a.heads + h) * 2 + side;
  char* dst = a.cache + a.data + ((size_t)blk * a.heads + h) * lay.head_bytes + (side ? (size_t)B * lay.ds : 0) + (size_t)wave * (16 * lay.ds);
  float before = *gbl(scale);
  Group<NPC> q;
  const bool here = W == 1 || __any(map[16 * wave + (lane & 15)] >= 0);  // new rows in the wave's group
  uint32_t top = 0;  // the largest magnitude as bits, which order like it, NaN on top
  if (here) {
    if (!anew) load_old(q, dst, side, np, lane);
    load_group<T>(q, a, x, map, wave, h, side, np, lane);
#pragma unroll
    for (int c = 0; c < NPC; ++c)
#pragma unroll
      for (int i = 0; i < 16; ++i) top = max(top, __float_as_uint(q.x[c][i]) & 0x7fffffffu);
    top = lanes_max<64>(top);
  }
  if constexpr (W > 1) {
    if (lane == 0) tops[wave] = top;
    asm volatile("" : "+v"(before));  // every wave has the old scale before one writes the new
    __syncthreads();
#pragma unroll
    for (int k = 0; k < W; ++k) top = max(top, tops[k]);
  }
  const float old = anew ? 0.0f : before, fresh = kv_scale(__uint_as_float(top));
  const float s = old >= fresh ? old : fresh > old ? fresh : __uint_as_float(0x7fc00000u);  // either NaN: NaN
  const float r = !(s > 0.0f) ? 0.0f : s == old ? 1.0f : __fdiv_rn(old, s);
  if (lane == 0 && wave == 0) *gbl(scale) = s;
  if (!here) {
    if (!anew && r == 1.0f) return;
    q.named = 0;
#pragma unroll
    for (int c = 0; c < NPC; ++c)
#pragma unroll
      for (int i = 0; i < 16; ++i) q.x[c][i] = 0.0f;
    if (!anew) load_old(q, dst, side, np, lane);
  }
  store_group(q, Quantiser(s), anew, r, dst, side, np, lane);
}

template <class T, int NPC, int W>
__global__ __launch_bounds__(W == 1 ? 256 : 64 * W) void kv_write_kernel(KvWriteArgs a) {
  __shared__ int s_map[W == 1 ? 64 : 16 * W];
  __shared__ uint32_t s_top[W];
  const int lane = threadIdx.x & 63, tw = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), wave = W == 1 ? 0 : tw;
  // a row's heads and sides one after another
  const uint32_t item = W == 1 ? blockIdx.x * 4 + tw : blockIdx.x, sides = 2 * a.heads;
  const int r0 = (int)(item / sides) * a.each;
  if (r0 >= a.rows) return;
  const int rest = item % sides, side = rest & 1, h = rest >> 1;
  // rows that begin a run of their block: the row before, padding aside, is another's;
  // the first lane has the row before the item's
  const int slot = slots_of(a, r0 - 1, lane), blk = block_of<W>(a, slot);
  int prev = __shfl_up(blk, 1);
  const uint64_t there = __ballot(blk >= 0);
  if (__builtin_expect((~there & ((2ull << a.each) - (r0 ? 1 : 2))) != 0, 0)) {  // padding, or the call's last rows
    const uint64_t below = there & ((1ull << lane) - 1);
    prev = __shfl(blk, below ? 63 - __builtin_clzll(below) : 0);
    if (!(there & 1) && (there & ((2ull << a.each) - 1))) {  // rows that have only padding before them here
      int base = r0 - 1, s = -1;
      const bool found = base > 0 && pass_padding<-64>(a, base, s, lane);
      const uint64_t last = __ballot(in_pool(a, s));
      const int back = found ? __builtin_amdgcn_readlane(block_of<W>(a, s), 63 - __builtin_clzll(last)) : -1;
      if (!below) prev = back;
    }
  }
  uint64_t lead = __ballot(lane > 0 && lane <= a.each && blk >= 0 && blk != prev);
  while (lead) {
    const int i = __builtin_ctzll(lead);
    lead &= lead - 1;
    write_block<T, NPC, W>(a, s_map + (W == 1 ? 16 * tw : 0), s_top, r0 - 1, i, slot, __builtin_amdgcn_readlane(blk, i), h, side, lane, wave);
    if constexpr (W > 1) __syncthreads();  // the map and the maxima are free again
  }
}

template <class T>
__global__ __launch_bounds__(256) void kv_read_kernel(KvReadArgs a) {
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const long r = (long)blockIdx.x * 4 + wave;
  if (r >= a.rows) return;
  const int slot = __builtin_amdgcn_readfirstlane(gbl(a.slots)[r]);
  const bool there = slot >= 0 && slot < (long)a.blocks * a.block;
  if (!there && !a.fill) return;
  const int blk = there ? slot / a.block : 0, tok = there ? slot - blk * a.block : 0, n = tok & 15;
  const KvLayout lay(a.blocks, a.block, a.heads, a.d);
  const char* base = a.cache + a.data + (size_t)blk * a.heads * lay.head_bytes + (size_t)(tok >> 4) * (16 * lay.ds);
  const float* scales = reinterpret_cast<const float*>(a.cache) + (long)blk * a.heads * 2;
  T* ko = static_cast<T*>(const_cast<void*>(a.x[0].p)) + r * a.x[0].row;
  T* vo = static_cast<T*>(const_cast<void*>(a.x[1].p)) + r * a.x[1].row;
  const int per = a.d / 8, units = a.heads * per;
#pragma unroll 2
  for (int u = lane; u < units; u += 64) {
    const int h = per == 1 ? u : (int)__umulhi((uint32_t)u, a.per_inv), d = (u - h * per) * 8;  // u / per: u < 2^15
    const char* at = base + (size_t)h * lay.head_bytes;
    const u32x2_t k = *(const INCVIT_GLOBAL u32x2_t*)(at + (d >> 4) * 256 + n * 16 + (d & 15));
    const int chunk = d >> 6, wide = min(64, lay.ds - 64 * chunk);
    const char* vp = at + (size_t)a.block * lay.ds + chunk * 1024 + (n >> 2) * 4 * wide + 4 * (d & 63);
    const u32x4_t v0 = *(const INCVIT_GLOBAL u32x4_t*)vp, v1 = *(const INCVIT_GLOBAL u32x4_t*)(vp + 16);
    const u32x2_t sc = *(const INCVIT_GLOBAL u32x2_t*)(scales + 2 * h);
    const float ks = __uint_as_float(sc[0]), vs = __uint_as_float(sc[1]);
    float y[8], z[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      y[i] = there ? (float)(int8_t)(k[i >> 2] >> (8 * (i & 3))) * ks : 0.0f;
      z[i] = there ? (float)(int8_t)((i < 4 ? v0[i & 3] : v1[i & 3]) >> (8 * (n & 3))) * vs : 0.0f;
    }
    T* kd = ko + (long)h * a.x[0].head + d;
    T* vd = vo + (long)h * a.x[1].head + d;
    if constexpr (sizeof(T) == 2) {
      *(INCVIT_GLOBAL u32x4_t*)kd = u32x4_t{f2bf2(y[0], y[1]), f2bf2(y[2], y[3]), f2bf2(y[4], y[5]), f2bf2(y[6], y[7])};
      *(INCVIT_GLOBAL u32x4_t*)vd = u32x4_t{f2bf2(z[0], z[1]), f2bf2(z[2], z[3]), f2bf2(z[4], z[5]), f2bf2(z[6], z[7])};
    } else {
      store_out4<T>(kd, y);
      store_out4<T>(kd + 4, y + 4);
      store_out4<T>(vd, z);
      store_out4<T>(vd + 4, z + 4);
    }
  }
}

template <class T, int NPC>
hipError_t launch_write_np(const KvWriteArgs& a, unsigned items, hipStream_t s) {
  if (a.block == 16) return launch_k(kv_write_kernel<T, NPC, 1>, dim3((items + 3) / 4), dim3(256), 0, s, a);
  if (a.block == 32) return launch_k(kv_write_kernel<T, NPC, 2>, dim3(items), dim3(128), 0, s, a);
  if (a.block == 64) return launch_k(kv_write_kernel<T, NPC, 4>, dim3(items), dim3(256), 0, s, a);
  return launch_k(kv_write_kernel<T, NPC, 8>, dim3(items), dim3(512), 0, s, a);
}
template <class T>
hipError_t launch_write_t(const KvWriteArgs& a, unsigned items, hipStream_t s) {
  const int np = kv_dims(a.d) / 16;
  if (np <= 4) return launch_write_np<T, 1>(a, items, s);
  if (np <= 8) return launch_write_np<T, 2>(a, items, s);
  return launch_write_np<T, 4>(a, items, s);
}

}  // namespace

hipError_t launch_kv_write(const KvWriteArgs& a0, hipStream_t s) {
  KvWriteArgs a = a0;
  const int64_t items = (int64_t)a.rows * 2 * a.heads;
  a.each = items <= kFewItems ? 1 : items <= kManyItems ? 4 : a.block == 16 ? 16 : 32;
  const unsigned n = (unsigned)((a.rows + a.each - 1) / a.each * 2 * a.heads);
  return a.dtype == INCVIT_BF16 ? launch_write_t<uint16_t>(a, n, s) : launch_write_t<float>(a, n, s);
}

hipError_t launch_kv_read(const KvReadArgs& a0, hipStream_t s) {
  KvReadArgs a = a0;
  const int per = a.d / 8;
  a.per_inv = 0xffffffffu / per + 1u;
  const dim3 grid((unsigned)((a.rows + 3) / 4));
  return a.dtype == INCVIT_BF16 ? launch_k(kv_read_kernel<uint16_t>, grid, dim3(256), 0, s, a)
                                : launch_k(kv_read_kernel<float>, grid, dim3(256), 0, s, a);
}

}  // namespace incvit
