// Keys and values written into a cache in 8 bits, and read back.
//
// Write: one wave for the rows of a block, of one head, keys or values.  Of the
// launch's waves (one for each row, head and side) those whose row begins a run of
// rows of one block work, the others end at once.  A wave puts the run's rows at
// their places (a map in LDS; of rows of one slot the last), finds their largest
// magnitude, and goes through the block's groups of 16 tokens: new rows are
// quantised, kept integers are rounded anew where the scale has grown, and only
// what changes is written.  Bound by the latency of three dependent loads (slots,
// rows and scale, kept integers) for a few rows, and by memory for many.
//
// Read: a thread has 4 dims of a row and head: 4 bytes of the keys and 16 of the
// values (4 tokens together, of which it takes a byte of each dim).
#include "attend.hpp"

namespace incvit {

namespace {

constexpr int kMaxBlock = 128;

__device__ __forceinline__ float kv_scale(float top) {
  return __builtin_isfinite(top) ? __fdiv_rn(top, 127.0f) : __uint_as_float(0x7fc00000u);
}
// x / s rounded to fp32, then to the nearest integer, within 127; 0 for a scale of 0 or NaN
__device__ __forceinline__ uint32_t kv_int(float x, float s) {
  const float r = rintf(__fdiv_rn(x, s));
  return s > 0.0f ? (uint32_t)(int)fminf(fmaxf(r, -127.0f), 127.0f) & 0xffu : 0u;
}
// a kept integer (byte i of w) under a larger scale
__device__ __forceinline__ uint32_t kv_again(uint32_t w, int i, float r) {
  return (uint32_t)(int)rintf(__fmul_rn((float)(int8_t)(w >> (8 * i)), r)) & 0xffu;
}

template <class T, int P>
__device__ __forceinline__ void load_dims(const T* p, float* x) {
  if constexpr (P == 1) {
    x[0] = Elem<T>::f(*gbl(p));
  } else if constexpr (sizeof(T) == 4) {
#pragma unroll
    for (int i = 0; i < P; i += 2) {
      const u32x2_t v = *(const INCVIT_GLOBAL u32x2_t*)(p + i);
      x[i] = __uint_as_float(v[0]);
      x[i + 1] = __uint_as_float(v[1]);
    }
  } else {
#pragma unroll
    for (int i = 0; i < P; i += 2) {
      const uint32_t v = *(const INCVIT_GLOBAL uint32_t*)(p + i);
      x[i] = __uint_as_float(v << 16);
      x[i + 1] = __uint_as_float(v & 0xffff0000u);
    }
  }
}

// What a wave knows of its block.
struct BlockJob {
  const int* map;  // LDS: row of a token, or -1
  bool anew;       // nothing is kept
  float s, r;      // the scale; what kept integers are multiplied by (1: unchanged)
};

// Values of a chunk of 16 P dims from dim d0 on, for the tokens 4 g .. 4 g + 3 of group `grp`.
template <class T, int P>
__device__ __forceinline__ void write_values(const BlockJob& j, const KvSide& x, int grp, int h, int d0, int d, char* dst, int lane) {
  const int g = lane >> 4, m = lane & 15, dim = d0 + P * m;
  int rows[4];
  int named = 0;
#pragma unroll
  for (int t = 0; t < 4; ++t) {
    rows[t] = j.map[16 * grp + 4 * g + t];
    named |= (rows[t] >= 0 ? 1 : 0) << t;
  }
  if (!named && !j.anew && j.r == 1.0f) return;
  char* at = dst + lane * 4 * P;
  float v[4][P];
#pragma unroll
  for (int t = 0; t < 4; ++t) {
#pragma unroll
    for (int p = 0; p < P; ++p) v[t][p] = 0.0f;
    if (rows[t] >= 0 && dim < d)
      load_dims<T, P>(static_cast<const T*>(x.p) + (long)rows[t] * x.row + (long)h * x.head + dim, v[t]);
  }
#pragma unroll
  for (int p = 0; p < P; ++p) {
    uint32_t out = 0;
    if (named != 15 && !j.anew) {
      const uint32_t old = *(const INCVIT_GLOBAL uint32_t*)(at + 4 * p);
#pragma unroll
      for (int t = 0; t < 4; ++t) out |= (j.r == 1.0f ? old >> (8 * t) & 0xffu : kv_again(old, t, j.r)) << (8 * t);
    }
#pragma unroll
    for (int t = 0; t < 4; ++t)
      if (named >> t & 1) out = (out & ~(0xffu << (8 * t))) | kv_int(v[t][p], j.s) << (8 * t);
    *(INCVIT_GLOBAL uint32_t*)(at + 4 * p) = out;
  }
}

template <class T>
__global__ __launch_bounds__(256) void kv_write_kernel(KvWriteArgs a) {
  __shared__ int s_map[4][kMaxBlock];
  const int lane = threadIdx.x & 63, g = lane >> 4, n = lane & 15;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  // a row's heads and sides one after another
  const long item = (long)blockIdx.x * 4 + wave;
  const int each = 2 * a.heads;
  const long r0 = item / each;
  if (r0 >= a.rows) return;
  const int side = (int)(item - r0 * each) & 1, h = (int)(item - r0 * each) >> 1;
  const long pool = (long)a.blocks * a.block;
  const int slot = gbl(a.slots)[r0], blk = slot / a.block;
  if (slot < 0 || slot >= pool) return;
  if (r0 > 0) {
    const int before = gbl(a.slots)[r0 - 1];
    if (before >= 0 && before < pool && before / a.block == blk) return;
  }
  int* map = s_map[wave];
  for (int t = lane; t < a.block; t += 64) map[t] = -1;
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  // the run: rows of the block from r0 on; r0 + (row of the map) is below 2^31
  for (long r = r0;; r += 64) {
    const int sl = r + lane < a.rows ? gbl(a.slots)[r + lane] : -1;
    const uint64_t in = __ballot(sl >= 0 && sl < pool && sl / a.block == blk);
    const int run = in == ~0ull ? 64 : __builtin_ctzll(~in);
    if (lane < run) atomicMax(&map[sl - blk * a.block], (int)(r + lane));
    if (run < 64) break;
  }
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  int named = 0;
  for (int t = 0; t < a.block; t += 64) named += __popcll(__ballot(t + lane < a.block && map[min(t + lane, a.block - 1)] >= 0));
  BlockJob j;
  j.map = map;
  j.anew = named == a.block || (a.begin && map[0] >= 0);

  const KvLayout lay(a.blocks, a.block, a.heads, a.d);
  const KvSide x = side ? a.x[1] : a.x[0];
  float* scale = reinterpret_cast<float*>(a.cache) + ((long)blk * a.heads + h) * 2 + side;
  const float old = j.anew ? 0.0f : *gbl(scale);
  // the largest magnitude, as bits, which order like it and put NaN on top
  uint32_t top = 0;
  for (int grp = 0; grp < a.block / 16; ++grp) {
    const int row = map[16 * grp + n];
    if (row < 0) continue;
    const T* src = static_cast<const T*>(x.p) + (long)row * x.row + (long)h * x.head;
    for (int d = 8 * g; d < a.d; d += 32) {
      V8<T> v;
      v.load(src + d);
      if constexpr (sizeof(T) == 2) {
        const uint32_t q[4] = {v.v.x, v.v.y, v.v.z, v.v.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) top = max(top, max(q[i] << 16 & 0x7fffffffu, q[i] & 0x7fff0000u));
      } else {
        const float q[8] = {v.a.x, v.a.y, v.a.z, v.a.w, v.b.x, v.b.y, v.b.z, v.b.w};
#pragma unroll
        for (int i = 0; i < 8; ++i) top = max(top, __float_as_uint(q[i]) & 0x7fffffffu);
      }
    }
  }
  top = lanes_max<64>(top);
  const float fresh = kv_scale(__uint_as_float(top));
  j.s = old >= fresh ? old : fresh > old ? fresh : __uint_as_float(0x7fc00000u);  // either NaN: NaN
  j.r = j.s == old ? 1.0f : j.s > 0.0f ? __fdiv_rn(old, j.s) : 0.0f;
  if (!(j.s > 0.0f)) j.r = 0.0f;
  if (lane == 0) *gbl(scale) = j.s;

  char* dst = a.cache + a.data + ((size_t)blk * a.heads + h) * lay.head_bytes + (side ? (size_t)a.block * lay.ds : 0);
  const int ds = lay.ds, np = ds / 16;
  for (int grp = 0; grp < a.block / 16; ++grp, dst += 16 * ds) {
    if (side) {
      for (int c = 0; c < np / 4; ++c) write_values<T, 4>(j, x, grp, h, 64 * c, a.d, dst + 1024 * c, lane);
      if (np % 4 == 1) write_values<T, 1>(j, x, grp, h, 64 * (np / 4), a.d, dst + 1024 * (np / 4), lane);
      if (np % 4 == 2) write_values<T, 2>(j, x, grp, h, 64 * (np / 4), a.d, dst + 1024 * (np / 4), lane);
      continue;
    }
    const int row = map[16 * grp + n];
    for (int p = g; p < np; p += 4) {  // 16 dims of token n
      char* at = dst + p * 256 + n * 16;
      uint32_t out[4] = {0, 0, 0, 0};
      if (row >= 0) {
        const T* src = static_cast<const T*>(x.p) + (long)row * x.row + (long)h * x.head;
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const int d = 16 * p + 8 * e;
          if (d >= a.d) continue;
          V8<T> y;
          y.load(src + d);
          float v[8];
          floats_of(y, v);
#pragma unroll
          for (int i = 0; i < 8; ++i) out[2 * e + (i >> 2)] |= kv_int(v[i], j.s) << (8 * (i & 3));
        }
      } else if (!j.anew) {
        if (j.r == 1.0f) continue;
        const u32x4_t w = *(const INCVIT_GLOBAL u32x4_t*)at;
#pragma unroll
        for (int i = 0; i < 16; ++i) out[i >> 2] |= kv_again(w[i >> 2], i & 3, j.r) << (8 * (i & 3));
      }
      *(INCVIT_GLOBAL u32x4_t*)at = u32x4_t{out[0], out[1], out[2], out[3]};
    }
  }
}

template <class T>
__global__ __launch_bounds__(256) void kv_read_kernel(KvReadArgs a) {
  const int quads = a.d / 4, each = a.heads * quads;
  const long at = (long)blockIdx.x * 256 + threadIdx.x;
  const long r = at / each;
  if (r >= a.rows) return;
  const int rest = (int)(at - r * each), h = rest / quads, d = (rest - h * quads) * 4;
  const int slot = gbl(a.slots)[r];
  if (slot < 0 || slot >= (long)a.blocks * a.block) return;
  const int blk = slot / a.block, tok = slot - blk * a.block, n = tok & 15;
  const KvLayout lay(a.blocks, a.block, a.heads, a.d);
  const char* base = a.cache + a.data + ((size_t)blk * a.heads + h) * lay.head_bytes + (size_t)(tok >> 4) * (16 * lay.ds);
  const float* s = reinterpret_cast<const float*>(a.cache) + ((long)blk * a.heads + h) * 2;
  const uint32_t k = *(const INCVIT_GLOBAL uint32_t*)(base + (d >> 4) * 256 + n * 16 + (d & 15));
  const int chunk = d >> 6, wide = min(64, lay.ds - 64 * chunk);
  const u32x4_t v = *(const INCVIT_GLOBAL u32x4_t*)(base + (size_t)a.block * lay.ds + chunk * 1024 + (n >> 2) * 4 * wide + 4 * (d & 63));
  const float ks = gbl(s)[0], vs = gbl(s)[1];
  float y[4], z[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    y[i] = (float)(int8_t)(k >> (8 * i)) * ks;
    z[i] = (float)(int8_t)(v[i] >> (8 * (n & 3))) * vs;
  }
  T* ko = static_cast<T*>(const_cast<void*>(a.x[0].p)) + r * a.x[0].row + (long)h * a.x[0].head + d;
  T* vo = static_cast<T*>(const_cast<void*>(a.x[1].p)) + r * a.x[1].row + (long)h * a.x[1].head + d;
  store_out4<T>(ko, y);
  store_out4<T>(vo, z);
}

}  // namespace

hipError_t launch_kv_write(const KvWriteArgs& a, hipStream_t s) {
  const dim3 grid((unsigned)((a.rows * 2 * a.heads + 3) / 4));
  return a.dtype == INCVIT_BF16 ? launch_k(kv_write_kernel<uint16_t>, grid, dim3(256), 0, s, a)
                                : launch_k(kv_write_kernel<float>, grid, dim3(256), 0, s, a);
}

hipError_t launch_kv_read(const KvReadArgs& a, hipStream_t s) {
  const dim3 grid((unsigned)((a.rows * a.heads * (a.d / 4) + 255) / 256));
  return a.dtype == INCVIT_BF16 ? launch_k(kv_read_kernel<uint16_t>, grid, dim3(256), 0, s, a)
                                : launch_k(kv_read_kernel<float>, grid, dim3(256), 0, s, a);
}

}  // namespace incvit
