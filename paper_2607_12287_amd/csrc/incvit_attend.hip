// C ABI of the cache in 8 bits and of the attention operators: argument checks,
// the split of the work, launches.
#include <algorithm>
#include <cmath>

#include "attend.hpp"

using namespace incvit;

namespace {

// Workgroups of a call that shares keys, where waves have keys and where they have
// rows, and the key tiles of one at least.  32 sequences over 152 k keys, heads of 128
// (cached): 39, 38, 37, 35 us with 512, 768, 1024, 1536.
constexpr long kWant = 1536, kWantRows = 512, kLeast = 16, kLeastRows = 8;

// Rows times query heads of a call, up to which waves share keys for longer sequences
// (a workgroup of waves with rows takes four times the rows, and so leaves the chip
// idle sooner).  Measured, us, heads of 64 in groups of 4, waves with keys | rows.
// 8192 keys of one sequence, 4 key heads, 16 rows: 15 | 26 cached, 15 | 19 plain; 32
// rows: 16 | 27, 18 | 24; 64 rows: 21 | 29, 27 | 26.  16 sequences of 2048 keys, 4, 8,
// 16, 24 rows: cached 15 | 24, 19 | 25, 26 | 27, 35 | 29; plain 21 | 20, 31 | 21,
// 28 | 25, 29 | 28.
constexpr long kFewRows = 1024;

// Rows times query heads, up to which a wave has one tile of 16 rows and not two, so
// that there are more workgroups: twice as many up to 128 dims, where two fit a CU's
// LDS.  Only for sequences of enough rows, which do not wait for memory, and whose
// keys are not shared anyway.  Measured, 16 heads in groups of 4, one tile | two, us, a
// prompt that sees everything, then with a window of 512:
//   1024 rows, heads of 64: 18 | 25, 13 | 18; 128: 29 | 35, 19 | 24; 256: 48 | 69, 31 | 45;
//   2048 rows,          64: 34 | 45, 16 | 18; 128: 57 | 63, 23 | 25; 256: 99 | 129, 60 | 49;
//   4096 rows,          64: 72 | 91, 24 | 23; 128: 126 | 130, 44 | 32; 256: 358 | 270, 121 | 96.
// Rows alone decide: where a window turns the order (2048 rows of 256, 4096 of 64), two.
// 64 sequences of 24 rows and 1024 keys, 128: 74 | 46; 512 rows, 8192 keys: 76 | 59.
constexpr long kOneTileRows = 16384, kOneTileEach = 256;

constexpr int64_t kMostStride = (int64_t)1 << 40;
constexpr float kLog2e = 1.44269504088896340736f;

bool is_dtype(int32_t t) { return t == INCVIT_F32 || t == INCVIT_BF16; }

incvit_status launched(hipError_t e, const char* what) {
  if (e == hipSuccess) return INCVIT_OK;
  char buf[160];
  snprintf(buf, sizeof buf, "%s: %s", what, hipGetErrorString(e));
  return op_fail(INCVIT_ERR_HIP, buf);
}

bool dims_ok(int32_t d) { return d >= 8 && d <= 256 && d % 8 == 0; }

bool kv_ok(const incvit_kv& c) {
  return (c.block == 16 || c.block == 32 || c.block == 64 || c.block == 128) && c.blocks >= 1 && c.heads >= 1 && c.heads <= 1024 &&
         dims_ok(c.head_dim) && (int64_t)c.blocks * c.block < ((int64_t)1 << 31);
}

// Whether rows x heads runs of d elements at r * row + h * head never overlap.
bool apart(int64_t rows, int64_t row, int64_t heads, int64_t head, int64_t d) {
  if (rows <= 1) return heads <= 1 || head >= d;
  if (heads <= 1) return row >= d;
  const int64_t lo = std::min(row, head), hi = std::max(row, head), n = row < head ? rows : heads;
  return lo >= d && n - 1 <= (hi - d) / lo;
}

incvit_status check_rows(int32_t dtype, const void* p, int64_t row, int64_t head, const char* what) {
  const int64_t per = dtype == INCVIT_BF16 ? 8 : 4;
  char buf[96];
  if (!p) snprintf(buf, sizeof buf, "%s: null", what);
  else if ((uintptr_t)p % 16 || row % per || head % per) snprintf(buf, sizeof buf, "%s: rows and heads must be 16-byte aligned", what);
  else if (row < 0 || head < 0 || row > kMostStride || head > kMostStride)
    snprintf(buf, sizeof buf, "%s: strides must be in [0, 2^40] elements", what);
  else return INCVIT_OK;
  return op_fail(INCVIT_ERR_ARG, buf);
}

incvit_status check_kv(const incvit_kv* c, int32_t dtype, int64_t rows, const void* cache, const int32_t* slots) {
  if (!c || !kv_ok(*c)) return op_fail(c ? INCVIT_ERR_UNSUPPORTED : INCVIT_ERR_ARG, "cache out of range (blocks, block, heads or head_dim)");
  if (!is_dtype(dtype)) return op_fail(INCVIT_ERR_UNSUPPORTED, "dtype must be INCVIT_F32 or INCVIT_BF16");
  // a launch counts its threads in 32 bits
  if (rows < 0 || rows > ((int64_t)1 << 24) / c->heads) return op_fail(INCVIT_ERR_ARG, "rows must be >= 0 and rows * heads <= 2^24");
  if (rows == 0) return INCVIT_OK;
  if (!cache || (uintptr_t)cache % 256) return op_fail(INCVIT_ERR_ARG, "the cache must be non-null and 256-byte aligned");
  if (!slots || (uintptr_t)slots % 4) return op_fail(INCVIT_ERR_ARG, "slots must be non-null and 4-byte aligned");
  return INCVIT_OK;
}

bool attention_ok(const incvit_attention& a) {
  return is_dtype(a.dtype) && dims_ok(a.head_dim) && a.q_heads >= 1 && a.q_heads <= 1024 && a.kv_heads >= 1 &&
         a.q_heads % a.kv_heads == 0 && (a.causal == 0 || a.causal == 1) && (a.fill == 0 || a.fill == 1) && a.window >= 0 && a.window <= (1 << 30) && a.sinks >= 0 &&
         a.sinks <= (1 << 30) && a.scale > 0.0f && std::isfinite(a.scale * kLog2e);
}

incvit_status check_attention(const incvit_attention* a, int32_t n, int64_t rows) {
  if (!a) return op_fail(INCVIT_ERR_ARG, "null configuration");
  if (!is_dtype(a->dtype)) return op_fail(INCVIT_ERR_UNSUPPORTED, "dtype must be INCVIT_F32 or INCVIT_BF16");
  if (!dims_ok(a->head_dim)) return op_fail(INCVIT_ERR_UNSUPPORTED, "head_dim must be a multiple of 8 in [8, 256]");
  if (!attention_ok(*a))
    return op_fail(INCVIT_ERR_ARG, "attention out of range (heads, causal, window, sinks, fill or scale)");
  if (n < 0 || rows < 0 || n > (1 << 24)) return op_fail(INCVIT_ERR_ARG, "n must be in [0, 2^24] and rows >= 0");
  if (rows > ((int64_t)1 << 30) / (a->q_heads / a->kv_heads) - 1)
    return op_fail(INCVIT_ERR_ARG, "rows * (q_heads / kv_heads) must be < 2^30");
  return INCVIT_OK;
}

incvit_status check_plan(const incvit_attention& a, const AttendPlan& p, const void* workspace) {
  if (p.shares * a.kv_heads >= (1 << 24)) return op_fail(INCVIT_ERR_UNSUPPORTED, "too many rows and sequences for one launch");
  if (p.bytes && (!workspace || (uintptr_t)workspace % 256))
    return op_fail(INCVIT_ERR_ARG, "the workspace must be non-null and 256-byte aligned");
  return INCVIT_OK;
}

AttendArgs attend_args(const incvit_attention& a, const AttendPlan& p, int32_t n, int64_t rows, const int32_t* q_start,
                       const incvit_rows* q, const incvit_rows* out, void* workspace) {
  AttendArgs r = {};
  r.q_start = q_start;
  r.q = KvSide{q->p, (long)q->row, (long)q->head};
  r.out = KvSide{out->p, (long)out->row, (long)out->head};
  r.parts = static_cast<float*>(workspace);
  r.rows = (long)rows;
  r.n = n;
  r.q_len = q_start ? 0 : (int)(rows / n);
  r.hk = a.kv_heads;
  r.group = a.q_heads / a.kv_heads;
  r.d = a.head_dim;
  r.causal = a.causal;
  r.window = a.window;
  r.sinks = a.sinks;
  r.fill = q_start ? a.fill : 0;
  r.scale_log2 = a.scale * kLog2e;
  r.most_rows = (int)((q_start ? rows : rows / n) * r.group);
  r.row_log = p.row_log;
  r.key_log = p.key_log;
  r.tiles = (int)p.tiles;
  r.tiles_each = p.tiles_each;
  r.splits = p.splits;
  r.chunk = p.chunk;
  r.even = p.even;
  r.shares = p.shares;
  return r;
}

// Rows of a workgroup by those of a sequence; then, where the row tiles alone
// leave the chip idle, the keys of each are shared by several workgroups.
AttendPlan plan_with(const incvit_attention& a, bool cached, long n, long rows, bool ragged, long max_len, int most) {
  AttendPlan p = {};
  const bool bf16 = a.dtype == INCVIT_BF16;
  const long group = a.q_heads / a.kv_heads, each = (rows + n - 1) / n * group;
  const int ds = kv_dims(a.head_dim);
  p.key_log = 5;
  const long all = rows * a.q_heads;
  if (each > (cached ? (all <= kFewRows ? 256 : 64) : bf16 ? (all <= kFewRows / 2 ? 128 : 16) : 32) && (bf16 || !cached)) {
    p.by_rows = 1;
    p.nt = cached ? cached_wave_tiles(ds) : std::min(most_wave_tiles(bf16, ds), each <= 64 ? 1 : most);
    p.row_log = 5 + p.nt;
    p.key_log = cached ? 6 : rows_key_log(bf16, ds);
  } else {
    p.nt = cached ? std::min(most_row_tiles(bf16, ds), each <= 16 ? 1 : 2) : 1;
    p.row_log = 3 + p.nt;
  }
  const long tr = 1L << p.row_log, kt = 1L << p.key_log;
  p.tiles_each = (int)((rows / n * group + tr - 1) / tr);
  p.tiles = ragged ? rows * group / tr + n + a.fill : n * p.tiles_each;
  // key tiles of a row tile at most: the kernels see no more keys of a sequence, and
  // counts of their tiles stay within 32 bits
  long span = std::min(max_len, (long)kMostKeys);
  if (a.window) span = std::min(span, (long)a.window * (a.causal ? 1 : 2) + tr / group + 1 + a.sinks + 3 * kt);
  const long tiles = std::max(1L, (span + kt - 1) / kt);
  const long wgs = std::max(1L, p.tiles * a.kv_heads);
  p.splits = 1;
  p.shares = p.tiles;
  p.chunk = (int)(p.by_rows ? kLeastRows : kLeast);
  if (tiles <= 2 * p.chunk) return p;  // a second launch takes as long as the keys that it saves
  if (!p.by_rows && !ragged && n > 1 && n <= kEvenTiles && p.tiles_each == 1) {
    p.even = (int)std::max(1L, kWant / a.kv_heads);
    p.shares = p.even + p.tiles;
  } else if (wgs < 256) {
    const long want = (p.by_rows ? kWantRows : kWant) / wgs;
    p.chunk = (int)std::max((long)p.chunk, (tiles + want - 1) / want);
    p.splits = (int)std::min((long)kMostShares, (tiles + p.chunk - 1) / p.chunk);
    p.shares = p.tiles * p.splits;
  }
  if (p.splits > 1 || p.even) p.bytes = (size_t)p.shares * a.kv_heads * tr * (ds + 2) * 4;
  return p;
}

}  // namespace

AttendPlan incvit::attend_plan(const incvit_attention& a, bool cached, long n, long rows, bool ragged, long max_len) {
  const AttendPlan p = plan_with(a, cached, n, rows, ragged, max_len, 2);
  const bool few = rows * a.q_heads <= (kv_dims(a.head_dim) <= 128 ? 2 : 1) * kOneTileRows;
  const long each = (rows + n - 1) / n * (a.q_heads / a.kv_heads);
  if (cached || !p.by_rows || p.splits > 1 || !few || each < kOneTileEach) return p;
  return plan_with(a, cached, n, rows, ragged, max_len, 1);
}

extern "C" {

size_t incvit_kv_bytes(const incvit_kv* c) {
  return c && kv_ok(*c) ? KvLayout(c->blocks, c->block, c->heads, c->head_dim).total : 0;
}

incvit_status incvit_kv_write(const incvit_kv* c, int32_t dtype, int64_t rows, const void* k, int64_t k_row, int64_t k_head,
                              const void* v, int64_t v_row, int64_t v_head, const int32_t* slots, int32_t begin, void* cache,
                              void* stream) {
  incvit_status st = check_kv(c, dtype, rows, cache, slots);
  if (st != INCVIT_OK || rows == 0) return st;
  if ((st = check_rows(dtype, k, k_row, k_head, "k")) != INCVIT_OK) return st;
  if ((st = check_rows(dtype, v, v_row, v_head, "v")) != INCVIT_OK) return st;
  if (begin != 0 && begin != 1) return op_fail(INCVIT_ERR_ARG, "begin must be 0 or 1");
  KvWriteArgs a = {};
  a.x[0] = KvSide{k, (long)k_row, (long)k_head};
  a.x[1] = KvSide{v, (long)v_row, (long)v_head};
  a.slots = slots;
  a.cache = static_cast<char*>(cache);
  a.data = KvLayout(c->blocks, c->block, c->heads, c->head_dim).data;
  a.rows = (long)rows;
  a.blocks = c->blocks;
  a.block = c->block;
  a.heads = c->heads;
  a.d = c->head_dim;
  a.begin = begin;
  a.dtype = dtype;
  return launched(launch_kv_write(a, static_cast<hipStream_t>(stream)), "kv_write");
}

incvit_status incvit_kv_read(const incvit_kv* c, const void* cache, int32_t dtype, int64_t rows, const int32_t* slots,
                             int32_t fill, void* k, int64_t k_row, int64_t k_head, void* v, int64_t v_row, int64_t v_head,
                             void* stream) {
  incvit_status st = check_kv(c, dtype, rows, cache, slots);
  if (st != INCVIT_OK || rows == 0) return st;
  if ((st = check_rows(dtype, k, k_row, k_head, "k")) != INCVIT_OK) return st;
  if ((st = check_rows(dtype, v, v_row, v_head, "v")) != INCVIT_OK) return st;
  if (fill != 0 && fill != 1) return op_fail(INCVIT_ERR_ARG, "fill must be 0 or 1");
  if (!apart(rows, k_row, c->heads, k_head, c->head_dim) || !apart(rows, v_row, c->heads, v_head, c->head_dim))
    return op_fail(INCVIT_ERR_SHAPE, "heads of the output overlap");
  KvReadArgs a = {};
  a.x[0] = KvSide{k, (long)k_row, (long)k_head};
  a.x[1] = KvSide{v, (long)v_row, (long)v_head};
  a.slots = slots;
  a.cache = static_cast<const char*>(cache);
  a.data = KvLayout(c->blocks, c->block, c->heads, c->head_dim).data;
  a.rows = (long)rows;
  a.blocks = c->blocks;
  a.block = c->block;
  a.heads = c->heads;
  a.d = c->head_dim;
  a.dtype = dtype;
  a.fill = fill;
  return launched(launch_kv_read(a, static_cast<hipStream_t>(stream)), "kv_read");
}

size_t incvit_attention_workspace_bytes(const incvit_attention* a, int32_t cached, int32_t n, int64_t rows, int32_t ragged,
                                        int64_t max_len) {
  if (!a || !attention_ok(*a) || n < 1 || n > (1 << 24) || rows < 1 || max_len < 0 || max_len > kMostStride ||
      rows > ((int64_t)1 << 30) / (a->q_heads / a->kv_heads) - 1)
    return 0;
  return attend_plan(*a, cached != 0, n, (long)rows, ragged != 0, (long)max_len).bytes;
}

incvit_status incvit_kv_attend(const incvit_attention* a, const incvit_kv* c, const void* cache, int32_t n, int64_t rows,
                               const int32_t* q_start, const int32_t* table, int64_t table_stride, int32_t width, const int32_t* lens,
                               int64_t max_len, const incvit_rows* q, const incvit_rows* out, void* workspace, void* stream) {
  incvit_status st = check_attention(a, n, rows);
  if (st != INCVIT_OK) return st;
  if (!c || !kv_ok(*c)) return op_fail(c ? INCVIT_ERR_UNSUPPORTED : INCVIT_ERR_ARG, "cache out of range (blocks, block, heads or head_dim)");
  if (c->heads != a->kv_heads || c->head_dim != a->head_dim)
    return op_fail(INCVIT_ERR_SHAPE, "the cache's heads and head_dim must be the attention's");
  if (n == 0 || rows == 0) return INCVIT_OK;
  if (!q || !out) return op_fail(INCVIT_ERR_ARG, "null queries or output");
  if (!cache || (uintptr_t)cache % 256) return op_fail(INCVIT_ERR_ARG, "the cache must be non-null and 256-byte aligned");
  if ((!table && width > 0) || !lens) return op_fail(INCVIT_ERR_ARG, "null table or lens");
  if (((uintptr_t)table | (uintptr_t)lens | (uintptr_t)q_start) % 4)
    return op_fail(INCVIT_ERR_ARG, "q_start, table and lens must be 4-byte aligned");
  if (width < 0 || table_stride < 0 || table_stride > kMostStride)
    return op_fail(INCVIT_ERR_ARG, "width must be >= 0 and table_stride in [0, 2^40]");
  if (!q_start && rows % n) return op_fail(INCVIT_ERR_SHAPE, "without q_start rows must be a multiple of n");
  if (max_len < 0 || max_len > kMostStride) return op_fail(INCVIT_ERR_ARG, "max_len must be in [0, 2^40]");
  if ((st = check_rows(a->dtype, q->p, q->row, q->head, "q")) != INCVIT_OK) return st;
  if ((st = check_rows(a->dtype, out->p, out->row, out->head, "out")) != INCVIT_OK) return st;
  if (!apart(rows, out->row, a->q_heads, out->head, a->head_dim)) return op_fail(INCVIT_ERR_SHAPE, "heads of the output overlap");
  const AttendPlan p = attend_plan(*a, true, n, (long)rows, q_start != nullptr, max_len ? (long)max_len : (long)width * c->block);
  if ((st = check_plan(*a, p, workspace)) != INCVIT_OK) return st;
  AttendArgs r = attend_args(*a, p, n, rows, q_start, q, out, workspace);
  const KvLayout lay(c->blocks, c->block, c->heads, c->head_dim);
  r.cache = static_cast<const char*>(cache);
  r.data = lay.data;
  r.lens = lens;
  r.table = table;
  r.table_stride = (long)table_stride;
  r.width = width;
  r.blocks = c->blocks;
  r.lb = lay.lb;
  hipStream_t s = static_cast<hipStream_t>(stream);
  if ((st = launched(p.by_rows ? launch_kv_attend_rows(r, s) : launch_kv_attend(r, p, a->dtype, s), "kv_attend")) != INCVIT_OK) return st;
  return launched(launch_attend_join(r, a->dtype, s), "kv_attend");
}

incvit_status incvit_attend(const incvit_attention* a, int32_t n, int64_t rows, const int32_t* q_start, int64_t key_rows,
                            const int32_t* k_start, int64_t max_len, const incvit_rows* q, const incvit_rows* k, const incvit_rows* v,
                            const incvit_rows* out, void* workspace, void* stream) {
  incvit_status st = check_attention(a, n, rows);
  if (st != INCVIT_OK) return st;
  if (key_rows < 0 || key_rows > (1 << 30)) return op_fail(INCVIT_ERR_ARG, "key_rows must be in [0, 2^30]");
  if (n == 0 || rows == 0) return INCVIT_OK;
  if (!q || !k || !v || !out) return op_fail(INCVIT_ERR_ARG, "null queries, keys, values or output");
  if (((uintptr_t)q_start | (uintptr_t)k_start) % 4) return op_fail(INCVIT_ERR_ARG, "q_start and k_start must be 4-byte aligned");
  if (!q_start && rows % n) return op_fail(INCVIT_ERR_SHAPE, "without q_start rows must be a multiple of n");
  if (!k_start && key_rows % n) return op_fail(INCVIT_ERR_SHAPE, "without k_start key_rows must be a multiple of n");
  if (max_len < 0 || max_len > kMostStride) return op_fail(INCVIT_ERR_ARG, "max_len must be in [0, 2^40]");
  if ((st = check_rows(a->dtype, q->p, q->row, q->head, "q")) != INCVIT_OK) return st;
  if ((st = check_rows(a->dtype, out->p, out->row, out->head, "out")) != INCVIT_OK) return st;
  if (key_rows > 0) {
    if ((st = check_rows(a->dtype, k->p, k->row, k->head, "k")) != INCVIT_OK) return st;
    if ((st = check_rows(a->dtype, v->p, v->row, v->head, "v")) != INCVIT_OK) return st;
    // a tile's rows are addressed with 31 bits
    if (k->row > (1 << 23) || v->row > (1 << 23)) return op_fail(INCVIT_ERR_UNSUPPORTED, "rows of keys and values more than 2^23 elements apart");
  }
  if (!apart(rows, out->row, a->q_heads, out->head, a->head_dim)) return op_fail(INCVIT_ERR_SHAPE, "heads of the output overlap");
  const AttendPlan p = attend_plan(*a, false, n, (long)rows, q_start != nullptr, max_len ? (long)max_len : (long)((key_rows + n - 1) / n));
  if ((st = check_plan(*a, p, workspace)) != INCVIT_OK) return st;
  AttendArgs r = attend_args(*a, p, n, rows, q_start, q, out, workspace);
  r.k = KvSide{k->p, (long)k->row, (long)k->head};
  r.v = KvSide{v->p, (long)v->row, (long)v->head};
  r.k_start = k_start;
  r.key_rows = (long)key_rows;
  r.k_len = k_start ? 0 : (int)(key_rows / n);
  hipStream_t s = static_cast<hipStream_t>(stream);
  if ((st = launched(p.by_rows ? launch_attend_rows(r, p, a->dtype, s) : launch_attend(r, a->dtype, s), "attend")) != INCVIT_OK) return st;
  return launched(launch_attend_join(r, a->dtype, s), "attend");
}

}  // extern "C"
