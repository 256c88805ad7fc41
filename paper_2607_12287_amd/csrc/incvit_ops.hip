// C ABI of the stand-alone operators: argument checks and launches.
#include <algorithm>
#include <cmath>

#include "ops.hpp"

using namespace incvit;

namespace {

bool is_dtype(int32_t t) { return t == INCVIT_F32 || t == INCVIT_BF16; }

incvit_status launched(hipError_t e, const char* what) {
  if (e == hipSuccess) return INCVIT_OK;
  char buf[160];
  snprintf(buf, sizeof buf, "%s: %s", what, hipGetErrorString(e));
  return op_fail(INCVIT_ERR_HIP, buf);
}

// Whether rows x heads runs of d elements at r * row + h * head never overlap.
bool disjoint(int64_t rows, int64_t row, int64_t heads, int64_t head, int64_t d) {
  if (rows <= 1) return heads <= 1 || head >= d;
  if (heads <= 1) return row >= d;
  const int64_t lo = row < head ? row : head, hi = row < head ? head : row, n = row < head ? rows : heads;
  return lo >= d && (n - 1 <= (hi - d) / lo) && hi >= d;
}

incvit_status check_heads(const incvit_qk& c, int64_t rows, int64_t out_rows, const incvit_heads* h, QkSide& s) {
  s = QkSide{};
  if (!h || h->heads == 0) return INCVIT_OK;
  const uintptr_t eb = c.dtype == INCVIT_BF16 ? 2 : 4;
  if (h->heads < 0 || h->heads > 65536) return op_fail(INCVIT_ERR_ARG, "heads must be in [0, 65536]");
  if (!h->in || !h->out) return op_fail(INCVIT_ERR_ARG, "null rows of queries or keys");
  if (((uintptr_t)h->in | (uintptr_t)h->out | (uintptr_t)h->gamma | (uintptr_t)h->beta) % eb)
    return op_fail(INCVIT_ERR_ARG, "rows, gammas and betas must be aligned to their elements");
  if (h->beta && c.norm != INCVIT_NORM_LAYER) return op_fail(INCVIT_ERR_ARG, "beta is given without a LayerNorm");
  const int64_t most = (int64_t)1 << 40;
  for (int64_t st : {h->in_row, h->in_head, h->out_row, h->out_head})
    if (st < 0 || st > most) return op_fail(INCVIT_ERR_ARG, "strides must be in [0, 2^40] elements");
  if (!disjoint(out_rows, h->out_row, h->heads, h->out_head, c.head_dim))
    return op_fail(INCVIT_ERR_SHAPE, "heads of the output overlap");
  if (h->in == h->out && ((rows > 1 && h->in_row != h->out_row) || (h->heads > 1 && h->in_head != h->out_head)))
    return op_fail(INCVIT_ERR_SHAPE, "in place, the output's strides must be the input's");
  s = QkSide{h->in, h->out, h->gamma, h->beta, (long)h->in_row, (long)h->in_head, (long)h->out_row, (long)h->out_head, h->heads};
  return INCVIT_OK;
}

bool q_sizes(int32_t K, int32_t N) {
  return K >= 1 && K <= 65536 && N >= 1 && N <= (1 << 20) &&
         (uint64_t)((N + 15) / 16) * ((K + 63) / 64) * 1024 < ((uint64_t)1 << 32);
}

incvit_status check_q(int64_t rows, int32_t K, int32_t N) {
  if (!q_sizes(K, N)) return op_fail(INCVIT_ERR_UNSUPPORTED, "K must be in [1, 65536], N in [1, 2^20] and the packed weights below 4 GiB");
  if (rows < 0 || rows > INT32_MAX - 64) return op_fail(INCVIT_ERR_ARG, "rows must be in [0, 2^31 - 64)");
  return INCVIT_OK;
}

incvit_status check_x(int32_t dtype, const void* x, int64_t x_stride, const void* qrows) {
  if (!is_dtype(dtype)) return op_fail(INCVIT_ERR_UNSUPPORTED, "dtype must be INCVIT_F32 or INCVIT_BF16");
  if (!x || !qrows) return op_fail(INCVIT_ERR_ARG, "null rows");
  if ((uintptr_t)x % (dtype == INCVIT_BF16 ? 2 : 4)) return op_fail(INCVIT_ERR_ARG, "rows must be aligned to their elements");
  if ((uintptr_t)qrows % 256) return op_fail(INCVIT_ERR_ARG, "quantised rows must be 256-byte aligned");
  if (x_stride < 0 || x_stride > ((int64_t)1 << 40)) return op_fail(INCVIT_ERR_ARG, "x_stride must be in [0, 2^40] elements");
  return INCVIT_OK;
}

incvit_status check_out(int32_t dtype, int64_t rows, int32_t N, const void* weights, int32_t gelu, const void* residual,
                        int64_t res_stride, const void* out, int64_t out_stride) {
  if (!is_dtype(dtype)) return op_fail(INCVIT_ERR_UNSUPPORTED, "dtype must be INCVIT_F32 or INCVIT_BF16");
  if (!weights || !out) return op_fail(INCVIT_ERR_ARG, "null weights or output");
  if ((uintptr_t)weights % 256) return op_fail(INCVIT_ERR_ARG, "weights must be 256-byte aligned");
  if (((uintptr_t)out | (uintptr_t)residual) % (dtype == INCVIT_BF16 ? 2 : 4))
    return op_fail(INCVIT_ERR_ARG, "out and residual must be aligned to their elements");
  if (gelu != 0 && gelu != 1) return op_fail(INCVIT_ERR_ARG, "gelu must be 0 or 1");
  const int64_t most = (int64_t)1 << 40;
  if ((rows > 1 && out_stride < N) || out_stride < 0 || out_stride > most) return op_fail(INCVIT_ERR_SHAPE, "out_stride must be in [N, 2^40]");
  if (residual && (res_stride < 0 || res_stride > most)) return op_fail(INCVIT_ERR_ARG, "res_stride must be in [0, 2^40]");
  if (residual == out && residual && rows > 1 && res_stride != out_stride)
    return op_fail(INCVIT_ERR_SHAPE, "a residual in place must have the output's stride");
  return INCVIT_OK;
}

// Rows per launch: the large-row GEMM addresses its rows' integers with 32 bits,
// and a launch counts its threads in as many.
int64_t q_slab(int32_t K) { return std::min((((int64_t)1 << 31) / ((K + 63) / 64 * 64)) / 256 * 256, (int64_t)1 << 21); }

incvit_status q_rows(int32_t dtype, int64_t rows, int32_t K, const void* x, int64_t x_stride, const void* gamma, const void* beta,
                     float eps, void* qrows, hipStream_t s) {
  const QRowsLayout l(rows, K);
  const size_t eb = dtype == INCVIT_BF16 ? 2 : 4;
  QRowsArgs a = {};
  a.ld = (long)x_stride;
  a.gamma = gamma;
  a.beta = beta;
  a.eps = eps;
  a.K = K;
  a.dtype = dtype;
  const int64_t slab = q_slab(K);
  for (int64_t r = 0; r < rows; r += slab) {
    a.x = static_cast<const char*>(x) + (size_t)r * x_stride * eb;
    a.dst = static_cast<char*>(qrows) + (size_t)(r / 16) * l.kc * 1024;
    a.scale = reinterpret_cast<float*>(static_cast<char*>(qrows) + l.scale) + r;
    a.rows = (long)(rows - r < slab ? rows - r : slab);
    const incvit_status st = launched(launch_q_rows(a, s), "qlinear_quantize_rows");
    if (st != INCVIT_OK) return st;
  }
  return INCVIT_OK;
}

// Whether rows of n elements every `stride` from p on and the same from q on share
// a span of memory.
bool spans_meet(int64_t rows, size_t eb, const void* p, int64_t n, int64_t stride, const void* q, int64_t m, int64_t ostride) {
  const uintptr_t a = (uintptr_t)p, b = (uintptr_t)q;
  return a < b + ((rows - 1) * ostride + m) * eb && b < a + ((rows - 1) * stride + n) * eb;
}

// What a product has but its rows and outputs.
GemmArgs q_args(int32_t K, int32_t N, const void* weights, int32_t gelu, int64_t res_stride, int64_t out_stride) {
  const QWeightsLayout wl(K, N);
  const char* w = static_cast<const char*>(weights);
  GemmArgs a = {};
  a.W = w;
  a.col_scale = reinterpret_cast<const float*>(w + wl.scale);
  a.bias = reinterpret_cast<const float*>(w + wl.bias);
  a.lda = 64 * wl.kc;
  a.kchunks = wl.kc;
  a.Nout = 16 * wl.blocks;
  a.n = N;
  a.ksplit = 1;
  a.gelu = gelu;
  a.out_ld = (long)out_stride;
  a.res_ld = (long)res_stride;
  return a;
}

incvit_status q_multiply(int32_t dtype, int64_t rows, int32_t K, int32_t N, const void* qrows, const void* weights, int32_t gelu,
                         const void* residual, int64_t res_stride, void* out, int64_t out_stride, hipStream_t s) {
  const QRowsLayout rl(rows, K);
  const size_t eb = dtype == INCVIT_BF16 ? 2 : 4;
  GemmArgs a = q_args(K, N, weights, gelu, res_stride, out_stride);
  const int64_t slab = q_slab(K);
  for (int64_t r = 0; r < rows; r += slab) {
    const int m = (int)(rows - r < slab ? rows - r : slab);
    a.A = static_cast<const char*>(qrows) + (size_t)(r / 16) * a.kchunks * 1024;
    a.row_scale = reinterpret_cast<const float*>(static_cast<const char*>(qrows) + rl.scale) + r;
    a.out = static_cast<char*>(out) + (size_t)r * out_stride * eb;
    a.resid = residual ? static_cast<const char*>(residual) + (size_t)r * res_stride * eb : nullptr;
    a.m_host = m;
    a.mpad = (m + 15) / 16 * 16;
    const incvit_status st = launched(launch_q_gemm(a, dtype == INCVIT_F32, m, m, s), "qlinear_multiply");
    if (st != INCVIT_OK) return st;
  }
  return INCVIT_OK;
}

}  // namespace

extern "C" {

incvit_status incvit_rope_table(const incvit_rope* r, int64_t tokens, const int32_t* pos, int64_t axis_stride, int64_t token_stride,
                                float* table, void* stream) {
  RopeArgs a = {};
  if (!r) return op_fail(INCVIT_ERR_ARG, "null rope");
  if (!rope_pairs(*r, a)) return op_fail(INCVIT_ERR_ARG, "rope out of range (axes, pairs, ladder, layout, theta or scale)");
  if (tokens < 0 || tokens > INT32_MAX / a.pairs) return op_fail(INCVIT_ERR_ARG, "tokens must be >= 0 and tokens * pairs < 2^31");
  if (tokens == 0) return INCVIT_OK;
  if (!pos || !table) return op_fail(INCVIT_ERR_ARG, "null positions or table");
  if ((uintptr_t)pos % 4 || (uintptr_t)table % 8) return op_fail(INCVIT_ERR_ARG, "positions must be 4-byte and the table 8-byte aligned");
  const int64_t most = (int64_t)1 << 40;
  if (axis_stride < 0 || axis_stride > most || token_stride < 0 || token_stride > most)
    return op_fail(INCVIT_ERR_ARG, "strides must be in [0, 2^40] elements");
  a.tokens = (int)tokens;
  a.pos = pos;
  a.axis_stride = (long)axis_stride;
  a.token_stride = (long)token_stride;
  a.table = table;
  return launched(launch_rope(a, static_cast<hipStream_t>(stream)), "rope_table");
}

incvit_status incvit_rope_table_grids(const incvit_rope* r, int32_t n, const incvit_grid* grids, int32_t merge, float* table,
                                      void* stream) {
  RopeArgs a = {};
  if (!r) return op_fail(INCVIT_ERR_ARG, "null rope");
  if (!rope_pairs(*r, a)) return op_fail(INCVIT_ERR_ARG, "rope out of range (axes, pairs, ladder, layout, theta or scale)");
  if (n < 0) return op_fail(INCVIT_ERR_ARG, "n must be >= 0");
  if (n == 0) return INCVIT_OK;
  if (!grids || !table) return op_fail(INCVIT_ERR_ARG, "null grids or table");
  if ((uintptr_t)table % 8) return op_fail(INCVIT_ERR_ARG, "the table must be 8-byte aligned");
  if (merge < 1) return op_fail(INCVIT_ERR_ARG, "merge must be >= 1");
  int64_t tokens = 0;
  for (int32_t i = 0; i < n; ++i) {
    const incvit_grid& g = grids[i];
    if (g.t < 1 || g.h < 1 || g.w < 1) return op_fail(INCVIT_ERR_ARG, "grid sizes must be >= 1");
    if (g.h % merge || g.w % merge) return op_fail(INCVIT_ERR_SHAPE, "grid height and width must be multiples of merge");
    const int64_t frame = (int64_t)g.h * g.w;
    if (frame > INT32_MAX || g.t > INT32_MAX / frame) tokens = INT64_MAX / 2;
    else tokens += frame * g.t;
    if (tokens > INT32_MAX / a.pairs) return op_fail(INCVIT_ERR_ARG, "tokens * pairs must be < 2^31");
  }
  a.merge = merge;
  for (int32_t i = 0; i < n; i += kGridsPerLaunch) {
    for (int j = 0; j < kGridsPerLaunch && i + j < n; ++j) rope_grid(a, j, grids[i + j]);
    a.table = table;
    table += (size_t)a.tokens * a.pairs * 2;
    const incvit_status st = launched(launch_rope(a, static_cast<hipStream_t>(stream)), "rope_table_grids");
    if (st != INCVIT_OK) return st;
  }
  return INCVIT_OK;
}

incvit_status incvit_qk_norm_rope(const incvit_qk* c, int64_t rows, const incvit_heads* q, const incvit_heads* k,
                                  const float* table, int64_t table_rows, const int32_t* index, const int32_t* k_rows,
                                  int64_t k_out_rows, void* stream) {
  if (!c) return op_fail(INCVIT_ERR_ARG, "null configuration");
  if (!is_dtype(c->dtype)) return op_fail(INCVIT_ERR_UNSUPPORTED, "dtype must be INCVIT_F32 or INCVIT_BF16");
  if (c->head_dim < 2 || c->head_dim > 2 * kMaxPairs || c->head_dim % 2)
    return op_fail(INCVIT_ERR_UNSUPPORTED, "head_dim must be even and in [2, 256]");
  if (c->rot_dim < 0 || c->rot_dim > c->head_dim || c->rot_dim % 2)
    return op_fail(INCVIT_ERR_SHAPE, "rot_dim must be even and in [0, head_dim]");
  if (c->pairing != INCVIT_PAIR_HALVES && c->pairing != INCVIT_PAIR_ADJACENT)
    return op_fail(INCVIT_ERR_ARG, "pairing must be INCVIT_PAIR_HALVES or INCVIT_PAIR_ADJACENT");
  if (c->norm != INCVIT_NORM_NONE && c->norm != INCVIT_NORM_RMS && c->norm != INCVIT_NORM_LAYER)
    return op_fail(INCVIT_ERR_ARG, "norm must be INCVIT_NORM_NONE, _RMS or _LAYER");
  if (!(c->eps >= 0.0f) || !std::isfinite(c->eps)) return op_fail(INCVIT_ERR_ARG, "eps must be >= 0 and finite");
  if (rows < 0) return op_fail(INCVIT_ERR_ARG, "rows must be >= 0");
  if (rows == 0) return INCVIT_OK;
  if (c->rot_dim > 0) {
    if (!table || (uintptr_t)table % 8) return op_fail(INCVIT_ERR_ARG, "the table must be non-null and 8-byte aligned");
    if (table_rows < 1 || table_rows > INT32_MAX) return op_fail(INCVIT_ERR_ARG, "table_rows must be in [1, 2^31)");
  }
  if (((uintptr_t)index | (uintptr_t)k_rows) % 4) return op_fail(INCVIT_ERR_ARG, "index and k_rows must be 4-byte aligned");
  if (k_rows && (k_out_rows < 1 || k_out_rows > INT32_MAX)) return op_fail(INCVIT_ERR_ARG, "k_out_rows must be in [1, 2^31)");
  QkArgs a = {};
  incvit_status st = check_heads(*c, rows, rows, q, a.q);
  if (st != INCVIT_OK) return st;
  if ((st = check_heads(*c, rows, k_rows ? k_out_rows : rows, k, a.k)) != INCVIT_OK) return st;
  if (k_rows && a.k.heads && a.k.in == a.k.out) return op_fail(INCVIT_ERR_SHAPE, "k_rows cannot move keys in place");
  const int64_t heads = (int64_t)a.q.heads + a.k.heads;
  if (heads == 0) return INCVIT_OK;
  if (rows > INT32_MAX / heads) return op_fail(INCVIT_ERR_ARG, "rows * heads must be < 2^31");
  a.dtype = c->dtype;
  a.head_dim = c->head_dim;
  a.rot_pairs = c->rot_dim / 2;
  a.adjacent = c->pairing;
  a.norm = c->norm;
  a.eps = c->eps;
  a.rows = (long)rows;
  a.table = table;
  a.table_rows = (long)table_rows;
  a.index = index;
  a.k_rows = k_rows;
  a.k_out_rows = (long)k_out_rows;
  return launched(launch_qk(a, static_cast<hipStream_t>(stream)), "qk_norm_rope");
}

size_t incvit_qlinear_weights_bytes(int32_t K, int32_t N) { return q_sizes(K, N) ? QWeightsLayout(K, N).total : 0; }

size_t incvit_qlinear_rows_bytes(int64_t rows, int32_t K) {
  if (rows < 0 || rows > INT32_MAX - 64 || K < 1 || K > 65536) return 0;
  return QRowsLayout((long)rows, K).total;
}

incvit_status incvit_qlinear_pack_weights(int32_t dtype, int32_t K, int32_t N, const void* w, int64_t k_stride, int64_t n_stride,
                                          const float* scales, const void* bias, void* weights, void* stream) {
  const incvit_status st = check_q(0, K, N);
  if (st != INCVIT_OK) return st;
  if (!is_dtype(dtype) && dtype != INCVIT_I8) return op_fail(INCVIT_ERR_UNSUPPORTED, "dtype must be INCVIT_F32, INCVIT_BF16 or INCVIT_I8");
  if (!w || !weights) return op_fail(INCVIT_ERR_ARG, "null weights");
  if ((uintptr_t)weights % 256) return op_fail(INCVIT_ERR_ARG, "packed weights must be 256-byte aligned");
  if ((dtype == INCVIT_I8) != (scales != nullptr)) return op_fail(INCVIT_ERR_ARG, "scales belong to INCVIT_I8 weights, and those need them");
  const uintptr_t eb = dtype == INCVIT_F32 ? 4 : dtype == INCVIT_BF16 ? 2 : 1;
  if ((uintptr_t)w % eb || (uintptr_t)bias % (dtype == INCVIT_BF16 ? 2 : 4) || (uintptr_t)scales % 4)
    return op_fail(INCVIT_ERR_ARG, "weights, scales and bias must be aligned to their elements");
  const int64_t most = (int64_t)1 << 40;
  if (k_stride < 0 || n_stride < 0 || k_stride > most || n_stride > most)
    return op_fail(INCVIT_ERR_ARG, "strides must be in [0, 2^40] elements");
  const QPackArgs a = {w, (long)k_stride, (long)n_stride, scales, bias, static_cast<char*>(weights), K, N, dtype};
  return launched(launch_q_pack(a, static_cast<hipStream_t>(stream)), "qlinear_pack_weights");
}

incvit_status incvit_qlinear_quantize_rows(int32_t dtype, int64_t rows, int32_t K, const void* x, int64_t x_stride,
                                           const void* gamma, const void* beta, float eps, void* qrows, void* stream) {
  incvit_status st = check_q(rows, K, 1);
  if (st != INCVIT_OK) return st;
  if (rows == 0) return INCVIT_OK;
  if ((st = check_x(dtype, x, x_stride, qrows)) != INCVIT_OK) return st;
  if (beta && !gamma) return op_fail(INCVIT_ERR_ARG, "beta is given without gamma");
  if (((uintptr_t)gamma | (uintptr_t)beta) % (dtype == INCVIT_BF16 ? 2 : 4))
    return op_fail(INCVIT_ERR_ARG, "gamma and beta must be aligned to their elements");
  if (gamma && (!(eps >= 0.0f) || !std::isfinite(eps))) return op_fail(INCVIT_ERR_ARG, "eps must be >= 0 and finite");
  return q_rows(dtype, rows, K, x, x_stride, gamma, beta, eps, qrows, static_cast<hipStream_t>(stream));
}

incvit_status incvit_qlinear_multiply(int32_t dtype, int64_t rows, int32_t K, int32_t N, const void* qrows, const void* weights,
                                      int32_t gelu, const void* residual, int64_t res_stride, void* out, int64_t out_stride,
                                      void* stream) {
  incvit_status st = check_q(rows, K, N);
  if (st != INCVIT_OK) return st;
  if (rows == 0) return INCVIT_OK;
  if (!qrows || (uintptr_t)qrows % 256) return op_fail(INCVIT_ERR_ARG, "quantised rows must be non-null and 256-byte aligned");
  if ((st = check_out(dtype, rows, N, weights, gelu, residual, res_stride, out, out_stride)) != INCVIT_OK) return st;
  return q_multiply(dtype, rows, K, N, qrows, weights, gelu, residual, res_stride, out, out_stride, static_cast<hipStream_t>(stream));
}

incvit_status incvit_qlinear(int32_t dtype, int64_t rows, int32_t K, int32_t N, const void* x, int64_t x_stride,
                             const void* weights, int32_t gelu, const void* residual, int64_t res_stride, void* out,
                             int64_t out_stride, void* workspace, void* stream) {
  incvit_status st = check_q(rows, K, N);
  if (st != INCVIT_OK) return st;
  if (rows == 0) return INCVIT_OK;
  if ((st = check_x(dtype, x, x_stride, workspace)) != INCVIT_OK) return st;
  if ((st = check_out(dtype, rows, N, weights, gelu, residual, res_stride, out, out_stride)) != INCVIT_OK) return st;
  hipStream_t s = static_cast<hipStream_t>(stream);
  // in one launch only where no workgroup's output can be another's input
  if (q_token_fits(rows, K) && !spans_meet(rows, dtype == INCVIT_BF16 ? 2 : 4, x, K, x_stride, out, N, out_stride)) {
    GemmArgs a = q_args(K, N, weights, gelu, res_stride, out_stride);
    a.A = x;
    a.x_ld = (long)x_stride;
    a.k = K;
    a.out = out;
    a.resid = residual;
    a.m_host = (int)rows;
    return launched(launch_q_token(a, dtype == INCVIT_F32, s), "qlinear");
  }
  if ((st = q_rows(dtype, rows, K, x, x_stride, nullptr, nullptr, 0.0f, workspace, s)) != INCVIT_OK) return st;
  return q_multiply(dtype, rows, K, N, workspace, weights, gelu, residual, res_stride, out, out_stride, s);
}

}  // extern "C"
