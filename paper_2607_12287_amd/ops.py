"""The library's stand-alone operators on torch tensors (reached as attributes of
:mod:`paper_2607_12287_amd.incvit`).  Argument checks and memory only: a call is
one or two kernels of a few microseconds, so the checks build nothing that they do
not need.  Work goes to the current stream of the tensors' device; results carry
no gradient.
"""
from __future__ import annotations

import struct
from typing import Optional

import torch

from . import incvit as _c

_BF16, _F32 = torch.bfloat16, torch.float32
_CODES = {_F32: _c.INCVIT_F32, _BF16: _c.INCVIT_BF16, torch.int8: _c.INCVIT_I8}
# incvit_heads and incvit_qk as their bytes: 0.1 us each, a ctypes structure 0.4
_HEADS, _QK = struct.Struct("4P4qi4x"), struct.Struct("5if")
assert _HEADS.size == _c.ctypes.sizeof(_c.incvit_heads) and _QK.size == _c.ctypes.sizeof(_c.incvit_qk)
_KV, _ATTENTION, _ROWS = struct.Struct("4i"), struct.Struct("8if"), struct.Struct("P2q")
assert (_KV.size == _c.ctypes.sizeof(_c.incvit_kv) and _ATTENTION.size == _c.ctypes.sizeof(_c.incvit_attention) and
        _ROWS.size == _c.ctypes.sizeof(_c.incvit_rows))
_stream_of = torch._C._cuda_getCurrentRawStream
_current = torch._C._cuda_getDevice


def _call(f, device, *args):
    """f(*args, stream) with `device` current, on its current stream."""
    i = device.index
    if i == _current():
        st = f(*args, _stream_of(i))
    else:
        with torch.cuda.device(device):
            st = f(*args, _stream_of(i))
    if st:
        _c._check(st)


def _ptr(t):
    return None if t is None else t.data_ptr()


# ------------------------------------------------------- rotary positions --


def rope_table(rope: _c.incvit_rope, positions=None, grids=None, merge: int = 1, out=None, device=None):
    """[tokens][pairs][2] fp32 cosines and sines.  positions: device int32
    [axes][tokens], any strides; or grids: (t, h, w[, t0[, y0[, x0]]]) on the host,
    whose tokens follow one another (frame by frame, in merge x merge windows)."""
    n = sum(rope.pairs[:rope.axes])
    if (positions is None) == (grids is None):
        raise ValueError("either positions or grids")
    if positions is not None:
        if not (positions.is_cuda and positions.dtype == torch.int32 and positions.dim() == 2 and positions.shape[0] == rope.axes):
            raise ValueError("positions: device int32 [axes][tokens]")
        tokens, device = positions.shape[1], positions.device
    else:
        n_grids, arr = _c.grid_array(grids, merge)
        tokens = 0
        for g in grids:
            tokens += g[0] * g[1] * g[2]
        if device is None:
            device = out.device if out is not None else torch.device("cuda", torch.cuda.current_device())
        elif not isinstance(device, torch.device) or device.index is None:
            device = torch.empty(0, device=device).device
    if out is None:
        out = torch.empty(max(tokens, 0), n, 2, dtype=_F32, device=device)
    elif not (out.device == device and out.is_cuda and out.dtype == _F32 and out.is_contiguous() and out.numel() == tokens * n * 2):
        raise ValueError("out: device fp32 [tokens][pairs][2]")
    if positions is not None:
        _call(_c.lib().incvit_rope_table, device, _c.ctypes.byref(rope), tokens, positions.data_ptr(), *positions.stride(),
              out.data_ptr())
    else:
        _call(_c.lib().incvit_rope_table_grids, device, _c.ctypes.byref(rope), n_grids, arr, merge, out.data_ptr())
    return out


# ------------------------------------------- head norms with the rotation --


def _heads(x, out, gamma, beta, who: str) -> bytes:
    """The bytes of the incvit_heads of x and out."""
    for t in (gamma, beta):
        if t is not None and not (t.dtype == x.dtype and t.device == x.device and t.is_contiguous() and t.numel() == x.shape[2]):
            raise ValueError(f"{who}_gamma, {who}_beta: [head_dim] of the rows' type and device")
    s, o = x.stride(), out.stride()
    if not (out.dtype == x.dtype and out.device == x.device and out.dim() == 3 and out.shape[1:] == x.shape[1:]):
        raise ValueError(f"{who}_out: rows of the same heads, type and device")
    if s[2] != 1 or o[2] != 1:
        raise ValueError(f"{who}, {who}_out: the values of a head lie one after another")
    return _HEADS.pack(x.data_ptr(), out.data_ptr(), 0 if gamma is None else gamma.data_ptr(), 0 if beta is None else beta.data_ptr(),
                       s[0], s[1], o[0], o[1], x.shape[1])


def qk_norm_rope(q=None, k=None, table=None, pairing: str = "halves", norm: Optional[str] = "rms", q_gamma=None, k_gamma=None,
                 q_beta=None, k_beta=None, eps: float = 1e-6, index=None, k_rows=None, q_out=None, k_out=None):
    """Norm of every head of q [rows][q heads][d] and k [rows][k heads][d] (views
    with any row and head strides; either may be None), then the rotation by the
    table rows `index` (device int32 [rows]; without it row r % table rows) of
    `table` (rope_table's; None: no rotation).  k_rows (device int32 [rows]): the
    rows of k_out (a cache [..][k heads][d], then required) that the new keys go
    to.  q_out, k_out may be q and k (in place); made here they are new tensors.  A
    row whose index is outside the table (padding: negative) gets no output: it
    stays what it was in a given q_out or k_out and is zeros in a new one.  Returns
    (q_out, k_out)."""
    x = q if q is not None else k
    if x is None:
        raise ValueError("q or k")
    dt, dev = x.dtype, x.device
    if not (x.is_cuda and x.dim() == 3 and (dt == _BF16 or dt == _F32)):
        raise ValueError("q, k: device tensors [rows][heads][d], fp32 or bf16")
    rows, _, d = x.shape
    if q is not None and k is not None and not (k.dim() == 3 and k.shape[0] == rows and k.shape[2] == d and k.dtype == dt and
                                                k.device == dev):
        raise ValueError("q and k: [rows][heads][d] of one type on one device")
    rot = trows = 0
    if table is not None:
        if not (table.device == dev and table.dtype == _F32 and table.dim() == 3 and table.shape[2] == 2 and table.is_contiguous()):
            raise ValueError("table: device fp32 [rows][pairs][2]")
        trows, rot = table.shape[0], 2 * table.shape[1]
    new = torch.zeros if index is not None and rot else torch.empty  # rows that the kernel leaves out
    for t in (index, k_rows):
        if t is not None and not (t.dtype == torch.int32 and t.device == dev and t.is_contiguous() and t.numel() == rows):
            raise ValueError("index, k_rows: device int32 [rows]")
    if not norm:
        q_gamma = k_gamma = None
    hq = hk = None
    k_out_rows = 0
    if q is not None:
        if q_out is None:
            q_out = new(rows, q.shape[1], d, dtype=dt, device=dev)
        elif q_out.shape[0] != rows:
            raise ValueError("q_out: as many rows as q")
        hq = _heads(q, q_out, q_gamma, q_beta, "q")
    if k is not None:
        if k_rows is not None:
            if k_out is None:
                raise ValueError("k_rows: rows of k_out, which has to be given")
            k_out_rows = k_out.shape[0]
        elif k_out is None:
            k_out = new(rows, k.shape[1], d, dtype=dt, device=dev)
        elif k_out.shape[0] != rows:
            raise ValueError("k_out: as many rows as k")
        hk = _heads(k, k_out, k_gamma, k_beta, "k")
    elif k_rows is not None:
        raise ValueError("k_rows: rows of k_out, without k")
    c = _QK.pack(_CODES[dt], d, rot, _c.PAIRINGS[pairing], _c.NORMS[norm], eps)
    _call(_c.lib().incvit_qk_norm_rope, dev, c, rows, hq, hk, _ptr(table), trows, _ptr(index), _ptr(k_rows),
          k_out_rows)
    return q_out, k_out


# ----------------------------------------------------------- 8-bit products --


_MOST_K, _MOST_N = 65536, 1 << 20  # the library's, which takes both in 32 bits


def _rows_of(x):
    """(type code, rows, K) of rows that the 8-bit operators take."""
    code = _CODES.get(x.dtype, _c.INCVIT_I8)
    if not (x.is_cuda and code != _c.INCVIT_I8 and x.dim() == 2 and (x.stride(1) == 1 or x.shape[1] == 1)):
        raise ValueError("x: device fp32 or bf16 [rows][K], the values of a row one after another")
    if x.shape[1] > _MOST_K:
        raise _c.IncvitError(_c.INCVIT_ERR_UNSUPPORTED, f"rows of K = {x.shape[1]}")
    return code, x.shape[0], x.shape[1]


def _buffer(n: int, device):
    return torch.empty(n, dtype=torch.uint8, device=device)


class QRows:
    """Rows quantised to 8 bits (quantize_rows), for any number of products."""

    def __init__(self, rows: int, K: int, dtype, buf):
        self.rows, self.K, self.dtype, self.buf = rows, K, dtype, buf


def quantize_rows(x, gamma=None, beta=None, eps: float = 1e-6) -> QRows:
    """The rows of x [rows][K] in 8-bit integers with a scale each; with gamma
    (and beta), [K] of x's type, after a LayerNorm."""
    code, rows, K = _rows_of(x)
    for t in (gamma, beta):
        if t is not None and not (t.device == x.device and t.dtype == x.dtype and t.is_contiguous() and t.numel() == K):
            raise ValueError("gamma, beta: [K] of x's type and device")
    L = _c.lib()
    buf = _buffer(L.incvit_qlinear_rows_bytes(rows, K), x.device)
    _call(L.incvit_qlinear_quantize_rows, x.device, code, rows, K, x.data_ptr(), x.stride(0), _ptr(gamma), _ptr(beta), eps,
          buf.data_ptr())
    return QRows(rows, K, x.dtype, buf)


class QLinear:
    """y = x W + b in 8-bit integers: W [K][N] (any strides: pass linear.weight.t()
    for one stored [N][K]) is quantised and packed once.  W fp32 or bf16, bias [N]
    of its type; or W int8 with `scales` (fp32 [N]) and an fp32 bias."""

    def __init__(self, weight, bias=None, scales=None):
        code = _CODES.get(weight.dtype)
        if code is None or not weight.is_cuda or weight.dim() != 2:
            raise ValueError("weight: device [K][N], fp32, bf16 or int8")
        self.K, self.N = weight.shape
        self.device = weight.device
        if (code == _c.INCVIT_I8) != (scales is not None):
            raise ValueError("scales: with int8 weights, and only with them")
        for t, dt in ((bias, _F32 if code == _c.INCVIT_I8 else weight.dtype), (scales, _F32)):
            if t is not None and not (t.device == self.device and t.dtype == dt and t.is_contiguous() and t.numel() == self.N):
                raise ValueError("bias: [N] of the weights' type (fp32 with int8 weights); scales: fp32 [N]; on the weights' device")
        L = _c.lib()
        n = L.incvit_qlinear_weights_bytes(self.K, self.N) if self.K <= _MOST_K and self.N <= _MOST_N else 0
        if n == 0:
            raise _c.IncvitError(_c.INCVIT_ERR_UNSUPPORTED, f"a product of K = {self.K}, N = {self.N}")
        self.weights = _buffer(n, self.device)
        _call(L.incvit_qlinear_pack_weights, self.device, code, self.K, self.N, weight.data_ptr(), *weight.stride(), _ptr(scales),
              _ptr(bias), self.weights.data_ptr())

    def __call__(self, x, gelu: bool = False, residual=None, out=None):
        """act(x W + b) + residual for x [rows][K] (fp32 or bf16, the values of a row
        one after another) or QRows; residual and out [rows][N] of x's type (out may
        be residual, or overlap x).  Returns out."""
        q = isinstance(x, QRows)
        if q:
            code, rows, K, dev = _CODES[x.dtype], x.rows, x.K, x.buf.device
        else:
            code, rows, K = _rows_of(x)
            dev = x.device
        if K != self.K or dev != self.device:
            raise ValueError("x: rows of K values on the weights' device")
        N, dt = self.N, x.dtype
        if out is None:
            out = torch.empty(rows, N, dtype=dt, device=dev)
        elif not (out.dtype == dt and out.device == dev and out.shape == (rows, N) and (out.stride(1) == 1 or N == 1)):
            raise ValueError("out: [rows][N] of x's type, the values of a row one after another")
        r = None
        rs = 0
        if residual is not None:
            if not (residual.dtype == dt and residual.device == dev and residual.shape == (rows, N) and
                    (residual.stride(1) == 1 or N == 1)):
                raise ValueError("residual: [rows][N] of x's type, the values of a row one after another")
            r, rs = residual.data_ptr(), residual.stride(0)
        L = _c.lib()
        if q:
            _call(L.incvit_qlinear_multiply, dev, code, rows, K, N, x.buf.data_ptr(), self.weights.data_ptr(), bool(gelu), r, rs,
                  out.data_ptr(), out.stride(0))
        else:
            ws = _buffer(L.incvit_qlinear_rows_bytes(rows, K), dev)
            _call(L.incvit_qlinear, dev, code, rows, K, N, x.data_ptr(), x.stride(0), self.weights.data_ptr(), bool(gelu), r, rs,
                  out.data_ptr(), out.stride(0), ws.data_ptr())
        return out


# ------------------------------- a cache of keys and values in 8 bits --------


def _head_rows(t, who: str):
    """Checks rows of heads [rows][heads][d], the values of a head one after another; the type code."""
    code = _CODES.get(t.dtype, _c.INCVIT_I8)
    if not (t.is_cuda and code != _c.INCVIT_I8 and t.dim() == 3 and (t.stride(2) == 1 or t.shape[2] == 1)):
        raise ValueError(f"{who}: device fp32 or bf16 [rows][heads][d], the values of a head one after another")
    return code


def _indexes(t, n: int, device, who: str):
    if not (t.dtype == torch.int32 and t.device == device and t.dim() == 1 and t.shape[0] == n and t.is_contiguous()):
        raise ValueError(f"{who}: device int32 [{n}]")
    return t.data_ptr()


def _starts(t, device, who: str):
    """(address, sequences) of starts [n + 1]."""
    if not (t.dtype == torch.int32 and t.device == device and t.dim() == 1 and t.shape[0] >= 1 and t.is_contiguous()):
        raise ValueError(f"{who}: device int32 [sequences + 1]")
    return t.data_ptr(), t.shape[0] - 1


def _int32(x, who: str) -> int:
    if not 0 <= x <= 0x7fffffff:
        raise ValueError(f"{who}: in [0, 2^31)")
    return int(x)


def _attention(code: int, hq: int, hk: int, d: int, causal, window, sinks, fill, scale) -> bytes:
    if hk < 1 or hq % hk or hq < 1:
        raise ValueError("as many query heads as keys' or a multiple")
    return _ATTENTION.pack(code, hq, hk, d, bool(causal), _int32(window, "window"), _int32(sinks, "sinks"), fill,
                           d ** -0.5 if scale is None else scale)


def _output(q, out):
    if out is None:
        return torch.empty(q.shape, dtype=q.dtype, device=q.device)
    if not (out.dtype == q.dtype and out.device == q.device and out.shape == q.shape and (out.stride(2) == 1 or out.shape[2] == 1)):
        raise ValueError("out: rows of q's shape, type and device, the values of a head one after another")
    return out


def _rows(t) -> bytes:
    return _ROWS.pack(t.data_ptr(), t.stride(0), t.stride(1))


def _workspace(L, a: bytes, cached: int, n: int, rows: int, ragged: bool, max_len: int, device):
    """(tensor or None, its address) of an attention call."""
    nbytes = L.incvit_attention_workspace_bytes(a, cached, n, rows, ragged, max_len)
    if nbytes == 0:
        return None, None
    t = _buffer(nbytes, device)
    return t, t.data_ptr()


class KVCache:
    """Keys and values of `heads` heads in 8 bits, in `blocks` blocks of `block` (16,
    32, 64 or 128) tokens with a scale for each block and head; zeros at first.  The
    caller hands blocks out to sequences: slot = block number * block + place."""

    def __init__(self, blocks: int, heads: int, head_dim: int, block: int = 16, device=None):
        for x, who in ((blocks, "blocks"), (heads, "heads"), (head_dim, "head_dim"), (block, "block")):
            _int32(x, who)
        self.blocks, self.heads, self.head_dim, self.block = blocks, heads, head_dim, block
        self.config = _KV.pack(blocks, block, heads, head_dim)
        n = _c.lib().incvit_kv_bytes(self.config)
        if n == 0:
            raise _c.IncvitError(_c.INCVIT_ERR_UNSUPPORTED, f"a cache of {blocks} blocks of {block} tokens, {heads} heads of {head_dim}")
        self.buf = torch.zeros(n, dtype=torch.uint8, device="cuda" if device is None else device)
        if not self.buf.is_cuda:
            raise ValueError("device: a GPU")
        self.device = self.buf.device

    def _sides(self, k, v):
        code = _head_rows(k, "k")
        if v.dtype != k.dtype or v.shape != k.shape or v.device != k.device or _head_rows(v, "v") != code:
            raise ValueError("k and v: of one shape and type on one device")
        if k.shape[1:] != (self.heads, self.head_dim) or k.device != self.device:
            raise ValueError("k, v: [rows][heads][head_dim] on the cache's device")
        return code

    def write(self, k, v, slots, begin: bool = False):
        """Quantise new keys and values [rows][heads][d] (fp32 or bf16, any 16-byte
        aligned row and head strides) into `slots` (device int32 [rows], negative:
        nowhere; the rows of one block one after another, with any of those between).  A block keeps what it
        holds, rounded anew if its scale grows; with `begin` one whose first slot is
        written holds nothing else afterwards (a sequence that goes on into a block
        used before)."""
        code = self._sides(k, v)
        rows = k.shape[0]
        at = _indexes(slots, rows, self.device, "slots")
        _call(_c.lib().incvit_kv_write, self.device, self.config, code, rows, k.data_ptr(), k.stride(0), k.stride(1), v.data_ptr(),
              v.stride(0), v.stride(1), at, bool(begin), self.buf.data_ptr())

    def read(self, slots, dtype=_BF16, k_out=None, v_out=None):
        """(keys, values) [rows][heads][d] of `slots`, in `dtype` or in given tensors.  A
        row whose slot is outside the cache (negative) stays what it was in a given
        tensor and is zeros in a new one."""
        if (k_out is None) != (v_out is None):
            raise ValueError("k_out and v_out: both or neither")
        new = k_out is None
        if new:
            if dtype is not _BF16 and dtype is not _F32:
                raise ValueError("dtype: fp32 or bf16")
            shape = (slots.shape[0], self.heads, self.head_dim)
            k_out, v_out = torch.empty(shape, dtype=dtype, device=self.device), torch.empty(shape, dtype=dtype, device=self.device)
        code = self._sides(k_out, v_out)
        rows = k_out.shape[0]
        at = _indexes(slots, rows, self.device, "slots")
        _call(_c.lib().incvit_kv_read, self.device, self.config, self.buf.data_ptr(), code, rows, at, new, k_out.data_ptr(),
              k_out.stride(0), k_out.stride(1), v_out.data_ptr(), v_out.stride(0), v_out.stride(1))
        return k_out, v_out

    def attend(self, q, table, lens, q_start=None, causal: bool = True, window: int = 0, sinks: int = 0, scale=None, max_len: int = 0,
               out=None):
        """Attention of q [rows][q heads][d] over the cached tokens of `table` (device
        int32 [sequences][blocks of a sequence]), `lens` (device int32 [sequences]) of
        them.  A sequence's queries are its last tokens: rows q_start[i] to q_start[i +
        1] (device int32 [sequences + 1]) or rows / sequences for each.  Query at
        position p sees key j where j <= p (causal) and |p - j| < window (window 0:
        all) or j < sinks; a row that sees nothing gives zeros.  scale: 1 / sqrt(d)
        unless given.  max_len: about the longest sequence, if the table is much wider.
        Rows behind the last sequence stay what they were in a given out, and are zeros
        in a new one."""
        code = _head_rows(q, "q")
        dev = self.device
        rows, hq, d = q.shape
        if q.device != dev or d != self.head_dim:
            raise ValueError("q: [rows][heads][head_dim] on the cache's device")
        if not (table.dtype == torch.int32 and table.device == dev and table.dim() == 2 and (table.stride(1) == 1 or table.shape[1] < 2)):
            raise ValueError("table: device int32 [sequences][blocks], a sequence's blocks one after another")
        n, width = table.shape
        at = _indexes(lens, n, dev, "lens")
        starts = None
        if q_start is not None:
            starts, m = _starts(q_start, dev, "q_start")
            if m != n:
                raise ValueError("q_start: device int32 [sequences + 1]")
        a = _attention(code, hq, self.heads, d, causal, window, sinks, out is None, scale)
        new, out = out is None, _output(q, out)
        if rows == 0 or n == 0:
            return out.zero_() if new else out
        most = max_len or width * self.block
        L = _c.lib()
        ws, wp = _workspace(L, a, 1, n, rows, starts is not None, most, dev)
        _call(L.incvit_kv_attend, dev, a, self.config, self.buf.data_ptr(), n, rows, starts, table.data_ptr(), table.stride(0), width, at,
              most, _rows(q), _rows(out), wp)
        return out


# ---------------------------------------------------------------- attention --


def attend(q, k, v, q_start=None, k_start=None, causal: bool = True, window: int = 0, sinks: int = 0, scale=None, max_len: int = 0,
           out=None):
    """Attention of q [rows][q heads][d] over keys and values [key rows][heads][d]
    (fp32 or bf16, any 16-byte aligned row and head strides), sequences one after
    another: q_start and k_start (device int32 [sequences + 1]), or one sequence.
    Masks, positions and what is returned as KVCache.attend's."""
    code = _head_rows(q, "q")
    dev = q.device
    rows, hq, d = q.shape
    for t, who in ((k, "k"), (v, "v")):
        if _head_rows(t, who) != code or t.device != dev or t.shape != k.shape or t.shape[2] != d:
            raise ValueError("k and v: of one shape, of q's type, head_dim and device")
    if (q_start is None) != (k_start is None):
        raise ValueError("q_start and k_start: both or neither")
    qs = ks = None
    n = 1
    if q_start is not None:
        (qs, n), (ks, m) = _starts(q_start, dev, "q_start"), _starts(k_start, dev, "k_start")
        if m != n:
            raise ValueError("q_start and k_start: device int32 [sequences + 1]")
    a = _attention(code, hq, k.shape[1], d, causal, window, sinks, out is None, scale)
    new, out = out is None, _output(q, out)
    if rows == 0 or n == 0:
        return out.zero_() if new else out
    keys = k.shape[0]
    most = max_len or -(-keys // n)
    L = _c.lib()
    ws, wp = _workspace(L, a, 0, n, rows, qs is not None, most, dev)
    _call(L.incvit_attend, dev, a, n, rows, qs, keys, ks, most, _rows(q), _rows(k), _rows(v), _rows(out), wp)
    return out
