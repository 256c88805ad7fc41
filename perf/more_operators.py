"""Calls of the library's cache of keys and values in 8 bits and of its attention, as cases that can be timed and compared.

Four operators, which a decoder or an encoder of long streams has behind the head norms and their rotation:

* `store`: new keys and values quantised as they are written into the blocks of a cache, with a scale for each block of
  tokens and head, and the tokens of the written sequences read back;
* `cached`: attention of new queries over the keys and values held in that cache, through a table of each sequence's blocks;
* `window`: attention of packed sequences over keys and values in their own type.

Both attentions are causal or not, over all keys or over a sliding window with a few first tokens that stay visible.

With `own` the calls go to the library; without it the same mathematics runs in elementary torch operations.
"""
import math
import random

import torch

own = False

MOST_BYTES = 1.4e8                            # drawn cases stay below what the largest listed ones move
MOST_FLOPS = {"bf16": 2.7e11, "f32": 1.7e10}  # and compute (fp32 products run at a sixteenth of bf16's rate)


def _store(name, lens, new, heads, head, dtype, *, block=16, append=True, packed=False):
    c = dict(op="store", lens=lens, new=new, heads=heads, head=head, dtype=dtype, block=block, append=append, packed=packed)
    return dict(c, name=name) if name else c


def _cached(name, lens, new, hq, hk, head, dtype, *, block=16, causal=True, window=0, sinks=0):
    c = dict(op="cached", lens=lens, new=new, hq=hq, hk=hk, head=head, dtype=dtype, block=block, causal=causal, window=window,
             sinks=sinks)
    return dict(c, name=name) if name else c


def _window(name, lens, new, hq, hk, head, dtype, *, causal=True, window=0, sinks=0, packed=False):
    c = dict(op="window", lens=lens, new=new, hq=hq, hk=hk, head=head, dtype=dtype, causal=causal, window=window, sinks=sinks,
             packed=packed)
    return dict(c, name=name) if name else c


def _text(values):
    return ",".join(str(v) for v in values)


def _spread(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def listed():
    rng = random.Random(5)
    ragged = _text(_spread(rng, 200, 16384) for _ in range(31)) + ",16384"  # a server's batch: many short, a few long
    return [
        # the newest token of one stream: latency alone
        _store("store_token", "39", "1", 4, 128, "bf16"),
        # the headline's step: 23 refreshed tokens of a frame's 256, whose blocks keep the other tokens
        _store("store_step", "256", "23", 16, 72, "bf16", append=False),
        # 32 streams of 256 tokens, whole frames, keys and values inside the projection's output
        _store("store_vitl_x32", _text([256] * 32), "256", 16, 64, "bf16", packed=True),
        # odd frames in fp32 that go on in the middle of a block
        _store("store_odd_f32", "300,273,41", "273,100,7", 12, 80, "f32", block=32),
        # a single stream's next token over a short past: latency
        _cached("cached_token", "777", "1", 16, 4, 128, "bf16"),
        # a server's batch, a token of each sequence: the bytes of the caches
        _cached("cached_batch", ragged, "1", 16, 4, 128, "bf16"),
        # long streams with a window and their first tokens, a few tokens at once, odd sizes, fp32
        _cached("cached_stream_f32", "20011,9973,4099,1201,77", "3", 12, 12, 80, "f32", block=64, window=4000, sinks=4),
        # the next 1024 tokens of a long prompt over its past
        _cached("cached_chunk", "8192", "1024", 16, 4, 128, "bf16", block=32),
        # 448x448 frames: every token sees its own frame, the projection's output in place
        _window("window_frames", _text([1024] * 8), "", 16, 16, 72, "bf16", causal=False, packed=True),
        # a prompt through a layer with a sliding window and first tokens
        _window("window_prompt", "8192", "", 16, 4, 128, "bf16", window=1024, sinks=16),
        # a prompt through a layer that sees everything: the largest
        _window("window_full", "8192", "", 16, 4, 128, "bf16"),
        # odd frames in fp32, a window to both sides
        _window("window_odd_f32", "273,273,546,1,130", "", 12, 12, 80, "f32", causal=False, window=100, sinks=1),
    ]


def draw(rng):
    """A case of the same ranges: lengths from one token on, odd and even sizes, every option."""
    while True:
        op = rng.choice(["store", "cached", "cached", "window", "window"])
        dtype = rng.choice(["bf16", "bf16", "f32"])
        head = rng.choice([32, 40, 64, 64, 72, 80, 96, 128, 128, 192, 256])
        hk = rng.choice([1, 2, 3, 4, 8, 12, 16])
        hq = hk * rng.choice([1, 1, 2, 3, 4, 8])
        block = rng.choice([16, 16, 32, 64, 128])
        n = _spread(rng, 1, 40)
        kw = dict(causal=rng.random() < 0.7)
        if rng.random() < 0.5:
            kw.update(window=_spread(rng, 1, 5000), sinks=rng.choice([0, 1, 4, 16, 100]))
        if op == "store":
            lens = [_spread(rng, 1, 10000) for _ in range(n)]
            most = rng.choice([1, 4, 10000])
            new = [rng.randint(1, min(m, most)) for m in lens]
            case = _store("", _text(lens), _text(new), hk, head, dtype, block=block, append=rng.random() < 0.6,
                          packed=rng.random() < 0.4)
        elif op == "cached":
            lens = [_spread(rng, 1, 30000) for _ in range(n)]
            most = rng.choice([1, 1, 5, 2000])
            new = [rng.randint(1, min(m, most)) for m in lens]
            case = _cached("", _text(lens), _text(new), hq, hk, head, dtype, block=block, **kw)
        else:
            lens = [_spread(rng, 1, 10000) for _ in range(n)]
            most = rng.choice([1, 100000, 100000])  # the newest token's query alone, or every token's
            new = [min(m, most) for m in lens]
            case = _window("", _text(lens), _text(new), hq, hk, head, dtype, packed=most > 1 and rng.random() < 0.5, **kw)
        w = work(case)
        if w["bytes"] <= MOST_BYTES and w["flops"] <= MOST_FLOPS[dtype]:
            return case


# ---------------------------------------------------------------- inputs --


def _gen(seed, what):
    return torch.Generator(device="cuda").manual_seed((int(seed) * 1000003 + what * 7919 + 31) % (1 << 62))


def _dt(case):
    return torch.bfloat16 if case["dtype"] == "bf16" else torch.float32


def _lens(case):
    """([keys of each sequence], [new tokens of each])."""
    lens = [int(x) for x in case["lens"].split(",")]
    new = [int(x) for x in case["new"].split(",")] if case["new"] else lens
    return lens, new * len(lens) if len(new) == 1 else new


def _starts(lens):
    out = [0]
    for m in lens:
        out.append(out[-1] + m)
    return out


def _blocks(case):
    """(table [sequences][widest] on the host, blocks of the pool)."""
    lens, B = _lens(case)[0], case["block"]
    need = [-(-m // B) for m in lens]
    order = list(range(sum(need) + 3))
    random.Random(sum(need)).shuffle(order)  # blocks as a pool hands them out
    table, at = [], 0
    for k in need:
        table.append(order[at:at + k] + [-1] * (max(need) - k))
        at += k
    return table, len(order)


def _slots(case, table):
    """Slots in the pool of every token of every sequence, one list for each."""
    B = case["block"]
    return [[table[i][t // B] * B + t % B for t in range(m)] for i, m in enumerate(_lens(case)[0])]


def _values(rows, heads, head, dt, g, channels):
    """Tokens of different sizes, and for keys channels of different sizes, as projections give them."""
    x = torch.empty((rows, heads, head), device="cuda").normal_(0.0, 1.0, generator=g)
    x *= torch.rand((rows, 1, 1), device="cuda", generator=g) + 0.5
    if channels:
        x *= 0.5 + 2.5 * torch.rand((1, heads, head), device="cuda", generator=g) ** 4
    return x.to(dt)


class State:
    """Inputs, the cache that a program keeps, and what its tables say."""


def _inputs(case, seed):
    """What the call is given, the same for both sides."""
    s = State()
    s.case = case
    g, dt = _gen(seed, 1), _dt(case)
    lens, new = _lens(case)
    d, rows = case["head"], sum(new)
    i32 = dict(dtype=torch.int32, device="cuda")
    s.q_start = torch.tensor(_starts(new), **i32)
    if case["op"] != "window":
        table, s.blocks = _blocks(case)
        slots = _slots(case, table)
        s.table, s.lens = torch.tensor(table, **i32), torch.tensor(lens, **i32)
    if case["op"] == "store":
        h = case["heads"]
        pick = random.Random(seed)
        past, fresh = [], []  # what the cache holds before, and the slots of the new rows
        for sl, m, n in zip(slots, lens, new):
            past += sl[:m - n] if case["append"] else sl
            fresh += sl[m - n:] if case["append"] else [sl[t] for t in sorted(pick.sample(range(m), n))]
        s.past, s.slots = torch.tensor(past, **i32), torch.tensor(fresh, **i32)
        s.all = torch.tensor([x for sl in slots for x in sl], **i32)
        s.k0, s.v0 = _values(len(past), h, d, dt, g, True), _values(len(past), h, d, dt, g, False)
        if case["packed"]:  # views of a projection's output [rows][q | k | v]
            x = torch.empty((rows, 3 * h * d), dtype=dt, device="cuda")
            s.k, s.v = x[:, h * d:2 * h * d].unflatten(1, (h, d)), x[:, 2 * h * d:].unflatten(1, (h, d))
            s.k.copy_(_values(rows, h, d, dt, g, True))
            s.v.copy_(_values(rows, h, d, dt, g, False))
        else:
            s.k, s.v = _values(rows, h, d, dt, g, True), _values(rows, h, d, dt, g, False)
        return s
    hq, hk = case["hq"], case["hk"]
    if case["op"] == "cached":
        s.q = _values(rows, hq, d, dt, g, False)
        s.past = torch.tensor([x for sl in slots for x in sl], **i32)
        s.k0, s.v0 = _values(len(s.past), hk, d, dt, g, True), _values(len(s.past), hk, d, dt, g, False)
        return s
    s.k_start = torch.tensor(_starts(lens), **i32)
    if case["packed"]:
        x = torch.empty((rows, (hq + 2 * hk) * d), dtype=dt, device="cuda")
        s.q, s.k, s.v = (y.unflatten(1, (-1, d)) for y in x.split([hq * d, hk * d, hk * d], dim=1))
        for t, ch in ((s.q, False), (s.k, True), (s.v, False)):
            t.copy_(_values(rows, t.shape[1], d, dt, g, ch))
    else:
        s.q = _values(rows, hq, d, dt, g, False)
        s.k, s.v = _values(sum(lens), hk, d, dt, g, True), _values(sum(lens), hk, d, dt, g, False)
    return s


def prepare(case, seed):
    s = _inputs(case, seed)
    if case["op"] == "window":
        return s
    h = case["heads"] if case["op"] == "store" else case["hk"]
    if own:
        from paper_2607_12287_amd import incvit
        s.cache = incvit.KVCache(s.blocks, h, case["head"], block=case["block"])
        s.cache.write(s.k0, s.v0, s.past, begin=True)
    else:
        s.held = [_Held(s.blocks, case["block"], h, case["head"]) for _ in range(2)]
        for held, x in zip(s.held, (s.k0, s.v0)):
            held.write(x, s.past.long(), True)
    return s


# ------------------------------------------------------------------- run --


class _Held:
    """Keys or values in 8 bits: whole numbers [blocks][tokens][heads][head] and scales [blocks][heads]."""

    def __init__(self, blocks, block, heads, head):
        self.q = torch.zeros((blocks, block, heads, head), dtype=torch.int8, device="cuda")
        self.s = torch.zeros((blocks, heads), device="cuda")

    def write(self, x, slots, begin):
        """A block's scale is the larger of the one it has and max|x| / 127 of its new rows; what it keeps is rounded anew.
        With `begin` a block whose first slot is written keeps nothing, and so does one whose slots are all written."""
        n, B = self.q.shape[:2]
        x, b = x.float(), slots // B
        named = torch.zeros((n * B,), dtype=torch.bool, device="cuda")
        named[slots] = True
        named = named.view(n, B)
        hit = named.any(1)
        anew = named.all(1) | (named[:, 0] & hit if begin else torch.zeros_like(hit))
        top = torch.zeros_like(self.s).index_reduce_(0, b, x.abs().amax(-1), "amax", include_self=True)
        fresh = (top.double() / 127.0).float()  # one rounding
        old = torch.where(anew[:, None], torch.zeros_like(self.s), self.s)
        s = torch.where(hit[:, None], torch.maximum(old, fresh), self.s)
        ratio = torch.where(s > 0, (old.double() / s.double()).float(), torch.zeros_like(s))  # 1 where the scale stays
        change = hit[:, None] & ((ratio != 1) | anew[:, None])
        kept = (self.q.float() * ratio[:, None, :, None]).round().to(torch.int8)
        self.q = torch.where(change[:, None, :, None], kept, self.q)
        sx = s[b].double()[..., None]
        q = (x.double() / sx).float().round().clamp_(-127.0, 127.0)  # a quotient next to a border: 64 bits
        q = torch.where(sx > 0, q, torch.zeros_like(q))
        self.q.view(n * B, *self.q.shape[2:])[slots] = q.to(torch.int8)
        self.s = s

    def read(self, slots):
        B = self.q.shape[1]
        return self.q.view(-1, *self.q.shape[2:])[slots].float() * self.s[slots // B][..., None]


def run(s):
    return _run_own(s) if own else _run_plain(s)


def _run_own(s):
    c = s.case
    if c["op"] == "store":
        s.cache.write(s.k, s.v, s.slots, begin=c["append"])
        return s.cache.read(s.all, dtype=s.k.dtype)
    kw = dict(causal=c["causal"], window=c["window"], sinks=c["sinks"])
    lens, new = _lens(c)
    if c["op"] == "cached":
        return s.cache.attend(s.q, s.table, s.lens, q_start=s.q_start if min(new) != max(new) else None, **kw)
    from paper_2607_12287_amd import incvit
    many = len(lens) > 1
    return incvit.attend(s.q, s.k, s.v, q_start=s.q_start if many else None, k_start=s.k_start if many else None, **kw)


def _visible(case, nq, nk, dev="cuda"):
    """[queries][keys]: what each of a sequence's last nq tokens sees of its nk keys."""
    p = torch.arange(nk - nq, nk, device=dev)[:, None]
    j = torch.arange(nk, device=dev)[None, :]
    see = (j <= p) if case["causal"] else torch.ones((nq, nk), dtype=torch.bool, device=dev)
    if case["window"]:
        see = see & (((p - j).abs() < case["window"]) | (j < case["sinks"]))
    return see


def _attention(case, q, k, v):
    """[nq][hq][d] over [nk][hk][d] in fp32; a query that sees nothing gives zeros."""
    nq, hq, d = q.shape
    nk, hk = k.shape[:2]
    rows = q.view(nq, hk, hq // hk, d).permute(1, 2, 0, 3).reshape(hk, -1, d)
    x = (rows @ k.permute(1, 2, 0).contiguous()).view(hk, hq // hk, nq, nk) * (1.0 / math.sqrt(d))
    x = x.masked_fill_(~_visible(case, nq, nk), -math.inf)
    top = x.amax(-1, keepdim=True)
    p = (x - torch.where(top == -math.inf, torch.zeros_like(top), top)).exp_()
    total = p.sum(-1, keepdim=True)
    o = p.view(hk, -1, nk) @ v.permute(1, 0, 2).contiguous()
    o = o / torch.where(total == 0, torch.ones_like(total), total).view(hk, -1, 1)
    return o.view(hk, hq // hk, nq, d).permute(2, 0, 1, 3).reshape(nq, hq, d)


def _run_plain(s):
    c = s.case
    lens, new = _lens(c)
    if c["op"] == "store":
        for held, x in zip(s.held, (s.k, s.v)):
            held.write(x, s.slots.long(), c["append"])
        return tuple(held.read(s.all.long()).to(s.k.dtype) for held in s.held)
    qs, ks = _starts(new), _starts(lens)
    out = torch.empty_like(s.q, memory_format=torch.contiguous_format)
    if c["op"] == "cached":
        B = c["block"]
        for i, m in enumerate(lens):
            at = s.table[i, :-(-m // B)].long()
            at = (at[:, None] * B + torch.arange(B, device="cuda")).flatten()[:m]
            out[qs[i]:qs[i + 1]] = _attention(c, s.q[qs[i]:qs[i + 1]].float(), s.held[0].read(at), s.held[1].read(at))
        return out
    for i in range(len(lens)):
        out[qs[i]:qs[i + 1]] = _attention(c, s.q[qs[i]:qs[i + 1]].float(), s.k[ks[i]:ks[i + 1]].float(), s.v[ks[i]:ks[i + 1]].float())
    return out


# ------------------------------------------------------------------ work --


def _seen(case):
    """(query and key pairs, keys that some query sees) of all sequences."""
    pairs = keys = 0
    w = case["window"]
    for nk, nq in zip(*_lens(case)):
        first = nk - nq
        for p in range(first, nk):
            hi = p + 1 if case["causal"] else (min(nk, p + w) if w else nk)
            lo = max(0, p - w + 1) if w else 0
            pairs += hi - lo + (min(lo, case["sinks"]) if w else 0)
        keys += nk - max(0, first - w + 1) + min(max(0, first - w + 1), case["sinks"]) if w else nk
    return pairs, keys


def work(case):
    e = 2.0 if case["dtype"] == "bf16" else 4.0
    lens, new = _lens(case)
    d, rows = case["head"], sum(new)
    if case["op"] == "store":
        n = 2.0 * case["heads"] * d  # keys and values of a token
        scales = 8.0 * case["heads"] / case["block"]
        return {"bytes": rows * (n * (e + 1.0) + 4.0 + scales) + sum(lens) * (n * (e + 1.0) + 4.0 + scales), "flops": 4.0 * n * (rows + sum(lens))}
    pairs, keys = _seen(case)
    io = 2.0 * rows * case["hq"] * d * e
    n = 2.0 * case["hk"] * d
    if case["op"] == "cached":
        past = keys * (n + 8.0 * case["hk"] / case["block"] + 4.0 / case["block"])
    else:
        past = keys * n * e
    return {"bytes": io + past, "flops": 4.0 * pairs * case["hq"] * d}


# ----------------------------------------------------------------- exact --


def _exact_store(x0, past, x, slots, case, blocks):
    """Values of the pool's slots [blocks * tokens][heads][head] after both writes, in 64 bits but for the scales and quotients,
    which are fp32 by definition."""
    B = case["block"]
    q = torch.zeros((blocks * B,) + x.shape[1:], dtype=torch.float64, device="cuda")
    s = torch.zeros((blocks, x.shape[1]), dtype=torch.float64, device="cuda")
    for rows, at, begin in ((x0, past, True), (x, slots, case["append"])):
        if not len(at):
            continue
        rows, at = rows.double(), at.long()
        order = torch.argsort(at)
        b, count = torch.unique_consecutive(at[order] // B, return_counts=True)
        most = int(count.max())
        ends = torch.cumsum(count, 0)
        place = (ends - count)[:, None] + torch.arange(most, device="cuda").clamp(max=most)
        there = place < ends[:, None]
        place = order[torch.where(there, place, torch.zeros_like(place))]  # [blocks hit][most] rows
        top = torch.where(there[..., None], rows.abs().amax(-1)[place], 0.0).amax(1)
        first = ((at[place] % B == 0) & there).any(1) if begin else torch.zeros_like(count, dtype=torch.bool)
        old = torch.where((first | (count == B))[:, None], 0.0, s[b])
        scale = torch.maximum(old, (top / 127.0).float().double())
        shrink = torch.where(scale > 0, old / scale.clamp_min(1e-300), 0.0).float().double()
        whole = q.view(blocks, B, *x.shape[1:])
        whole[b] = torch.round((whole[b] * shrink[:, None, :, None]).float().double())
        s[b] = scale
        sc = s[at // B][..., None]
        q[at] = torch.where(sc > 0, torch.round((rows / sc.clamp_min(1e-300)).float().double()).clamp(-127.0, 127.0), 0.0)
    return (q.view(blocks, B, *x.shape[1:]) * s[:, None, :, None]).view_as(q)


def exact(case, seed):
    s = _inputs(case, seed)
    if case["op"] == "store":
        k, v = (_exact_store(x0, s.past, x, s.slots, case, s.blocks) for x0, x in ((s.k0, s.k), (s.v0, s.v)))
        return k[s.all.long()], v[s.all.long()]
    if case["op"] == "cached":
        at = s.past.long()
        none = s.past[:0]
        k, v = (_exact_store(x, s.past, x[:0], none, dict(case, append=True), s.blocks)[at] for x in (s.k0, s.v0))
    else:
        k, v = s.k.double(), s.v.double()
    lens, new = _lens(case)
    qs, ks = _starts(new), _starts(lens)
    group = case["hq"] // case["hk"]
    out = torch.zeros(s.q.shape, dtype=torch.float64, device="cuda")
    for i, (nk, nq) in enumerate(zip(lens, new)):
        pos = nk - nq + torch.arange(nq, device="cuda")
        key = torch.arange(nk, device="cuda")
        gap = pos[:, None] - key
        see = torch.ones_like(gap, dtype=torch.bool)
        if case["causal"]:
            see &= gap >= 0
        if case["window"]:
            see &= (gap.abs() < case["window"]) | (key < case["sinks"])[None, :]
        for h in range(case["hq"]):
            x = s.q[qs[i]:qs[i + 1], h].double() @ k[ks[i]:ks[i + 1], h // group].t().contiguous() / math.sqrt(case["head"])
            x = torch.where(see, x, torch.full_like(x, -math.inf))
            p = torch.softmax(x, dim=-1).nan_to_num(0.0)
            out[qs[i]:qs[i + 1], h] = p @ v[ks[i]:ks[i + 1], h // group].contiguous()
    return out
