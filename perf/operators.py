"""The operators that take several new tokens of a sequence at once, for timing them and comparing their results.

A program that serves a model over the quantised KV cache of this library meets more than single tokens: prompts in
chunks, drafts of a few tokens to verify, batches in which some sequences bring one token and others hundreds.  Three
operators carry that work:

* ``rotate``: rotary positions of queries and keys, in a projection's output as it lies there, with one to three axes;
* ``append``: new keys and values join the cache (windows, quantised store, pages), the keys rotated on the way, every
  sequence with its own number of tokens if need be;
* ``attend``: the queries of several new tokens attend to the cached tokens, as the cache holds them, and causally to
  the new ones.

``listed()`` names twelve pieces of such work and ``draw(rng)`` gives more of the same ranges; ``prepare`` makes what the
program holds before the call, ``run`` makes the call once: in elementary torch operations, or, with ``own`` set, through
the library.

An append moves the cache on.  ``run`` takes the counts back, so that a pass can be repeated; a second pass then finds
the first one's tokens in the ring of recent tokens.  Packed codes are compared as the bytes they are: whole numbers,
defined to the last bit by the 32-bit operations that form them.
"""
from __future__ import annotations

import math

import torch

own = False

D = 128
SINK = 4
PAGE = 64
SYM, ASYM, HYBRID = 0, 1, 2

# Cost bounds of a drawn case, those of the largest listed ones: scores of an attention (queries x keys over all query
# heads), cached (sequence, kv head, token) units, (sequence, head, token) rows of a rotation or an append.
MOST_SCORES = 32 * 2048 * (32768 + 2048)
MOST_UNITS = 8 * 8 * 32768
MOST_ROTATED = 40 * 32768
MOST_APPENDED = 4 * 8 * 32768


def _case(name, op, batch, q_heads, kv_heads, cached, new, **more):
    c = dict(op=op, batch=batch, q_heads=q_heads, kv_heads=kv_heads, cached=cached, new=new, ragged=False, paged=False,
             bits=2, v_bits=0, group=32, recent=128, k_mode=HYBRID, v_mode=HYBRID, heavy=True, norm=False,
             rot_dim=D, interleaved=False, axes=1)
    c.update(more)
    if name is not None:
        c = dict(name=name, **c)
    return c


def listed():
    return [
        # Queries and keys of one decode step of eight sequences, out of the fused projection's output: latency.
        _case("rotate_step", "rotate", 8, 32, 8, 4000, 1),
        # Two image prompts: positions with a time, a height and a width axis, an odd number of tokens.
        _case("rotate_three_axes_4099", "rotate", 2, 32, 8, 0, 4099, axes=3),
        # A long prompt of a model that rotates half of the channels, in adjacent pairs.
        _case("rotate_prompt_32k_partial", "rotate", 1, 32, 8, 0, 32768, rot_dim=64, interleaved=True),
        # Continuous batching, one token of each of 32 sequences, counts on the device, paged store, 4 bits.
        _case("append_step_ragged", "append", 32, 32, 8, 8000, 1, ragged=True, paged=True, bits=4),
        # A chunk of a long prompt of a multi-head layer, keys divided by the key-norm factors on their way, 4 bits.
        _case("append_chunk_512", "append", 1, 32, 32, 4097, 512, bits=4, norm=True),
        # First prompts of 17 to 2048 tokens in one batch, three axes, paged store, wide groups.
        _case("append_prompts_ragged", "append", 16, 32, 8, 0, 2048, ragged=True, paged=True, group=64, axes=3),
        # Long prompts, 2-bit codes: all bytes and hardly any latency.
        _case("append_prompt_32k", "append", 4, 32, 8, 0, 32768),
        # A draft of four tokens over a short conversation at 4 bits: latency.
        _case("attend_draft_4_of_500", "attend", 1, 32, 8, 500, 4, bits=4),
        # Drafts of five tokens over a batch of long contexts: the cache's bytes count.
        _case("attend_draft_5_of_32k", "attend", 8, 32, 8, 32763, 5),
        # A mixed batch: sequences that bring one token beside chunks of up to 256, over 1k to 16k, paged store, 4 bits.
        _case("attend_mixed_ragged", "attend", 16, 32, 8, 16000, 256, ragged=True, paged=True, bits=4),
        # A chunk of a long prompt, 4 bits: matrix products.
        _case("attend_chunk_2048_of_32k", "attend", 1, 32, 8, 32768, 2048, bits=4, group=64),
        # A first prompt of a multi-head layer: nothing cached yet, causal attention among the new tokens alone.
        _case("attend_first_prompt_4k", "attend", 1, 32, 32, 0, 4096, bits=4),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    """One more case of the listed ranges."""
    op = rng.choice(["rotate", "append", "append", "attend", "attend", "attend"])
    kv_heads = rng.choice([1, 2, 4, 8, 8, 8, 16, 32])
    q_heads = kv_heads * rng.choice([1, 2, 3, 4, 4, 4, 5, 8])
    batch = _log_int(rng, 1, 32)
    bits, v_bits, k_mode, v_mode = rng.choice([
        (2, 0, HYBRID, HYBRID), (2, 0, SYM, HYBRID), (4, 0, HYBRID, HYBRID), (4, 0, HYBRID, HYBRID), (4, 0, SYM, ASYM),
        (3, 0, SYM, SYM), (3, 2, SYM, HYBRID), (4, 2, HYBRID, HYBRID)])
    more = dict(bits=bits, v_bits=v_bits, k_mode=k_mode, v_mode=v_mode, group=rng.choice([32, 32, 64]),
                recent=rng.choice([32, 100, 128, 128]), heavy=rng.random() < 0.7, ragged=rng.random() < 0.4,
                paged=rng.random() < 0.5, norm=op == "append" and rng.random() < 0.3, axes=rng.choice([1, 1, 3]),
                interleaved=rng.random() < 0.3, rot_dim=rng.choice([D, D, D, 96, 64]))
    cached = 0 if rng.random() < 0.2 else None
    if op == "rotate":
        new = _log_int(rng, 1, max(1, min(32768, MOST_ROTATED // (batch * (q_heads + kv_heads)))))
        return _case(None, op, batch, q_heads, kv_heads, cached or 1000, new, **more)
    if op == "append":
        new = _log_int(rng, 1, max(1, min(32768, MOST_APPENDED // (batch * kv_heads))))
        if cached is None:
            cached = _log_int(rng, 100, 8000)
        return _case(None, op, batch, q_heads, kv_heads, cached, new, **more)
    if cached is None:
        cached = _log_int(rng, 300, max(301, min(32768, MOST_UNITS // (batch * kv_heads))))
    most = MOST_SCORES // (batch * q_heads)
    new = _log_int(rng, 1, max(1, min(4096, int((math.sqrt(cached ** 2 + 4.0 * most) - cached) / 2))))
    return _case(None, op, batch, q_heads, kv_heads, cached, new, **more)


# ------------------------------------------------------------------------------------------------ inputs


def _bits(c, which):
    return c["v_bits"] if which == 1 and c["v_bits"] else c["bits"]


def _mode(c, which):
    return c["v_mode"] if which == 1 else c["k_mode"]


def _slots(c, which):
    return c["recent"] + (c["group"] if which == 1 else 1)


def _quantised(c, which, n):
    """Rows of the store of keys (0) or values (1) when n tokens (a number or a tensor) are cached."""
    mid = n - SINK - c["recent"]
    mid = max(0, mid) if isinstance(mid, int) else mid.clamp_min(0)
    return mid - mid % c["group"] if which == 1 else mid


def _spread(least, most, count):
    return [int(round(most * (least / most) ** ((count - 1 - i) / max(1, count - 1)))) for i in range(count)]


def _counts(c):
    """Cached and new tokens of every sequence of the batch."""
    B, n, t = c["batch"], c["cached"], c["new"]
    if not c["ragged"]:
        return [n] * B, [t] * B
    ns = [0] * B if n == 0 else _spread(max(1, n // 16), n, B)
    least = max(1, t // 128)
    ts = _spread(least, t, B)
    turn = B // 2 + 1                       # (neither count goes with the other)
    return ns, [ts[(i * 5 + turn) % B] for i in range(B)] if math.gcd(5, B) == 1 else ts[turn:] + ts[:turn]


def _axis_of_pair(c):
    """The axis whose position turns each pair: three sections of about a quarter, three and three eighths."""
    pairs = c["rot_dim"] // 2
    if c["axes"] == 1:
        return [0] * pairs
    first = pairs // 4
    second = (pairs - first) // 2
    return [0] * first + [1] * second + [2] * (pairs - first - second)


class _Random:
    def __init__(self, seed):
        self.gen = torch.Generator(device="cuda")
        self.gen.manual_seed(1000003 * (seed % (1 << 40)) + 29)

    def normal(self, *shape):
        return torch.randn(shape, generator=self.gen, device="cuda")

    def half(self, *shape):
        out = torch.empty(shape, dtype=torch.float16, device="cuda")
        for part in out:                    # (a large draw in pieces)
            part.copy_(torch.randn(part.shape, generator=self.gen, device="cuda"))
        return out

    def integers(self, low, high, shape):
        return torch.randint(low, high, shape, generator=self.gen, device="cuda", dtype=torch.int32)


def _rotation_inputs(c, r):
    """fp32 cosine and sine tables and the tokens' positions (int32 [axes][B][new])."""
    B, T = c["batch"], c["new"]
    ns, _ = _counts(c)
    rows = max(ns) + T + 16
    turn = 10000.0 ** (-torch.arange(0, c["rot_dim"], 2, device="cuda", dtype=torch.float64) / c["rot_dim"])
    angle = torch.arange(rows, device="cuda", dtype=torch.float64)[:, None] * turn
    start = torch.tensor(ns, dtype=torch.int32, device="cuda")
    along = start[:, None] + torch.arange(T, dtype=torch.int32, device="cuda")
    if c["axes"] == 1:
        positions = along[None].contiguous()
    else:                                   # patches of a picture: one time, rows and columns of a grid
        wide = max(1, int(math.sqrt(T)))
        i = torch.arange(T, dtype=torch.int32, device="cuda").expand(B, T)
        positions = torch.stack([start[:, None].expand(B, T), i // wide + start[:, None], i % wide + start[:, None]]).contiguous()
        positions += r.integers(0, 8, (3, B, 1))
    return dict(cos=angle.cos().float().contiguous(), sin=angle.sin().float().contiguous(), positions=positions)


def _key_spread(c, r):
    """Standard deviation of every key channel: 1, or 1 + |Student-t with 3 degrees of freedom|."""
    H = c["kv_heads"]
    if not c["heavy"]:
        return torch.ones(H, D, device="cuda")
    z = r.normal(4, H, D)
    return 1.0 + (z[0] / ((z[1] ** 2 + z[2] ** 2 + z[3] ** 2) / 3.0).sqrt()).abs()


def _projection(c, r, sigma):
    """The fused projection's output [B][new][q heads, keys, values][D] and its three parts as [B][heads][new][D]."""
    hq, hk = c["q_heads"], c["kv_heads"]
    x = r.half(c["batch"], c["new"], hq + 2 * hk, D)
    x[:, :, hq:hq + hk] *= sigma.half()
    parts = x.transpose(1, 2)
    return parts[:, :hq], parts[:, hq:hq + hk], parts[:, hq + hk:], parts[:, :hq + hk]


def _fields(x, bits, mode):
    """Fields, scales and zero-points of fp16 groups [G, M], a group a column, every 32-bit operation rounded on its own."""
    x = x.float()
    top, half = (1 << bits) - 1, 1 << (bits - 1)
    low, high = x.amin(0), x.amax(0)
    over = lambda a, d: (a / torch.full_like(a, float(d))).half()  # noqa: E731  (a true division)
    sa, ss = over(high - low, top), over(torch.maximum(low.abs(), high.abs()), half - 1)
    quotient = lambda a, s: torch.where(s == 0, 0.0, a / torch.where(s == 0, 1.0, s))  # noqa: E731
    ca = quotient(x - low, sa.float()).round_().clamp_(0, top)
    cs = quotient(x, ss.float()).round_().clamp_(-half, half - 1)
    if mode == HYBRID:
        da = (x - (sa.float() * ca + low)).abs()
        ds = (x - ss.float() * cs).abs()
        ea, es = torch.zeros_like(low), torch.zeros_like(low)
        for i in range(x.shape[0]):         # the definition's sum: one value after the other
            ea += da[i]
            es += ds[i]
        asym = ea < es
    else:
        asym = torch.full_like(low, mode == ASYM, dtype=torch.bool)
    fields = torch.where(asym, ca, cs + half).to(torch.uint8)
    return fields, torch.where(asym, -sa, ss), torch.where(asym, low.half(), torch.zeros_like(sa))


def _packed(f, bits):
    """uint8 fields [..., L] as bytes [..., L * bits / 8], the first field lowest."""
    if bits == 3:                           # the low two bits of all fields, then the high ones
        return torch.cat([_packed(f & 3, 2), _packed(f >> 2, 1)], dim=-1)
    per = 8 // bits
    f = f.view(*f.shape[:-1], f.shape[-1] // per, per)
    return (f << torch.arange(0, 8, bits, dtype=torch.uint8, device=f.device)).sum(-1, dtype=torch.uint8)


def _key_rows(c, x):
    """Rows fp16 [M, D] of keys as packed rows: groups of channels inside a row."""
    G, M = c["group"], x.shape[0]
    f, s, z = _fields(x.view(M * (D // G), G).T, _bits(c, 0), _mode(c, 0))
    return _packed(f.T.reshape(M, D), _bits(c, 0)), s.view(M, D // G), z.view(M, D // G)


def _value_groups(c, x):
    """Token groups fp16 [M, G, D] of values as packed groups: G tokens of a channel."""
    G, M = c["group"], x.shape[0]
    f, s, z = _fields(x.permute(1, 0, 2).reshape(G, M * D), _bits(c, 1), _mode(c, 1))
    return _packed(f.view(G, M, D).permute(1, 2, 0).contiguous(), _bits(c, 1)), s.view(M, D), z.view(M, D)


def _store_rows(s, b, h, row):
    """Where row `row` of sequence b's kv head h lies in the store buffers, in rows."""
    c = s["case"]
    if not c["paged"]:
        return (b * c["kv_heads"] + h) * s["capacity"] + row
    return (s["page_table"].long()[b, row // PAGE] * c["kv_heads"] + h) * PAGE + row % PAGE


def _empty_cache(s):
    """Zeroed buffers of the cache in the layout of the library, and a page table whose pages lie anywhere."""
    c = s["case"]
    B, H, G = c["batch"], c["kv_heads"], c["group"]
    ns, ts = _counts(c)
    s["capacity"] = -(-(max(n + t for n, t in zip(ns, ts)) + 2) // PAGE) * PAGE
    rows = B * H * s["capacity"]
    s["pages"] = 0
    if c["paged"]:
        blocks = [-(-(n + t + 1) // PAGE) for n, t in zip(ns, ts)]
        s["pages"] = sum(blocks) + 5
        ids = torch.randperm(s["pages"], generator=s["random"].gen, device="cuda").to(torch.int32)
        table = torch.zeros(B, s["capacity"] // PAGE, dtype=torch.int32, device="cuda")
        at = 0
        for b, n in enumerate(blocks):
            table[b, :n] = ids[at:at + n]
            at += n
        s["page_table"] = table
        rows = s["pages"] * H * PAGE
    zeros = lambda *shape, **kw: torch.zeros(shape, device="cuda", **kw)  # noqa: E731
    half = dict(dtype=torch.float16)
    buf = {
        "k_codes": zeros(rows, D * _bits(c, 0) // 8, dtype=torch.uint8),
        "k_scales": zeros(rows, D // G, **half),
        "k_zeros": zeros(rows, D // G, **half) if c["k_mode"] != SYM else None,
        "v_codes": zeros(rows // G, D, G * _bits(c, 1) // 8, dtype=torch.uint8),
        "v_scales": zeros(rows // G, D, **half),
        "v_zeros": zeros(rows // G, D, **half) if c["v_mode"] != SYM else None,
        "k_sink": zeros(B, H, SINK, D, **half), "v_sink": zeros(B, H, SINK, D, **half),
        "k_recent": zeros(B, H, _slots(c, 0), D, **half), "v_recent": zeros(B, H, _slots(c, 1), D, **half),
    }
    s["buffers"] = buf


def _fill_cache(s, sigma):
    """The cache of tokens drawn at random, sequence by sequence: windows, and the rest packed."""
    c, r, buf = s["case"], s["random"], s["buffers"]
    H, G = c["kv_heads"], c["group"]
    heads = torch.arange(H, device="cuda")[:, None]
    for b, n in enumerate(_counts(c)[0]):
        if n == 0:
            continue
        k, v = (r.normal(H, n, D) * sigma[:, None]).half(), r.normal(H, n, D).half()
        for which, x, name in ((0, k, "k"), (1, v, "v")):
            m = min(n, SINK)
            buf[name + "_sink"][b, :, :m] = x[:, :m]
            nq = _quantised(c, which, n)
            live = torch.arange(min(n, SINK) + nq, n, device="cuda")
            buf[name + "_recent"][b, :, live % _slots(c, which)] = x[:, live]
            if nq == 0:
                continue
            rows = x[:, SINK:SINK + nq]
            if which == 0:
                at = _store_rows(s, b, heads, torch.arange(nq, device="cuda")[None]).view(-1)
                packed = _key_rows(c, rows.reshape(-1, D))
            else:
                at = _store_rows(s, b, heads, torch.arange(0, nq, G, device="cuda")[None]).view(-1) // G
                packed = _value_groups(c, rows.reshape(-1, G, D))
            for part, p in zip(("_codes", "_scales", "_zeros"), packed):
                if buf[name + part] is not None:
                    buf[name + part][at] = p


def prepare(case, seed):
    c = dict(case)
    s = dict(case=c, random=_Random(seed))
    r = s["random"]
    if c["op"] in ("rotate", "append"):
        s.update(_rotation_inputs(c, r))
    sigma = _key_spread(c, r)
    s["q"], s["k"], s["v"], s["qk"] = _projection(c, r, sigma)
    if c["op"] == "rotate":
        s["out"] = torch.empty(c["batch"], c["new"], c["q_heads"] + c["kv_heads"], D, dtype=torch.float16, device="cuda").transpose(1, 2)
        return s
    s["inv"] = (0.5 + torch.rand(c["kv_heads"], D, generator=r.gen, device="cuda")).contiguous() if c["norm"] else None
    ns, ts = _counts(c)
    s["cached"] = torch.tensor(ns, dtype=torch.int32, device="cuda")
    s["new"] = torch.tensor(ts, dtype=torch.int32, device="cuda")
    s["most"] = max(n + t for n, t in zip(ns, ts))
    s["counts"] = s["cached"].clone()
    _empty_cache(s)
    _fill_cache(s, sigma)
    if c["op"] == "attend":
        s["out"] = torch.zeros(c["batch"], c["new"], c["q_heads"], D, dtype=torch.float16, device="cuda").transpose(1, 2)
    return s


# ------------------------------------------------------------------------------------------------ the plain forms


def _angles(s):
    """Cosine and sine of every token's pairs, [B, 1, T, pairs]."""
    c = s["case"]
    axis = torch.tensor(_axis_of_pair(c), device="cuda")
    p = s["positions"].long().clamp(0, s["cos"].shape[0] - 1)[axis]                   # [pairs, B, T]
    pair = torch.arange(len(axis), device="cuda")[:, None, None]
    return s["cos"][p, pair].permute(1, 2, 0)[:, None], s["sin"][p, pair].permute(1, 2, 0)[:, None]


def _pairs(c, x):
    """The two halves of every pair as views of x [..., D]."""
    n = c["rot_dim"]
    return (x[..., 0:n:2], x[..., 1:n:2]) if c["interleaved"] else (x[..., :n // 2], x[..., n // 2:n])


def _rotated(s, x):
    c = s["case"]
    cos, sin = _angles(s)
    a, b = _pairs(c, x.float())
    y = x.clone()
    first, second = _pairs(c, y)
    first.copy_(a * cos - b * sin)
    second.copy_(b * cos + a * sin)
    return y


def _append(s):
    """The rows that leave the windows are packed into the store, the new ones that stay join the windows."""
    c, buf = s["case"], s["buffers"]
    G, H, T = c["group"], c["kv_heads"], c["new"]
    k = _rotated(s, s["k"])
    if s["inv"] is not None:
        k = (k.float() * s["inv"][None, :, None]).half()
    n, t = s["cached"].long(), s["new"].long()
    # the store of a ragged batch is left one step ahead of the cache
    ahead = (n + t + (1 if c["ragged"] else 0)).clamp_max(s["capacity"])
    heads = torch.arange(H, device="cuda")
    writes = []
    for which, x, name in ((0, k, "k"), (1, s["v"], "v")):
        ring, sink, slots = buf[name + "_recent"], buf[name + "_sink"], _slots(c, which)
        first, end = _quantised(c, which, n), _quantised(c, which, ahead)
        step = G if which == 1 else 1
        i = torch.arange(0, T + 2 + (G if which == 1 else 0), step, device="cuda")
        row = first[:, None] + i
        b, j = torch.nonzero(row < end[:, None], as_tuple=True)
        row = row[b, j]
        token = (SINK + row)[:, None] + torch.arange(step, device="cuda")             # [M, step]
        seq = b[:, None].expand_as(token)
        fresh = (token >= n[seq])[:, None, :, None]
        at = seq[:, None], heads[None, :, None]
        old = ring[at[0], at[1], (token % slots)[:, None]]                            # [M, H, step, D]
        new = x[at[0], at[1], (token - n[seq]).clamp(0, T - 1)[:, None]]
        rows = torch.where(fresh, new, old)
        packed = _key_rows(c, rows.view(-1, D)) if which == 0 else _value_groups(c, rows.view(-1, G, D))
        where = _store_rows(s, b[:, None], heads, row[:, None]).view(-1)
        writes.append((name, which, where // step, packed))
        stays = SINK + _quantised(c, which, n + t)
        token = n[:, None] + torch.arange(T, device="cuda")
        is_new = torch.arange(T, device="cuda") < t[:, None]
        for b, j, dst, m in ((*torch.nonzero(is_new & (token < SINK), as_tuple=True), sink, SINK),
                             (*torch.nonzero(is_new & (token >= torch.maximum(stays, torch.full_like(stays, SINK))[:, None]), as_tuple=True), ring, slots)):
            dst[b, :, token[b, j] % m] = x[b, :, j]
    for name, which, where, packed in writes:
        for part, p in zip(("_codes", "_scales", "_zeros"), packed):
            if buf[name + part] is not None:
                buf[name + part][where] = p
    s["counts"].copy_(s["cached"] + s["new"])


def _unpacked(codes, bits):
    if bits == 3:
        n = codes.shape[-1] // 3
        return _unpacked(codes[..., :2 * n], 2) | _unpacked(codes[..., 2 * n:], 1) << 2
    shift = torch.arange(0, 8, bits, dtype=torch.uint8, device=codes.device)
    return ((codes[..., None] >> shift) & ((1 << bits) - 1)).flatten(-2)


def _decoded(c, buf, name, which):
    """fp32 values of the whole store: rows [R, D]."""
    bits, G = _bits(c, which), c["group"]
    scale = buf[name + "_scales"]
    low = torch.where(torch.signbit(scale), buf[name + "_zeros"].float(), scale.float() * -(1 << (bits - 1))) if buf[name + "_zeros"] is not None \
        else scale.float() * -(1 << (bits - 1))
    f = _unpacked(buf[name + "_codes"], bits).float()
    if which == 0:
        f = f.view(-1, D // G, G)
        return (scale.float().abs()[..., None] * f + low[..., None]).view(-1, D)
    return (scale.float().abs()[..., None] * f + low[..., None]).transpose(1, 2).reshape(-1, D)


def _all_tokens(s, which):
    """fp32 [B, H, tokens, D]: the cached tokens as the cache holds them, then the new ones, every sequence from 0 on."""
    c, buf = s["case"], s["buffers"]
    name, B, H = "kv"[which], c["batch"], c["kv_heads"]
    n = s["cached"].long()
    j = torch.arange(s["most"], device="cuda")
    x = _decoded(c, buf, name, which)
    b, h = torch.arange(B, device="cuda")[:, None, None], torch.arange(H, device="cuda")[None, :, None]
    row = (j - SINK).clamp_min(0).expand(B, 1, -1)
    x = x[_store_rows(s, b, h, row)]                                                  # [B, H, tokens, D]
    x[:, :, :SINK] = buf[name + "_sink"][:, :, :s["most"]]
    recent = j >= (SINK + _quantised(c, which, n))[:, None]                           # [B, tokens]
    x = torch.where(recent[:, None, :, None], buf[name + "_recent"][:, :, j % _slots(c, which)].float(), x)
    sink = (j < SINK)[None, None, :, None]
    x = torch.where(sink, torch.nn.functional.pad(buf[name + "_sink"].float(), (0, 0, 0, max(0, s["most"] - SINK)))[:, :, :s["most"]], x)
    i = (j - n[:, None]).clamp(0, c["new"] - 1)                                       # [B, tokens]
    fresh = s["kv"[which]][b, h, i[:, None]].float()
    return torch.where((j >= n[:, None])[:, None, :, None], fresh, x)


def _attend(s):
    c = s["case"]
    B, H, T, r = c["batch"], c["kv_heads"], c["new"], c["q_heads"] // c["kv_heads"]
    k, v = _all_tokens(s, 0), _all_tokens(s, 1)
    q = s["q"].float().reshape(B, H, r * T, D)
    score = torch.matmul(q, k.transpose(2, 3).contiguous()).mul_(1.0 / math.sqrt(D)).view(B, H, r, T, -1)
    i, j = torch.arange(T, device="cuda"), torch.arange(s["most"], device="cuda")
    hidden = j[None, None] > (s["cached"].long()[:, None] + i)[:, :, None]            # [B, T, tokens]
    score.masked_fill_(hidden[:, None, None], -math.inf)
    score -= score.amax(-1, keepdim=True)
    score.exp_()
    total = score.sum(-1, keepdim=True)
    out = torch.matmul(score.view(B, H, r * T, -1), v).view(B, H, r, T, D).div_(total).reshape(B, H * r, T, D)
    rows = (i < s["new"][:, None])[:, None, :, None]
    s["out"].copy_(torch.where(rows, out.half(), s["out"]))


def _library(s):
    """What a program keeps of the library: the cache over its buffers, the rotation's tables, a workspace."""
    if "iq" not in s:
        from paper_2602_23200_amd import binding as iq
        c = s["case"]
        s["iq"] = iq
        if "cos" in s:
            s["rotation"] = iq.make_rotation(s["cos"], s["sin"], interleaved=c["interleaved"], pair_axis=_axis_of_pair(c))
        s["config"] = iq.make_config(c["batch"], c["q_heads"], c["kv_heads"], D, c["bits"], c["group"], SINK, c["recent"], c["k_mode"],
                                     c["v_mode"], 0, iq.KIND_INNER, s.get("capacity", PAGE), c["v_bits"], 0, s.get("pages", 0))
        if c["op"] != "rotate":
            handle = iq.innerq_cache_t()
            for name, t in s["buffers"].items():
                setattr(handle, name, None if t is None else t.data_ptr())
            if c["paged"]:
                handle.page_table = s["page_table"].data_ptr()
            handle.n_tokens = handle.store_ahead_tokens = 0 if c["ragged"] else c["cached"]
            s["cache"] = iq.Cache(s["config"], s["buffers"], handle)
        if c["op"] == "attend":
            s["workspace"] = iq.allocate_chunk_workspace(s["config"], c["new"])
    return s["iq"]


def run(s):
    c = s["case"]
    if c["op"] == "rotate":
        if own:
            iq = _library(s)
            iq.innerq_rotate(s["config"], s["rotation"], s["qk"], out=s["out"], positions=s["positions"])
        else:
            s["out"].copy_(_rotated(s, s["qk"]))
        return {"out": s["out"]}
    if c["op"] == "append":
        if own:
            iq = _library(s)
            if c["ragged"]:
                s["counts"].copy_(s["cached"])              # the scheduler's lengths; the call advances them
                iq.innerq_append_rotated_ragged(s["cache"], s["counts"], s["new"], s["k"], s["v"], s["rotation"],
                                                positions=s["positions"], k_inv_norm=s["inv"])
            else:
                s["cache"].c.n_tokens = s["cache"].c.store_ahead_tokens = c["cached"]
                iq.innerq_append_rotated(s["cache"], s["k"], s["v"], s["rotation"], positions=s["positions"], k_inv_norm=s["inv"])
        else:
            _append(s)
        kept = {name: t for name, t in s["buffers"].items() if t is not None}
        return {**kept, "counts": s["counts"]} if c["ragged"] else kept
    if own:
        iq = _library(s)
        if c["ragged"]:
            iq.innerq_chunk_attention_ragged(s["cache"], s["cached"], s["new"], s["most"], s["k"], s["v"], s["q"], s["workspace"], out=s["out"])
        else:
            iq.innerq_chunk_attention(s["cache"], s["k"], s["v"], s["q"], s["workspace"], out=s["out"])
    else:
        _attend(s)
    return {"out": s["out"]}


# ------------------------------------------------------------------------------------------------ the least work


def _row_bytes(c, which):
    """Bytes of one quantised (token, kv head): codes, scales, zero-points."""
    return D * _bits(c, which) / 8 + D / c["group"] * (2 if _mode(c, which) == SYM else 4)


def work(case):
    c = case
    ns, ts = _counts(c)
    tables = 4.0 * c["rot_dim"] * c["batch"] * c["new"] + 4.0 * c["axes"] * c["batch"] * c["new"]
    if c["op"] == "rotate":
        rows = c["batch"] * (c["q_heads"] + c["kv_heads"]) * c["new"]
        return {"bytes": rows * D * 4.0 + tables, "flops": rows * c["rot_dim"] * 3.0}
    total, flops = 0.0, 0.0
    if c["op"] == "append":
        total += tables
        for n, t in zip(ns, ts):
            for which in (0, 1):
                gone = _quantised(c, which, n + t) - _quantised(c, which, n)
                old = max(0, min(n, SINK + _quantised(c, which, n + t)) - SINK - _quantised(c, which, n))
                new_gone = gone - old
                rows = t * D * 2 + old * D * 2 + gone * _row_bytes(c, which) + (t - new_gone) * D * 2
                total += c["kv_heads"] * rows
                flops += c["kv_heads"] * D * (gone * (16 if _mode(c, which) == HYBRID else 8) + (t * 3 if which == 0 else 0))
        return {"bytes": total, "flops": flops}
    for n, t in zip(ns, ts):
        for which in (0, 1):
            nq = _quantised(c, which, n)
            total += c["kv_heads"] * (nq * _row_bytes(c, which) + (n - nq + t) * D * 2)
        total += c["q_heads"] * t * D * 4
        flops += 4.0 * c["q_heads"] * D * (t * n + t * (t + 1) / 2)
    return {"bytes": total, "flops": flops}


# ------------------------------------------------------------------------------------------------ the definition, in 64 bits


def _turned(s, x, b):
    """Heads x [H, T, D] of sequence b, rotated in 64 bits."""
    c, n = s["case"], s["case"]["rot_dim"]
    y = x.double().clone()
    place = s["positions"][:, b].long().clamp(0, s["cos"].shape[0] - 1)
    for i, a in enumerate(_axis_of_pair(c)):
        lo, hi = (2 * i, 2 * i + 1) if c["interleaved"] else (i, i + n // 2)
        z = torch.complex(y[:, :, lo], y[:, :, hi]) * torch.complex(s["cos"][place[a], i].double(), s["sin"][place[a], i].double())
        y[:, :, lo], y[:, :, hi] = z.real, z.imag
    return y


def _group_exact(x, bits, mode):
    """Scale and zero-point, in 64 bits, of groups along the last dimension of fp16 values."""
    x = x.double()
    lo, hi = x.min(-1).values, x.max(-1).values
    levels, half = 2 ** bits - 1, 2 ** (bits - 1)
    wide, even = (hi - lo) / levels, torch.max(lo.abs(), hi.abs()) / (half - 1)
    if mode == SYM:
        return even, torch.zeros_like(lo)
    if mode == HYBRID:
        w, e = wide.half().double()[..., None], even.half().double()[..., None]
        m = lo[..., None]
        ca = torch.nan_to_num((x - m) / w).round().clamp(0, levels)
        cs = torch.nan_to_num(x / e).round().clamp(-half, half - 1)
        asym = (x - m - w * ca).abs().sum(-1) < (x - e * cs).abs().sum(-1)
        return torch.where(asym, -wide, even), torch.where(asym, lo, torch.zeros_like(lo))
    return -wide, lo


def _append_exact(s):
    c, G, H = s["case"], s["case"]["group"], s["case"]["kv_heads"]
    got = {k: (None if v is None or v.dtype == torch.uint8 else v.double()) for k, v in s["buffers"].items()}
    for b, (n, t) in enumerate(zip(*_counts(c))):
        k = _turned(s, s["k"][b, :, :, :], b)
        kept = k.half()
        if s["inv"] is not None:
            kept = (kept.double() * s["inv"].double()[:, None]).half()
            k = k * s["inv"].double()[:, None]
        for which, exact, x, name in ((0, k, kept, "k"), (1, s["v"][b].double(), s["v"][b], "v")):
            slots, ring = _slots(c, which), s["buffers"][name + "_recent"][b]
            r0, r1 = _quantised(c, which, n), _quantised(c, which, min(s["capacity"], n + t + (1 if c["ragged"] else 0)))
            if r1 > r0:
                old = [ring[:, u % slots] for u in range(SINK + r0, min(n, SINK + r1))]
                rows = x[:, max(0, SINK + r0 - n):max(0, SINK + r1 - n)]
                rows = torch.cat([torch.stack(old, 1), rows], 1) if old else rows
                for h in range(H):
                    at = _store_rows(s, torch.tensor(b, device="cuda"), h, torch.arange(r0, r1, device="cuda"))
                    if which == 0:
                        sc, z = _group_exact(rows[h].view(r1 - r0, D // G, G), _bits(c, 0), c["k_mode"])
                    else:
                        at = at[::G] // G
                        sc, z = _group_exact(rows[h].view(-1, G, D).transpose(1, 2), _bits(c, 1), c["v_mode"])
                    got[name + "_scales"][at] = sc
                    if got[name + "_zeros"] is not None:
                        got[name + "_zeros"][at] = z
            stays = SINK + _quantised(c, which, n + t)
            for u in range(n, min(n + t, SINK)):
                got[name + "_sink"][b, :, u] = exact[:, u - n]
            first = max(n, stays, SINK)
            if first < n + t:
                u = torch.arange(first, n + t, device="cuda")
                got[name + "_recent"][b, :, u % slots] = exact[:, u - n]
    kept = {name: got[name] for name in s["buffers"] if s["buffers"][name] is not None}
    return {**kept, "counts": None} if c["ragged"] else kept


def _values(s, which, b, h, n):
    """The n cached tokens of one kv head as the cache holds them, in 64 bits."""
    c, G, name = s["case"], s["case"]["group"], "kv"[which]
    buf, bits = s["buffers"], _bits(s["case"], which)
    nq = _quantised(c, which, n)
    parts = [buf[name + "_sink"][b, h, :min(n, SINK)].double()]
    if nq:
        at = _store_rows(s, torch.tensor(b, device="cuda"), h, torch.arange(0, nq, G if which else 1, device="cuda")) // (G if which else 1)
        byte, sc = buf[name + "_codes"][at].long(), buf[name + "_scales"][at].double()
        length = byte.shape[-1] * 8 // bits
        i = torch.arange(length, device="cuda")
        if bits == 3:
            code = (byte[..., i // 4] >> (i % 4 * 2) & 3) + 4 * (byte[..., length // 4 + i // 8] >> i % 8 & 1)
        else:
            code = byte[..., i * bits // 8] >> (i * bits % 8) & (2 ** bits - 1)
        asym = torch.signbit(sc)
        zero = buf[name + "_zeros"][at].double() if buf[name + "_zeros"] is not None else torch.zeros_like(sc)
        code = code.double().view(*sc.shape, G)
        x = sc.abs()[..., None] * (code - torch.where(asym, 0.0, 2.0 ** (bits - 1))[..., None]) + torch.where(asym, zero, torch.zeros_like(zero))[..., None]
        parts.append(x.transpose(1, 2).reshape(nq, D) if which else x.reshape(nq, D))
    if n > SINK + nq:
        parts.append(buf[name + "_recent"][b, h, torch.arange(SINK + nq, n, device="cuda") % _slots(c, which)].double())
    return torch.cat(parts)


def exact(case, seed):
    s = prepare(case, seed)
    c = s["case"]
    if c["op"] == "rotate":
        return {"out": torch.stack([_turned(s, s["qk"][b], b) for b in range(c["batch"])])}
    if c["op"] == "append":
        return _append_exact(s)
    r = c["q_heads"] // c["kv_heads"]
    out = s["out"].double()
    for b, (n, t) in enumerate(zip(*_counts(c))):
        later = torch.arange(n + t, device="cuda") > n + torch.arange(t, device="cuda")[:, None]
        for h in range(c["kv_heads"]):
            k, v = (torch.cat([_values(s, w, b, h, n), s["kv"[w]][b, h, :t].double()]) for w in (0, 1))
            for g in range(h * r, (h + 1) * r):
                a = s["q"][b, g, :t].double() @ k.T / math.sqrt(D)
                out[b, g, :t] = torch.softmax(a.masked_fill(later, -math.inf), -1) @ v
    return {"out": out}
