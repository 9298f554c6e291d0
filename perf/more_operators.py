"""The operators around a KV cache held in 8 bits with a scale for each block of tokens and head, for timing them and comparing
their results.

A program that serves a model beside the 2- to 4-bit caches of this library has layers, and whole models, that do not bear them:
their keys and values stay in 8 bits (integers, or floating point with three bits of mantissa), 32 or 64 tokens of a head to a
scale.  Four operators carry such a cache:

* ``write``: new keys and values join it.  Tokens of a block that is not complete yet wait in fp16 (its "open" rows); a block is
  packed when its last token arrives, so the cache does not depend on how the tokens came;
* ``read``: tokens come back as fp16 rows (a context that moves to another place, or into another kind of cache);
* ``attend``: the queries of one or several new tokens attend to the cached tokens and causally to the new ones;
* ``cross``: queries of a decoder attend to all tokens of an encoder's states, which the cache holds: another length for every
  sequence, none for some.

``listed()`` names twelve pieces of such work and ``draw(rng)`` gives more of the same ranges; ``prepare`` makes what the
program holds before the call, ``run`` makes the call once: in elementary torch operations, or, with ``own`` set, through
the library.

A write moves the cache on.  ``run`` takes the counts back, so that a pass can be repeated; a second pass then finds the first
one's tokens in the open rows.  Packed values are compared as what they are, in units of their block's scale: the stored integer or
floating-point number, which 32-bit operations define to the last bit.
"""
from __future__ import annotations

import math

import torch

own = False

D = 128
PAGE = 64

# Cost bounds of a drawn case, those of the largest listed ones: scores of an attention (queries x keys over all query heads),
# cached (sequence, kv head, token) units that an attention reads, and those that a write or a read moves.
MOST_SCORES = 32 * 2048 * (32768 + 2048)
MOST_UNITS = 8 * 8 * 32768
MOST_MOVED = 4 * 8 * 32768


def _case(name, op, batch, q_heads, kv_heads, cached, new, **more):
    c = dict(op=op, batch=batch, q_heads=q_heads, kv_heads=kv_heads, cached=cached, new=new, ragged=False, paged=False,
             e4m3=False, block=32, heavy=True)
    c.update(more)
    if name is not None:
        c = dict(name=name, **c)
    return c


def listed():
    return [
        # Continuous batching: one token of each of 32 sequences, counts on the device, paged store: latency.
        _case("write_step_ragged", "write", 32, 32, 8, 8000, 1, ragged=True, paged=True, e4m3=True),
        # First prompts of 16 to 2048 tokens in one batch, paged store, wide blocks.
        _case("write_prompts_ragged", "write", 16, 32, 8, 0, 2048, ragged=True, paged=True, block=64),
        # Long prompts: all bytes and hardly any latency.
        _case("write_prompt_32k", "write", 4, 32, 8, 0, 32768, e4m3=True),
        # The newest 257 tokens of a batch of conversations, which end inside a block, out of the paged store.
        _case("read_newest_257_ragged", "read", 8, 32, 8, 8000, 257, ragged=True, paged=True, e4m3=True, block=64),
        # Long contexts as a whole.
        _case("read_context_32k", "read", 4, 32, 8, 32765, 32765),
        # One token behind a short conversation: latency.
        _case("attend_step_500", "attend", 1, 32, 8, 500, 1, e4m3=True),
        # One token of each of eight long contexts: the cache's bytes.
        _case("attend_step_32k", "attend", 8, 32, 8, 32763, 1),
        # Drafts of five tokens over the same contexts, floating point, wide blocks.
        _case("attend_draft_5_of_32k", "attend", 8, 32, 8, 32763, 5, e4m3=True, block=64),
        # A mixed batch: sequences that bring one token beside chunks of up to 256, over 1k to 16k, paged store.
        _case("attend_mixed_ragged", "attend", 16, 32, 8, 16000, 256, ragged=True, paged=True, e4m3=True),
        # A chunk of a long prompt: matrix products.
        _case("attend_chunk_2048_of_32k", "attend", 1, 32, 8, 32768, 2048, block=64),
        # One decoder token of 32 requests over encoder states of 90 to 1437 tokens, one request without any: every head its own keys.
        _case("cross_step_ragged", "cross", 32, 16, 16, 1437, 1, ragged=True, heavy=False),
        # A decoder's prompt of 300 tokens over the states of 4099.
        _case("cross_prompt_300_of_4099", "cross", 4, 32, 8, 4099, 300, paged=True, e4m3=True, heavy=False),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    """One more case of the listed ranges."""
    op = rng.choice(["write", "write", "read", "attend", "attend", "attend", "cross"])
    kv_heads = rng.choice([1, 2, 4, 8, 8, 8, 16, 32])
    q_heads = kv_heads * rng.choice([1, 2, 3, 4, 4, 4, 5, 8])
    batch = _log_int(rng, 1, 32)
    more = dict(e4m3=rng.random() < 0.5, block=rng.choice([32, 32, 64]), heavy=rng.random() < 0.6,
                ragged=rng.random() < 0.4, paged=rng.random() < 0.5)
    if op == "write":
        cached = 0 if rng.random() < 0.3 else _log_int(rng, 1, 8000)
        new = _log_int(rng, 1, max(1, min(32768, MOST_MOVED // (batch * kv_heads))))
        return _case(None, op, batch, q_heads, kv_heads, cached, new, **more)
    if op == "read":
        new = _log_int(rng, 1, max(1, min(32768, MOST_MOVED // (batch * kv_heads))))
        return _case(None, op, batch, q_heads, kv_heads, new + rng.choice([0, 1, 31, 500]), new, **more)
    if op == "attend" and rng.random() < 0.2:
        cached = 0
    else:
        cached = _log_int(rng, 1 if rng.random() < 0.2 else 300, max(301, min(32768, MOST_UNITS // (batch * kv_heads))))
    most = MOST_SCORES // (batch * q_heads)
    if op == "attend":
        new = int((math.sqrt(cached ** 2 + 4.0 * most) - cached) / 2)
    else:
        new = most // cached
    return _case(None, op, batch, q_heads, kv_heads, cached, _log_int(rng, 1, max(1, min(4096, new))), **more)


# ------------------------------------------------------------------------------------------------ inputs


def _spread(least, most, count):
    """`count` numbers from `least` to `most`, each the same multiple of the one before."""
    return [int(round(most * (least / most) ** ((count - 1 - i) / max(1, count - 1)))) for i in range(count)]


def _counts(c):
    """Cached tokens, and rows that come (write, attend, cross) or go (read), of every sequence of the batch."""
    B, n, t = c["batch"], c["cached"], c["new"]
    if not c["ragged"]:
        return [n] * B, [t] * B
    ns = [0] * B if n == 0 else _spread(max(1, n // 16), n, B)
    if c["op"] == "read":
        return ns, [min(t, x) for x in ns]
    if c["op"] == "cross" and B > 2:
        ns[1] = 0                           # (a request that has no encoder states)
    ts = _spread(max(1, t // 128), t, B)
    turn = B // 2 + 1                       # (neither count goes with the other)
    return ns, [ts[(i * 7 + turn) % B] for i in range(B)] if B % 7 else ts[turn:] + ts[:turn]


class _Random:
    def __init__(self, seed):
        self.gen = torch.Generator(device="cuda")
        self.gen.manual_seed(999983 * (seed % (1 << 40)) + 17)

    def normal(self, *shape):
        return torch.randn(shape, generator=self.gen, device="cuda")

    def half(self, *shape):
        out = torch.empty(shape, dtype=torch.float16, device="cuda")
        for part in out:                    # (a large draw in pieces)
            part.copy_(torch.randn(part.shape, generator=self.gen, device="cuda"))
        return out


def _key_spread(c, r):
    """Standard deviation of every key channel: 1, or 1 + |Student-t with 3 degrees of freedom|."""
    H = c["kv_heads"]
    if not c["heavy"]:
        return torch.ones(H, D, device="cuda")
    z = r.normal(4, H, D)
    return 1.0 + (z[0] / ((z[1] ** 2 + z[2] ** 2 + z[3] ** 2) / 3.0).sqrt()).abs()


def _code_type(c):
    return torch.float8_e4m3fn if c["e4m3"] else torch.int8


def _packed(c, x):
    """Blocks fp16 [M, block, D] as codes of the same shape and fp32 scales [M]; every 32-bit operation rounded on its own."""
    x = x.float()
    most = x.abs().amax((1, 2))
    scale = most / torch.full_like(most, 448.0 if c["e4m3"] else 127.0)
    y = torch.where(scale[:, None, None] == 0, 0.0, x / torch.where(scale == 0, 1.0, scale)[:, None, None])
    return (y if c["e4m3"] else y.round_()).to(_code_type(c)), scale


def _empty_store(s, r):
    """The store in the order of its tokens: codes [P, H, S, D] and scales [P, H, S / block], P sequences of S tokens or P pages of 64."""
    c = s["case"]
    B, H = c["batch"], c["kv_heads"]
    ns, ts = _counts(c)
    grow = c["op"] == "write"
    most = max(n + (t if grow else 0) for n, t in zip(ns, ts))
    if c["op"] == "attend":
        most = max(n + t for n, t in zip(ns, ts))
    s["capacity"] = max(1, -(-most // PAGE)) * PAGE
    P, S = B, s["capacity"]
    if c["paged"]:
        need = [-(-(n + (t if grow else 0)) // PAGE) for n, t in zip(ns, ts)]
        P, S = sum(need) + 5, PAGE
        ids = torch.randperm(P, generator=r.gen, device="cuda").to(torch.int32)
        table = torch.zeros(B, s["capacity"] // PAGE, dtype=torch.int32, device="cuda")
        at = 0
        for b, m in enumerate(need):
            table[b, :m] = ids[at:at + m]
            at += m
        s["page_table"] = table
    s["places"] = (P, S)
    s["store"] = {w: (torch.zeros(P, H, S, D, dtype=torch.int8, device="cuda").view(_code_type(c)),
                      torch.zeros(P, H, S // c["block"], device="cuda")) for w in "kv"}
    s["open"] = {w: torch.zeros(B, H, c["block"], D, dtype=torch.float16, device="cuda") for w in "kv"}


def _put(s, w, b, first, codes, scales):
    """Packed blocks [H, m, block, D] of sequence b, from token `first` on, into the store."""
    c = s["case"]
    H, m, G = codes.shape[0], codes.shape[1], c["block"]
    to, scale_to = s["store"][w]
    to = to.view(torch.int8)
    codes = codes.view(torch.int8)
    if not c["paged"]:
        to[b, :, first:first + m * G] = codes.reshape(H, m * G, D)
        scale_to[b, :, first // G:first // G + m] = scales
        return
    token = first + G * torch.arange(m, device="cuda")
    page, row = s["page_table"][b].long()[token // PAGE], token % PAGE
    to.view(to.shape[0], H, PAGE // G, G, D)[page, :, row // G] = codes.transpose(0, 1)
    scale_to[page, :, row // G] = scales.T


def _fill(s, r, sigma):
    """The cache of tokens drawn at random, sequence by sequence."""
    c, G = s["case"], s["case"]["block"]
    for b, n in enumerate(_counts(c)[0]):
        if n == 0:
            continue
        for w, spread in (("k", sigma), ("v", None)):
            x = r.normal(c["kv_heads"], n, D)
            x = (x if spread is None else x * spread[:, None]).half()
            m = n // G
            if m:
                codes, scales = _packed(c, x[:, :m * G].reshape(-1, G, D))
                _put(s, w, b, 0, codes.view(-1, m, G, D), scales.view(-1, m))
            s["open"][w][b, :, :n - m * G] = x[:, m * G:]


# The library's order of the bytes of 32 tokens and how its axes are those of the order above: axes of a key byte are token = 16 a + c,
# channel = 32 g + 16 h + e, of a value byte channel = 32 q + 2 c + m, token = 16 i + 4 g + j.

def _key_axes(x, P, H, S):
    """[P, H, S, D] as [P, H, tiles, a, c, g, h, e]."""
    return x.view(P, H, S // 32, 2, 16, 4, 2, 16)


def _value_axes(x, P, H, S):
    """[P, H, S, D] as [P, H, tiles, i, g, j, q, c, m]."""
    return x.view(P, H, S // 32, 2, 4, 4, 4, 16, 2)


def _library_axes(s, buffers):
    """The library's code buffers as views with those axes."""
    c, (P, S) = s["case"], s["places"]
    H, kind = c["kv_heads"], _code_type(c)
    k = buffers["k_codes"].view(kind).view(P, H, S // 32, 2, 2, 4, 16, 16).permute(0, 1, 2, 3, 6, 5, 4, 7)
    v = buffers["v_codes"].view(kind).view(P, H, S // 32, 4, 4, 16, 2, 2, 4).permute(0, 1, 2, 7, 4, 8, 3, 5, 6)
    return k, v


def _library_cache(s):
    """The same cache as the library's."""
    from paper_2602_23200_amd import binding as iq
    c, (P, S) = s["case"], s["places"]
    H = c["kv_heads"]
    cfg = iq.make_block_config(c["batch"], c["q_heads"], H, D, type=iq.E4M3 if c["e4m3"] else iq.INT8, block=c["block"],
                               capacity_tokens=s["capacity"], page_pool_pages=P if c["paged"] else 0)
    cache = iq.allocate_block_cache(cfg, page_table=s.get("page_table"))
    for w, axes, view in zip("kv", (_key_axes, _value_axes), _library_axes(s, cache.buffers)):
        codes, scales = s["store"][w]
        view.view(torch.int8).copy_(axes(codes.view(torch.int8), P, H, S))
        cache.buffers[w + "_scales"].view(torch.float32).view(scales.shape).copy_(scales)
        cache.buffers[w + "_open"].view(torch.float16).view(s["open"][w].shape).copy_(s["open"][w])
    cache.c.n_tokens = c["cached"]
    s["cache"], s["store"], s["open"] = cache, None, None
    if c["op"] in ("attend", "cross"):
        s["workspace"] = iq.allocate_block_workspace(cfg, c["new"])


def _inputs(case, seed):
    """Everything that the program holds, the cache in the order of its tokens."""
    c = dict(case)
    s, r = dict(case=c), _Random(seed)
    B, hq, hk, T = c["batch"], c["q_heads"], c["kv_heads"], c["new"]
    ns, ts = _counts(c)
    sigma = _key_spread(c, r)
    if c["op"] in ("write", "attend"):      # the output of a fused projection, [B, T, heads, D], and its parts as [B, heads, T, D]
        x = r.half(B, T, hq + 2 * hk, D)
        x[:, :, hq:hq + hk] *= sigma.half()
        x = x.transpose(1, 2)
        s["q"], s["k"], s["v"] = x[:, :hq], x[:, hq:hq + hk], x[:, hq + hk:]
    elif c["op"] == "cross":
        s["q"] = r.half(B, T, hq, D).transpose(1, 2)
    _empty_store(s, r)
    _fill(s, r, sigma)
    s["cached"] = torch.tensor(ns, dtype=torch.int32, device="cuda")
    s["new"] = torch.tensor(ts, dtype=torch.int32, device="cuda")
    s["counts"] = s["cached"].clone()
    s["first"] = s["cached"] - s["new"]
    s["most"] = max(n + (t if c["op"] == "attend" else 0) for n, t in zip(ns, ts))
    if c["op"] == "read":
        s["out"] = [torch.zeros(B, T, hk, D, dtype=torch.float16, device="cuda").transpose(1, 2) for _ in "kv"]
    elif c["op"] != "write":
        s["out"] = torch.zeros(B, T, hq, D, dtype=torch.float16, device="cuda").transpose(1, 2)
    return s


def prepare(case, seed):
    s = _inputs(case, seed)
    if own:
        _library_cache(s)
    return s


# ------------------------------------------------------------------------------------------------ the plain forms


def _held(s, w, b, first, last, kind=torch.float32):
    """Tokens first .. last of sequence b as the cache holds them, [H, last - first, D]."""
    c, G = s["case"], s["case"]["block"]
    H, n = c["kv_heads"], _counts(c)[0][b]
    packed = n - n % G
    codes, scales = s["store"][w]
    parts = []
    if first < min(last, packed):
        g0, g1 = first // G, -(-min(last, packed) // G)
        if c["paged"]:
            block = torch.arange(g0, g1, device="cuda")
            page, at = s["page_table"][b].long()[block * G // PAGE], block % (PAGE // G)
            x = codes.view(torch.int8).view(-1, H, PAGE // G, G, D)[page, :, at].view(codes.dtype).to(kind)
            x = (x * scales[page, :, at].to(kind)[:, :, None, None]).transpose(0, 1).reshape(H, -1, D)
        else:
            x = codes[b, :, g0 * G:g1 * G].to(kind).view(H, -1, G, D) * scales[b, :, g0:g1].to(kind)[:, :, None, None]
            x = x.view(H, -1, D)
        parts.append(x[:, first - g0 * G:min(last, packed) - g0 * G])
    if last > packed:
        parts.append(s["open"][w][b, :, max(first, packed) - packed:last - packed].to(kind))
    return torch.cat(parts, 1) if parts else torch.zeros(H, 0, D, dtype=kind, device="cuda")


def _state(s):
    """A cache as what it holds: axes as the library has them."""
    c, (P, S) = s["case"], s["places"]
    out = {}
    for w, axes in (("k", _key_axes), ("v", _value_axes)):
        codes, scales = s["store"][w]
        out[w + "_codes"], out[w + "_scales"], out[w + "_open"] = axes(codes, P, c["kv_heads"], S), scales, s["open"][w]
    if c["ragged"]:
        out["counts"] = s["counts"]
    return out


def _write(s):
    c, G = s["case"], s["case"]["block"]
    s["counts"].copy_(s["cached"] + s["new"])
    for b, (n, t) in enumerate(zip(*_counts(c))):
        for w in "kv":
            waits = s["open"][w][b]
            x = torch.cat([waits[:, :n % G], s[w][b, :, :t]], 1)
            m = x.shape[1] // G
            if m:
                codes, scales = _packed(c, x[:, :m * G].reshape(-1, G, D))
                _put(s, w, b, n - n % G, codes.view(-1, m, G, D), scales.view(-1, m))
            rest = x.shape[1] - m * G
            waits[:, :rest] = x[:, m * G:]
    return _state(s)


def _read(s):
    for b, (n, t) in enumerate(zip(*_counts(s["case"]))):
        for w, out in zip("kv", s["out"]):
            out[b, :, :t] = _held(s, w, b, n - t, n).half()
    return s["out"]


def _attend(s):
    """Both attentions: softmax(q K^T / sqrt(D)) V, a row without a token zero."""
    c, out = s["case"], s["out"]
    H, r, causal = c["kv_heads"], c["q_heads"] // c["kv_heads"], c["op"] == "attend"
    for b, (n, t) in enumerate(zip(*_counts(c))):
        k, v = (_held(s, w, b, 0, n) for w in "kv")
        if causal:
            k, v = torch.cat([k, s["k"][b, :, :t].float()], 1), torch.cat([v, s["v"][b, :, :t].float()], 1)
        if k.shape[1] == 0:
            out[b, :, :t] = 0
            continue
        q = s["q"][b, :, :t].float().reshape(H, r * t, D)
        together = max(1, (1 << 28) // (r * t * k.shape[1]))
        for h in range(0, H, together):
            a = torch.matmul(q[h:h + together], k[h:h + together].transpose(1, 2).contiguous())
            a *= 1.0 / math.sqrt(D)
            if causal:
                hidden = torch.arange(n + t, device="cuda") > n + torch.arange(t, device="cuda")[:, None]
                a.view(-1, r, t, n + t).masked_fill_(hidden, -math.inf)
            a -= a.amax(-1, keepdim=True)
            a.exp_()
            o = torch.matmul(a, v[h:h + together]) / a.sum(-1, keepdim=True)
            out[b, h * r:h * r + o.shape[0] * r, :t] = o.view(-1, t, D).half()
    return out


def _own(s):
    from paper_2602_23200_amd import binding as iq
    c, cache = s["case"], s["cache"]
    op, ragged = c["op"], c["ragged"]
    if op == "write":
        if ragged:
            s["counts"].copy_(s["cached"])
            iq.innerq_block_append_ragged(cache, s["counts"], s["new"], s["k"], s["v"])
        else:
            cache.c.n_tokens = c["cached"]
            iq.innerq_block_append(cache, s["k"], s["v"])
        k, v = _library_axes(s, cache.buffers)
        shape = s["places"][0], c["kv_heads"], s["places"][1] // c["block"]
        out = {"k_codes": k, "v_codes": v}
        for w in "kv":
            out[w + "_scales"] = cache.buffers[w + "_scales"].view(torch.float32).view(shape)
            out[w + "_open"] = cache.buffers[w + "_open"].view(torch.float16).view(c["batch"], c["kv_heads"], c["block"], D)
        if ragged:
            out["counts"] = s["counts"]
        return out
    if op == "read":
        if ragged:
            iq.innerq_block_read_ragged(cache, s["cached"], s["first"], *s["out"])
        else:
            iq.innerq_block_read(cache, c["cached"] - c["new"], *s["out"])
        return s["out"]
    if op == "attend":
        if ragged:
            return iq.innerq_block_attention_ragged(cache, s["cached"], s["new"], s["most"], s["k"], s["v"], s["q"], s["workspace"], out=s["out"])
        return iq.innerq_block_attention(cache, s["k"], s["v"], s["q"], s["workspace"], out=s["out"])
    if ragged:
        return iq.innerq_block_cross_attention_ragged(cache, s["cached"], s["new"], s["most"], s["q"], s["workspace"], out=s["out"])
    return iq.innerq_block_cross_attention(cache, s["q"], s["workspace"], out=s["out"])


def run(state):
    if own:
        out = _own(state)
    else:
        out = {"write": _write, "read": _read, "attend": _attend, "cross": _attend}[state["case"]["op"]](state)
    return out if isinstance(out, dict) else {"out": out}


# ------------------------------------------------------------------------------------------------ the least work


def work(case):
    c, G = case, case["block"]
    H, total, flops = c["kv_heads"], 0.0, 0.0
    for n, t in zip(*_counts(c)):
        held = 2 * H * ((n - n % G) * (D + 4.0 / G) + n % G * 2 * D)           # bytes of the cached tokens, keys and values
        if c["op"] == "write":
            gone = (n % G + t) // G * G                                        # tokens that are packed
            old = n % G if gone else 0
            total += 2 * H * (t * 2 * D + old * 2 * D + gone * (D + 4.0 / G) + (n + t - (n - n % G) - gone - (n % G - old)) * 2 * D)
            flops += 2 * H * gone * D * 4.0
        elif c["op"] == "read":
            still = min(t, n % G)                                              # of the open rows
            total += 2 * H * ((t - still) * (D + 4.0 / G) + still * 2 * D + t * 2 * D)
            flops += 2 * H * (t - still) * D
        else:
            total += held + c["q_heads"] * t * D * 4
            flops += 4.0 * c["q_heads"] * D * t * n
            if c["op"] == "attend":
                total += 2 * H * t * 2 * D
                flops += 4.0 * c["q_heads"] * D * t * (t + 1) / 2
    return {"bytes": total, "flops": flops}


# ------------------------------------------------------------------------------------------------ the definition, in 64 bits


def _token(s, w, b, i):
    """Tokens i (a tensor) of sequence b, one by one out of where they lie, in 64 bits: [H, len(i), D]."""
    c, G = s["case"], s["case"]["block"]
    n = _counts(c)[0][b]
    packed = i < n - n % G
    place = torch.where(packed, i, 0)
    codes, scales = s["store"][w]
    P, S = s["places"]
    page = s["page_table"][b].long()[place // S] if c["paged"] else torch.full_like(place, b)
    x = codes.view(torch.int8)[page, :, place % S].view(codes.dtype).double() * scales[page, :, place % S // G].double()[..., None]
    y = s["open"][w][b][:, i % G].double().transpose(0, 1)
    return torch.where(packed[:, None, None], x, y).transpose(0, 1)


def _write_exact(s):
    c, G = s["case"], s["case"]["block"]
    top = 448 if c["e4m3"] else 127
    out = {w + "_codes": None for w in "kv"}                                   # (fields of 8 bits)
    if c["ragged"]:
        out["counts"] = None
    for w in "kv":
        scale, waits = s["store"][w][1].double(), s["open"][w].double()
        for b, (n, t) in enumerate(zip(*_counts(c))):
            last = (n + t) // G * G
            for g in range(n // G, last // G):
                size = s[w][b, :, max(0, g * G - n):g * G + G - n].abs().amax((1, 2)).double()
                if g == n // G and n % G:
                    size = torch.maximum(size, s["open"][w][b, :, :n % G].abs().amax((1, 2)).double())
                if c["paged"]:
                    scale[s["page_table"][b, g * G // PAGE].long(), :, g * G % PAGE // G] = size / top
                else:
                    scale[b, :, g] = size / top
            for i in range(max(n, last), n + t):
                waits[b, :, i % G] = s[w][b, :, i - n].double()
        out[w + "_scales"], out[w + "_open"] = scale, waits
    return out


def exact(case, seed):
    s = _inputs(case, seed)
    c = s["case"]
    if c["op"] == "write":
        return _write_exact(s)
    if c["op"] == "read":
        out = []
        for w in "kv":
            rows = s["out"][0].double()
            for b, (n, t) in enumerate(zip(*_counts(c))):
                rows[b, :, :t] = _token(s, w, b, torch.arange(n - t, n, device="cuda"))
            out.append(rows)
        return {"out": out}
    r = c["q_heads"] // c["kv_heads"]
    out = s["out"].double()
    for b, (n, t) in enumerate(zip(*_counts(c))):
        k, v = (_token(s, w, b, torch.arange(n, device="cuda")) for w in "kv")
        if c["op"] == "attend":
            k, v = (torch.cat([x, s[w][b, :, :t].double()], 1) for w, x in (("k", k), ("v", v)))
        if k.shape[1] == 0:
            continue
        for g in range(c["q_heads"]):
            a = s["q"][b, g, :t].double() @ k[g // r].T / math.sqrt(D)
            if c["op"] == "attend":
                a = a.masked_fill(torch.ones_like(a, dtype=torch.bool).triu(n + 1), -math.inf)
            out[b, g, :t] = torch.softmax(a, -1) @ v[g // r]
    return {"out": out}
