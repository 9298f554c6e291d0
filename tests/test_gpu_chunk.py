"""innerq_chunk_attention and its ragged form against attention in 64 bits over what the cache holds (decoded by the oracle) and the
new rows."""
from dataclasses import replace

import numpy as np
import pytest

from oracle import innerq_oracle as orc
from paper_2602_23200_amd import workloads as wl
from tests.helpers import gpu_config, oracle_config
from tests.rows import projection
from tests.test_gpu_paged import paged_cache

pytestmark = pytest.mark.gpu
SYM, ASYM, HYBRID = orc.SYM, orc.ASYM, orc.HYBRID


@pytest.fixture(scope="module")
def env():
    import torch
    from paper_2602_23200_amd import binding as iq
    assert torch.cuda.is_available(), "these tests need the MI355X"
    iq.lib()
    return torch, iq


def small(**kw):
    base = dict(name="c", batch=1, n_q_heads=4, n_kv_heads=1, head_dim=128, n_tokens=1, bits=2, group=32, w_sink=4, w_recent=48, seed=3)
    base.update(kw)
    return wl.Workload(**base)


def filled(torch, iq, o, lengths, rng, scale=1.0, pages=None):
    """A cache whose sequence b holds lengths[b] tokens, and the oracle's caches of them (batch 1 each)."""
    cfg = gpu_config(o)
    cache = paged_cache(torch, iq, o, [n + 1 for n in lengths], seed=pages) if pages is not None else iq.allocate_cache(cfg)
    o1 = replace(o, batch=1)
    refs, T = [], max(max(lengths), 1)
    spread = 1.0 + np.abs(rng.standard_t(3, (1, o.n_kv_heads, 1, 128)))
    k = np.clip(rng.standard_normal((len(lengths), o.n_kv_heads, T, 128)) * spread * scale, -60000.0, 60000.0).astype(np.float16)
    v = rng.standard_normal((len(lengths), o.n_kv_heads, T, 128)).astype(np.float16)
    for b, n in enumerate(lengths):
        refs.append(orc.cache_new(o1))
        if n:
            orc.quantize_append(o1, refs[b], k[b:b + 1, :, :n], v[b:b + 1, :, :n])
    counts = torch.zeros(len(lengths), dtype=torch.int32, device="cuda")
    iq.innerq_append_rotated_ragged(cache, counts, torch.tensor(lengths, dtype=torch.int32, device="cuda"), torch.from_numpy(k).cuda(),
                                    torch.from_numpy(v).cuda())
    cache.c.n_tokens = lengths[0]                          # (for the calls with one count for all)
    cache.c.store_ahead_tokens = lengths[0] + 1
    return cache, o1, refs, counts


def held(o1, ref, which):
    """What the cache holds of one sequence, in token order: 64-bit values [Hk, n, d]."""
    if ref.n_tokens == 0:
        return np.zeros((o1.n_kv_heads, 0, 128))
    return np.stack([np.asarray(orc.effective_tensor(o1, ref, which, 0, h), dtype=np.float64) for h in range(o1.n_kv_heads)])


def expected(o1, ref, q, k, v):
    """q [Hq, t, d], k, v [Hk, t, d] -> [Hq, t, d] in 64 bits."""
    r = q.shape[0] // k.shape[0]
    K = np.concatenate([held(o1, ref, "k"), k.astype(np.float64)], axis=1)
    V = np.concatenate([held(o1, ref, "v"), v.astype(np.float64)], axis=1)
    t, n = q.shape[1], K.shape[1]
    s = np.einsum("gtd,gnd->gtn", q.astype(np.float64), K.repeat(r, 0)) / np.sqrt(128.0)
    s[:, np.arange(n)[None] > n - t + np.arange(t)[:, None]] = -np.inf
    p = np.exp(s - s.max(-1, keepdims=True))
    return np.einsum("gtn,gnd->gtd", p / p.sum(-1, keepdims=True), V.repeat(r, 0)), s, V


def tolerance(want, s, V, q, K_most):
    """Bound of an element's error.  Keys, values and weights are fp16 roundings, half a step of 2^-10 (u = 2^-11 relative each).  A
    weight's error is u of itself for its own rounding plus that of its score, at most sum |q k| u / sqrt(d); normalised weights
    sum to one, so an output is off by at most (2 u + 2 ds) max |V| over the tokens attended to, ds the largest score error, and by
    1e-5 of that for all fp32 sums."""
    u = 2.0 ** -11
    ds = u * (np.abs(q.astype(np.float64)).sum(-1).max() * K_most) / np.sqrt(128.0)
    return (2 * u + 2 * min(ds, 1.0) + 1e-5) * np.abs(V).max()


def check(torch, o1, refs, lengths, ts, q, k, v, out, half):
    worst = 0.0
    for b, t in enumerate(ts):
        if not t:
            continue
        qb, kb, vb = (x[b, :, :t].cpu().numpy() for x in (q, k, v))
        want, s, V = expected(o1, refs[b], qb, kb, vb)
        got = out[b, :, :t].float().cpu().numpy().astype(np.float64)
        assert np.isfinite(got).all()
        # the root mean square over a row: roundings are independent, so their sum over tokens is far below the bound of an element;
        # three times 2^-11 for the three roundings, the score's share by its spread, and the output's own rounding
        err = np.abs(got - want)
        spread = 2.0 ** -11 * np.sqrt((qb.astype(np.float64) ** 2).sum(-1).max() / 128.0) * np.abs(held_most(o1, refs[b], kb))
        bound = tolerance(want, s, V, qb, held_most(o1, refs[b], kb)) + (2.0 ** -11 * np.abs(want) if half else 0.0)
        assert (err <= bound).all(), (b, (err / bound).max())
        rms = np.sqrt((err ** 2).mean() / (want ** 2).mean())
        assert rms <= 2.0 ** -11 * 3 + 2 * spread, (b, rms)
        worst = max(worst, rms)
    return worst


def held_most(o1, ref, k):
    return max(np.abs(held(o1, ref, "k")).max(initial=0.0), np.abs(k.astype(np.float64)).max())


FORMS = [dict(bits=2), dict(bits=4), dict(bits=3, k_mode=SYM, v_mode=SYM), dict(bits=4, group=64, k_mode=ASYM, v_mode=SYM),
         dict(bits=3, group=64, k_mode=HYBRID, v_mode=ASYM), dict(bits=2, group=64, w_recent=1, w_sink=0), dict(bits=3, v_bits=2, w_recent=130)]


@pytest.mark.parametrize("form", range(len(FORMS)))
@pytest.mark.parametrize("n", [0, 1, 4, 53, 85, 116, 117, 400, 1003])
def test_chunks(env, form, n):
    torch, iq = env
    over = dict(FORMS[form])
    v_bits = over.pop("v_bits", 0)
    r, heads = [(4, 1), (1, 3), (8, 1), (5, 2)][(form + n) % 4]
    w = small(n_q_heads=r * heads, n_kv_heads=heads, **over)
    rng = np.random.default_rng(form * 1000 + n)
    o = oracle_config(w, capacity=1280, v_bits=v_bits)
    cache, o1, refs, counts = filled(torch, iq, o, [n], rng)
    before = {name: x.clone() for name, x in cache.buffers.items() if x is not None}
    for t in (1, 5, 33, 130):
        _, q, k, v = projection(torch, rng, 1, t, r * heads, heads)
        half = (form + t) % 2 == 0
        out = torch.empty(1, t, r * heads, 128, dtype=torch.float16 if half else torch.float32, device="cuda").transpose(1, 2)
        ws = iq.allocate_chunk_workspace(cache.cfg, t)
        ws.fill_(255)                                      # (its content may be anything: NaN here)
        iq.innerq_chunk_attention(cache, k, v, q, ws, out=out)
        check(torch, o1, refs, [n], [t], q, k, v, out, half)
    for name, x in before.items():
        assert torch.equal(x, cache.buffers[name]), name


@pytest.mark.parametrize("paged", [None, 5])
@pytest.mark.parametrize("form", [0, 1, 4])
@pytest.mark.parametrize("T", [1, 7, 200])
def test_ragged(env, form, paged, T):
    torch, iq = env
    w = small(batch=6, n_q_heads=8, n_kv_heads=2, **FORMS[form])
    rng = np.random.default_rng(form * 10 + T)
    o = oracle_config(w, capacity=1536)
    lengths = [0, 3, 90, 700, 1200, 64]
    ts = [min(T, x) for x in (T, 1, 0, 150, 2, 33)]
    cache, o1, refs, counts = filled(torch, iq, o, lengths, rng, pages=paged)
    x, q, k, v = projection(torch, rng, 6, T, 8, 2)
    for b, t in enumerate(ts):
        x[b, t:] = float("nan")                             # (padding is not read)
    out = torch.full((6, T, 8, 128), 7.0, dtype=torch.float16, device="cuda").transpose(1, 2)
    ws = iq.allocate_chunk_workspace(cache.cfg, T)
    ws.fill_(255)
    iq.innerq_chunk_attention_ragged(cache, counts, torch.tensor(ts, dtype=torch.int32, device="cuda"), 1400, k, v, q, ws, out=out)
    check(torch, o1, refs, lengths, ts, q, k, v, out, True)
    for b, t in enumerate(ts):
        assert (out[b, :, t:] == 7.0).all()
    assert counts.tolist() == lengths


def test_one_token_is_the_decode_step(env):
    """A chunk of one token behind a store that is not run ahead attends to what innerq_decode_attention_next attends to, but for the
    token that leaves the window in that step; behind an empty window of change (n + 1 <= sinks + window) they are the same."""
    torch, iq = env
    rng = np.random.default_rng(1)
    w = small(batch=2, n_q_heads=8, n_kv_heads=2, bits=4)
    o = oracle_config(w, capacity=256)
    cache, o1, refs, counts = filled(torch, iq, o, [40, 40], rng)
    _, q, k, v = projection(torch, rng, 2, 1, 8, 2)
    a = iq.innerq_chunk_attention(cache, k, v, q, iq.allocate_chunk_workspace(cache.cfg, 1))
    cache.c.store_ahead_tokens = 41
    b = iq.innerq_decode_attention_next(cache, k.contiguous(), v.contiguous(), q[:, :, 0].contiguous(), iq.allocate_workspace(cache.cfg))
    # fp16 weights and the fp32 sums of the short form: 2 x 2^-11 of the largest value
    assert (a[:, :, 0] - b).abs().max() <= 2.0 ** -10 * v.abs().max().item() * 2


def test_query_scale_and_extreme_magnitudes(env):
    """The factors applied by the call; keys near the end of fp16 against small queries, and the other way round."""
    torch, iq = env
    rng = np.random.default_rng(2)
    for bits, scale in ((2, 3000.0), (4, 3000.0), (4, 2.0 ** -10), (3, 1000.0)):
        w = small(n_q_heads=4, n_kv_heads=2, bits=bits)
        o = oracle_config(w, capacity=640)
        cache, o1, refs, counts = filled(torch, iq, o, [500], rng, scale=scale)
        _, q, k, v = projection(torch, rng, 1, 20, 4, 2)
        k = (k.float() * scale).half()
        factor = torch.from_numpy((rng.random((2, 128)) / scale).astype(np.float32)).cuda()
        out = iq.innerq_chunk_attention(cache, k, v, q, iq.allocate_chunk_workspace(cache.cfg, 20), q_scale=factor)
        scaled = (q.float() * factor.repeat_interleave(2, 0)[None, :, None]).half()
        check(torch, o1, refs, [500], [20], scaled, k, v, out, False)


def test_scores_that_rise_and_fall(env):
    """Keys ever larger along the tokens (the level is raised again and again), and the same backwards."""
    torch, iq = env
    rng = np.random.default_rng(12)
    w = small(n_q_heads=2, n_kv_heads=1, bits=4)
    o = oracle_config(w, capacity=1280)
    o1 = replace(o, batch=1)
    for back in (False, True):
        n, t = 900, 70
        ramp = np.linspace(0.05, 6.0, n + t)[:, None]
        ramp = ramp[::-1] if back else ramp
        direction = rng.standard_normal(128)
        k = (direction * ramp + 0.1 * rng.standard_normal((n + t, 128))).astype(np.float16)[None, None]
        v = rng.standard_normal((1, 1, n + t, 128)).astype(np.float16)
        q = np.broadcast_to(direction, (1, 2, t, 128)).astype(np.float16)
        cache, ref = iq.allocate_cache(gpu_config(o)), orc.cache_new(o1)
        orc.quantize_append(o1, ref, k[:, :, :n], v[:, :, :n])
        kd, vd, qd = (torch.from_numpy(np.ascontiguousarray(x)).cuda() for x in (k, v, q))
        iq.innerq_append_rotated(cache, kd[:, :, :n], vd[:, :, :n])
        out = iq.innerq_chunk_attention(cache, kd[:, :, n:], vd[:, :, n:], qd, iq.allocate_chunk_workspace(cache.cfg, t))
        check(torch, o1, [ref], [n], [t], qd, kd[:, :, n:], vd[:, :, n:], out, False)


def test_long_context_and_long_chunk(env):
    """Enough keys for many splits, enough rows for many work-groups; one (sequence, head) of several compared."""
    torch, iq = env
    rng = np.random.default_rng(7)
    for (B, heads, r, n, t, bits, group) in ((3, 8, 4, 6000, 6, 2, 32), (1, 2, 4, 9000, 600, 4, 64), (1, 4, 1, 0, 1500, 4, 32), (2, 1, 1, 5000, 1, 2, 32),
                                             (1, 1, 71, 700, 3, 4, 32)):
        w = small(batch=B, n_q_heads=heads * r, n_kv_heads=heads, bits=bits, group=group, w_recent=128)
        o = oracle_config(w, capacity=-(-(n + t + 2) // 64) * 64)
        cache = iq.allocate_cache(gpu_config(o))
        K, V = (torch.randn(B, heads, max(n, 1), 128, device="cuda").half() for _ in range(2))
        if n:
            iq.innerq_append_rotated(cache, K, V)
        _, q, k, v = projection(torch, rng, B, t, heads * r, heads)
        out = iq.innerq_chunk_attention(cache, k, v, q, iq.allocate_chunk_workspace(cache.cfg, t))
        b, h = B - 1, heads - 1
        o1 = replace(o, batch=1, n_q_heads=r, n_kv_heads=1)
        ref = orc.cache_new(o1)
        if n:
            orc.quantize_append(o1, ref, K[b:b + 1, h:h + 1].cpu().numpy(), V[b:b + 1, h:h + 1].cpu().numpy())
        sel = slice(h * r, (h + 1) * r)
        check(torch, o1, [ref], [n], [t], q[b:b + 1, sel], k[b:b + 1, h:h + 1], v[b:b + 1, h:h + 1], out[b:b + 1, sel], False)


def test_recorded_and_replayed_with_appends(env):
    """Rotation, ragged attention and ragged append in one graph, replayed: the sequences grow from replay to replay.  Against eager
    calls on a second cache, bit for bit."""
    from tests.rows import rotation_tables
    torch, iq = env
    rng = np.random.default_rng(3)
    w = small(batch=3, n_q_heads=8, n_kv_heads=2, bits=4)
    o = oracle_config(w, capacity=1024)
    cos, sin = rotation_tables(1024, 128)
    rot = iq.make_rotation(torch.from_numpy(cos).cuda(), torch.from_numpy(sin).cuda())
    T = 20
    x = torch.empty(3, T, 12, 128, dtype=torch.float16, device="cuda")
    ts = torch.tensor([20, 1, 7], dtype=torch.int32, device="cuda")
    sides = []
    for _ in range(2):
        cache = iq.allocate_cache(gpu_config(o))
        sides.append(dict(cache=cache, n=torch.zeros(3, dtype=torch.int32, device="cuda"), x=x.clone(), ws=iq.allocate_chunk_workspace(cache.cfg, T),
                          out=torch.zeros(3, T, 8, 128, dtype=torch.float16, device="cuda").transpose(1, 2)))

    def step(s):
        p = s["x"].transpose(1, 2)
        iq.innerq_rotate(s["cache"].cfg, rot, p[:, :10], out=p[:, :10], n_tokens_dev=s["n"], t_new_dev=ts)
        iq.innerq_chunk_attention_ragged(s["cache"], s["n"], ts, 1024, p[:, 8:10], p[:, 10:], p[:, :8], s["ws"], out=s["out"])
        iq.innerq_append_rotated_ragged(s["cache"], s["n"], ts, p[:, 8:10], p[:, 10:])

    step(sides[0])
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(sides[0])
    for b in sides[0]["cache"].buffers.values():
        if b is not None:
            b.zero_()
    sides[0]["n"].zero_()
    sides[0]["out"].zero_()
    for i in range(30):
        new = torch.from_numpy(rng.standard_normal((3, T, 12, 128)).astype(np.float16)).cuda()
        for s in sides:
            s["x"].copy_(new)
        graph.replay()
        step(sides[1])
        torch.cuda.synchronize()
        assert torch.equal(sides[0]["n"], sides[1]["n"]) and sides[0]["n"].tolist() == [20 * (i + 1), i + 1, 7 * (i + 1)]
        assert torch.equal(sides[0]["out"], sides[1]["out"])
    for name, b in sides[0]["cache"].buffers.items():
        assert b is None or torch.equal(b, sides[1]["cache"].buffers[name]), name


def test_what_no_token_wrote_is_not_read(env):
    """Every byte of the cache is a NaN's before the tokens come: rows behind the last one, free ring slots and unused sinks stay out."""
    torch, iq = env
    rng = np.random.default_rng(21)
    for bits, group, lengths in ((2, 32, [0, 2, 100, 517]), (4, 64, [3, 60, 250, 700]), (3, 32, [1, 84, 85, 116])):
        w = small(batch=4, n_q_heads=4, n_kv_heads=2, bits=bits, group=group)
        o = oracle_config(w, capacity=768)
        o1 = replace(o, batch=1)
        cache = iq.allocate_cache(gpu_config(o))
        for x in cache.buffers.values():
            if x is not None:
                x.fill_(255)
        T = max(lengths)
        _, _, K, V = projection(torch, rng, 4, T, 1, 2)
        counts = torch.zeros(4, dtype=torch.int32, device="cuda")
        iq.innerq_append_rotated_ragged(cache, counts, torch.tensor(lengths, dtype=torch.int32, device="cuda"), K, V)
        refs = []
        for b, n in enumerate(lengths):
            refs.append(orc.cache_new(o1))
            if n:
                orc.quantize_append(o1, refs[b], K[b:b + 1, :, :n].cpu().numpy(), V[b:b + 1, :, :n].cpu().numpy())
        for t in (1, 40):
            _, q, k, v = projection(torch, rng, 4, t, 4, 2)
            ts = torch.full((4,), t, dtype=torch.int32, device="cuda")
            out = iq.innerq_chunk_attention_ragged(cache, counts, ts, 768, k, v, q, iq.allocate_chunk_workspace(cache.cfg, t))
            check(torch, o1, refs, lengths, [t] * 4, q, k, v, out, False)


@pytest.mark.parametrize("batch", [256, 257])
def test_many_sequences(env, batch):
    """As many sequences as a list holds, and one more (whose launch is planned without it)."""
    torch, iq = env
    rng = np.random.default_rng(batch)
    w = small(batch=batch, n_q_heads=2, n_kv_heads=1, bits=4)
    o = oracle_config(w, capacity=256)
    lengths = [int(x) for x in rng.integers(0, 200, batch)]
    ts = [int(x) for x in rng.integers(0, 41, batch)]
    cache, o1, refs, counts = filled(torch, iq, o, lengths, rng)
    T = max(ts)
    _, q, k, v = projection(torch, rng, batch, T, 2, 1)
    out = torch.full((batch, T, 2, 128), 9.0, dtype=torch.float16, device="cuda").transpose(1, 2)
    iq.innerq_chunk_attention_ragged(cache, counts, torch.tensor(ts, dtype=torch.int32, device="cuda"), 256, k, v, q,
                                     iq.allocate_chunk_workspace(cache.cfg, T), out=out)
    check(torch, o1, refs, lengths, ts, q, k, v, out, True)
    for b, t in enumerate(ts):
        assert (out[b, :, t:] == 9.0).all()


def test_counts_outside_their_bounds_touch_nothing_else(env):
    torch, iq = env
    rng = np.random.default_rng(5)
    w = small(batch=4, n_q_heads=4, n_kv_heads=1, bits=4)
    o = oracle_config(w, capacity=256)
    lengths, t = [100, 0, 30, 0], 12
    cache, o1, refs, counts = filled(torch, iq, o, lengths, rng)
    _, q, k, v = projection(torch, rng, 4, t, 4, 1)
    bad = torch.tensor([100, -7, 30, 1 << 20], dtype=torch.int32, device="cuda")
    ts = torch.tensor([12, 500, -3, 5], dtype=torch.int32, device="cuda")
    out = torch.full((4, t, 4, 128), 3.0, device="cuda").transpose(1, 2)
    iq.innerq_chunk_attention_ragged(cache, bad, ts, 256, k, v, q, iq.allocate_chunk_workspace(cache.cfg, t), out=out)
    check(torch, o1, refs, lengths, [12, 0, 0, 0], q, k, v, out, False)
    assert (out[2] == 3.0).all() and (out[3, :, 5:] == 3.0).all()


def test_two_streams(env):
    """Two calls at once, each with its own workspace: the bits of one after the other."""
    torch, iq = env
    rng = np.random.default_rng(6)
    w = small(batch=2, n_q_heads=8, n_kv_heads=2, bits=2)
    o = oracle_config(w, capacity=4096)
    cache = iq.allocate_cache(gpu_config(o))
    _, _, K, V = projection(torch, rng, 2, 3000, 1, 2)
    iq.innerq_append_rotated(cache, K, V)
    jobs = []
    for t in (5, 90):
        _, q, k, v = projection(torch, rng, 2, t, 8, 2)
        ws = iq.allocate_chunk_workspace(cache.cfg, t)
        jobs.append((k, v, q, ws, iq.innerq_chunk_attention(cache, k, v, q, ws).clone()))
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in jobs]
    for _ in range(5):
        outs = [iq.innerq_chunk_attention(cache, k, v, q, ws, stream=s) for (k, v, q, ws, _), s in zip(jobs, streams)]
        torch.cuda.synchronize()
        for out, job in zip(outs, jobs):
            assert torch.equal(out, job[4])


def test_offsets_beyond_32_bits(env):
    """Nine sequences of a million tokens on eight heads, 4.8 GB of packed keys: the last sequence by itself gives the same."""
    torch, iq = env
    n = (1 << 20) - 40
    cfg = iq.make_config(9, 16, 8, 128, 4, 32, 4, 128, capacity_tokens=1 << 20)
    cache = iq.allocate_cache(cfg)
    gen = torch.Generator(device="cuda")
    gen.manual_seed(1)
    for name in ("k_codes", "v_codes"):
        for part in cache.buffers[name].view(9, -1):
            part.random_(0, 256, generator=gen)
    for name in ("k_scales", "v_scales"):                   # (symmetric: 0.1 to 0.3)
        x = cache.buffers[name].view(torch.float16).view(9, -1)
        for part in x:
            part.uniform_(0.1, 0.3, generator=gen)
    for name in ("k_recent", "v_recent", "k_sink", "v_sink"):
        cache.buffers[name].view(torch.float16).normal_(generator=gen)
    one = iq.sequence_view(cache, 8)
    cache.c.n_tokens = cache.c.store_ahead_tokens = one.c.n_tokens = one.c.store_ahead_tokens = n
    rng = np.random.default_rng(2)
    for t in (3, 20):
        _, q, k, v = projection(torch, rng, 9, t, 16, 8)
        out = iq.innerq_chunk_attention(cache, k, v, q, iq.allocate_chunk_workspace(cfg, t))
        alone = iq.innerq_chunk_attention(one, k[8:], v[8:], q[8:], iq.allocate_chunk_workspace(one.cfg, t))
        assert torch.isfinite(out).all()
        # the same fp16 operands, the fp32 sums in another order: weights taken at another level are rounded anew (2^-11 each,
        # independent), so means of values around 1 over a million tokens move by far less than 2^-11 of a value
        assert (out[8] - alone[0]).abs().max() <= 2.0 ** -11
        assert (out[8] - out[0]).abs().max() > 0
