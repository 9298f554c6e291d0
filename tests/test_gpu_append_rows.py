"""innerq_append_rotated and its ragged form against the oracle: the cache that rotating every key first and appending it then
leaves, bit for bit, whatever the sizes of the calls."""
from dataclasses import replace

import numpy as np
import pytest

from oracle import innerq_oracle as orc
from paper_2602_23200_amd import workloads as wl
from tests.helpers import assert_cache_equal, gpu_config, oracle_config
from tests.rows import projection, rotate, rotation_tables
from tests.test_gpu_paged import gathered, paged_cache

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def env():
    import torch
    from paper_2602_23200_amd import binding as iq
    assert torch.cuda.is_available(), "these tests need the MI355X"
    iq.lib()
    return torch, iq


def small(**kw):
    base = dict(name="r", batch=2, n_q_heads=4, n_kv_heads=2, head_dim=128, n_tokens=1, bits=2, group=32, w_sink=4, w_recent=48, seed=3)
    base.update(kw)
    return wl.Workload(**base)


SYM, ASYM, HYBRID = orc.SYM, orc.ASYM, orc.HYBRID
FORMS = [dict(bits=2), dict(bits=4, group=64), dict(bits=3, k_mode=SYM, v_mode=SYM), dict(bits=4, k_mode=ASYM, v_mode=SYM),
         dict(bits=3, group=64, k_mode=HYBRID, v_mode=ASYM), dict(bits=2, group=64, w_recent=1), dict(bits=2, w_sink=0, w_recent=5),
         dict(bits=4, n_q_heads=9, n_kv_heads=3)]
# first prompts that end in the sink, in the window and beyond it; chunks that overwrite what they evict; single tokens between
CALLS = [[1, 1, 1, 70, 1, 33, 200, 1, 64], [300, 1, 1, 2, 130, 5], [3, 49, 31, 1, 1, 1], [777]]


def tables(torch, iq, rows, rot_dim, interleaved, axes):
    cos, sin = rotation_tables(rows, rot_dim)
    return cos, sin, iq.make_rotation(torch.from_numpy(cos).cuda(), torch.from_numpy(sin).cuda(), interleaved, axes)


@pytest.mark.parametrize("form", range(len(FORMS)))
@pytest.mark.parametrize("calls", range(len(CALLS)))
def test_appends_of_any_size(env, form, calls):
    torch, iq = env
    w = small(**FORMS[form])
    rng = np.random.default_rng(100 * form + calls)
    n_axes, rot_dim, interleaved, norm = 1 + (form + calls) % 3, [128, 96, 64, 128][calls], (form + calls) % 2 == 1, form % 2 == 1
    axes = None if n_axes == 1 else [(i // 9) % n_axes for i in range(rot_dim // 2)]
    cos, sin, rot = tables(torch, iq, 400, rot_dim, interleaved, axes)
    total = sum(CALLS[calls])
    o = oracle_config(w, capacity=-(-total // 64) * 64)
    cache, ref = iq.allocate_cache(gpu_config(o)), orc.cache_new(o)
    inv = (0.5 + rng.random((w.n_kv_heads, 128))).astype(np.float32) if norm else None
    done = 0
    for t in CALLS[calls]:
        _, _, k, v = projection(torch, rng, w.batch, t, 1, w.n_kv_heads)
        if calls == 2:
            k, v = k.contiguous(), v.contiguous()          # (the layout of the other appends)
        positions = rng.integers(0, 400, (n_axes, w.batch, t)).astype(np.int32)
        if t == 1 and n_axes == 1:
            positions = np.full((1, w.batch, 1), done, np.int32)
            given = None                                   # (its place in the sequence)
        else:
            given = torch.from_numpy(positions).cuda()
        iq.innerq_append_rotated(cache, k, v, rot, positions=given, k_inv_norm=None if inv is None else torch.from_numpy(inv).cuda())
        turned = rotate(k.cpu().numpy(), cos, sin, positions, rot_dim, interleaved, axes)
        orc.quantize_append(o, ref, turned, v.cpu().numpy(), k_inv_norm=inv)
        done += t
        assert cache.n_tokens == done and cache.c.store_ahead_tokens == done
        assert_cache_equal(cache, ref, o, what=f"after {done}")


def test_without_a_rotation_it_is_the_ordinary_append(env):
    torch, iq = env
    w = small(bits=4)
    o = oracle_config(w, capacity=512)
    rng = np.random.default_rng(1)
    a, b = iq.allocate_cache(gpu_config(o)), iq.allocate_cache(gpu_config(o))
    for t in (90, 1, 40, 1, 1, 200):
        _, _, k, v = projection(torch, rng, w.batch, t, 1, w.n_kv_heads)
        iq.innerq_append_rotated(a, k, v)
        iq.innerq_quantize_append(b, k.contiguous(), v.contiguous())
        for name, x in a.buffers.items():
            assert x is None or torch.equal(x, b.buffers[name]), (name, t)


@pytest.mark.parametrize("heads", [1, 2, 5, 8])
def test_long_prompt_takes_ranges_of_heads(env, heads):
    """Long enough that a work-group takes several heads, an odd number of them among others."""
    torch, iq = env
    for group in (32, 64):
        w = small(batch=1, n_q_heads=heads, n_kv_heads=heads, bits=2, group=group, w_recent=128)
        n = 20000 if heads > 1 else 5000
        o = oracle_config(w, capacity=-(-n // 64) * 64)
        rng = np.random.default_rng(heads)
        cos, sin, rot = tables(torch, iq, n, 128, False, None)
        _, _, k, v = projection(torch, rng, 1, n, 1, heads, spare=0)
        cache = iq.allocate_cache(gpu_config(o))
        iq.innerq_append_rotated(cache, k, v, rot)
        turned = torch.from_numpy(rotate(k.cpu().numpy(), cos, sin, np.arange(n)[None, None], 128)).cuda()
        plain = iq.allocate_cache(gpu_config(o))
        iq.innerq_quantize_append(plain, turned, v.contiguous())
        for name, x in cache.buffers.items():
            assert x is None or torch.equal(x, plain.buffers[name]), name
        h = heads - 1                                       # (and one head against the oracle)
        o1 = replace(o, n_q_heads=1, n_kv_heads=1, capacity_tokens=1024)
        ref = orc.cache_new(o1)
        orc.quantize_append(o1, ref, turned[:, h:h + 1, :1000].cpu().numpy(), v[:, h:h + 1, :1000].cpu().numpy())
        rows = orc.partition(o1, "k", 1000)[1]
        got = cache.buffers["k_codes"].view(heads, o.capacity_tokens, -1)[h, :rows].cpu().numpy()
        assert np.array_equal(got, ref.k_codes[0, 0, :rows])


def ahead(o, ref):
    """The state the ragged append leaves: the store of a sequence one step ahead of its windows."""
    return orc.partition(o, "k", min(ref.n_tokens + 1, o.capacity_tokens))[1], orc.partition(o, "v", min(ref.n_tokens + 1, o.capacity_tokens))[1]


@pytest.mark.parametrize("paged", [False, True])
@pytest.mark.parametrize("form", range(len(FORMS)))
def test_ragged(env, form, paged):
    torch, iq = env
    w = small(batch=5, **FORMS[form])
    rng = np.random.default_rng(form)
    rounds = [[0, 1, 17, 90, 300], [1, 1, 0, 1, 1], [1, 1, 1, 1, 1], [64, 2, 33, 0, 5], [1, 0, 1, 1, 1], [200, 4, 100, 31, 1]]
    total = np.array(rounds).sum(0)
    o = oracle_config(w, capacity=512 if w.group == 64 else 448)
    cos, sin, rot = tables(torch, iq, 500, 128, False, [0] * 20 + [1] * 20 + [2] * 24)
    cache = paged_cache(torch, iq, o, list(total + 1), seed=form) if paged else iq.allocate_cache(gpu_config(o))
    o1 = replace(o, batch=1)
    refs = [orc.cache_new(o1) for _ in total]
    runs = [orc.cache_new(o1) for _ in total]
    n_dev = torch.zeros(5, dtype=torch.int32, device="cuda")
    for ts in rounds:
        T = max(ts)
        x, _, k, v = projection(torch, rng, 5, T, 1, w.n_kv_heads)
        for b, t in enumerate(ts):
            x[b, t:] = float("nan")                         # (padding is not read)
        positions = rng.integers(0, 500, (3, 5, T)).astype(np.int32)
        iq.innerq_append_rotated_ragged(cache, n_dev, torch.tensor(ts, dtype=torch.int32, device="cuda"), k, v, rot,
                                        positions=torch.from_numpy(positions).cuda())
        turned = rotate(k.cpu().numpy(), cos, sin, positions, 128, False, [0] * 20 + [1] * 20 + [2] * 24)
        g = gathered(torch, iq, cache) if paged else cache
        for b, t in enumerate(ts):
            if t:
                orc.quantize_append(o1, refs[b], turned[b:b + 1, :, :t], v[b:b + 1, :, :t].cpu().numpy())
            assert int(n_dev[b]) == refs[b].n_tokens
            if refs[b].n_tokens:
                assert_cache_equal(g, refs[b], o1, bsel=slice(b, b + 1), what=f"sequence {b} after {refs[b].n_tokens}", per_sequence=True)
    # the store is one step ahead: a decode step may follow, and does what it does behind the ordinary calls
    one = [torch.from_numpy(rng.standard_normal((5, h, 128)).astype(np.float16)).cuda() for h in (w.n_kv_heads, w.n_kv_heads, w.n_q_heads)]
    k1, v1, q1 = one[0][:, :, None].contiguous(), one[1][:, :, None].contiguous(), one[2]
    out = iq.innerq_decode_step_ragged(cache, n_dev, o.capacity_tokens, k1, v1, q1, iq.allocate_workspace(cache.cfg)).cpu().numpy()
    for b in range(5):
        orc.quantize_append(o1, refs[b], k1[b:b + 1].cpu().numpy(), v1[b:b + 1].cpu().numpy())
        want = orc.decode_attention(o1, refs[b], q1[b:b + 1].cpu().numpy())
        err = (np.abs(out[b] - want[0]).max(-1) / np.abs(want[0]).max(-1)).max()
        assert err <= 2e-3, (b, err)


def test_counts_outside_their_bounds_are_clamped(env):
    """A sequence that would pass the capacity takes what fits; a bad count touches no other sequence."""
    torch, iq = env
    w = small(batch=3, bits=4)
    o = oracle_config(w, capacity=128)
    rng = np.random.default_rng(0)
    cache = iq.allocate_cache(gpu_config(o))
    guard = {n: x.clone() for n, x in cache.buffers.items() if x is not None}
    n_dev = torch.tensor([0, -5, 0], dtype=torch.int32, device="cuda")
    _, _, k, v = projection(torch, rng, 3, 100, 1, w.n_kv_heads)
    iq.innerq_append_rotated_ragged(cache, n_dev, torch.tensor([100, 0, -1], dtype=torch.int32, device="cuda"), k, v)
    assert n_dev.tolist() == [100, -5, 0]
    _, _, k2, v2 = projection(torch, rng, 3, 64, 1, w.n_kv_heads)
    iq.innerq_append_rotated_ragged(cache, n_dev, torch.tensor([64, 0, 500], dtype=torch.int32, device="cuda"), k2, v2)
    assert n_dev.tolist() == [128, -5, 64]
    o1 = replace(o, batch=1)
    for b, parts in ((0, [(k, v, 100), (k2, v2, 28)]), (2, [(k2, v2, 64)])):
        ref = orc.cache_new(o1)
        for kk, vv, t in parts:
            orc.quantize_append(o1, ref, kk[b:b + 1, :, :t].cpu().numpy(), vv[b:b + 1, :, :t].cpu().numpy())
        assert_cache_equal(cache, ref, o1, bsel=slice(b, b + 1), per_sequence=True)
    for name, x in cache.buffers.items():
        if x is not None:
            assert torch.equal(x.view(3, -1)[1], guard[name].view(3, -1)[1]), name


def test_recorded_and_replayed(env):
    """A ragged append in a graph: the counts move on from replay to replay."""
    torch, iq = env
    w = small(batch=2, bits=2)
    o = oracle_config(w, capacity=512)
    rng = np.random.default_rng(2)
    cos, sin, rot = tables(torch, iq, 600, 128, False, None)
    for T in (1, 24):
        cache = iq.allocate_cache(gpu_config(o))
        _, _, k, v = projection(torch, rng, 2, T, 1, w.n_kv_heads)
        n_dev = torch.zeros(2, dtype=torch.int32, device="cuda")
        t_dev = torch.tensor([T, max(1, T // 2)], dtype=torch.int32, device="cuda")
        iq.innerq_append_rotated_ragged(cache, n_dev, t_dev, k, v, rot)      # (first use outside the capture)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            iq.innerq_append_rotated_ragged(cache, n_dev, t_dev, k, v, rot)
        o1 = replace(o, batch=1)
        refs = [orc.cache_new(o1) for _ in range(2)]
        n_dev.zero_()
        for step in range(200 if T == 1 else 15):
            if step % 5 == 0:
                v.mul_(-1.0)
                torch.cuda.synchronize()
            graph.replay()
            for b in range(2):
                t = int(t_dev[b])
                place = refs[b].n_tokens + np.arange(T)[None, None]
                turned = rotate(k[b:b + 1].cpu().numpy(), cos, sin, place, 128)
                orc.quantize_append(o1, refs[b], turned[:, :, :t], v[b:b + 1, :, :t].cpu().numpy())
        for b in range(2):
            assert int(n_dev[b]) == refs[b].n_tokens
            assert_cache_equal(cache, refs[b], o1, bsel=slice(b, b + 1), per_sequence=True)
