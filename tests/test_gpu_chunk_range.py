"""innerq_chunk_attention where scores lie far apart or are very large: weights far below the largest one, and scores whose neighbours in fp32
are whole powers of two apart."""
import math
from dataclasses import replace

import numpy as np
import pytest

from oracle import innerq_oracle as orc
from tests.chunk_reference import attend, check, operands
from tests.helpers import gpu_config, oracle_config
from tests.test_gpu_chunk import small

pytestmark = pytest.mark.gpu
# new tokens and query heads a kv head of every row form: up to 32 rows, up to 128, more (most keys cached)
FORMS = [(2, 4), (20, 4), (40, 4)]


@pytest.fixture(scope="module")
def env():
    import torch
    from paper_2602_23200_amd import binding as iq
    assert torch.cuda.is_available(), "these tests need the MI355X"
    iq.lib()
    return torch, iq


@pytest.mark.parametrize("form", range(3))
@pytest.mark.parametrize("strong", [0, 4, 30, 700])
@pytest.mark.parametrize("nats", [5.0, 12.0, 16.0, 17.0, 18.0, 21.0])
def test_one_token_far_above_the_others(env, nats, strong, form):
    """A sink, the first packed token, one of the first tile, one of the window: its value is 0, so that the output is what the others' weights
    are.  They are `nats` below it; in fp16 at a level equal to the largest score they would lose their bits (from 9.7 nats on) and vanish (from
    17.3 on)."""
    torch, iq = env
    t, r = FORMS[form]
    n, heads = 720, 512
    w = small(n_q_heads=heads * r, n_kv_heads=heads, bits=4)
    o = oracle_config(w, capacity=1024)
    o1 = replace(o, n_q_heads=r, n_kv_heads=1)
    rng = np.random.default_rng(form)
    # one value in a row: asymmetric groups of one zero-point, nothing is rounded; many equal heads, so that the keys are not split
    k = np.full((1, 1, n + t, 128), 0.25, np.float16)
    k[:, :, strong] = 1.25
    v = (1.0 + rng.random((1, 1, n + t, 128))).astype(np.float16)
    v[:, :, strong] = 0.0
    q = np.full((1, r, t, 128), nats / math.sqrt(128.0), np.float16)
    cache, ref = iq.allocate_cache(gpu_config(o)), orc.cache_new(o1)
    orc.quantize_append(o1, ref, k[:, :, :n], v[:, :, :n])
    kd, vd = (torch.from_numpy(x).cuda().expand(-1, heads, -1, -1) for x in (k, v))
    qd = torch.from_numpy(q).cuda().repeat(1, heads, 1, 1)
    iq.innerq_append_rotated(cache, kd[:, :, :n], vd[:, :, :n])
    out = iq.innerq_chunk_attention(cache, kd[:, :, n:], vd[:, :, n:], qd, iq.allocate_chunk_workspace(cache.cfg, t))
    assert torch.equal(out[:, :r], out[:, -r:])
    want, bound = attend(q[0], operands(o1, ref, "k", k[0, :, n:]), operands(o1, ref, "v", v[0, :, n:]), False)
    print(check(out[0, :r].cpu().numpy(), want, bound))


@pytest.mark.parametrize("nats", [12.0, 17.0, 21.0])
def test_one_new_token_far_above_the_others(env, nats):
    """The same within a first prompt, where the strong token is the first new one."""
    torch, iq = env
    t, heads = 900, 64
    w = small(n_q_heads=heads, n_kv_heads=heads, bits=4)
    o = oracle_config(w, capacity=1024)
    rng = np.random.default_rng(1)
    k = np.full((1, t, 128), 0.25, np.float16)
    k[:, 0] = 1.25
    v = (1.0 + rng.random((1, t, 128))).astype(np.float16)
    v[:, 0] = 0.0
    q = np.full((1, t, 128), nats / math.sqrt(128.0), np.float16)
    cache = iq.allocate_cache(gpu_config(o))
    kd, vd, qd = (torch.from_numpy(x).cuda()[None].expand(-1, heads, -1, -1) for x in (k, v, q))
    out = iq.innerq_chunk_attention(cache, kd, vd, qd, iq.allocate_chunk_workspace(cache.cfg, t))
    want, bound = attend(q, k.astype(np.float64), v.astype(np.float64), False)
    print(check(out[0, :1].cpu().numpy(), want, bound))
    assert torch.equal(out[0, 0], out[0, -1])


@pytest.mark.parametrize("form", range(3))
@pytest.mark.parametrize("nats", [15.0, 17.4, 20.0])
def test_a_long_flat_tail(env, nats, form):
    """A million tokens `nats` below one strong token, in a range of their own: together they hold 24 % to 0.2 % of the weight.  All blocks of the
    store but the first are one page."""
    torch, iq = env
    t, r = FORMS[form]
    n, B, heads = 1 << 20, [128, 64, 64][form], 8
    cfg = iq.make_config(B, heads * r, heads, 128, 4, 32, 4, 128, orc.ASYM, orc.ASYM, capacity_tokens=n + 64, page_pool_pages=2)
    table = torch.ones(B, (n + 64) // 64, dtype=torch.int32, device="cuda")
    table[:, 0] = 0
    cache = iq.allocate_cache(cfg, page_table=table)
    # codes and scales 0: every value is its group's zero-point
    for name, x in cache.buffers.items():
        if name != "page_table":
            x.zero_()
    for which, low in (("k", 0.25), ("v", 1.0)):
        cache.buffers[f"{which}_scales"].view(torch.float16).fill_(-0.0)
        for part in ("zeros", "sink", "recent"):
            cache.buffers[f"{which}_{part}"].view(torch.float16).fill_(low)
    rows = cache.buffers["k_zeros"].view(torch.float16).view(2, heads, 64, 4)
    rows[0, :, 0] = 1.25
    # (a value's group is 32 tokens of a channel: the strong token's group says 0 for all of them, which are 31 of a million)
    cache.buffers["v_zeros"].view(torch.float16).view(2, heads, 2, 128)[0, :, 0] = 0.0
    cache.c.n_tokens = cache.c.store_ahead_tokens = n
    k = torch.full((B, heads, t, 128), 0.25, dtype=torch.float16, device="cuda")
    v = torch.ones(B, heads, t, 128, dtype=torch.float16, device="cuda")
    x = np.float16(nats / math.sqrt(128.0))
    q = torch.full((B, heads * r, t, 128), float(x), dtype=torch.float16, device="cuda")
    out = iq.innerq_chunk_attention(cache, k, v, q, iq.allocate_chunk_workspace(cfg, t))
    low = math.exp(-float(x) * 128.0 / math.sqrt(128.0))
    for i in range(t):
        others = n + i
        want = (others - 31) * low / (1.0 + others * low)
        # 2^-11 each for the roundings of the strong weight and of the tail's (all alike), 2^-34 of the strong one for those below the normal
        # range; sums in fp32, whose addends are all alike, so that their roundings may be: 2^-24 of the sum for each of a wavefront's additions
        most = 1.0 / (1.0 + others * low)
        bound = 2 * want * (1 - want) * 2.0 ** -11 + 2.0 ** -34 * most * others + 2.0 ** -24 * (n / 16 + 600) * want
        err = (out[:, :, i] - want).abs().max().item()
        assert err <= bound, (i, err, bound, want)


MAGNITUDES = [(60.0, 100.0), (3000.0, 1000.0), (3000.0, 60000.0), (60000.0, 60000.0)]


@pytest.mark.parametrize("sign", [1.0, -1.0])
@pytest.mark.parametrize("magnitude", MAGNITUDES)
@pytest.mark.parametrize("order", ["random", "rising", "falling"])
@pytest.mark.parametrize("form", range(3))
def test_large_scores(env, form, order, magnitude, sign):
    """Scores of 10^5 to 4 10^10, all positive or all negative: keys along one direction in steps of 2 % from the largest score down, so that it is a
    token's alone and the output that token's value."""
    torch, iq = env
    t, r = FORMS[form]
    n = 300
    w = small(n_q_heads=2 * r, n_kv_heads=2, bits=4)
    o = oracle_config(w, capacity=512)
    o1 = replace(o, batch=1)
    rng = np.random.default_rng(form)
    direction = np.where(rng.random(128) < 0.5, -1.0, 1.0)
    place = rng.permutation(n + t) if order == "random" else np.arange(n + t)[::-1 if order == "rising" else 1]
    size = magnitude[1] * (1.02 ** -place.clip(0, 40) if sign > 0 else 0.45 * 1.02 ** place.clip(0, 40))
    k = np.broadcast_to(size[None, :, None] * direction, (2, n + t, 128)).astype(np.float16)
    v = rng.standard_normal((2, n + t, 128)).astype(np.float16)
    q = (sign * magnitude[0] * direction * (1.0 + 0.05 * rng.random((2 * r, t, 1)))).astype(np.float16)
    cache, ref = iq.allocate_cache(gpu_config(o)), orc.cache_new(o1)
    orc.quantize_append(o1, ref, k[None, :, :n], v[None, :, :n])
    kd, vd, qd = (torch.from_numpy(np.ascontiguousarray(x)).cuda()[None] for x in (k, v, q))
    iq.innerq_append_rotated(cache, kd[:, :, :n], vd[:, :, :n])
    out = iq.innerq_chunk_attention(cache, kd[:, :, n:], vd[:, :, n:], qd, iq.allocate_chunk_workspace(cache.cfg, t))[0].cpu().numpy()
    assert np.isfinite(out).all()
    K, V = operands(o1, ref, "k", k[:, n:]), operands(o1, ref, "v", v[:, n:])
    alone = 0
    for g in range(2 * r):
        s = q[g].astype(np.float64) @ K[g // r].T / math.sqrt(128.0)
        a = np.abs(q[g].astype(np.float64)) @ np.abs(K[g // r]).T / math.sqrt(128.0)
        s[np.arange(n + t)[None] > n + np.arange(t)[:, None]] = -np.inf
        for i in range(t):
            order = np.argsort(s[i])
            # clear of the second one by what 128 additions in fp32 can move a score (2^-24 of the sum of magnitudes each, both ways) and 40 nats
            if s[i, order[-1]] - s[i, order[-2]] > 2 * 128 * 2.0 ** -24 * a[i].max() + 40.0:
                alone += 1
                assert np.abs(out[g, i] - V[g // r, order[-1]]).max() <= 2.0 ** -20 * 4, (g, i)
    assert alone == 2 * r * t
