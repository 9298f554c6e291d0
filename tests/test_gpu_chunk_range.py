"""innerq_chunk_attention where scores are very large: their neighbours in fp32 are whole numbers apart."""
import math
from dataclasses import replace

import numpy as np
import pytest

from oracle import innerq_oracle as orc
from tests.chunk_reference import operands
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
