"""The reference that the attention of several new tokens is held against (tests/chunk_reference.py), held against a model of the kernel's
roundings: right results pass, and results with one mistake planted do not."""
from dataclasses import replace

import numpy as np
import pytest

from oracle import innerq_oracle as orc
from paper_2602_23200_amd import workloads as wl
from tests.chunk_reference import aimed, attend, borders_of, check, operands
from tests.helpers import oracle_config

CASES = [(2, 32, 400, 5, 4), (4, 64, 400, 40, 4), (3, 32, 1003, 33, 2), (4, 32, 117, 130, 1), (2, 64, 0, 70, 1)]


def case(bits, group, n, t, r, heads=2):
    w = wl.Workload(name="c", batch=1, n_q_heads=r * heads, n_kv_heads=heads, head_dim=128, n_tokens=1, bits=bits, group=group, w_sink=4, w_recent=48, seed=3)
    o1 = replace(oracle_config(w, capacity=1280), batch=1)
    rng = np.random.default_rng(bits * n + t)
    spread = 1.0 + np.abs(rng.standard_t(3, (heads, 1, 128)))
    k = (rng.standard_normal((heads, n + t, 128)) * spread).astype(np.float16)
    v = rng.standard_normal((heads, n + t, 128)).astype(np.float16)
    ref = orc.cache_new(o1)
    if n:
        orc.quantize_append(o1, ref, k[None, :, :n], v[None, :, :n])
    K, V = operands(o1, ref, "k", k[:, n:]), operands(o1, ref, "v", v[:, n:])
    return o1, aimed(rng, K, n, t, r, borders_of(o1, n, t)), K, V


def model(q, K, V, hidden=None, above=9.0, most=15.0, tile=64, weight_bits=None):
    """Tile by tile in fp32, the weights rounded to fp16 at a running level of 2^above below the score that raised it."""
    Hq, t, d = q.shape
    r, N = Hq // K.shape[0], K.shape[1]
    if hidden is None:
        hidden = np.arange(N)[None] > N - t + np.arange(t)[:, None]
    out = np.empty((Hq, t, d))
    scale = np.float32(np.log2(np.e) / np.sqrt(d))
    for g in range(Hq):
        s = (q[g].astype(np.float32) @ K[g // r].astype(np.float32).T) * scale
        s[hidden] = -np.inf
        m, l, o = np.full(t, -np.inf), np.zeros(t), np.zeros((t, d))
        for j in range(0, N, tile):
            top = s[:, j:j + tile].max(-1).astype(np.float64)
            raised = top > m + most
            level = np.where(raised, top - above, m)
            f = np.where(raised, np.exp2(np.where(np.isinf(m), -np.inf, m - np.where(raised, level, 0.0))), 1.0)
            m, l, o = level, l * f, o * f[:, None]
            w = np.exp2(s[:, j:j + tile] - np.where(np.isinf(m), 0.0, m)[:, None]).astype(np.float16).astype(np.float64)
            l += w.sum(-1)
            o += w @ V[g // r][j:j + tile]
        out[g] = o / l[:, None]
    return out


@pytest.mark.parametrize("c", CASES)
@pytest.mark.parametrize("half", [False, True])
def test_a_right_result_passes(c, half):
    o1, q, K, V = case(*c)
    want, bound = attend(q, K, V, half)
    got = model(q, K, V)
    print(check(got.astype(np.float16) if half else got, want, bound, str(c)))


def bfloat(x):
    w = x.astype(np.float32).view(np.uint32)
    return ((w + 0x7fff + ((w >> 16) & 1)) & 0xffff0000).view(np.float32).astype(np.float64)


@pytest.mark.parametrize("c", CASES)
def test_results_with_a_mistake_do_not(c):
    """One token hidden or shown, two values changed places, operands of fewer bits: each is beyond the bound, in fp16 outputs, too."""
    o1, q, K, V = case(*c)
    n, t = c[2], c[3]
    N = n + t
    want, bound = attend(q, K, V, True)
    causal = np.arange(N)[None] > n + np.arange(t)[:, None]
    rows = np.arange(t)

    def wrong(what, **kw):
        with pytest.raises(AssertionError):
            check(model(q, kw.get("K", K), kw.get("V", V), kw.get("hidden", causal)).astype(np.float16), want, bound)
            print("not seen:", what)

    own = causal.copy()
    own[rows[1:], n + rows[1:]] = True                      # (a row keeps at least one token)
    wrong("own token hidden", hidden=own)
    shown = causal.copy()
    shown[rows[:-1], n + rows[:-1] + 1] = False
    wrong("next token shown", hidden=shown)
    if t > 64:
        wrong("a tile of later tokens shown", hidden=causal & (np.arange(N)[None] >= n + (rows[:, None] // 64 + 1) * 64))
    for j in borders_of(o1, n, t)[:-1]:
        if (~causal[:, j]).sum() < 3:
            continue
        less = causal.copy()
        less[:, j] = True
        less[rows, n + rows] = False
        wrong(f"token {j} left out", hidden=less)
        swapped = V.copy()
        swapped[:, [j, j + 1]] = V[:, [j + 1, j]]
        wrong(f"values {j} and {j + 1} changed places", V=swapped)
    wrong("bfloat16 values", V=bfloat(V))
    wrong("bfloat16 keys", K=bfloat(K))


def test_the_lower_end_of_the_weights():
    """One token holds nearly all of the weight and comes first; the others are 12 to 21 nats below it.  At a level equal to the largest score
    their weights lose their bits and then vanish; 2^9 below it they keep them within the bound."""
    rng = np.random.default_rng(0)
    for nats in (12.0, 16.0, 17.0, 18.0, 21.0):
        K = np.zeros((1, 1001, 128))
        K[0, 0] = 1.0
        q = np.full((1, 1, 128), nats / np.sqrt(128.0)).astype(np.float16)
        V = 1.0 + rng.random((1, 1001, 128)).astype(np.float16).astype(np.float64)
        V[0, 0] = 0.0
        want, bound = attend(q, K, V, False)
        check(model(q, K, V), want, bound)
        if nats >= 16.0:
            with pytest.raises(AssertionError):
                check(model(q, K, V, above=0.0, most=6.0), want, bound)
