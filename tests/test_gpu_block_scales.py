"""Attention over the 8-bit cache where scales of values lie far apart: blocks far below another one, and long tails of small weights beside a strong token
in a block of another scale.

Tolerances are the header's words.  Keys and queries are made so that every score is a sum of equal products of few bits, exact in fp32 in any order; what is left
of a score's error are its factor, the sum with the logarithm of the scale (below 40), the level's subtraction and the exponential, 2^-24 each of magnitudes
up to the largest |score| (in units of log2) and that logarithm: e (12 most + 100), most in nats.  A weight is moved by that share of itself, by its own
rounding (u = 2^-22, or 2^-11 of more than 32 rows) and by 2^-34 of the row's largest one, which is never more than all of it.  Sums in fp32 add 2^-23 of
sum p |v| for each of a lane's additions (one a tile) and for those within a tile and of the joins."""
import math

import numpy as np
import pytest

from tests import block_cache as bc
from tests import block_reference as ref

pytestmark = pytest.mark.gpu
D, H, R = 128, 320, 4                                      # (many equal heads, so that keys are not split)
# new tokens, four query heads a kv head: up to 16 rows, 32, 64, 128, more
FORMS = [1, 5, 12, 20, 40]


@pytest.fixture(scope="module")
def env():
    import torch
    from paper_2602_23200_amd import binding as iq
    assert torch.cuda.is_available(), "these tests need the MI355X"
    iq.lib()
    return torch, iq


def attend(env, k, v, q, n, e4, block):
    """k, v [n + t, D] of every head, q [R, t, D] -> [R, t, D] of the first and the last head, fp32."""
    torch, iq = env
    t = len(k) - n
    cache, _ = bc.empty(torch, iq, 1, H * R, H, -(-(n + t) // 64) * 64, e4, block)
    kd, vd = (torch.from_numpy(x).cuda()[None, None].expand(1, H, -1, -1) for x in (k, v))
    if n:
        iq.innerq_block_append(cache, kd[:, :, :n], vd[:, :, :n])
    out = iq.innerq_block_attention(cache, kd[:, :, n:], vd[:, :, n:], torch.from_numpy(q).cuda()[None].repeat(1, H, 1, 1),
                                    iq.allocate_block_workspace(cache.cfg, t))
    return [out[0, h * R:(h + 1) * R].cpu().numpy().astype(np.float64) for h in (0, H - 1)]


def held(x, n, e4, block):
    return np.concatenate([ref.held(x[None, :n], block, e4)[0], x[n:].astype(np.float64)])


@pytest.mark.parametrize("t", FORMS)
@pytest.mark.parametrize("e4", [False, True])
@pytest.mark.parametrize("ratio", [0, 3, 5, 12, 19, 22, 24, 26, 27, 28, 29, 30, 31, 32, 34])
def test_a_block_far_below_another(env, ratio, e4, t):
    """Every other block's values are 2^-ratio of the others'; queries have all of their weight on one token of the small ones: its value, to 2^-35 of
    the largest value."""
    n, rng = 22 * 32, np.random.default_rng(ratio)
    size = np.where(np.arange(n + t) // 32 % 2 == 0, 60000.0, 60000.0 * 2.0 ** -ratio)
    v = (rng.uniform(-1.0, 1.0, (n + t, D)) * size[:, None]).astype(np.float16)
    aim = rng.permutation(np.flatnonzero(np.arange(n) // 32 % 2))[:D]                       # (a channel of the keys for each)
    k, q = np.zeros((n + t, D), np.float16), np.zeros((R * t, D), np.float16)
    k[aim, np.arange(D)] = 8.0
    channel = np.arange(R * t) % D
    q[np.arange(R * t), channel] = 96.0                    # (68 nats)
    token = aim[channel]
    K, V = held(k, n, e4, 32), held(v, n, e4, 32)
    score = (q.astype(np.float64) * K[token]).sum(1) / math.sqrt(D)
    assert (score > 60).all()
    for got in attend(env, k, v, q.reshape(R, t, D), n, e4, 32):
        # (the others' weights are 0 in any form; a value and the sum it is divided by carry the same weight, rounded in a few operations)
        bound = 2.0 ** -35 * np.abs(V).max() + 2.0 ** -20 * np.abs(V[token])
        err = np.abs(got.reshape(R * t, D) - V[token])
        assert (err <= bound).all(), (ratio, float((err / bound).max()))


def promised(q, K, V, hidden, many):
    """Attention of q [R, t, D] over K, V [N, D] in 64 bits, and the bound of every element (see above)."""
    out, bound = np.zeros(q.shape), np.zeros(q.shape)
    u, e, far = (2.0 ** -11 if many else 2.0 ** -22), 2.0 ** -24, 2.0 ** -35 * np.abs(V).max()
    for r in range(len(q)):
        s = q[r].astype(np.float64) @ K.T / math.sqrt(D)
        most = np.where(hidden, 0.0, np.abs(s)).max(-1, keepdims=True)
        s[hidden] = -np.inf
        p = np.exp(s - s.max(-1, keepdims=True))
        share = p * (u + e * (12 * most + 100)) + np.minimum(p, 2.0 ** -34)
        total = p.sum(-1, keepdims=True)
        p, share = p / total, share / total
        out[r] = p @ V
        for i in range(q.shape[1]):
            bound[r, i] = 1.01 * share[i] @ np.abs(V - out[r, i])
        bound[r] += 2.0 ** -23 * (len(K) / 32 + 100) * (p @ np.abs(V)) + far * (p @ (V != 0))
    return out, bound


def check_tail(env, strong, outlier, n, t, nats, e4, block):
    """Blocks `strong` (of 32 tokens) have one token `nats` above the others, with values of 0, and 31 without any weight, with values of `outlier`; other tokens
    have a key of 0 and values of 1."""
    k, v = np.zeros((n + t, D), np.float16), np.ones((n + t, D), np.float16)
    for g in strong:
        k[32 * g:32 * g + 32], v[32 * g:32 * g + 32] = -127.0 / 32, outlier
        k[32 * g + 3 * g % 32], v[32 * g + 3 * g % 32] = 1.0, 0.0
    K, V = held(k, n, e4, block), held(v, n, e4, block)
    top = K[32 * strong[0] + 3 * strong[0] % 32, 0]
    x = nats / (top * math.sqrt(D))
    step = 2.0 ** (math.floor(math.log2(x)) - 7)           # (eight bits)
    q = np.full((R, t, D), round(x / step) * step, np.float16)
    hidden = ref.causal(n, t)
    want, bound = promised(q, K, V, hidden, t * R > 32)
    assert (want > 0).all() and (want < 0.6).all()
    worst = 0.0
    for got in attend(env, k, v, q, n, e4, block):
        worst = max(worst, float((np.abs(got - want) / bound).max()))
    assert worst <= 1.0, worst


@pytest.mark.parametrize("t", FORMS)
@pytest.mark.parametrize("e4", [False, True])
@pytest.mark.parametrize("block", [32, 64])
@pytest.mark.parametrize("outlier", [1.0, 1.9, 4.1, 7.9, 15.0, 15.9, 16.1, 40.0, 900.0, 60000.0])
@pytest.mark.parametrize("nats", [14.2, 16.0, 17.4])
def test_a_tail_beside_a_strong_token_of_a_larger_scale(env, nats, outlier, block, e4, t):
    check_tail(env, list(range(0, 44, 4)), outlier, 44 * 32 + 5, t, nats, e4, block)


@pytest.mark.parametrize("t", FORMS)
@pytest.mark.parametrize("e4", [False, True])
@pytest.mark.parametrize("block", [32, 64])
@pytest.mark.parametrize("outlier", [1.0, 30.0, 900.0, 4100.0, 60000.0])
@pytest.mark.parametrize("nats", [14.2, 16.0, 17.4])
def test_a_tail_of_open_and_new_rows(env, nats, outlier, block, e4, t):
    check_tail(env, list(range(14)), outlier, 14 * 32 + (31 if block == 32 else 63), t, nats, e4, block)


@pytest.mark.parametrize("t", FORMS)
@pytest.mark.parametrize("e4", [False, True])
def test_large_values_of_new_rows_behind_larger_ones_of_the_cache(env, e4, t):
    """Open and new rows up to 65504 and down to the smallest numbers beside blocks of any scale, queries aimed at one of them."""
    n, rng = 14 * 32 + 31, np.random.default_rng(t)
    v = (rng.uniform(-1.0, 1.0, (n + t, D)) * 65504.0 * 2.0 ** -rng.integers(0, 33, (n + t, 1))).astype(np.float16)
    v[:32] = 65504.0
    k, q = np.zeros((n + t, D), np.float16), np.zeros((R, t, D), np.float16)
    token = np.concatenate([np.arange(14 * 32, n)[::3], n + np.zeros(1, np.int64)])         # (seen by all rows)
    k[token, np.arange(len(token))] = 8.0
    channel = np.arange(R * t).reshape(R, t) % len(token)
    np.put_along_axis(q, channel[..., None], np.float16(96.0), 2)
    V = held(v, n, e4, 32)[token[channel]]
    for got in attend(env, k, v, q, n, e4, 32):
        bound = 2.0 ** -35 * 65504.0 + 2.0 ** -20 * np.abs(V)
        assert (np.abs(got - V) <= bound).all(), float((np.abs(got - V) / bound).max())
