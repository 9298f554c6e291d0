"""Attention over the 8-bit cache where the scales of values lie far apart: blocks far below another one."""
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
