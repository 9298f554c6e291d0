"""Attention over the 8-bit cache where scores lie far apart or are very large, and where scales do."""
import math

import numpy as np
import pytest

from tests import block_cache as bc
from tests import block_reference as ref
from tests.chunk_reference import check

pytestmark = pytest.mark.gpu
D = 128
# new tokens, four query heads a kv head: up to 16 rows, 32, 64, 128, more
FORMS = [1, 5, 12, 20, 40]


@pytest.fixture(scope="module")
def env():
    import torch
    from paper_2602_23200_amd import binding as iq
    assert torch.cuda.is_available(), "these tests need the MI355X"
    iq.lib()
    return torch, iq


@pytest.mark.parametrize("t", FORMS)
@pytest.mark.parametrize("nats", [5.0, 12.0, 17.0, 21.0])
@pytest.mark.parametrize("strong", [0, 40, 700, 723])
def test_one_token_far_above_the_others(env, nats, strong, t):
    """Packed first, in a later tile, open, or new: its value is 0, so that the output is what the others' weights are, `nats` below it."""
    torch, iq = env
    n, r, H = 720, 4, 320                                  # (many equal heads, so that keys are not split)
    if strong >= n + t:
        pytest.skip("not there")
    rng = np.random.default_rng(t)
    k = np.full((1, 1, n + t, D), 0.25, np.float16)
    k[:, :, strong] = 1.25
    v = (1.0 + rng.random((1, 1, n + t, D))).astype(np.float16)
    v[:, :, strong] = 0.0
    q = np.full((r, t, D), nats / math.sqrt(128.0), np.float16)
    cache, _ = bc.empty(torch, iq, 1, H * r, H, 832, t % 2 == 0, 32)
    kd, vd = (torch.from_numpy(x).cuda().expand(-1, H, -1, -1) for x in (k, v))
    iq.innerq_block_append(cache, kd[:, :, :n], vd[:, :, :n])
    out = iq.innerq_block_attention(cache, kd[:, :, n:], vd[:, :, n:], torch.from_numpy(q).cuda()[None].repeat(1, H, 1, 1),
                                    iq.allocate_block_workspace(cache.cfg, t))
    K, V = (np.concatenate([ref.held(x[0, :, :n], 32, t % 2 == 0), x[0, :, n:].astype(np.float64)], 1) for x in (k, v))
    want, bound = ref.attend(q, K, V, False, t * r > 32, ref.causal(n, t))
    for h in (0, H - 1):
        check(out[0, h * r:(h + 1) * r].cpu().numpy(), want, bound)


@pytest.mark.parametrize("t", FORMS)
@pytest.mark.parametrize("nats", [15.0, 17.4, 20.0])
def test_a_long_flat_tail(env, nats, t):
    """A million tokens `nats` below one strong token: together they hold 24 % to 0.2 % of the weight.  All blocks of the store but the first are one page."""
    torch, iq = env
    n, B, H, r = 1 << 20, 32, 8, 4
    cfg = iq.make_block_config(B, H * r, H, type=iq.INT8, block=32, capacity_tokens=n + 64, page_pool_pages=2)
    table = torch.ones(B, (n + 64) // 64, dtype=torch.int32, device="cuda")
    table[:, 0] = 0
    cache = iq.allocate_block_cache(cfg, page_table=table)
    # keys: 25 steps of 0.01, the strong one 127 of them; values: one, those of the strong token's block zero
    cache.buffers["k_codes"].fill_(25)
    cache.buffers["k_codes"].view(2, H, 2, 2, 2, 4, 16, 16)[0, :, 0, 0, :, :, 0] = 127     # (page, head, tile, a, h, g, c, e: token 0)
    cache.buffers["k_scales"].view(torch.float32).fill_(0.01)
    cache.buffers["v_codes"].fill_(127)
    cache.buffers["v_codes"].view(2, H, 2, 4096)[0, :, 0] = 0
    cache.buffers["v_scales"].view(torch.float32).fill_(float(np.float32(1.0) / np.float32(127.0)))
    cache.buffers["v_scales"].view(torch.float32).view(2, H, 2)[0, :, 0] = 0.0
    cache.c.n_tokens = n
    k = torch.full((B, H, t, D), 0.25, dtype=torch.float16, device="cuda")
    v = torch.ones(B, H, t, D, dtype=torch.float16, device="cuda")
    q = torch.full((B, H * r, t, D), nats / 1.02 / math.sqrt(128.0), dtype=torch.float16, device="cuda")
    out = iq.innerq_block_attention(cache, k, v, q, iq.allocate_block_workspace(cfg, t))
    x, step = float(q[0, 0, 0, 0]), float(np.float32(0.01))
    low, new = math.exp(-x * 102 * step * math.sqrt(128.0)), math.exp(x * (0.25 - 127 * step) * math.sqrt(128.0))
    u = 2.0 ** -11 if t * r > 32 else 2.0 ** -22
    for i in range(t):
        weight, value = (n - 1) * low + (i + 1) * new, (n - 32) * low + (i + 1) * new
        want = value / (1.0 + weight)
        # u each for the roundings of the strong weight and of the tail's (all alike), 2^-34 of the strong one for those below the normal range, scores of
        # 20 off by 50 2^-24; sums in fp32, whose addends are all alike, so that their roundings may be: 2^-23 of the sum for each of a lane's additions
        most = 1.0 / (1.0 + weight)
        bound = 2 * want * (1 - want) * (u + 1500 * 2.0 ** -24) + 2.0 ** -34 * most * n + 2.0 ** -23 * (n / 16 + 600) * want
        err = (out[:, :, i] - want).abs().max().item()
        assert err <= bound, (i, err, bound, want)


@pytest.mark.parametrize("sign", [1.0, -1.0])
@pytest.mark.parametrize("magnitude", [(60.0, 100.0), (3000.0, 1000.0), (3000.0, 60000.0), (60000.0, 60000.0)])
@pytest.mark.parametrize("order", ["random", "rising", "falling"])
@pytest.mark.parametrize("t", FORMS)
def test_large_scores(env, t, order, magnitude, sign):
    """Scores of 10^5 to 4 10^10, all positive or all negative: keys along one direction in steps of 2 %, so that the largest score is a token's alone and the
    output that token's value."""
    torch, iq = env
    n, r = 300, 4
    rng = np.random.default_rng(t)
    direction = np.where(rng.random(D) < 0.5, -1.0, 1.0)
    place = rng.permutation(n + t) if order == "random" else np.arange(n + t)[::-1 if order == "rising" else 1]
    size = magnitude[1] * (1.02 ** -place.clip(0, 40) if sign > 0 else 0.45 * 1.02 ** place.clip(0, 40))
    k = np.broadcast_to(size[None, :, None] * direction, (2, n + t, D)).astype(np.float16)
    v = rng.standard_normal((2, n + t, D)).astype(np.float16)
    q = (sign * magnitude[0] * direction * (1.0 + 0.05 * rng.random((2 * r, t, 1)))).astype(np.float16)
    cache, _ = bc.empty(torch, iq, 1, 2 * r, 2, 512, False, 32)
    kd, vd, qd = (torch.from_numpy(np.ascontiguousarray(x)).cuda()[None] for x in (k, v, q))
    iq.innerq_block_append(cache, kd[:, :, :n], vd[:, :, :n])
    out = iq.innerq_block_attention(cache, kd[:, :, n:], vd[:, :, n:], qd, iq.allocate_block_workspace(cache.cfg, t))[0].cpu().numpy()
    assert np.isfinite(out).all()
    K, V = (np.concatenate([ref.held(x[:, :n], 32, False), x[:, n:].astype(np.float64)], 1) for x in (k, v))
    alone = 0
    for g in range(2 * r):
        s = q[g].astype(np.float64) @ K[g // r].T / math.sqrt(128.0)
        a = np.abs(q[g].astype(np.float64)) @ np.abs(K[g // r]).T / math.sqrt(128.0)
        s[ref.causal(n, t)] = -np.inf
        for i in range(t):
            last = np.argsort(s[i])
            # clear of the second one by what 128 additions in fp32 can move a score (2^-23 of the sum of magnitudes each, both ways) and 40 nats
            if s[i, last[-1]] - s[i, last[-2]] > 2 * 128 * 2.0 ** -23 * a[i].max() + 40.0:
                alone += 1
                assert np.abs(out[g, i] - V[g // r, last[-1]]).max() <= 2.0 ** -20 * 4, (g, i)
    assert alone > 0.8 * 2 * r * t


@pytest.mark.parametrize("t", FORMS)
@pytest.mark.parametrize("e4", [False, True])
@pytest.mark.parametrize("seed", range(3))
def test_scales_far_apart(env, t, e4, seed):
    """Blocks of keys and values from the smallest fp16 numbers to the largest, blocks of zeros among them, queries aimed at tokens of any of them."""
    torch, iq = env
    rng = np.random.default_rng(100 * t + seed)
    n, r, block = 1100, 4, 32
    V = rng.standard_normal((1, 1, n + t, D)) * 10.0 ** rng.uniform(-7.0, 4.3, (n + t + 31) // 32).repeat(32)[:n + t, None]
    K = rng.standard_normal((1, 1, n + t, D)) * 10.0 ** rng.uniform(-1.0, 1.0, (n + t + 31) // 32).repeat(32)[:n + t, None]
    for x in (V, K):
        for g in rng.integers(0, n // 32, 3):
            x[:, :, 32 * g:32 * g + 32] = 0.0
    k, v = (np.clip(x, -65504, 65504).astype(np.float16) for x in (K, V))
    cache, _ = bc.empty(torch, iq, 1, r, 1, 1280, e4, block)
    kd, vd = torch.from_numpy(k).cuda(), torch.from_numpy(v).cuda()
    iq.innerq_block_append(cache, kd[:, :, :n], vd[:, :, :n])
    K, V = (np.concatenate([ref.held(x[0, :, :n], block, e4), x[0, :, n:].astype(np.float64)], 1) for x in (k, v))
    q = rng.standard_normal((r, t, D))
    for g in range(r):
        for i in range(t):
            j = int(rng.integers(n + i + 1))
            size = (K[0, j] ** 2).sum()
            if size > 0 and rng.random() < 0.8:
                q[g, i] = K[0, j] * rng.choice([6.0, 20.0, 60.0]) * math.sqrt(D) / size
    q = np.clip(q, -60000, 60000).astype(np.float16)
    out = iq.innerq_block_attention(cache, kd[:, :, n:], vd[:, :, n:], torch.from_numpy(q).cuda()[None], iq.allocate_block_workspace(cache.cfg, t))
    want, bound = ref.attend(q, K, V, False, t * r > 32, ref.causal(n, t))
    check(out[0].cpu().numpy(), want, bound, (t, e4, seed))
