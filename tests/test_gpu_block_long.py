"""Attention over a cache in 8 bits of the largest length, whose tokens all count: two thirds of the weight lie on 2^24 equal tokens, one third on a marked one, so
that a range of tokens that is left out, or taken twice, shows."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu
D = 128


@pytest.fixture(scope="module")
def cache():
    import torch
    from paper_2602_23200_amd import binding as iq
    assert torch.cuda.is_available(), "these tests need the MI355X"
    n, H = (1 << 24) - 265, 3
    cache = iq.allocate_block_cache(iq.make_block_config(1, H, H, type=iq.INT8, block=64, capacity_tokens=1 << 24))
    row = torch.full((1, H, 1, D), 0.5, dtype=torch.float16, device="cuda")
    mark = n // 3
    for part in (mark, 1, n - mark - 1):
        x = row * 4 if part == 1 else row.expand(1, H, part, D)
        iq.innerq_block_append(cache, x, x)
    return torch, iq, cache, n, H


@pytest.mark.parametrize("cross", [False, True])
@pytest.mark.parametrize("ragged", [False, True])
@pytest.mark.parametrize("t", [1, 20, 50, 100, 200])
def test_every_token_counts(cache, t, ragged, cross):
    torch, iq, cache, n, H = cache
    nats = 16.0
    q = torch.full((1, H, t, D), nats / 1.5 / 128.0 ** 0.5, dtype=torch.float16, device="cuda")
    new = torch.full((1, H, t, D), 0.5, dtype=torch.float16, device="cuda")
    ws, count = iq.allocate_block_workspace(cache.cfg, t), torch.tensor([n], dtype=torch.int32, device="cuda")
    if cross:
        out = iq.innerq_block_cross_attention_ragged(cache, count, None, n, q, ws) if ragged else iq.innerq_block_cross_attention(cache, q, ws)
    elif ragged:
        out = iq.innerq_block_attention_ragged(cache, count, None, 1 << 24, new, new, q, ws)
    else:
        out = iq.innerq_block_attention(cache, new, new, q, ws)
    x = float(q[0, 0, 0, 0])
    rest = (n - 1 + np.zeros(t) if cross else n + np.arange(t)) * np.exp(-1.5 * x * 128.0 ** 0.5)
    want = (2.0 + 0.5 * rest) / (1.0 + rest)
    # the tail's weights, all alike: one fp16 rounding (2^-11, of few rows 2^-34 of the strong one), the roundings of scores of 21 nats; moved by a share they move the
    # output by 1.5 rest / (1 + rest)^2 of it.  Sums over tiles in fp32: each of a wavefront's additions is off by 2^-23 of what it has so far, half of its share in
    # the mean, in numerator and normaliser; a row is spread over 64 ranges and more.  63 tokens of the marked block are a step larger (6 % in weight, 1 % in value)
    share = (2.0 ** -11 if t > 32 else 2.0 ** -34 * np.exp(nats)) + 2.0 ** -24 * (12 * 21 + 100) + 63 * 0.07 / n
    sums = 2.0 ** -24 * (n / 32 / 64 + 600)
    bound = 1.5 * rest / (1 + rest) ** 2 * share + sums * (0.5 + want) * rest / (1 + rest) + 1e-6
    left_out = 1.5 * rest / (1 + rest) ** 2 / 256          # what a 256th of the tail is
    assert (bound < 0.6 * left_out).all()
    err = np.abs(out[0].cpu().numpy().astype(np.float64) - want[None, :, None])
    assert (err <= bound[None, :, None]).all(), float((err / bound[None, :, None]).max())
