"""Counts in device memory at and beyond the ends of their ranges, for the calls over several new tokens."""
from dataclasses import replace

import numpy as np
import pytest

from oracle import innerq_oracle as orc
from tests.helpers import assert_cache_equal, gpu_config, oracle_config
from tests.rows import projection, rotate, rotation_tables
from tests.test_gpu_append_rows import small

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def env():
    import torch
    from paper_2602_23200_amd import binding as iq
    assert torch.cuda.is_available(), "these tests need the MI355X"
    iq.lib()
    return torch, iq


@pytest.mark.parametrize("T", [1, 40])
@pytest.mark.parametrize("bad", [-1, -(1 << 31), 129, (1 << 31) - 1])
def test_a_sequence_with_a_count_outside_the_cache_takes_nothing(env, bad, T):
    """Neither its buffers nor its count change, whether or not it brings tokens, and its neighbours take theirs."""
    torch, iq = env
    w = small(batch=3, bits=4)
    o = oracle_config(w, capacity=128)
    rng = np.random.default_rng(T)
    cache = iq.allocate_cache(gpu_config(o))
    for x in cache.buffers.values():
        if x is not None:
            x.fill_(77)
    guard = {n: x.clone() for n, x in cache.buffers.items() if x is not None}
    n_dev = torch.tensor([0, bad, 0], dtype=torch.int32, device="cuda")
    o1 = replace(o, batch=1)
    refs = {b: orc.cache_new(o1) for b in (0, 2)}
    for ts in ([T, T, T], [T, T, 0], [T, 0, T]):
        _, _, k, v = projection(torch, rng, 3, T, 1, w.n_kv_heads)
        iq.innerq_append_rotated_ragged(cache, n_dev, torch.tensor(ts, dtype=torch.int32, device="cuda"), k, v)
        for b, ref in refs.items():
            if ts[b]:
                t = min(ts[b], 128 - ref.n_tokens)
                orc.quantize_append(o1, ref, k[b:b + 1, :, :t].cpu().numpy(), v[b:b + 1, :, :t].cpu().numpy())
        assert n_dev.tolist() == [refs[0].n_tokens, bad, refs[2].n_tokens]
    for b, ref in refs.items():
        assert_cache_equal(cache, ref, o1, bsel=slice(b, b + 1), per_sequence=True)
    for name, x in cache.buffers.items():
        if x is not None:
            assert torch.equal(x.view(3, -1)[1], guard[name].view(3, -1)[1]), name


def test_places_at_the_end_of_32_bits(env):
    """Without positions a token stands at n_b + t: sums that 32 bits do not hold are beyond the table, as the largest ones are."""
    torch, iq = env
    rng = np.random.default_rng(4)
    B, T, H = 4, 9, 2
    x = projection(torch, rng, B, T, H, 1)[1]
    cos, sin = rotation_tables(300, 128)
    rot = iq.make_rotation(torch.from_numpy(cos).cuda(), torch.from_numpy(sin).cuda())
    cfg = iq.make_config(B, 4, 2, 128, 2, 32, 4, 128, capacity_tokens=64)
    n = np.array([(1 << 31) - 1, (1 << 31) - 4, -(1 << 31), -5], np.int32)
    y = iq.innerq_rotate(cfg, rot, x, n_tokens_dev=torch.from_numpy(n).cuda()).cpu().numpy()
    place = n.astype(np.int64)[None, :, None] + np.arange(T)[None, None]
    assert np.array_equal(y, rotate(x.cpu().numpy(), cos, sin, place, 128))
