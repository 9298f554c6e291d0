"""Counts in device memory at and beyond the ends of their ranges, for the calls over several new tokens."""
from dataclasses import replace

import numpy as np
import pytest

from oracle import innerq_oracle as orc
from tests.helpers import assert_cache_equal, gpu_config, oracle_config
from tests.rows import projection
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
