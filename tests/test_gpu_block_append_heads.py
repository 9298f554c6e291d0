"""Ragged appends of up to a block of rows to caches of few and of many heads (a work-group has a sequence, or a wavefront a block), to the bit."""
import numpy as np
import pytest

from tests import block_cache as bc

pytestmark = pytest.mark.gpu
D = 128


@pytest.fixture(scope="module")
def env():
    import torch
    from paper_2602_23200_amd import binding as iq
    assert torch.cuda.is_available(), "these tests need the MI355X"
    iq.lib()
    return torch, iq


@pytest.mark.parametrize("H", [1, 8, 9, 16, 17, 40])
@pytest.mark.parametrize("block,t_new", [(32, 1), (32, 4), (32, 5), (32, 32), (64, 8), (64, 9), (64, 64)])
@pytest.mark.parametrize("paged", [False, True])
def test_steps(env, H, block, t_new, paged):
    torch, iq = env
    rng = np.random.default_rng(H + t_new)
    cap, start = 192, [0, block - 1, block, 63, 128 - t_new, 190, 192]
    new = [t_new, 1, 0, t_new, t_new, t_new, t_new]
    B = len(start)
    takes = [min(t, cap - n) for n, t in zip(start, new)]
    k, v = bc.keys_and_values(rng, [cap + t_new] * B, H)
    cache, table = bc.empty(torch, iq, B, H, H, cap, False, block, [n + t for n, t in zip(start, takes)] if paged else None, rng, dirt=0x33)
    counts = torch.zeros(B, dtype=torch.int32, device="cuda")
    first = torch.tensor(start, dtype=torch.int32, device="cuda")
    iq.innerq_block_append_ragged(cache, counts, first, torch.from_numpy(k[:, :, :cap]).cuda(), torch.from_numpy(v[:, :, :cap]).cuda())
    kn, vn = (np.full((B, H, t_new, D), np.nan, dtype=np.float16) for _ in range(2))
    for b, (n, t) in enumerate(zip(start, takes)):
        kn[b, :, :t], vn[b, :, :t] = k[b, :, n:n + t], v[b, :, n:n + t]
    iq.innerq_block_append_ragged(cache, counts, torch.tensor(new, dtype=torch.int32, device="cuda"), bc.rows(torch, kn, "projection", rng),
                                  bc.rows(torch, vn, "projection", rng))
    assert counts.tolist() == [n + t for n, t in zip(start, takes)]
    for b, (n, t) in enumerate(zip(start, takes)):
        bc.check_contents(iq, cache, table, b, k[b, :, :n + t], v[b, :, :n + t], False, (n, t))
