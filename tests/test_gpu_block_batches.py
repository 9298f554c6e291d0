"""Ragged attention over the 8-bit cache in batches of any number of sequences whose longest one has many rows: every sequence is held to what its own number of
rows promises (weights of 22 bits up to 32 rows of a kv head).  Keys are multiples of 1/32 of one magnitude for all channels, queries powers of two, so that scores are
exact and weights of 11 bits lie beyond the bound of 22 (tests/test_gpu_block_scales.py has it)."""
import numpy as np
import pytest

from tests import block_cache as bc
from tests import block_reference as ref
from tests.test_gpu_block_scales import promised

pytestmark = pytest.mark.gpu
D = 128


@pytest.fixture(scope="module")
def env():
    import torch
    from paper_2602_23200_amd import binding as iq
    assert torch.cuda.is_available(), "these tests need the MI355X"
    iq.lib()
    return torch, iq


def dev(torch, x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def exact_rows(rng, shape):
    """Keys [.., T, D] whose blocks of 32 have a scale of 1/32, values, and queries for them."""
    k = np.broadcast_to(rng.integers(-64, 65, (*shape[:-1], 1)) / 32.0, shape).astype(np.float16)
    k[..., ::32, :] = 127.0 / 32
    return k, rng.standard_normal(shape, dtype=np.float32).astype(np.float16)


def checked(q, got, K, V, hidden, many, r, what):
    for h in range(len(K)):
        rows = slice(h * r, h * r + r)
        want, bound = promised(q[rows], K[h], V[h], hidden, many) if len(K[h]) else (np.zeros_like(got[rows]), 1e-30)
        assert (np.abs(got[rows] - want) <= bound).all(), (what, h, float((np.abs(got[rows] - want) / bound).max()))


@pytest.mark.parametrize("B,Hk,r,t,longest", [(100, 2, 4, 40, 500), (255, 1, 1, 90, 500), (256, 1, 4, 12, 500), (257, 1, 4, 12, 500), (257, 2, 4, 40, 500),
                                              (257, 1, 4, 20, 5000), (300, 1, 1, 90, 500), (520, 1, 4, 20, 500)])
@pytest.mark.parametrize("paged", [False, True])
@pytest.mark.parametrize("block", [32, 64])
def test_every_sequence_has_its_own_precision(env, B, Hk, r, t, longest, paged, block):
    torch, iq = env
    rng = np.random.default_rng(B + t)
    lengths = [int(n) for n in rng.integers(0, 90, B)]
    new = [int(x) for x in rng.integers(0, 3, B)]
    looked = sorted({0, 1, 7, 99, B // 2, B // 2 + 1, 173, 174, 254, 255, 256, 259, 260, 261, 347, B - 2, B - 1} & set(range(B)))
    for i, b in enumerate(looked):
        new[b] = (t, 1, 32 // r, 0, 32 // r + 1, t - 1, 2)[i % 7]
        lengths[b] = (longest, 0, 131, 64, 33, 1, 40)[i % 7]
    cap = -(-(longest + 76) // 64) * 64
    cache, _ = bc.empty(torch, iq, B, Hk * r, Hk, cap, False, block, lengths if paged else None, rng)
    k, v = exact_rows(rng, (B, Hk, max(lengths), D))
    counts = dev(torch, [0] * B)
    iq.innerq_block_append_ragged(cache, counts, dev(torch, lengths), torch.from_numpy(k).cuda(), torch.from_numpy(v).cuda())
    kn, vn = exact_rows(rng, (B, Hk, t, D))
    q = (np.where(rng.random((B, Hk * r, t, D)) < 0.9, 0.0625, -0.0625)).astype(np.float16)
    rows = [bc.rows(torch, x, "projection", rng) for x in (kn, vn, q)]
    ws = iq.allocate_block_workspace(cache.cfg, t)
    ws.fill_(0xff)
    out, cross = (torch.full((B, t, Hk * r, D), 4.0, device="cuda").transpose(1, 2) for _ in range(2))
    iq.innerq_block_attention_ragged(cache, counts, dev(torch, new), cap, *rows, ws, out=out)
    iq.innerq_block_cross_attention_ragged(cache, counts, dev(torch, new), max(lengths), rows[2], ws, out=cross)
    assert counts.tolist() == lengths
    out, cross = (x.cpu().numpy().astype(np.float64) for x in (out, cross))
    for b in looked:
        n, m = lengths[b], new[b]
        held = [ref.held(x[b, :, :n], block, False) for x in (k, v)]
        assert np.array_equal(held[0], k[b, :, :n].astype(np.float64))
        full = [np.concatenate([h, x[b, :, :m].astype(np.float64)], 1) for h, x in zip(held, (kn, vn))]
        checked(q[b, :, :m], out[b, :, :m], *full, ref.causal(n, m), m * r > 32, r, (b, n, m))
        checked(q[b, :, :m], cross[b, :, :m], *held, np.zeros((m, n), dtype=bool), m * r > 32, r, (b, n, m, "cross"))
    for b in range(B):
        assert (out[b, :, new[b]:] == 4.0).all() and (cross[b, :, new[b]:] == 4.0).all(), b


def test_a_large_batch_in_a_graph(env):
    """Parts of a batch one behind the other in a graph, replayed with other counts."""
    torch, iq = env
    rng = np.random.default_rng(3)
    B, Hk, r, t = 300, 1, 4, 20
    lengths = [int(n) for n in rng.integers(0, 200, B)]
    cache, _, counts, _, _ = bc.filled(torch, iq, rng, lengths, Hk * r, Hk, False, 32, capacity=576)
    q, k, v = (torch.from_numpy(rng.standard_normal((B, H, t, D)).astype(np.float16)).cuda() for H in (Hk * r, Hk, Hk))
    ws = [iq.allocate_block_workspace(cache.cfg, t) for _ in range(2)]
    new = dev(torch, [t] * B)
    outs = [torch.zeros(B, Hk * r, t, D, device="cuda") for _ in range(2)]
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        iq.innerq_block_attention_ragged(cache, counts, new, 300, k, v, q, ws[0], out=outs[0])
    for i in range(6):
        new.copy_(dev(torch, [int(x) for x in rng.integers(0, t + 1, B)]))
        ws[0].fill_(i)
        graph.replay()
        iq.innerq_block_attention_ragged(cache, counts, new, 300, k, v, q, ws[1], out=outs[1])
        torch.cuda.synchronize()
        assert torch.equal(outs[0], outs[1]), i
