"""Attention and cross attention over the cache in 8 bits with block scales, against 64 bits over what the cache stands for."""
import numpy as np
import pytest

from tests import block_cache as bc
from tests import block_reference as ref
from tests.chunk_reference import check

pytestmark = pytest.mark.gpu
D = 128
MANY = 32                                                  # rows of a kv head up to which weights keep 22 bits


@pytest.fixture(scope="module")
def env():
    import torch
    from paper_2602_23200_amd import binding as iq
    assert torch.cuda.is_available(), "these tests need the MI355X"
    iq.lib()
    return torch, iq


def dev(torch, x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def aimed(rng, K, n, t, r, causal):
    """Queries [Hk r, t, D], most of them along the key of one token, which then has nearly all of the weight: the row's own, the first hidden one, one on
    either side of where packed tokens, tiles and ranges end, or any."""
    Hk, N, _ = K.shape
    q = rng.standard_normal((Hk * r, t, D))
    edges = [j for x in (0, 16, 32, 64, 128, n // 64 * 64, n // 32 * 32, n, N) for j in (x - 1, x) if 0 <= j < N]
    for g in range(Hk * r):
        for i in range(t):
            kind = rng.random()
            if kind < 0.25 or N == 0:
                continue
            j = n + i if kind < 0.4 else n + i + 1 if kind < 0.5 else edges[int(rng.integers(len(edges)))] if kind < 0.8 else int(rng.integers(N))
            if 0 <= j < N:
                k = K[g // r, j]
                q[g, i] = k * (12.0 * np.sqrt(D) / max((k ** 2).sum(), 1e-6))
    return np.clip(q, -60000, 60000).astype(np.float16)


def run_uniform(env, rng, n, t, Hq, Hk, e4, block, paged=False, B=2, half=True, cross=False, how="projection", what=""):
    torch, iq = env
    cache, _, _, k, v = bc.filled(torch, iq, rng, [n] * B, Hq, Hk, e4, block, capacity=-(-(n + t) // 64) * 64, paged=paged)
    kn, vn = bc.keys_and_values(rng, [t] * B, Hk)
    K, V, q = [], [], []
    for b in range(B):
        K.append(ref.held(k[b, :, :n], block, e4))
        V.append(ref.held(v[b, :, :n], block, e4))
        if not cross:
            K[b] = np.concatenate([K[b], kn[b].astype(np.float64)], 1)
            V[b] = np.concatenate([V[b], vn[b].astype(np.float64)], 1)
        q.append(aimed(rng, K[b], n, t, Hq // Hk, not cross))
    ws = iq.allocate_block_workspace(cache.cfg, t)
    ws.fill_(0xff)                                         # (NaN everywhere)
    out = torch.empty(B, t, Hq, D, dtype=torch.float16 if half else torch.float32, device="cuda").transpose(1, 2)
    rows = [bc.rows(torch, x, how, rng) for x in (np.stack(q), kn, vn)]
    if cross:
        iq.innerq_block_cross_attention(cache, rows[0], ws, out=out)
    else:
        iq.innerq_block_attention(cache, rows[1], rows[2], rows[0], ws, out=out)
    got = out.cpu().numpy()
    worst = 0.0
    for b in range(B):
        want, bound = ref.attend(q[b], K[b], V[b], half, t * (Hq // Hk) > MANY, None if cross else ref.causal(n, t))
        worst = max(worst, check(got[b], want, bound, (what, n, t, Hq, Hk, e4, block, b)))
    return worst


@pytest.mark.parametrize("e4", [False, True])
@pytest.mark.parametrize("block", [32, 64])
@pytest.mark.parametrize("n", [0, 1, 31, 32, 33, 64, 127, 500, 1025, 4100])
def test_one_token(env, e4, block, n):
    rng = np.random.default_rng(n + block)
    run_uniform(env, rng, n, 1, 8, 2, e4, block, paged=n % 2 == 1)


@pytest.mark.parametrize("r", [1, 2, 3, 4, 5, 8, 16, 17, 40])
def test_query_heads_of_a_kv_head(env, r):
    rng = np.random.default_rng(r)
    run_uniform(env, rng, 333, 1, 2 * r, 2, r % 2 == 0, 32, half=r % 3 == 0)
    run_uniform(env, rng, 170, 3, 2 * r, 2, r % 2 == 1, 64, half=r % 3 == 1)


@pytest.mark.parametrize("e4", [False, True])
@pytest.mark.parametrize("t", [2, 5, 8, 16, 17, 33, 64, 130, 300])
@pytest.mark.parametrize("n", [0, 40, 700])
def test_several_tokens(env, e4, t, n):
    rng = np.random.default_rng(t + n)
    run_uniform(env, rng, n, t, 4, 1, e4, 64 if t % 2 else 32, paged=t % 3 == 0, half=t % 4 != 1, how="plain" if t % 2 else "projection")


@pytest.mark.parametrize("e4", [False, True])
@pytest.mark.parametrize("t,n", [(1, 0), (1, 5), (1, 64), (1, 1437), (4, 99), (30, 640), (100, 333), (300, 1), (65, 2048)])
def test_cross(env, e4, t, n):
    rng = np.random.default_rng(t + n)
    run_uniform(env, rng, n, t, 6, 3, e4, 32, paged=n % 2 == 0, half=t % 2 == 1, cross=True)


@pytest.mark.parametrize("t_new", [1, 6, 40, 200])
@pytest.mark.parametrize("cross", [False, True])
@pytest.mark.parametrize("paged", [False, True])
def test_ragged(env, t_new, cross, paged):
    torch, iq = env
    rng = np.random.default_rng(t_new + 2 * cross)
    lengths = [0, 1, 700, 64, 33, 2500, 130, 31, 96]
    new = [t_new, 0, t_new // 2 + 1, 1, t_new, t_new, 0, t_new, max(1, t_new - 1)]
    Hq, Hk, e4, block, B = 8, 2, t_new % 4 == 2, 64 if paged else 32, len(lengths)
    cache, _, counts, k, v = bc.filled(torch, iq, rng, lengths, Hq, Hk, e4, block, paged=paged)
    kn, vn = bc.keys_and_values(rng, [t_new] * B, Hk)
    q = np.zeros((B, Hq, t_new, D), dtype=np.float16)
    K, V = [], []
    for b, (n, t) in enumerate(zip(lengths, new)):
        K.append(ref.held(k[b, :, :n], block, e4))
        V.append(ref.held(v[b, :, :n], block, e4))
        if not cross:
            K[b] = np.concatenate([K[b], kn[b, :, :t].astype(np.float64)], 1)
            V[b] = np.concatenate([V[b], vn[b, :, :t].astype(np.float64)], 1)
        q[b, :, :t] = aimed(rng, K[b], n, t, Hq // Hk, not cross)
        q[b, :, t:], kn[b, :, t:], vn[b, :, t:] = np.nan, np.nan, np.nan     # (rows beyond a count are not read)
    rows = [bc.rows(torch, x, "projection", rng) for x in (q, kn, vn)]
    most = max(n + (0 if cross else t) for n, t in zip(lengths, new))
    for bound_by in (most, cache.cfg.capacity_tokens):
        ws = iq.allocate_block_workspace(cache.cfg, t_new)
        ws.fill_(0xff)
        out = torch.full((B, t_new, Hq, D), 5.0, dtype=torch.float32, device="cuda").transpose(1, 2)
        if cross:
            iq.innerq_block_cross_attention_ragged(cache, counts, dev(torch, new), bound_by, rows[0], ws, out=out)
        else:
            iq.innerq_block_attention_ragged(cache, counts, dev(torch, new), bound_by, rows[1], rows[2], rows[0], ws, out=out)
        got = out.cpu().numpy()
        for b, (n, t) in enumerate(zip(lengths, new)):
            many = t * (Hq // Hk) > MANY
            want, bound = ref.attend(q[b, :, :t], K[b], V[b], False, many, None if cross else ref.causal(n, t))
            check(got[b, :, :t], want, bound, (n, t))
            assert (got[b, :, t:] == 5.0).all()
        assert counts.tolist() == lengths
    if cross:
        assert (got[0] == 0.0).all()                       # (no token: zero)
