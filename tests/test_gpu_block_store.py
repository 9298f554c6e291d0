"""Writing the cache in 8 bits with block scales and reading it back, to the bit against the definition."""
import numpy as np
import pytest

from tests import block_cache as bc
from tests import block_reference as ref

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


@pytest.mark.parametrize("e4", [False, True])
@pytest.mark.parametrize("block", [32, 64])
@pytest.mark.parametrize("paged", [False, True])
@pytest.mark.parametrize("how", ["plain", "projection"])
def test_append_in_calls_of_any_length(env, e4, block, paged, how):
    torch, iq = env
    rng = np.random.default_rng(17 + block)
    B, H = 2, 3
    calls = [1, 30, 1, 1, 62, 200, 64, 32, 7, 128, 1]
    n = sum(calls)
    k, v = bc.keys_and_values(rng, [n, n], H)
    cache, table = bc.empty(torch, iq, B, 2 * H, H, 640, e4, block, [n, n] if paged else None, rng, dirt=0x5a)
    at = 0
    for t in calls:
        iq.innerq_block_append(cache, bc.rows(torch, k[:, :, at:at + t], how, rng), bc.rows(torch, v[:, :, at:at + t], how, rng))
        at += t
        assert cache.n_tokens == at
        for b in range(B):
            bc.check_contents(iq, cache, table, b, k[b, :, :at], v[b, :, :at], e4, (at, t))
    # what no block reached is as it was
    for w in "kv":
        codes, scales, _ = bc.contents(iq, cache, table, 0)[w]
        if not paged:
            assert (codes[:, n // block * block // 32:] == 0x5a).all() and (scales[:, n // block:].view(np.uint8) == 0x5a).all()


@pytest.mark.parametrize("e4", [False, True])
@pytest.mark.parametrize("t_new", [1, 5, 64, 65, 200])
@pytest.mark.parametrize("paged", [False, True])
def test_append_ragged(env, e4, t_new, paged):
    torch, iq = env
    rng = np.random.default_rng(31 + t_new)
    block = 64 if t_new % 2 else 32
    H, cap = 2, 448
    start = [0, 1, 31, 63, 64, 100, cap - 1, cap, 200, 333]
    new = [t_new, t_new // 2, 0, t_new, 1, t_new, t_new, t_new, t_new + 9, -4]
    B = len(start)
    takes = [max(0, min(t, t_new, cap - n)) for n, t in zip(start, new)]
    k, v = bc.keys_and_values(rng, [cap + t_new] * B, H)
    cache, table = bc.empty(torch, iq, B, H, H, cap, e4, block, [n + t for n, t in zip(start, takes)] if paged else None, rng, dirt=0x33)
    counts = dev(torch, [0] * B)
    iq.innerq_block_append_ragged(cache, counts, dev(torch, start), torch.from_numpy(k[:, :, :cap]).cuda(), torch.from_numpy(v[:, :, :cap]).cuda())
    assert counts.tolist() == start
    kn, vn = (np.full((B, H, t_new, D), np.nan, dtype=np.float16) for _ in range(2))     # (rows that are not taken are not read)
    for b, (n, t) in enumerate(zip(start, takes)):
        kn[b, :, :t], vn[b, :, :t] = k[b, :, n:n + t], v[b, :, n:n + t]
    iq.innerq_block_append_ragged(cache, counts, dev(torch, new), bc.rows(torch, kn, "projection", rng), bc.rows(torch, vn, "projection", rng))
    assert counts.tolist() == [n + t for n, t in zip(start, takes)]
    for b, (n, t) in enumerate(zip(start, takes)):
        bc.check_contents(iq, cache, table, b, k[b, :, :n + t], v[b, :, :n + t], e4, (n, t))


@pytest.mark.parametrize("t_new", [1, 100])
def test_append_ragged_leaves_alone_what_has_a_bad_count(env, t_new):
    torch, iq = env
    rng = np.random.default_rng(5)
    H, cap = 2, 128
    counts = dev(torch, [-1, cap + 1, 3, 2 ** 31 - 1, -2 ** 31])
    before = counts.tolist()
    cache, _ = bc.empty(torch, iq, 5, H, H, cap, False, 32, dirt=0x77)
    k, v = bc.keys_and_values(rng, [t_new] * 5, H)
    iq.innerq_block_append_ragged(cache, counts, None, torch.from_numpy(k).cuda(), torch.from_numpy(v).cuda())
    assert counts.tolist() == [before[0], before[1], 3 + t_new, before[3], before[4]]
    for name in iq.BLOCK_BUFFER_NAMES:
        x = cache.buffers[name].view(5, -1)
        assert (x[[0, 1, 3, 4]] == 0x77).all(), name


@pytest.mark.parametrize("e4", [False, True])
def test_values_at_the_edges_of_the_codes(env, e4):
    """Ties of the rounding, zero blocks, the largest and smallest fp16 numbers, negative zero."""
    torch, iq = env
    rng = np.random.default_rng(3)
    top = 448.0 if e4 else 127.0
    x = np.zeros((1, 6, 32, D), dtype=np.float16)
    grid = np.arange(-1016, 1017) / 8.0                                     # halves and quarters of steps: a scale of exactly one
    x[0, 0] = rng.choice(grid, (32, D)).astype(np.float16)
    x[0, 0, 0, 0] = top
    x[0, 0, 1, :8] = [0.5, 1.5, 2.5, -0.5, -1.5, 126.5, -126.5, 3.5]
    x[0, 2] = rng.choice([65504.0, -65504.0, 1.0, 0.0], (32, D)).astype(np.float16)
    x[0, 3] = rng.choice([2.0 ** -24, -2.0 ** -24, 0.0, -0.0], (32, D)).astype(np.float16)
    x[0, 4] = (rng.standard_normal((32, D)) * 10.0 ** rng.uniform(-7, 4, (32, D))).astype(np.float16)
    x[0, 5] = (rng.integers(-1792, 1793, (32, D)) / 4.0 if e4 else rng.integers(-254, 255, (32, D)) / 2.0).astype(np.float16)
    x[0, 5, 31, 127] = -top
    v = x[:, ::-1].copy()
    cache, _ = bc.empty(torch, iq, 1, 6, 6, 64, e4, 32)
    iq.innerq_block_append(cache, torch.from_numpy(x).cuda(), torch.from_numpy(v).cuda())
    bc.check_contents(iq, cache, None, 0, x[0], v[0], e4)
    out = torch.empty(1, 6, 32, D, dtype=torch.float16, device="cuda"), torch.empty(1, 6, 32, D, dtype=torch.float16, device="cuda")
    iq.innerq_block_read(cache, 0, *out)
    for got, t in zip(out, (x, v)):
        assert np.array_equal(got[0].cpu().numpy(), expected_rows(t[0], 32, e4))


def expected_rows(x, block, e4):
    """fp16(fl(S * code)) of packed tokens, open ones as they came."""
    n = x.shape[1] // block * block
    codes, scale = ref.pack(x[:, :n], block, e4)
    out = x.copy()
    with np.errstate(over="ignore"):
        out[:, :n] = (codes.astype(np.float32) * scale.repeat(block, 1)[..., None]).astype(np.float16)
    return out


@pytest.mark.parametrize("e4", [False, True])
@pytest.mark.parametrize("block", [32, 64])
@pytest.mark.parametrize("paged", [False, True])
def test_read(env, e4, block, paged):
    torch, iq = env
    rng = np.random.default_rng(9)
    H, n = 2, 300
    cache, _, _, k, v = bc.filled(torch, iq, rng, [n, n], 2 * H, H, e4, block, paged=paged)
    want = [np.stack([expected_rows(x[b], block, e4) for b in range(2)]) for x in (k, v)]
    for first, count in ((0, n), (0, 1), (299, 1), (31, 2), (5, 27), (60, 200), (256, 44), (288, 12), (33, 31), (100, 0)):
        wide = torch.full((2, max(count, 1) + 2, 2 * H + 3, D), 7.0, dtype=torch.float16, device="cuda")
        keys, values = wide[:, 1:1 + count, :H].transpose(1, 2), wide[:, 1:1 + count, H + 1:2 * H + 1].transpose(1, 2)
        if count:
            iq.innerq_block_read(cache, first, keys, values)
        for got, w in ((keys, want[0]), (values, want[1])):
            same = got.cpu().numpy().view(np.uint16) == w[:, :, first:first + count].view(np.uint16)
            assert same.all(), (first, count)
        keys.fill_(7.0)
        values.fill_(7.0)
        assert (wide == 7.0).all()
    one = torch.zeros(2, H, n, D, dtype=torch.float16, device="cuda")
    for i in range(2):
        iq.innerq_block_read(cache, 0, *([one, None] if i == 0 else [None, one]))
        assert np.array_equal(one.cpu().numpy(), want[i])


@pytest.mark.parametrize("paged", [False, True])
def test_read_ragged(env, paged):
    torch, iq = env
    rng = np.random.default_rng(12)
    H, lengths = 2, [0, 1, 40, 64, 333, 511, 130, 200]
    cache, _, counts, k, v = bc.filled(torch, iq, rng, lengths, H, H, True, 64, paged=paged)
    for count in (1, 70, 512):
        for first in (None, [0, 0, 39, -3, 300, 2 ** 31 - 1, -2 ** 31, 131]):
            out = [torch.full((len(lengths), H, count, D), 9.0, dtype=torch.float16, device="cuda") for _ in "kv"]
            iq.innerq_block_read_ragged(cache, counts, None if first is None else dev(torch, first), *out)
            for got, x in zip(out, (k, v)):
                got = got.cpu().numpy()
                for b, n in enumerate(lengths):
                    rows = expected_rows(x[b, :, :n], 64, True)
                    want = np.full((H, count, D), 9.0, dtype=np.float16)
                    for i in range(count):
                        token = (0 if first is None else first[b]) + i
                        if 0 <= token < n:
                            want[:, i] = rows[:, token]
                    assert np.array_equal(got[b], want), (count, b)


def test_counts_beyond_the_capacity_are_clamped_by_a_read(env):
    torch, iq = env
    rng = np.random.default_rng(2)
    cache, _, _, k, v = bc.filled(torch, iq, rng, [192, 192, 192], 1, 1, False, 64, capacity=192)
    out = [torch.full((3, 1, 192, D), 9.0, dtype=torch.float16, device="cuda") for _ in "kv"]
    iq.innerq_block_read_ragged(cache, dev(torch, [5000, -7, 192]), None, *out)
    for got, x in zip(out, (k, v)):
        for b in (0, 2):
            assert np.array_equal(got[b].cpu().numpy(), expected_rows(x[b], 64, False))
        assert (got[1] == 9.0).all()


def test_what_is_read_can_be_written_again(env):
    """Integers: the largest magnitude of a block comes back as 127 steps, so codes survive a round trip when the scale does."""
    torch, iq = env
    rng = np.random.default_rng(8)
    cache, _, _, k, v = bc.filled(torch, iq, rng, [128], 2, 2, False, 32)
    rows = [torch.empty(1, 2, 128, D, dtype=torch.float16, device="cuda") for _ in "kv"]
    iq.innerq_block_read(cache, 0, *rows)
    again, _ = bc.empty(torch, iq, 1, 2, 2, 128, False, 32)
    iq.innerq_block_append(again, *rows)
    for w, x in zip("kv", rows):
        bc.check_contents(iq, again, None, 0, rows[0][0].cpu().numpy(), rows[1][0].cpu().numpy(), False)
