"""innerq_rotate against the formula: bit for bit in 32 bits with every operation rounded, and in 64 bits."""
import numpy as np
import pytest

from tests.rows import projection, rotate, rotation_tables

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def env():
    import torch
    from paper_2602_23200_amd import binding as iq
    assert torch.cuda.is_available(), "these tests need the MI355X"
    iq.lib()
    return torch, iq


def config(iq, B, Hq=4, Hk=2):
    return iq.make_config(B, Hq, Hk, 128, 2, 32, 4, 128, capacity_tokens=64)


def sections(P, n):
    """Axis of every pair: uneven sections, their borders inside a group of eight pairs."""
    cut = [0, P // 4 + 1, P // 4 + 1 + (P - P // 4) // 2, P] if n == 3 else [0, P // 2 - 3, P]
    return [a for a in range(n) for _ in range(cut[a], cut[a + 1])]


def run(torch, iq, rng, B, T, H, rot_dim, interleaved, n_axes, in_place=False, axes=None, x=None, positions=None, rows=333):
    cos, sin = rotation_tables(rows, rot_dim)
    axes = axes if axes is not None else None if n_axes == 1 else sections(rot_dim // 2, n_axes)
    rot = iq.make_rotation(torch.from_numpy(cos).cuda(), torch.from_numpy(sin).cuda(), interleaved, axes)
    if x is None:
        x = projection(torch, rng, B, T, H, 1)[1]
    if positions is None:
        positions = rng.integers(-3, rows + 40, (n_axes, B, T)).astype(np.int32)     # (outside the table: clamped into it)
    before = x.cpu().numpy()
    y = iq.innerq_rotate(config(iq, B), rot, x, out=x if in_place else None, positions=torch.from_numpy(positions).cuda())
    got = y.cpu().numpy()
    want = rotate(before, cos, sin, positions, rot_dim, interleaved, axes)
    assert np.array_equal(got.view(np.uint16), want.view(np.uint16))
    exact = rotate(before, cos, sin, positions, rot_dim, interleaved, axes, np.float64)
    # two products and a sum in fp32 (3 x 2^-24 of the products' magnitude, at most sqrt(2) of the pair's norm), one rounding to fp16
    # (2^-11 of the result, 2^-25 where it is a denormal)
    norm = np.sqrt((before.astype(np.float64) ** 2).max())
    assert np.all(np.abs(got - exact) <= np.abs(exact) * 2.0 ** -11 + 3 * 2.0 ** -24 * 1.5 * norm + 2.0 ** -25)


@pytest.mark.parametrize("rot_dim", [16, 64, 96, 128])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("n_axes", [1, 2, 3])
def test_forms(env, rot_dim, interleaved, n_axes):
    torch, iq = env
    run(torch, iq, np.random.default_rng(rot_dim + n_axes), 3, 37, 5, rot_dim, interleaved, n_axes)


@pytest.mark.parametrize("B,T,H", [(1, 1, 1), (1, 1, 40), (7, 1, 40), (1, 4097, 3), (2, 1024, 40), (300, 1, 9), (33, 31, 1)])
@pytest.mark.parametrize("in_place", [False, True])
def test_sizes(env, B, T, H, in_place):
    torch, iq = env
    run(torch, iq, np.random.default_rng(B + T), B, T, H, 128, False, 1, in_place)


def test_axes_of_pairs_need_not_be_sections(env):
    torch, iq = env
    run(torch, iq, np.random.default_rng(5), 2, 20, 3, 128, False, 3, axes=[(i * 7 + i // 5) % 3 for i in range(64)])


def test_what_lies_between_the_rows_stays(env):
    """Rotating queries and keys in place in a projection's output leaves the values and the spare head alone."""
    torch, iq = env
    rng = np.random.default_rng(9)
    x, q, k, v = projection(torch, rng, 2, 50, 4, 2)
    before = x.cpu().numpy()
    run(torch, iq, rng, 2, 50, 6, 128, False, 1, True, x=x.transpose(1, 2)[:, :6])
    assert np.array_equal(x.cpu().numpy()[:, :, 6:], before[:, :, 6:])
    assert not np.array_equal(x.cpu().numpy()[:, :, :6], before[:, :, :6])


def test_one_row_for_all(env):
    """An input stride of 0: the same row for every token."""
    torch, iq = env
    rng = np.random.default_rng(3)
    row = torch.from_numpy(rng.standard_normal((2, 3, 1, 128)).astype(np.float16)).cuda()
    run(torch, iq, rng, 2, 19, 3, 128, True, 1, x=row.expand(2, 3, 19, 128))


def test_place_in_the_sequence(env):
    """Without positions a token stands behind the cached ones; counts on the device; rows beyond a count are left alone."""
    torch, iq = env
    rng = np.random.default_rng(4)
    B, T, H = 3, 24, 2
    x = projection(torch, rng, B, T, H, 1)[1]
    cos, sin = rotation_tables(300, 128)
    rot = iq.make_rotation(torch.from_numpy(cos).cuda(), torch.from_numpy(sin).cuda())
    along = np.arange(T)[None, None]
    y = iq.innerq_rotate(config(iq, B), rot, x, n_tokens=77).cpu().numpy()
    assert np.array_equal(y, rotate(x.cpu().numpy(), cos, sin, np.broadcast_to(77 + along, (1, B, T)), 128))
    n, t = np.array([0, 13, 290], np.int32), np.array([24, 0, 7], np.int32)
    out = torch.full((B, H, T, 128), 5.0, dtype=torch.float16, device="cuda")
    iq.innerq_rotate(config(iq, B), rot, x, out=out, n_tokens_dev=torch.from_numpy(n).cuda(), t_new_dev=torch.from_numpy(t).cuda())
    want = rotate(x.cpu().numpy(), cos, sin, n[None, :, None] + along, 128)
    for b in range(B):
        assert np.array_equal(out[b, :, :t[b]].cpu().numpy(), want[b, :, :t[b]])
        assert (out[b, :, t[b]:] == 5.0).all()


def test_inverse(env):
    """The sines negated turn back: two roundings of 2^-11 of the pair's norm (at most sqrt(2) of its larger channel) each way."""
    torch, iq = env
    rng = np.random.default_rng(6)
    x = projection(torch, rng, 2, 65, 4, 1)[1]
    cos, sin = rotation_tables(100, 128)
    c, s = torch.from_numpy(cos).cuda(), torch.from_numpy(sin).cuda()
    y = iq.innerq_rotate(config(iq, 2), iq.make_rotation(c, s), x)
    z = iq.innerq_rotate(config(iq, 2), iq.make_rotation(c, -s), y).cpu().numpy().astype(np.float64)
    w = x.cpu().numpy().astype(np.float64)
    norm = np.sqrt(w[..., :64] ** 2 + w[..., 64:] ** 2)
    assert (np.abs(z - w) <= np.concatenate([norm, norm], -1) * 2.0 ** -11 * 3).all()


def test_another_stream_and_replays(env):
    """Recorded in a graph with counts on the device, replayed with other counts and inputs."""
    torch, iq = env
    rng = np.random.default_rng(8)
    B, T, H = 2, 16, 3
    x = projection(torch, rng, B, T, H, 1)[1]
    cos, sin = rotation_tables(500, 128)
    rot = iq.make_rotation(torch.from_numpy(cos).cuda(), torch.from_numpy(sin).cuda())
    cfg, n = config(iq, B), torch.zeros(B, dtype=torch.int32, device="cuda")
    out = torch.empty(B, H, T, 128, dtype=torch.float16, device="cuda")
    iq.innerq_rotate(cfg, rot, x, out=out, n_tokens_dev=n)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        iq.innerq_rotate(cfg, rot, x, out=out, n_tokens_dev=n)
    for step in range(3):
        n.copy_(torch.tensor([step * 5, 100 + step]))
        x.mul_(0.5)
        graph.replay()
        torch.cuda.synchronize()
        want = rotate(x.cpu().numpy(), cos, sin, n.cpu().numpy()[None, :, None] + np.arange(T)[None, None], 128)
        assert np.array_equal(out.cpu().numpy(), want)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    out.zero_()
    side.wait_stream(torch.cuda.current_stream())
    iq.innerq_rotate(cfg, rot, x, out=out, n_tokens_dev=n, stream=side)
    side.synchronize()
    assert np.array_equal(out.cpu().numpy(), want)


def test_offsets_beyond_32_bits(env):
    """2.3 billion elements: rows at both ends against the formula."""
    torch, iq = env
    T, H = 375000, 48
    x = torch.empty(1, T, H, 128, dtype=torch.float16, device="cuda")
    for part in x[0].split(25000):
        part.normal_()
    cos, sin = rotation_tables(T, 128)
    rot = iq.make_rotation(torch.from_numpy(cos).cuda(), torch.from_numpy(sin).cuda())
    picks = np.array([0, 1, 187499, T - 2, T - 1])
    before = x[:, picks].transpose(1, 2).cpu().numpy()
    v = x.transpose(1, 2)
    iq.innerq_rotate(config(iq, 1), rot, v, out=v)
    got = x[:, picks].transpose(1, 2).cpu().numpy()
    assert np.array_equal(got, rotate(before, cos, sin, picks[None, None], 128))
