"""The calls of the 8-bit cache together, as a program uses them: growing conversations, drafts, graphs, streams, beams, and sizes beyond 32 bits."""
import numpy as np
import pytest

from tests import block_cache as bc
from tests import block_reference as ref
from tests.chunk_reference import check

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


@pytest.mark.parametrize("e4,block,paged", [(False, 32, True), (True, 64, False)])
def test_conversations(env, e4, block, paged):
    """Prompts of different lengths, then rounds of rotated drafts of which a part is kept: attention, append, and at the end everything is read back and
    a decoder's cross attention runs over it."""
    torch, iq = env
    rng = np.random.default_rng(6)
    B, Hk, r, cap = 3, 2, 4, 512
    lengths, T = [70, 0, 301], 6
    kept = [[6, 1, 3], [2, 2, 0], [1, 6, 5], [5, 4, 6]]
    total = [n + sum(x[b] for x in kept) for b, n in enumerate(lengths)]
    cache, table = bc.empty(torch, iq, B, Hk * r, Hk, cap, e4, block, total if paged else None, rng, dirt=0x11)
    k, v = bc.keys_and_values(rng, lengths, Hk)
    counts = dev(torch, [0] * B)
    iq.innerq_block_append_ragged(cache, counts, dev(torch, lengths), torch.from_numpy(k).cuda(), torch.from_numpy(v).cuda())
    K, V = ([x[b, :, :n] for b, n in enumerate(lengths)] for x in (k, v))
    cfg = iq.make_config(B, Hk * r, Hk, D, 4, 32, 4, 32, capacity_tokens=cap)               # (for the rotation)
    angle = np.arange(cap)[:, None] * 10000.0 ** (-np.arange(0, D, 2) / D)
    rotation = iq.make_rotation(torch.from_numpy(np.cos(angle).astype(np.float32)).cuda(), torch.from_numpy(np.sin(angle).astype(np.float32)).cuda())
    ws = iq.allocate_block_workspace(cache.cfg, T)
    for keep in kept:
        x = torch.from_numpy(rng.standard_normal((B, T, Hk * (r + 2), D)).astype(np.float16)).cuda().transpose(1, 2)
        qk = x[:, :Hk * (r + 1)]
        iq.innerq_rotate(cfg, rotation, qk, out=qk, n_tokens_dev=counts)
        q, kn, vn = x[:, :Hk * r], x[:, Hk * r:Hk * (r + 1)], x[:, Hk * (r + 1):]
        ns = counts.tolist()
        out = iq.innerq_block_attention_ragged(cache, counts, None, max(ns) + T, kn, vn, q, ws).cpu().numpy()
        iq.innerq_block_append_ragged(cache, counts, dev(torch, keep), kn, vn)
        qh, kh, vh = (y.cpu().numpy() for y in (q, kn, vn))
        for b, n in enumerate(ns):
            full = [np.concatenate([ref.held(y[b], block, e4), z[b].astype(np.float64)], 1) for y, z in ((K, kh), (V, vh))]
            want, bound = ref.attend(qh[b], *full, False, False, ref.causal(n, T))
            check(out[b], want, bound, (n, b))
            K[b], V[b] = (np.concatenate([y[b], z[b][:, :keep[b]]], 1) for y, z in ((K, kh), (V, vh)))
    assert counts.tolist() == total
    back = [torch.full((B, Hk, cap, D), 3.0, dtype=torch.float16, device="cuda") for _ in "kv"]
    iq.innerq_block_read_ragged(cache, counts, None, *back)
    q = torch.from_numpy(rng.standard_normal((B, Hk * r, 2, D)).astype(np.float16)).cuda()
    out = iq.innerq_block_cross_attention_ragged(cache, counts, None, cap, q, ws).cpu().numpy()
    for b, n in enumerate(total):
        bc.check_contents(iq, cache, table, b, K[b], V[b], e4)
        held = [ref.held(y[b], block, e4) for y in (K, V)]
        for got, h in zip(back, held):
            got = got[b].cpu().numpy()
            assert np.abs(got[:, :n] - h).max() <= 2.0 ** -11 * np.abs(h).max() * 1.001 and (got[:, n:] == 3.0).all()
        check(out[b], *ref.attend(q[b].cpu().numpy(), *held, False))


def test_a_step_in_a_graph(env):
    """Attention, then the append, of a ragged step in one graph: replayed, the sequences grow; between replays the program works on its own and the inputs
    change.  Every replay against the same calls made eagerly on a second cache."""
    torch, iq = env
    rng = np.random.default_rng(1)
    B, Hk, r, T = 4, 2, 4, 3
    lengths = [30, 0, 127, 500]
    caches = [bc.filled(torch, iq, np.random.default_rng(2), lengths, Hk * r, Hk, True, 32, capacity=640) for _ in range(2)]
    new = dev(torch, [3, 1, 2, 3])
    x = torch.zeros(B, T, Hk * (r + 2), D, dtype=torch.float16, device="cuda").transpose(1, 2)
    q, k, v = x[:, :Hk * r], x[:, Hk * r:Hk * (r + 1)], x[:, Hk * (r + 1):]
    ws = [iq.allocate_block_workspace(caches[0][0].cfg, T) for _ in range(2)]
    outs = [torch.zeros(B, Hk * r, T, D, dtype=torch.float32, device="cuda") for _ in range(2)]

    def step(i):
        cache, _, counts, _, _ = caches[i]
        iq.innerq_block_attention_ragged(cache, counts, new, 640, k, v, q, ws[i], out=outs[i])
        iq.innerq_block_append_ragged(cache, counts, new, k, v)

    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        step(0)
    assert caches[0][2].tolist() == lengths                # (a capture runs nothing)
    for i in range(20):
        x.copy_(torch.from_numpy(rng.standard_normal(x.shape).astype(np.float16)).cuda())
        ws[0].fill_(i)
        graph.replay()
        step(1)
        if i % 3 == 0:
            torch.cuda.synchronize()
            x.sum().item()
        assert torch.equal(outs[0], outs[1]) and torch.equal(caches[0][2], caches[1][2]), i
    assert caches[0][2].tolist() == [n + 20 * t for n, t in zip(lengths, new.tolist())]
    for name in iq.BLOCK_BUFFER_NAMES:
        assert torch.equal(caches[0][0].buffers[name], caches[1][0].buffers[name]), name


def test_chunks_in_a_graph_and_other_streams(env):
    """A long ragged chunk (sequences of few rows and of many, and a merge) in a graph on a side stream, two calls on two streams at once, and a given stream."""
    torch, iq = env
    rng = np.random.default_rng(4)
    lengths, T, Hk, r = [900, 64, 2000], 90, 2, 4
    cache, _, counts, _, _ = bc.filled(torch, iq, rng, lengths, Hk * r, Hk, False, 64, capacity=2560)
    q, k, v = (torch.from_numpy(rng.standard_normal((3, H, T, D)).astype(np.float16)).cuda() for H in (Hk * r, Hk, Hk))
    new = dev(torch, [90, 5, 33])
    ws = [iq.allocate_block_workspace(cache.cfg, T) for _ in range(3)]
    blank = torch.zeros(3, Hk * r, T, D, device="cuda")
    want = iq.innerq_block_attention_ragged(cache, counts, new, 2200, k, v, q, ws[0], out=blank.clone())
    torch.cuda.synchronize()
    side, other = torch.cuda.Stream(), torch.cuda.Stream()
    outs = [blank.clone() for _ in range(3)]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        iq.innerq_block_attention_ragged(cache, counts, new, 2200, k, v, q, ws[0], out=outs[0])
    assert not outs[0].any()
    for i in range(4):
        for o in outs:
            o.zero_()
        torch.cuda.synchronize()
        graph.replay()
        with torch.cuda.stream(side):
            iq.innerq_block_attention_ragged(cache, counts, new, 2200, k, v, q, ws[1], out=outs[1])
        iq.innerq_block_attention_ragged(cache, counts, new, 2200, k, v, q, ws[2], out=outs[2], stream=other)
        torch.cuda.synchronize()
        for o in outs:
            assert torch.equal(o, want), i


@pytest.mark.parametrize("B,Hk,r,t", [(300, 1, 4, 1), (300, 2, 4, 40), (700, 8, 4, 1), (260, 1, 1, 200)])
def test_batches_without_a_list(env, B, Hk, r, t):
    """More sequences than a list holds, or more heads than one round of work-groups: the same work-groups for every sequence."""
    torch, iq = env
    rng = np.random.default_rng(B + t)
    lengths = [int(n) for n in rng.integers(0, 200, B)]
    lengths[3], lengths[B - 1] = 0, 331
    cache, _, counts, k, v = bc.filled(torch, iq, rng, lengths, Hk * r, Hk, True, 32, capacity=576)
    new = [int(x) for x in rng.integers(0, t + 1, B)]
    new[B - 1] = t
    q, kn, vn = (rng.standard_normal((B, H, t, D)).astype(np.float16) for H in (Hk * r, Hk, Hk))
    ws = iq.allocate_block_workspace(cache.cfg, t)
    out = torch.full((B, Hk * r, t, D), 4.0, device="cuda")
    iq.innerq_block_attention_ragged(cache, counts, dev(torch, new), 576, *(torch.from_numpy(x).cuda() for x in (kn, vn, q)), ws, out=out)
    cross = torch.full((B, Hk * r, t, D), 4.0, device="cuda")
    iq.innerq_block_cross_attention_ragged(cache, counts, dev(torch, new), 400, torch.from_numpy(q).cuda(), ws, out=cross)
    out, cross = out.cpu().numpy(), cross.cpu().numpy()
    for b in [3, 0, 1, 2, B // 2, B - 2, B - 1]:
        n, m = lengths[b], new[b]
        held = [ref.held(x[b, :, :n], 32, True) for x in (k, v)]
        full = [np.concatenate([h, x[b, :, :m].astype(np.float64)], 1) for h, x in zip(held, (kn, vn))]
        many = t * r > 32
        check(out[b, :, :m], *ref.attend(q[b, :, :m], *full, False, many, ref.causal(n, m)), b)
        check(cross[b, :, :m], *ref.attend(q[b, :, :m], *held, False, many), b)
        assert (out[b, :, m:] == 4.0).all() and (cross[b, :, m:] == 4.0).all()


@pytest.mark.parametrize("B,Hk,r,t", [(256, 2, 4, 40), (100, 8, 1, 90), (64, 4, 8, 4)])
def test_lists_of_many_sequences(env, B, Hk, r, t):
    """Few and many rows, splits and none, empty sequences side by side; work-groups of the merge take rows one after the other.  Twice over one workspace, the
    second time with other counts."""
    torch, iq = env
    rng = np.random.default_rng(B)
    lengths = [int(n) for n in rng.integers(0, 100, B)]
    for b, n in zip((0, 7, B // 2, B - 1), (3000, 0, 1500, 2211)):
        lengths[b] = n
    cache, _, counts, k, v = bc.filled(torch, iq, rng, lengths, Hk * r, Hk, True, 32, capacity=3136)
    q, kn, vn = (rng.standard_normal((B, H, t, D)).astype(np.float16) for H in (Hk * r, Hk, Hk))
    ws = iq.allocate_block_workspace(cache.cfg, t)
    for turn in range(2):
        new = [int(x) for x in (rng.integers(0, 3, B) if turn else rng.integers(0, t + 1, B))]
        new[0], new[1], new[B - 1] = (1, t, 2) if turn else (t, 1, t)
        out = torch.full((B, Hk * r, t, D), 4.0, device="cuda")
        iq.innerq_block_attention_ragged(cache, counts, dev(torch, new), 3136, *(torch.from_numpy(x).cuda() for x in (kn, vn, q)), ws, out=out)
        out = out.cpu().numpy()
        for b in [0, 1, 2, 7, B // 2, B - 1]:
            n, m = lengths[b], new[b]
            full = [np.concatenate([ref.held(x[b, :, :n], 32, True), y[b, :, :m].astype(np.float64)], 1) for x, y in ((k, kn), (v, vn))]
            check(out[b, :, :m], *ref.attend(q[b, :, :m], *full, False, t * r > 32, ref.causal(n, m)), (turn, b))
            assert (out[b, :, m:] == 4.0).all()


@pytest.mark.parametrize("t", [1, 100])
def test_rows_of_all_heads_and_sequences_the_same(env, t):
    """New keys and values broadcast over sequences and heads, queries over sequences (strides of zero); and more rows than the merge has work-groups for."""
    torch, iq = env
    rng = np.random.default_rng(t)
    B, Hk, r, n = 8, 8, 4, 2000
    cache, _, counts, k, v = bc.filled(torch, iq, rng, [n] * B, Hk * r, Hk, False, 64, capacity=2112)
    q, kn, vn = (rng.standard_normal((1, H, t, D)).astype(np.float16) for H in (Hk * r, 1, 1))
    rows = [torch.from_numpy(x).cuda().expand(B, H, t, D) for x, H in ((kn, Hk), (vn, Hk), (q, Hk * r))]
    ws = iq.allocate_block_workspace(cache.cfg, t)
    out = torch.empty(B, Hk * r, t, D, device="cuda")
    iq.innerq_block_attention(cache, *rows, ws, out=out)
    for b in (0, B - 1):
        for h in (0, Hk - 1):
            full = [np.concatenate([ref.held(x[b, h:h + 1], 64, False), y[0].astype(np.float64)], 1) for x, y in ((k, kn), (v, vn))]
            at = slice(h * r, h * r + r)
            check(out[b, at].cpu().numpy(), *ref.attend(q[0, at], *full, False, t * r > 32, ref.causal(n, t)), (b, h))
    iq.innerq_block_append(cache, rows[0], rows[1])
    for b in (0, B - 1):
        bc.check_contents(iq, cache, None, b, *(np.concatenate([x[b], np.broadcast_to(y[0], (Hk, t, D))], 1) for x, y in ((k, kn), (v, vn))), False)


def test_a_prefix_of_shared_pages(env):
    """Two sequences whose tables name the same pages for their first 128 tokens and pages of their own behind: read and attended to by both, and left as they are
    by what either appends."""
    torch, iq = env
    rng = np.random.default_rng(12)
    Hk, r, cap, n = 2, 4, 320, 128
    table = torch.tensor([[4, 2, 0, 1, 3], [4, 2, 7, 6, 5]], dtype=torch.int32, device="cuda")
    cfg = iq.make_block_config(2, Hk * r, Hk, type=iq.E4M3, block=32, capacity_tokens=cap, page_pool_pages=8)
    cache = iq.allocate_block_cache(cfg, page_table=table)
    k, v = bc.keys_and_values(rng, [n + 90], Hk)
    own_k, own_v = bc.keys_and_values(rng, [90], Hk)
    K, V = ([x[0], np.concatenate([x[0, :, :n], y[0]], 1)] for x, y in ((k, own_k), (v, own_v)))
    counts = dev(torch, [0, 0])
    prefix = [torch.from_numpy(x[:, :, :n]).cuda().expand(2, Hk, n, D) for x in (k, v)]
    iq.innerq_block_append_ragged(cache, counts, dev(torch, [n, 0]), *prefix)               # (by the first one)
    counts[1] = n
    before = {name: cache.buffers[name].cpu().numpy() for name in iq.BLOCK_BUFFER_NAMES if "open" not in name}
    own = [torch.from_numpy(np.stack([x[b][:, n:] for b in range(2)])).cuda() for x in (K, V)]
    iq.innerq_block_append_ragged(cache, counts, dev(torch, [90, 67]), *own)
    lengths = [n + 90, n + 67]
    for name, was in before.items():
        pages = was.reshape(8, -1)
        assert np.array_equal(cache.buffers[name].cpu().numpy().reshape(8, -1)[[2, 4]], pages[[2, 4]]), name
    for b, m in enumerate(lengths):
        bc.check_contents(iq, cache, table.cpu().numpy(), b, K[b][:, :m], V[b][:, :m], True)
    q = rng.standard_normal((2, Hk * r, 3, D)).astype(np.float16)
    out = iq.innerq_block_cross_attention_ragged(cache, counts, None, cap, torch.from_numpy(q).cuda(), iq.allocate_block_workspace(cfg, 3)).cpu().numpy()
    for b, m in enumerate(lengths):
        check(out[b], *ref.attend(q[b], *(ref.held(x[b][:, :m], 32, True) for x in (K, V)), True), b)


def test_beams_share_a_sequence(env):
    """Cross attention of the beams of a sequence as so many rows of it, their queries token by token out of another layout."""
    torch, iq = env
    rng = np.random.default_rng(3)
    beams, Hk, r = 5, 2, 3
    cache, _, counts, k, v = bc.filled(torch, iq, rng, [200, 77], Hk * r, Hk, False, 32)
    x = torch.from_numpy(rng.standard_normal((2, beams, Hk * r, D)).astype(np.float16)).cuda()             # [sequence, beam, head, D]
    out = torch.empty(2, beams, Hk * r, D, device="cuda")
    iq.innerq_block_cross_attention_ragged(cache, counts, None, 200, x.transpose(1, 2), iq.allocate_block_workspace(cache.cfg, beams), out=out.transpose(1, 2))
    for b, n in enumerate([200, 77]):
        want, bound = ref.attend(x[b].transpose(0, 1).cpu().numpy(), *(ref.held(y[b, :, :n], 32, False) for y in (k, v)), False)
        check(out[b].transpose(0, 1).cpu().numpy(), want, bound)


def test_bad_counts_are_clamped(env):
    """Counts of cached tokens outside 0 .. capacity, of new ones outside 0 .. T: every other sequence is right, nothing beyond the buffers is touched, and a
    clamped sequence is the clamped one's."""
    torch, iq = env
    rng = np.random.default_rng(8)
    cache, _, counts, k, v = bc.filled(torch, iq, rng, [192, 192, 192, 50], 4, 1, False, 64, capacity=192)
    q, kn, vn = (rng.standard_normal((4, H, 3, D)).astype(np.float16) for H in (4, 1, 1))
    ws = iq.allocate_block_workspace(cache.cfg, 3)
    out = torch.full((4, 4, 3, D), 6.0, device="cuda")
    iq.innerq_block_cross_attention_ragged(cache, dev(torch, [5000, -3, 192, 50]), dev(torch, [9, 3, -2, 2]), 192, torch.from_numpy(q).cuda(), ws, out=out)
    got = out.cpu().numpy()
    for b, (n, m) in enumerate([(192, 3), (0, 3), (192, 0), (50, 2)]):
        check(got[b, :, :m], *ref.attend(q[b, :, :m], *(ref.held(x[b, :, :n], 64, False) for x in (k, v)), False), b)
        assert (got[b, :, m:] == 6.0).all()


def test_pages_beyond_32_bits(env):
    """A pool of more than 4 GB a tensor, pages at its end, entries outside of it clamped."""
    torch, iq = env
    rng = np.random.default_rng(9)
    B, H, n, pool, cap = 2, 8, 200, 70000, 320
    table = torch.full((B, cap // 64), 2 ** 31 - 1, dtype=torch.int32, device="cuda")
    pages = rng.permutation(8)[:8] + pool - 8
    table[:, :4] = torch.from_numpy(pages.reshape(2, 4).astype(np.int32)).cuda()
    cfg = iq.make_block_config(B, 2 * H, H, type=iq.E4M3, block=64, capacity_tokens=cap, page_pool_pages=pool)
    assert iq.innerq_block_buffer_bytes(cfg, 0) > 2 ** 32
    cache = iq.allocate_block_cache(cfg, page_table=table)
    k, v = bc.keys_and_values(rng, [n] * B, H)
    kd, vd = torch.from_numpy(k).cuda(), torch.from_numpy(v).cuda()
    iq.innerq_block_append(cache, kd[:, :, :130], vd[:, :, :130])
    iq.innerq_block_append(cache, kd[:, :, 130:], vd[:, :, 130:])
    back = [torch.empty(B, H, n, D, dtype=torch.float16, device="cuda") for _ in "kv"]
    iq.innerq_block_read(cache, 0, *back)
    for t in (1, 40):
        q = rng.standard_normal((B, 2 * H, t, D)).astype(np.float16)
        out = iq.innerq_block_cross_attention(cache, torch.from_numpy(q).cuda(), iq.allocate_block_workspace(cfg, t)).cpu().numpy()
        for b in range(B):
            K, V = (ref.held(x[b], 64, True) for x in (k, v))
            check(out[b], *ref.attend(q[b], K, V, False, 2 * t > 32), (t, b))
            for got, h in zip(back, (K, V)):
                assert np.abs(got[b].cpu().numpy() - h).max() <= 2.0 ** -11 * np.abs(h).max() * 1.001
    assert not cache.buffers["k_codes"][:pool // 2].any()  # (nothing wrapped round to the pool's beginning)


def test_a_sequence_of_the_largest_length(env):
    """2^24 tokens of three heads (more than 4 GB a tensor), every token's rows the same but a marked one's: queries that see it, far to the end."""
    torch, iq = env
    n, H = (1 << 24) - 65, 3
    cfg = iq.make_block_config(1, H, H, type=iq.INT8, block=64, capacity_tokens=1 << 24)
    cache = iq.allocate_block_cache(cfg)
    row = torch.full((1, H, 1, D), 0.5, dtype=torch.float16, device="cuda")
    plain = row.expand(1, H, n, D)
    mark = n - 1000
    for part in (mark, 1, n - mark - 1):                   # (the marked token's block comes in three calls)
        x = row * 4 if part == 1 else plain[:, :, :part]
        iq.innerq_block_append(cache, x, x)
    assert cache.n_tokens == n
    ends = [torch.empty(1, H, 70, D, dtype=torch.float16, device="cuda") for _ in "kv"]
    iq.innerq_block_read(cache, mark - 35, *ends)
    for x in ends:
        # (2.0 is 127 steps; 0.5 is 31.75 of them, rounded to 32 in the marked token's block)
        size = x[0, :, :, 0].float().cpu().numpy()
        assert (size[:, 35] == 2.0).all() and np.abs(np.delete(size, 35, 1) - 0.5).max() < 0.005
    for t in (1, 50):
        # keys 1.5 apart in every channel: 1.5 x sqrt(128) nats times the query
        q = torch.full((1, H, t, D), 25.0 / 1.5 / 128.0 ** 0.5, dtype=torch.float16, device="cuda")
        new = row.expand(1, H, t, D)
        out = iq.innerq_block_attention(cache, new, new, q, iq.allocate_block_workspace(cfg, t))
        x = float(q[0, 0, 0, 0])
        low = np.exp(-1.5 * x * 128.0 ** 0.5)
        want = (2.0 + 0.5 * n * low) / (1.0 + n * low)
        # (63 tokens of the marked block differ by 0.004 in key and value: 2^-20 of all; sums of equal addends: 2^-23 each)
        assert (out - want).abs().max().item() <= want * 2.0 ** -23 * (n / 512 / 16 + 3000) + 1e-3, t


def test_rows_of_another_device_are_refused(env, monkeypatch):
    """Calls launch on the current device: with rows of another one nothing is launched."""
    torch, iq = env
    cache, _ = bc.empty(torch, iq, 1, 4, 1, 64, False, 32)
    q, k, v = (torch.zeros(1, H, 2, D, dtype=torch.float16, device="cuda") for H in (4, 1, 1))
    ws, counts = iq.allocate_block_workspace(cache.cfg, 2), dev(torch, [0])
    monkeypatch.delattr(torch._C, "_cuda_getDevice", raising=False)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 1)
    for call in (lambda: iq.innerq_block_append(cache, k, v), lambda: iq.innerq_block_append_ragged(cache, counts, None, k, v),
                 lambda: iq.innerq_block_read(cache, 0, k, v), lambda: iq.innerq_block_read_ragged(cache, counts, None, None, v),
                 lambda: iq.innerq_block_attention(cache, k, v, q, ws), lambda: iq.innerq_block_attention_ragged(cache, counts, None, 64, k, v, q, ws),
                 lambda: iq.innerq_block_cross_attention(cache, q, ws), lambda: iq.innerq_block_cross_attention_ragged(cache, counts, None, 64, q, ws)):
        with pytest.raises(AssertionError):
            call()
    monkeypatch.undo()
    with pytest.raises(AssertionError):
        iq.innerq_block_cross_attention(cache, q, ws.cpu())
    assert cache.c.n_tokens == 0 and counts.tolist() == [0]
