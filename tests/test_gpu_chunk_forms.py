"""Every compiled form of innerq_chunk_attention (pairs of widths, groups, wavefronts a tile, contiguous and paged stores) against attention
in 64 bits over the same operands, with queries that put their weight on one token: the borders of the cache, the row's own token, the first
hidden one (tests/chunk_reference.py; tests/test_chunk_reference_cpu.py shows which mistakes that finds)."""
import numpy as np
import pytest

from oracle import innerq_oracle as orc
from tests.chunk_reference import aimed, attend, borders_of, check, operands
from tests.helpers import oracle_config
from tests.rows import projection
from tests.test_gpu_chunk import filled, small

pytestmark = pytest.mark.gpu
SYM, ASYM, HYBRID = orc.SYM, orc.ASYM, orc.HYBRID
PAIRS = [(k, v) for k in (2, 3, 4) for v in (2, 3, 4)]
MODES = [(HYBRID, HYBRID), (SYM, HYBRID), (ASYM, SYM), (SYM, SYM), (HYBRID, ASYM)]
# (new tokens, query heads a kv head): up to 32 rows; up to 128; more, most keys cached; more, most keys new
SIZES = {"few": (5, 4), "four": (31, 3), "eight": (47, 4), "new": (290, 1)}


@pytest.fixture(scope="module")
def env():
    import torch
    from paper_2602_23200_amd import binding as iq
    assert torch.cuda.is_available(), "these tests need the MI355X"
    iq.lib()
    return torch, iq


def rows_of(torch, rng, o1, refs, lengths, ts, T, r, heads):
    """New rows as a projection's parts and queries aimed at the tokens of every sequence; padding is NaN."""
    x, q, k, v = projection(torch, rng, len(lengths), T, r * heads, heads)
    spread = torch.from_numpy((1.0 + np.abs(rng.standard_t(3, (1, heads, 1, 128)))).astype(np.float16)).cuda()
    k.mul_(spread)
    for b, (n, t) in enumerate(zip(lengths, ts)):
        if t:
            K = operands(o1, refs[b], "k", k[b, :, :t].cpu().numpy())
            q[b, :, :t] = torch.from_numpy(aimed(rng, K, n, t, r, borders_of(o1, n, t))).cuda()
        x[b, t:] = float("nan")
    return q, k, v


def compare(o1, refs, ts, q, k, v, out, half, what):
    worst = 0.0
    for b, t in enumerate(ts):
        if t:
            qb, kb, vb = (y[b, :, :t].cpu().numpy() for y in (q, k, v))
            want, bound = attend(qb, operands(o1, refs[b], "k", kb), operands(o1, refs[b], "v", vb), half)
            worst = max(worst, check(out[b, :, :t].float().cpu().numpy(), want, bound, f"{what} sequence {b}"))
    return worst


@pytest.mark.parametrize("paged", [False, True])
@pytest.mark.parametrize("group", [32, 64])
@pytest.mark.parametrize("pair", PAIRS)
def test_widths(env, pair, group, paged):
    """One count for all: every row form of a pair of widths, behind two sequences of the same length."""
    torch, iq = env
    at = PAIRS.index(pair) + 3 * (group == 64) + paged
    modes, n = MODES[at % 5], [405, 213, 340, 628][at % 4]
    rng = np.random.default_rng(1000 * at + group)
    for name, (t, r) in SIZES.items():
        w = small(batch=2, n_q_heads=2 * r, n_kv_heads=2, bits=pair[0], group=group, k_mode=modes[0], v_mode=modes[1], w_recent=[48, 130, 64][at % 3])
        o = oracle_config(w, capacity=1024, v_bits=pair[1])
        cache, o1, refs, counts = filled(torch, iq, o, [n, n], rng, pages=at if paged else None)
        half = (at + t) % 2 == 0
        q, k, v = rows_of(torch, rng, o1, refs, [n, n], [t, t], t, r, 2)
        ws = iq.allocate_chunk_workspace(cache.cfg, t)
        ws.fill_(255)
        out = torch.empty(2, t, 2 * r, 128, dtype=torch.float16 if half else torch.float32, device="cuda").transpose(1, 2)
        iq.innerq_chunk_attention(cache, k, v, q, ws, out=out)
        print(name, compare(o1, refs, [t, t], q, k, v, out, half, name), flush=True)


@pytest.mark.parametrize("paged", [False, True])
@pytest.mark.parametrize("pair", PAIRS)
def test_widths_of_ragged_batches(env, pair, paged):
    """Counts on the device: sequences of few and of many rows in one batch, empty caches and empty chunks among them."""
    torch, iq = env
    at = PAIRS.index(pair) + paged
    group, modes = (32, 64)[at % 2], MODES[(at + 1) % 5]
    rng = np.random.default_rng(at)
    w = small(batch=5, n_q_heads=8, n_kv_heads=2, bits=pair[0], group=group, k_mode=modes[0], v_mode=modes[1], w_recent=[48, 130, 64][at % 3])
    o = oracle_config(w, capacity=1024, v_bits=pair[1])
    lengths, ts = [0, 3, 417, 700, 256], [37, 8, 0, 70, 1]
    cache, o1, refs, counts = filled(torch, iq, o, lengths, rng, pages=at if paged else None)
    q, k, v = rows_of(torch, rng, o1, refs, lengths, ts, 70, 4, 2)
    ws = iq.allocate_chunk_workspace(cache.cfg, 70)
    ws.fill_(255)
    out = torch.full((5, 70, 8, 128), 5.0, device="cuda").transpose(1, 2)
    iq.innerq_chunk_attention_ragged(cache, counts, torch.tensor(ts, dtype=torch.int32, device="cuda"), 800, k, v, q, ws, out=out)
    print(compare(o1, refs, ts, q, k, v, out, False, str(pair)), flush=True)
    for b, t in enumerate(ts):
        assert (out[b, :, t:] == 5.0).all()


@pytest.mark.parametrize("n", [0, 1, 4, 53, 85, 116, 117, 150])
def test_short_caches(env, n):
    """Caches that end in the sink, in the window and shortly beyond it."""
    torch, iq = env
    rng = np.random.default_rng(n)
    for bits, group, (t, r) in ((2, 32, (1, 4)), (4, 32, (33, 2)), (3, 64, (140, 1)), (4, 64, (9, 3))):
        w = small(n_q_heads=2 * r, n_kv_heads=2, bits=bits, group=group)
        o = oracle_config(w, capacity=512)
        cache, o1, refs, counts = filled(torch, iq, o, [n], rng)
        q, k, v = rows_of(torch, rng, o1, refs, [n], [t], t, r, 2)
        out = iq.innerq_chunk_attention(cache, k, v, q, iq.allocate_chunk_workspace(cache.cfg, t))
        print(compare(o1, refs, [t], q, k, v, out, False, f"{bits} {group} {t}"), flush=True)


def shared_list(torch, iq, rng, B, heads, r, lengths, ts, capacity):
    w = small(batch=B, n_q_heads=heads * r, n_kv_heads=heads, bits=4)
    o = oracle_config(w, capacity=capacity)
    cache, o1, refs, counts = filled(torch, iq, o, lengths, rng)
    T = max(ts)
    q, k, v = rows_of(torch, rng, o1, refs, lengths, ts, T, r, heads)
    ws = iq.allocate_chunk_workspace(cache.cfg, T)
    ws.fill_(255)
    guard = ws.clone()
    out = torch.full((B, T, heads * r, 128), 5.0, device="cuda").transpose(1, 2)
    iq.innerq_chunk_attention_ragged(cache, counts, torch.tensor(ts, dtype=torch.int32, device="cuda"), capacity, k, v, q, ws, out=out)
    print(compare(o1, refs, ts, q, k, v, out, False, f"{B} x {heads}"), flush=True)
    return ws, guard


def test_a_list_of_more_units_than_items(env):
    """Over 512 (head, block of rows) units in either launch: no sequence is split, and nothing is written to the partial results."""
    torch, iq = env
    rng = np.random.default_rng(1)
    B, heads = 40, 16
    lengths = [int(x) for x in rng.integers(0, 300, B)]
    few = [int(x) for x in rng.integers(1, 9, B)]
    ws, guard = shared_list(torch, iq, rng, B, heads, 4, lengths, few, 384)
    assert torch.equal(ws[2048:], guard[2048:])             # (behind the table)
    ws, guard = shared_list(torch, iq, rng, B, heads, 4, lengths, [9 + x for x in few], 384)
    assert torch.equal(ws[2048:], guard[2048:])


def test_a_list_whose_ranges_are_lengthened(env):
    """Ranges of the least length would be more than 512 items: they are lengthened until they fit, some sequences are split and others are not."""
    torch, iq = env
    rng = np.random.default_rng(2)
    lengths = [3000, 20, 2500, 100, 700, 3100]
    shared_list(torch, iq, rng, 6, 16, 1, lengths, [140, 33, 150, 130, 300, 1], 3520)
    shared_list(torch, iq, rng, 6, 16, 4, [7000, 60, 5000, 300, 2000, 3500], [5, 1, 8, 8, 3, 2], 7040)


def test_offsets_beyond_32_bits_against_the_formula(env):
    """Nine sequences of a million tokens on eight heads: the last head of the last sequence against attention in 64 bits over its packed rows."""
    torch, iq = env
    n, B, H, rows = (1 << 20) - 40, 9, 8, (1 << 20) + 64
    cfg = iq.make_config(B, 2 * H, H, 128, 4, 32, 4, 128, SYM, SYM, capacity_tokens=rows)
    cache = iq.allocate_cache(cfg)
    gen = torch.Generator(device="cuda").manual_seed(1)
    for name in ("k_codes", "v_codes"):
        for part in cache.buffers[name].view(B, -1):
            part.random_(0, 256, generator=gen)
    for name in ("k_scales", "v_scales"):
        for part in cache.buffers[name].view(torch.float16).view(B, -1):
            part.uniform_(0.1, 0.3, generator=gen)
    for name in ("k_recent", "v_recent", "k_sink", "v_sink"):
        cache.buffers[name].view(torch.float16).normal_(generator=gen)
    cache.c.n_tokens = cache.c.store_ahead_tokens = n

    def held(which):
        """fp16 values [n, 128] of the last head of the last sequence."""
        slots = 128 + (1 if which == "k" else 32)
        nq = n - 132 if which == "k" else (n - 132) // 32 * 32
        last = lambda name: cache.buffers[f"{which}_{name}"].view(B * H, -1)[-1]          # noqa: E731
        field = torch.stack([last("codes") & 15, last("codes") >> 4], -1).flatten().float() - 8.0
        scale = last("scales").view(torch.float16).float()
        if which == "k":
            x = (field.view(rows, 4, 32) * scale.view(rows, 4, 1)).view(rows, 128)
        else:
            x = (field.view(rows // 32, 128, 32) * scale.view(rows // 32, 128, 1)).transpose(1, 2).reshape(rows, 128)
        ring = last("recent").view(torch.float16).view(slots, 128)
        at = torch.arange(4 + nq, n, device="cuda") % slots
        return torch.cat([last("sink").view(torch.float16).view(4, 128), x[:nq].half(), ring[at]])

    K, V = held("k"), held("v")
    rng = np.random.default_rng(3)
    for t in (3, 20, 80):
        _, q, k, v = projection(torch, rng, B, t, 2 * H, H)
        for i in range(t):                                  # (rows along keys all over the sequence)
            for g in (0, 1):
                j = [n - 1, 5, 4, 1 << 19, n - 200, n - 133, int(rng.integers(n))][(2 * i + g) % 7]
                x = K[j].float()
                q[B - 1, 2 * H - 2 + g, i] = (x * (14.0 * 128 ** 0.5 / (x * x).sum())).half()
        out = iq.innerq_chunk_attention(cache, k, v, q, iq.allocate_chunk_workspace(cfg, t))
        Kt, Vt = (torch.cat([y, z[B - 1, H - 1]]).double() for y, z in ((K, k), (V, v)))
        for g in (0, 1):
            s = q[B - 1, 2 * H - 2 + g].double() @ Kt.T / 128 ** 0.5
            s[torch.arange(n + t, device="cuda") > n + torch.arange(t, device="cuda")[:, None]] = -float("inf")
            p = torch.softmax(s, -1)
            want = p @ Vt
            # a rounded weight moves the output by p 2^-11 |v - out|; scores of at most a few dozen in fp32, 128 additions of 2^-24 of at most 150;
            # fp32 sums over a range of the tokens (seven or more of them): 2^-24 for each addition, and for those of the joins
            bound = 1.01 * (2.0 ** -11 + 2.0 ** -24 * 128 * 150) * (p @ Vt.abs() + want.abs()) + (n / 7 + 512) * 2.0 ** -24 * (p @ Vt.abs())
            got = out[B - 1, 2 * H - 2 + g].double()
            assert ((got - want).abs() <= bound).all(), (t, g, ((got - want).abs() / bound).max().item())
