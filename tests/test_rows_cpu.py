"""What the calls over several new tokens refuse, on the host and before any launch (no GPU here; pointers are made up)."""
import ctypes as C

import pytest

from paper_2602_23200_amd import binding as iq

P = 4096                                                  # an aligned address nobody follows
L = iq.lib()


def config(**over):
    c = iq.make_config(2, 8, 2, 128, 4, 32, 4, 64, capacity_tokens=1024)
    for k, v in over.items():
        setattr(c, k, v)
    return c


def cache_of(n=100, **over):
    cache = iq.innerq_cache_t()
    for name in iq.BUFFER_NAMES:
        setattr(cache, name, P)
    cache.n_tokens = n
    for k, v in over.items():
        setattr(cache, k, v)
    return cache


def rotation(**over):
    r = iq.innerq_rotation_t(P, P, 100, 128, 0, 1)
    for k, v in over.items():
        setattr(r, k, v)
    return r


def strides(batch=16384, head=128, token=1280):
    return iq.innerq_strides_t(batch, head, token)


def ref(x):
    return None if x is None else C.byref(x)


def call_rotate(cfg=None, rot=None, positions=P, n=0, n_dev=None, t_dev=None, x=P, xs=None, y=P, ys=None, heads=4, t=3, **null):
    return L.innerq_rotate(ref(cfg or config()), None if "rot" in null.get("none", ()) else ref(rot or rotation()), positions, n, n_dev, t_dev,
                           x, None if "xs" in null.get("none", ()) else ref(xs or strides()), y,
                           None if "ys" in null.get("none", ()) else ref(ys or strides()), heads, t, None)


ROTATIONS = [
    (dict(cos_table=None), iq.E_NULL), (dict(sin_table=None), iq.E_NULL), (dict(cos_table=P + 4), iq.E_ALIGN), (dict(sin_table=P + 8), iq.E_ALIGN),
    (dict(table_positions=0), iq.E_ARG), (dict(table_positions=1 << 31), iq.E_ARG), (dict(rot_dim=0), iq.E_ARG), (dict(rot_dim=130), iq.E_ARG),
    (dict(rot_dim=63), iq.E_ARG), (dict(rot_dim=24), iq.E_UNSUPPORTED), (dict(rot_dim=2), iq.E_UNSUPPORTED), (dict(interleaved=2), iq.E_ARG),
    (dict(n_axes=0), iq.E_ARG), (dict(n_axes=4), iq.E_ARG), (dict(pair_axis=(C.c_uint8 * 64)(*[0] * 63, 1)), iq.E_ARG)]


@pytest.mark.parametrize("over,want", ROTATIONS)
def test_rotations(over, want):
    assert call_rotate(rot=rotation(**over)) == want
    s, c = strides(), config()
    assert L.innerq_append_rotated(ref(c), ref(cache_of()), ref(rotation(**over)), P, P, ref(s), P, ref(s), 3, None, None) == want


def test_axes_of_pairs_that_are_not_turned_are_ignored():
    r = rotation(rot_dim=64, pair_axis=(C.c_uint8 * 64)(*[0] * 32, *[9] * 32))
    assert call_rotate(rot=r, t=0) == iq.OK


@pytest.mark.parametrize("over,want", [
    (dict(none=("rot",)), iq.E_NULL), (dict(none=("xs",)), iq.E_NULL), (dict(none=("ys",)), iq.E_NULL), (dict(x=None), iq.E_NULL), (dict(y=None), iq.E_NULL),
    (dict(x=P + 8), iq.E_ALIGN), (dict(y=P + 2), iq.E_ALIGN), (dict(positions=P + 2), iq.E_ALIGN), (dict(n_dev=P + 1), iq.E_ALIGN), (dict(t_dev=P + 2), iq.E_ALIGN),
    (dict(xs=strides(token=644)), iq.E_ALIGN), (dict(xs=strides(head=-128)), iq.E_ARG), (dict(ys=strides(token=0)), iq.E_ARG), (dict(ys=strides(head=64)), iq.E_ARG),
    (dict(heads=0), iq.E_ARG), (dict(heads=65536), iq.E_ARG), (dict(t=-1), iq.E_ARG), (dict(t=1 << 31), iq.E_ARG), (dict(t=1 << 30), iq.E_ARG), (dict(n=-1), iq.E_ARG),
    (dict(n=(1 << 31) - 2), iq.E_ARG), (dict(t=0), iq.OK), (dict(cfg=config(bits=5)), iq.E_UNSUPPORTED)])
def test_rotate(over, want):
    assert call_rotate(**over) == want


@pytest.mark.parametrize("s", [strides(head=128, token=128), strides(token=384), strides(head=384, token=128, batch=384), strides(batch=2560), strides(batch=2944, head=256)])
def test_rows_that_are_written_do_not_overlap(s):
    # two sequences, three tokens, four (rotation) or eight (attention) heads
    assert call_rotate(ys=s) == iq.E_ARG
    assert attentions(outs=strides(s.batch, s.head, s.token)) == (iq.E_ARG, iq.E_ARG)


def test_rows_next_to_each_other_in_any_order_are_written():
    for order in ((0, 1, 2), (0, 2, 1), (1, 0, 2), (2, 1, 0)):
        n, at, s = (2, 4, 3), 128, [0, 0, 0]
        for d in reversed(order):
            s[d] = at
            at *= n[d]
        assert call_rotate(ys=strides(*s), n_dev=P + 1) == iq.E_ALIGN      # (what is looked at next: the rows are accepted, nothing is launched)


def appends(cfg, cache, k=P, ks=None, v=P, vs=None, t=3, inv=None, n_dev=P, t_dev=P, rot=None, positions=None):
    ks, vs = ks or strides(), vs or strides()
    before = cache.n_tokens if cache else None
    a = L.innerq_append_rotated(ref(cfg), ref(cache), ref(rot), positions, k, ref(ks), v, ref(vs), t, inv, None)
    b = L.innerq_append_rotated_ragged(ref(cfg), ref(cache), ref(rot), positions, n_dev, t_dev, k, ref(ks), v, ref(vs), t, inv, None)
    assert cache is None or cache.n_tokens == before
    return a, b


@pytest.mark.parametrize("over,want", [
    (dict(k=None), iq.E_NULL), (dict(v=None), iq.E_NULL), (dict(k=P + 8), iq.E_ALIGN), (dict(v=P + 4), iq.E_ALIGN), (dict(ks=strides(batch=4)), iq.E_ALIGN),
    (dict(vs=strides(token=-8)), iq.E_ARG), (dict(inv=P + 4), iq.E_ALIGN), (dict(t=-1), iq.E_ARG), (dict(t=0), iq.OK), (dict(t=1025), iq.E_CAPACITY),
    (dict(rot=rotation(), positions=P + 1), iq.E_ALIGN)])
def test_append(over, want):
    assert appends(config(), cache_of(), **over) == (want, want)


def test_append_states():
    assert appends(config(), None) == (iq.E_NULL, iq.E_NULL)
    assert appends(config(), cache_of(k_codes=None)) == (iq.E_NULL, iq.E_NULL)
    for kind in (iq.KIND_OUTER, iq.KIND_FP16):
        assert appends(config(kind=kind), cache_of()) == (iq.E_UNSUPPORTED, iq.E_UNSUPPORTED)
    assert appends(config(capacity_tokens=(1 << 24) + 32), cache_of()) == (iq.E_UNSUPPORTED, iq.E_UNSUPPORTED)
    s, c, cache = strides(), config(), cache_of(1022)
    assert L.innerq_append_rotated(ref(c), ref(cache), None, None, P, ref(s), P, ref(s), 3, None, None) == iq.E_CAPACITY
    assert cache.n_tokens == 1022
    for n_dev, t_dev, want in ((None, P, iq.E_NULL), (P, None, iq.E_NULL), (P + 2, P, iq.E_ALIGN), (P, P + 1, iq.E_ALIGN)):
        assert appends(config(), cache_of(), n_dev=n_dev, t_dev=t_dev, t=0)[1] == want


def test_struct_layout_matches_the_header():
    assert C.sizeof(iq.innerq_strides_t) == 24 and iq.innerq_strides_t.token.offset == 16
    assert C.sizeof(iq.innerq_rotation_t) == 3 * 8 + 3 * 4 + 64 + 4 and iq.innerq_rotation_t.pair_axis.offset == 36


def attentions(cfg=None, cache=None, k=P, ks=None, v=P, vs=None, q=P, qs=None, t=3, scale=None, out=P, outs=None, fp32=0, ws=P, ws_bytes=1 << 40,
               n_dev=P, t_dev=P, most=500):
    cfg, cache = cfg or config(), cache or cache_of()
    s = [x or strides() for x in (ks, vs, qs, outs)]
    rows = [k, ref(s[0]), v, ref(s[1]), q, ref(s[2]), t, scale, out, ref(s[3]), fp32, ws, ws_bytes, None]
    return (L.innerq_chunk_attention(ref(cfg), ref(cache), *rows), L.innerq_chunk_attention_ragged(ref(cfg), ref(cache), n_dev, t_dev, most, *rows))


@pytest.mark.parametrize("over,want", [
    (dict(k=None), iq.E_NULL), (dict(v=None), iq.E_NULL), (dict(q=None), iq.E_NULL), (dict(out=None), iq.E_NULL), (dict(ws=None), iq.E_NULL),
    (dict(k=P + 8), iq.E_ALIGN), (dict(v=P + 2), iq.E_ALIGN), (dict(q=P + 4), iq.E_ALIGN), (dict(out=P + 8), iq.E_ALIGN), (dict(ws=P + 8), iq.E_ALIGN),
    (dict(scale=P + 4), iq.E_ALIGN), (dict(qs=strides(head=132)), iq.E_ALIGN), (dict(ks=strides(token=-8)), iq.E_ARG), (dict(outs=strides(token=0)), iq.E_ARG),
    (dict(outs=strides(head=132), fp32=0), iq.E_ALIGN), (dict(t=-1), iq.E_ARG), (dict(t=0), iq.OK), (dict(t=1025), iq.E_CAPACITY), (dict(ws_bytes=63), iq.E_WORKSPACE),
    (dict(cfg=config(kind=iq.KIND_OUTER)), iq.E_UNSUPPORTED), (dict(cfg=config(kind=iq.KIND_FP16)), iq.E_UNSUPPORTED),
    (dict(cfg=config(capacity_tokens=(1 << 24) + 32)), iq.E_UNSUPPORTED), (dict(cfg=config(n_q_heads=1 << 24, capacity_tokens=1 << 20), t=1 << 10), iq.E_UNSUPPORTED)])
def test_chunk_attention(over, want):
    assert attentions(**over) == (want, want)


def test_chunk_attention_states():
    assert L.innerq_chunk_attention(ref(config()), None, *([P, None] * 3), 3, None, P, None, 0, P, 1 << 40, None) == iq.E_NULL
    assert attentions(cache=cache_of(1022))[0] == iq.E_CAPACITY
    for over, want in ((dict(n_dev=None), iq.E_NULL), (dict(t_dev=None), iq.E_NULL), (dict(n_dev=P + 2), iq.E_ALIGN), (dict(most=0), iq.E_ARG), (dict(most=1025), iq.E_CAPACITY)):
        assert attentions(**over)[1] == want
    # too little workspace, by a byte, where the keys may be split
    need = iq.innerq_chunk_workspace_bytes(config(), 3)
    assert need > 64 and attentions(ws_bytes=need - 1) == (iq.E_WORKSPACE, iq.E_WORKSPACE)


def test_chunk_workspace():
    for bad in (config(bits=5), config(kind=iq.KIND_FP16)):
        assert iq.innerq_chunk_workspace_bytes(bad, 4) == 0
    assert iq.innerq_chunk_workspace_bytes(config(), 0) == 0 and iq.innerq_chunk_workspace_bytes(config(), -1) == 0
    assert iq.innerq_chunk_workspace_bytes(config(), 1 << 25) == 0
    # never more than two rounds of work-groups, whatever the sizes: 1024 of 128 rows or 512 of 256 (a list: 512 of 32 and of 128)
    for batch, hk, r, cap, t in ((1, 1, 1, 1 << 20, 1), (1, 8, 4, 1 << 17, 2048), (64, 8, 8, 32768, 5), (4, 32, 1, 65536, 33)):
        c = iq.make_config(batch, hk * r, hk, 128, 2, 32, 4, 128, capacity_tokens=cap)
        assert 64 <= iq.innerq_chunk_workspace_bytes(c, t) <= 1024 * 128 * 130 * 4 + 4096
