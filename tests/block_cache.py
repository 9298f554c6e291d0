"""Caches in 8 bits on the device with what they hold known on the host (shared by the tests of those calls)."""
import numpy as np

from tests import block_reference as ref

D = 128


def keys_and_values(rng, lengths, H, heavy=True):
    """fp16 [B, H, max length, D] of either tensor; some channels of the keys far larger than others."""
    T = max(max(lengths), 1)
    spread = 1.0 + np.abs(rng.standard_t(3, (1, H, 1, D))) * heavy
    k = np.clip(rng.standard_normal((len(lengths), H, T, D)) * spread, -60000, 60000).astype(np.float16)
    v = rng.standard_normal((len(lengths), H, T, D)).astype(np.float16)
    return k, v


def page_table(rng, lengths, capacity, spare=3):
    """A random injection of the pages that the sequences need into a pool; entries nobody may follow lie outside of it."""
    need = [-(-n // 64) for n in lengths]
    pool = sum(need) + spare
    ids = rng.permutation(pool).astype(np.int32)
    table = np.full((len(lengths), capacity // 64), 0x7ffffff0, dtype=np.int32)
    table[:, 1::2] = -5
    at = 0
    for b, m in enumerate(need):
        table[b, :m] = ids[at:at + m]
        at += m
    return table, pool


def empty(torch, iq, B, Hq, Hk, capacity, e4, block, lengths=None, rng=None, dirt=0):
    """A cache; lengths (with rng): paged, with pages for that many tokens.  dirt: the byte that its buffers hold."""
    table, pool = (None, 0) if lengths is None else page_table(rng, lengths, capacity)
    cfg = iq.make_block_config(B, Hq, Hk, type=iq.E4M3 if e4 else iq.INT8, block=block, capacity_tokens=capacity, page_pool_pages=pool)
    cache = iq.allocate_block_cache(cfg, page_table=None if table is None else torch.from_numpy(table).cuda())
    for name in iq.BLOCK_BUFFER_NAMES:
        cache.buffers[name].fill_(dirt)
    return cache, table


def contents(iq, cache, table, b):
    """Tiles [Hk, tiles, 4096] of codes, scales [Hk, blocks] and open rows [Hk, block, D] of sequence b, of keys and values."""
    cfg = cache.cfg
    H, G, out = cfg.n_kv_heads, cfg.block, {}
    for w in "kv":
        codes, scales, rows = (cache.buffers[w + x].cpu().numpy() for x in ("_codes", "_scales", "_open"))
        scales = scales.view(np.float32)
        if table is None:
            codes = codes.reshape(cfg.batch, H, -1, 4096)[b]
            scales = scales.reshape(cfg.batch, H, -1)[b]
        else:
            pages = np.clip(table[b], 0, cfg.page_pool_pages - 1)
            codes = codes.reshape(-1, H, 2, 4096)[pages].transpose(1, 0, 2, 3).reshape(H, -1, 4096)
            scales = scales.reshape(-1, H, 64 // G)[pages].transpose(1, 0, 2).reshape(H, -1)
        out[w] = codes, scales, rows.view(np.float16).reshape(cfg.batch, H, G, D)[b]
    return out


def check_contents(iq, cache, table, b, k, v, e4, what=""):
    """The cache holds tokens k, v fp16 [Hk, n, D] of sequence b, to the bit."""
    G, n = cache.cfg.block, k.shape[1]
    m = n // G * G
    for w, x, tiles in (("k", k, ref.key_tiles), ("v", v, ref.value_tiles)):
        codes, scales, rows = contents(iq, cache, table, b)[w]
        want, scale = ref.pack(x[:, :m], G, e4)
        assert np.array_equal(scales[:, :m // G], scale), (what, b, w, "scales")
        assert np.array_equal(codes[:, :m // 32], tiles(ref.code_bytes(want, e4))), (what, b, w, "codes")
        assert np.array_equal(rows[:, :n - m].view(np.uint16), x[:, m:].view(np.uint16)), (what, b, w, "open rows")


def rows(torch, x, how, rng):
    """fp16 [B, H, T, D] on the device: "plain", "projection" (between the rows of other heads, tokens outermost) or "broadcast" over the batch."""
    x = torch.from_numpy(x)
    if how == "plain":
        return x.cuda()
    if how == "broadcast":
        return x[:1].cuda().expand(x.shape)
    B, H, T, d = x.shape
    wide = torch.from_numpy(rng.standard_normal((B, T, H + 3, d)).astype(np.float16)).cuda()
    wide[:, :, 2:2 + H] = x.transpose(1, 2).cuda()
    return wide[:, :, 2:2 + H].transpose(1, 2)


def filled(torch, iq, rng, lengths, Hq, Hk, e4, block, capacity=None, paged=False, heavy=True):
    """A cache whose sequence b holds lengths[b] tokens, its counts on the device, and those tokens [B, Hk, n, D]."""
    capacity = capacity or -(-(max(lengths) + 300) // 64) * 64
    cache, table = empty(torch, iq, len(lengths), Hq, Hk, capacity, e4, block, lengths if paged else None, rng)
    k, v = keys_and_values(rng, lengths, Hk, heavy)
    counts = torch.zeros(len(lengths), dtype=torch.int32, device="cuda")
    iq.innerq_block_append_ragged(cache, counts, torch.tensor(lengths, dtype=torch.int32, device="cuda"), torch.from_numpy(k).cuda(),
                                  torch.from_numpy(v).cuda())
    cache.c.n_tokens = lengths[0]                          # (for the calls with one count for all)
    return cache, table, counts, k, v
