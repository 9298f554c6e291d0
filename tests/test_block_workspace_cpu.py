"""A workspace of the 8-bit cache's attention for so many rows of a sequence also serves every call of fewer: a program makes one for its longest chunk."""
import pytest

from paper_2602_23200_amd import binding as iq


@pytest.mark.parametrize("batch", [1, 3, 8, 48, 49, 64, 96, 97, 256, 257, 1000])
@pytest.mark.parametrize("kv_heads,r", [(1, 1), (8, 4), (8, 5), (32, 1), (2, 71), (4, 17)])
def test_never_more_for_fewer_rows(batch, kv_heads, r):
    cfg = iq.make_block_config(batch, kv_heads * r, kv_heads, capacity_tokens=1 << 15)
    rows = sorted({t + e for t in (2 ** i for i in range(15)) for e in (-1, 0, 1) if t + e > 0} | {16 * i // r for i in range(1, 40)} - {0})
    rows = [t for t in rows if t * r * kv_heads * batch < 1 << 31]                           # (more are refused)
    sizes = [iq.innerq_block_workspace_bytes(cfg, t) for t in rows]
    assert sizes[0] > 0 and sizes == sorted(sizes), [(t, a, b) for t, a, b in zip(rows[1:], sizes, sizes[1:]) if b < a]
    assert sizes[-1] <= 80 << 20
