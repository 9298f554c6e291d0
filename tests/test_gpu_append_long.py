"""innerq_append_rotated beyond 2 M key groups, where its launch decides between the variants of a hybrid group on a shorter error sum: byte for
byte the cache of the same tokens in parts below that line, and of innerq_quantize_append of keys rotated beforehand."""
import pytest

from oracle import innerq_oracle as orc
from tests.rows import rotation_tables
from tests.test_gpu_bulk_append import device_values

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def env():
    import torch
    from paper_2602_23200_amd import binding as iq
    assert torch.cuda.is_available(), "these tests need the MI355X"
    iq.lib()
    return torch, iq


@pytest.mark.parametrize("dist", ["normal", "ties", "denormal", "wide", "offset"])
@pytest.mark.parametrize("bits,group,modes", [(2, 32, (orc.HYBRID, orc.HYBRID)), (2, 64, (orc.HYBRID, orc.HYBRID)), (4, 64, (orc.HYBRID, orc.HYBRID)),
                                              (4, 32, (orc.HYBRID, orc.ASYM)), (3, 64, (orc.HYBRID, orc.HYBRID)), (2, 32, (orc.ASYM, orc.SYM))])
def test_shorter_error_sum(env, bits, group, modes, dist):
    torch, iq = env
    H, n = 8, (1 << 21) // 8 * group // 128 + 200
    assert H * (n - 132) * (128 // group) >= 1 << 21
    cfg = iq.make_config(1, H, H, 128, bits, group, 4, 128, modes[0], modes[1], capacity_tokens=-(-n // 64) * 64)
    gen = torch.Generator(device="cuda").manual_seed(bits * group)
    x = torch.empty(1, n, 2 * H, 128, dtype=torch.float16, device="cuda").transpose(1, 2)       # (a projection's output)
    for part in x.split(H, dim=1):
        part.copy_(device_values(torch, gen, (1, H, n, 128), dist))
    k, v = x[:, :H], x[:, H:]
    inv = torch.rand(H, 128, device="cuda", generator=gen) + 0.5 if group == 64 else None
    cos, sin = (torch.from_numpy(t).cuda() for t in rotation_tables(n, 64))
    rot = iq.make_rotation(cos, sin)                        # (half of the channels: the others keep their ties and denormals)
    whole, parts, plain = (iq.allocate_cache(cfg) for _ in range(3))
    iq.innerq_append_rotated(whole, k, v, rot, k_inv_norm=inv)
    for a, b in ((0, n // 3), (n // 3, n // 3 * 2 - 5), (n // 3 * 2 - 5, n)):
        iq.innerq_append_rotated(parts, k[:, :, a:b], v[:, :, a:b], rot, k_inv_norm=inv)
    iq.innerq_quantize_append(plain, iq.innerq_rotate(cfg, rot, k).contiguous(), v.contiguous(), inv)
    for name, buf in whole.buffers.items():
        if buf is not None:
            assert torch.equal(buf, plain.buffers[name]), name
            assert name.endswith("recent") or torch.equal(buf, parts.buffers[name]), name       # (a ring's spare slots hold older tokens)
