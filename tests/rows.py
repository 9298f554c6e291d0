"""Plain forms of the calls over several new tokens, and rows laid out as a projection leaves them (shared by their tests)."""
import numpy as np


def rotation_tables(positions, rot_dim, base=10000.0):
    """fp32 cosines and sines [positions, rot_dim / 2], angles in 64 bits."""
    turn = base ** (-np.arange(0, rot_dim, 2, dtype=np.float64) / rot_dim)
    angle = np.arange(positions, dtype=np.float64)[:, None] * turn
    return np.cos(angle).astype(np.float32), np.sin(angle).astype(np.float32)


def rotate(x, cos, sin, positions, rot_dim, interleaved=False, axes=None, dtype=np.float32):
    """x fp16 [B, H, T, d]; positions [axes, B, T].  dtype float32: every operation rounded (the definition, to the bit);
    float64: the formula."""
    P = rot_dim // 2
    axes = np.zeros(P, dtype=np.int64) if axes is None else np.asarray(axes)
    place = np.clip(positions, 0, cos.shape[0] - 1)[axes]                  # [P, B, T]
    pair = np.arange(P)[:, None, None]
    c = np.moveaxis(cos[place, pair], 0, -1)[:, None].astype(dtype)        # [B, 1, T, P]
    s = np.moveaxis(sin[place, pair], 0, -1)[:, None].astype(dtype)
    first, second = (slice(0, rot_dim, 2), slice(1, rot_dim, 2)) if interleaved else (slice(0, P), slice(P, rot_dim))
    a, b = x[..., first].astype(dtype), x[..., second].astype(dtype)
    y = x.astype(dtype) if dtype == np.float64 else x.copy()
    y[..., first] = (a * c - b * s).astype(y.dtype)
    y[..., second] = (b * c + a * s).astype(y.dtype)
    return y


def projection(torch, rng, B, T, Hq, Hk, d=128, spare=1):
    """A projection's output [B, T, Hq + 2 Hk + spare, d] on the device and its parts q, k, v as [B, H, T, d] views."""
    x = torch.from_numpy(rng.standard_normal((B, T, Hq + 2 * Hk + spare, d)).astype(np.float16)).cuda()
    p = x.transpose(1, 2)
    return x, p[:, :Hq], p[:, Hq:Hq + Hk], p[:, Hq + Hk:Hq + 2 * Hk]
