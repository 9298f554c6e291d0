"""The cache in 8 bits with block scales from its definition (include/innerq.h), and attention over it in 64 bits with how far a result may
be from it (shared by the tests of those calls).

What is left between a right result and attention in 64 bits over the values that the cache stands for, with p the softmax weights, e =
2^-24, u = 2^-11, everything to first order (second orders are below 2^-10 of it, in the factor 1.01):
* a score is a sum of 128 products, exact in fp32 (11 bits of a query, 8 of a code; new and open rows 11), each of whose additions is off by 2 e (a matrix
  core may cut instead of rounding) of at most a = sum |q_c k_c| / sqrt(d); its factor, the sum with the logarithm of the values' scale (below 40) and the
  level's subtraction round magnitudes up to the largest |score| and that logarithm a few times, the exponential, the logarithm and the scale's reciprocal
  add 2 e each.  A weight moved by a share s moves the output by p s (v - out);
* a weight enters the second product as two fp16 pieces, the second one rounded by u of what the first one left, which is u of the weight: u^2.  Below
  fp16's normal range the pieces' smallest step counts, 2^-25 at a level 2^9 below the largest weight: 2^-34 of that one;
* many rows: one piece, u of the weight (the normaliser sums the same rounded weights);
* the codes of a block of values whose scale is below 1/16 of the largest enter times 2^-k, multiples of 2^-24: exact down to 2^-28 of that scale, below it off
  by 2^-25 at a scale of at most 1/8 of the largest, which is 2^-35 of the largest value;
* sums over tokens in fp32: 2 e of sum p |v| for every token and for every wavefront and range that a row is spread over;
* an fp16 output is rounded by u of itself (2^-25 where it is a denormal)."""
import numpy as np


def e4m3(y):
    """Nearest numbers of four exponent and three mantissa bits (bias 7, half to even), as floats."""
    y = np.asarray(y, dtype=np.float64)
    e = np.maximum(np.floor(np.log2(np.maximum(np.abs(y), 1e-30))), -6)
    return np.rint(y / 2.0 ** (e - 3)) * 2.0 ** (e - 3)


def e4m3_bytes(values):
    """Their bytes."""
    values = np.asarray(values, dtype=np.float64)
    size = np.abs(values)
    e = np.maximum(np.floor(np.log2(np.maximum(size, 1e-30))), -6)
    mantissa = np.rint(size / 2.0 ** (e - 3)).astype(np.int64)             # 8 .. 15, below 8: subnormal
    byte = np.where(mantissa >= 8, ((e.astype(np.int64) + 7) << 3) + (mantissa - 8), mantissa)
    return (byte + np.where(np.signbit(values), 128, 0)).astype(np.uint8)


def pack(x, block, e4):
    """fp16 [H, m * block, d] -> codes (numbers) [H, m * block, d], scales fp32 [H, m]: every fp32 operation rounded."""
    H, n, d = x.shape
    g = x.astype(np.float32).reshape(H, n // block, block * d)
    scale = np.abs(g).max(-1) / np.float32(448.0 if e4 else 127.0)
    q = g / np.where(scale == 0, np.float32(1), scale)[..., None]
    assert q.dtype == np.float32
    return (e4m3(q) if e4 else np.rint(q).astype(np.float64) + 0.0).reshape(H, n, d), scale      # (an integer's zero has no sign)


def code_bytes(codes, e4):
    return e4m3_bytes(codes) if e4 else codes.astype(np.int8).view(np.uint8)


def key_tiles(b):
    """Bytes [..., 32 m, 128] of keys in the store's order: [..., m, 4096]."""
    b = b.reshape(*b.shape[:-2], -1, 2, 16, 4, 2, 16)                       # a c g h e
    return np.moveaxis(b, (-5, -4, -3, -2), (-5, -2, -3, -4)).reshape(*b.shape[:-5], 4096)


def value_tiles(b):
    b = b.reshape(*b.shape[:-2], -1, 2, 4, 4, 4, 16, 2)                     # i g j q c m
    return np.moveaxis(b, (-6, -5, -4, -3, -2, -1), (-2, -5, -1, -6, -4, -3)).reshape(*b.shape[:-6], 4096)


def held(x, block, e4):
    """What the cache holds of tokens x fp16 [H, n, d], in token order: 64-bit values."""
    n = x.shape[1] // block * block
    codes, scale = pack(x[:, :n], block, e4)
    out = x.astype(np.float64)
    out[:, :n] = codes * scale.astype(np.float64).repeat(block, 1)[..., None]
    return out


def attend(q, K, V, half, many=False, hidden=None):
    """q [Hq, t, d], K, V [Hk, N, d] in 64 bits; hidden [t, N].  -> outputs [Hq, t, d] and the bound of every element."""
    Hq, t, d = q.shape
    Hk, N, _ = K.shape
    r = Hq // Hk
    out, bound = np.zeros((Hq, t, d)), np.zeros((Hq, t, d))
    if N == 0:
        return out, bound
    hidden = np.zeros((t, N), dtype=bool) if hidden is None else hidden
    u, e = 2.0 ** -11, 2.0 ** -24
    for g in range(Hq):
        k, v, x = K[g // r], V[g // r], q[g].astype(np.float64)
        s = x @ k.T / np.sqrt(d)
        a = np.abs(x) @ np.abs(k).T / np.sqrt(d)
        s[hidden] = -np.inf
        most = np.where(hidden, 0.0, np.abs(s)).max(-1, keepdims=True)
        p = np.exp(s - s.max(-1, keepdims=True))
        p /= p.sum(-1, keepdims=True)
        out[g] = p @ v
        share = p * ((u if many else u * u) + e * (256 * a + 8 * most + 50)) + 2.0 ** -34 * p.max(-1, keepdims=True) * ~hidden
        for i in range(t):                                  # (differences to the output: a row at a time)
            bound[g, i] = 1.01 * share[i] @ np.abs(v - out[g, i])
        bound[g] += 2 * (N + 600) * e * (p @ np.abs(v)) + 2.0 ** -35 * np.abs(v).max()
    if half:
        bound += u * np.abs(out) + 2.0 ** -25
    return out, bound


def causal(n, t):
    return np.arange(n + t)[None] > n + np.arange(t)[:, None]
