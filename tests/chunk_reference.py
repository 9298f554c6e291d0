"""Attention of several new tokens in 64 bits over the fp16 operands that the library multiplies, and how far a result may be from it
(shared by the tests of that call).

The operands are the definition's: queries and new rows fp16 as given, cached windows fp16, stored values rounded once to fp16.  What is
left between a right result and this reference, with p the softmax weights, u = 2^-11 and everything to first order (second orders are
below 2^-10 of it, in the factor 1.01):
* a weight is rounded to fp16, by u of itself, and its score is a sum of 128 exact products in fp32, each addition off by 2^-24 of at most
  a = sum |q_c k_c| / sqrt(d); scaling, the level's subtraction (magnitudes up to the largest |score|) and the exponential add a few steps of
  2^-24.  A weight moved by a share e moves the output by p e (v - out), because the normaliser is the sum of the same weights;
* a weight below fp16's normal range is off by half its smallest step, 2^-25, at a level that is 2^9 or more below the largest weight:
  2^-34 of the largest weight;
* sums over tokens in fp32: an addition each for the wavefronts and ranges that a row is spread over and for its tokens, 2^-24 of
  sum p |v| each;
* an fp16 output is rounded by u of itself (2^-25 where it is a denormal)."""
import numpy as np

from oracle import innerq_oracle as orc


def operands(o1, ref, which, fresh):
    """fp16 values, as 64-bit ones, of all tokens of one sequence: [Hk, n + t, d].  ref: the oracle's cache of it; fresh [Hk, t, d]."""
    n = ref.n_tokens
    held = [orc.effective_tensor(o1, ref, which, 0, h) if n else np.zeros((0, 128)) for h in range(o1.n_kv_heads)]
    return np.concatenate([np.stack(held).astype(np.float16), fresh], axis=1).astype(np.float64)


def attend(q, K, V, half, hidden=None):
    """q [Hq, t, d], K, V [Hk, n + t, d] -> outputs [Hq, t, d] and the bound of every element.  hidden (t, n + t): instead of the causal mask."""
    Hq, t, d = q.shape
    Hk, N, _ = K.shape
    r = Hq // Hk
    n = N - t
    if hidden is None:
        hidden = np.arange(N)[None] > n + np.arange(t)[:, None]
    out, bound = np.empty((Hq, t, d)), np.empty((Hq, t, d))
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
        share = p * (u + e * (128 * a + 8 * most + 8)) + 2.0 ** -34 * p.max(-1, keepdims=True) * ~hidden
        for i in range(t):                                  # (differences to the output: a row at a time)
            bound[g, i] = 1.01 * share[i] @ np.abs(v - out[g, i])
        bound[g] += (N + 128) * e * (p @ np.abs(v))
    if half:
        bound += u * np.abs(out) + 2.0 ** -25
    return out, bound


def aimed(rng, K, n, t, r, borders):
    """Queries [Hk r, t, d] fp16, most of them along the key of one token, which then has nearly all of the weight: the row's own token, the first
    one that is hidden from it, a border of the cache, or any token; the rest are random."""
    Hk, N, d = K.shape
    q = rng.standard_normal((Hk * r, t, d))
    for g in range(Hk * r):
        for i in range(t):
            kind = rng.random()
            if kind < 0.2:
                continue
            if kind < 0.4:
                j = n + i
            elif kind < 0.6:
                j = n + i + 1
            elif kind < 0.8 and borders:
                j = borders[int(rng.integers(len(borders)))]
            else:
                j = int(rng.integers(n + i + 1))
            if not 0 <= j < N:
                continue
            k = K[g // r, j]
            q[g, i] = k * (12.0 * np.sqrt(d) / max((k ** 2).sum(), 1e-6))
    return np.clip(q, -60000.0, 60000.0).astype(np.float16)


def borders_of(o1, n, t):
    """Tokens on either side of where a cache of n tokens and t new ones change from one kind to the next, and ends of tiles of either kind."""
    at = {0, n, n + t}
    for which in "kv":
        n_s, n_q, _ = orc.partition(o1, which, n)
        at |= {n_s, n_s + n_q}
        at |= {n_s + x for x in (32, 64, n_q - 32, n_q - 64) if 0 < x < n_q}
    at |= {n + x for x in (32, 64, 128) if x < t}
    return sorted({j for x in at for j in (x - 1, x) if 0 <= j < n + t})


def check(got, want, bound, what=""):
    got = np.asarray(got, dtype=np.float64)
    assert np.isfinite(got).all(), what
    over = np.abs(got - want) / np.maximum(bound, 1e-300)
    assert over.max(initial=0.0) <= 1.0, (what, float(over.max()), np.unravel_index(over.argmax(), over.shape))
    return float(over.max(initial=0.0))
