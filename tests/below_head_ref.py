"""64-bit references of the operators below the vocabulary head, in numpy."""
import numpy as np

U = np.uint64
LOW = U(0xFFFFFFFF)


def philox(counter, seed):
    """Words [n, 4] (uint32) of Philox4x32-10 for the 64-bit counters, upper words zero."""
    with np.errstate(over="ignore"):
        ctr = np.asarray(counter, dtype=U)
    x = [ctr & LOW, ctr >> U(32), np.zeros_like(ctr), np.zeros_like(ctr)]
    return _rounds(x, seed & 0xFFFFFFFF, seed >> 32)


def _rounds(x, k0, k1):
    for _ in range(10):
        a, b = x[0] * U(0xD2511F53), x[2] * U(0xCD9E8D57)
        x = [(b >> U(32)) ^ x[1] ^ U(k0), b & LOW, (a >> U(32)) ^ x[3] ^ U(k1), a & LOW]
        k0, k1 = (k0 + 0x9E3779B9) & 0xFFFFFFFF, (k1 + 0xBB67AE85) & 0xFFFFFFFF
    return np.stack(x, 1).astype(np.uint32)


def threshold(p):
    return int((1.0 - p) * 65536 + 0.5)


def kept(n, p, seed, offset):
    """Which of n values a dropout keeps."""
    with np.errstate(over="ignore"):
        w = philox(np.arange((n + 7) // 8, dtype=U) + U(offset), seed)
    return w.astype("<u4").view("<u2").reshape(-1)[:n] < threshold(p)


def dropout(x, p, seed, offset, residual=None):
    x = np.asarray(x, np.float64)
    y = np.where(kept(x.size, p, seed, offset).reshape(x.shape), x * (65536 / threshold(p)), 0.0)
    return y if residual is None else y + residual


def embedding(table, tokens, scale):
    t = np.asarray(table, np.float64)
    ok = (tokens >= 0) & (tokens < len(t))
    return np.where(ok[..., None], t[np.where(ok, tokens, 0)] * scale, 0.0)


def embedding_backward(dy, tokens, V, scale):
    """The gradient and, for its tolerance, the scaled sums of magnitudes and the number of terms of each class."""
    D = dy.shape[-1]
    dy, t = np.asarray(dy, np.float64).reshape(-1, D), np.asarray(tokens).reshape(-1)
    ok = (t >= 0) & (t < V)
    dW, mag, n = np.zeros((V, D)), np.zeros((V, D)), np.zeros(V, np.int64)
    np.add.at(dW, t[ok], dy[ok] * scale)
    np.add.at(mag, t[ok], np.abs(dy[ok] * scale))
    np.add.at(n, t[ok], 1)
    return dW, mag, n
