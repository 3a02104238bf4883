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


def policy(H, W, bias, tokens, adv, old, ref, w, lo, hi, kl):
    """Policy loss on the head and its gradients, in 64 bits (old, ref, w, bias: None as in the library)."""
    H, W = np.asarray(H, np.float64), np.asarray(W, np.float64)
    M, V = len(H), len(W)
    z = H @ W.T + (0.0 if bias is None else np.asarray(bias, np.float64))
    top = z.max(1, keepdims=True) if M else np.zeros((0, 1))
    lam = top + np.log(np.exp(z - top).sum(1, keepdims=True))
    p = np.exp(z - lam)
    ok = (tokens >= 0) & (tokens < V)
    rows = np.nonzero(ok)[0]
    logp, losses, g = np.zeros(M), np.zeros(M), np.zeros(M)
    w = np.ones(M) if w is None else np.asarray(w, np.float64)
    for m in rows:
        lp = logp[m] = z[m, tokens[m]] - lam[m, 0]
        r = 1.0 if old is None else np.exp(lp - float(old[m]))
        A = float(adv[m])
        a, b = r * A, min(max(r, 1 - lo), 1 + hi) * A
        losses[m] = -min(a, b)
        g[m] = -A * r if a <= b else 0.0
        if ref is not None:
            d = float(ref[m]) - lp
            losses[m] += kl * (np.exp(d) - d - 1)
            g[m] += kl * (1 - np.exp(d))
    g *= w
    dZ = -g[:, None] * p
    dZ[rows, tokens[rows]] += g[rows]
    return {"loss": float((losses * w)[rows].sum()), "losses": losses, "logp": logp, "g": g, "p": p, "dZ": dZ,
            "dH": dZ @ W, "dW": dZ.T @ H, "db": dZ.sum(0)}


def _act(a, name):
    """act(a) and its derivative."""
    from scipy.special import erfc, expit
    if name == "silu":
        s = expit(a)
        return a * s, s * (1 + a * (1 - s))
    c = 0.5 * erfc(-a / np.sqrt(2.0))
    return a * c, c + a * np.exp(-0.5 * a * a) / np.sqrt(2 * np.pi)


def gated_ffn(x, wg, wu, wd, act, dy=None, r=lambda v, n: v):
    """The block and, with dy, its gradients.  r(v, name): what is done to an intermediate result (nothing)."""
    a, b = r(x @ wg.T, "gate"), r(x @ wu.T, "up")
    f, df = _act(a, act)
    h = r(f * b, "h")
    out = {"gate": a, "up": b, "h": h, "y": h @ wd.T}
    if dy is not None:
        dh = dy @ wd
        da, db = r(dh * b * df, "da"), r(dh * f, "db")
        out.update(dh=dh, da=da, db=db, dx=da @ wg + db @ wu, dw_gate=da.T @ x, dw_up=db.T @ x, dw_down=dy.T @ h)
    return out
