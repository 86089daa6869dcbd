"""The operators of a next-word model's layers and answers in 64 bits on the CPU, for tests: dropout's draws, a dense layer with what
follows it, log probabilities with entropy and alternatives, their gradients, and bounds for what 32-bit sums and roundings may do."""
import math

import numpy as np

from tests.head_ref import EPS32, HALF_BF16

GELU = math.sqrt(2 / math.pi), 0.044715


# ---- dropout ---------------------------------------------------------------------------------------------------------
def philox(counter, key):
    """Philox4x32-10 of arrays of four words and two"""
    m = np.uint64(0xffffffff)
    c, k = [np.asarray(v, dtype=np.uint64) for v in counter], [int(v) for v in key]
    for _ in range(10):
        a, b = c[0] * np.uint64(0xD2511F53), c[2] * np.uint64(0xCD9E8D57)
        c = [(b >> np.uint64(32)) ^ c[1] ^ np.uint64(k[0]), b & m, (a >> np.uint64(32)) ^ c[3] ^ np.uint64(k[1]), a & m]
        k = [(k[0] + 0x9E3779B9) % 2 ** 32, (k[1] + 0xBB67AE85) % 2 ** 32]
    return c


def limit(p):
    """65536 p as the library rounds it, of the float that it is given"""
    return min(65535, int(65536.0 * float(np.float32(p)) + 0.5))


def kept(n, rows, cols, p, seed, call):
    """-> which values stay [n, rows, cols], what they are multiplied by"""
    k, r, j = np.meshgrid(np.arange(n), np.arange(rows), np.arange(-(-cols // 8)), indexing="ij")
    call %= 2 ** 64
    words = philox((r, j + 65536 * k, np.full_like(r, call % 2 ** 32), np.full_like(r, call >> 32)), (seed % 2 ** 32, seed >> 32))
    u = np.stack([(w >> np.uint64(s)) & np.uint64(0xffff) for w in words for s in (0, 16)], -1).reshape(n, rows, -1)[:, :, :cols]
    return u >= limit(p), 65536.0 / (65536 - limit(p))


def dropped(x, p, seed, call):
    stay, scale = kept(*x.shape, p, seed, call)
    return np.where(stay, x * scale, 0.0)


# ---- dense layer -----------------------------------------------------------------------------------------------------
def _sigmoid(t):
    with np.errstate(over="ignore"):
        return 1 / (1 + np.exp(-t))


def activate(z, kind):
    if kind == "relu":
        return np.maximum(z, 0)
    if kind == "silu":
        return z * _sigmoid(z)
    if kind == "gelu":
        return 0.5 * z * (1 + np.tanh(GELU[0] * (z + GELU[1] * z ** 3)))
    return z


def slope(z, kind):
    if kind == "relu":
        return (z > 0).astype(np.float64)
    if kind == "silu":
        s = _sigmoid(z)
        return s + z * s * _sigmoid(-z)
    if kind == "gelu":
        u = 2 * GELU[0] * (z + GELU[1] * z ** 3)
        return _sigmoid(u) + z * _sigmoid(u) * _sigmoid(-u) * 2 * GELU[0] * (1 + 3 * GELU[1] * z ** 2)
    return np.ones_like(z)


def layer(x, w, bias, residual, kind, p, seed, call, bf16):
    """-> pre, y and the bounds of both.  A sum of k terms is allowed k + 16 unit roundings of its terms' magnitudes.  The activations rise
    by 1.13 at most for each unit of z; the exponential's argument t is off by 3 roundings of itself and its value by 2 more, which reaches
    s(t) times 1 - s(t), at most 0.28 / |t|: with the additions, the reciprocal and the last product 8 roundings of z."""
    z = np.matmul(x, w)
    terms = np.matmul(np.abs(x), np.abs(w))
    if bias is not None:
        z, terms = z + bias[:, None], terms + np.abs(bias[:, None])
    zerr = (x.shape[-1] + 16) * EPS32 * terms
    out = HALF_BF16 if bf16 else EPS32
    a = activate(z, kind)
    aerr = 1.13 * zerr + 8 * EPS32 * np.abs(z)
    stay, scale = kept(*z.shape, p, seed, call) if limit(p) else (np.ones(z.shape, bool), 1.0)
    y, yerr = np.where(stay, a * scale, 0.0), np.where(stay, aerr * scale, 0.0) + 2 * EPS32 * np.abs(a) * scale
    if residual is not None:
        y, yerr = y + residual, yerr + EPS32 * (np.abs(y) + np.abs(residual))
    return dict(pre=z, y=y), dict(pre=zerr + out * (np.abs(z) + zerr), y=yerr + out * (np.abs(y) + yerr))


def layer_grad(dy, pre, x, w, kind, p, seed, call, bf16):
    """-> dx, dw, db and their bounds.  The slope is a sum of a sigmoid, off as in layer(), and z times it times its complement times a factor
    that stays under 4 where the complement is not nothing: 32 roundings."""
    d = dropped(dy, p, seed, call) if limit(p) else dy
    dz = d * (slope(pre, kind) if kind != "none" else 1.0)
    err = 32 * EPS32 * np.abs(d) * (kind in ("gelu", "silu")) + 4 * EPS32 * np.abs(dz)
    op = err + (HALF_BF16 * (np.abs(dz) + err) if bf16 and (kind != "none" or limit(p)) else 0)
    out = HALF_BF16 if bf16 else EPS32
    t = lambda a: np.swapaxes(a, -1, -2)  # noqa: E731
    rows, n_out = dz.shape[1:]
    dx, dw, db = np.matmul(dz, t(w)), np.matmul(t(x), dz), dz.sum(1)
    bx = np.matmul(op, np.abs(t(w))) + (n_out + 16) * EPS32 * np.matmul(np.abs(dz), np.abs(t(w)))
    bw = np.matmul(np.abs(t(x)), op) + (rows + 16) * EPS32 * np.matmul(np.abs(t(x)), np.abs(dz))
    bb = err.sum(1) + (rows + 16) * EPS32 * np.abs(dz).sum(1)
    return dict(dx=dx, dw=dw, db=db), dict(dx=bx + out * (np.abs(dx) + bx), dw=bw + out * (np.abs(dw) + bw), db=bb)


# ---- log probabilities -------------------------------------------------------------------------------------------------
def scores(z, tokens, n_top):
    """z [rows][v] without NaN or +inf, tokens [rows][k] -> dict; rows of -inf alone as the header says"""
    rows, v = z.shape
    top = z.max(1, keepdims=True)
    empty = ~np.isfinite(top[:, 0])
    d = np.where(empty[:, None], -np.inf, z - np.where(np.isfinite(top), top, 0))
    s = np.exp(d).sum(1, keepdims=True)
    log_s = np.log(np.where(empty[:, None], 1, s))
    lp = d - log_s
    p = np.exp(lp)
    plp = np.where(p > 0, p * np.where(p > 0, lp, 0), 0)
    valid = (tokens >= 0) & (tokens < v)
    at = np.where(valid, tokens, 0)
    logp = np.where(valid, np.take_along_axis(lp, at, 1), 0.0)
    order = np.argsort(-z, axis=1, kind="stable")[:, :n_top]
    return dict(logp=logp, entropy=-plp.sum(1), top=order, top_logp=np.take_along_axis(lp, order, 1), p=p, lp=lp, plp=plp, d=d, log_s=log_s, empty=empty,
                valid=valid, at=at)


def scores_grad(r, dlogp, dentropy):
    g = np.where(r["valid"], dlogp, 0.0) * ~r["empty"][:, None]
    dz = -r["p"] * g.sum(1, keepdims=True) - dentropy[:, None] * (r["plp"] + r["p"] * r["entropy"][:, None])
    for i in range(g.shape[1]):
        dz[np.arange(len(dz)), r["at"][:, i]] += g[:, i]
    return dz


def scores_bounds(r, dlogp=None, dentropy=None, bf16=0):
    """A thread adds 64 terms at most, some 32 additions join the threads and pieces: 112 roundings with those of a term's own; its exp is off by
    2 |d| + 2 roundings, d the distance to the largest."""
    e, p = EPS32, r["p"]
    d = np.where(np.isfinite(r["d"]), np.abs(r["d"]), 0)
    rel = (p * (2 * d + 112)).sum(1, keepdims=True) * e                      # of S
    lerr = rel + 2 * e * np.abs(r["log_s"])
    lp = np.where(np.isfinite(r["lp"]), np.abs(r["lp"]), 0)
    mean = (p * d).sum(1, keepdims=True)
    herr = (lerr + (p * d * (2 * d + 114)).sum(1, keepdims=True) * e + mean * (rel + 4 * e) + 2 * e * np.abs(r["entropy"])[:, None])[:, 0]
    one = e * d + lerr + e * lp                                             # of a log p
    out = dict(entropy=herr, lp=one)
    if dlogp is not None:
        g = np.where(r["valid"], np.abs(dlogp), 0).sum(1, keepdims=True)
        a = g + np.abs(dentropy)[:, None] * (lp + r["entropy"][:, None])
        perr = one + (2 * lp + 4) * e
        # a p below the smallest normal float, 2^-126, may be taken for zero: exp2 has no subnormal results.  What it would be times a is lost
        dz = 2.0 ** -126 * a + p * (perr * a + (dlogp.shape[1] + 4) * e * a + np.abs(dentropy)[:, None] * (one + herr[:, None]))
        for i in range(dlogp.shape[1]):
            dz[np.arange(len(dz)), r["at"][:, i]] += (dlogp.shape[1] + 4) * e * (g + a.max(1, keepdims=True) * (p > 0).any(1, keepdims=True))[:, 0] * r["valid"][:, i]
        out["dz"] = dz + (HALF_BF16 if bf16 else e) * (np.abs(scores_grad(r, dlogp, dentropy)) + dz)
    return out
