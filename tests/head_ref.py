"""The operators of a language model's head in 64 bits on the CPU, for tests: layer norm, 8-bit checkpoints, softmax cross
entropy, their gradients, and bounds for what 32-bit sums and bf16 roundings may do to them."""
import numpy as np

EPS32, HALF_BF16 = 2.0 ** -24, 2.0 ** -8          # unit roundings: half a step, relative


def layer_norm(x, gamma, beta, eps):
    mean = x.mean(-1, keepdims=True)
    rstd = 1 / np.sqrt(((x - mean) ** 2).mean(-1, keepdims=True) + eps)
    return (x - mean) * rstd * gamma + beta, mean, rstd


def layer_norm_grad(dy, x, gamma, mean, rstd):
    """-> dx, dgamma, dbeta; x: the values the backward pass sees (a checkpoint's, say), mean, rstd: of the forward pass"""
    xh = (x - mean) * rstd
    g = dy * gamma
    dx = rstd * (g - g.mean(-1, keepdims=True) - xh * (g * xh).mean(-1, keepdims=True))
    return dx, (dy * xh).sum(-2), dy.sum(-2)


def checkpoint(x):
    """-> values, int8 q, byte e + 127, of float32 x [..., d]"""
    x = np.asarray(x, dtype=np.float64)
    d = x.shape[-1]
    f = -(-d // 32) * 32
    g = np.zeros(x.shape[:-1] + (f,))
    g[..., :d] = x
    g = g.reshape(x.shape[:-1] + (f // 32, 32))
    top = np.abs(g).max(-1)
    poison = ~np.isfinite(top)
    e = np.full(top.shape, -126, dtype=np.int64)
    for cand in range(-126, 123):                  # the least that holds the group, by definition
        need = (top > 127.0 * 2.0 ** (cand - 1)) & ~poison
        e = np.where(need & (cand > -126), cand, e)
    q = np.where(poison[..., None], 0, np.rint(np.where(poison[..., None], 0, g) * 2.0 ** -e[..., None].astype(np.float64)))
    v = np.where(poison[..., None], np.nan, q * 2.0 ** e[..., None].astype(np.float64))
    shape = x.shape[:-1] + (f,)
    return v.reshape(shape)[..., :d], q.reshape(shape).astype(np.int8), np.where(poison, 255, e + 127).astype(np.uint8)


def class_loss(x, w, bias, y):
    """x [T][D], w [D][V], bias [V] or None, y [T] -> dict with loss, row_loss, dx, dw, db and the pieces of their bounds"""
    T, V = x.shape[0], w.shape[1]
    live = (y >= 0) & (y < V)
    x = np.where(live[:, None], x, 0.0)            # rows without a label take no part, whatever they hold
    z = x @ w + (0 if bias is None else bias)
    top = z.max(1, keepdims=True) if T else z[:, :1]
    e = np.exp(z - top)
    total = e.sum(1, keepdims=True)
    lse = (top + np.log(total))[:, 0]
    at = np.where(live, y, 0)
    row = np.where(live, lse - z[np.arange(T), at], 0.0)
    n = max(1, int(live.sum()))
    g = e / total * live[:, None]
    p = g.copy()
    g[np.arange(T)[live], at[live]] -= 1
    g /= n
    return dict(loss=row.sum() / n, row_loss=row, dx=g @ w.T, dw=x.T @ g, db=g.sum(0), g=g, p=p / n, z=z, x=x, live=live, n=n)


def class_loss_bounds(r, w, bias, bf16):
    """How far 32-bit sums (and bf16 operands of the two gradient products) may be off: every sum of k terms is allowed k + 16 unit
    roundings of the sum of its terms' magnitudes."""
    x, g, p = r["x"], r["g"], r["p"]
    (T, D), V = x.shape, w.shape[1]
    ax, aw = np.abs(x), np.abs(w)
    zerr = ((D + 16) * EPS32 * (ax @ aw) + 4 * EPS32 * np.abs(np.where(np.isfinite(r["z"]), r["z"], 0))).max(1) if T else np.zeros(0)
    big = np.abs(np.where(np.isfinite(r["z"]), r["z"], 0)).max(1) if T else np.zeros(0)
    row = 2 * zerr + (V ** 0.5 + 40) * EPS32 * (1 + big)
    gerr = p * (2 * zerr + (V ** 0.5 + 40 + 2 * big) * EPS32)[:, None] + 4 * EPS32 * np.abs(g)
    gop = gerr + (HALF_BF16 * np.abs(g) if bf16 else 4 * EPS32 * np.abs(g))
    out = HALF_BF16 if bf16 else EPS32
    ag = np.abs(g)
    return dict(row_loss=row, loss=row.sum() / r["n"] + (T + 16) * EPS32 * abs(r["loss"]),
                dx=gop @ aw.T + (V + 16) * EPS32 * (ag @ aw.T) + out * np.abs(r["dx"]),
                dw=ax.T @ gop + (T + 16) * EPS32 * (ax.T @ ag) + out * np.abs(r["dw"]),
                db=gerr.sum(0) + (T + 16) * EPS32 * ag.sum(0))
