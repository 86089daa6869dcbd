"""Operators of a next-word model's layers and answers on replicas, as cases that can be timed and compared: a dense layer with
bias, activation, dropout and residual in one pass and its gradient, dropout on its own, and the log probabilities of given
tokens with entropy and top alternatives, with their gradient.

Every operator is grouped: replica k of a federated round has its own activations, weights and gradients.  Types are
"f32" and "bf16" (activations, weights, logits and the gradients of these; biases, their gradients, log probabilities and
entropies are 32-bit floats always).
"""
import math

import torch

own = False
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
GELU = math.sqrt(2 / math.pi), 0.044715


def listed():
    return [
        # serving: one token through a widening layer
        dict(name="layer-token", op="layer", mode="forward", n=1, rows=1, inputs=512, outputs=2048, activation="gelu", bias=True,
             residual=False, drop=0.0, type="bf16"),
        # a small network's hidden layer (784 inputs, 128 units, batch 32, four replicas)
        dict(name="layer-small-f32", op="layer", mode="forward", n=4, rows=32, inputs=784, outputs=128, activation="relu", bias=True,
             residual=False, drop=0.0, type="f32"),
        # fp32 training at sizes that divide by nothing: what follows an activation, back onto the residual
        dict(name="layer-odd-f32", op="layer", mode="forward", n=2, rows=1001, inputs=777, outputs=1111, activation="silu", bias=True,
             residual=True, drop=0.1, type="f32"),
        # the largest: long batches through a 4096-wide layer, with dropout onto the residual
        dict(name="layer-large-bf16", op="layer", mode="forward", n=4, rows=8192, inputs=4096, outputs=4096, activation="none", bias=True,
             residual=True, drop=0.1, type="bf16"),
        # a gradient at sizes that divide by nothing
        dict(name="layer-grad-odd-f32", op="layer", mode="grad", n=3, rows=500, inputs=777, outputs=1000, activation="silu", bias=True,
             residual=False, drop=0.1, type="f32"),
        # sixteen replicas' widening layers, 16 sequences of 64 tokens
        dict(name="layer-grad-n16-bf16", op="layer", mode="grad", n=16, rows=1024, inputs=512, outputs=2048, activation="gelu", bias=True,
             residual=False, drop=0.0, type="bf16"),
        # dropout of a small batch's embeddings
        dict(name="drop-small-f32", op="drop", mode="train", n=4, rows=255, features=129, p=0.1, residual=False, type="f32"),
        # dropout onto the residual stream, long batches
        dict(name="drop-large-bf16", op="drop", mode="train", n=16, rows=2048, features=4096, p=0.2, residual=True, type="bf16"),
        # answering: one token's alternatives
        dict(name="scores-token", op="scores", mode="forward", n=1, rows=1, classes=32000, tokens=1, top=8, masked=0.0, type="bf16"),
        # evaluation of replicas on held-out text
        dict(name="scores-n4-f32", op="scores", mode="forward", n=4, rows=512, classes=20011, tokens=1, top=5, masked=0.1, type="f32"),
        # evaluation with candidates, a large vocabulary
        dict(name="scores-large-bf16", op="scores", mode="forward", n=2, rows=4096, classes=65536, tokens=4, top=5, masked=0.0, type="bf16"),
        # training on weighted log probabilities and entropy
        dict(name="scores-train-bf16", op="scores", mode="train", n=4, rows=1000, classes=32000, tokens=2, top=0, masked=0.0, type="bf16"),
    ]


def draw(rng):
    def size(lo, hi):                                     # spread over the logarithm; one in two divides by 8 or more
        v = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
        if rng.random() < 0.5 and v >= 64:
            v = v // 32 * 32
        return min(hi, max(lo, v))

    typ = rng.choice(["f32", "bf16"])
    op = rng.choice(["layer", "layer", "drop", "scores"])
    if op == "layer":
        case = dict(op=op, mode=rng.choice(["forward", "grad"]), n=size(1, 16), rows=size(1, 8192), inputs=size(48, 4096), outputs=size(33, 4096),
                    activation=rng.choice(["none", "relu", "gelu", "silu"]), bias=rng.random() < 0.7, residual=rng.random() < 0.5,
                    drop=rng.choice([0.0, 0.0, 0.1, 0.5]), type=typ)
        most = (5e11 if typ == "bf16" else 1e11) / (2 if case["mode"] == "grad" else 1)
        while case["n"] > 1 and case["n"] * case["inputs"] * case["outputs"] * max(256, case["rows"]) > most:
            case["n"] -= 1
    elif op == "drop":
        case = dict(op=op, mode=rng.choice(["forward", "train"]), n=size(1, 16), rows=size(1, 4096), features=size(33, 8192),
                    p=rng.choice([0.05, 0.1, 0.5]), residual=rng.random() < 0.5, type=typ)
        while case["n"] > 1 and case["n"] * case["rows"] * case["features"] > 67e6:
            case["n"] -= 1
    else:
        case = dict(op=op, mode=rng.choice(["forward", "train"]), n=size(1, 8), rows=size(1, 4096), classes=size(1000, 131072), tokens=size(1, 16),
                    top=rng.choice([0, 1, 5, 20]), masked=rng.choice([0.0, 0.0, 0.3]), type=typ)
        while case["n"] > 1 and case["n"] * case["rows"] * case["classes"] > 268e6:
            case["n"] -= 1
        if case["rows"] * case["classes"] > 268e6:
            case["rows"] = 2048
    return case


# ---- inputs ----------------------------------------------------------------------------------------------------------
class _Make:
    def __init__(self, seed):
        self.g = torch.Generator(device="cuda").manual_seed(int(seed))

    def normal(self, *shape, std=1.0, dtype=torch.float32):
        out = torch.empty(shape, dtype=torch.float32, device="cuda").normal_(0.0, std, generator=self.g)
        return out.to(dtype)

    def uniform(self, *shape):
        return torch.rand(shape, generator=self.g, device="cuda")


def _draw_state(s, m, seed):
    """What decides which values are dropped: a run's seed, a layer's call number and the step's counter on the device."""
    s["seed"], s["call"] = int(seed) * 0x9E3779B97F4A7C15 % 2 ** 64, 7 << 32
    s["counter"] = torch.full((1,), int(seed) % 1000 + 3, dtype=torch.int64, device="cuda")


def prepare(case, seed):
    m, t, n, rows = _Make(seed), TYPES[case["type"]], case["n"], case["rows"]
    bf16 = int(case["type"] == "bf16")
    s = dict(case=case)
    if case["op"] == "layer":
        i, o = case["inputs"], case["outputs"]
        s["x"], s["w"] = m.normal(n, rows, i, dtype=t), m.normal(n, i, o, std=1 / math.sqrt(i), dtype=t)
        s["bias"] = m.normal(n, o, std=0.2) if case["bias"] else None
        s["residual"] = m.normal(n, rows, o, dtype=t) if case["residual"] and case["mode"] == "forward" else None
        if case["mode"] == "grad":
            s["dy"] = m.normal(n, rows, o, std=1e-2, dtype=t)
            s["pre"] = m.normal(n, rows, o, dtype=t) if case["activation"] != "none" else None       # as the forward pass left it
        _draw_state(s, m, seed)
    elif case["op"] == "drop":
        d = case["features"]
        s["x"] = m.normal(n, rows, d, dtype=t)
        s["residual"] = m.normal(n, rows, d, dtype=t) if case["residual"] else None
        if case["mode"] == "train":
            s["dy"] = m.normal(n, rows, d, std=1e-2, dtype=t)
        _draw_state(s, m, seed)
    else:
        v, k = case["classes"], case["tokens"]
        z = m.normal(n, rows, v, std=2.0) + 3 * m.normal(n, rows, 1)
        # a model's row has a few likely words: some logits of every row are raised
        at = (m.uniform(n, rows, 16) * v).long().clamp(max=v - 1)
        z.scatter_reduce_(2, at, 4 * m.normal(n, rows, 16).abs() + 4 + 3 * m.normal(n, rows, 1), "amax")
        if case["masked"]:
            z.masked_fill_(m.uniform(n, 1, v) < case["masked"], -math.inf)         # words that an answer may not hold
            z[:, :, 0] = 0.0                                                       # one at least that it may
        s["logits"] = z.to(t)
        # word frequencies fall off as in a text: log-uniform ranks; -1 is no token (padding)
        tokens = (torch.exp(m.uniform(n, rows, k) * math.log(v)).floor() - 1).clamp(0, v - 1).to(torch.int32)
        s["tokens"] = torch.where(m.uniform(n, rows, 1) < 0.05, torch.full_like(tokens, -1), tokens)
        if case["mode"] == "train":
            s["dlogp"], s["dentropy"] = m.normal(n, rows, k, std=1e-2), m.normal(n, rows, std=1e-2)
    if own:
        from paper_2111_08274_amd import hadfl
        if case["op"] == "layer":
            s["plan"] = hadfl.DenseLayer(n, rows, case["inputs"], case["outputs"], bf16=bf16, activation=case["activation"], drop=case["drop"],
                                         grad=case["mode"] == "grad")
        elif case["op"] == "drop":
            s["plan"] = hadfl.Dropout(n, rows, case["features"], case["p"], bf16=bf16)
        else:
            s["plan"] = hadfl.TokenScores(n, rows, case["classes"], n_tokens=case["tokens"], n_top=case["top"], bf16=bf16)
    return s


# ---- the plain forms ---------------------------------------------------------------------------------------------------
def _threshold(p):
    return min(65535, math.floor(65536 * p + 0.5))


def _kept(s, n, rows, cols, p):
    """Which of [n, rows, cols] stay: Philox4x32-10 with the seed as key, its counter (row, column / 8 + 2^16 replica, the call's two
    words), eight 16-bit numbers for eight columns, each at least 65536 p."""
    low = 0xffffffff
    call = s["call"] + s["counter"]
    dev, chunks = call.device, (cols + 7) // 8
    c1 = torch.arange(chunks, device=dev) + (torch.arange(n, device=dev) << 16)[:, None, None]
    c0, c1 = torch.broadcast_tensors(torch.arange(rows, device=dev)[None, :, None], c1)
    c2, c3 = (call & low).expand(c0.shape), ((call >> 32) & low).expand(c0.shape)
    k0, k1 = s["seed"] & low, s["seed"] >> 32
    for _ in range(10):
        a, b = c0 * 0xD2511F53, c2 * 0xCD9E8D57                # modulo 2^64: all 64 bits of the products
        c0, c1, c2, c3 = ((b >> 32) & low) ^ c1 ^ k0, b & low, ((a >> 32) & low) ^ c3 ^ k1, a & low
        k0, k1 = (k0 + 0x9E3779B9) & low, (k1 + 0xBB67AE85) & low
    u = torch.stack([c0 & 0xffff, c0 >> 16, c1 & 0xffff, c1 >> 16, c2 & 0xffff, c2 >> 16, c3 & 0xffff, c3 >> 16], -1)
    return (u >= _threshold(p)).flatten(2)[:, :, :cols]


def _drop(s, x, p):
    if _threshold(p) == 0:
        return x
    return torch.where(_kept(s, *x.shape, p), x * (65536 / (65536 - _threshold(p))), torch.zeros_like(x))


def _act(z, kind):
    if kind == "relu":
        return torch.where(z > 0, z, torch.zeros_like(z))
    if kind == "gelu":
        return 0.5 * z * (1 + torch.tanh(GELU[0] * (z + GELU[1] * z * z * z)))
    if kind == "silu":
        return z / (1 + torch.exp(-z))
    return z


def _slope(z, kind):
    if kind == "relu":
        return (z > 0).to(z.dtype)
    if kind == "gelu":
        t = torch.tanh(GELU[0] * (z + GELU[1] * z * z * z))
        return 0.5 * (1 + t) + 0.5 * z * (1 - t * t) * GELU[0] * (1 + 3 * GELU[1] * z * z)
    if kind == "silu":
        e = 1 / (1 + torch.exp(-z))
        return e * (1 + z * (1 - e))
    return torch.ones_like(z)


def _layer(s, case):
    x, w, t = s["x"].float(), s["w"].float(), s["x"].dtype
    if case["mode"] == "forward":
        z = torch.matmul(x, w)
        if s["bias"] is not None:
            z += s["bias"][:, None]
        y = _drop(s, _act(z, case["activation"]), case["drop"])
        if s["residual"] is not None:
            y = s["residual"].float() + y
        out = {"y": y.to(t)}
        if case["activation"] != "none":
            out["pre"] = z.to(t)
        return out
    dz = _drop(s, s["dy"].float(), case["drop"])
    if s["pre"] is not None:
        dz = dz * _slope(s["pre"].float(), case["activation"])
    out = {"dx": torch.matmul(dz, w.transpose(1, 2).contiguous()).to(t), "dw": torch.matmul(x.transpose(1, 2).contiguous(), dz).to(t)}
    if case["bias"]:
        out["db"] = dz.sum(1)
    return out


def _dropout(s, case):
    y = _drop(s, s["x"].float(), case["p"])
    if s["residual"] is not None:
        y = s["residual"].float() + y
    out = {"y": y.to(s["x"].dtype)}
    if case["mode"] == "train":
        out["dx"] = _drop(s, s["dy"].float(), case["p"]).to(s["x"].dtype)
    return out


def _scores(s, case):
    z, tokens = s["logits"].float(), s["tokens"]
    v = case["classes"]
    top = z.amax(-1, keepdim=True)
    e = torch.exp(z - top)
    total = e.sum(-1, keepdim=True)
    log_total = torch.log(total)
    p = e / total
    lp = z - top - log_total
    weighted = torch.where(p > 0, p * lp, torch.zeros_like(p))
    entropy = -weighted.sum(-1)
    at = tokens.clamp(min=0).long()
    logp = torch.where(tokens >= 0, lp.gather(2, at), torch.zeros((), device=z.device))
    out = {"logp": logp, "entropy": entropy}
    if case["top"]:
        left, order = z.clone(), torch.arange(v, device=z.device, dtype=torch.int32)
        index = []
        for _ in range(case["top"]):                       # the largest that is left, the first of equals
            best = left.amax(-1, keepdim=True)
            first = torch.where(left == best, order, v).amin(-1, keepdim=True)
            index.append(first)
            left.scatter_(2, first.long(), -math.inf)
        out["top"] = torch.cat(index, -1)
        out["top_logp"] = lp.gather(2, out["top"].long())
    if case["mode"] == "train":
        g = torch.where(tokens >= 0, s["dlogp"], torch.zeros_like(s["dlogp"]))
        h = s["dentropy"][..., None]
        dz = -p * g.sum(-1, keepdim=True) - h * (weighted + p * entropy[..., None])
        for i in range(case["tokens"]):                    # one after the other: a token may be given twice
            dz.scatter_add_(2, at[..., i:i + 1], g[..., i:i + 1])
        out["dlogits"] = dz.to(s["logits"].dtype)
    return out


# ---- one pass ----------------------------------------------------------------------------------------------------------
def run(state):
    s, case = state, state["case"]
    if not own:
        return {"layer": _layer, "drop": _dropout, "scores": _scores}[case["op"]](s, case)
    plan = s["plan"]
    if case["op"] == "scores":
        logp, entropy, top, top_logp = plan.forward(s["logits"], s["tokens"])
        out = {"logp": logp, "entropy": entropy}
        if case["top"]:
            out["top"], out["top_logp"] = top, top_logp
        if case["mode"] == "train":
            out["dlogits"] = plan.backward(s["logits"], s["tokens"], s["dlogp"], s["dentropy"])
        return out
    draw_of = dict(seed=s["seed"], call=s["call"], counter=s["counter"])
    if case["op"] == "drop":
        out = {"y": plan.forward(s["x"], residual=s["residual"], **draw_of)}
        if case["mode"] == "train":
            out["dx"] = plan.backward(s["dy"], **draw_of)
        return out
    if case["mode"] == "forward":
        out = {}
        if case["activation"] != "none":
            out["pre"] = torch.empty((case["n"], case["rows"], case["outputs"]), dtype=s["x"].dtype, device=s["x"].device)
        out["y"] = plan.forward(s["x"], s["w"], s["bias"], residual=s["residual"], pre=out.get("pre"), **draw_of)
        return out
    want = ("dx", "dw", "db") if case["bias"] else ("dx", "dw")
    dx, dw, db = plan.backward(s["dy"], s["x"], s["w"], pre=s["pre"], want=want, **draw_of)
    out = {"dx": dx, "dw": dw}
    if case["bias"]:
        out["db"] = db
    return out


def work(case):
    n, rows, size = case["n"], case["rows"], {"f32": 4, "bf16": 2}[case["type"]]
    if case["op"] == "layer":
        i, o = case["inputs"], case["outputs"]
        act = case["activation"] != "none"
        if case["mode"] == "forward":
            tensors = rows * i + i * o + rows * o * (1 + act + case["residual"])
            return {"bytes": n * (tensors * size + (4 * o if case["bias"] else 0)), "flops": 2 * n * rows * i * o}
        tensors = 2 * rows * i + 2 * i * o + rows * o * (1 + act)
        return {"bytes": n * (tensors * size + (4 * o if case["bias"] else 0)), "flops": 4 * n * rows * i * o}
    if case["op"] == "drop":
        tensors = 2 + case["residual"] + (2 if case["mode"] == "train" else 0)
        return {"bytes": n * rows * case["features"] * size * tensors, "flops": 2 * n * rows * case["features"] * tensors}
    v, k, top = case["classes"], case["tokens"], case["top"]
    once = rows * (v * size + 8 * k + 4 + 8 * top)
    if case["mode"] == "train":
        once += rows * (v * size + 4 * k + 4)
    return {"bytes": n * once, "flops": n * rows * v * (5 if case["mode"] == "forward" else 12)}


# ---- the definitions in 64 bits ------------------------------------------------------------------------------------------
def exact(case, seed):
    s = prepare(case, seed)
    one = {"layer": _layer64, "drop": _drop64, "scores": _scores64}[case["op"]]
    outs = [one(case, s, k) for k in range(case["n"])]
    return {name: torch.stack([o[name] for o in outs]) for name in outs[0]}


def _words(value):
    return int(value) % 2 ** 32, int(value) // 2 ** 32 % 2 ** 32


def _times(c, factor):
    """High and low 32 bits of c * factor, the factor in two halves of 16 bits."""
    upper = c * (factor >> 16)                             # below 2^48
    lower = c * (factor & 0xffff)
    whole = upper + (lower >> 16)
    return whole >> 16, ((whole & 0xffff) << 16) | (lower & 0xffff)


def _factor64(s, k, rows, cols, p):
    """What a value of replica k is multiplied by: 0, or one over the share that stays."""
    limit = min(65535, math.floor(65536 * p + 0.5))
    x = torch.arange(rows, device="cuda")[:, None].expand(rows, -(-cols // 8))
    y = (torch.arange(x.shape[1], device="cuda") + 65536 * k)[None].expand(x.shape)
    call = _words(s["call"] + int(s["counter"]))
    z, w = torch.full_like(x, call[0]), torch.full_like(x, call[1])
    key = list(_words(s["seed"]))
    for _ in range(10):
        high_x, low_x = _times(x, 0xD2511F53)
        high_z, low_z = _times(z, 0xCD9E8D57)
        x, y, z, w = high_z ^ y ^ key[0], low_z, high_x ^ w ^ key[1], low_x
        key = [(key[0] + 0x9E3779B9) % 2 ** 32, (key[1] + 0xBB67AE85) % 2 ** 32]
    out = torch.empty(rows, x.shape[1], 4, 2, dtype=torch.float64, device="cuda")
    for i, word in enumerate((x, y, z, w)):
        for half in range(2):
            out[:, :, i, half] = ((word // 65536 ** half) % 65536 >= limit).double()
    return out.view(rows, -1)[:, :cols] * (65536 / (65536 - limit))


def _dropped64(s, k, x, p):
    f = _factor64(s, k, *x.shape, p)
    return torch.where(f > 0, x * f, torch.zeros_like(x))


def _layer64(case, s, k):
    x, w, kind = s["x"][k].double(), s["w"][k].double(), case["activation"]
    if case["mode"] == "forward":
        z = x @ w if s["bias"] is None else x @ w + s["bias"][k].double()
        sigmoid = {"gelu": lambda: torch.sigmoid(2 * GELU[0] * (z + GELU[1] * z ** 3)), "silu": lambda: torch.sigmoid(z)}
        y = z if kind == "none" else z.clamp(min=0) if kind == "relu" else z * sigmoid[kind]()
        y = _dropped64(s, k, y, case["drop"])
        if s["residual"] is not None:
            y = y + s["residual"][k].double()
        return {"y": y} if kind == "none" else {"y": y, "pre": z}
    dz = _dropped64(s, k, s["dy"][k].double(), case["drop"])
    if s["pre"] is not None:
        z = s["pre"][k].double()
        if kind == "relu":
            dz = torch.where(z > 0, dz, torch.zeros_like(dz))
        else:
            inner = 2 * GELU[0] * (z + GELU[1] * z ** 3) if kind == "gelu" else z
            along = 2 * GELU[0] * (1 + 3 * GELU[1] * z ** 2) if kind == "gelu" else torch.ones_like(z)
            up = torch.sigmoid(inner)
            dz = dz * (up + z * up * torch.sigmoid(-inner) * along)
    out = {"dx": dz @ w.t().contiguous(), "dw": x.t().contiguous() @ dz}
    if case["bias"]:
        out["db"] = dz.sum(0)
    return out


def _drop64(case, s, k):
    y = _dropped64(s, k, s["x"][k].double(), case["p"])
    out = {"y": y if s["residual"] is None else y + s["residual"][k].double()}
    if case["mode"] == "train":
        out["dx"] = _dropped64(s, k, s["dy"][k].double(), case["p"])
    return out


def _scores64(case, s, k):
    z, tokens = s["logits"][k].double(), s["tokens"][k].long()
    lp = torch.log_softmax(z, 1)
    plp = torch.special.entr(torch.exp(lp))                # -p log p
    entropy = plp.sum(1)
    valid = tokens >= 0
    row = torch.arange(case["rows"], device=z.device)[:, None].expand(tokens.shape)
    logp = torch.zeros(tokens.shape, dtype=torch.float64, device=z.device)
    logp[valid] = lp[row[valid], tokens[valid]]
    out = {"logp": logp, "entropy": entropy}
    if case["top"]:
        order = torch.sort(z, dim=1, descending=True, stable=True).indices[:, :case["top"]]
        out["top"], out["top_logp"] = order.to(torch.int32), lp.gather(1, order)
    if case["mode"] == "train":
        g = s["dlogp"][k].double() * valid
        p = torch.exp(lp)
        d = s["dentropy"][k].double()[:, None] * (plp - p * entropy[:, None]) - p * g.sum(1, keepdim=True)
        d.index_put_((row[valid], tokens[valid]), g[valid], accumulate=True)
        out["dlogits"] = d
    return out
