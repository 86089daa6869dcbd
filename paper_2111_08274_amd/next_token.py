"""Federated training of a next-token head on replicas: the cycle's selection and aggregation around the operators of a
language model's head.

    python -m paper_2111_08274_amd.next_token [--replicas 4] [--vocab 2003] [--width 128] [--cycles 20] [--blocks 0] [--drop 0] [--bf16]

Every replica holds one row of parameters (a bare row: the library trains nothing itself) with a dense layer, a layer norm and
the last dense layer over the vocabulary,

    h = relu(x W1 + b1),   y = layer_norm(h; gamma, beta),   loss = cross_entropy(y W2 + b2, next token),

x the fixed embedding of the last token.  With --blocks, h passes as many blocks h <- h + D(gelu(h U + a) V + c) before the norm, with --drop D
drops values (and of x too), other ones in every step.  A step is grouped over the replicas: what the backward pass needs of x and of h
is kept in 8 bits, the logits live in the loss's workspace alone, and a replica that has done its local steps of the round sits the others
out with rows that have no label.  After the rounds the aggregated model answers freshly drawn tokens of the training distribution, whose
right next ones have no noise: their log probabilities, entropies and alternatives, from its logits.  After the local steps the library selects replicas by their versions and aggregates their rows.

Tokens are synthetic: the next token is a fixed permutation of the last one, replaced by a uniform one with probability 1/8;
replica k sees mostly tokens of its own part of the vocabulary (shards that differ, as the method's devices do).
"""
import argparse
import json

import numpy as np

LOGITS = 1 << 28                   # that answers hold at once: 1 GiB of floats
COLUMNS = 1 << 17                  # of a dense layer


class Head:
    """Parameters of all replicas in rows [n, row_stride] (views into them), their gradients and the operators' plans."""

    def __init__(self, rows, n, batch, width, hidden, vocab, bf16=0, blocks=0, drop=0.0, seed=0):
        import torch
        from . import hadfl
        self.torch, self.rows, self.bf16 = torch, rows, bf16
        self.n, self.batch, self.width, self.hidden, self.vocab = n, batch, width, hidden, vocab
        self.blocks, self.drop, self.seed = blocks, drop, seed
        self.dtype = torch.bfloat16 if bf16 else torch.float32
        self.grads = torch.zeros_like(rows)
        at, self.p, self.g = 0, {}, {}
        for name, shape in self.layout(width, hidden, vocab, blocks):
            size = int(np.prod(shape))
            for views, t in ((self.p, rows), (self.g, self.grads)):
                views[name] = t[:, at:at + size].unflatten(1, shape)
            at += size
        self.kept_x = hadfl.PackedRows(n, batch, width, bf16)
        self.kept_h = hadfl.PackedRows(n, batch, hidden, bf16)
        self.norm = hadfl.LayerNorm(n, batch, hidden, bf16)
        self.dense = hadfl.DenseGrad(n, batch, width, hidden, bf16)
        self.loss = hadfl.ClassLoss(n, batch, hidden, vocab, bf16)
        self.drop_x = hadfl.Dropout(n, batch, width, drop, bf16) if drop else None
        if blocks:
            self.up = hadfl.DenseLayer(n, batch, hidden, 2 * hidden, bf16, activation="gelu")
            self.down = hadfl.DenseLayer(n, batch, 2 * hidden, hidden, bf16, drop=drop)
            self.kept = [(hadfl.PackedRows(n, batch, hidden, bf16), hadfl.PackedRows(n, batch, 2 * hidden, bf16),
                          torch.empty((n, batch, 2 * hidden), dtype=self.dtype, device=rows.device)) for _ in range(blocks)]
        self.steps = torch.zeros(1, dtype=torch.int64, device=rows.device)        # the dropouts' counter

    @staticmethod
    def layout(width, hidden, vocab, blocks=0):
        inner = [q for i in range(blocks) for q in (("u%d" % i, (hidden, 2 * hidden)), ("a%d" % i, (2 * hidden,)), ("v%d" % i, (2 * hidden, hidden)), ("c%d" % i, (hidden,)))]
        return (("w1", (width, hidden)), ("b1", (hidden,)), *inner, ("gamma", (hidden,)), ("beta", (hidden,)), ("w2", (hidden, vocab)), ("b2", (vocab,)))

    @staticmethod
    def size(width, hidden, vocab, blocks=0):
        return sum(int(np.prod(s)) for _, s in Head.layout(width, hidden, vocab, blocks))

    def weights(self, name):
        return self.p[name].to(self.dtype) if self.bf16 else self.p[name]

    def drawn(self, call):
        """Which values a dropout of the present step keeps: calls are 2^32 apart, the steps lie between."""
        return dict(seed=self.seed, call=call << 32, counter=self.steps)

    def first(self, x):
        torch, p = self.torch, self.p
        h = torch.relu(torch.baddbmm(p["b1"][:, None], x.float(), p["w1"]))
        return h.to(self.dtype), h > 0

    def step(self, x, labels):
        """x [n, batch, width] of the plan's type, labels [n, batch] int32 -> mean losses [n]; the gradients are left in `grads`."""
        p, g = self.p, self.g
        if self.drop:
            x = self.drop_x.forward(x, **self.drawn(0))
        self.kept_x.pack(x)
        h, on = self.first(x)
        for i in range(self.blocks):
            kept_h, kept_a, pre = self.kept[i]
            kept_h.pack(h)
            a = self.up.forward(h, self.weights("u%d" % i), p["a%d" % i], pre=pre)
            kept_a.pack(a)
            h = self.down.forward(a, self.weights("v%d" % i), p["c%d" % i], residual=h, **self.drawn(1 + i))
        self.kept_h.pack(h)
        y = self.norm.forward(h, p["gamma"], p["beta"])
        loss, _, dy, dw2, _ = self.loss.grad(y, self.weights("w2"), labels, p["b2"], dw=None if self.bf16 else g["w2"], db=g["b2"])
        if self.bf16:
            g["w2"].copy_(dw2)
        dh, _, _ = self.norm.backward(dy, self.kept_h, p["gamma"], dgamma=g["gamma"], dbeta=g["beta"])
        for i in reversed(range(self.blocks)):
            kept_h, kept_a, pre = self.kept[i]
            u, v = "u%d" % i, "v%d" % i
            da, dv, _ = self.down.backward(dh, kept_a, self.weights(v), dw=None if self.bf16 else g[v], db=g["c%d" % i], **self.drawn(1 + i))
            dx, du, _ = self.up.backward(da, kept_h, self.weights(u), pre=pre, dw=None if self.bf16 else g[u], db=g["a%d" % i])
            if self.bf16:
                g[u].copy_(du)
                g[v].copy_(dv)
            dh = dh + dx
        self.dense.backward(self.kept_x, dh * on, dw=g["w1"], db=g["b1"])
        self.steps.add_(1)
        return loss

    def answers(self, x, tokens, top=0):
        """What the model says of x [n, batch, width], without dropout: log probabilities of tokens [n, batch, k] int32, entropy [n, batch] and
        the top classes with theirs."""
        from . import hadfl
        p = self.p
        h, _ = self.first(x)
        for i in range(self.blocks):
            a = self.up.forward(h, self.weights("u%d" % i), p["a%d" % i])
            h = hadfl.DenseLayer(self.n, self.batch, 2 * self.hidden, self.hidden, self.bf16, grad=False).forward(a, self.weights("v%d" % i), p["c%d" % i], residual=h)
        y, w2 = self.norm.forward(h, p["gamma"], p["beta"], stats=False), self.weights("w2")
        rows = max(1, min(self.batch, LOGITS // (self.n * self.vocab)))       # of the batch, whose logits are there at once
        columns = -(-self.vocab // -(-self.vocab // COLUMNS))
        outs = []
        for at in range(0, max(1, self.batch), rows):
            x, given = y[:, at:at + rows], tokens[:, at:at + rows].contiguous()
            logits = self.torch.empty((self.n, x.shape[1], self.vocab), dtype=self.dtype, device=y.device)
            for c in range(0, self.vocab, columns):
                z = logits[:, :, c:c + columns]
                hadfl.DenseLayer(self.n, x.shape[1], self.hidden, z.shape[2], self.bf16, grad=False).forward(x, w2[:, :, c:c + columns], p["b2"][:, c:c + columns], y=z)
            outs.append(hadfl.TokenScores(self.n, x.shape[1], self.vocab, n_tokens=tokens.shape[2], n_top=top, bf16=self.bf16).forward(logits, given))
        return outs[0] if len(outs) == 1 else tuple(None if q[0] is None else self.torch.cat(q, 1) for q in zip(*outs))

    def update(self, lr):
        self.rows.sub_(self.grads, alpha=lr)


class Tokens:
    def __init__(self, n, vocab, seed=0):
        rng = np.random.default_rng(seed)
        self.rng, self.n, self.vocab = rng, n, vocab
        self.next = rng.permutation(vocab)

    def batch(self, size):
        own = (np.arange(self.n)[:, None] + self.rng.random((self.n, size))) * self.vocab / self.n
        last = np.where(self.rng.random((self.n, size)) < 0.75, own, self.rng.random((self.n, size)) * self.vocab).astype(np.int64)
        after = np.where(self.rng.random((self.n, size)) < 0.125, self.rng.integers(0, self.vocab, size=(self.n, size)), self.next[last])
        return last, after.astype(np.int32)


def run(replicas=4, n_select=2, vocab=2003, width=128, hidden=256, batch=256, cycles=20, steps_per_unit=2, lr=1.0, bf16=0, seed=0, blocks=0, drop=0.0):
    """-> dict with the mean training loss of every cycle and the members of every selection"""
    import torch
    from . import hadfl, synth
    dev = torch.device("cuda", torch.cuda.current_device())
    ratio = 1 + np.arange(replicas) % 4
    cfg = hadfl.make_config(replicas, n_select, net="none", m_none=Head.size(width, hidden, vocab, blocks), steps_per_unit=steps_per_unit, seed=synth.SELECT_SEED)
    stride = hadfl.param_count(cfg)[2]
    gen = torch.Generator(device=dev).manual_seed(seed)
    rows = torch.zeros((replicas, stride), dtype=torch.float32, device=dev)
    head = Head(rows, replicas, batch, width, hidden, vocab, bf16, blocks, drop, seed)
    # one start for all (Algorithm 1)
    head.p["w1"].copy_(torch.randn((width, hidden), generator=gen, device=dev) * (2 / width) ** 0.5)
    head.p["gamma"].fill_(1.0)
    head.p["w2"].copy_(torch.randn((hidden, vocab), generator=gen, device=dev) * hidden ** -0.5)
    for i in range(blocks):
        head.p["u%d" % i].copy_(torch.randn((hidden, 2 * hidden), generator=gen, device=dev) * (2 / hidden) ** 0.5)
        head.p["v%d" % i].copy_(torch.randn((2 * hidden, hidden), generator=gen, device=dev) * (2 * hidden * blocks) ** -0.5)
    embedding = torch.randn((vocab, width), generator=gen, device=dev).to(head.dtype)
    ctx = hadfl.Context(cfg, ratio, replicas=rows.view(-1))
    steps, tokens = hadfl.step_counts(ratio, 1, steps_per_unit), Tokens(replicas, vocab, seed)
    versions = torch.as_tensor(steps, dtype=torch.int32, device=dev)
    history, chosen = [], []
    for cycle in range(cycles):
        total, count = torch.zeros((), device=dev), 0
        for s in range(int(steps.max())):
            last, after = tokens.batch(batch)
            active = steps > s
            after[~active] = -1                                # done for this round: rows without labels
            loss = head.step(embedding[torch.as_tensor(last, device=dev)], torch.as_tensor(after, device=dev))
            head.update(lr)
            total += loss.sum()
            count += int(active.sum())
        ctx.select(cycle, versions=versions)
        ctx.aggregate(True)
        history.append(float(total) / count)
        chosen.append(ctx.selected()[0].tolist())
    ctx.close()
    last, _ = tokens.batch(batch)
    right = torch.as_tensor(tokens.next[last], dtype=torch.int32, device=dev)[..., None].contiguous()
    logp, entropy, top, _ = head.answers(embedding[torch.as_tensor(last, device=dev)], right, top=min(5, vocab))
    found = (top == right).float().sum(-1).mean()
    return dict(losses=history, selected=chosen, rows=rows, log_vocab=float(np.log(vocab)), answers=dict(logp=float(logp.mean()), entropy=float(entropy.mean()),
                                                                                                      in_top_5=float(found)))


def main():
    ap = argparse.ArgumentParser()
    ap.add_argument("--replicas", type=int, default=4)
    ap.add_argument("--select", type=int, default=2)
    ap.add_argument("--vocab", type=int, default=2003)
    ap.add_argument("--width", type=int, default=128)
    ap.add_argument("--hidden", type=int, default=256)
    ap.add_argument("--batch", type=int, default=256)
    ap.add_argument("--cycles", type=int, default=20)
    ap.add_argument("--lr", type=float, default=1.0)
    ap.add_argument("--blocks", type=int, default=0)
    ap.add_argument("--drop", type=float, default=0.0)
    ap.add_argument("--bf16", action="store_true")
    a = ap.parse_args()
    out = run(a.replicas, a.select, a.vocab, a.width, a.hidden, a.batch, a.cycles, lr=a.lr, bf16=int(a.bf16), blocks=a.blocks, drop=a.drop)
    print(json.dumps(dict(config=vars(a), first_loss=out["losses"][0], last_loss=out["losses"][-1], log_vocab=out["log_vocab"], selected=out["selected"], answers=out["answers"])))


if __name__ == "__main__":
    main()
