"""The next-token example with blocks and dropout: one step's gradients against their formulas in 64 bits, its answers, and rounds of it."""
import json
import subprocess
import sys

import numpy as np
import pytest

from paper_2111_08274_amd import next_token
from tests import head_ref, layer_ref

pytestmark = pytest.mark.gpu


def _head(n, batch, width, hidden, vocab, **k):
    import torch
    g = torch.Generator(device="cuda").manual_seed(3)
    rows = torch.randn((n, next_token.Head.size(width, hidden, vocab, k.get("blocks", 0)) + 7), generator=g, device="cuda") * 0.2
    x = torch.randn((n, batch, width), generator=g, device="cuda")
    y = torch.randint(0, vocab, (n, batch), generator=g, device="cuda", dtype=torch.int32)
    return next_token.Head(rows, n, batch, width, hidden, vocab, **k), x, y


def test_one_step_with_blocks_against_64_bits():
    # as for the head alone: with the checkpoints' values taken from the device what is left are 32-bit sums, 1e-4 of a tensor's largest gradient is far
    # above them
    n, batch, width, hidden, vocab, blocks, drop, seed = 2, 50, 24, 32, 101, 2, 0.25, 11
    head, x, y = _head(n, batch, width, hidden, vocab, blocks=blocks, drop=drop, seed=seed)
    y[1, ::3] = -1
    loss = head.step(x, y).double().cpu().numpy()
    p = {k: v.double().cpu().numpy() for k, v in head.p.items()}
    got = {k: v.double().cpu().numpy() for k, v in head.g.items()}
    value = lambda t: t.double().cpu().numpy()  # noqa: E731
    xd = layer_ref.dropped(value(x), drop, seed, 0)
    kept_x, kept_h = head_ref.checkpoint(value(head.kept_x.unpack()))[0], value(head.kept_h.unpack())
    kept = [(value(a.unpack()), value(b.unpack())) for a, b, _ in head.kept]
    masks = [layer_ref.kept(n, batch, hidden, drop, seed, (1 + i) << 32) for i in range(blocks)]
    assert np.abs(kept_x - xd).max() <= np.abs(xd).max() * 2.0 ** -7 and int(head.steps) == 1
    for k in range(n):
        h = np.maximum(xd[k] @ p["w1"][k] + p["b1"][k], 0)
        on, pres = h > 0, []
        for i in range(blocks):
            pre = h @ p["u%d" % i][k] + p["a%d" % i][k]
            z = layer_ref.activate(pre, "gelu") @ p["v%d" % i][k] + p["c%d" % i][k]
            h = h + np.where(masks[i][0][k], z * masks[i][1], 0)
            pres.append(pre)
        out, mean, rstd = head_ref.layer_norm(h, p["gamma"][k], p["beta"][k], 1e-5)
        r = head_ref.class_loss(out, p["w2"][k], p["b2"][k], y[k].cpu().numpy().astype(np.int64))
        assert abs(loss[k] - r["loss"]) <= 1e-5 * max(1, abs(r["loss"]))
        dh, dgamma, dbeta = head_ref.layer_norm_grad(r["dx"], kept_h[k], p["gamma"][k], mean, rstd)
        want = dict(gamma=dgamma, beta=dbeta, w2=r["dw"], b2=r["db"])
        for i in reversed(range(blocks)):
            dz = np.where(masks[i][0][k], dh * masks[i][1], 0)
            want["v%d" % i], want["c%d" % i] = kept[i][1][k].T @ dz, dz.sum(0)
            du = dz @ p["v%d" % i][k].T * layer_ref.slope(pres[i], "gelu")
            want["u%d" % i], want["a%d" % i] = kept[i][0][k].T @ du, du.sum(0)
            dh = dh + du @ p["u%d" % i][k].T
        du = dh * on
        want["w1"], want["b1"] = kept_x[k].T @ du, du.sum(0)
        assert set(want) == set(got)
        for name, w in want.items():
            assert np.abs(got[name][k] - w).max() <= 1e-4 * np.abs(w).max(), (k, name)


def test_the_model_answers_with_what_its_logits_say():
    import torch
    n, batch, width, hidden, vocab = 2, 30, 24, 32, 401
    head, x, y = _head(n, batch, width, hidden, vocab, blocks=1, drop=0.5)
    logp, entropy, top, top_logp = head.answers(x, y[..., None].contiguous(), top=3)
    h = torch.relu(x.double() @ head.p["w1"].double() + head.p["b1"].double()[:, None])
    z = h @ head.p["u0"].double() + head.p["a0"].double()[:, None]
    a = 0.5 * z * (1 + torch.tanh(layer_ref.GELU[0] * (z + layer_ref.GELU[1] * z ** 3)))
    h = h + a @ head.p["v0"].double() + head.p["c0"].double()[:, None]
    h = (h - h.mean(-1, keepdim=True)) / torch.sqrt(h.var(-1, unbiased=False, keepdim=True) + 1e-5) * head.p["gamma"].double()[:, None] + head.p["beta"].double()[:, None]
    lp = torch.log_softmax(h @ head.p["w2"].double() + head.p["b2"].double()[:, None], -1)
    assert (logp[..., 0] - lp.gather(2, y[..., None].long())[..., 0]).abs().max() < 1e-4
    assert (entropy + (lp.exp() * lp).sum(-1)).abs().max() < 1e-4
    best = lp.topk(3, -1)
    assert (top_logp - best.values).abs().max() < 1e-4 and (lp.gather(2, top.long()) - best.values).abs().max() < 1e-4
    # without dropout in the way the loss of a step says the same
    plain, _, _ = _head(n, batch, width, hidden, vocab, blocks=1)
    loss = plain.step(x, y)
    assert (loss + logp[..., 0].mean(1)).abs().max() < 1e-4


@pytest.mark.parametrize("bf16", [0, 1])
def test_rounds_with_blocks_and_dropout_run_and_stay_in_step(bf16):
    import torch
    kw = dict(replicas=3, n_select=2, vocab=200, width=32, hidden=64, batch=64, bf16=bf16, blocks=2, drop=0.1, lr=0.1)
    out = next_token.run(cycles=3, **kw)
    assert all(np.isfinite(out["losses"])) and bool(torch.isfinite(out["rows"]).all())
    assert all(torch.equal(out["rows"][0], out["rows"][k]) for k in (1, 2))
    assert -20 < out["answers"]["logp"] < 0 <= out["answers"]["entropy"] <= out["log_vocab"] + 1e-3 and 0 <= out["answers"]["in_top_5"] <= 1
    again = next_token.run(cycles=3, **kw)
    assert again["selected"] == out["selected"] and torch.equal(again["rows"], out["rows"])          # the same values dropped


def test_the_command_takes_blocks_and_dropout():
    r = subprocess.run([sys.executable, "-m", "paper_2111_08274_amd.next_token", "--vocab", "100", "--width", "16", "--hidden", "32", "--batch", "32", "--cycles", "1",
                        "--blocks", "1", "--drop", "0.1"], capture_output=True, text=True, timeout=100)
    assert r.returncode == 0, r.stderr[-2000:]
    assert set(json.loads(r.stdout)["answers"]) == {"logp", "entropy", "in_top_5"}
