"""The operators of a language model's head together, as they are used: one step of the next-token head against its formula in
64 bits, and rounds of it under the library's selection and aggregation."""
import numpy as np
import pytest

from paper_2111_08274_amd import next_token
from tests import head_ref as ref

pytestmark = pytest.mark.gpu


def test_one_step_of_the_head_against_64_bits():
    # x and h are kept in 8 bits for the backward pass, as the step does; with the reference's own h rounding its checkpoint to the
    # same multiples, what is left are 32-bit sums: 1e-4 of the largest gradient of a tensor is far above them and far below
    # what a wrong operand or a missing checkpoint (a step is 2^-7 of a group's largest) would show.  Values of h next to a rounding
    # boundary of the checkpoint may fall on either side: they are taken from the device
    import torch
    n, batch, width, hidden, vocab = 3, 70, 48, 96, 203
    g = torch.Generator(device="cuda").manual_seed(3)
    rows = torch.randn((n, next_token.Head.size(width, hidden, vocab) + 7), generator=g, device="cuda") * 0.2
    head = next_token.Head(rows, n, batch, width, hidden, vocab)
    x = torch.randn((n, batch, width), generator=g, device="cuda")
    y = torch.randint(0, vocab, (n, batch), generator=g, device="cuda", dtype=torch.int32)
    y[1] = -1                                                 # a replica that sits the step out
    y[2, ::3] = -1
    loss = head.step(x, y).double().cpu().numpy()
    kept_h = head.kept_h.unpack().double().cpu().numpy()
    p = {k: v.double().cpu().numpy() for k, v in head.p.items()}
    grads = {k: v.double().cpu().numpy() for k, v in head.g.items()}
    for k in range(n):
        xk, yk = x[k].double().cpu().numpy(), y[k].cpu().numpy().astype(np.int64)
        u = xk @ p["w1"][k] + p["b1"][k]
        h = np.maximum(u, 0)
        out, mean, rstd = ref.layer_norm(h, p["gamma"][k], p["beta"][k], 1e-5)
        r = ref.class_loss(out, p["w2"][k], p["b2"][k], yk)
        dh, dgamma, dbeta = ref.layer_norm_grad(r["dx"], kept_h[k], p["gamma"][k], mean, rstd)
        du = dh * (u > 0)
        want = dict(w1=ref.checkpoint(x[k].cpu().numpy())[0].T @ du, b1=du.sum(0), gamma=dgamma, beta=dbeta, w2=r["dw"], b2=r["db"])
        assert abs(loss[k] - r["loss"]) <= 1e-5 * max(1, abs(r["loss"]))
        assert np.abs(kept_h[k] - h).max() <= h.max() * 2.0 ** -7
        for name, w in want.items():
            top = np.abs(w).max()
            assert np.abs(grads[name][k] - w).max() <= 1e-4 * top, (k, name)
            assert (top == 0) == (k == 1)
    before = rows.clone()
    head.update(0.5)
    assert torch.equal(rows[1], before[1]) and torch.equal(rows[:, -7:], before[:, -7:])


@pytest.mark.parametrize("bf16", [0, 1])
def test_rounds_of_the_head_learn_and_stay_in_step(bf16):
    import torch
    out = next_token.run(replicas=4, n_select=2, vocab=512, width=64, hidden=128, batch=128, cycles=12, bf16=bf16)
    assert out["losses"][0] > 0.8 * out["log_vocab"] and out["losses"][-1] < 0.6 * out["losses"][0]
    assert all(len(set(s)) == 2 and 0 <= min(s) and max(s) < 4 for s in out["selected"])
    assert all(torch.equal(out["rows"][0], out["rows"][k]) for k in range(1, 4))          # the global synchronisation
    again = next_token.run(replicas=4, n_select=2, vocab=512, width=64, hidden=128, batch=128, cycles=2, bf16=bf16)
    assert again["selected"] == out["selected"][:2]
