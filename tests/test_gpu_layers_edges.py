"""The layers' operators on the GPU where sizes and calls end: tensors whose offsets pass 32 bits, more rows than one launch has threads for, two plans at
once on two streams, a graph whose plan also runs eagerly."""
import numpy as np
import pytest

from paper_2111_08274_amd import hadfl
from tests import layer_ref as ref
from tests.test_gpu_head import _check, _dtype, _torch, _values

pytestmark = pytest.mark.gpu
FAR = (1 << 32) + 24


def _far(shape, dtype, g):
    """Replicas more than 2^32 elements apart, rows with a gap"""
    torch = _torch()
    n, rows, cols = shape
    flat = torch.empty((n - 1) * FAR + (rows - 1) * (cols + 8) + cols, dtype=dtype, device="cuda")
    t = flat.as_strided(shape, (FAR, cols + 8, 1))
    t.copy_(torch.randn(shape, device="cuda", generator=g).to(dtype))
    return t


@pytest.mark.parametrize("rows", [20, 300])
@pytest.mark.parametrize("bf16", [0, 1])
def test_offsets_that_pass_32_bits(rows, bf16):
    torch = _torch()
    torch.cuda.empty_cache()
    if torch.cuda.mem_get_info()[0] < 150 << 30:
        pytest.skip("needs 120 GB of device memory")
    g = torch.Generator(device="cuda").manual_seed(1)
    t, n, i, o = _dtype(bf16), 2, 72, 136
    x, w, r = _far((n, rows, i), t, g), _far((n, i, o), t, g), _far((n, rows, o), t, g)
    y, pre = _far((n, rows, o), t, g), _far((n, rows, o), t, g)
    plan, kw = hadfl.DenseLayer(n, rows, i, o, bf16=bf16, activation="gelu", drop=0.1), dict(seed=1, call=2)
    plan.forward(x, w, residual=r, pre=pre, y=y, **kw)
    near = [q.contiguous() for q in (x, w, r)]
    pre2 = torch.empty((n, rows, o), dtype=t, device="cuda")
    assert torch.equal(plan.forward(*near[:2], residual=near[2], pre=pre2, **kw), y) and torch.equal(pre, pre2)
    want = plan.backward(near[2], *near[:2], pre=pre2, **kw)
    dx, dw = _far((n, rows, i), t, g), _far((n, i, o), t, g)
    got = plan.backward(r, x, w, pre=pre, dx=dx, dw=dw, **kw)
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    drop = hadfl.Dropout(n, rows, o, 0.3, bf16=bf16)
    assert torch.equal(drop.forward(r, residual=y, y=pre, **kw), drop.forward(near[2], residual=y.contiguous(), **kw))
    scores, tokens = hadfl.TokenScores(n, rows, o, n_tokens=2, n_top=3, bf16=bf16), torch.randint(0, o, (n, rows, 2), device="cuda", dtype=torch.int32)
    assert all(torch.equal(a, b) for a, b in zip(scores.forward(r, tokens), scores.forward(near[2], tokens)))
    d = torch.randn((n, rows, 2), device="cuda")
    assert torch.equal(scores.backward(r, tokens, d, dlogits=pre), scores.backward(near[2], tokens, d))


def test_more_rows_than_one_launch_has_threads_for():
    # 2^20 rows of 2^15 values: 2^32 chunks of eight, a thread each
    torch = _torch()
    torch.cuda.empty_cache()
    if torch.cuda.mem_get_info()[0] < 90 << 30:
        pytest.skip("needs 69 GB of device memory")
    rows, cols = 1 << 20, 1 << 15
    x = torch.ones((1, 1, cols), device="cuda", dtype=torch.bfloat16)
    y = hadfl.Dropout(1, rows, cols, 0.5, bf16=1).forward(x.expand(1, rows, cols), seed=3, call=4)
    for t in (0, 1, 1 << 19, rows - 1):
        words = ref.philox((np.full(cols // 8, t), np.arange(cols // 8), np.full(cols // 8, 4), np.zeros(cols // 8, int)), (3, 0))
        u = np.stack([(w >> np.uint64(s)) & np.uint64(0xffff) for w in words for s in (0, 16)], -1).reshape(-1)
        assert np.array_equal(_values(y[0, t]), np.where(u >= 32768, 2.0, 0.0))
    del y
    torch.cuda.empty_cache()


def test_rows_beyond_65535_blocks_in_the_scores():
    # 2^24 rows of 40 logits, two kinds of them; entropies and alternatives of the first and the last
    torch = _torch()
    n, rows, v = 16, 1 << 20, 40
    z = torch.randn((n, 1, v), device="cuda", generator=torch.Generator(device="cuda").manual_seed(0)).bfloat16()
    plan = hadfl.TokenScores(n, rows, v, n_tokens=0, n_top=2, bf16=1)
    _, entropy, top, top_logp = plan.forward(z.expand(n, rows, v))
    r = [ref.scores(_values(z[k]), np.zeros((1, 1), int), 2) for k in range(n)]
    for k in range(n):
        _check(_values(entropy[k, -1:]), r[k]["entropy"], ref.scores_bounds(r[k])["entropy"], "entropy")
        assert top[k, -1].tolist() == r[k]["top"][0].tolist()
    assert bool((entropy == entropy[:, :1]).all()) and bool((top == top[:, :1]).all()) and bool((top_logp == top_logp[:, :1]).all())


def test_two_plans_at_once_on_two_streams():
    torch = _torch()
    g = torch.Generator(device="cuda").manual_seed(5)
    n, rows, i, o = 2, 700, 520, 264
    runs = []
    for bf16 in (0, 1):
        x, w, dy = (torch.randn(s, device="cuda", generator=g).to(_dtype(bf16)) for s in ((n, rows, i), (n, i, o), (n, rows, o)))
        plans = [hadfl.DenseLayer(n, rows, i, o, bf16=bf16, activation="silu", drop=0.1) for _ in range(2)]
        scores = [hadfl.TokenScores(n, rows, o, n_tokens=0, n_top=4, bf16=bf16) for _ in range(2)]

        def step(k, x=x, w=w, dy=dy, plans=plans, scores=scores):
            pre = torch.empty_like(dy)
            y = plans[k].forward(x, w, pre=pre, seed=1)
            return (y,) + plans[k].backward(dy, x, w, pre=pre, seed=1) + scores[k].forward(y)[1:]
        runs.append((step, step(0)))
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    for step, want in runs:
        got = [[], []]
        for _ in range(10):
            for k in range(2):
                with torch.cuda.stream(streams[k]):
                    got[k].append(step(k))
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for side in got for out in side for a, b in zip(out, want))


def test_two_graphs_of_one_plan_and_eager_calls_between():
    # a plan's working memory serves both, one after the other on one stream
    torch = _torch()
    n, rows, i, o = 2, 300, 96, 520
    for bf16 in (0, 1):
        g = torch.Generator(device="cuda").manual_seed(6)
        x, w, dy = (torch.randn(s, device="cuda", generator=g).to(_dtype(bf16)) for s in ((n, rows, i), (n, i, o), (n, rows, o)))
        plan, counter = hadfl.DenseLayer(n, rows, i, o, bf16=bf16, activation="relu", drop=0.2), torch.zeros(1, dtype=torch.int64, device="cuda")
        pre = torch.empty_like(dy)

        def forward():
            return plan.forward(x, w, pre=pre, seed=2, counter=counter)

        def backward():
            return plan.backward(dy, x, w, pre=pre, seed=2, counter=counter)

        forward(), backward()
        torch.cuda.synchronize()
        graphs, outs = [torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()], []
        for graph, call in zip(graphs, (forward, backward)):
            with torch.cuda.graph(graph):
                outs.append(call())
        for step in range(4):
            counter.fill_(step * 7)
            x.copy_(torch.randn(x.shape, device="cuda", generator=g))
            for graph in graphs:
                graph.replay()
            torch.cuda.synchronize()
            got = [outs[0].clone()] + [q.clone() for q in outs[1]]
            assert torch.equal(got[0], forward()) and all(torch.equal(a, b) for a, b in zip(got[1:], backward()))
