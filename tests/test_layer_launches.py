"""What the layers' operators ask the GPU to launch, checked without one (tests/native/head_launches.cpp stands in for the HIP runtime)."""
import json
import os
import re
import subprocess
import sys

import pytest

HERE = os.path.dirname(os.path.abspath(__file__))


@pytest.fixture(scope="session")
def launched(tmp_path_factory):
    so = str(tmp_path_factory.mktemp("hip") / "layer_launches.so")
    subprocess.run(["/opt/rocm/llvm/bin/clang++", "-std=c++17", "-O1", "-shared", "-fPIC", "-D__HIP_PLATFORM_AMD__", "-I/opt/rocm/include",
                    os.path.join(HERE, "native", "head_launches.cpp"), "-o", so], check=True)

    def run(cases):
        r = subprocess.run([sys.executable, os.path.join(HERE, "native", "run_layers.py"), so], input=json.dumps(cases), text=True,
                           capture_output=True, cwd=os.path.dirname(HERE), env=dict(os.environ, PYTHONPATH=os.path.dirname(HERE)))
        assert r.returncode == 0, r.stderr[-3000:]
        return json.loads(r.stdout)
    return run


def _name(launch):
    return re.search(r"\d+([a-z_]+_kernel)", launch[0]).group(1)


def _both(**c):
    return [dict(c, op="layer"), dict(c, op="layer", grad=1), dict(c, op="layer", grad=1, act=2, drop=0.1), dict(c, op="layer", grad=1, packed=1)]


def test_no_operand_through_registers_has_fewer_columns_than_a_load_takes(launched):
    cases = [q for t in (1, 5, 40, 64, 65, 100) for i in (1, 7, 8, 9, 40) for o in (1, 7, 8, 9, 40) for b in (0, 1) for q in _both(n=2, rows=t, inputs=i, outputs=o, bf16=b)]
    through = 0
    for c, r in zip(cases, launched(cases)):
        assert r["status"] == 0, (c, r["text"])
        for v in r["launches"]:
            if _name(v) == "layer_product_kernel":
                assert len(v) == 9 and all(int(q) >= 8 for q in v[7:]), (c, v)
                through += 1
    assert through > 100


def test_rows_that_overlap_are_laid_out_for_products_of_planes(launched):
    # a plane's rows end where the next begins: what lies beyond the last is told by its offset
    cases = [q for t, i, o in ((200, 200, 264), (1000, 2048, 1024), (130, 72, 72)) for b in (0, 1) for name, cols in (("x", i), ("w", o), ("y", o))
             for s in ([0, 0], [cols, 0], [1 << 24, 16], [1 << 24, cols - 8], [1 << 24, cols + 8], [1 << 30, 1 << 23])
             for q in _both(n=2, rows=t, inputs=i, outputs=o, bf16=b, **{name: s})]
    seen = 0
    for c, r in zip(cases, launched(cases)):
        assert r["status"] == 0, (c, r["text"])
        for v in r["launches"]:
            if _name(v) == "layer_planes_kernel":
                q = [int(x) for x in v[7:13]]
                assert q[0] >= q[2] and q[3] >= q[5] and max(q[0], q[3]) <= 1 << 22, (c, v)
                seen += 1
    assert seen > 100


def test_no_launch_has_more_threads_than_a_dimension_holds(launched):
    big = dict(n=16, rows=1 << 20)
    cases = [dict(op="drop", features=4128, bf16=1, **big), dict(op="drop", features=1 << 17, **big)]
    cases += [dict(op="scores", classes=1 << 20, bf16=b, top=32, grad=g, **big) for b in (0, 1) for g in (0, 1)]
    cases += [dict(op="scores", classes=40, bf16=b, top=32, grad=g, n=1024, rows=1 << 14) for b in (0, 1) for g in (0, 1)]
    cases += [q for b in (0, 1) for q in _both(inputs=1 << 10, outputs=1 << 12, bf16=b, **big) + _both(n=1024, rows=64, inputs=1 << 13, outputs=1 << 15, bf16=b)
              + _both(n=1024, rows=1 << 14, inputs=1 << 13, outputs=520, bf16=b) + _both(n=1024, rows=8, inputs=1 << 14, outputs=1 << 16, bf16=b)]
    for c, r in zip(cases, launched(cases)):
        assert r["status"] == 0, (c, r["text"])
        for v in r["launches"]:
            size = [int(q) for q in v[1:7]]
            assert all(size[i] * size[i + 1] < 1 << 32 for i in (0, 2, 4)) and size[2] < 1 << 16 and size[4] < 1 << 16, (c, v)


def test_the_gpu_tests_reach_every_kernel_of_the_layers(launched):
    from tests import test_gpu_layers as gpu
    odd = lambda t, i, o: dict(x=[t * (i + 3) + 7, i + 3], w=[i * (o + 3) + 7, o + 3], y=[t * (o + 3) + 7, o + 3])  # noqa: E731
    cases = [q for n, t, i, o in gpu.LAYER for b in (0, 1) for s in ({}, odd(t, i, o)) for q in _both(n=n, rows=t, inputs=i, outputs=o, bf16=b, **s)]
    cases += [q for n, t, i, o, b in gpu.ROUTES + gpu.LARGE for q in _both(n=n, rows=t, inputs=i, outputs=o, bf16=b)[:3]]
    cases += [dict(op="layer", grad=1, want=["db"], act=1, n=2, rows=5, inputs=40, outputs=40, bf16=b) for b in (0, 1)]
    cases += [dict(op="scores", n=n, rows=t, classes=v, bf16=b, tokens=3, top=min(v, 5), grad=g) for n, t, v in gpu.SCORES + [(2, 1100, 20011), (2, 1100, 33001), (2, 1100, 60000)]
              for b in (0, 1) for g in (0, 1)]
    cases += [dict(op="drop", n=2, rows=5, features=40, bf16=b) for b in (0, 1)]
    got = launched([dict(op="kernels")] + cases)
    kernels, reached = {k for k in got[0] if "hadfl5layer" in k}, set()
    for c, r in zip(cases, got[1:]):
        assert r["status"] == 0, (c, r["text"])
        reached |= {v[0] for v in r["launches"] if "hadfl5layer" in v[0]}
    assert len(kernels) > 30 and reached <= kernels
    assert not kernels - reached, "\n".join(sorted(kernels - reached))
