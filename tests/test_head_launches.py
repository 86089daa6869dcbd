"""What the head's operators ask the GPU to launch, checked without one: the library's real launch path on a stand-in for the HIP runtime
(tests/native/head_launches.cpp)."""
import json
import os
import re
import subprocess
import sys

import pytest

HERE = os.path.dirname(os.path.abspath(__file__))


@pytest.fixture(scope="session")
def launched(tmp_path_factory):
    so = str(tmp_path_factory.mktemp("hip") / "head_launches.so")
    subprocess.run(["/opt/rocm/llvm/bin/clang++", "-std=c++17", "-O1", "-shared", "-fPIC", "-D__HIP_PLATFORM_AMD__", "-I/opt/rocm/include",
                    os.path.join(HERE, "native", "head_launches.cpp"), "-o", so], check=True)

    def run(cases):
        r = subprocess.run([sys.executable, os.path.join(HERE, "native", "run_head.py"), so], input=json.dumps(cases), text=True,
                           capture_output=True, cwd=os.path.dirname(HERE), env=dict(os.environ, PYTHONPATH=os.path.dirname(HERE)))
        assert r.returncode == 0, r.stderr[-3000:]
        return json.loads(r.stdout)
    return run


def _name(launch):
    return re.search(r"\d+([a-z_]+_kernel)", launch[0]).group(1)


def _planes(launch):
    """(row stride, rows, columns) of both operands of a product of planes"""
    v = [int(q) for q in launch[7:13]]
    return v[:3], v[3:]


DENSE = [(1, 1000, 2048, 2048, 1), (4, 1000, 2048, 2048, 1), (1, 8200, 896, 896, 1), (1, 1100, 4104, 3592, 0)]


def test_rows_that_overlap_are_laid_out_for_products_of_planes_in_the_dense_gradient(launched):
    # a plane's rows end where the next begins: what lies beyond the last is told by its offset
    cases = [dict(op="dense", n=n, rows=t, inputs=i, outputs=o, bf16=b, dy=dy) for n, t, i, o, b in DENSE
             for dy in (None, [0, 0], [o, 0], [t * o, 0], [t * o, 16], [t * o, o - 8], [t * (o + 8), o + 8])]
    for c, r in zip(cases, launched(cases)):
        direct = [v for v in r["launches"] if _name(v) == "direct_kernel"]
        assert r["status"] == 0 and direct, c
        assert all(ld >= cols for v in direct for ld, _, cols in _planes(v)), c
        whole = not c["dy"] or c["dy"][1] >= c["outputs"]
        assert ("lay_out_kernel" in map(_name, r["launches"])) == (not c["bf16"] or not whole), c


@pytest.mark.parametrize("grad", [0, 1])
def test_rows_that_overlap_are_laid_out_for_products_of_planes_in_the_loss(launched, grad):
    cases = [dict(op="loss", n=n, rows=t, features=d, classes=v, bf16=b, grad=grad, w=w) for n, t, d, v, b in [(1, 400, 200, 2056, 1), (2, 1000, 776, 4200, 1), (1, 400, 200, 2056, 0)]
             for w in (None, [0, 0], [v, 0], [d * v, 0], [d * v, 16], [d * v, v - 8], [d * (v + 8), v + 8])]
    for c, r in zip(cases, launched(cases)):
        direct = [v for v in r["launches"] if _name(v) == "direct_kernel"]
        assert r["status"] == 0 and direct, c
        assert all(ld >= cols for v in direct for ld, _, cols in _planes(v)), c
        whole = not c["w"] or c["w"][1] >= c["classes"]
        assert [_name(v) for v in r["launches"]].count("lay_out_kernel") == (1 if c["bf16"] and whole else 2), c      # x always, W where it has to be


def test_no_operand_through_registers_has_fewer_columns_than_a_load_takes(launched):
    # pieces of a vocabulary whose last one would hold one to eight classes; sizes of fewer than eight columns, which are laid out
    cases = [dict(op="loss", n=1024, rows=t, features=16, classes=v, bf16=b) for b in (0, 1) for t in (30, 130) for v in list(range(7165, 7181)) + [8193, 20487, 61441, 65537, 131073]]
    cases += [dict(op="loss", n=64, rows=40, features=64, classes=v) for v in range(58881, 58890)]
    cases += [dict(op="loss", n=2, rows=5, features=f, classes=v, bf16=b) for f in (1, 7, 8, 9) for v in (1, 7, 8, 9) for b in (0, 1)]
    cases += [dict(op="dense", n=2, rows=5, inputs=f, outputs=v, bf16=b) for f in (1, 7, 8, 9) for v in (1, 7, 8, 9) for b in (0, 1)]
    pieces = set()
    for c, r in zip(cases, launched(cases)):
        assert r["status"] == 0, c
        through = [v for v in r["launches"] if _name(v) == "product_kernel"]
        assert all(int(q) >= 8 for v in through for q in v[7:]), (c, through)
        pieces.add(sum("Gradient" in v[0] for v in through))
    assert len(pieces) > 3


def test_no_launch_has_more_threads_than_a_dimension_holds(launched):
    # sizes within the header's limits whose workgroups, in one line, would be 2^32 threads or more
    cases = [dict(op="pack", n=16, rows=1 << 20, features=4128, bf16=1), dict(op="pack", n=16, rows=1 << 20, features=1 << 17), dict(op="unpack", n=16, rows=1 << 20, features=1 << 17, bf16=1),
             dict(op="loss", n=1024, rows=4096, features=8, classes=1 << 17, bf16=1, grad=0), dict(op="loss", n=16, rows=1 << 20, features=1 << 12, classes=1 << 17, bf16=1),
             dict(op="loss", n=16, rows=1 << 20, features=1 << 12, classes=1 << 17), dict(op="loss", n=1024, rows=64, features=1 << 17, classes=1 << 20),
             dict(op="loss", n=1024, rows=8, features=1 << 17, classes=1 << 18, bf16=1), dict(op="dense", n=1024, rows=64, inputs=1 << 16, outputs=1 << 16),
             dict(op="dense", n=1024, rows=1 << 14, inputs=1 << 13, outputs=1 << 16, bf16=1), dict(op="norm", n=16, rows=1 << 20, features=1 << 17),
             dict(op="norm", n=1024, rows=1 << 14, features=512)]
    folded = 0
    for c, r in zip(cases, launched(cases)):
        assert r["status"] == 0, (c, r["text"])
        for v in r["launches"]:
            size = [int(q) for q in v[1:7]]
            assert all(size[i] * size[i + 1] < 1 << 32 for i in (0, 2, 4)), (c, v)
            folded += size[2] > 1 and _name(v) in ("pack_rows_kernel", "unpack_rows_kernel", "direct_kernel", "product_kernel", "few_weights_kernel", "lay_out_kernel", "join_shares_kernel")
    assert folded > 8


def _shapes(launched):
    """The sizes of the GPU tests, in the layouts that change a route: as they lie, and with odd strides."""
    from tests import test_gpu_head as head
    from tests import test_gpu_head_edges as edges
    cases = []
    for n, t, i, o, b in [s + (b,) for s in head.DENSE for b in (0, 1)] + edges.DENSE:
        cases += [dict(op="dense", n=n, rows=t, inputs=i, outputs=o, bf16=b, dy=dy) for dy in (None, [t * (o + 3) + 7, o + 3])]
    for n, t, d, v, b in [s + (b,) for s in head.LOSS for b in (0, 1)] + edges.LOSS:
        cases += [dict(op="loss", n=n, rows=t, features=d, classes=v, bf16=b, bias=1, grad=g, w=w) for w in (None, [d * (v + 3) + 7, v + 3]) for g in (0, 1)]
    cases += [dict(op="loss", n=n, rows=t, features=d, classes=v, bf16=b, bias=1) for n, t, d, v, b in edges.PIECES]
    pieces = next(m for m in head.test_a_vocabulary_in_pieces.pytestmark if m.name == "parametrize").args[1]
    cases += [dict(op="loss", n=64, rows=t, features=d, classes=v, bf16=b, bias=1) for b, t, d, v in pieces]
    cases += [dict(op="norm", n=n, rows=t, features=f, bf16=b) for n, t, f in head.NORM for b in (0, 1)]
    cases += [dict(op=op, n=2, rows=5, features=40, bf16=b) for op in ("pack", "unpack") for b in (0, 1)]
    return cases


def test_the_gpu_tests_reach_every_kernel_of_the_head(launched):
    cases = _shapes(launched)
    got = launched([dict(op="kernels")] + cases)
    kernels, reached = {k for k in got[0] if "hadfl4head" in k}, set()
    for c, r in zip(cases, got[1:]):
        assert r["status"] == 0, (c, r["text"])
        reached |= {v[0] for v in r["launches"]}
    assert len(kernels) > 100 and reached <= kernels
    assert not kernels - reached, "\n".join(sorted(kernels - reached))


def test_the_gpu_tests_reach_planes_that_lie_in_the_callers_tensors(launched):
    cases = _shapes(launched)
    tiles = set()
    for c, r in zip(cases, launched(cases)):
        if c["op"] in ("dense", "loss") and c["bf16"]:
            laid = [_name(v) for v in r["launches"]].count("lay_out_kernel")
            for v in r["launches"]:
                if _name(v) == "direct_kernel" and laid < (1 if c["op"] == "dense" else 2):
                    tiles.add((c["op"],) + tuple(re.search(r"ELi(\d+)ELi(\d+)ELi\dELi\dEN", v[0]).groups()))
    assert {("dense", "128", "128"), ("dense", "256", "256"), ("loss", "128", "128"), ("loss", "256", "256")} <= tiles, tiles
