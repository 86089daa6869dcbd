"""The operators of a language model's head on the GPU where their routes, strides and values end: each kernel that a plan can choose, inputs
whose rows overlap, tensors whose offsets pass 32 bits, logits near the largest float.  References and bounds as in test_gpu_head.py."""
import numpy as np
import pytest

from paper_2111_08274_amd import hadfl
from tests import head_ref as ref
from tests import test_gpu_head as base

pytestmark = pytest.mark.gpu


def _dense(n, rows, i, o, bf16, x, dy, layout="whole"):
    """Checks dw and db for the tensors x, dy"""
    plan, packed = hadfl.DenseGrad(n, rows, i, o, bf16=bf16), hadfl.PackedRows(n, rows, i, bf16=bf16).pack(x)
    dw, db = base._out((n, i, o), 0, layout), base._out((n, o), 0, layout)
    plan.backward(packed, dy, dw=dw.t, db=db.t)
    v, d = ref.checkpoint(x.float().cpu().numpy())[0], base._values(dy)
    base._check(db.get(), d.sum(1), (rows + 16) * ref.EPS32 * np.abs(d).sum(1), "db")
    base._check(dw.get(), np.matmul(v.transpose(0, 2, 1), d), (rows + 16) * ref.EPS32 * np.matmul(np.abs(v).transpose(0, 2, 1), np.abs(d)), "dw")
    assert dw.untouched() and db.untouched()


# rows that do not fill the last 64, in the sizes' different kernels
@pytest.mark.parametrize("n,rows,i,o,bf16", [(1, 1000, 2048, 2048, 1), (4, 1000, 2048, 2048, 1), (1, 8200, 896, 896, 1), (2, 70, 64, 128, 1), (1, 1100, 4104, 3592, 0)])
@pytest.mark.parametrize("stride", [0, 16])
def test_dense_gradient_of_rows_that_overlap(n, rows, i, o, bf16, stride):
    # one row for all rows (the gradient behind a mean over tokens), and rows that begin 16 values after another
    torch = base._torch()
    g = torch.Generator(device="cuda").manual_seed(1)
    x = torch.randn((n, rows, i), device="cuda", generator=g).to(base._dtype(bf16))
    line = torch.randn(rows * stride + n * o + 64, device="cuda", generator=g).to(base._dtype(bf16))
    _dense(n, rows, i, o, bf16, x, line.as_strided((n, rows, o), (o if n > 1 else 0, stride, 1)))
