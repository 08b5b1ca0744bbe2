"""The operators of a training pass at the largest sizes that their argument checks admit, against a runtime that launches nothing (and
refuses launches of 2^32 threads and more along a dimension, as HIP does), and their workspaces there."""
import ctypes

import pytest

import host_hip
from paper_2309_06497_amd import binding as B


@pytest.fixture(scope="module")
def lib(tmp_path_factory):
    return host_hip.build(str(tmp_path_factory.mktemp("hip")))


ROWS = r"""
P = ctypes.c_void_p(1 << 40)
S = ctypes.c_void_p(STREAM)
for rows, cols in ((1, 1), (1 << 26, 64), ((1 << 24) + 1, 1500), (1 << 24, 4096), ((1 << 23) + 3, 16384), ((1 << 31) - 1, 1), ((1 << 31) - 1, 16384)):
    k = B.ResidualNorm(rows, cols, 1, 1, 1, 0, 1e-5, 1.0, 1 << 40, None, None, 1 << 40, None)
    reset()
    rc = L.shampoo_residual_norm_forward(ctypes.byref(k), P, cols, P, cols, P, cols, P, cols, None, None, 0, S)
    each = 4 if cols <= 2048 else 1                # rows of a workgroup
    print(rows, cols, rc, sum(e.a for e in launches("residual_norm_forward")) * each)
"""


def test_residual_norm_forward_of_as_many_rows_as_it_admits(lib):
    seen = [list(map(int, line.split())) for line in host_hip.run(lib, ROWS) if line]
    assert len(seen) == 7
    for rows, cols, rc, covered in seen:
        assert rc == 0, (rows, cols, rc)
        assert rows <= covered < rows + 4, (rows, cols, covered)


BIAS = r"""
P = ctypes.c_void_p(1 << 40)
S = ctypes.c_void_p(STREAM)
for rows, n, out, act, dtype in ((16384, 8, 1 << 22, 0, 1), (16384, 40, (1 << 22) - 3, 3, 0), (1 << 20, 8, 1 << 22, 0, 1), (1 << 20, 8, 1 << 20, 0, 1), (16384, 8, 3000000, 2, 1),
                                  ((1 << 31) - 1, 1, 1, 0, 1), (8192, 8192, 2048, 0, 1)):
    b = L.shampoo_checkpoint_bytes(rows, n)
    ws = L.shampoo_checkpoint_weight_grad_workspace_bytes(rows, n, out, act, dtype, out, dtype, 1)
    reset()
    rc = L.shampoo_checkpoint_weight_grad(P, b, rows, n, act, P, dtype, out, out, P, dtype, 0, n, P, P, ws, S)
    print(rows, out, rc)
"""


def test_bias_gradients_of_as_many_outputs_as_it_admits(lib):
    seen = [list(map(int, line.split())) for line in host_hip.run(lib, BIAS) if line]
    assert len(seen) == 7 and all(rc == 0 for _, _, rc in seen), seen


def test_cross_entropy_workspace_does_not_grow_with_the_rows_of_a_bias_gradient():
    """A piece of the rows takes the same memory whatever their number: logits, and partial sums of the bias's gradient.  From the first size on
    which is one piece of its own (2^14 rows of 131072 classes)."""
    L = B.lib()
    for dtype, grad in ((1, 1), (1, 0), (0, 0)):
        for bias in (0, 1):
            need = []
            for rows in (1 << 16, 1 << 20, (1 << 31) - 1):
                c = B.CrossEntropy(rows, 2048, 131072, dtype, grad, 0, bias, 1, 2048, 2048, 2048, 2048)
                need.append(L.shampoo_linear_cross_entropy_workspace_bytes(ctypes.byref(c)))
                if dtype == 0:         # planes of all of x
                    need[-1] -= 3 * rows * 2048 * 2
            assert 0 < min(need) and max(need) - min(need) < 64 << 20, (dtype, grad, bias, need)
            assert max(need) < 10 << 30
