"""Which kernel the rows of logits go to, without a GPU: the batches that the GPU tests compare with the definition have every form of it among them."""
import re

import pytest

import host_hip
import test_gpu_log_probs_rows as rows


@pytest.fixture(scope="module")
def lib(tmp_path_factory):
    return host_hip.build(str(tmp_path_factory.mktemp("hip")))


FORMS = r"""
P, S = ctypes.c_void_p(1 << 40), ctypes.c_void_p(STREAM)
for n, v in BATCHES:
    for dtype in (0, 1):
        for top in (0, 20):
            c = B.Logits(n, v, 3, top, dtype, 1.0, v)
            size = L.shampoo_log_probs_workspace_bytes(ctypes.byref(c))
            reset()
            assert L.shampoo_log_probs(ctypes.byref(c), P, P, P, P, P, P, P, P, size, S) == 0
            print(n, v, dtype, top, *[e.name.decode() for e in launches()])
"""


def test_the_batches_of_the_gpu_tests_reach_every_form(lib):
    seen = {}
    for line in host_hip.run(lib, "BATCHES = %r\n" % (rows.BATCHES,) + FORMS):
        if not line:
            continue
        n, v, dtype, top, first, *join = line.split()
        form = re.search(r"log_probs_kernelI([ft])Li(\d)ELb([01])E", first)
        assert form and (form[1] == "f") == (dtype == "0") and (form[3] == "1") == (top != "0"), line
        assert all("log_probs_join_kernel" in k for k in join) and len(join) <= 1, line
        seen[int(n), int(v), dtype, top] = int(form[2]), len(join)
    for dtype in "01":
        for top in ("0", "20"):
            assert [seen[n, v, dtype, top] for n, v in rows.BATCHES] == [(1, 0), (1, 0), (2, 0), (2, 0), (4, 0), (8, 0), (8, 1), (8, 1), (4, 1)]
