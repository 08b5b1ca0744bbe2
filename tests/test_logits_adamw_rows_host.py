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


RETRY = r"""
P, S, n = ctypes.c_void_p(1 << 40), ctypes.c_void_p(STREAM), 600
cfg = B.AdamWConfig(n, (i64 * n)(*[7] * n), None, 8, 0, 1, 0, 0.9, 0.999, 1e-8, 0.01)
h = ctypes.c_void_p()
assert L.shampoo_adamw_create(ctypes.byref(cfg), P, L.shampoo_adamw_workspace_bytes(ctypes.byref(cfg)), S, ctypes.byref(h)) == 0
w, g = ((ctypes.c_void_p * n)(*[(k + 1) << 20 for k in range(n)]) for _ in range(2))
step = lambda t: L.shampoo_adamw_step(h, w, g, None, 0.1, t, None, 1.0, S)
for fail in range(3):
    reset(fail=fail)
    print(step(5), len(launches("adamw_kernel")))
reset()
print(step(5), len(launches("adamw_kernel")))
reset()
print(step(5), len(launches("adamw_kernel")))
"""


def test_a_step_that_failed_in_the_middle_is_whole_when_it_is_tried_again(lib):
    """What the header says: launches before the failing one were made, the step does not count, the next try makes all of them"""
    assert [line for line in host_hip.run(lib, RETRY) if line] == ["-6 1", "-6 2", "-6 3", "0 3", "-5 0"]
