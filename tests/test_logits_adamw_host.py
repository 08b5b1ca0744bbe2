"""Log probabilities, gradient norms and AdamW without a GPU: refusals (nothing is enqueued: the pointers are never touched), workspaces, the largest
sizes that the checks admit against a runtime that launches nothing (and refuses launches of 2^32 threads and more), and what a call returns when a
launch or an allocation fails."""
import ctypes

import pytest

import host_hip
from paper_2309_06497_amd import binding as B

P, ODD, BIG = ctypes.c_void_p(1 << 20), ctypes.c_void_p((1 << 20) + 4), 1 << 50
NAN, INF = float("nan"), float("inf")


@pytest.fixture(scope="module")
def lib(tmp_path_factory):
    return host_hip.build(str(tmp_path_factory.mktemp("hip")))


def logits(**kw):
    good = dict(rows=10, classes=100, tokens=2, top=3, dtype=1, inverse_temperature=1.0, ld=100)
    return B.Logits(*[{**good, **kw}[f[0]] for f in B.Logits._fields_])


def test_log_probs_refusals():
    L = B.lib()

    def call(z=P, t=P, lp=P, h=P, tt=P, tlp=P, st=P, ws=P, nbytes=BIG, **kw):
        return L.shampoo_log_probs(ctypes.byref(logits(**kw)), z, t, lp, h, tt, tlp, st, ws, nbytes, None)

    def grad(z=P, t=P, st=P, a=P, b=P, dz=P, ld=100, **kw):
        return L.shampoo_log_probs_grad(ctypes.byref(logits(**kw)), z, t, st, a, b, dz, ld, None)

    assert L.shampoo_log_probs(None, P, P, P, P, P, P, P, P, BIG, None) == -1 and L.shampoo_log_probs_grad(None, P, P, P, P, P, P, 100, None) == -1
    for f in (call, grad):
        assert f(z=None) == -1 and f(t=None) == -1 and f(st=None) == -1
        assert f(rows=-1) == -2 and f(classes=0) == -2 and f(tokens=-1) == -2 and f(top=-1) == -2 and f(classes=101) == -2
        assert f(dtype=2) == -3 and f(inverse_temperature=0.0) == -3 and f(inverse_temperature=-1.0) == -3 and f(inverse_temperature=NAN) == -3 and f(inverse_temperature=INF) == -3 and f(inverse_temperature=3e38) == -3
        assert f(rows=1 << 31) == -7 and f(tokens=65) == -7 and f(top=65) == -7
        assert f(st=ODD) == -7
        assert f(rows=0, z=None, t=None, st=None) == 0
    assert call(classes=(1 << 22) + 1, ld=1 << 23) == -7 and grad(classes=(1 << 22) + 1, ld=1 << 23) == -2
    assert call(lp=None) == -1 and call(h=None) == -1 and call(tt=None) == -1 and call(tlp=None) == -1
    assert grad(dz=None) == -1 and grad(ld=99) == -2
    long = dict(rows=1, classes=1 << 20, ld=1 << 20)
    need = L.shampoo_log_probs_workspace_bytes(ctypes.byref(logits(**long)))
    assert need > 0
    assert call(ws=None, **long) == -4 and call(ws=ODD, **long) == -4 and call(nbytes=need - 1, **long) == -4
    assert L.shampoo_log_probs_workspace_bytes(None) == 0 and L.shampoo_log_probs_workspace_bytes(ctypes.byref(logits(classes=0))) == 0


ROWS = r"""
P = ctypes.c_void_p(1 << 40)
S = ctypes.c_void_p(STREAM)
for rows in (1, 63, 64, 1000, 4097, (1 << 22) + 1, (1 << 31) - 1):
    for classes in (1, 512, 2048, 2049, 8193, 65537, 131072, 131080, 1 << 22):
        for skew in (0, 2):
            for top in (0, 64):
                ld = classes + skew // 2
                c = B.Logits(rows, classes, 1, top, 1, 1.0, ld)
                n = L.shampoo_log_probs_workspace_bytes(ctypes.byref(c))
                z = ctypes.c_void_p((1 << 40) + skew)
                reset()
                rc = L.shampoo_log_probs(ctypes.byref(c), z, P, P, P, P, P, P, P, n, S)
                small, parts, joins = (sum(e.a * k for e in launches(name)) for name, k in (("log_probs_row_kernel", 4), ("log_probs_kernel", 1), ("log_probs_join_kernel", 1)))
                one = all(e.stream == STREAM for e in entries())
                reset()
                rg = L.shampoo_log_probs_grad(ctypes.byref(c), z, P, P, P, P, P, ld, S)
                print(rows, classes, rc, rg, small, parts, joins, sum(e.a for e in launches("log_probs_grad_kernel")), one and all(e.stream == STREAM for e in entries()))
"""


def test_log_probs_of_as_many_rows_and_classes_as_they_admit(lib):
    seen = [line.split() for line in host_hip.run(lib, ROWS) if line]
    assert len(seen) == 7 * 9 * 2 * 2
    for line in seen:
        rows, classes, rc, rg, small, parts, joins, grads = map(int, line[:8])
        assert rc == 0 and rg == 0 and line[8] == "True", line
        if classes <= 2048:
            assert rows <= small < rows + 4 and parts == 0 and joins == 0, line
        else:
            assert small == 0 and parts % rows == 0 and parts // rows <= 64, line
            assert joins == (rows if parts > rows else 0), line
            assert parts // rows >= -(-classes // 131072), line
        assert rows <= 4 * grads < rows + 4 if classes <= 4096 else grads % rows == 0, line


def test_gradient_norm_refusals():
    L = B.lib()

    def call(n=2, grads=(1 << 20, 1 << 21), numel=(5, 6), dtype=0, norm=P, ws=P, nbytes=BIG):
        g = (ctypes.c_void_p * len(grads))(*grads) if grads else None
        m = (ctypes.c_int64 * len(numel))(*numel) if numel else None
        return L.shampoo_gradient_norm(n, g, m, dtype, norm, P, ws, nbytes, None)

    assert call(grads=None) == -1 and call(numel=None) == -1 and call(norm=None) == -1 and call(grads=(1 << 20, None)) == -1
    assert call(n=0) == -2 and call(n=-1) == -2 and call(numel=(5, -1)) == -2 and call(dtype=2) == -3
    assert call(numel=(1 << 39, 1)) == -7 and call(numel=((1 << 63) - 1, (1 << 63) - 1)) == -7
    two = (ctypes.c_int64 * 2)(5, 6)
    need = L.shampoo_gradient_norm_workspace_bytes(2, two)
    assert need > 0 and call(ws=None) == -4 and call(ws=ODD) == -4 and call(nbytes=need - 1) == -4
    assert L.shampoo_gradient_norm_workspace_bytes(0, two) == 0 and L.shampoo_gradient_norm_workspace_bytes(2, None) == 0


NORMS = r"""
P, S = ctypes.c_void_p(1 << 40), ctypes.c_void_p(STREAM)
for sizes in ([0], [1], [0, 0, 5], [(1 << 39)], [1 << 38, (1 << 38) - 1, 0], [7] * 1000, [0] * 191 + [3] + [0] * 200, [1] * (1 << 20)):
    n = len(sizes)
    g = (ctypes.c_void_p * n)(*[(k + 1) << 20 for k in range(n)])
    m = (i64 * n)(*sizes)
    ws = L.shampoo_gradient_norm_workspace_bytes(n, m)
    reset()
    rc = L.shampoo_gradient_norm(n, g, m, 1, P, P, P, ws, S)
    k = launches("square_sums")
    print(n, rc, len(k), len(entries()) - len(k), ws >> 20)
"""


def test_gradient_norms_of_as_many_elements_as_they_admit(lib):
    seen = [list(map(int, line.split())) for line in host_hip.run(lib, NORMS) if line]
    assert len(seen) == 8
    for n, rc, sums, others, megabytes in seen:
        assert rc == 0 and sums == -(-n // 192) and others == 1 and megabytes < 80, (n, rc, sums, others, megabytes)


def config(sizes=(5, 6), **kw):
    good = dict(n_params=len(sizes), numel=(ctypes.c_int64 * max(len(sizes), 1))(*sizes), decay=None, state_bits=32, param_dtype=0, grad_dtype=0, device=0, beta1=0.9, beta2=0.999,
                epsilon=1e-8, weight_decay=0.01)
    return B.AdamWConfig(*[{**good, **kw}[f[0]] for f in B.AdamWConfig._fields_])


def test_adamw_configurations():
    L = B.lib()
    out = ctypes.c_void_p()

    def create(cfg, ws=P, nbytes=BIG):
        return L.shampoo_adamw_create(ctypes.byref(cfg), ws, nbytes, None, ctypes.byref(out))

    bad = [(config(n_params=0), -2), (config(numel=None), -1), (config((5, -1)), -2), (config((1 << 39, 1)), -7), (config(n_params=(1 << 20) + 1), -7), (config(state_bits=16), -3),
           (config(param_dtype=2), -3), (config(grad_dtype=-1), -3), (config(beta1=1.0), -3), (config(beta2=-0.1), -3), (config(beta1=NAN), -3), (config(epsilon=0.0), -3),
           (config(epsilon=NAN), -3), (config(epsilon=INF), -3), (config(weight_decay=-1.0), -3), (config(weight_decay=INF), -3)]
    for cfg, code in bad:
        assert create(cfg) == code and L.shampoo_adamw_workspace_bytes(ctypes.byref(cfg)) == 0
    assert L.shampoo_adamw_create(None, P, BIG, None, ctypes.byref(out)) == -1 and L.shampoo_adamw_create(ctypes.byref(config()), P, BIG, None, None) == -1
    need = L.shampoo_adamw_workspace_bytes(ctypes.byref(config()))
    assert create(config(), ws=None) == -4 and create(config(), ws=ODD) == -4 and create(config(), nbytes=need - 1) == -4
    for call in (lambda: L.shampoo_adamw_step(None, None, None, None, 0.1, 0, None, 1.0, None), lambda: L.shampoo_adamw_get(None, P, P, 0, None),
                 lambda: L.shampoo_adamw_set(None, P, P, None), lambda: L.shampoo_adamw_destroy(None)):
        assert call() == -1
    n = 1 << 30
    size = lambda **kw: L.shampoo_adamw_workspace_bytes(ctypes.byref(config((n,), **kw))) / n
    assert 8.0 <= size() < 8.03 and 2.0 <= size(state_bits=8) < 2.05


STEPS = r"""
S = ctypes.c_void_p(STREAM)
P = ctypes.c_void_p(1 << 40)
def config(sizes, **kw):
    good = dict(n_params=len(sizes), numel=(i64 * len(sizes))(*sizes), decay=None, state_bits=8, param_dtype=0, grad_dtype=1, device=0, beta1=0.9, beta2=0.999, epsilon=1e-8, weight_decay=0.01)
    return B.AdamWConfig(*[{**good, **kw}[f[0]] for f in B.AdamWConfig._fields_])
def create(sizes, **kw):
    cfg, h = config(sizes, **kw), ctypes.c_void_p()
    return L.shampoo_adamw_create(ctypes.byref(cfg), P, L.shampoo_adamw_workspace_bytes(ctypes.byref(cfg)), S, ctypes.byref(h)), h
def step(h, n, t, copies=False, lr=0.1, norm=None, most=1.0, hole=None):
    w, g, c = ((ctypes.c_void_p * n)(*[None if k == hole else (k + 1) << 20 for k in range(n)]) for _ in range(3))
    return L.shampoo_adamw_step(h, w, g, c if copies else None, lr, t, norm, most, S)
for sizes, copies in (([5, 0, 4096], False), ([7] * 240, False), ([7] * 241, False), ([7] * 161, True), ([0] * 500, False), ([1 << 36], False), ([(1 << 35) - 1] * 3, True)):
    n = len(sizes)
    reset()
    rc, h = create(sizes)
    made = [(e.what, e.name.decode()) for e in entries()]
    reset()
    rs = step(h, n, 3, copies)
    k = launches("adamw_kernel")
    print(n, rc, rs, len(k), sum(e.a for e in k), sum(-(-s // 2048) for s in sizes), all(e.stream == STREAM for e in entries()))
    reset()
    assert step(h, n, 3) == -5 and step(h, n, -1) == -5 and step(h, n, 4, lr=float("nan")) == -3 and step(h, n, 4, lr=1e39) == -3 and step(h, n, 4, norm=P, most=0.0) == -3 and step(h, n, 4, norm=P, most=float("nan")) == -3
    if sizes[0]:
        assert step(h, n, 4, hole=0) == -1 and L.shampoo_adamw_get(h, None, P, 0, S) == -1 and L.shampoo_adamw_set(h, P, None, S) == -1
    assert L.shampoo_adamw_get(h, P, P, 3, S) == -3 and not entries()
    assert step(h, n, 4, norm=P, most=float("inf")) == 0
    assert L.shampoo_adamw_destroy(h) == 0
rc, h = create([5, 6], param_dtype=1)
assert step(h, 2, 0, copies=True) == -3 and step(h, 2, 0) == 0
# a launch that fails: the step does not count
rc, h = create([7] * 600)
codes = list(failing(lambda: step(h, 600, 0)))
assert [c for _, c in codes] == [-6] * 3, codes
reset()
assert step(h, 600, 0) == -5 and step(h, 600, 1) == 0
made = []
reset()
for rc in out_of_memory(lambda: made.append(create([5, 6])) or made[-1][0]):
    assert rc == -6 and not made[-1][1].value
assert [rc for _, rc in failing(lambda: create([5, 6])[0])] and all(rc == -6 for _, rc in failing(lambda: create([5, 6])[0]))
reset()
z = B.Logits(1, 1 << 20, 1, 3, 1, 1.0, 1 << 20)
for call in (lambda: L.shampoo_log_probs(ctypes.byref(z), P, P, P, P, P, P, P, P, 1 << 30, S), lambda: L.shampoo_log_probs_grad(ctypes.byref(z), P, P, P, P, P, P, 1 << 20, S)):
    assert all(rc == -6 for _, rc in failing(call))
g, m = (ctypes.c_void_p * 2)(1 << 20, 1 << 21), (i64 * 2)(5, 6)
assert [rc for _, rc in failing(lambda: L.shampoo_gradient_norm(2, g, m, 0, P, P, P, 1 << 20, S))] == [-6, -6]
print("done")
"""


def test_adamw_steps_and_failures(lib):
    seen = [line for line in host_hip.run(lib, STEPS) if line]
    assert seen[-1] == "done" and len(seen) == 8
    for line in seen[:-1]:
        n, rc, rs, count, blocks, want, stream = line.split()
        n, count = int(n), int(count)
        assert int(rc) == 0 and int(rs) == 0 and blocks == want and stream == "True", line
    launches = [int(line.split()[3]) for line in seen[:-1]]
    assert launches[:5] == [1, 1, 2, 2, 0] and launches[5] == -(-(1 << 25) // (1 << 22))


def test_tensors_that_the_binding_refuses():
    torch = pytest.importorskip("torch")
    t = torch.zeros((3, 4))
    k = torch.zeros((3,), dtype=torch.int64)
    for call in (lambda: B.shampoo_log_probs(t, k), lambda: B.shampoo_gradient_norm([t]), lambda: B.shampoo_gradient_norm([]), lambda: B.shampoo_gradient_norm([1])):
        with pytest.raises(AssertionError):
            call()
    with pytest.raises(TypeError):
        B.shampoo_gradient_norm(1)
    with pytest.raises(B.ShampooError) as e:
        B.AdamW([(3, 4)], beta1=1.5)
    assert e.value.code == -3
    with pytest.raises(ValueError):
        B.AdamW([(3, 4)], decay=[True, False])
