"""Refusals of the training operators (nothing is enqueued: the pointers are never touched), their workspaces, and what they return
when a launch fails (a runtime that launches nothing)."""
import ctypes

import pytest

import host_hip
from paper_2309_06497_amd import binding as B

P, BIG = ctypes.c_void_p(1 << 20), 1 << 50
NAN = float("nan")


def test_cross_entropy_refusals():
    L = B.lib()
    names = [f[0] for f in B.CrossEntropy._fields_]
    good = dict(rows=10, features=16, classes=100, dtype=1, grad_dtype=1, w_layout=0, has_bias=1, gradients=1, ldx=16, ldw=16, lddx=16, lddw=16)

    def call(x=P, w=P, bias=P, t=P, scale=1.0, loss=P, ws=P, nbytes=BIG, **kw):
        c = B.CrossEntropy(*[{**good, **kw}[n] for n in names])
        return L.shampoo_linear_cross_entropy(ctypes.byref(c), x, w, bias, t, None, scale, loss, P, P, P, ws, nbytes, None)

    odd = ctypes.c_void_p((1 << 20) + 8)
    assert L.shampoo_linear_cross_entropy(None, P, P, P, P, None, 1.0, P, P, P, P, P, BIG, None) == -1
    assert call(x=None) == -1 and call(w=None) == -1 and call(bias=None) == -1 and call(t=None) == -1 and call(loss=None) == -1
    assert call(rows=-1) == -2 and call(features=0) == -2 and call(classes=0) == -2
    assert call(ldx=15) == -2 and call(ldw=15) == -2 and call(lddx=15) == -2 and call(lddw=15) == -2
    assert call(w_layout=1, ldw=99, lddw=100) == -2 and call(w_layout=1, ldw=100, lddw=99) == -2
    assert call(dtype=2) == -3 and call(grad_dtype=-1) == -3 and call(w_layout=2) == -3 and call(dtype=0) == -3
    assert call(scale=NAN) == -3 and call(scale=float("inf")) == -3
    assert call(classes=(1 << 22) + 1) == -7 and call(features=65537, ldx=65537, ldw=65537) == -7 and call(rows=1 << 31) == -7
    assert call(x=odd) == -7 and call(w=odd) == -7
    assert call(ws=None) == -4 and call(ws=odd) == -4
    c = B.CrossEntropy(*[good[n] for n in names])
    need = L.shampoo_linear_cross_entropy_workspace_bytes(ctypes.byref(c))
    assert need > 0 and call(nbytes=need - 1) == -4
    c.classes = 0
    assert L.shampoo_linear_cross_entropy_workspace_bytes(ctypes.byref(c)) == 0
    assert L.shampoo_linear_cross_entropy_workspace_bytes(None) == 0


def test_cross_entropy_workspace_is_bounded():
    """The logits of all rows are never there: a piece of them, at most 4 GiB with what the gradients need of it."""
    L = B.lib()
    for rows in (1 << 14, 1 << 20, (1 << 31) - 1):
        c = B.CrossEntropy(rows, 2048, 131072, 1, 0, 0, 0, 1, 2048, 2048, 2048, 2048)
        assert L.shampoo_linear_cross_entropy_workspace_bytes(ctypes.byref(c)) < 5 << 30
        c.grad_dtype = 1          # bf16 weight gradients of several pieces are summed in float32
        assert L.shampoo_linear_cross_entropy_workspace_bytes(ctypes.byref(c)) < (5 << 30) + 131072 * 2048 * 4


def test_checkpoint_refusals():
    L = B.lib()
    size = L.shampoo_checkpoint_bytes
    assert size(0, 5) == 0 and size(-1, 5) == 0 and size(5, 0) == 0 and size(5, (1 << 20) + 1) == 0 and size(1 << 31, 8) == 0
    assert size(3, 33) == 256 + 256 and size(1000, 1024) == 1024000 + 32000 and size((1 << 31) - 1, 1 << 20) > 1 << 50
    n = size(10, 40)

    def pack(x=P, dtype=1, rows=10, cols=40, ld=40, packed=P, nbytes=n):
        return L.shampoo_checkpoint_pack(x, dtype, rows, cols, ld, packed, nbytes, None)

    def unpack(packed=P, nbytes=n, rows=10, cols=40, act=0, y=P, dtype=1, ld=40):
        return L.shampoo_checkpoint_unpack(packed, nbytes, rows, cols, act, y, dtype, ld, None)

    def grad(packed=P, nbytes=n, rows=10, cols=40, act=2, dy=P, dtype=1, ld=40, dx=P, lddx=40):
        return L.shampoo_checkpoint_activation_grad(packed, nbytes, rows, cols, act, dy, dtype, ld, dx, lddx, None)

    assert pack(x=None) == -1 and unpack(y=None) == -1 and grad(dy=None) == -1 and grad(dx=None) == -1
    for call in (pack, unpack, grad):
        assert call(packed=None) == -1 and call(packed=ctypes.c_void_p((1 << 20) + 16)) == -4 and call(nbytes=n - 1) == -4
        assert call(rows=-1) == -2 and call(cols=0) == -2 and call(ld=39) == -2 and call(dtype=7) == -3
        assert call(cols=(1 << 20) + 1, nbytes=BIG) == -7
        assert call(rows=0) == 0
    assert unpack(act=4) == -3 and unpack(act=-1) == -3 and grad(act=4) == -3 and grad(lddx=39) == -2


def test_weight_gradient_refusals():
    L = B.lib()
    n = L.shampoo_checkpoint_bytes(10, 40)
    need = L.shampoo_checkpoint_weight_grad_workspace_bytes(10, 40, 24, 0, 1, 24, 1, 1)

    def call(packed=P, pbytes=n, rows=10, cols=40, act=0, dy=P, dtype=1, out=24, ld=24, dw=P, grad=1, layout=1, lddw=24, db=P, ws=P, nbytes=max(need, 1)):
        return L.shampoo_checkpoint_weight_grad(packed, pbytes, rows, cols, act, dy, dtype, out, ld, dw, grad, layout, lddw, db, ws, nbytes, None)

    odd = ctypes.c_void_p((1 << 20) + 8)
    assert call(packed=None) == -1 and call(dy=None) == -1 and call(dw=None) == -1
    assert call(rows=-1) == -2 and call(cols=0) == -2 and call(out=0) == -2 and call(ld=23) == -2 and call(lddw=23) == -2
    assert call(layout=0, lddw=39) == -2 and call(layout=2) == -3
    assert call(act=4) == -3 and call(dtype=2) == -3 and call(grad=2) == -3 and call(dtype=0, grad=1) == -3
    assert call(cols=65537, pbytes=BIG) == -7 and call(out=(1 << 22) + 1, ld=1 << 23) == -7 and call(dy=odd) == -7
    assert call(packed=odd) == -4 and call(pbytes=n - 1) == -4
    assert call(ws=None) == -4 and call(ws=odd) == -4 and call(nbytes=need - 1) == -4
    assert L.shampoo_checkpoint_weight_grad_workspace_bytes(10, 0, 24, 0, 1, 24, 1, 1) == 0


def test_residual_norm_refusals():
    L = B.lib()
    names = [f[0] for f in B.ResidualNorm._fields_]
    good = dict(rows=12, cols=40, dtype=1, post=1, pre=2, gates=3, epsilon=1e-5, scale=1.0, w_post=1 << 20, b_post=None, gate=1 << 20,
                w_pre=1 << 20, b_pre=None)
    n = L.shampoo_checkpoint_bytes(12, 40)

    def forward(r=P, ldr=40, f=P, ldf=40, o=P, ldo=40, h=P, ldh=40, pr=P, pf=P, nbytes=n, **kw):
        c = B.ResidualNorm(*[{**good, **kw}[k] for k in names])
        return L.shampoo_residual_norm_forward(ctypes.byref(c), r, ldr, f, ldf, o, ldo, h, ldh, pr, pf, nbytes, None)

    def backward(packed=1, r=P, ldr=40, f=P, ldf=40, do=P, lddo=40, dh=P, lddh=40, dr=P, lddr=40, df=P, lddf=40, ws=P, nbytes=BIG, **kw):
        c = B.ResidualNorm(*[{**good, **kw}[k] for k in names])
        return L.shampoo_residual_norm_backward(ctypes.byref(c), packed, r, ldr, f, ldf, do, lddo, dh, lddh, dr, lddr, df, lddf, P, P, P, P, P,
                                                ws, nbytes, None)

    odd = ctypes.c_void_p((1 << 20) + 8)
    for call in (forward, backward):
        assert call(r=None) == -1 and call(f=None) == -1 and call(w_post=None) == -1 and call(w_pre=None) == -1 and call(gate=None) == -1
        assert call(rows=-1) == -2 and call(cols=0) == -2 and call(gates=-1) == -2 and call(gates=5) == -2
        assert call(cols=16385) == -7 and call(rows=1 << 31) == -7
        assert call(dtype=3) == -3 and call(post=3) == -3 and call(pre=-1) == -3
        assert call(epsilon=-1.0) == -3 and call(epsilon=NAN) == -3 and call(scale=NAN) == -3
    assert forward(ldr=39) == -2 and forward(ldf=39) == -2 and forward(ldo=39) == -2 and forward(ldh=39) == -2
    assert forward(o=None) == -1 and forward(h=None) == -1 and forward(pr=None) == -1 and forward(pf=None) == -1
    assert forward(pr=odd) == -4 and forward(nbytes=n - 1) == -4
    assert backward(dh=None) == -1 and backward(dr=None) == -1 and backward(df=None) == -1
    assert backward(packed=0, ldr=39) == -2 and backward(packed=0, ldf=39) == -2
    assert backward(lddo=39) == -2 and backward(lddh=39) == -2 and backward(lddr=39) == -2 and backward(lddf=39) == -2
    assert backward(r=odd) == -4 and backward(ws=None) == -4 and backward(ws=odd) == -4
    c = B.ResidualNorm(*[good[k] for k in names])
    need = L.shampoo_residual_norm_backward_workspace_bytes(ctypes.byref(c))
    assert need > 0 and backward(nbytes=need - 1) == -4
    assert L.shampoo_residual_norm_forward(None, P, 1, P, 1, P, 1, P, 1, None, None, 0, None) == -1
    assert L.shampoo_residual_norm_backward_workspace_bytes(None) == 0


def test_binding_refuses_other_types_and_devices():
    import torch
    x = torch.zeros((4, 8))
    with pytest.raises(AssertionError):
        B.shampoo_checkpoint_pack(x)
    with pytest.raises(AssertionError):
        B.shampoo_checkpoint_pack(x.half())
    with pytest.raises(AssertionError):
        B.shampoo_linear_cross_entropy(x, x, torch.zeros(4, dtype=torch.int64))


def test_a_launch_that_fails_is_reported(tmp_path):
    lib = host_hip.build(str(tmp_path))
    out = host_hip.run(lib, r"""
P = ctypes.c_void_p(1 << 40)
S = ctypes.c_void_p(STREAM)
c = B.CrossEntropy(300, 1000, 50001, 1, 0, 1, 1, 1, 1000, 50001, 1000, 50001)
n = L.shampoo_linear_cross_entropy_workspace_bytes(ctypes.byref(c))
k = B.ResidualNorm(64, 100, 1, 1, 2, 4, 1e-5, 1.0, 1 << 40, 1 << 40, 1 << 40, 1 << 40, 1 << 40)
m = L.shampoo_residual_norm_backward_workspace_bytes(ctypes.byref(k))
b = L.shampoo_checkpoint_bytes(64, 100)
calls = {
    "head": lambda: L.shampoo_linear_cross_entropy(ctypes.byref(c), P, P, P, P, P, 1.0, P, P, P, P, P, n, S),
    "pack": lambda: L.shampoo_checkpoint_pack(P, 1, 64, 100, 100, P, b, S),
    "unpack": lambda: L.shampoo_checkpoint_unpack(P, b, 64, 100, 1, P, 0, 100, S),
    "act": lambda: L.shampoo_checkpoint_activation_grad(P, b, 64, 100, 2, P, 1, 100, P, 100, S),
    "wgrad": lambda: L.shampoo_checkpoint_weight_grad(P, b, 64, 100, 3, P, 0, 77, 80, P, 0, 0, 100, P, P, 1 << 40, S),
    "forward": lambda: L.shampoo_residual_norm_forward(ctypes.byref(k), P, 100, P, 100, P, 100, P, 100, P, P, b, S),
    "backward": lambda: L.shampoo_residual_norm_backward(ctypes.byref(k), 1, P, 100, P, 100, P, 100, P, 100, P, 100, P, 100, P, P, P, P, P, P, m, S),
}
for name, call in calls.items():
    codes = [rc for _, rc in failing(call)]
    reset()
    assert call() == 0
    assert all(e.what == b"K" and e.stream == STREAM for e in entries()), name      # kernels on the caller's stream and nothing else
    print(name, len(codes), set(codes))
""")
    seen = [line.split(" ", 2) for line in out if line]
    assert len(seen) == 7 and all(codes == "{-6}" and int(k) > 0 for _, k, codes in seen), seen
