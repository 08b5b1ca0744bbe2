"""The operators of a training pass at the ends of their ranges, against float64: logits far from zero, values that bf16 does not reach,
rows in several pieces, strided outputs, results in place.

e = 2^-24 is the rounding of float32, u = 2^-8 that of bf16.  Bars are derived at each test."""
import math

import pytest

from paper_2309_06497_amd import binding as B

pytestmark = pytest.mark.gpu
U = 2.0 ** -8
KINDS = [("bf16", "bf16"), ("bf16", "f32"), ("f32", "f32")]


def torch_():
    import torch
    return torch


def gen(seed):
    g = torch_().Generator(device="cuda")
    g.manual_seed(seed)
    return g


def types(kind):
    torch = torch_()
    return [{"bf16": torch.bfloat16, "f32": torch.float32}[k] for k in kind]


def rel(got, want):
    torch = torch_()
    return float(torch.linalg.vector_norm(got.double() - want) / torch.linalg.vector_norm(want))


# ----------------------------------------------------------------------------
# Logits far from zero
# ----------------------------------------------------------------------------
def quarters(g, *shape):
    """-2/4 ... 2/4: products are sixteenths, which a float32 sum holds exactly beside 2^18"""
    torch = torch_()
    return torch.randint(-2, 3, shape, generator=g, device="cuda") * 0.25


def softmax_gradients(z, x, w, t):
    torch = torch_()
    z = z - z.amax(1, keepdim=True)
    total = torch.exp(z).sum(1, keepdim=True)
    i = torch.arange(z.shape[0], device="cuda")
    loss = torch.log(total)[:, 0] - z[i, t]
    g = torch.exp(z) / total
    g[i, t] -= 1.0
    return loss, g @ w, g.t() @ x, g.sum(0)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("by_bias", [False, True])
@pytest.mark.parametrize("offset", [2.0 ** 13, -2.0 ** 13, 2.0 ** 18])
@pytest.mark.parametrize("n,d,v", [(40, 64, 300), (200, 1024, 300), (70, 256, 2500), (600, 712, 16500)])
def test_a_common_offset_of_the_logits_changes_nothing(n, d, v, offset, by_bias, kind):
    """Logits are exact here (sixteenths beside at most 2^18: 23 bits), so what separates the result from the definition is what it is without an
    offset: exponents of |z - largest| < 64 off by 64 e, sums of exponentials by less than that again: 2^-17 in a loss and
    in float32 gradients; 3 u in bf16 ones."""
    torch = torch_()
    dt, grad = types(kind)
    g = gen(n + v)
    x, w = quarters(g, n, d), quarters(g, v, d)
    bias = None
    if by_bias:
        bias = torch.full((v,), offset, device="cuda")
    else:
        x[:, 0], w[:, 0] = math.copysign(2.0 ** 7, offset), abs(offset) / 2.0 ** 7
    t = torch.randint(0, v, (n,), generator=g, device="cuda")
    z = x.double() @ w.double().t() + (offset if by_bias else 0.0)
    loss64, dx64, dw64, db64 = softmax_gradients(z, x.double(), w.double(), t)
    loss, dx, dw, db = B.shampoo_linear_cross_entropy(x.to(dt), w.to(dt), t, bias=bias, grad_dtype=grad)
    alone = B.shampoo_linear_cross_entropy(x.to(dt), w.to(dt), t, bias=bias, gradients=False)
    for l in (loss, alone):
        assert float((l.double() - loss64).abs().max()) <= 2.0 ** -17 * max(1.0, float(loss64.max()))
    if not by_bias:        # the common feature's gradient: a sum of p - [t] over the classes, 0, times the offset
        dx, dx64 = dx[:, 1:], dx64[:, 1:]
    assert rel(dx, dx64) <= (3 * U if kind[0] == "bf16" else 2.0 ** -16)
    assert rel(dw, dw64) <= (3 * U if kind[1] == "bf16" else 2.0 ** -16)
    if by_bias:
        assert rel(db, db64) <= 2.0 ** -16


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("n,d,v", [(40, 64, 300), (200, 1024, 300), (600, 64, 16500)])
def test_the_softmax_of_equal_logits_however_low(n, d, v, kind):
    """A bias of the type's lowest value leaves nothing of x w^T: probabilities of 1 / classes, a loss of log(classes)."""
    torch = torch_()
    dt, grad = types(kind)
    g = gen(12)
    x, w = torch.randn((n, d), generator=g, device="cuda").to(dt), (torch.randn((v, d), generator=g, device="cuda") * 0.1).to(dt)
    t = torch.randint(0, v, (n,), generator=g, device="cuda")
    for low in (torch.finfo(torch.float32).min, -3.0e20):
        bias = torch.full((v,), low, device="cuda")
        loss64, dx64, dw64, db64 = softmax_gradients(torch.zeros((n, v), dtype=torch.float64, device="cuda"), x.double(), w.double(), t)
        loss, dx, dw, db = B.shampoo_linear_cross_entropy(x, w, t, bias=bias, grad_dtype=grad)
        assert float((loss.double() - loss64).abs().max()) <= 2.0 ** -20 * math.log(v)
        assert rel(dx, dx64) <= (3 * U if kind[0] == "bf16" else 2.0 ** -16)
        assert rel(dw, dw64) <= (3 * U if kind[1] == "bf16" else 2.0 ** -16)
        assert rel(db, db64) <= 2.0 ** -16


# ----------------------------------------------------------------------------
# Float32 values that bf16 does not reach
# ----------------------------------------------------------------------------
LARGEST = 3.4028234663852886e38


@pytest.mark.parametrize("out_in", [False, True])
@pytest.mark.parametrize("act", [B.ACT_NONE, B.ACT_SILU])
@pytest.mark.parametrize("n", [1, 64, 70, 999])
def test_weight_gradient_of_the_largest_and_of_infinite_float32_values(n, act, out_in):
    """dy's columns: ordinary, the largest float32, an infinity, two of one sign, two of different sign; in the last row too.  A
    result is what the sum is: within 2^-18 of the sum of its terms' sizes (float32 sums of n terms), infinite, or NaN."""
    torch = torch_()
    g = gen(n)
    x = torch.randint(0, 2, (n, 40), generator=g, device="cuda") * 0.25 + 0.25
    x *= torch.randint(0, 2, (n, 40), generator=g, device="cuda") * 2 - 1              # codes of 32 and 64 steps, or 64 and 128: held exactly
    dy = torch.randn((n, 9), generator=g, device="cuda")
    k = torch.tensor(sorted({0, n // 2, n - 1}), device="cuda")
    dy[k[-1], 1], dy[k[0], 2], dy[k[-1], 3], dy[k[0], 4], dy[k[-1], 5] = LARGEST, -LARGEST, math.inf, -math.inf, -math.inf
    dy[k[0], 6] = dy[k[-1], 6] = math.inf
    dy[k[0], 7], dy[k[-1], 7] = -math.inf, math.inf
    dy[k[-1], 8] = 3.397e38                                                           # rounds to an infinity of bf16
    c = B.shampoo_checkpoint_pack(x)
    assert torch.equal(B.shampoo_checkpoint_unpack(c), x)
    a = x.double() if act == B.ACT_NONE else x.double() * torch.sigmoid(x.double())
    want = (a[:, :, None] * dy.double()[:, None, :]).sum(0)
    size = (a[:, :, None] * dy.double()[:, None, :]).abs().sum(0)
    dw, db = B.shampoo_checkpoint_weight_grad(c, dy, act, out_in=out_in, bias=True)
    dw = dw.t() if out_in else dw
    fin = torch.isfinite(want)
    assert torch.equal(torch.isnan(dw), torch.isnan(want))
    assert torch.equal(dw[torch.isinf(want)].double(), want[torch.isinf(want)])
    assert bool(((dw.double() - want).abs()[fin] <= 2.0 ** -18 * size[fin]).all())
    want = dy.double().sum(0)
    assert torch.equal(torch.isnan(db), torch.isnan(want)) and torch.equal(db[torch.isinf(want)].double(), want[torch.isinf(want)])


def test_head_with_the_largest_float32_weight():
    torch = torch_()
    g = gen(4)
    for n, d, v in ((40, 64, 300), (90, 200, 2500)):
        x, w = torch.randn((n, d), generator=g, device="cuda"), torch.randn((v, d), generator=g, device="cuda") * 0.1
        x[:, 0], w[5, 0] = 2.0 ** -126, LARGEST                                         # 4 in a logit
        t = torch.randint(0, v, (n,), generator=g, device="cuda")
        loss64, dx64, dw64, _ = softmax_gradients(x.double() @ w.double().t(), x.double(), w.double(), t)
        loss, dx, dw, _ = B.shampoo_linear_cross_entropy(x, w, t)
        assert float((loss.double() - loss64).abs().max()) <= 2.0 ** -17 * float(loss64.max())
        assert rel(dw, dw64) <= 2.0 ** -16
        for part in (slice(0, 1), slice(1, d)):
            assert rel(dx[:, part], dx64[:, part]) <= 2.0 ** -16


# ----------------------------------------------------------------------------
# Many rows
# ----------------------------------------------------------------------------
def test_residual_norm_forward_in_several_launches():
    """2^22 workgroups of four rows a launch: the rows around each of their ends, and the last ones."""
    torch = torch_()
    g = gen(5)
    n, d = 2 * (1 << 24) + 5, 8
    r, f = torch.randn((n, d), generator=g, device="cuda").bfloat16(), torch.randn((n, d), generator=g, device="cuda").bfloat16()
    w = torch.rand((d,), generator=g, device="cuda") + 0.5
    r_out, h, r8, f8 = B.shampoo_residual_norm_forward(r, f, post=B.NORM_NONE, pre=B.NORM_RMS, w_pre=w, scale=0.5, checkpoint=True)
    held = [B.shampoo_checkpoint_unpack(c) for c in (r8, f8)]
    for k in range(0, n, 1 << 22):
        part = slice(k, min(n, k + (1 << 22)))
        out = r[part].double() + 0.5 * f[part].double()
        norm = out / torch.sqrt(out.square().mean(1, keepdim=True) + 1e-5) * w.double()
        assert float((r_out[part].double() - out).abs().max()) <= U * float(out.abs().max())
        assert float((h[part].double() - norm).abs().max()) <= U * float(norm.abs().max())
        for x, y in zip((r, f), held):
            assert float((x[part].double() - y[part].double()).abs().max()) <= float(x[part].abs().max()) / 127.5


@pytest.mark.parametrize("kind,n,d,bias,in_out", [
    (("bf16", "bf16"), 300, 200, False, False), (("bf16", "bf16"), 530, 40, True, True), (("bf16", "f32"), 300, 648, False, False),
    (("bf16", "f32"), 300, 40, True, False), (("f32", "f32"), 300, 104, False, True), (("f32", "f32"), 530, 24, True, False)])
def test_head_in_several_pieces_of_rows_whose_logits_are_kept(kind, n, d, bias, in_out):
    """256 rows of 4194301 classes are a piece: 16-bit logits, float32 ones, and a bias gradient that later pieces add to.  |z| < 16: exponents
    off by 2^-19, float32 gradients by less than 2^-16 of their norm; bf16 ones 3 u."""
    torch = torch_()
    dt, grad = types(kind)
    g = gen(n + d)
    v = 4194301
    x, w = torch.randn((n, d), generator=g, device="cuda").to(dt), (torch.randn((v, d), generator=g, device="cuda") * (2 / math.sqrt(d))).to(dt)
    t = torch.randint(0, v, (n,), generator=g, device="cuda")
    b = torch.randn((v,), generator=g, device="cuda") if bias else None
    wv = w.t().contiguous().t() if in_out else w
    loss, dx, dw, db = B.shampoo_linear_cross_entropy(x, wv, t, bias=b, scale=1.0 / n, grad_dtype=grad)
    x64, w64, b64 = x.double(), w.double(), b.double() if bias else 0.0
    loss64, dx64 = torch.zeros(n, dtype=torch.float64, device="cuda"), torch.zeros_like(x64)
    dw64, db64, largest = torch.zeros_like(w64), torch.zeros(v, dtype=torch.float64, device="cuda"), 0.0
    for k in range(0, n, 100):                 # 2^31 elements and more in one float64 product came out wrong in places
        z, tk = x64[k:k + 100] @ w64.t() + b64, t[k:k + 100]
        largest = max(largest, float(z.abs().max()))
        i = torch.arange(z.shape[0], device="cuda")
        lse = torch.logsumexp(z, 1)
        loss64[k:k + 100] = lse - z[i, tk]
        p = z.sub_(lse[:, None]).exp_()
        p[i, tk] -= 1.0
        p /= n
        dx64[k:k + 100] = p @ w64
        dw64 += p.t() @ x64[k:k + 100]
        db64 += p.sum(0)
    assert float((loss.double() - loss64).abs().max()) <= 2.0 ** -23 * (math.sqrt(d) + 16) * largest
    assert rel(dx, dx64) <= (3 * U if kind[0] == "bf16" else 2.0 ** -16)
    assert rel(dw, dw64) <= (3 * U if kind[1] == "bf16" else 2.0 ** -16)
    if bias:
        assert rel(db, db64) <= 2.0 ** -16


# ----------------------------------------------------------------------------
# Float32 accuracy takes all three bf16 terms
# ----------------------------------------------------------------------------
def two_terms(x):
    """What two bf16 terms hold of float32 x"""
    h = x.bfloat16().float()
    return h + (x - h).bfloat16().float()


@pytest.mark.parametrize("d,bias", [(8, False), (704, False), (8, True)])
@pytest.mark.parametrize("v", [251, 2 * 1190 + 1])
def test_float32_weight_gradient_of_bf16_rows_has_24_bits_of_g(v, d, bias):
    """One row, x = 1, w = 0: every logit is 0, p = 1 / v and dw is g itself, 1 / v and 1 / v - 1.  1 / v and the product with it are off by 2 e,
    three terms by less than e, their sum by 2 e: 2^-21 of each element.  Two terms of 1 / v are further off (2^-17.0 of it for 251)."""
    torch = torch_()
    x, w = torch.ones((1, d), device="cuda").bfloat16(), torch.zeros((v, d), device="cuda").bfloat16()
    t = torch.tensor([v // 2], device="cuda")
    want = torch.full((v,), 1.0 / v, dtype=torch.float64, device="cuda")
    want[v // 2] -= 1.0
    bar = 2.0 ** -21
    if v == 251:
        assert float(((two_terms(want.float()).double() - want) / want).abs().max()) > 8 * bar
    _, _, dw, db = B.shampoo_linear_cross_entropy(x, w, t, bias=torch.zeros(v, device="cuda") if bias else None, grad_dtype=torch.float32)
    assert float(((dw.double() - want[:, None]) / want[:, None]).abs().max()) <= bar
    if bias:
        assert float(((db.double() - want) / want).abs().max()) <= bar


@pytest.mark.parametrize("kind", [("bf16", "f32"), ("f32", "f32")])
@pytest.mark.parametrize("act", [B.ACT_GELU, B.ACT_SILU])
def test_float32_weight_gradient_has_24_bits_of_the_activation(act, kind):
    """One row, dy = 1: dw is a(x) itself.  x > 0, where erf and exp do not cancel: a few 2^-23 of each, three terms less than e: 2^-20.  Two
    terms are off by up to 2^-17."""
    torch = torch_()
    dt, grad = types(kind)
    x = torch.arange(1, 4096, device="cuda").float()[None] * 2.0 ** -10
    c = B.shampoo_checkpoint_pack(x.to(dt))
    z = B.shampoo_checkpoint_unpack(c, dtype=torch.float32).double()
    want = z * torch.sigmoid(z) if act == B.ACT_SILU else z * 0.5 * torch.special.erfc(-z / math.sqrt(2))
    some = want[0] > 0
    assert int(some.sum()) > 4000
    bar = 2.0 ** -20
    assert float(((two_terms(want.float()).double() - want) / want)[0, some].abs().max()) > 4 * bar
    dw = B.shampoo_checkpoint_weight_grad(c, torch.ones((1, 1), device="cuda").to(dt), act, grad, out_in=True)
    assert float(((dw.double() - want) / want)[0, some].abs().max()) <= bar


# ----------------------------------------------------------------------------
# Results in place and in rows further apart, by the C interface
# ----------------------------------------------------------------------------
class Rows:
    """A matrix inside a buffer of one value: its rows `ld` apart, from an element on that is not aligned (aligned: on 256 bytes)"""
    FILL = 77.0

    def __init__(self, rows, cols, dtype, gap=5, values=None, aligned=False):
        torch = torch_()
        self.ld = -(-(cols + gap) // 8) * 8 if aligned else cols + gap
        first = 256 if aligned else self.ld + 3
        self.all = torch.full((first + (rows + 2) * self.ld,), self.FILL, dtype=dtype, device="cuda")
        self.view = torch.as_strided(self.all, (rows, cols), (self.ld, 1), first)
        if values is not None:
            self.view.copy_(values)

    def p(self):
        return self.view.data_ptr()

    def check(self, want):
        """The matrix as wanted, bit by bit, and nothing else touched"""
        torch = torch_()
        assert torch.equal(self.view, want)
        self.view.fill_(self.FILL)
        assert bool((self.all == self.FILL).all())


def done(rc):
    torch_().cuda.synchronize()
    assert rc == 0, rc


def stream():
    return torch_().cuda.current_stream().cuda_stream


def code(dt):
    return B.GRAD_F32 if dt == torch_().float32 else B.GRAD_BF16


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("in_out", [False, True])
@pytest.mark.parametrize("n,d,v,bias", [(3, 7, 5, False), (130, 201, 257, True), (65, 777, 1001, False), (600, 130, 16501, False), (1000, 257, 20003, True)])
def test_gradients_of_the_head_in_rows_further_apart(n, d, v, bias, in_out, kind):
    import ctypes
    torch = torch_()
    dt, grad = types(kind)
    g = gen(n)
    x, w = torch.randn((n, d), generator=g, device="cuda").to(dt), (torch.randn((v, d), generator=g, device="cuda") * 0.1).to(dt)
    t = torch.randint(0, v, (n,), generator=g, device="cuda")
    b = torch.randn((v,), generator=g, device="cuda") if bias else None
    wv = w.t().contiguous().t() if in_out else w
    loss, dx, dw, db = B.shampoo_linear_cross_entropy(x, wv, t, bias=b, grad_dtype=grad)
    dw = dw.t() if in_out else dw
    x2, w2 = Rows(n, d, dt, values=x, aligned=True), Rows(*dw.shape, dt, values=w.t() if in_out else w, aligned=True)
    dx2, dw2, loss2 = Rows(n, d, dt), Rows(*dw.shape, grad), Rows(1, n, torch.float32)
    db2 = Rows(1, v, torch.float32)
    c = B.CrossEntropy(n, d, v, code(dt), code(grad), B.IN_OUT if in_out else B.OUT_IN, int(bias), 1, x2.ld, w2.ld, dx2.ld, dw2.ld)
    need = B.lib().shampoo_linear_cross_entropy_workspace_bytes(ctypes.byref(c))
    ws = torch.full((need + 4096,), 255, dtype=torch.uint8, device="cuda")       # NaN, whatever is read of it
    done(B.lib().shampoo_linear_cross_entropy(ctypes.byref(c), x2.p(), w2.p(), b.data_ptr() if bias else None, t.data_ptr(), None, 1.0, loss2.p(), dx2.p(),
                                              dw2.p(), db2.p() if bias else None, ws.data_ptr(), need, stream()))
    assert bool((ws[need:] == 255).all())
    loss2.check(loss[None])
    dx2.check(dx)
    dw2.check(dw)
    x2.check(x)
    w2.check(w.t() if in_out else w)
    if bias:
        db2.check(db[None])


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("n,d", [(1, 1), (3, 7), (5, 33), (70, 200), (33, 1001)])
def test_checkpoints_of_rows_further_apart_and_gradients_in_place(n, d, dt):
    torch = torch_()
    dt, = types((dt,))
    L, g = B.lib(), gen(d)
    x, dy = torch.randn((n, d), generator=g, device="cuda").to(dt), torch.randn((n, d), generator=g, device="cuda").to(dt)
    c = B.shampoo_checkpoint_pack(x)
    need = L.shampoo_checkpoint_bytes(n, d)
    x2, packed = Rows(n, d, dt, values=x), torch.full((need + 512,), 77, dtype=torch.uint8, device="cuda")
    done(L.shampoo_checkpoint_pack(x2.p(), code(dt), n, d, x2.ld, packed.data_ptr(), need, stream()))
    x2.check(x)
    assert bool((packed[need:] == 77).all())
    for act in (B.ACT_NONE, B.ACT_SILU):
        y = Rows(n, d, dt)
        done(L.shampoo_checkpoint_unpack(packed.data_ptr(), need, n, d, act, y.p(), code(dt), y.ld, stream()))
        y.check(B.shampoo_checkpoint_unpack(c, act))
    want = B.shampoo_checkpoint_activation_grad(c, dy, B.ACT_GELU)
    dy2, dx2 = Rows(n, d, dt, values=dy), Rows(n, d, dt, gap=9)
    done(L.shampoo_checkpoint_activation_grad(packed.data_ptr(), need, n, d, B.ACT_GELU, dy2.p(), code(dt), dy2.ld, dx2.p(), dx2.ld, stream()))
    dx2.check(want)
    done(L.shampoo_checkpoint_activation_grad(packed.data_ptr(), need, n, d, B.ACT_GELU, dy2.p(), code(dt), dy2.ld, dy2.p(), dy2.ld, stream()))
    dy2.check(want)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("out_in", [False, True])
@pytest.mark.parametrize("n,i,o", [(1, 1, 1), (70, 33, 65), (999, 130, 331), (2500, 1000, 17001)])
def test_weight_gradient_in_rows_further_apart(n, i, o, out_in, kind):
    """The last size: tiles of 256 of which a last round is split"""
    torch = torch_()
    dt, grad = types(kind)
    L, g = B.lib(), gen(o)
    x, dy = torch.randn((n, i), generator=g, device="cuda").to(dt), torch.randn((n, o), generator=g, device="cuda").to(dt)
    c = B.shampoo_checkpoint_pack(x)
    dy2 = Rows(n, o, dt, values=dy, aligned=True)
    dw, db = B.shampoo_checkpoint_weight_grad(c, dy2.view, B.ACT_SILU, grad, out_in, True)
    dw2, db2 = Rows(*dw.shape, grad), Rows(1, o, torch.float32)
    need = L.shampoo_checkpoint_weight_grad_workspace_bytes(n, i, o, B.ACT_SILU, code(dt), dy2.ld, code(grad), 1)
    ws = torch.full((need + 4096,), 255, dtype=torch.uint8, device="cuda")       # NaN, whatever is read of it
    done(L.shampoo_checkpoint_weight_grad(c.packed.data_ptr(), c.packed.numel(), n, i, B.ACT_SILU, dy2.p(), code(dt), o, dy2.ld, dw2.p(), code(grad),
                                          B.OUT_IN if out_in else B.IN_OUT, dw2.ld, db2.p(), ws.data_ptr(), need, stream()))
    assert bool((ws[need:] == 255).all())
    dw2.check(dw)
    db2.check(db[None])
    dy2.check(dy)


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("packed", [False, True])
@pytest.mark.parametrize("n,d,gates", [(1, 1, 1), (6, 33, 3), (40, 520, 0), (300, 1001, 1), (24, 2049, 4), (9, 4100, 1), (6, 8201, 2)])
def test_residual_norms_in_place_in_rows_further_apart(n, d, gates, packed, dt):
    """r_out in the place of r, dr in that of dr_out, df in that of dh"""
    import ctypes
    torch = torch_()
    dt, = types((dt,))
    L, g = B.lib(), gen(d)
    r, f, dr_out, dh = (torch.randn((n, d), generator=g, device="cuda").to(dt) for _ in range(4))
    w_post, b_post, w_pre, b_pre = (torch.randn((d,), generator=g, device="cuda") for _ in range(4))
    gate = torch.randn((gates, d), generator=g, device="cuda") if gates else None
    kw = dict(post=B.NORM_LAYER, pre=B.NORM_LAYER, w_post=w_post, b_post=b_post, gate=gate, w_pre=w_pre, b_pre=b_pre, epsilon=1e-5, scale=0.5)
    out = B.shampoo_residual_norm_forward(r, f, checkpoint=packed, **kw)
    want = B.shampoo_residual_norm_backward(*(out[2:] if packed else (r, f)), dr_out, dh, **kw)
    c = B.ResidualNorm(n, d, code(dt), B.NORM_LAYER, B.NORM_LAYER, gates, 1e-5, 0.5, w_post.data_ptr(), b_post.data_ptr(), gate.data_ptr() if gates else None,
                       w_pre.data_ptr(), b_pre.data_ptr())
    size = L.shampoo_checkpoint_bytes(n, d)
    memory = [torch.full((size + 512,), 77, dtype=torch.uint8, device="cuda") for _ in range(2)] if packed else None
    r2, f2, h2 = Rows(n, d, dt, values=r), Rows(n, d, dt, gap=9, values=f), Rows(n, d, dt, gap=1)
    done(L.shampoo_residual_norm_forward(ctypes.byref(c), r2.p(), r2.ld, f2.p(), f2.ld, r2.p(), r2.ld, h2.p(), h2.ld,
                                         *((m.data_ptr() for m in memory) if packed else (None, None)), size, stream()))
    r2.check(out[0])
    h2.check(out[1])
    if packed:
        for m, have in zip(memory, out[2:]):
            again = B.Checkpoint(m[:size], (n, d), code(dt))
            assert torch.equal(B.shampoo_checkpoint_unpack(again), B.shampoo_checkpoint_unpack(have)) and bool((m[size:] == 77).all())
    r2.view.copy_(r)
    a2, b2 = Rows(n, d, dt, values=dr_out), Rows(n, d, dt, gap=2, values=dh)
    sums = {k: Rows(gates if k == "dgate" else 1, d, torch.float32, gap=0) for k in ("dgate", "dw_post", "db_post", "dw_pre", "db_pre")}
    need = L.shampoo_residual_norm_backward_workspace_bytes(ctypes.byref(c))
    ws = torch.full((need + 4096,), 255, dtype=torch.uint8, device="cuda")       # NaN, whatever is read of it
    rf = [(m.data_ptr(), 0) for m in memory] if packed else [(r2.p(), r2.ld), (f2.p(), f2.ld)]
    done(L.shampoo_residual_norm_backward(ctypes.byref(c), int(packed), *rf[0], *rf[1], a2.p(), a2.ld, b2.p(), b2.ld, a2.p(), a2.ld, b2.p(), b2.ld,
                                          *(sums[k].p() if gates or k != "dgate" else None for k in sums), ws.data_ptr(), need, stream()))
    assert bool((ws[need:] == 255).all())
    a2.check(want["dr"])
    b2.check(want["df"])
    r2.check(r)
    f2.check(f)
    for k, s in sums.items():
        if want[k] is not None:
            s.check(want[k].view(-1, d))
