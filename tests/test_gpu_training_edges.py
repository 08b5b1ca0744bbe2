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
