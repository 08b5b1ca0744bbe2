"""The operators of a training pass against their definitions in float64: the loss over many classes with its gradients, 8-bit
checkpoints with what reads them, residual norms in both directions.

Bars, all relative to the norm of the result unless said otherwise, u = 2^-8 the rounding of bf16 (8 significant bits), e = 2^-24 that of float32:
  loss             an absolute 2^-23 (sqrt(features) + 16) max|z|: float32 sums of `features` exact products, exp and log behind them
  bf16 gradients   3 u of the norm: up to two roundings of g and one of the result (independent ones add up to less)
  float32 dw from bf16 x   2^-15: g in two bf16 terms (2^-17), its exponent off by the error of z (|z| < 64: 2^-18)
  float32          2^-16: the exponent of g again, and sums of up to 2^13 float32 terms; db as dw
  checkpoints      codes exactly; what is computed from them u (bf16) or 2^-20 (float32: erf, exp and a product of a few 2^-23)
  norms            bf16 u, float32 and sums over rows 2^-18 (float32 sums of up to 2^14 terms, in pieces)
A bf16 result adds u / 2 of the largest element where a single one is compared."""
import math

import pytest

from paper_2309_06497_amd import binding as B

pytestmark = pytest.mark.gpu
U = 2.0 ** -8


def torch_():
    import torch
    return torch


def gen(seed):
    g = torch_().Generator(device="cuda")
    g.manual_seed(seed)
    return g


def normal(g, *shape, sigma=1.0):
    torch = torch_()
    return torch.randn(shape, generator=g, device="cuda") * sigma


def rel(got, want):
    torch = torch_()
    d = torch.linalg.vector_norm(got.double() - want)
    n = torch.linalg.vector_norm(want)
    return float(d / n) if float(n) > 0 else float(d)


def strided(x, how):
    """The same values as a view: rows further apart, or off any alignment"""
    torch = torch_()
    if how == "dense":
        return x
    if how == "rows":
        big = torch.full((x.shape[0] + 2, x.shape[1] + 24), float("nan"), dtype=x.dtype, device=x.device)
        view = big[1:1 + x.shape[0], 8:8 + x.shape[1]]
    else:
        flat = torch.full((x.numel() + x.shape[0] + 3,), float("nan"), dtype=x.dtype, device=x.device)
        view = flat[1:1 + x.shape[0] * (x.shape[1] + 1)].view(x.shape[0], x.shape[1] + 1)[:, :x.shape[1]]
    view.copy_(x)
    return view


# ----------------------------------------------------------------------------
# Cross entropy
# ----------------------------------------------------------------------------
def head_reference(x, w, t, bias, weight, scale):
    torch = torch_()
    x, w = x.double(), w.double()
    z = x @ w.t()
    if bias is not None:
        z = z + bias.double()
    n, v = z.shape
    valid = (t >= 0) & (t < v)
    i = torch.arange(n, device=t.device)[valid]
    lse = torch.logsumexp(z, 1)
    loss = torch.zeros(n, dtype=torch.float64, device=t.device)
    loss[i] = lse[i] - z[i, t[i]]
    loss[i[z[i, t[i]] == -math.inf]] = math.inf
    g = torch.zeros_like(z)
    c = (weight.double() if weight is not None else torch.ones(n, dtype=torch.float64, device=t.device)) * scale
    g[i] = torch.exp(z[i] - lse[i, None])
    g[i, t[i]] -= 1.0
    g[lse == -math.inf] = 0.0
    g *= torch.where(valid, c, torch.zeros_like(c))[:, None]
    finite = z[torch.isfinite(z)]
    largest = float(finite.abs().max()) if finite.numel() else 0.0
    return loss, g @ w, g.t() @ x, g.sum(0), largest


def check_head(out, want, d, bf16, grad_f32):
    torch = torch_()
    loss, dx, dw, db = out
    l64, dx64, dw64, db64, largest = want
    fin = torch.isfinite(l64)
    assert torch.equal(loss[~fin].double(), l64[~fin])
    assert float((loss[fin].double() - l64[fin]).abs().max() if fin.any() else 0.0) <= 2.0 ** -23 * (math.sqrt(d) + 16) * max(largest, 1.0)
    floor = 2.0 ** -40        # all gradients zero
    assert rel(dx, dx64) <= (3 * U if bf16 else 2.0 ** -16) + (floor if not dx64.any() else 0)
    assert rel(dw, dw64) <= (2.0 ** -15 if bf16 and grad_f32 else 3 * U if bf16 else 2.0 ** -16)
    if db is not None:
        assert rel(db, db64) <= 2.0 ** -15


# up to 192, 640 or 96 features (by type) the logits are made twice; many splits of the product for dx: few rows and features, many classes
SIZES = [(2, 66, 20001), (129, 704, 300), (1, 1, 1), (1, 8, 2), (2, 3, 5), (3, 64, 64), (65, 40, 129), (130, 200, 257), (255, 1000, 1003), (64, 96, 4099), (300, 72, 10)]
KINDS = [("bf16", "bf16"), ("bf16", "f32"), ("f32", "f32")]


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("in_out", [False, True])
@pytest.mark.parametrize("bias", [False, True])
@pytest.mark.parametrize("n,d,v", SIZES)
def test_head_and_its_gradients(n, d, v, bias, in_out, kind):
    torch = torch_()
    g = gen(1000 * n + v)
    types = {"bf16": torch.bfloat16, "f32": torch.float32}
    dt = types[kind[0]]
    x, w = normal(g, n, d).to(dt), normal(g, v, d, sigma=2 / math.sqrt(d)).to(dt)
    t = torch.randint(-1, v + 1, (n,), generator=g, device="cuda")       # -1 and v: ignored
    b = normal(g, v) if bias else None
    weight = torch.rand((n,), generator=g, device="cuda") + 0.5 if n % 2 else None
    want = head_reference(x, w, t, b, weight, 1.0 / n)
    wv = w.t().contiguous().t() if in_out else w
    out = B.shampoo_linear_cross_entropy(x, wv, t, bias=b, weight=weight, scale=1.0 / n, grad_dtype=types[kind[1]])
    assert out[1].dtype == dt and out[2].dtype == types[kind[1]] and tuple(out[2].shape) == (v, d)
    check_head(out, want, d, kind[0] == "bf16", kind[1] == "f32")
    loss = B.shampoo_linear_cross_entropy(x, wv, t, bias=b, gradients=False)
    assert torch.allclose(loss, out[0], rtol=1e-5, atol=1e-5)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("in_out", [False, True])
@pytest.mark.parametrize("n,d,v", [(200, 300, 8000), (17, 2048, 1500), (520, 1000, 4001)])
def test_head_whose_gradients_share_a_launch_of_more_workgroups_than_cus(n, d, v, in_out, kind):
    test_head_and_its_gradients(n, d, v, True, in_out, kind)


@pytest.mark.parametrize("d", [64, 256])
@pytest.mark.parametrize("bias", [False, True])
@pytest.mark.parametrize("scale", [1.0 / 255, 1.0 / 509, -3.02, 1.0])
def test_head_gradients_in_bf16_are_not_scaled_as_a_whole(scale, bias, d):
    """Against the definition's gradients rounded once (one product of a bf16 x and the scale is many a dw's only term, so that roundings
    of the result all go one way): roundings of single elements of g average out in <got, want> / <want, want> (over 255 d of them, and
    more); one of the scale, which every row shares, would not: 2^-11, of which 2^-13 is the largest probability, which 1 - p may lose."""
    torch = torch_()
    g = gen(31)
    n, v = 255, 20000
    x, w = normal(g, n, d, sigma=0.1).bfloat16(), normal(g, v, d, sigma=0.1).bfloat16()
    t = torch.randint(0, v, (n,), generator=g, device="cuda")
    b = normal(g, v, sigma=0.01) if bias else None
    out = B.shampoo_linear_cross_entropy(x, w, t, bias=b, scale=scale)
    want = head_reference(x, w, t, b, None, scale)
    want = [want[0], want[1].bfloat16().double(), want[2].bfloat16().double(), want[3]]
    for k in (1, 2) + ((3,) if bias else ()):
        dot = float((out[k].double() * want[k]).sum() / (want[k] * want[k]).sum())
        assert abs(dot - 1.0) <= 2.0 ** -11
    none = B.shampoo_linear_cross_entropy(x, w, t, bias=b, scale=0.0)
    assert not none[1].any() and not none[2].any()
    tiny = B.shampoo_linear_cross_entropy(x, w, t, bias=b, scale=1.7e-38, grad_dtype=torch.float32)
    assert torch.isfinite(tiny[2]).all() and torch.isfinite(tiny[1].float()).all()


@pytest.mark.parametrize("how", ["rows", "odd"])
@pytest.mark.parametrize("dt", ["bf16", "f32"])
def test_head_on_strided_views(how, dt):
    torch = torch_()
    g = gen(7)
    dt = torch.bfloat16 if dt == "bf16" else torch.float32
    n, d, v = 100, 136, 520
    x, w = normal(g, n, d).to(dt), normal(g, v, d, sigma=0.2).to(dt)
    t = torch.randint(0, v, (n,), generator=g, device="cuda")
    want = head_reference(x, w, t, None, None, 1.0)
    for wv in (strided(w, how), strided(w.t().contiguous(), how).t()):
        out = B.shampoo_linear_cross_entropy(strided(x, how), wv, t)
        check_head(out, want, d, dt == torch.bfloat16, dt == torch.float32)


def test_head_with_masked_classes_and_rows_that_are_not_finite():
    torch = torch_()
    g = gen(8)
    n, d, v = 70, 64, 300
    x, w = normal(g, n, d), normal(g, v, d, sigma=0.2)
    t = torch.randint(0, v, (n,), generator=g, device="cuda")
    bias = normal(g, v)
    bias[100:] = -math.inf                       # masked classes, some of them targets
    for dt in (torch.bfloat16, torch.float32):
        xs, ws = x.to(dt), w.to(dt)
        out = B.shampoo_linear_cross_entropy(xs, ws, t, bias=bias)
        want = head_reference(xs, ws, t, bias, None, 1.0)
        assert bool((out[0][t >= 100] == math.inf).all())
        check_head(out, want, d, dt == torch.bfloat16, dt == torch.float32)
        assert torch.isfinite(out[1]).all() and torch.isfinite(out[2]).all()
        # nothing left: no gradient
        out = B.shampoo_linear_cross_entropy(xs, ws, t, bias=torch.full_like(bias, -math.inf))
        assert bool((out[0] == math.inf).all()) and not out[1].any() and not out[2].any() and not out[3].any()
        # the lowest finite value instead of -infinity: the same probabilities
        low = torch.where(torch.isinf(bias), torch.full_like(bias, torch.finfo(torch.float32).min), bias)
        ref = B.shampoo_linear_cross_entropy(xs, ws, t.clamp(max=99), bias=bias)
        out = B.shampoo_linear_cross_entropy(xs, ws, t.clamp(max=99), bias=low)
        assert all(torch.equal(a, b) for a, b in zip(out, ref))
        # an ignored row that is not finite: its own outputs are zero; a counted one is NaN, and only there
        bad = xs.clone()
        bad[5] = math.nan
        ti = t.clamp(max=99)
        ti[5] = -100
        out = B.shampoo_linear_cross_entropy(bad, ws, ti, bias=bias)
        assert float(out[0][5]) == 0.0 and not out[1][5].any() and torch.isfinite(out[0]).all() and torch.isfinite(out[1]).all()
        ti[5] = 3
        out = B.shampoo_linear_cross_entropy(bad, ws, ti, bias=bias)
        assert bool(torch.isnan(out[0][5])) and bool(torch.isnan(out[1][5]).all())
        rest = torch.arange(n, device="cuda") != 5
        assert torch.isfinite(out[0][rest]).all() and torch.isfinite(out[1][rest]).all()


def test_head_where_every_class_is_masked_by_the_lowest_value():
    """The softmax of equal logits, however low: 1 / classes each (z + lowest is lowest: nothing of z is left)."""
    torch = torch_()
    g = gen(12)
    for n, d, v in ((40, 64, 300), (200, 1024, 300), (600, 64, 16500)):          # one product, several splits, large tiles
        for dt in (torch.bfloat16, torch.float32):
            x, w = normal(g, n, d).to(dt), normal(g, v, d, sigma=0.1).to(dt)
            t = torch.randint(0, v, (n,), generator=g, device="cuda")
            low = torch.full((v,), torch.finfo(torch.float32).min, device="cuda")
            loss, dx, dw, db = B.shampoo_linear_cross_entropy(x, w, t, bias=low)
            # lse = lowest + log(classes) rounds to lowest, and so does z: the loss is what float32 leaves, 0
            assert not loss.any() and torch.isfinite(dx).all() and torch.isfinite(dw).all() and torch.isfinite(db).all()


def test_head_whose_logits_span_the_whole_range():
    """Differences beyond 64 powers of two, and beyond float32's exponents, next to ordinary ones."""
    torch = torch_()
    g = gen(13)
    for n, d, v in ((40, 64, 300), (600, 64, 16500)):
        x, w = normal(g, n, d, sigma=3.0).bfloat16(), normal(g, v, d, sigma=3.0).bfloat16()
        t = torch.randint(0, v, (n,), generator=g, device="cuda")
        want = head_reference(x, w, t, None, None, 1.0)
        out = B.shampoo_linear_cross_entropy(x, w, t)
        check_head(out, want, d, True, False)


def test_head_of_large_logits_does_not_overflow():
    torch = torch_()
    g = gen(9)
    x, w = normal(g, 33, 64, sigma=30.0).bfloat16(), normal(g, 777, 64, sigma=30.0).bfloat16()
    t = torch.randint(0, 777, (33,), generator=g, device="cuda")
    want = head_reference(x, w, t, None, None, 1.0)
    out = B.shampoo_linear_cross_entropy(x, w, t)
    assert all(torch.isfinite(o).all() for o in out[:3])
    # |z| is in the thousands: the exponents are off by 2^-24 of that
    assert float((out[0].double() - want[0]).abs().max()) <= 2.0 ** -23 * 24 * want[4]
    assert rel(out[1], want[1]) <= 3 * U and rel(out[2], want[2]) <= 3 * U


def test_head_gradient_against_differences():
    torch = torch_()
    g = gen(10)
    n, d, v = 20, 24, 50
    x, w, b = normal(g, n, d), normal(g, v, d, sigma=0.4), normal(g, v)
    t = torch.randint(0, v, (n,), generator=g, device="cuda")
    weight = torch.rand((n,), generator=g, device="cuda")
    _, dx, dw, db = B.shampoo_linear_cross_entropy(x, w, t, bias=b, weight=weight, scale=0.3)

    def value(x, w, b):
        z = x @ w.t() + b
        return float((0.3 * weight.double() * (torch.logsumexp(z, 1) - z.gather(1, t[:, None])[:, 0])).sum())

    at = [x.double(), w.double(), b.double()]
    for k, grad in enumerate((dx, dw, db)):
        v_ = normal(g, *at[k].shape).double()
        h = 1e-5                                   # differences of second order: h^2 = 1e-10
        up, down = list(at), list(at)
        up[k], down[k] = at[k] + h * v_, at[k] - h * v_
        slope = (value(*up) - value(*down)) / (2 * h)
        assert abs(float((grad.double() * v_).sum()) - slope) <= 1e-5 * (1 + abs(slope))


def test_head_in_several_pieces_of_rows():
    """4 GiB of logits: 256 rows of 4194304 classes are a piece by themselves, 300 rows two."""
    torch = torch_()
    g = gen(11)
    n, d, v = 300, 8, 4194304
    x, w = normal(g, n, d).bfloat16(), normal(g, v, d).bfloat16()
    t = torch.randint(0, v, (n,), generator=g, device="cuda")
    z = x.double() @ w.double().t()
    lse = torch.logsumexp(z, 1)
    i = torch.arange(n, device="cuda")
    want_loss, largest = lse - z[i, t], float(z.abs().max())
    p = z.sub_(lse[:, None]).exp_()
    p[i, t] -= 1.0
    dx64, dw64 = p @ w.double(), p.t() @ x.double()
    for grad in (torch.bfloat16, torch.float32):
        loss, dx, dw, _ = B.shampoo_linear_cross_entropy(x, w, t, grad_dtype=grad)
        assert float((loss.double() - want_loss).abs().max()) <= 2.0 ** -23 * (math.sqrt(d) + 16) * largest
        assert rel(dx, dx64) <= 3 * U and rel(dw, dw64) <= (3 * U if grad == torch.bfloat16 else 2.0 ** -15)


def test_head_without_rows():
    torch = torch_()
    x, w, t = torch.empty((0, 16), device="cuda"), torch.ones((9, 16), device="cuda"), torch.empty((0,), dtype=torch.int64, device="cuda")
    loss, dx, dw, db = B.shampoo_linear_cross_entropy(x, w, t, bias=torch.ones(9, device="cuda"))
    assert loss.numel() == 0 and dx.numel() == 0 and not dw.any() and not db.any()


# ----------------------------------------------------------------------------
# Checkpoints
# ----------------------------------------------------------------------------
def held(x):
    """What a checkpoint holds of x, from the definition, in float64"""
    torch = torch_()
    n, d = x.shape
    v = torch.nn.functional.pad(x.double(), (0, -d % 32)).view(n, -1, 32)
    largest = v.abs().amax(2, keepdim=True)
    s = torch.full_like(largest, -120.0)
    step = torch.ones_like(largest)
    for k in (128.0, 64.0, 32.0, 16.0, 8.0, 4.0, 2.0, 1.0):    # the largest s + 1 for which the code is above 127, bit by bit
        up = torch.round(largest * torch.exp2(-(s + k - 1))) > 127
        s = torch.where(up, s + k, s)
    q = torch.round(v * torch.exp2(-s)) * torch.exp2(s)
    q = torch.where(largest < 2.0 ** -100, torch.zeros_like(q), q)
    return torch.where(torch.isfinite(largest), q, torch.full_like(q, math.nan)).view(n, -1)[:, :d]


def activations(g, n, d):
    size = normal(g, d).mul(0.5).exp()
    return normal(g, n, d) * size


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("how", ["dense", "rows", "odd"])
@pytest.mark.parametrize("n,d", [(1, 1), (3, 31), (5, 32), (7, 33), (64, 1000), (130, 2049)])
def test_checkpoint_holds_what_it_should(n, d, how, dt):
    torch = torch_()
    dt = torch.bfloat16 if dt == "bf16" else torch.float32
    x = activations(gen(n + d), n, d).to(dt)
    if n > 2:
        x[1] = 0.0
        x[2] *= 2.0 ** -60
        x[0, ::3] = 1.9921875 * torch.sign(x[0, ::3])           # 127.5 steps: the next exponent
    c = B.shampoo_checkpoint_pack(strided(x, how))
    assert c.packed.numel() <= 256 + 256 + n * (-(-d // 32)) * 33
    want = held(x)
    assert torch.equal(B.shampoo_checkpoint_unpack(c, dtype=torch.float32).double(), want)
    assert torch.equal(B.shampoo_checkpoint_unpack(c, dtype=torch.bfloat16).double(), want)
    # half a step, where the largest is at least 63.75 steps
    assert float((want - x.double()).abs().max()) <= float(x.double().abs().max()) / 127.5


def test_checkpoint_of_extreme_groups():
    torch = torch_()
    x = torch.zeros((9, 64), device="cuda")
    x[0, 3] = math.inf
    x[1, 40] = math.nan
    x[2, 0], x[2, 1] = 3.0e38, -1.0
    x[3, 0] = 2.0 ** -100
    x[4, 0] = 2.0 ** -100 * 0.999
    x[5, 0] = 1e-45
    x[6, 0], x[6, 1] = 1.0, 1e-3
    x[7, 5], x[8, 5] = 255 * 2.0 ** 120, -255 * 2.0 ** 119
    y = B.shampoo_checkpoint_unpack(B.shampoo_checkpoint_pack(x))
    assert torch.isnan(y[0, :32]).all() and not y[0, 32:].any()
    assert torch.isnan(y[1, 32:]).all() and not y[1, :32].any()
    assert torch.isnan(y[7, :32]).all() and torch.isfinite(y[8]).all()
    ok = [2, 3, 4, 5, 6, 8]
    assert torch.equal(y[ok].double(), held(x[ok]))
    assert float(y[3, 0]) == 2.0 ** -100 and not y[4].any() and not y[5].any()


def activation(z, kind):
    """a and a' in float64"""
    torch = torch_()
    if kind == B.ACT_RELU:
        return z.clamp(min=0), (z > 0).double()
    if kind == B.ACT_SILU:
        s = torch.sigmoid(z)
        return z * s, s * (1 + z * (1 - s))
    if kind == B.ACT_GELU:
        phi = 0.5 * torch.special.erfc(-z / math.sqrt(2))
        return z * phi, phi + z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi)
    return z, torch.ones_like(z)


@pytest.mark.parametrize("kind", [B.ACT_NONE, B.ACT_RELU, B.ACT_GELU, B.ACT_SILU])
@pytest.mark.parametrize("n,d,how", [(1, 1, "dense"), (33, 70, "odd"), (64, 256, "rows"), (100, 1001, "dense")])
def test_activations_and_their_gradients_from_a_checkpoint(n, d, how, kind):
    torch = torch_()
    g = gen(n)
    x = activations(g, n, d) * 2
    x[0, 0] = 90.0                                              # exp overflows beyond
    c = B.shampoo_checkpoint_pack(x)
    a, slope = activation(held(x), kind)
    for dt, bar in ((torch.float32, 2.0 ** -20), (torch.bfloat16, U)):
        dy = strided(normal(g, n, d).to(dt), how)
        assert rel(B.shampoo_checkpoint_unpack(c, kind, dt), a) <= bar
        assert rel(B.shampoo_checkpoint_activation_grad(c, dy, kind), dy.double() * slope) <= bar


def test_activation_gradient_against_differences():
    torch = torch_()
    g = gen(5)
    x = activations(g, 8, 64)
    c = B.shampoo_checkpoint_pack(x)
    z = held(x)
    for kind in (B.ACT_GELU, B.ACT_SILU):
        h = 1e-5
        slope = (activation(z + h, kind)[0] - activation(z - h, kind)[0]) / (2 * h)
        got = B.shampoo_checkpoint_activation_grad(c, torch.ones_like(x), kind)
        assert float((got.double() - slope).abs().max()) <= 1e-6


@pytest.mark.parametrize("kinds", KINDS)
@pytest.mark.parametrize("out_in", [False, True])
@pytest.mark.parametrize("act", [B.ACT_NONE, B.ACT_GELU])
@pytest.mark.parametrize("n,i,o,how", [(1, 1, 1, "dense"), (1, 40, 9, "dense"), (70, 33, 65, "odd"), (257, 256, 128, "rows"), (999, 130, 331, "dense"), (2000, 264, 72, "rows")])
def test_weight_gradient_from_a_checkpoint(n, i, o, how, act, out_in, kinds):
    torch = torch_()
    types = {"bf16": torch.bfloat16, "f32": torch.float32}
    g = gen(n + i + o)
    x, dy = activations(g, n, i).to(types[kinds[0]]), normal(g, n, o, sigma=1e-3).to(types[kinds[0]])
    c = B.shampoo_checkpoint_pack(x)
    a = activation(held(x), act)[0]
    want = a.t() @ dy.double()
    dw, db = B.shampoo_checkpoint_weight_grad(c, strided(dy, how), act, types[kinds[1]], out_in, True)
    # exact operands but for a(x): bf16 result u, and u for a(x); float32 result 2^-17 for a(x) and sums of 2^11 terms
    bar = (U if act == B.ACT_NONE else 2 * U) if kinds[1] == "bf16" else 2.0 ** -16 if kinds[0] == "bf16" and act != B.ACT_NONE else 2.0 ** -18
    assert dw.dtype == types[kinds[1]]
    assert rel(dw, want.t() if out_in else want) <= bar
    assert rel(db, dy.double().sum(0)) <= 2.0 ** -18


@pytest.mark.parametrize("out_in", [False, True])
def test_weight_gradient_whose_last_round_of_tiles_is_split(out_in):
    """4 x 67 tiles of 256: 256 of them, and twelve that are split along the tokens."""
    torch = torch_()
    g = gen(21)
    n, i, o = 2500, 1000, 17000
    for dt, grad, bar in ((torch.bfloat16, torch.bfloat16, U), (torch.bfloat16, torch.float32, 2.0 ** -18), (torch.float32, torch.float32, 2.0 ** -18)):
        x, dy = activations(g, n, i).to(dt), normal(g, n, o).to(dt)
        c = B.shampoo_checkpoint_pack(x)
        want = held(x).t() @ dy.double()
        got = B.shampoo_checkpoint_weight_grad(c, dy, grad_dtype=grad, out_in=out_in)
        got = got.t() if out_in else got
        assert rel(got, want) <= bar
        # each tile of the last round by itself, and the one before
        for k in range(o - 13 * 256, o, 128):
            assert rel(got[:, k:k + 128], want[:, k:k + 128]) <= 2 * bar
        for k in range(0, i, 128):
            assert rel(got[k:k + 128, -3000:], want[k:k + 128, -3000:]) <= 2 * bar


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("n,i,o", [(1, 40, 9), (257, 256, 128), (999, 130, 331)])
def test_weight_gradient_of_relu_is_exact_up_to_sums(n, i, o, dt):
    """relu(x) of a checkpoint is a bf16 value: as without an activation, nothing but float32 sums of n terms."""
    torch = torch_()
    g = gen(n + 7)
    dt = torch.bfloat16 if dt == "bf16" else torch.float32
    x, dy = activations(g, n, i).to(dt), normal(g, n, o).to(dt)
    c = B.shampoo_checkpoint_pack(x)
    want = held(x).clamp_min(0.0).t() @ dy.double()
    assert rel(B.shampoo_checkpoint_weight_grad(c, dy, B.ACT_RELU, torch.float32), want) <= 2.0 ** -18


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("n,i,o", [(64, 40, 63), (128, 40, 64), (129, 200, 65), (192, 40, 300), (1000, 8, 1), (16385, 40, 130), (20001, 33, 7)])
def test_bias_gradients_by_parts_of_the_rows(n, i, o, dt):
    """Every column by itself: a term goes through less than 40 float32 additions, so 40 e of the sum of |dy|."""
    torch = torch_()
    g = gen(n + o)
    dt = torch.bfloat16 if dt == "bf16" else torch.float32
    x, dy = activations(g, n, i).to(dt), normal(g, n, o).to(dt)
    dy[:, ::3] += 1.0
    c = B.shampoo_checkpoint_pack(x)
    for grad in {dt, torch.float32}:
        dw, db = B.shampoo_checkpoint_weight_grad(c, dy, grad_dtype=grad, bias=True)
        assert ((db.double() - dy.double().sum(0)).abs() <= 40 * 2.0 ** -24 * dy.double().abs().sum(0)).all()
        alone = B.shampoo_checkpoint_weight_grad(c, dy, grad_dtype=grad)
        assert torch.equal(dw, alone)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("in_out", [False, True])
@pytest.mark.parametrize("n,d,v", [(40, 300, 1100), (250, 520, 700), (32, 2048, 1000), (700, 1100, 900)])
def test_head_whose_small_gradients_share_a_launch(n, d, v, in_out, kind):
    test_head_and_its_gradients(n, d, v, True, in_out, kind)
    test_head_and_its_gradients(n, d, v, False, in_out, kind)


def test_weight_gradient_in_several_pieces_of_rows():
    torch = torch_()
    g = gen(3)
    n, i, o = 70000, 8192, 24                      # 1 GiB of bf16 activations: 65536 rows of 8192
    x, dy = activations(g, n, i).bfloat16(), normal(g, n, o).bfloat16()
    c = B.shampoo_checkpoint_pack(x)
    want = torch.zeros((i, o), dtype=torch.float64, device="cuda")
    for k in range(0, n, 10000):
        want += B.shampoo_checkpoint_unpack(c, dtype=torch.float32)[k:k + 10000].double().t() @ dy[k:k + 10000].double()
    assert rel(B.shampoo_checkpoint_weight_grad(c, dy), want) <= U
    assert rel(B.shampoo_checkpoint_weight_grad(c, dy, grad_dtype=torch.float32), want) <= 2.0 ** -18


def test_checkpoints_without_rows():
    torch = torch_()
    c = B.shampoo_checkpoint_pack(torch.empty((0, 40), device="cuda"))
    assert B.shampoo_checkpoint_unpack(c).shape == (0, 40)
    assert B.shampoo_checkpoint_activation_grad(c, torch.empty((0, 40), device="cuda"), B.ACT_SILU).shape == (0, 40)
    dw, db = B.shampoo_checkpoint_weight_grad(c, torch.empty((0, 9), device="cuda"), bias=True)
    assert tuple(dw.shape) == (40, 9) and not dw.any() and not db.any()


# ----------------------------------------------------------------------------
# Residual norms
# ----------------------------------------------------------------------------
EPS = 1e-5
NORMS = [(B.NORM_RMS, B.NORM_RMS), (B.NORM_NONE, B.NORM_LAYER), (B.NORM_LAYER, B.NORM_LAYER), (B.NORM_RMS, B.NORM_NONE), (B.NORM_NONE, B.NORM_NONE)]


def norm64(x, kind, w, b):
    torch = torch_()
    if kind == B.NORM_NONE:
        return x
    if kind == B.NORM_LAYER:
        x = x - x.mean(1, keepdim=True)
    y = x / torch.sqrt(x.square().mean(1, keepdim=True) + EPS) * w
    return y + b if b is not None else y


def sandwich64(r, f, post, pre, p, scale):
    torch = torch_()
    u = norm64(f, post, p.get("w_post"), p.get("b_post"))
    if "gate" in p:
        u = (u.view(p["gate"].shape[0], -1, u.shape[1]) * p["gate"][:, None]).reshape(u.shape)
    r_out = r + scale * u
    return r_out, norm64(r_out, pre, p.get("w_pre"), p.get("b_pre")) if pre != B.NORM_NONE else None


def norm_parameters(g, d, post, pre, gates, biases=True):
    p = {}
    if gates:
        p["gate"] = normal(g, gates, d, sigma=0.5)
    for side, kind in (("post", post), ("pre", pre)):
        if kind != B.NORM_NONE:
            p["w_" + side] = 1 + 0.1 * normal(g, d)
        if kind == B.NORM_LAYER and biases:
            p["b_" + side] = 0.1 * normal(g, d)
    return p


def check_norm(n, d, dt, post, pre, gates, checkpoint, how="dense", biases=True, seed=0):
    torch = torch_()
    g = gen(n + d + seed)
    r, f = (normal(g, n, d) * normal(g, d).mul(0.5).exp() + 0.5).to(dt), normal(g, n, d, sigma=0.7).to(dt)
    dr_out, dh = normal(g, n, d).to(dt), normal(g, n, d).to(dt)
    p = norm_parameters(g, d, post, pre, gates, biases)
    kw = dict(post=post, pre=pre, epsilon=EPS, scale=0.5, **p)
    bar = U if dt == torch.bfloat16 else 2.0 ** -18
    rs, fs = strided(r, how), strided(f, how)
    out = B.shampoo_residual_norm_forward(rs, fs, checkpoint=checkpoint, **kw)
    p64 = {k: v.double() for k, v in p.items()}
    r_out, h = sandwich64(r.double(), f.double(), post, pre, p64, 0.5)
    assert rel(out[0], r_out) <= bar
    if pre == B.NORM_NONE:
        assert out[1] is None
    elif d > 1 or pre == B.NORM_RMS:
        assert rel(out[1], h) <= bar
    if checkpoint:
        r64, f64 = held(r), held(f)
        assert torch.equal(B.shampoo_checkpoint_unpack(out[2], dtype=torch.float32).double(), r64)
        assert torch.equal(B.shampoo_checkpoint_unpack(out[3], dtype=torch.float32).double(), f64)
    else:
        r64, f64 = r.double(), f.double()
    got = B.shampoo_residual_norm_backward(out[2] if checkpoint else rs, out[3] if checkpoint else fs, strided(dr_out, how),
                                           strided(dh, how) if pre != B.NORM_NONE else None, **kw)
    leaves = {"r": r64.requires_grad_(), "f": f64.requires_grad_(), **{k: v.requires_grad_() for k, v in p64.items()}}
    r_out, h = sandwich64(leaves["r"], leaves["f"], post, pre, p64, 0.5)
    value = (r_out * dr_out.double()).sum() + ((h * dh.double()).sum() if h is not None else 0)
    want = dict(zip(leaves, torch.autograd.grad(value, list(leaves.values()))))
    for k, w in want.items():
        e = got["d" + k]
        assert e is not None and tuple(e.shape) == tuple(w.shape), k
        if float(torch.linalg.vector_norm(w)) < 1e-12:                      # one feature: the norm leaves nothing
            assert float(e.abs().max()) <= 1e-2
            continue
        assert rel(e, w) <= (bar if k in ("r", "f") else 2.0 ** -18), (k, rel(e, w))
    for k in ("gate", "w_post", "b_post", "w_pre", "b_pre"):
        assert k in want or got["d" + k] is None


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("post,pre", NORMS)
@pytest.mark.parametrize("n,d,gates,checkpoint", [
    (1, 40, 1, False), (5, 7, 0, False), (6, 33, 3, True), (64, 512, 1, True), (12, 520, 12, False), (33, 1000, 1, True),
    (40, 1024, 2, False), (300, 2048, 1, True), (20, 2049, 4, True), (9, 4100, 0, False), (6, 8200, 1, True), (5, 16384, 5, False)])
def test_residual_norm_forward_and_backward(n, d, gates, checkpoint, post, pre, dt):
    check_norm(n, d, torch_().bfloat16 if dt == "bf16" else torch_().float32, post, pre, gates, checkpoint)


@pytest.mark.parametrize("how", ["rows", "odd"])
def test_residual_norm_on_strided_views(how):
    torch = torch_()
    for dt in (torch.bfloat16, torch.float32):
        check_norm(50, 264, dt, B.NORM_RMS, B.NORM_LAYER, 5, False, how)
        check_norm(50, 264, dt, B.NORM_RMS, B.NORM_LAYER, 5, True, how, biases=False)


def test_residual_norm_with_more_gates_than_workgroups():
    torch = torch_()
    check_norm(3 * 2500, 64, torch.float32, B.NORM_RMS, B.NORM_RMS, 2500, True)
    check_norm(2500, 72, torch.bfloat16, B.NORM_NONE, B.NORM_RMS, 2500, False)


def test_residual_norm_of_many_rows():
    torch = torch_()
    check_norm(5000, 320, torch.float32, B.NORM_LAYER, B.NORM_RMS, 1, True)


def test_residual_norm_extremes():
    torch = torch_()
    w = torch.ones(64, device="cuda")
    r, f = torch.zeros((4, 64), device="cuda"), torch.zeros((4, 64), device="cuda")
    r[1], f[1] = 1e15, 1e15                       # squares of 1e30 stay in range
    r[2, 3], f[3, 5] = math.nan, math.inf
    r_out, h, r8, f8 = B.shampoo_residual_norm_forward(r, f, w_post=w, w_pre=w, checkpoint=True)
    assert not r_out[0].any() and not h[0].any()
    assert torch.isfinite(h[1]).all() and torch.isnan(h[2]).all() and torch.isnan(h[3]).all()
    g = B.shampoo_residual_norm_backward(r8, f8, torch.ones_like(r), torch.ones_like(r), w_post=w, w_pre=w)
    assert torch.isfinite(g["dr"][:2]).all() and torch.isfinite(g["df"][:2]).all()
    assert torch.isnan(g["dr"][2]).all() and torch.isnan(g["df"][3]).all()
    assert B.shampoo_residual_norm_forward(r[:0], f[:0], w_post=w, w_pre=w)[0].shape == (0, 64)
    g = B.shampoo_residual_norm_backward(r[:0], f[:0], r[:0], r[:0], w_post=w, w_pre=w)
    assert not g["dw_post"].any() and not g["dw_pre"].any()


def test_residual_norm_gradient_against_differences():
    torch = torch_()
    g = gen(77)
    n, d = 6, 40
    r, f, a, b = (normal(g, n, d) for _ in range(4))
    p = norm_parameters(g, d, B.NORM_LAYER, B.NORM_RMS, 2)
    kw = dict(post=B.NORM_LAYER, pre=B.NORM_RMS, epsilon=EPS, scale=0.7, **p)
    got = B.shampoo_residual_norm_backward(r, f, a, b, **kw)
    at = {"r": r.double(), "f": f.double(), **{k: v.double() for k, v in p.items()}}

    def value(at):
        q = {k: v for k, v in at.items() if k not in "rf"}
        r_out, h = sandwich64(at["r"], at["f"], B.NORM_LAYER, B.NORM_RMS, q, 0.7)
        return float((r_out * a.double()).sum() + (h * b.double()).sum())

    for k in at:
        v, s = normal(g, *at[k].shape).double(), 1e-5
        slope = (value({**at, k: at[k] + s * v}) - value({**at, k: at[k] - s * v})) / (2 * s)
        assert abs(float((got["d" + k].double() * v).sum()) - slope) <= 1e-4 * (1 + abs(slope)), k


# ----------------------------------------------------------------------------
# Streams, graphs, repetition
# ----------------------------------------------------------------------------
def all_three(x, w, t, bias, dy):
    out = list(B.shampoo_linear_cross_entropy(x, w, t, bias=bias, grad_dtype=torch_().float32))
    c = B.shampoo_checkpoint_pack(x)
    out += list(B.shampoo_checkpoint_weight_grad(c, dy, B.ACT_SILU, bias=True))
    ones = torch_().ones(x.shape[1], device="cuda")
    r_out, h, r8, f8 = B.shampoo_residual_norm_forward(x, dy, w_post=ones, w_pre=ones, gate=ones, checkpoint=True)
    g = B.shampoo_residual_norm_backward(r8, f8, dy, x, w_post=ones, w_pre=ones, gate=ones)
    return out + [r_out, h] + [v for v in g.values() if v is not None]


def three_inputs(seed):
    torch = torch_()
    g = gen(seed)
    x, dy, w = normal(g, 500, 200).bfloat16(), normal(g, 500, 200).bfloat16(), normal(g, 1500, 200, sigma=0.1).bfloat16()
    return x, w, torch.randint(0, 1500, (500,), generator=g, device="cuda"), normal(g, 1500), dy


def test_the_same_call_gives_the_same_bits_on_any_stream():
    torch = torch_()
    inputs = three_inputs(1)
    first = all_three(*inputs)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        second = all_three(*inputs)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(first, second))


def test_replays_of_a_graph():
    torch = torch_()
    inputs = three_inputs(2)
    all_three(*inputs)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = all_three(*inputs)
    for seed in (3, 4, 5):
        for a, b in zip(inputs, three_inputs(seed)):
            a.copy_(b)
        graph.replay()
        torch.cuda.synchronize()
        got = [o.clone() for o in out]
        want = all_three(*inputs)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want))
