"""Log probabilities, entropies, most probable tokens and the gradient of the logits against the definitions in 64 bits.

Tolerances.  u = 2^-24 is half a step of float32.  A logit's distance from the largest, in units of log 2, has three roundings (the subtraction, the scale
1 / T over log 2, the product): 3 u |x|.  2^x and log2 by the GPU's instructions are off by one step, 2 u of the result, at most.  A sum of n positive terms, added
up in `chain` steps one behind the other, is off by chain u of itself: a thread adds at most classes / 256 + 8 values and the joins are 20 more.  A term
that is e^-y of the largest has 3 u y / log 2 of itself, and p y summed over a row is at most H + log p_max, so at most log(classes) + 1.  Together
  s:    delta = u (chain + 2 + 5 (log(classes) + 1))  of itself
  log p: delta + 5 u |log p| + 2 u log2(classes)
  H:    two terms, log s and sum p x, of at most log(classes) + 1 each and delta of themselves: 3 delta (log(classes) + 1)
  dz:   p (A + b (log p + H)) / T:  p is off by delta + 5 u |log p| of itself, the bracket by 8 u of the sum of its magnitudes and b's part of the errors of log p and
        H; the GPU's 2^x is zero below 2^-126, so that p is off by 1.2e-38 in any case, and dz by that times the bracket; then the rounding to the result's type (2^-8 of a
        bf16 value, u of a float32 one, and a product that is that small may also lose all of itself below 1.2e-38)."""
import math

import pytest

from paper_2309_06497_amd import binding as B

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


def make(n, v, m, dtype, seed, spread=2.0, ignored=0.2):
    import torch
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    z = (torch.randn((n, v), generator=g, device="cuda") * spread).to(dtype)
    t = torch.randint(0, v, (n, m), generator=g, device="cuda")
    t[torch.rand((n, m), generator=g, device="cuda") < ignored] = -100
    return z, t, g


def definition(z, t, temperature):
    """log p of all tokens, log p of the given ones, entropy"""
    import torch
    x = z.double() / temperature
    m = x.amax(1, keepdim=True)
    m = torch.where(m == -math.inf, torch.zeros_like(m), m)
    lp = x - m - torch.log(torch.exp(x - m).sum(1, keepdim=True))
    lp = torch.where(torch.isnan(lp) & ~torch.isnan(z).any(1, keepdim=True) & ~(z == math.inf).any(1, keepdim=True), torch.full_like(lp, -math.inf), lp)
    p = torch.exp(lp)
    h = -(torch.where(p == 0, torch.zeros_like(p), p * lp)).sum(1)
    ok = (t >= 0) & (t < z.shape[1])
    given = torch.where(ok, lp.gather(1, torch.where(ok, t, torch.zeros_like(t))), torch.zeros_like(lp[:, :1]))
    return lp, given, h


def order(z, top):
    """The `top` largest logits of every row, ties to the lower token; -1 where none is left"""
    import numpy as np
    z = z.double().cpu().numpy()
    out = np.full((z.shape[0], top), -1)
    for i, row in enumerate(z):
        at = np.flatnonzero(row > -np.inf)                   # NaN: no
        at = at[np.lexsort((at, -(row[at] + 0.0)))][:top]
        out[i, :len(at)] = at
    return out


def delta(v):
    return U * (v / 256 + 28 + 2 + 5 * (math.log(v) + 1))


def lp_tolerance(lp, v):
    return delta(v) + 5 * U * lp.abs() + 2 * U * math.log2(v + 1)


def near(got, want, tolerance, what):
    import torch
    got, want = got.double(), want.double()
    want = torch.where(want.abs() > 3.4028235677973366e38, torch.copysign(torch.full_like(want, math.inf), want), want)      # what float32 rounds to infinity
    assert torch.equal(torch.isfinite(got), torch.isfinite(want)), what
    assert torch.equal(torch.isnan(got), torch.isnan(want)), what
    same = (got == want) | torch.isnan(want)
    off = torch.where(same, torch.zeros_like(got), (got - want).abs())
    tolerance = torch.as_tensor(tolerance, device=got.device, dtype=torch.float64).expand_as(off)
    tolerance = torch.where(same, torch.ones_like(off), tolerance)
    assert bool((off <= tolerance).all()), (what, float((off / tolerance).max()))


def check(z, t, top, temperature, r=None):
    import torch
    v = z.shape[1]
    r = r or B.shampoo_log_probs(z, t, top=top, temperature=temperature)
    lp, given, h = definition(z, t if t.dim() == 2 else t[:, None], temperature)
    assert r.log_probs.shape == t.shape and r.log_probs.dtype == torch.float32 and r.entropy.shape == (z.shape[0],)
    near(r.log_probs.view(given.shape), given, lp_tolerance(given, v), "log p")
    near(r.entropy, h, 3 * delta(v) * (math.log(v) + 1), "entropy")
    if top == 0:
        assert r.top_tokens is None and r.top_log_probs is None
        return r
    want = order(z, top)
    assert r.top_tokens.dtype == torch.int64 and (r.top_tokens.cpu().numpy() == want).all()
    at = torch.from_numpy(want).to(z.device)
    alp = torch.where(at < 0, torch.where(torch.isnan(lp).any(1, keepdim=True), math.nan, -math.inf), lp.gather(1, at.clamp(min=0)))
    near(r.top_log_probs, alp, lp_tolerance(alp, v), "log p of the most probable")
    return r


def gradient(z, t, a, b, temperature):
    """By the definition, and its tolerance before the rounding to the result's type"""
    import torch
    n, v = z.shape
    lp, given, h = definition(z, t, temperature)
    p = torch.exp(lp)
    ok = (t >= 0) & (t < v) & (p.sum(1, keepdim=True) > 0)
    a = torch.where(ok, a.double(), torch.zeros_like(given))
    total, size = a.sum(1, keepdim=True), a.abs().sum(1, keepdim=True)
    lp0 = torch.where(p == 0, torch.zeros_like(lp), lp)
    bb = b.double()[:, None] if b is not None else torch.zeros((n, 1), device=z.device, dtype=torch.float64)
    dz = -p * (total + bb * (lp0 + h[:, None]))
    for j in range(t.shape[1]):
        i = ok[:, j].nonzero()[:, 0]
        dz[i, t[i, j]] += a[i, j]
    d = delta(v)
    magnitude = size + bb.abs() * (lp0.abs() + h[:, None])
    off = p * (magnitude * (d + 5 * U * lp0.abs() + 8 * U) + bb.abs() * (lp_tolerance(lp0, v) + 3 * d * (math.log(v) + 1))) + 1.2e-38 * magnitude
    spot = torch.zeros_like(dz)
    for j in range(t.shape[1]):
        i = ok[:, j].nonzero()[:, 0]
        spot[i, t[i, j]] += size[i, 0] * (t.shape[1] + 4) * U
    return dz / temperature, (off + spot) / temperature


def check_gradient(z, t, a, b, temperature, got=None):
    import torch
    want, off = gradient(z, t, a if a is not None else torch.zeros(t.shape, device=z.device), b, temperature)
    if got is None:
        got = B.shampoo_log_probs_grad(z, t, B.shampoo_log_probs(z, t, temperature=temperature), a, b)
    assert got.dtype == z.dtype and got.shape == z.shape
    half = torch.finfo(z.dtype).eps / 2
    near(got, want, off * (1 + half) + half * want.abs() + 1.2e-38, "gradient")
    return got


SIZES = [(1, 1, 1, 1, 1.0), (1, 2, 1, 2, 0.5), (3, 7, 2, 7, 1.0), (4, 8, 1, 3, 2.0), (5, 33, 4, 5, 1.0), (6, 511, 3, 64, 1.0), (6, 513, 3, 64, 1.3), (17, 1000, 16, 20, 0.7),
         (2, 4097, 64, 64, 2.0), (64, 2048, 1, 1, 1.0), (9, 2049, 1, 50, 1.0), (1, 16384, 1, 20, 1.0), (3, 16389, 5, 33, 1.0), (1, 131072, 1, 20, 1.0), (2, 131071, 2, 64, 0.9),
         (1, 262147, 1, 64, 1.0), (300, 5003, 4, 10, 1.0), (700, 999, 1, 0, 1.0), (1025, 257, 1, 2, 1.0), (40, 33000, 1, 12, 1.0), (2000, 64, 1, 64, 1.0)]


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("n,v,m,top,temperature", SIZES)
def test_log_probs(n, v, m, top, temperature, dtype):
    import torch
    z, t, _ = make(n, v, m, getattr(torch, dtype), n + v)
    check(z, t, top, temperature)
    if m == 1:
        check(z, t[:, 0], top, temperature)


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("n,v,m,top,temperature", SIZES)
def test_gradient_of_logits(n, v, m, top, temperature, dtype):
    import torch
    z, t, g = make(n, v, m, getattr(torch, dtype), n + v)
    a = torch.randn((n, m), generator=g, device="cuda")
    b = torch.randn((n,), generator=g, device="cuda")
    check_gradient(z, t, a, b, temperature)
    check_gradient(z, t, a, None, temperature)
    check_gradient(z, t, None, b, temperature)


def test_gradient_against_differences():
    """Of sum a log p + sum b H in 64 bits, along a random direction.  Central differences at 2^-17: their own error is the third derivative (a few units) times
    2^-34 / 6 and rounding 2^-53 / 2^-17 of a sum of 16 x 6 terms of size one: 1e-9; the gradient's is float32's, 2^-24 of sums of 50 products of size one: 1e-5."""
    import torch
    z, t, g = make(16, 50, 3, torch.float32, 5)
    a, b, u = torch.randn((16, 3), generator=g, device="cuda"), torch.randn((16,), generator=g, device="cuda"), torch.randn((16, 50), generator=g, device="cuda")
    for temperature in (1.0, 0.6):
        r = B.shampoo_log_probs(z, t, temperature=temperature)
        got = float((B.shampoo_log_probs_grad(z, t, r, a, b).double() * u.double()).sum())

        def value(s):
            _, given, h = definition(z.double() + s * u.double(), t, temperature)
            return float((a.double() * given).sum() + (b.double() * h).sum())

        e = 2.0 ** -17
        assert abs((value(e) - value(-e)) / (2 * e) - got) < 1e-5 * (1 + abs(got))


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("v", [40, 300, 5000, 40007])
def test_ties_go_to_the_lower_token(v, dtype):
    import torch
    dtype = getattr(torch, dtype)
    g = torch.Generator(device="cuda")
    g.manual_seed(v)
    few = torch.randint(0, 3, (5, v), generator=g, device="cuda").to(dtype)
    equal = torch.full((2, v), -2.5, device="cuda", dtype=dtype)
    zeros = torch.where(torch.rand((2, v), generator=g, device="cuda") < 0.5, 0.0, -0.0).to(dtype)
    low = torch.full((2, v), torch.finfo(dtype).min, device="cuda", dtype=dtype)
    low[1, v // 2], low[1, v - 1] = 1.0, 3.0
    late = torch.full((1, v), -1.0, device="cuda", dtype=dtype)
    late[0, -9:] = 1.0
    z = torch.cat([few, equal, zeros, low, late])
    t = torch.randint(0, v, (z.shape[0], 2), generator=g, device="cuda")
    for top in (1, 5, 20, 64):
        check(z, t, top, 1.0)


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("v", [100, 3000, 33333])
def test_rows_in_order(v, dtype):
    """Every logit larger than all before it, and the other way round; the largest all side by side, or one in each stretch"""
    import torch
    up = torch.arange(v, device="cuda", dtype=torch.float32)
    z = torch.stack([up, -up, up % 129, -(up % 8) * 4, (up // 8) % 70, up // 2048]).to(getattr(torch, dtype)) * 0.01
    t = torch.tensor([[0, v - 1]] * 6, device="cuda")
    for top in (3, 64):
        check(z, t, top, 1.0)


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("v", [100, 1500, 5000, 40000, 150000])
def test_rows_that_are_sure_of_one_token(v, dtype):
    """The others far behind: 10 ... 300, and more than any exponent holds; spreads that are next to nothing"""
    import torch
    z, t, _ = make(7, v, 2, getattr(torch, dtype), v)
    for i, (lead, spread) in enumerate(((10.0, 1.0), (60.0, 1.0), (300.0, 3.0), (1e4, 1.0), (20.0, 1e-3), (0.0, 1e-30), (3e38, 1.0))):
        z[i] *= spread
        z[i, (v * i) // 7] = lead
    for top in (1, 20, 64):
        for temperature in (1.0, 0.1, 30.0):
            check(z, t, top, temperature)


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("v", [9, 700, 9001])
def test_masked_tokens(v, dtype):
    """Few left, one left, nothing left; masked and ignored tokens given"""
    import torch
    z, t, g = make(7, v, 3, getattr(torch, dtype), v)
    z[0, torch.rand((v,), generator=g, device="cuda") < 0.9] = -math.inf
    z[1, 1:] = -math.inf
    z[2, :-1] = -math.inf
    z[3] = -math.inf
    z[4, ::2] = -math.inf
    t[:, 0], t[:, 1], t[:, 2] = 0, v - 1, v
    for top in (0, 4, 64):
        r = check(z, t, top, 1.0)
    assert float(r.entropy[1]) == 0 and float(r.entropy[2]) == 0 and float(r.entropy[3]) == 0
    assert float(r.log_probs[1, 0]) == 0 and float(r.log_probs[1, 1]) == -math.inf and (r.log_probs[:, 2] == 0).all()
    a, b = torch.randn((7, 3), generator=g, device="cuda"), torch.randn((7,), generator=g, device="cuda")
    got = check_gradient(z, t, a, b, 1.0)
    assert (got[3] == 0).all()
    assert (got[4, 2::2][: (v - 2) // 2] == 0).all()


def test_the_lowest_value_in_a_whole_row_and_far_offsets():
    """Equal logits have log p = -log(classes) wherever they are; a common offset takes nothing"""
    import torch
    v = 1000
    for dtype in (torch.float32, torch.bfloat16):
        z = torch.empty((4, v), device="cuda", dtype=dtype)
        z[0], z[1], z[2], z[3] = torch.finfo(dtype).min, torch.finfo(dtype).max, 0.0, 1e4
        t = torch.full((4,), 5, device="cuda")
        for temperature in (0.25, 1.0, 100.0):
            r = check(z, t, 3, temperature)
            near(r.log_probs, torch.full((4,), -math.log(v), device="cuda"), delta(v) + 20 * U * math.log(v), "equal logits")
            check_gradient(z, t[:, None], torch.ones((4, 1), device="cuda"), torch.ones((4,), device="cuda"), temperature)
    y = torch.randn((3, v), device="cuda").mul_(64).round_().div_(64)           # whole 64ths: 2^14 + y is exact
    t = torch.arange(3, device="cuda")
    one, two = B.shampoo_log_probs(y, t), B.shampoo_log_probs(y + 16384.0, t)
    assert torch.equal(one.log_probs, two.log_probs) and torch.equal(one.entropy, two.entropy)


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("v", [30, 5003])
def test_values_that_are_not_finite(v, dtype):
    import torch
    z, t, g = make(5, v, 2, getattr(torch, dtype), 3, ignored=0.0)
    z[0, 7], z[1, v - 1], z[2, 3], z[2, 4] = math.nan, math.inf, math.nan, -math.inf
    z[3] = math.nan
    t[2, 0], t[1, 1] = 4, v - 1
    r = B.shampoo_log_probs(z, t, top=6)
    bad = torch.tensor([True, True, True, True, False], device="cuda")
    assert torch.isnan(r.log_probs[bad]).all() and torch.isnan(r.entropy[bad]).all() and torch.isnan(r.top_log_probs[bad]).all()
    assert (r.top_tokens.cpu().numpy() == order(z, 6)).all()
    check(z[4:], t[4:], 6, 1.0)
    a = torch.randn((5, 2), generator=g, device="cuda")
    got = B.shampoo_log_probs_grad(z, t, r, a, torch.ones((5,), device="cuda"))
    assert torch.isnan(got[bad]).all() and torch.isfinite(got[4]).all()
    got = B.shampoo_log_probs_grad(z, torch.full_like(t, -1), r, a)            # ignored rows: nothing, whatever their logits are
    assert (got == 0).all()


def test_a_token_given_twice():
    import torch
    z, t, g = make(6, 300, 64, torch.float32, 8)
    t[:, 32:] = t[:, :32]
    t[0] = 5
    a = torch.randn((6, 64), generator=g, device="cuda")
    check(z, t, 0, 1.0)
    check_gradient(z, t, a, None, 1.0)
    a[0] = torch.tensor([1.0, -1.0] * 32, device="cuda")                       # coefficients that cancel
    check_gradient(z, t, a, None, 1.0)


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("v", [37, 1000, 8200, 70001])
def test_strides_alignments_and_results_in_place(v, dtype):
    import torch
    dtype = getattr(torch, dtype)
    wide, t, g = make(9, 2 * v + 5, 2, dtype, v)
    t %= v
    a, b = torch.randn((9, 2), generator=g, device="cuda"), torch.randn((9,), generator=g, device="cuda")
    for z in (wide[:, 1:v + 1], wide[:, v + 2:2 * v + 2], wide[::2, 3:v + 3], wide[:, ::2][:, :v], wide[:, :v].t().contiguous().t()):
        n = z.shape[0]
        check(z, t[:n], 5, 1.0)
        want = check_gradient(z, t[:n], a[:n], b[:n], 1.0)
        # the gradient is made element by element; sums are in an order that goes by a row's address, so that the last bits of log p and entropy may differ
        same = B.shampoo_log_probs(z, t[:n])
        assert torch.equal(B.shampoo_log_probs_grad(z.contiguous(), t[:n], same, a[:n], b[:n]), want)
    # in place, and beside the logits in the same matrix: the other columns stay
    z = wide[:, 1:v + 1]
    r = B.shampoo_log_probs(z, t)
    want = B.shampoo_log_probs_grad(z, t, r, a, b)
    before = wide.clone()
    out = wide[:, v + 2:2 * v + 2]
    assert B.shampoo_log_probs_grad(z, t, r, a, b, out=out).data_ptr() == out.data_ptr()
    assert torch.equal(out, want)
    before[:, v + 2:2 * v + 2] = want
    assert torch.equal(wide, before)
    B.shampoo_log_probs_grad(z, t, r, a, b, out=z)
    before[:, 1:v + 1] = want
    assert torch.equal(wide, before)
    for bad in (wide[:, 2:v + 2], wide[:, :v], wide.view(-1)[1:1 + 9 * v].view(9, v)):
        with pytest.raises(AssertionError):
            B.shampoo_log_probs_grad(z, t, r, a, b, out=bad)


def test_no_rows_and_no_tokens():
    import torch
    z = torch.randn((0, 50), device="cuda")
    r = B.shampoo_log_probs(z, torch.empty((0,), dtype=torch.int64, device="cuda"), top=3)
    assert r.log_probs.shape == (0,) and r.top_tokens.shape == (0, 3)
    assert B.shampoo_log_probs_grad(z, torch.empty((0,), dtype=torch.int64, device="cuda"), r, r.log_probs).shape == (0, 50)
    z, t, _ = make(4, 50, 1, torch.float32, 1)
    r = check(z, t[:, :0], 3, 1.0)
    check_gradient(z, t[:, :0], None, torch.ones((4,), device="cuda"), 1.0)
    assert (B.shampoo_log_probs_grad(z, t[:, :0], r, None) == 0).all()


def test_refusals():
    import torch
    z, t, _ = make(4, 50, 2, torch.float32, 1)
    r = B.shampoo_log_probs(z, t)
    for call in (lambda: B.shampoo_log_probs(z.half(), t), lambda: B.shampoo_log_probs(z[0], t), lambda: B.shampoo_log_probs(z.cpu(), t), lambda: B.shampoo_log_probs(z, t.cpu()),
                 lambda: B.shampoo_log_probs(z, t.int()), lambda: B.shampoo_log_probs(z, t[:3]), lambda: B.shampoo_log_probs(z, t[..., None]),
                 lambda: B.shampoo_log_probs_grad(z, t, r, torch.ones((4,), device="cuda")), lambda: B.shampoo_log_probs_grad(z, t, r, t),
                 lambda: B.shampoo_log_probs_grad(z[:3], t[:3], r, None), lambda: B.shampoo_log_probs_grad(z, t, r, None, torch.ones((3,), device="cuda")),
                 lambda: B.shampoo_log_probs_grad(z, t, r, None, out=z.bfloat16()), lambda: B.shampoo_log_probs_grad(z, t, r, None, out=z.t().contiguous().t())):
        with pytest.raises(AssertionError):
            call()
    for call, code in ((lambda: B.shampoo_log_probs(z, t, top=65), -7), (lambda: B.shampoo_log_probs(z, t.repeat(1, 33)), -7), (lambda: B.shampoo_log_probs(z, t, top=-1), -2),
                       (lambda: B.shampoo_log_probs(z, t, temperature=-1.0), -3), (lambda: B.shampoo_log_probs(z, t, temperature=math.nan), -3),
                       (lambda: B.shampoo_log_probs(z[:, :0], t), -2), (lambda: B.shampoo_log_probs(z, t, temperature=1e-45), -3)):
        with pytest.raises(B.ShampooError) as e:
            call()
        assert e.value.code == code
    with pytest.raises((ZeroDivisionError, B.ShampooError)):
        B.shampoo_log_probs(z, t, temperature=0.0)


def test_other_streams_and_replayed_graphs():
    """Work on a stream of its own; two captured calls, replayed between eager ones, on new values in the same memory"""
    import torch
    calls = []
    for n, v, top in ((3, 40000, 20), (60, 3000, 5)):
        z, t, g = make(n, v, 2, torch.bfloat16, v)
        a, b = torch.randn((n, 2), generator=g, device="cuda"), torch.randn((n,), generator=g, device="cuda")
        calls.append((z, t, top, a, b))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graphs = []
    for z, t, top, a, b in calls:
        with torch.cuda.stream(side):
            r = B.shampoo_log_probs(z, t, top=top)
            dz = B.shampoo_log_probs_grad(z, t, r, a, b)
        torch.cuda.synchronize()
        check(z, t, top, 1.0, r)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            r = B.shampoo_log_probs(z, t, top=top)
            dz = B.shampoo_log_probs_grad(z, t, r, a, b)
        graphs.append((graph, r, dz))
    for seed in range(3):
        for (z, t, top, a, b), (graph, r, dz) in zip(calls, graphs):
            z.copy_(make(z.shape[0], z.shape[1], 2, torch.bfloat16, 100 + seed)[0])
        for graph, _, _ in graphs:
            graph.replay()
        torch.cuda.synchronize()
        for (z, t, top, a, b), (graph, r, dz) in zip(calls, graphs):
            want = check(z, t, top, 1.0)
            assert torch.equal(want.log_probs, r.log_probs) and torch.equal(want.top_tokens, r.top_tokens) and torch.equal(want.entropy, r.entropy)
            assert torch.equal(want.top_log_probs, r.top_log_probs) and torch.equal(B.shampoo_log_probs_grad(z, t, want, a, b), dz)


def test_offsets_beyond_32_bits():
    """70000 rows of 65537 logits: 4.6e9 elements.  The rows behind 2^32 are looked at."""
    import torch
    n, v = 70000, 65537
    z = torch.zeros((n, v), device="cuda", dtype=torch.bfloat16)
    some = torch.tensor([0, 32767, 65534, 65535, 65536, 69998, 69999], device="cuda")
    y, t, g = make(len(some), v, 1, torch.bfloat16, 1, ignored=0.0)
    z[some] = y
    tokens = torch.full((n, 1), 3, device="cuda")
    tokens[some] = t
    r = B.shampoo_log_probs(z, tokens, top=5)
    check(y, t, 5, 1.0, B.LogProbs(*(x[some] for x in (r.log_probs, r.entropy, r.top_tokens, r.top_log_probs, r.statistics)), 1.0))
    assert (r.top_tokens[60000] == torch.arange(5, device="cuda")).all()
    a, b = torch.ones((n, 1), device="cuda"), torch.ones((n,), device="cuda")
    got = B.shampoo_log_probs_grad(z, tokens, r, a, b, out=z)
    check_gradient(y, t, a[some], b[some], 1.0, got[some])


def test_the_same_call_gives_the_same_bits():
    import torch
    z, t, g = make(50, 50001, 3, torch.bfloat16, 2)
    a, b = torch.randn((50, 3), generator=g, device="cuda"), torch.randn((50,), generator=g, device="cuda")
    first = None
    for _ in range(3):
        r = B.shampoo_log_probs(z, t, top=9)
        now = (r.log_probs, r.entropy, r.top_tokens, r.top_log_probs, B.shampoo_log_probs_grad(z, t, r, a, b))
        assert first is None or all(torch.equal(x, y) for x, y in zip(first, now))
        first = now
