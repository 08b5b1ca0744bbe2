"""Rows of logits against the definition in 64 bits, with a bar for every row by what its own terms are.

u = 2^-24 is half a step of float32.  With m the largest logit of a row, x = (z - m) / T, p the probabilities, q = 1 - max p, M1 = sum p |x|, M2 = sum p x^2:

A term 2^x is made in two steps, about a reference that may lie 8 log 2 = 5.6 below m and from there to m: two powers of two by the GPU's instruction, one step (2 u) each, and
their product: 5 u; the exponent has 4 roundings (difference, 1 / T, its product with 1 / log 2, the product): 4 u |x|, and 4 u 11.2 where a term lies between reference and m.  The
largest logit's own exponents are one value with both signs, so that it has the 5 u alone.  An addition is off by u of its result, and never by more than the smaller
of the two.  A thread adds at most 272 values (16384 classes by two wavefronts, 131072 by eight, and what the row's ends add), its wavefront, workgroup and row 20 more, and adding
zeros is exact: chain = min(292, terms that are not zero), and at most twice min(chain u, q).  Together
  s:     e = u (5 + 50 q + 4 M1) + 2 min(chain u, q)  of itself
  log p: e + u (2 + 5 log s + 5 |log p|)        (log2 one step, log 2 and its product; z - m, 1 / T, the sum)
  H:     log s and sum p x: e (1 + M1) + u (24 + 5 log s + 55 M1 + 4 M2) + 2 min(chain u (M1 + 5.6), M1 + 5.6 q)        (terms count from the reference: up to 5.6 p on top)
  dz:    p (A + b (log p + H)) / T: p is off by e + u (5 |x| + 4), the bracket by 12 u of its magnitudes and b times the bars of log p and H; 2^x is zero below 2^-126; the
         sum over a row's tokens; the result's type (half a step of a bf16 or float32 value)."""
import math

import pytest

from paper_2309_06497_amd import binding as B

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


class Row:
    """Definitions of a matrix of logits [n, v] and the bars above, all [n, 1] or [n, v]"""

    def __init__(self, z, temperature):
        import torch
        v = z.shape[1]
        x = z.double() / temperature
        m = x.amax(1, keepdim=True)
        x = x - torch.where(m == -math.inf, 0.0, m)
        e = torch.exp(x)
        s = e.sum(1, keepdim=True)
        self.some = s > 0
        log_s = torch.where(self.some, torch.log(s), 0.0)
        self.lp = x - log_s
        self.p = torch.where(self.some, e / s, 0.0)
        near = torch.where(self.p == 0, 0.0, x)
        self.h = torch.where(self.some, log_s - (self.p * near).sum(1, keepdim=True), 0.0)
        q = torch.where(self.some, 1 - self.p.amax(1, keepdim=True), 0.0)
        m1, m2 = (self.p * near.abs()).sum(1, keepdim=True), (self.p * near * near).sum(1, keepdim=True)
        chain = (e > 2.0 ** -126).sum(1, keepdim=True).clamp(max=292).double()
        self.e = U * (5 + 50 * q + 4 * m1) + 2 * torch.minimum(chain * U, q)
        self.lp_bar = self.e + U * (2 + 5 * log_s + 5 * torch.where(self.lp == -math.inf, 0.0, self.lp).abs())
        self.h_bar = self.e * (1 + m1) + U * (24 + 5 * log_s + 55 * m1 + 4 * m2) + 2 * torch.minimum(chain * U * (m1 + 5.6), m1 + 5.6 * q)
        self.p_bar = self.p * (self.e + U * (5 * near.abs() + 4))
        self.near_lp = torch.where(self.p == 0, 0.0, self.lp)


def within(got, want, bar, what):
    """got: float32; what float32 rounds to infinity is infinite"""
    import torch
    got = got.double()
    want = torch.where(want.abs() > 3.4028235677973366e38, torch.copysign(torch.full_like(want, math.inf), want), want)
    assert torch.equal(torch.isfinite(got), torch.isfinite(want)) and not bool(torch.isnan(got).any()), what
    off = torch.where(got == want, 0.0, (got - want).abs())
    bar = bar.expand_as(off)
    assert bool((off <= bar).all()), (what, float((off / bar).max()))


def given(row, t, v):
    import torch
    ok = (t >= 0) & (t < v)
    at = torch.where(ok, t, 0)
    return ok, at, torch.where(ok, row.lp.gather(1, at), 0.0), torch.where(ok, row.lp_bar.gather(1, at), 0.0)


def check(z, t, top, temperature, row=None):
    """Of one call; the order of tokens by a stable sort"""
    import torch
    v = z.shape[1]
    row = row or Row(z, temperature)
    r = B.shampoo_log_probs(z, t, top=top, temperature=temperature)
    _, _, want, bar = given(row, t, v)
    within(r.log_probs, want, bar, "log p")
    within(r.entropy[:, None], row.h, row.h_bar, "entropy")
    if top:
        value, at = torch.sort(z.float() + 0.0, dim=1, descending=True, stable=True)
        value, at = value[:, :top], at[:, :top]
        none = value == -math.inf
        short = torch.nn.functional.pad(torch.where(none, -1, at), (0, top - at.shape[1]), value=-1)
        assert torch.equal(r.top_tokens, short)
        near = torch.where(none, -math.inf, row.lp.gather(1, at))
        within(r.top_log_probs[:, :at.shape[1]], near, row.lp_bar.gather(1, at), "log p of the most probable")
        assert bool((r.top_log_probs[:, at.shape[1]:] == -math.inf).all())
    return r, row


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("n,v", [(500, 9000), (4200, 8192), (3, 70000), (70, 140000)])
def test_a_sure_token_read_behind_a_less_probable_one(n, v, dtype):
    """All but two tokens masked, 4096 apart, so that one thread reads both, one behind the other, the second 4 to 5.5 larger: what it sums about is the first.  The larger one's own
    term has 5 u, the other's 0.02 times 50 u, their sum u, its log2 one step of a number about one: 9 u for log p of either, and 5 u |log p| more for the smaller one."""
    import torch
    g = torch.Generator(device="cuda")
    g.manual_seed(n)
    z = torch.full((n, v), -math.inf, device="cuda")
    low = torch.randint(0, v - 4096, (n, 1), generator=g, device="cuda")
    t = torch.cat([low + 4096, low], 1)
    first = torch.randn((n, 1), generator=g, device="cuda")
    lead = torch.rand((n, 1), generator=g, device="cuda") * 1.5 + 4.0
    z = z.scatter_(1, t, torch.cat([first + lead, first], 1)).to(getattr(torch, dtype))
    r, row = check(z, t, 2, 1.0)
    want = row.lp.gather(1, t)
    off = (r.log_probs.double() - want).abs() / (9 * U + torch.tensor([0.0, 5 * U], device="cuda") * want.abs())
    worst = float(off.max())
    assert worst <= 1, worst


def check_gradient(z, t, a, b, temperature, r, row):
    """a [n, m] or None, b [n] or None"""
    import torch
    n, v = z.shape
    got = B.shampoo_log_probs_grad(z, t, r, a, b)
    assert got.dtype == z.dtype and got.shape == z.shape
    ok, at, _, _ = given(row, t, v)
    ok = ok & row.some
    coef = torch.where(ok, a.double(), 0.0) if a is not None else torch.zeros(t.shape, device=z.device, dtype=torch.float64)
    bb = b.double()[:, None] if b is not None else torch.zeros((n, 1), device=z.device, dtype=torch.float64)
    total, size = coef.sum(1, keepdim=True), coef.abs().sum(1, keepdim=True)
    want = -row.p * (total + bb * (row.near_lp + row.h))
    magnitude = size + bb.abs() * (row.near_lp.abs() + row.h)
    bar = row.p_bar * magnitude + row.p * (12 * U * magnitude + bb.abs() * (torch.where(row.p == 0, 0.0, row.lp_bar) + row.h_bar)) + 1.2e-38 * magnitude
    want.scatter_add_(1, at, coef)
    bar.scatter_add_(1, at, torch.where(ok, size * (t.shape[1] + 4) * U, 0.0))
    half = torch.finfo(z.dtype).eps / 2
    want, bar = want / temperature, bar / temperature
    within(got, want, bar * (1 + half) + half * want.abs() + 1.2e-38, "gradient")
    return got


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("v", [50, 3000, 9000])
@pytest.mark.parametrize("temperature", [1e-38, 1e-30, 1e-12])
def test_gradients_of_small_temperatures(v, dtype, temperature):
    """Coefficients over T that float32 does not hold: nothing for tokens of no probability, and for a token that has all of it"""
    import torch
    g = torch.Generator(device="cuda")
    g.manual_seed(v)
    z = torch.randn((40, v), generator=g, device="cuda").to(getattr(torch, dtype))
    z[:, 1] = torch.where(torch.arange(40, device="cuda") % 2 == 0, -math.inf, 8.0)
    t = torch.randint(0, v, (40, 2), generator=g, device="cuda")
    t[:, 0] = torch.where(torch.arange(40, device="cuda") % 3 == 0, z.float().argmax(1), 1)
    t[::5, 1] = -100
    a = torch.randn((40, 2), generator=g, device="cuda") * 8
    b = torch.randn((40,), generator=g, device="cuda") * 8
    r, row = check(z, t, 5, temperature)
    for x, y in ((a, None), (a, b), (None, b)):
        got = check_gradient(z, t, x, y, temperature, r, row)
        assert not bool(torch.isnan(got).any())


# Rows in a workgroup of one, two, four and eight wavefronts, and rows in parts of eight that a second launch joins (test_logits_adamw_rows_host.py holds that they are)
BATCHES = [(4100, 2049), (4099, 8191), (2050, 2500), (4097, 16381), (4097, 16393), (2100, 33000), (65, 131075), (64, 262147), (63, 131077)]


def many_kinds(n, v, dtype, seed):
    """Rows of sixteen kinds by turns, the last rows too: what makes the choice of tokens easy, and what sends it through each of its searches"""
    import torch
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    z = torch.randn((n, v), generator=g, device="cuda").mul_(2.0)
    rand = lambda *shape: torch.rand(shape, generator=g, device="cuda")
    up = torch.arange(v, device="cuda", dtype=torch.float32)
    kinds = [None,
             lambda i: torch.floor(rand(v) * 3),                                         # few values
             lambda i: torch.full((v,), -2.5, device="cuda"),                            # one
             lambda i: torch.where(rand(v) < 0.5, 0.0, -0.0),
             lambda i: torch.full((v,), torch.finfo(dtype).min, device="cuda").index_fill_(0, torch.tensor([v // 2, v - 1], device="cuda"), 1.0),
             lambda i: up * 0.01, lambda i: up * -0.01,                                  # in order
             lambda i: (up // 8) % 70 * 0.01,
             lambda i: up // 512 % 40,                                                   # the largest side by side
             lambda i: z[i].clone().index_fill_(0, (rand(1) * v).long(), 14.0),          # sure of one
             lambda i: (z[i] * 0.1).index_fill_(0, (rand(1) * v).long(), 300.0),
             lambda i: torch.where(rand(v) < 0.98, -math.inf, z[i]),                     # few left
             lambda i: torch.full((v,), -math.inf, device="cuda").index_fill_(0, (rand(1) * v).long(), -3.0),
             lambda i: torch.full((v,), -math.inf, device="cuda"),
             lambda i: z[i] * 1e-30,                                                     # spreads next to nothing
             lambda i: torch.where(up < v - 9, -1.0, 1.0)]                               # the largest last
    for i in list(range(64 if n > 64 else n)) + list(range(max(n - 16, 64), n)):
        if kinds[i % 16]:
            z[i] = kinds[i % 16](i)
    t = torch.randint(0, v, (n, 3), generator=g, device="cuda")
    t[:, 2] = z.argmax(1)
    t[rand(n, 3) < 0.1] = -100
    a, b = torch.randn((n, 3), generator=g, device="cuda"), torch.randn((n,), generator=g, device="cuda")
    return z.to(dtype), t, a, b


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("n,v", BATCHES)
def test_batches_of_every_kind_of_row(n, v, dtype):
    import torch
    z, t, a, b = many_kinds(n, v, getattr(torch, dtype), v)
    for temperature, tops in ((1.0, (0, 20, 64)), (0.6, (5,))):
        row = Row(z, temperature)
        for top in tops:
            r, _ = check(z, t, top, temperature, row)
    check_gradient(z, t, a, b, temperature, r, row)


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("n,v", [(4100, 2050), (2050, 4100), (65, 131076)])
def test_batches_between_the_columns_of_a_matrix(n, v, dtype):
    """Rows that begin anywhere"""
    import torch
    z, t, a, b = many_kinds(n, v, getattr(torch, dtype), v + 1)
    wide = torch.full((n, v + 3), math.inf, device="cuda", dtype=z.dtype)
    for first in (1, 2):
        view = wide[:, first:first + v]
        view.copy_(z)
        r, row = check(view, t, 20, 1.0)
        check_gradient(view, t, a, b, 1.0, r, row)
        view.fill_(math.inf)


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("v", [37, 500, 700, 1025, 2048])
def test_short_rows_of_every_kind(v, dtype):
    import torch
    z, t, a, b = many_kinds(300, v, getattr(torch, dtype), v)
    for top in (0, 1, 20, 64):
        r, row = check(z, t, top, 1.0)
    check_gradient(z, t, a, b, 1.0, r, row)


@pytest.mark.parametrize("top", [65, 1 << 20, (1 << 31) - 1])
def test_more_tokens_than_are_ordered_are_refused_before_their_memory_is_asked_for(top):
    import torch
    z, t = torch.zeros((1 << 15, 8), device="cuda"), torch.zeros((1 << 15,), dtype=torch.int64, device="cuda")
    torch.cuda.synchronize()
    before = torch.cuda.memory_reserved()
    with pytest.raises(B.ShampooError) as e:
        B.shampoo_log_probs(z, t, top=top)
    assert e.value.code == -7 and torch.cuda.memory_reserved() - before < 1 << 28
