"""Reading the state of AdamW through the C interface in both types, and steps whose norm is zero or rounded."""
import ctypes
import math

import numpy as np
import pytest

from paper_2309_06497_amd import binding as B

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
SHAPES = [(1,), (3, 5), (0,), (129,), (2048,), (4097,), (1000, 33), (7,), ()]


def get(opt, dtype):
    """m and v by shampoo_adamw_get, between values that it must leave"""
    import torch
    n, kind = opt.total, {B.GRAD_F32: torch.float32, B.GRAD_BF16: torch.bfloat16}[dtype]
    m, v = (torch.full((n + 16,), 7.0, device="cuda", dtype=kind) for _ in range(2))
    stream = ctypes.c_void_p(torch.cuda.current_stream().cuda_stream)
    at = lambda x: ctypes.c_void_p(x.data_ptr() + 3 * x.element_size())
    assert B.lib().shampoo_adamw_get(opt.handle, at(m), at(v), dtype, stream) == 0
    for x in (m, v):
        assert bool((x[:3] == 7).all()) and bool((x[3 + n:] == 7).all())
    return m[3:3 + n], v[3:3 + n]


@pytest.mark.parametrize("bits", [32, 8])
def test_states_in_both_types(bits):
    """float32: what the optimizer holds, bit by bit; bf16: that to the nearest, which with 8 bits is the same"""
    import torch
    gen = torch.Generator(device="cuda")
    gen.manual_seed(bits)
    opt = B.AdamW(SHAPES, state_bits=bits)
    normal = lambda s: torch.randn(s, generator=gen, device="cuda")
    w = [normal(s) for s in SHAPES]
    for t in range(3):
        opt.step(w, [normal(s) * torch.exp(2 * normal(s)) for s in SHAPES], 1e-2, t)
        held = opt.state()
        for x, y, z in zip(get(opt, B.GRAD_F32), get(opt, B.GRAD_BF16), held):
            assert torch.equal(x, z.float()) and torch.equal(y, z.bfloat16())
            assert bool((x != 0).any())


@pytest.mark.parametrize("bits", [32, 8])
def test_states_at_the_ends_of_their_range_in_both_types(bits):
    """Codes of every binade of groups from 2^-100 to 2^126, and of groups below and above, that are zero and NaN"""
    import torch
    exponents = np.arange(-110, 128)
    m = np.ldexp(np.ones((len(exponents), 128)), exponents[:, None] - np.arange(128)[None] % 14) * (1 + np.arange(128) % 8 / 8) * np.where(np.arange(128) % 3 == 0, -1, 1)
    v = np.ldexp(np.ones((len(exponents), 128)), exponents[:, None] - np.arange(128)[None] % 30) * (1 + np.arange(128) % 8 / 8)
    m, v = (torch.from_numpy(x.astype(np.float32)).cuda().reshape(-1) for x in (m, v))
    opt = B.AdamW([(m.numel(),)], state_bits=bits)
    opt.load(m, v)
    some = torch.from_numpy(np.repeat((exponents >= -100) & (exponents < 127), 128)).cuda()
    zero = torch.from_numpy(np.repeat(exponents < -100, 128)).cuda()
    for got, half, want in zip(get(opt, B.GRAD_F32), get(opt, B.GRAD_BF16), (m, v)):
        if bits == 32:
            assert torch.equal(got, want) and torch.equal(half, want.bfloat16())
            continue
        assert torch.equal(got[some], want[some]) and torch.equal(half[some].float(), want[some])
        assert bool((got[zero] == 0).all()) and bool((half[zero] == 0).all())
        assert bool(torch.isnan(got[~some & ~zero]).all()) and bool(torch.isnan(half[~some & ~zero]).all())


@pytest.mark.parametrize("bits", [32, 8])
def test_a_step_whose_norm_is_zero(bits):
    """Nothing but decay: the parameters are w times 1 - lr wd in float32, exactly, and the states stay zero"""
    import torch
    opt = B.AdamW([(300,), (40, 7)], state_bits=bits, weight_decay=0.3, decay=[True, False])
    w = [torch.randn(s, device="cuda") for s in [(300,), (40, 7)]]
    g = [torch.zeros_like(x) for x in w]
    want = [w[0] * np.float32(1.0 - 1e-2 * 0.3), w[1].clone()]
    norm = B.shampoo_gradient_norm(g)[0]
    assert float(norm) == 0
    opt.step(w, g, 1e-2, 0, norm=norm, max_norm=1.0)
    assert all(torch.equal(x, y) for x, y in zip(w, want)) and all(bool((x == 0).all()) for x in opt.state())


def test_a_norm_that_float32_rounds():
    """sqrt(3): the norm is the nearest float32 (sums in 64 bits), the factor 1 / norm is off by u, m = (1 - beta1) g 1 / sqrt(3) by that, the weight's u and the two products': 5 u"""
    import torch
    g = [torch.ones((3,), device="cuda")]
    norm, norms = B.shampoo_gradient_norm(g)
    assert float(norm) == float(np.float32(math.sqrt(3))) == float(norms[0])
    opt = B.AdamW([(3,)], beta1=0.5)
    opt.step([torch.zeros((3,), device="cuda")], g, 1e-2, 0, norm=norm, max_norm=1.0)
    want = 0.5 / math.sqrt(3)
    assert all(abs(float(x) - want) <= 5 * U * want for x in opt.state()[0])
