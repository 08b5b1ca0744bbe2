"""The operators of a training pass that make the gradients of a Shampoo step, as cases that can be timed.

  "head"    softmax cross entropy of a linear layer over many classes, with the gradients of its input, weight and bias; or the
            loss alone
  "pack"    a checkpoint of an activation in 8 bits, and back
  "act"     the gradient of an activation function from the checkpoint of its input
  "wgrad"   the gradient of a linear layer's weight and bias from the checkpoint of its input
  "norm"    residual sum with the norms after and before a block, forward, or forward and backward through 8-bit checkpoints

`own` chooses between the package's kernels and the plain form: elementary torch operations in float32.
"""
import math

import torch

own = False        # True: the calls of the package; False: the plain form

GROUP = 32         # neighbouring features that share a scale in a checkpoint
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


def listed():
    return [
        # A fine-tuning step on a few short rows, small classifier: launches and latency.
        {"name": "head_small", "kind": "head", "rows": 32, "features": 256, "classes": 1000, "type": "bf16", "grad": "bf16",
         "in_out": False, "bias": False, "ignored": 0.0, "gradients": True},
        # The last layer of a convolutional network (2048 features, 1000 classes, a bias), float32 throughout.
        {"name": "head_fc", "kind": "head", "rows": 256, "features": 2048, "classes": 1000, "type": "f32", "grad": "f32",
         "in_out": True, "bias": True, "ignored": 0.0, "gradients": True},
        # A language model of width 2048 with a vocabulary of ordinary size.
        {"name": "head_ordinary", "kind": "head", "rows": 4096, "features": 2048, "classes": 32000, "type": "bf16", "grad": "bf16",
         "in_out": False, "bias": False, "ignored": 0.1, "gradients": True},
        # Nothing divides: width 1000, an odd vocabulary kept as (in, out), float32 weight gradients, padded rows.
        {"name": "head_ragged", "kind": "head", "rows": 1999, "features": 1000, "classes": 50001, "type": "bf16", "grad": "f32",
         "in_out": True, "bias": True, "ignored": 0.3, "gradients": True},
        # The largest: a multilingual vocabulary.
        {"name": "head_large", "kind": "head", "rows": 8192, "features": 2048, "classes": 131072, "type": "bf16", "grad": "bf16",
         "in_out": False, "bias": False, "ignored": 0.1, "gradients": True},
        # The hidden activation of an MLP of width 2048, kept for the backward pass and read again.
        {"name": "pack_hidden", "kind": "pack", "rows": 8192, "features": 8192, "type": "bf16"},
        # GELU's gradient from it, ragged and in float32.
        {"name": "act_ragged", "kind": "act", "rows": 3001, "features": 4001, "type": "f32", "activation": "gelu"},
        # The second weight of that MLP: 8192 x 2048 from 8192 tokens.
        {"name": "wgrad_down", "kind": "wgrad", "rows": 8192, "features": 8192, "out": 2048, "type": "bf16", "grad": "bf16",
         "activation": "none", "out_in": False, "bias": False},
        # A ragged layer (out, in) with float32 gradients behind SiLU.
        {"name": "wgrad_ragged", "kind": "wgrad", "rows": 999, "features": 1000, "out": 331, "type": "f32", "grad": "f32",
         "activation": "silu", "out_in": True, "bias": True},
        # One sequence of a small model, forward only.
        {"name": "norm_small", "kind": "norm", "rows": 128, "features": 512, "type": "bf16", "post": "rms", "pre": "rms",
         "gates": 1, "backward": False},
        # A training step's tokens at width 2048: RMS norms on both sides, gate per channel, both directions.
        {"name": "norm_train", "kind": "norm", "rows": 16384, "features": 2048, "type": "bf16", "post": "rms", "pre": "rms",
         "gates": 1, "backward": True},
        # Layer norm before the next block only, float32, odd width, gates of 3 samples.
        {"name": "norm_ragged", "kind": "norm", "rows": 3003, "features": 1001, "type": "f32", "post": "none", "pre": "layer",
         "gates": 3, "backward": True},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _width(rng, lo, hi):
    """A size, half of the time a multiple of 64."""
    n = _log(rng, lo, hi)
    return max(64, n // 64 * 64) if rng.random() < 0.5 else n


def draw(rng):
    kind = rng.choice(["head", "head", "pack", "act", "wgrad", "wgrad", "norm", "norm"])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    if kind == "head":
        features, classes = _width(rng, 32, 4096), _width(rng, 10, 131072)
        most = 8192 * 2048 * 131072 // (8 if dtype == "f32" else 1)
        rows = max(1, min(_log(rng, 1, 8192), most // (features * classes)))
        return {"kind": kind, "rows": rows, "features": features, "classes": classes, "type": dtype,
                "grad": "f32" if dtype == "f32" else rng.choice(["bf16", "bf16", "f32"]), "in_out": rng.random() < 0.4,
                "bias": rng.random() < 0.4, "ignored": rng.choice([0.0, 0.1, 0.5]), "gradients": rng.random() < 0.8}
    if kind == "wgrad":
        return {"kind": kind, "rows": _log(rng, 1, 16384), "features": _width(rng, 16, 8192), "out": _width(rng, 16, 8192),
                "type": dtype, "grad": "f32" if dtype == "f32" else rng.choice(["bf16", "bf16", "f32"]),
                "activation": rng.choice(["none", "none", "relu", "gelu", "silu"]), "out_in": rng.random() < 0.4,
                "bias": rng.random() < 0.4}
    features = _width(rng, 16, 8192)
    rows = max(1, min(_log(rng, 1, 32768), (1 << 26) // features))
    if kind == "pack":
        return {"kind": kind, "rows": rows, "features": features, "type": dtype}
    if kind == "act":
        return {"kind": kind, "rows": rows, "features": features, "type": dtype, "activation": rng.choice(["relu", "gelu", "silu"])}
    gates = rng.choice([0, 1, 1, 4])
    if gates > 1:
        rows = max(gates, rows // gates * gates)
    post, pre = rng.choice([("rms", "rms"), ("none", "rms"), ("none", "layer"), ("layer", "layer"), ("rms", "none")])
    return {"kind": kind, "rows": rows, "features": features, "type": dtype, "post": post, "pre": pre, "gates": gates,
            "backward": rng.random() < 0.7}


# ----------------------------------------------------------------------------
# Inputs
# ----------------------------------------------------------------------------
EPSILON, ALPHA = 1e-5, 0.5


def _inputs(case, seed):
    dev = torch.device("cuda", 0)
    gen = torch.Generator(device=dev)
    gen.manual_seed(seed)
    n, d, dtype = case["rows"], case["features"], TYPES[case["type"]]

    def normal(*shape, sigma=1.0):
        return torch.randn(shape, generator=gen, device=dev).mul_(sigma)

    s = {}
    if case["kind"] == "head":
        v = case["classes"]
        w = normal(v, d, sigma=2.0 / math.sqrt(d))
        t = torch.randint(0, v, (n,), generator=gen, device=dev)
        # hidden states after a norm, that have learned something of their target
        s["x"] = (normal(n, d) + w[t]).to(dtype)
        w = w.to(dtype)
        s["w"] = w.t().contiguous().t() if case["in_out"] else w        # (in, out) in memory, seen as (out, in)
        s["bias"] = normal(v, sigma=0.5) if case["bias"] else None
        t[torch.rand((n,), generator=gen, device=dev) < case["ignored"]] = -100
        s["targets"], s["weight"] = t, torch.rand((n,), generator=gen, device=dev) + 0.5
        return s
    if case["kind"] == "norm":
        # a residual stream: features of different size, some of them far out
        size = normal(d).mul_(0.5).exp_()
        size[::97] *= 20.0
        s["r"] = (normal(n, d) * size).to(dtype)
        s["f"] = normal(n, d, sigma=0.7).to(dtype)
        s["gate"] = normal(case["gates"], d, sigma=0.5) if case["gates"] else None
        for side in ("post", "pre"):
            s["w_" + side] = normal(d, sigma=0.1) + 1.0 if case[side] != "none" else None
            s["b_" + side] = normal(d, sigma=0.1) if case[side] == "layer" else None
        if case["backward"]:
            s["dr_out"] = normal(n, d, sigma=1e-3).to(dtype)
            s["dh"] = normal(n, d, sigma=1e-3).to(dtype) if case["pre"] != "none" else None
        return s
    # activations: tokens and features of different size
    size = normal(d).mul_(0.5).exp_()
    s["x"] = (normal(n, d) * size * normal(n, 1).mul_(0.3).exp_()).to(dtype)
    if case["kind"] == "act":
        s["dy"] = normal(n, d, sigma=1e-3).to(dtype)
    if case["kind"] == "wgrad":
        s["dy"] = normal(n, case["out"], sigma=1e-3).to(dtype)
    return s


def prepare(case, seed):
    s = _inputs(case, seed)
    if case["kind"] in ("act", "wgrad"):
        # what the forward pass has left: the checkpoint
        if own:
            from paper_2309_06497_amd import binding as B
            s["x"] = B.shampoo_checkpoint_pack(s["x"])
        else:
            s["x"] = _quantize(s["x"])
    return case, s


# ----------------------------------------------------------------------------
# The plain form
# ----------------------------------------------------------------------------
def _power(e):
    """2^e in float32, -126 <= e <= 127"""
    return ((e + 127) << 23).to(torch.int32).view(torch.float32)


def _quantize(x):
    """Codes (int8) and exponents (int32) of x [n, d]: groups of 32 features share a power of two 2^s, a code is x / 2^s rounded to
    even, and s is the smallest that keeps the codes within 127.  Groups below 2^-100 are zero."""
    n, d = x.shape
    x = torch.nn.functional.pad(x.float(), (0, -d % GROUP)).view(n, -1, GROUP)
    bits = x.abs().amax(2).view(torch.int32)
    e = ((bits + 0x10000) >> 23) - 127                  # largest = 2^e (1 ... 1.992), or the next e above that
    e = torch.where(e < -100, torch.full_like(e, -100), e)
    q = torch.round(x * _power(6 - e)[:, :, None])
    q = torch.where((bits < (27 << 23))[:, :, None], torch.zeros_like(q), q)
    return q.to(torch.int8), e - 6, d


def _values(packed):
    q, s, d = packed
    return (q.float() * _power(s)[:, :, None]).view(q.shape[0], -1)[:, :d]


def _activation(z, name):
    if name == "relu":
        return torch.where(z > 0, z, torch.zeros_like(z))
    if name == "gelu":
        return 0.5 * z * (1.0 + torch.erf(z * math.sqrt(0.5)))
    if name == "silu":
        return z / (1.0 + torch.exp(-z))
    return z


def _slope(z, name):
    if name == "relu":
        return torch.where(z > 0, torch.ones_like(z), torch.zeros_like(z))
    if name == "gelu":
        return 0.5 * (1.0 + torch.erf(z * math.sqrt(0.5))) + z * torch.exp(-0.5 * z * z) * (1.0 / math.sqrt(2.0 * math.pi))
    s = 1.0 / (1.0 + torch.exp(-z))
    return s * (1.0 + z * (1.0 - s))


def _head(case, s):
    x, w, t = s["x"].float(), s["w"].float(), s["targets"]
    z = x @ w.t()
    if s["bias"] is not None:
        z = z + s["bias"]
    m = z.amax(1, keepdim=True)
    p = torch.exp(z - m)
    total = p.sum(1, keepdim=True)
    valid = (t >= 0) & (t < case["classes"])
    at = torch.where(valid, t, torch.zeros_like(t))[:, None]
    loss = (torch.log(total) + m - z.gather(1, at))[:, 0]
    loss = torch.where(valid, loss, torch.zeros_like(loss))
    if not case["gradients"]:
        return (loss,)
    del z
    g = torch.where(valid, s["weight"] * (1.0 / case["rows"]), torch.zeros_like(loss))[:, None]
    p *= g / total
    p.scatter_add_(1, at, -g)
    grad = TYPES[case["grad"]]
    out = [loss, (p @ w).to(TYPES[case["type"]]), (p.t() @ x).to(grad)]
    if case["in_out"]:
        out[2] = out[2].t().contiguous().t()
    return tuple(out + ([p.sum(0)] if s["bias"] is not None else []))


def _wgrad(case, s):
    a, dy = _activation(_values(s["x"]), case["activation"]), s["dy"].float()
    dw = ((dy.t() @ a) if case["out_in"] else (a.t() @ dy)).to(TYPES[case["grad"]])
    return (dw, dy.sum(0)) if case["bias"] else (dw,)


def _normed(x, kind):
    """x minus its mean where that is taken out, over its root mean square, and one over that"""
    if kind == "layer":
        x = x - x.mean(1, keepdim=True)
    inv = torch.rsqrt((x * x).mean(1, keepdim=True) + EPSILON)
    return x * inv, inv


def _norm(x, kind, w, b):
    if kind == "none":
        return x
    y = _normed(x, kind)[0] * w
    return y + b if b is not None else y


def _norm_backward(x, kind, w, dy):
    """Gradients of x, w and b of _norm"""
    n, inv = _normed(x, kind)
    g = dy * w
    dx = g - n * (g * n).mean(1, keepdim=True)
    if kind == "layer":
        dx = dx - g.mean(1, keepdim=True)
    return dx * inv, (dy * n).sum(0), dy.sum(0)


def _norm_pass(case, s, r, f, dr_out, dh):
    """Forward outputs on r and f, then the gradients on what the checkpoints hold of them, all in the precision of the inputs"""
    n, d = r.shape
    gate = None
    if s["gate"] is not None:
        gate = s["gate"].to(r.dtype).repeat_interleave(n // case["gates"], 0)
    w = {k: s[k].to(r.dtype) if s[k] is not None else None for k in ("w_post", "b_post", "w_pre", "b_pre")}

    def forward(r, f):
        u = _norm(f, case["post"], w["w_post"], w["b_post"])
        return u, r + ALPHA * (u if gate is None else gate * u)

    r_out = forward(r, f)[1]
    out = [r_out]
    if case["pre"] != "none":
        out.append(_norm(r_out, case["pre"], w["w_pre"], w["b_pre"]))
    if not case["backward"]:
        return out
    r, f = (_values(_quantize(v)).to(v.dtype) for v in (r, f))
    u, r_out = forward(r, f)
    total, tail = dr_out, []
    if case["pre"] != "none":
        dx, dw, db = _norm_backward(r_out, case["pre"], w["w_pre"], dh)
        total, tail = dr_out + dx, [dw] + ([db] if case["pre"] == "layer" else [])
    df = ALPHA * total
    middle = []
    if gate is not None:
        middle.append((df * u).view(case["gates"], -1, d).sum(1))
        df = df * gate
    if case["post"] != "none":
        df, dw, db = _norm_backward(f, case["post"], w["w_post"], df)
        middle += [dw] + ([db] if case["post"] == "layer" else [])
    return out + [total, df] + middle + tail


def _rounded(case, outputs):
    """Tokens by features in the type of the inputs, gradients of weights in float32"""
    dtype = TYPES[case["type"]]
    shape = (case["rows"], case["features"])
    first = 1 + (case["pre"] != "none") + (2 if case["backward"] else 0)
    assert all(tuple(o.shape) == shape for o in outputs[:first])
    return tuple(o.to(dtype) for o in outputs[:first]) + tuple(outputs[first:])


# ----------------------------------------------------------------------------
# One pass
# ----------------------------------------------------------------------------
def run(state):
    case, s = state
    if own:
        return _run_own(case, s)
    kind = case["kind"]
    if kind == "head":
        return _head(case, s)
    if kind == "pack":
        return _values(_quantize(s["x"])).to(TYPES[case["type"]])
    if kind == "act":
        return (s["dy"].float() * _slope(_values(s["x"]), case["activation"])).to(TYPES[case["type"]])
    if kind == "wgrad":
        return _wgrad(case, s)
    wide = [s[k].float() if s.get(k) is not None else None for k in ("r", "f", "dr_out", "dh")]
    return _rounded(case, _norm_pass(case, s, *wide))


def _run_own(case, s):
    from paper_2309_06497_amd import binding as B
    kind = case["kind"]
    if kind == "head":
        out = B.shampoo_linear_cross_entropy(s["x"], s["w"], s["targets"], bias=s["bias"], weight=s["weight"],
                                             scale=1.0 / case["rows"], grad_dtype=TYPES[case["grad"]], gradients=case["gradients"])
        return tuple(o for o in out if o is not None) if case["gradients"] else (out,)
    if kind == "pack":
        return B.shampoo_checkpoint_unpack(B.shampoo_checkpoint_pack(s["x"]), dtype=TYPES[case["type"]])
    if kind in ("act", "wgrad"):
        activation = {"none": B.ACT_NONE, "relu": B.ACT_RELU, "gelu": B.ACT_GELU, "silu": B.ACT_SILU}[case["activation"]]
    if kind == "act":
        return B.shampoo_checkpoint_activation_grad(s["x"], s["dy"], activation)
    if kind == "wgrad":
        out = B.shampoo_checkpoint_weight_grad(s["x"], s["dy"], activation=activation, grad_dtype=TYPES[case["grad"]],
                                               out_in=case["out_in"], bias=case["bias"])
        return out if case["bias"] else (out,)
    norms = {"none": B.NORM_NONE, "rms": B.NORM_RMS, "layer": B.NORM_LAYER}
    options = dict(post=norms[case["post"]], pre=norms[case["pre"]], w_post=s["w_post"], b_post=s["b_post"], gate=s["gate"],
                   w_pre=s["w_pre"], b_pre=s["b_pre"], epsilon=EPSILON, scale=ALPHA)
    if not case["backward"]:
        r_out, h = B.shampoo_residual_norm_forward(s["r"], s["f"], **options)
        return (r_out, h) if h is not None else (r_out,)
    r_out, h, r8, f8 = B.shampoo_residual_norm_forward(s["r"], s["f"], checkpoint=True, **options)
    g = B.shampoo_residual_norm_backward(r8, f8, s["dr_out"], s["dh"], **options)
    names = ("dr", "df", "dgate", "dw_post", "db_post", "dw_pre", "db_pre")
    return tuple(t for t in (r_out, h, *(g[k] for k in names)) if t is not None)


# ----------------------------------------------------------------------------
# The definitions in 64 bits
# ----------------------------------------------------------------------------
def _exact_values(x):
    """What a checkpoint holds of x, by trying exponents: the smallest s with all of round(x 2^-s) within 127"""
    n, d = x.shape
    x = torch.nn.functional.pad(x.double(), (0, -d % GROUP)).view(n, -1, GROUP)
    largest = x.abs().amax(2, keepdim=True)
    s = torch.floor(torch.log2(largest.clamp(min=2.0 ** -110))) - 8
    for _ in range(3):
        s = torch.where(torch.round(largest * torch.exp2(-s)) > 127, s + 1, s)
    v = torch.round(x * torch.exp2(-s)) * torch.exp2(s)
    return torch.where(largest < 2.0 ** -100, torch.zeros_like(v), v).view(n, -1)[:, :d]


def _exact_activation(z, name):
    """The function and its derivative"""
    if name == "none":
        return z, torch.ones_like(z)
    if name == "relu":
        return z.clamp(min=0), (z > 0).double()
    if name == "silu":
        s = torch.sigmoid(z)
        return z * s, s + z * s * (1 - s)
    phi = 0.5 * torch.special.erfc(-z / math.sqrt(2))
    return z * phi, phi + z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi)


def _exact_head(case, s):
    x, w, t = s["x"].double(), s["w"].double(), s["targets"]
    valid = (t >= 0) & (t < case["classes"])
    rows = torch.arange(case["rows"], device=t.device)[valid]
    z = x @ w.t()
    if s["bias"] is not None:
        z += s["bias"].double()
    lse = torch.logsumexp(z, 1)
    loss = torch.zeros_like(lse)
    loss[rows] = lse[rows] - z[rows, t[rows]]
    if not case["gradients"]:
        return (loss,)
    g = z.sub_(lse[:, None]).exp_()
    g[rows, t[rows]] -= 1.0
    g *= (valid * s["weight"].double() / case["rows"])[:, None]
    dw = x.t() @ g if case["in_out"] else g.t() @ x
    return (loss, g @ w, dw.t() if case["in_out"] else dw) + ((g.sum(0),) if s["bias"] is not None else ())


def exact(case, seed):
    s = _inputs(case, seed)
    kind = case["kind"]
    if kind == "head":
        return _exact_head(case, s)
    if kind == "pack":
        return _exact_values(s["x"])
    if kind == "act":
        return s["dy"].double() * _exact_activation(_exact_values(s["x"]), case["activation"])[1]
    if kind == "wgrad":
        a, dy = _exact_activation(_exact_values(s["x"]), case["activation"])[0], s["dy"].double()
        dw = dy.t() @ a if case["out_in"] else a.t() @ dy
        return (dw, dy.sum(0)) if case["bias"] else (dw,)
    return _exact_norm(case, s)


def _exact_norm(case, s):
    """The gradients by differentiating the forward pass"""
    n, d = case["rows"], case["features"]
    leaf = {k: s[k].double().requires_grad_() for k in ("gate", "w_post", "b_post", "w_pre", "b_pre") if s[k] is not None}

    def norm(x, side):
        if case[side] == "none":
            return x
        if case[side] == "layer":
            x = x - x.mean(1, keepdim=True)
        y = x / torch.sqrt(x.square().mean(1, keepdim=True) + EPSILON) * leaf["w_" + side]
        return y + leaf["b_" + side] if "b_" + side in leaf else y

    def forward(r, f):
        u = norm(f, "post")
        if "gate" in leaf:
            u = (u.view(case["gates"], -1, d) * leaf["gate"][:, None]).view(n, d)
        r_out = r + ALPHA * u
        return (r_out, norm(r_out, "pre")) if case["pre"] != "none" else (r_out,)

    with torch.no_grad():
        out = forward(s["r"].double(), s["f"].double())
    if not case["backward"]:
        return out
    r, f = (_exact_values(s[k]).requires_grad_() for k in ("r", "f"))
    with torch.enable_grad():
        seen = forward(r, f)
        value = sum((a * b.double()).sum() for a, b in zip(seen, (s["dr_out"], s["dh"])))
        leaves = [r, f] + [leaf[k] for k in ("gate", "w_post", "b_post", "w_pre", "b_pre") if k in leaf]
        return tuple(out) + torch.autograd.grad(value, leaves)


# ----------------------------------------------------------------------------
# What a pass cannot do without
# ----------------------------------------------------------------------------
def work(case):
    """Each input read once and each output written once; a checkpoint is 33 / 32 byte per element.  Operations: the products
    (logits and both gradients); a few per element where there are none."""
    n, d, b = float(case["rows"]), float(case["features"]), 4.0 if case["type"] == "f32" else 2.0
    if case["kind"] == "head":
        v, g = float(case["classes"]), 4.0 if case["grad"] == "f32" else 2.0
        if not case["gradients"]:
            return {"bytes": b * (n + v) * d + 12 * n, "flops": 2 * n * d * v}
        return {"bytes": 2 * b * n * d + (b + g) * v * d + 16 * n, "flops": 6 * n * d * v}
    packed = 33.0 / 32.0
    if case["kind"] == "pack":
        return {"bytes": 2 * b * n * d, "flops": 4 * n * d}
    if case["kind"] == "act":
        return {"bytes": (packed + 2 * b) * n * d, "flops": 16 * n * d}
    if case["kind"] == "wgrad":
        m, g = float(case["out"]), 4.0 if case["grad"] == "f32" else 2.0
        return {"bytes": packed * n * d + b * n * m + g * d * m, "flops": 2 * n * d * m}
    outputs = 1 + (case["pre"] != "none")
    if not case["backward"]:
        return {"bytes": (2 + outputs) * b * n * d, "flops": 12 * n * d}
    return {"bytes": (2 + 2 * outputs + 2) * b * n * d, "flops": 48 * n * d}
