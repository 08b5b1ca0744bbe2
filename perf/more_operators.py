"""The operators around a training step that work on given logits and on all tensors of a model at once, as cases that can be timed.

  "logp"       log probabilities of given tokens, the entropy of every row and its most probable tokens, from logits
  "logp_grad"  the gradient of the logits from those of the log probabilities and of the entropy
  "adamw"      an AdamW step of all parameters, with states in 32 or in 8 bits, bf16 copies of the parameters, gradients limited by their norm
  "grad_norm"  the norm of all gradients together, and of each tensor's

`own` chooses between the package's kernels and the plain form: elementary torch operations in float32."""
import math

import torch

own = False        # True: the calls of the package; False: the plain form

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
GROUP = 128        # neighbouring elements of a tensor that share the scales of their 8-bit states


def listed():
    return [
        # One token of one sequence while it is generated: its log probability and 20 alternatives.
        {"name": "logp_token", "kind": "logp", "rows": 1, "classes": 131072, "type": "bf16", "tokens": 1, "top": 20, "temperature": 1.0,
         "masked": 0.0, "ignored": 0.0},
        # Scoring sampled answers under a vocabulary of ordinary size: the given tokens and the entropy, no alternatives.
        {"name": "logp_score", "kind": "logp", "rows": 4096, "classes": 32000, "type": "bf16", "tokens": 1, "top": 0, "temperature": 1.0,
         "masked": 0.0, "ignored": 0.2},
        # Nothing divides: float32, an odd vocabulary of which a grammar forbids a third, four candidates a row, a temperature.
        {"name": "logp_ragged", "kind": "logp", "rows": 999, "classes": 50001, "type": "f32", "tokens": 4, "top": 5, "temperature": 0.7,
         "masked": 0.3, "ignored": 0.1},
        # The largest: a teacher's 20 most probable tokens of every position, a multilingual vocabulary.
        {"name": "logp_large", "kind": "logp", "rows": 8192, "classes": 131072, "type": "bf16", "tokens": 1, "top": 20, "temperature": 1.0,
         "masked": 0.0, "ignored": 0.1},
        # The backward pass of that scoring: advantages on the given tokens and a bonus for entropy.
        {"name": "grad_score", "kind": "logp_grad", "rows": 4096, "classes": 32000, "type": "bf16", "tokens": 1, "temperature": 1.0,
         "masked": 0.0, "ignored": 0.2, "entropy": True},
        # Distillation onto 16 given tokens of every position, float32, odd sizes.
        {"name": "grad_ragged", "kind": "logp_grad", "rows": 999, "classes": 50001, "type": "f32", "tokens": 16, "temperature": 2.0,
         "masked": 0.3, "ignored": 0.1, "entropy": False},
        # The gates and norm weights of 64 blocks, which Shampoo has no factors for: 192 vectors in one call.
        {"name": "adamw_vectors", "kind": "adamw", "layers": 64, "width": 512, "classes": 0, "matrices": False, "params": "f32", "grads": "f32",
         "bits": 32, "copies": False, "clip": False},
        # A residual MLP of width 2048 and its head: float32 parameters, bf16 gradients and copies, states in 32 bits.
        {"name": "adamw_mlp", "kind": "adamw", "layers": 4, "width": 2048, "classes": 32000, "matrices": True, "params": "f32", "grads": "bf16",
         "bits": 32, "copies": True, "clip": True},
        # Odd sizes, so that tensors begin and groups end anywhere: bf16 parameters with states in 8 bits.
        {"name": "adamw_ragged", "kind": "adamw", "layers": 5, "width": 331, "classes": 5003, "matrices": True, "params": "bf16", "grads": "f32",
         "bits": 8, "copies": False, "clip": True},
        # The largest: twelve layers and the head of a multilingual vocabulary, states in 8 bits.
        {"name": "adamw_large", "kind": "adamw", "layers": 12, "width": 2048, "classes": 131072, "matrices": True, "params": "f32", "grads": "bf16",
         "bits": 8, "copies": True, "clip": False},
        # Its gradients' norms, and those of many small odd tensors.
        {"name": "norm_large", "kind": "grad_norm", "layers": 12, "width": 2048, "classes": 131072, "matrices": True, "grads": "bf16"},
        {"name": "norm_ragged", "kind": "grad_norm", "layers": 60, "width": 131, "classes": 999, "matrices": True, "grads": "f32"},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _width(rng, lo, hi):
    """A size, half of the time a multiple of 64."""
    n = _log(rng, lo, hi)
    return max(64, n // 64 * 64) if rng.random() < 0.5 else n


def draw(rng):
    kind = rng.choice(["logp", "logp", "logp", "logp_grad", "logp_grad", "adamw", "adamw", "adamw", "grad_norm"])
    if kind.startswith("logp"):
        dtype, classes = rng.choice(["bf16", "bf16", "f32"]), _width(rng, 32, 131072)
        rows = min(_log(rng, 1, 8192), (8192 * 131072 if dtype == "bf16" else 4096 * 131072) // (classes * (2 if kind == "logp_grad" else 1)))
        case = {"kind": kind, "rows": rows, "classes": classes, "type": dtype, "tokens": rng.choice([1, 1, 1, 4, 16]),
                "temperature": rng.choice([1.0, 1.0, 0.7, 2.0]), "masked": rng.choice([0.0, 0.0, 0.3, 0.9]), "ignored": rng.choice([0.0, 0.1, 0.5])}
        if kind == "logp":
            case["top"] = min(classes, rng.choice([0, 1, 5, 20, 64]))
        else:
            case["entropy"] = rng.random() < 0.6
        return case
    matrices, width, classes = rng.random() < 0.8, _width(rng, 32, 2048), rng.choice([0, _width(rng, 10, 131072)])
    layers = _log(rng, 1, 60)
    while matrices and layers > 1 and 8 * layers * width * width + classes * width > 600e6:
        layers -= 1
    case = {"kind": kind, "layers": layers, "width": width, "classes": classes, "matrices": matrices, "grads": rng.choice(["bf16", "bf16", "f32"])}
    if kind == "adamw":
        case["params"] = rng.choice(["f32", "f32", "bf16"])
        case["bits"], case["copies"], case["clip"] = rng.choice([8, 32]), case["params"] == "f32" and rng.random() < 0.5, rng.random() < 0.5
    return case


# ----------------------------------------------------------------------------
# Inputs
# ----------------------------------------------------------------------------
BETA1, BETA2, EPSILON, DECAY, LR, MAX_NORM = 0.9, 0.999, 1e-8, 0.1, 1e-3, 1.0
START = 100        # steps that the optimizer has taken before


def _shapes(case):
    """Matrices first: they decay, the vectors do not."""
    d, n = case["width"], case["layers"]
    matrices = [s for _ in range(n) for s in ((d, 4 * d), (4 * d, d))] if case["matrices"] else []
    return matrices + ([(case["classes"], d)] if case["classes"] else []), [(d,) for _ in range(3 * n)]


def _views(flat, shapes):
    at, out = 0, []
    for s in shapes:
        n = math.prod(s)
        out.append(flat[at:at + n].view(s))
        at += n
    return out


def _inputs(case, seed):
    dev = torch.device("cuda", 0)
    gen = torch.Generator(device=dev)
    gen.manual_seed(seed)

    def normal(*shape, sigma=1.0):
        return torch.randn(shape, generator=gen, device=dev).mul_(sigma)

    s = {}
    if case["kind"].startswith("logp"):
        n, v, m = case["rows"], case["classes"], case["tokens"]
        t = torch.randint(0, v, (n, m), generator=gen, device=dev)
        # logits that have learned something of the first token: some rows sure, some not
        z = normal(n, v, sigma=2.0)
        z.scatter_add_(1, t[:, :1], normal(n, 1, sigma=4.0).abs_().add_(3.0))
        if case["masked"]:
            z.masked_fill_(torch.rand((1, v), generator=gen, device=dev) < case["masked"], -math.inf)
            if n > 2:
                z[n // 2] = -math.inf                     # a row that the grammar leaves nothing
        s["logits"] = z.to(TYPES[case["type"]])
        ignored = torch.rand((n, m), generator=gen, device=dev) < case["ignored"]
        ignored[0, 0] = False
        t[ignored] = -100
        s["tokens"] = t
        if case["kind"] == "logp_grad":
            s["d_log_probs"] = normal(n, m, sigma=1.0 / n)
            s["d_entropy"] = torch.full((n,), 0.01 / n, device=dev) if case["entropy"] else None
        return s
    matrices, vectors = _shapes(case)
    shapes = matrices + vectors
    total = sum(math.prod(x) for x in shapes)
    # gradients of tensors and elements of different size, some elements not reached at all
    size = normal(total).exp_().mul_(1e-3)
    for k, x in enumerate(_views(size, shapes)):
        x.mul_(4.0 ** (k % 5 - 2))
    g = normal(total).mul_(size)
    g[torch.rand((total,), generator=gen, device=dev) < 0.05] = 0.0
    s["g"], s["shapes"] = g.to(TYPES[case["grads"]]), shapes
    del g
    s["decayed"] = sum(math.prod(x) for x in matrices)
    s["grads"] = _views(s["g"], shapes)
    if case["kind"] == "adamw":
        s["p"] = normal(total, sigma=0.02).to(TYPES[case["params"]])
        s["params"] = _views(s["p"], shapes)
        s["m"] = normal(total, sigma=0.3).mul_(size)
        s["v"] = normal(total).square_().add_(0.5).mul_(size.square_())
        s["step"] = START
        if case["copies"]:
            s["c"] = s["p"].to(torch.bfloat16)
            s["copies"] = _views(s["c"], shapes)
        if case["bits"] == 8:
            # states that 8 bits hold: those of an optimizer that has run
            s["slots"] = _slots(shapes, dev)
            s["m"], s["v"] = _state8(s["m"], s["slots"], 113, 0x80000), _state8(s["v"], s["slots"], 97, 0x80000)
    return s


def prepare(case, seed):
    s = _inputs(case, seed)
    if case["kind"] == "logp_grad":
        # what the forward pass has left
        if own:
            from paper_2309_06497_amd import binding as B
            s["forward"] = B.shampoo_log_probs(s["logits"], s["tokens"], temperature=case["temperature"])
        else:
            s["forward"] = _statistics(case, s)
    if case["kind"] == "adamw" and own:
        from paper_2309_06497_amd import binding as B
        codes = {"f32": B.GRAD_F32, "bf16": B.GRAD_BF16}
        s["opt"] = B.AdamW(s["shapes"], beta1=BETA1, beta2=BETA2, epsilon=EPSILON, weight_decay=DECAY, decay=[len(x) > 1 for x in s["shapes"]],
                           state_bits=case["bits"], param_dtype=codes[case["params"]], grad_dtype=codes[case["grads"]])
        s["opt"].load(s["m"], s["v"])
        del s["m"], s["v"]
    return case, s


# ----------------------------------------------------------------------------
# The plain form: logits
# ----------------------------------------------------------------------------
def _statistics(case, s):
    """Of every row: the largest logit, the log of the sum of exp((z - largest) / T), that sum, and the entropy"""
    z, tau = s["logits"].float(), 1.0 / case["temperature"]
    m = z.amax(1, keepdim=True)
    m = torch.where(m == -math.inf, torch.zeros_like(m), m)
    d = (z - m).mul_(tau)
    e = torch.exp(d)
    total = e.sum(1, keepdim=True)
    log_total = torch.log(total)
    d.mul_(e)
    entropy = log_total - d.masked_fill_(e == 0, 0.0).sum(1, keepdim=True) / total
    return m, log_total, total, torch.where(total > 0, entropy, torch.zeros_like(entropy))


def _given(case, s):
    """Whether a token is one, and the place of its logit"""
    t = s["tokens"]
    valid = (t >= 0) & (t < case["classes"])
    return valid, torch.where(valid, t, torch.zeros_like(t))


def _log_probs(case, s):
    m, log_total, total, entropy = _statistics(case, s)
    tau = 1.0 / case["temperature"]
    valid, at = _given(case, s)
    nothing = torch.full_like(log_total, -math.inf)

    def log_prob(z):
        x = (z - m) * tau - log_total
        return torch.where(z == -math.inf, nothing, x)

    lp = log_prob(s["logits"].gather(1, at).float())
    out = {"log_probs": torch.where(valid, lp, torch.zeros_like(lp)), "entropy": entropy[:, 0]}
    if case["top"]:
        # the order of the logits as they are given, ties to the lowest token: keys of which no two are alike
        bits = (s["logits"].float() + 0.0).view(torch.int32).to(torch.int64)
        key = torch.where(bits < 0, -(bits & 0x7FFFFFFF), bits).mul_(1 << 32).sub_(torch.arange(case["classes"], device=bits.device))
        del bits
        at = -torch.topk(key, case["top"], dim=1).values & 0xFFFFFFFF
        del key
        z = s["logits"].gather(1, at).float()
        out["top_tokens"] = torch.where(z == -math.inf, torch.full_like(at, -1), at)
        out["top_log_probs"] = log_prob(z)
    return out


def _log_probs_grad(case, s):
    m, log_total, total, entropy = s["forward"]
    tau = 1.0 / case["temperature"]
    valid, at = _given(case, s)
    a = torch.where(valid, s["d_log_probs"], torch.zeros_like(s["d_log_probs"]))
    weight = a.sum(1, keepdim=True).expand(-1, case["classes"])
    x = (s["logits"].float() - m).mul_(tau).sub_(log_total)
    p = torch.exp(x)
    if s["d_entropy"] is not None:
        weight = weight + s["d_entropy"][:, None] * (x + entropy)
    g = torch.where(p > 0, p * weight, torch.zeros_like(p)).neg_()
    a = torch.where(total > 0, a, torch.zeros_like(a))
    return g.scatter_add_(1, at, a).mul_(tau).to(s["logits"].dtype)


# ----------------------------------------------------------------------------
# The plain form: all tensors of a model
# ----------------------------------------------------------------------------
def _slots(shapes, device):
    """Where an element lies when every tensor begins with a group of its own, and how many places there are"""
    sizes = torch.tensor([math.prod(x) for x in shapes], device=device)
    padded = (sizes + GROUP - 1) // GROUP * GROUP
    shift = torch.cumsum(padded, 0) - padded - (torch.cumsum(sizes, 0) - sizes)
    return torch.arange(int(sizes.sum()), device=device) + torch.repeat_interleave(shift, sizes), int(padded.sum())


def _power(e):
    """2^e in float32, -126 <= e <= 127 (int32)"""
    return ((e + 127) << 23).view(torch.float32)


def _state8(x, slots, shift, add):
    """The values that 8 bits hold of x.  2^E is the power of two of the largest of a group; |x| 2^-E is kept with three bits behind its first, in as many
    binades as `shift` leaves above float32's smallest (113: 14, 97: 30), below them as multiples of the smallest value.  `add` in units of
    2^-20 of a step: 1/2 to the nearest, otherwise what a random number would be.  With 30 binades (squares) nothing but 0 becomes 0.  Groups below 2^-100 are zero."""
    slot, places = slots
    groups = torch.zeros(places, device=x.device)
    groups[slot] = x.abs()
    e = ((groups.view(-1, GROUP).amax(1).view(torch.int32) >> 23) - 127)[slot // GROUP]
    y = x.abs() * _power(-e) * 2.0 ** -shift
    code = (y.view(torch.int32) + add) >> 20
    if shift == 97:
        code = torch.where((code == 0) & (x > 0), torch.ones_like(code), code)
    value = (code << 20).view(torch.float32) * 2.0 ** shift * _power(e)
    return torch.copysign(torch.where(e < -100, torch.zeros_like(value), value), x)


def _low(x):
    return x & 0xFFFFFFFF


def _offsets(total, step, device):
    """Offsets of the roundings of element i in this step: of m and v in 2^-20, of a bf16 parameter in 2^-16"""
    i = torch.arange(total, device=device)
    x = _low(_low(i) * 0x9E3779B9 + (i >> 32) * 0xBB67AE85 + step * 0x6A09E667)
    del i
    x = _low((x ^ (x >> 16)) * 0xBB67AE85)
    x = _low((x ^ (x >> 15)) * 0xA54FF53B)
    x = x ^ (x >> 16)
    y = _low(x * 0x9E3779B9 + 0x6A09E667)
    y = y ^ (y >> 15)
    return (x >> 12).to(torch.int32), (y >> 12).to(torch.int32), (y & 0xFFFF).to(torch.int32)


def _norms(s):
    """Sums in 64 bits"""
    squares = torch.stack([g.double().square().sum() for g in s["grads"]])
    return squares.sum().sqrt().float(), squares.sqrt().float()


def _adamw(case, s):
    t, out, total = s["step"], {}, s["p"].numel()
    s["step"] = t + 1
    g = s["g"].float()
    if case["clip"]:
        out["norm"] = norm = _norms(s)[0]
        g = g * torch.where(norm > MAX_NORM, MAX_NORM / norm, torch.ones_like(norm))
    m = s["m"] * BETA1 + g * (1.0 - BETA1)
    v = s["v"] * BETA2 + (g * (1.0 - BETA2)) * g
    u = torch.sqrt(v).mul_(1.0 / math.sqrt(1.0 - BETA2 ** (t + 1))).add_(EPSILON)
    u = m / u
    p = s["p"].float()
    p[:s["decayed"]] *= 1.0 - LR * DECAY
    p -= u.mul_(LR / (1.0 - BETA1 ** (t + 1)))
    del u, g
    if case["bits"] == 8 or case["params"] == "bf16":
        rm, rv, rp = _offsets(total, t, p.device)
    if case["bits"] == 8:
        s["m"].copy_(_state8(m, s["slots"], 113, rm))
        s["v"].copy_(_state8(v, s["slots"], 97, rv))
        out["m"], out["v"] = s["m"].to(torch.bfloat16), s["v"].to(torch.bfloat16)
    else:
        out["m"], out["v"] = s["m"].copy_(m), s["v"].copy_(v)
    if case["params"] == "bf16":
        p = ((p.view(torch.int32) + rp) >> 16).to(torch.int16).view(torch.bfloat16)
    out["params"] = s["p"].copy_(p)
    if case["copies"]:
        out["copies"] = s["c"].copy_(p)
    return out


# ----------------------------------------------------------------------------
# One pass
# ----------------------------------------------------------------------------
def run(state):
    case, s = state
    if own:
        return _run_own(case, s)
    if case["kind"] == "logp":
        return _log_probs(case, s)
    if case["kind"] == "logp_grad":
        return _log_probs_grad(case, s)
    return _adamw(case, s) if case["kind"] == "adamw" else _norms(s)


def _run_own(case, s):
    from paper_2309_06497_amd import binding as B
    if case["kind"] == "logp":
        r = B.shampoo_log_probs(s["logits"], s["tokens"], top=case["top"], temperature=case["temperature"])
        out = {"log_probs": r.log_probs, "entropy": r.entropy}
        if case["top"]:
            out["top_tokens"], out["top_log_probs"] = r.top_tokens, r.top_log_probs
        return out
    if case["kind"] == "logp_grad":
        return B.shampoo_log_probs_grad(s["logits"], s["tokens"], s["forward"], s["d_log_probs"], s["d_entropy"])
    if case["kind"] == "grad_norm":
        return B.shampoo_gradient_norm(s["grads"])
    out = {}
    if case["clip"]:
        out["norm"] = B.shampoo_gradient_norm(s["grads"])[0]
    s["opt"].step(s["params"], s["grads"], LR, s["step"], copies=s.get("copies"), norm=out.get("norm"), max_norm=MAX_NORM)
    s["step"] += 1
    out["m"], out["v"] = s["opt"].state()
    out["params"] = s["p"]
    if case["copies"]:
        out["copies"] = s["c"]
    return out


# ----------------------------------------------------------------------------
# The definitions in 64 bits
# ----------------------------------------------------------------------------
def exact(case, seed):
    s = _inputs(case, seed)
    if case["kind"] == "logp":
        return _exact_log_probs(case, s)
    if case["kind"] == "logp_grad":
        return _exact_log_probs_grad(case, s)
    if case["kind"] == "grad_norm":
        each = torch.stack([torch.linalg.vector_norm(g.double()) for g in s["grads"]])
        return torch.linalg.vector_norm(s["g"].double()), each
    return _exact_adamw(case, s)


def _exact_log_probs(case, s):
    n, v = case["rows"], case["classes"]
    lp = torch.log_softmax(s["logits"].double() / case["temperature"], 1)
    empty = torch.isnan(lp[:, 0])
    lp[empty] = -math.inf
    out = {"entropy": torch.where(empty, 0.0, torch.special.entr(torch.exp(lp)).sum(1))}
    given = torch.zeros(s["tokens"].shape, dtype=torch.float64, device=lp.device)
    rows, cols = ((s["tokens"] >= 0) & (s["tokens"] < v)).nonzero(as_tuple=True)
    given[rows, cols] = lp[rows, s["tokens"][rows, cols]]
    out["log_probs"] = given
    if case["top"]:
        out["top_tokens"], out["top_log_probs"] = None, torch.topk(lp, case["top"], 1).values
    return out


def _exact_log_probs_grad(case, s):
    """By rows at a time: d log p_t / d z = (onehot - p) / T,  d H / d z = -p (log p + H) / T"""
    v, out = case["classes"], []
    for i in range(0, case["rows"], 512):
        lp = torch.log_softmax(s["logits"][i:i + 512].double() / case["temperature"], 1)
        lp[torch.isnan(lp[:, 0])] = -math.inf
        p, t, a = torch.exp(lp), s["tokens"][i:i + 512], s["d_log_probs"][i:i + 512].double()
        g = torch.zeros_like(p)
        for j in range(case["tokens"]):
            ok = ((t[:, j] >= 0) & (t[:, j] < v) & (p.sum(1) > 0)).nonzero()[:, 0]
            g[ok] -= a[ok, j, None] * p[ok]
            g[ok, t[ok, j]] += a[ok, j]
        if s["d_entropy"] is not None:
            h = torch.special.entr(p).sum(1, keepdim=True)
            g += s["d_entropy"][i:i + 512, None].double() * (torch.special.entr(p) - p * h)
        out.append(g / case["temperature"])
    return torch.cat(out)


def _exact_state8(x, shapes, binades, offset):
    """A group at a time: multiples of the step of a value's binade, rounded down after `offset` of a step has been added"""
    out, at = torch.empty_like(x), 0
    for shape in shapes:
        n = math.prod(shape)
        v = torch.nn.functional.pad(x[at:at + n], (0, -n % GROUP)).view(-1, GROUP)
        o = torch.nn.functional.pad(offset[at:at + n], (0, -n % GROUP)).view(-1, GROUP)
        top = torch.frexp(v.abs().amax(1, keepdim=True)).exponent - 1
        e = torch.maximum(torch.frexp(v.abs()).exponent - 1, top - binades + 1)
        unit = torch.exp2((e - 3).double())
        q = torch.floor(v.abs() / unit + o)
        if binades == 30:
            q = torch.where((q == 0) & (v > 0), 1.0, q)
        q = torch.where(top < -100, 0.0, q * unit) * torch.sign(v)
        out[at:at + n] = q.view(-1)[:n]
        at += n
    return out


def _exact_adamw(case, s):
    t, out, total = s["step"], {}, s["p"].numel()
    g = s["g"].double()
    if case["clip"]:
        out["norm"] = torch.linalg.vector_norm(g)
        g *= min(1.0, MAX_NORM / float(out["norm"]))
    m = s["m"].double().mul_(BETA1).add_(g, alpha=1.0 - BETA1)
    v = s["v"].double().mul_(BETA2).addcmul_(g, g, value=1.0 - BETA2)
    p = s["p"].double()
    decay = torch.zeros(total, device=p.device, dtype=torch.float64)
    decay[:s["decayed"]] = LR * DECAY
    p -= decay.mul_(p) + LR * (m / (1.0 - BETA1 ** (t + 1))) / (torch.sqrt(v / (1.0 - BETA2 ** (t + 1))) + EPSILON)
    del decay, g
    out["m"], out["v"] = m, v
    if case["bits"] == 8:
        rm, rv, _ = _offsets(total, t, p.device)
        out["m"] = _exact_state8(m, s["shapes"], 14, rm.double() * 2.0 ** -20)
        out["v"] = _exact_state8(v, s["shapes"], 30, rv.double() * 2.0 ** -20)
    out["params"] = p
    if case["params"] == "bf16":
        at = torch.frexp(p).exponent.sub(8).double().exp2_()                    # the step of eight bits
        out["params"] = torch.sign(p) * torch.floor(p.abs() / at + _offsets(total, t, p.device)[2].double() * 2.0 ** -16) * at
    if case["copies"]:
        out["copies"] = p
    return out


# ----------------------------------------------------------------------------
# What a pass cannot do without
# ----------------------------------------------------------------------------
def work(case):
    """Each input read once and each output written once; states in 8 bits are 1 1/128 byte, and are written again as bf16 values.  Operations: a few per element."""
    if case["kind"].startswith("logp"):
        n, v, b, m = float(case["rows"]), float(case["classes"]), 4.0 if case["type"] == "f32" else 2.0, float(case["tokens"])
        if case["kind"] == "logp":
            return {"bytes": b * n * v + n * (12 * m + 4 + 12 * case["top"]), "flops": 6 * n * v}
        return {"bytes": 2 * b * n * v + n * (12 * m + 20), "flops": 8 * n * v}
    matrices, vectors = _shapes(case)
    n = float(sum(math.prod(x) for x in matrices + vectors))
    g = 4.0 if case["grads"] == "f32" else 2.0
    if case["kind"] == "grad_norm":
        return {"bytes": g * n + 4 * len(matrices + vectors), "flops": 2 * n}
    p = 4.0 if case["params"] == "f32" else 2.0
    state = 16.0 if case["bits"] == 32 else 4 * (1 + 1 / GROUP) + 4
    return {"bytes": (g * (2 if case["clip"] else 1) + 2 * p + state + (2 if case["copies"] else 0)) * n, "flops": 16 * n}
