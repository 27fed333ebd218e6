"""The operators of a block around its mixer: the norm of a mixer's output with
its gate, the residual addition with the norms on both sides of it, the gated
linear recurrence, and the gated feed-forward projections.  Their sizes,
inputs, one pass through each, the work a pass cannot do without, and a 64-bit
reference.

A case names an operator and its form (`kind`) and its sizes:
  gnorm-forward  hla.gated_norm over n tokens (n = 1: decoding)
  gnorm-train    the same with its gradients
  rnorm-forward  hla.residual_norm over n tokens
  rnorm-train    the same with its gradients
  glr-forward    hla.glr_forward over whole sequences
  glr-prompt     hla.glr_prefill from and into a state
  glr-step       hla.glr_step, one token a sequence
  glr-train      hla.glr_scan and its gradients
  glu-forward    hla.glu over n tokens
  glu-train      the same with its gradients

Types: "bf16", "fp32", or "mixed": fp32 outputs of a mixer beside bf16 gates
(gnorm), an fp32 residual stream beside bf16 blocks (rnorm).

The plain forms compute in 32 bits with elementary torch operations and round
once at the end.
"""
import torch

own = False

EPS = 1e-6
C = 8.0
# dtype -> (y of a mixer or the residual stream, everything else)
DTYPES = {"bf16": (torch.bfloat16, torch.bfloat16), "fp32": (torch.float32, torch.float32),
          "mixed": (torch.float32, torch.bfloat16)}


def _gnorm(kind, B, n, G, d, dtype="bf16", gate=True, norm_first=False, heads_first=False, shared=True):
    return dict(kind=kind, B=B, n=n, G=G, d=d, dtype=dtype, gate=gate, norm_first=norm_first, heads_first=heads_first,
                shared=shared)


def _rnorm(kind, B, n, D, dtype="bf16", post=True, scale=True, alpha=1.0):
    return dict(kind=kind, B=B, n=n, D=D, dtype=dtype, post=post, scale=scale, alpha=alpha)


def _glr(kind, B, n, D, dtype="bf16", bias=True):
    return dict(kind=kind, B=B, n=n, D=D, dtype=dtype, bias=bias)


def _glu(kind, B, n, D, F, act="silu"):
    return dict(kind=kind, B=B, n=n, D=D, F=F, dtype="bf16", act=act)


def listed():
    return [
        # decoding: the outputs of 32 heads of 128 of one token for each of 64 sequences, with their gates
        dict(_gnorm("gnorm-forward", 64, 1, 32, 128), name="gnorm-step"),
        # a training batch of a d = 64 layer: the attention's fp32 outputs, heads before tokens, normed head by head
        dict(_gnorm("gnorm-train", 4, 4096, 16, 64, "mixed", norm_first=True, heads_first=True), name="gnorm-train"),
        # decoding: between two blocks of a wide model, norms before and after
        dict(_rnorm("rnorm-forward", 64, 1, 4096), name="rnorm-step"),
        # long prompts between two blocks, the pre-norm alone
        dict(_rnorm("rnorm-forward", 2, 16384, 4096, "bf16", False, False), name="rnorm-long"),
        # a training batch over an fp32 residual stream, norms before and after, learned residual scales
        dict(_rnorm("rnorm-train", 4, 4096, 1024, "mixed"), name="rnorm-train"),
        # an odd width and length in fp32: nothing is a multiple of a vector
        dict(_rnorm("rnorm-train", 3, 1021, 333, "fp32", False, True, 0.5), name="rnorm-train-fp32-odd"),
        # decoding: one token for each of 64 sequences
        dict(_glr("glr-step", 64, 1, 4096), name="glr-step"),
        # serving: a prompt of ragged length from and into a state
        dict(_glr("glr-prompt", 1, 8000, 4096), name="glr-prompt"),
        # a training batch: forward and gradients
        dict(_glr("glr-train", 4, 4096, 2048), name="glr-train"),
        # decoding: one token for each of 16 sequences, the weights streamed once
        dict(_glu("glu-forward", 16, 1, 2048, 8192), name="glu-step"),
        # serving: a prompt of ragged length, a feed-forward width that no tile divides
        dict(_glu("glu-forward", 1, 2001, 2048, 5464, "gelu"), name="glu-prompt"),
        # a training batch: forward and gradients, the largest case
        dict(_glu("glu-train", 4, 4096, 1024, 4096), name="glu-train"),
    ]


def _log_between(rng, low, high):
    return min(high, max(low, round(low * (high / low) ** rng.random())))


def draw(rng):
    kind = rng.choice(("gnorm-forward", "gnorm-train", "rnorm-forward", "rnorm-train", "glr-forward", "glr-prompt",
                       "glr-step", "glr-train", "glu-forward", "glu-forward", "glu-train"))
    B = rng.choice((1, 2, 3, 4, 8))
    if kind.startswith("gnorm"):
        d, G = rng.choice((16, 64, 80, 100, 128, 256, 333, 1024)), rng.choice((1, 1, 4, 7, 16, 32))
        top = min(16384, (1 << 25) // (B * G * d))
        return _gnorm(kind, B, _log_between(rng, 1, top), G, d, rng.choice(tuple(DTYPES)), rng.random() < 0.8,
                      rng.random() < 0.5, rng.random() < 0.3, rng.random() < 0.5)
    if kind.startswith("rnorm"):
        D = _log_between(rng, 64, 8192)
        D = rng.choice((D, D - D % 8))
        top = min(16384, (1 << 25) // (B * D))
        return _rnorm(kind, B, _log_between(rng, 1, top), D, rng.choice(tuple(DTYPES)), rng.random() < 0.5,
                      rng.random() < 0.5, rng.choice((1.0, 0.5)))
    if kind.startswith("glr"):
        D = _log_between(rng, 16, 8192)
        D = rng.choice((D, D - D % 8))
        dtype, bias = rng.choice(("bf16", "bf16", "fp32")), rng.random() < 0.7
        if kind == "glr-step":
            return _glr(kind, _log_between(rng, 1, 128), 1, D, dtype, bias)
        return _glr(kind, B, _log_between(rng, 1, min(16384, (1 << 25) // (B * D))), D, dtype, bias)
    D, F = 8 * _log_between(rng, 8, 512), 8 * _log_between(rng, 8, 1024)
    top = min(16384, (1 << (34 if kind == "glu-train" else 35)) // (B * D * F))
    return _glu(kind, B, _log_between(rng, 1, top), D, F, rng.choice(("silu", "silu", "gelu")))


def _randn(g, *shape):
    return torch.randn(*shape, generator=g, device="cuda")


def _inputs(c, seed):
    """Everything that is drawn, made from the seed alone: activations as a
    projection leaves them (views of one wide row where the layer has them
    so), weights as a trained layer's."""
    g = torch.Generator("cuda").manual_seed(seed)
    t0, t = DTYPES[c["dtype"]]
    s = dict(case=c)
    B, n = c["B"], c["n"]
    kind = c["kind"]
    if kind.startswith("gnorm"):
        G, d = c["G"], c["d"]
        if c["heads_first"]:
            s["y"] = (_randn(g, B, G, n, d) * 0.3).to(t0).transpose(1, 2)
        else:
            s["y"] = (_randn(g, B, n, G, d) * 0.3).to(t0)
        # the gate is the last part of a wider projection
        s["z"] = _randn(g, B, n, 2 * G * d).to(t)[..., G * d:].unflatten(-1, (G, d)) if c["gate"] else None
        s["w"] = (1 + 0.1 * _randn(g, *((d,) if c["shared"] else (G, d)))).to(t)
        if kind == "gnorm-train":
            s["gout"] = _randn(g, B, n, G, d).to(t)
    elif kind.startswith("rnorm"):
        D = c["D"]
        s["x"] = (_randn(g, B, n, D) * 2).to(t0)
        s["y"] = _randn(g, B, n, D).to(t)
        s["w"] = (1 + 0.1 * _randn(g, D)).to(t)
        s["post"] = (1 + 0.1 * _randn(g, D)).to(t) if c["post"] else None
        s["scale"] = (0.5 + 0.1 * _randn(g, D)).to(t) if c["scale"] else None
        if kind == "rnorm-train":
            s["gout"], s["gr"] = _randn(g, B, n, D).to(t), _randn(g, B, n, D).to(t0)
    elif kind.startswith("glr"):
        D = c["D"]
        s["x"] = _randn(g, B, n, D).to(t)
        fg = (1.5 * _randn(g, B, n, 2 * D)).to(t)
        s["f"], s["g"] = fg[..., :D], fg[..., D:]
        # a full gate keeps 0.9 to 0.999 of the state a token
        keep = 0.9 + 0.099 * torch.rand(D, generator=g, device="cuda", dtype=torch.float64)
        s["decay"] = torch.log(torch.expm1(-torch.log(keep) / C)).float()
        s["fb"], s["gb"] = (0.5 * _randn(g, D) if c["bias"] else None for _ in range(2))
        if kind == "glr-train":
            s["gout"] = _randn(g, B, n, D).to(t)
        elif kind != "glr-forward":
            s["state"] = _randn(g, B, D)
        if kind == "glr-step":
            s.update({k: s[k][:, 0] for k in ("x", "f", "g")})
    else:
        D, F = c["D"], c["F"]
        s["x"] = _randn(g, B, n, D).to(t)
        s["wg"], s["wu"] = ((_randn(g, F, D) * D ** -0.5).to(t) for _ in range(2))
        if kind == "glu-train":
            s["gout"] = _randn(g, B, n, F).to(t)
    return s


def _learned(s):
    return [s[k] for k in {"gnorm": ("y", "z", "w"), "rnorm": ("x", "y", "w", "post", "scale"),
                           "glr": ("x", "f", "g", "decay", "fb", "gb"),
                           "glu": ("x", "wg", "wu")}[s["case"]["kind"].split("-")[0]] if s[k] is not None]


def prepare(case, seed):
    s = _inputs(case, seed)
    if case["kind"].endswith("train"):
        for x in _learned(s):
            x.requires_grad_()
    return s


# ----------------------------------------------------------------------------
# Plain forms, fp32.
def _rms(x):
    return x * torch.rsqrt(x.square().mean(-1, keepdim=True) + EPS)


def _silu(z):
    return z * torch.sigmoid(z)


def _plain_gnorm(c, y, z, w):
    if z is None:
        return _rms(y) * w
    return _rms(y) * w * _silu(z) if c["norm_first"] else _rms(y * _silu(z)) * w


def _plain_rnorm(c, x, y, w, post, scale):
    u = y if post is None else _rms(y) * post
    if scale is not None:
        u = u * scale
    r = x + c["alpha"] * u
    return _rms(r) * w, r


def _plain_scan(a, b):
    """h_t = a_t h_{t-1} + b_t from zero over dimension 1, and the products of all a up to t: spans of doubling length."""
    span, n = 1, a.shape[1]
    while span < n:
        b = torch.cat([b[:, :span], torch.addcmul(b[:, span:], a[:, span:], b[:, :-span])], 1)
        a = torch.cat([a[:, :span], a[:, span:] * a[:, :-span]], 1)
        span *= 2
    return b, a


def _plain_gates(x, f, g, decay, fb, gb):
    """The recurrence's a and b."""
    f, g = (v if m is None else v + m for v, m in ((f, fb), (g, gb)))
    la = -C * torch.logaddexp(decay, torch.zeros_like(decay)) * torch.sigmoid(f)
    return la.exp(), torch.sqrt(-torch.expm1(2 * la)) * torch.sigmoid(g) * x


def _plain(s):
    c, kind = s["case"], s["case"]["kind"]
    t0, t = DTYPES[c["dtype"]]
    f = {k: v.float() if isinstance(v, torch.Tensor) else v for k, v in s.items()}
    if kind.startswith("gnorm"):
        out = _plain_gnorm(c, f["y"], f["z"], f["w"])
        grads = torch.autograd.grad(out, _learned(s), f["gout"]) if kind == "gnorm-train" else ()
        return [out.detach().to(t), *grads]
    if kind.startswith("rnorm"):
        out, r = _plain_rnorm(c, *(f[k] for k in ("x", "y", "w", "post", "scale")))
        grads = torch.autograd.grad([out, r], _learned(s), [f["gout"], f["gr"]]) if kind == "rnorm-train" else ()
        return [out.detach().to(t), r.detach().to(t0), *grads]
    if kind.startswith("glr"):
        a, b = _plain_gates(*(f[k] for k in ("x", "f", "g", "decay", "fb", "gb")))
        if kind == "glr-step":
            s["state"].copy_(a * s["state"] + b)
            return [s["state"].to(t), s["state"]]
        with torch.no_grad():
            h, through = _plain_scan(a, b)
            if kind == "glr-prompt":
                h = h + through * s["state"][:, None]
                s["state"].copy_(h[:, -1])
                return [h.to(t), s["state"]]
            if kind == "glr-forward":
                return h.to(t)
            later = torch.cat([a[:, 1:], torch.zeros_like(a[:, :1])], 1).flip(1)
            lam = _plain_scan(later, f["gout"].flip(1))[0].flip(1)
            before = torch.cat([torch.zeros_like(h[:, :1]), h[:, :-1]], 1)
        return [h.to(t), *torch.autograd.grad([a, b], _learned(s), [lam * before, lam])]
    x = f["x"].flatten(0, 1)
    p, u = x @ f["wg"].T, x @ f["wu"].T
    a = _silu(p) if c["act"] == "silu" else 0.5 * p * (1 + torch.erf(p * 0.5 ** 0.5))
    out = (a * u).unflatten(0, (c["B"], c["n"]))
    if kind == "glu-forward":
        return out.to(t)
    return [out.detach().to(t), *torch.autograd.grad(out, _learned(s), f["gout"])]


def run(s):
    if not own:
        return _plain(s)
    import paper_2510_27258_amd as hla
    c, kind = s["case"], s["case"]["kind"]
    if kind.startswith("gnorm"):
        out = hla.gated_norm(s["y"], s["z"], s["w"], eps=EPS, norm_first=c["norm_first"],
                             out_dtype=DTYPES[c["dtype"]][1])
        grads = torch.autograd.grad(out, _learned(s), s["gout"]) if kind == "gnorm-train" else ()
        return [out.detach(), *grads]
    if kind.startswith("rnorm"):
        out, r = hla.residual_norm(s["x"], s["y"], s["w"], post_weight=s["post"], scale=s["scale"], alpha=c["alpha"],
                                   eps=EPS)
        grads = torch.autograd.grad([out, r], _learned(s), [s["gout"], s["gr"]]) if kind == "rnorm-train" else ()
        return [out.detach(), r.detach(), *grads]
    if kind.startswith("glr"):
        args = [s[k] for k in ("x", "f", "g", "decay", "fb", "gb")]
        if kind == "glr-forward":
            return hla.glr_forward(*args, c=C)
        if kind == "glr-prompt":
            return [hla.glr_prefill(s["state"], *args, c=C), s["state"]]
        if kind == "glr-step":
            return [hla.glr_step(s["state"], *args, c=C), s["state"]]
        y = hla.glr_scan(*args, c=C)
        return [y.detach(), *torch.autograd.grad(y, _learned(s), s["gout"])]
    out = hla.glu(s["x"], s["wg"], s["wu"], act=c["act"])
    if kind == "glu-forward":
        return out
    return [out.detach(), *torch.autograd.grad(out, _learned(s), s["gout"])]


def work(case):
    """Bytes: inputs and outputs once.  Flops: the products of the feed-forward
    part; elsewhere the element-wise operations, roughly."""
    c, kind = case, case["kind"]
    e0, e = (torch.finfo(t).bits // 8 for t in DTYPES[c["dtype"]])
    train = kind.endswith("train")
    if kind.startswith("gnorm"):
        row = c["G"] * c["d"]
        tokens = c["B"] * c["n"] * row
        gate = e if c["gate"] else 0
        weights = (c["d"] if c["shared"] else row) * e
        if train:
            return {"bytes": tokens * (2 * e0 + 2 * e + 2 * gate) + 2 * weights, "flops": tokens * 30}
        return {"bytes": tokens * (e0 + e + gate) + weights, "flops": tokens * 10}
    if kind.startswith("rnorm"):
        tokens = c["B"] * c["n"] * c["D"]
        weights = c["D"] * e * (1 + c["post"] + c["scale"])
        if train:
            return {"bytes": tokens * (4 * e0 + 4 * e) + 2 * weights, "flops": tokens * 30}
        return {"bytes": tokens * (2 * e0 + 2 * e) + weights, "flops": tokens * 10}
    if kind.startswith("glr"):
        tokens = c["B"] * c["n"] * c["D"]
        weights = c["D"] * 4 * (1 + 2 * c["bias"])
        state = 0 if kind in ("glr-forward", "glr-train") else 2 * c["B"] * c["D"] * 4
        if train:
            return {"bytes": tokens * 8 * e + 2 * weights, "flops": tokens * 60}
        return {"bytes": tokens * 4 * e + weights + state, "flops": tokens * 20}
    M, D, F = c["B"] * c["n"], c["D"], c["F"]
    moved = (M * D + 2 * D * F) * e * (2 if train else 1) + M * F * e * (2 if train else 1)
    return {"bytes": moved, "flops": 4 * M * D * F * (3 if train else 1)}


# ----------------------------------------------------------------------------
# 64 bits, from the definitions; gradients by their formulas, the recurrence token by token.
def _norm_back(dhat, hat, inv):
    """The gradient of v for that of hat = v inv, inv = (mean v^2 + eps)^-1/2."""
    return inv * (dhat - hat * (dhat * hat).mean(-1, keepdim=True))


def _inv(v):
    return (v.square().sum(-1, keepdim=True) / v.shape[-1] + EPS) ** -0.5


def _exact_gnorm(s):
    c = s["case"]
    y, w = s["y"].double(), s["w"].double()
    z = s["z"].double() if c["gate"] else None
    sig = None if z is None else 1 / (1 + torch.exp(-z))
    gate = 1.0 if z is None else z * sig
    first = c["norm_first"]
    v = y if first else y * gate
    inv = _inv(v)
    hat = v * inv
    out = hat * w * gate if first else hat * w
    if c["kind"] == "gnorm-forward":
        return [out]
    go = s["gout"].double()
    gh = go * gate if first else go
    dv = _norm_back(gh * w, hat, inv)
    dw = (gh * hat).sum((0, 1, 2) if c["shared"] else (0, 1))
    grads = [dv if first else dv * gate]
    if z is not None:
        grads.append((go * w * hat if first else dv * y) * sig * (1 + z * (1 - sig)))
    return [out, *grads, dw]


def _exact_rnorm(s):
    c = s["case"]
    x, y, w = (s[k].double() for k in ("x", "y", "w"))
    post, scale = (None if s[k] is None else s[k].double() for k in ("post", "scale"))
    u, inv_y = y, None
    if post is not None:
        inv_y = _inv(y)
        u = y * inv_y * post
    step = c["alpha"] if scale is None else c["alpha"] * scale
    r = x + step * u
    inv = _inv(r)
    hat = r * inv
    if c["kind"] == "rnorm-forward":
        return [hat * w, r]
    go, gr = s["gout"].double(), s["gr"].double()
    dr = gr + _norm_back(go * w, hat, inv)
    du = dr * step
    grads = [dr, du if post is None else _norm_back(du * post, y * inv_y, inv_y), (go * hat).sum((0, 1))]
    if post is not None:
        grads.append((du * y * inv_y).sum((0, 1)))
    if scale is not None:
        grads.append((c["alpha"] * dr * u).sum((0, 1)))
    return [hat * w, r, *grads]


def _exact_glr(s):
    c, kind = s["case"], s["case"]["kind"]
    x, f, g = ((s[k][:, None] if kind == "glr-step" else s[k]).double() for k in ("x", "f", "g"))
    decay = s["decay"].double()
    if c["bias"]:
        f, g = f + s["fb"].double(), g + s["gb"].double()
    r, i = 1 / (1 + torch.exp(-f)), 1 / (1 + torch.exp(-g))
    soft = torch.log1p(torch.exp(decay))
    la = -C * soft * r
    a, root = la.exp(), torch.sqrt(-torch.expm1(2 * la))
    b = root * i * x
    n = x.shape[1]
    h = s["state"].double() if "state" in s else torch.zeros_like(b[:, 0])
    ys, befores = torch.empty_like(b), torch.empty_like(b)
    for t in range(n):
        befores[:, t] = h
        h = torch.addcmul(b[:, t], a[:, t], h)
        ys[:, t] = h
    if kind == "glr-step":
        return [ys[:, 0], h]
    if kind != "glr-train":
        return [ys, h] if kind == "glr-prompt" else ys
    dy = s["gout"].double()
    lam = torch.empty_like(b)
    carry = torch.zeros_like(h)
    for t in reversed(range(n)):
        carry = dy[:, t] + carry
        lam[:, t] = carry
        carry = carry * a[:, t]
    dla = lam * (a * befores - i * x * a * a / root)
    dg = lam * root * x * i * (1 - i)
    df = dla * la * (1 - r)
    ddecay = (dla * -C * r).sum((0, 1)) / (1 + torch.exp(-decay))
    biases = [df.sum((0, 1)), dg.sum((0, 1))] if c["bias"] else []
    return [ys, lam * root * i, df, dg, ddecay, *biases]


def _exact_glu(s):
    c = s["case"]
    x, wg, wu = s["x"].double().flatten(0, 1), s["wg"].double(), s["wu"].double()
    p, u = x @ wg.T, x @ wu.T
    if c["act"] == "silu":
        sig = 1 / (1 + torch.exp(-p))
        a, da = p * sig, sig * (1 + p * (1 - sig))
    else:
        phi = 0.5 * torch.special.erfc(-p * 0.5 ** 0.5)
        a, da = p * phi, phi + p * torch.exp(-0.5 * p * p) * (2 * torch.pi) ** -0.5
    out = (a * u).unflatten(0, (c["B"], c["n"]))
    if c["kind"] == "glu-forward":
        return out
    go = s["gout"].double().flatten(0, 1)
    dp, du = go * u * da, go * a
    dx = (dp @ wg + du @ wu).unflatten(0, (c["B"], c["n"]))
    return [out, dx, dp.T.contiguous() @ x, du.T.contiguous() @ x]


def exact(case, seed):
    s = _inputs(case, seed)
    with torch.no_grad():
        return {"gnorm": _exact_gnorm, "rnorm": _exact_rnorm, "glr": _exact_glr,
                "glu": _exact_glu}[case["kind"].split("-")[0]](s)
