"""More operators of a party's local step and of the answers after it, as timed cases.

Between two aggregations a party trains adapters beside shared projections, and the common model answers requests. Around those
projections a block of the model has norms: of what the block gives, before it is gated and added to the stream that runs past it, and of
the stream, before the next block reads it. The adapters' gradients, one matrix of a short and a long side for every party, may be
orthogonalised by Newton-Schulz products before they are applied. And the common model, its adapters merged into the projections,
answers with weights of eight bits: one scale for each output, one for each row of the input.

Every case runs in two forms on the same inputs: written out in elementary torch operations in 32 bits, and, where
`own` is set, through `paper_2107_13797_amd.api`.
"""
import math

import torch

own = False

_TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
_SIZE = {"f32": 4, "f16": 2, "bf16": 2}
_EPS, _TINY = 1e-6, 1e-7
# a step of the quintic X <- a X + b (X X^T) X + c (X X^T)^2 X, five times
_STEP = (3.4445, -4.7750, 2.0315)

_LISTED = [
    # one request's row behind one block: launches only
    dict(name="norm_bf16_1x4096", op="norm", type="bf16", rows=1, cols=4096, pad=0, block=True, post=True, gate="cols", pre=True, scale=1.0, grad=False),
    # a step on rows of the forward benchmark's features
    dict(name="norm_f32_step_4096x256", op="norm", type="f32", rows=4096, cols=256, pad=0, block=True, post=True, gate="cols", pre=True, scale=0.5, grad=True),
    # a step with a gate for every element, odd sizes, rows that are a slice of a wider array
    dict(name="norm_f16_step_3001x1001_slice", op="norm", type="f16", rows=3001, cols=1001, pad=6, block=True, post=True, gate="full", pre=True, scale=1.0, grad=True),
    # a large step of a wide model: memory traffic
    dict(name="norm_bf16_step_16384x4096", op="norm", type="bf16", rows=16384, cols=4096, pad=0, block=True, post=True, gate="cols", pre=True, scale=1.0, grad=True),
    # adapters of a narrow model, one of each of eight parties: latency
    dict(name="orth_f32_8x4x256", op="orth", type="f32", parties=8, short=4, long=256, tall=False, base=False, steps=5),
    # eight parties' adapters of a wide projection, applied to what they held
    dict(name="orth_f32_8x16x4096_base", op="orth", type="f32", parties=8, short=16, long=4096, tall=False, base=True, steps=5),
    # nothing even, in 16 bits, the long side first
    dict(name="orth_bf16_7x1001x37", op="orth", type="bf16", parties=7, short=37, long=1001, tall=True, base=False, steps=5),
    # many parties' large adapters, the long side first
    dict(name="orth_f32_64x4096x64_base", op="orth", type="f32", parties=64, short=64, long=4096, tall=True, base=True, steps=5),
    # one request: the latency of reading the weights once
    dict(name="int8_bf16_1x4096x4096", op="int8", type="bf16", rows=1, inner=4096, outer=4096, fresh=False, bias=False, residual=False),
    # one row of each of 64 requests
    dict(name="int8_bf16_64x4096x4096", op="int8", type="bf16", rows=64, inner=4096, outer=4096, fresh=False, bias=False, residual=False),
    # a new common model, whose weights are brought to eight bits first; nothing even
    dict(name="int8_f16_fresh_3001x1001x515", op="int8", type="f16", rows=3001, inner=1001, outer=515, fresh=True, bias=True, residual=True),
    # the answers of all rows that the common model is judged by
    dict(name="int8_bf16_8192x4096x4096", op="int8", type="bf16", rows=8192, inner=4096, outer=4096, fresh=False, bias=False, residual=False),
]


def listed():
    return [dict(c) for c in _LISTED]


def work(case):
    """Bytes: inputs read once, outputs written once. Flops: two per multiply-add of the products; a few per element elsewhere."""
    e = _SIZE[case["type"]]
    if case["op"] == "norm":
        n, cols, full = case["rows"] * case["cols"], case["cols"], int(case["block"] and case["gate"] == "full")
        streams = 1 + (2 + full if case["block"] else 0) + int(case["pre"])
        if case["grad"]:
            streams += 1 + (2 + full if case["block"] else 0) + int(case["pre"])
        return dict(bytes=n * e * streams + 4 * cols * 6, flops=n * (12 + 24 * int(case["grad"])))
    if case["op"] == "orth":
        p, k, n = case["parties"], case["short"], case["long"]
        return dict(bytes=p * k * n * e * (2 + int(case["base"])), flops=p * (k * (k + 1) * n + 2 * k * k * n + case["steps"] * 4 * k ** 3))
    i, o, rows = case["inner"], case["outer"], case["rows"]
    b = rows * i * e + o * i * (e if case["fresh"] else 1) + o * 4 + rows * o * e * (1 + int(case["residual"]))
    return dict(bytes=b, flops=2 * rows * i * o)


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    """One more case: sizes spread over the logarithm of their ranges, none above the largest listed one."""
    most = {m: max(work(c)[m] for c in _LISTED) for m in ("bytes", "flops")}
    while True:
        op, kind = rng.choice(["norm", "orth", "int8"]), rng.choice(list(_TYPES))
        if op == "norm":
            block = rng.random() < 0.85
            case = dict(op=op, type=kind, rows=_log_int(rng, 1, 16384), cols=_log_int(rng, 8, 8192), pad=rng.choice([0, 0, 1, 8]), block=block,
                        post=block and rng.random() < 0.7, gate=rng.choice(["none", "cols", "full"]) if block else "none",
                        pre=not block or rng.random() < 0.8, scale=rng.choice([1.0, 0.5, 1.25]) if block else 1.0, grad=rng.random() < 0.6)
        elif op == "orth":
            short = _log_int(rng, 1, 128)
            case = dict(op=op, type=kind, parties=_log_int(rng, 1, 64), short=short, long=_log_int(rng, short, 16384), tall=rng.random() < 0.5,
                        base=rng.random() < 0.5, steps=rng.choice([3, 5, 5, 5]))
        else:
            case = dict(op=op, type=kind, rows=_log_int(rng, 1, 16384), inner=_log_int(rng, 16, 8192), outer=_log_int(rng, 16, 8192),
                        fresh=rng.random() < 0.3, bias=rng.random() < 0.5, residual=rng.random() < 0.5)
        w = work(case)
        if all(w[m] <= most[m] for m in most):
            return case


# ---------------------------------------------------------------------------------------------------
# inputs


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    kind = _TYPES[case["type"]]

    def normal(*shape, sigma=1.0):
        return torch.randn(shape, device="cuda", generator=gen).mul_(sigma)

    state = dict(case, kind=kind)
    if case["op"] == "norm":
        rows, cols = case["rows"], case["cols"]

        def wide(sigma, by=None):  # rows of a wider array where `pad` says so
            m = normal(rows, cols + case["pad"], sigma=sigma)
            if by is not None:
                m[:, :cols] *= by
            return m.to(kind)[:, :cols]

        loud = 1.0 + 8.0 * (torch.rand(cols, device="cuda", generator=gen) < 0.01)  # channels that a trained stream has
        state["x"] = wide(1.5, loud)
        state["f"] = wide(0.5) if case["block"] else None
        state["post_gain"] = normal(cols, sigma=0.1).add_(1.0) if case["post"] else None
        state["pre_gain"] = normal(cols, sigma=0.1).add_(1.0) if case["pre"] else None
        state["gates"] = dict(none=lambda: None, cols=lambda: normal(cols, sigma=0.2).add_(0.7), full=lambda: wide(0.4))[case["gate"]]()
        if case["grad"]:
            state["dnormed"] = wide(0.02) if case["pre"] else None
            state["dstream"] = wide(0.02) if case["block"] else None
        return state
    if case["op"] == "orth":
        p, k, n = case["parties"], case["short"], case["long"]
        # a gradient: some directions much stronger than others, and noise
        some = max(1, k // 4)
        g = normal(p, k, some) @ normal(p, some, n) * (some ** -0.5) + normal(p, k, n, sigma=0.3)
        g *= 1e-3
        state["g"] = (g.transpose(1, 2) if case["tall"] else g).to(kind).contiguous()
        state["held"] = normal(*state["g"].shape, sigma=0.05).to(kind) if case["base"] else None
        return state
    rows, i, o = case["rows"], case["inner"], case["outer"]
    x = normal(rows, i)
    x *= 1.0 + 5.0 * (torch.rand(i, device="cuda", generator=gen) < 0.01)
    w = normal(o, i, sigma=i ** -0.5).to(kind)
    state.update(x=x.to(kind), bias_values=normal(o, sigma=0.1) if case["bias"] else None,
                 residual_values=normal(rows, o).to(kind) if case["residual"] else None)
    if case["fresh"]:
        state["w"] = w
    else:  # the weights as such a program keeps them: eight bits, rows of a multiple of 128 with zeros behind what they hold
        q, scale = _eight_bits(w.float())
        state["wq"] = torch.zeros((o, (i + 127) // 128 * 128), dtype=torch.int8, device="cuda")
        state["wq"][:, :i] = q
        state["w_scale"] = scale
    return state


# ---------------------------------------------------------------------------------------------------
# the plain forms: elementary operations in 32 bits, rounded once at the end


def _eight_bits(x):
    """Whole numbers of -127 .. 127 as float32, and each row's scale: q = rint(x (127 / amax)) with both roundings to 32 bits."""
    amax = x.abs().amax(1, keepdim=True)
    some = amax > 0
    by = torch.where(some, torch.div(torch.full_like(amax, 127.0), torch.where(some, amax, 1.0)), 0.0)
    return torch.round(x * by), torch.div(amax, torch.full_like(amax, 127.0))[:, 0]


def _plain_norm(s):
    kind, x, scale = s["kind"], s["x"].float(), s["scale"]
    out = []
    if s["block"]:
        f = s["f"].float()
        q = torch.rsqrt((f * f).mean(1, keepdim=True) + _EPS) if s["post"] else None
        fn = f * q if s["post"] else f
        p = fn * s["post_gain"] if s["post"] else fn
        gate = None if s["gate"] == "none" else s["gates"].float()
        r = scale * x + (p if gate is None else gate * p)
        out.append(r.to(kind))
    else:
        r = x
    if s["pre"]:
        t = torch.rsqrt((r * r).mean(1, keepdim=True) + _EPS)
        rn = r * t
        out.append((rn * s["pre_gain"]).to(kind))
    if not s["grad"]:
        return out
    dr = s["dstream"].float() if s["block"] else 0.0
    if s["pre"]:
        dn = s["dnormed"].float()
        a = dn * s["pre_gain"]
        dr = dr + t * (a - rn * (a * rn).mean(1, keepdim=True))
        dpre = (dn * rn).sum(0)
    if s["block"]:
        out.append((scale * dr).to(kind))
        dp = dr if gate is None else dr * gate
        if s["post"]:
            b = dp * s["post_gain"]
            out.append((q * (b - fn * (b * fn).mean(1, keepdim=True))).to(kind))
            out.append((dp * fn).sum(0))
        else:
            out.append(dp.to(kind))
        if s["gate"] == "cols":
            out.append((dr * p).sum(0))
        elif s["gate"] == "full":
            out.append((dr * p).to(kind))
    else:
        out.append(dr.to(kind))
    if s["pre"]:
        out.append(dpre)
    return out


def _plain_orth(s):
    g = s["g"].float()
    x = g.transpose(1, 2).contiguous() if s["tall"] else g
    x = x / ((x * x).sum((1, 2), keepdim=True).sqrt() + _TINY)
    a, b, c = _STEP
    for _ in range(s["steps"]):
        k = torch.bmm(x, x.transpose(1, 2).contiguous())
        x = a * x + torch.bmm(b * k + c * torch.bmm(k, k), x)
    if s["tall"]:
        x = x.transpose(1, 2)
    if s["base"]:
        x = 0.99 * s["held"].float() - 0.02 * x
    return x.to(s["kind"]).contiguous()


def _plain_int8(s):
    if s["fresh"]:
        wq, w_scale = _eight_bits(s["w"].float())
    else:
        wq, w_scale = s["wq"][:, :s["inner"]].float(), s["w_scale"]
    xq, x_scale = _eight_bits(s["x"].float())
    y = (xq @ wq.t()) * (x_scale[:, None] * w_scale)
    if s["bias"]:
        y = y + s["bias_values"]
    if s["residual"]:
        y = y + s["residual_values"].float()
    return y.to(s["kind"])


# ---------------------------------------------------------------------------------------------------
# the framework's calls


def _own_norm(s):
    from paper_2107_13797_amd import api
    r, h, rstd = api.haflo_residual_norm(s["x"], s["f"], s["post_gain"], s["gates"], s["pre_gain"], s["scale"], _EPS)
    out = ([r] if s["block"] else []) + ([h] if s["pre"] else [])
    if not s["grad"]:
        return out
    dx, df, dpost, dgate, dpre = api.haflo_residual_norm_backward(s["dnormed"], s["dstream"], s["x"], s["f"], s["post_gain"], s["gates"],
                                                                  s["pre_gain"], rstd, s["scale"])
    return out + [t for t in (dx, df, dpost, dgate, dpre) if t is not None]


def _own_orth(s):
    from paper_2107_13797_amd import api
    if s["base"]:
        return api.haflo_orthogonal_update(s["g"], s["held"], keep=0.99, scale=-0.02, coefficients=[_STEP] * s["steps"], eps=_TINY)
    return api.haflo_orthogonal_update(s["g"], coefficients=[_STEP] * s["steps"], eps=_TINY)


def _own_int8(s):
    from paper_2107_13797_amd import api
    wq, w_scale = api.haflo_quantize_rows(s["w"]) if s["fresh"] else (s["wq"], s["w_scale"])
    return api.haflo_int8_forward(s["x"], wq, w_scale, bias=s["bias_values"], residual=s["residual_values"])


def run(state):
    if own:
        return {"norm": _own_norm, "orth": _own_orth, "int8": _own_int8}[state["op"]](state)
    return {"norm": _plain_norm, "orth": _plain_orth, "int8": _plain_int8}[state["op"]](state)


# ---------------------------------------------------------------------------------------------------
# the definitions in 64 bits


def _exact_norm(case, s):
    up = lambda t: None if t is None else t.double()  # noqa: E731
    x, f, post, pre, gate = (up(s[k]) for k in ("x", "f", "post_gain", "pre_gain", "gates"))
    width, out = case["cols"], []

    def length(v):  # the root of the mean square, and eps under the root
        return torch.sqrt(torch.linalg.vector_norm(v, dim=1, keepdim=True) ** 2 / width + _EPS)

    stream = x
    if case["block"]:
        lf = length(f) if post is not None else None
        part = f / lf * post if post is not None else f
        stream = case["scale"] * x + (part if gate is None else part * gate)
        out.append(stream)
    if pre is not None:
        lr = length(stream)
        unit = stream / lr
        out.append(unit * pre)
    if not case["grad"]:
        return out
    total = torch.zeros_like(x) if s["dstream"] is None else s["dstream"].double()
    if pre is not None:
        dn = s["dnormed"].double()
        # the gradient of v / length(v): what comes in less its part along v, over the length
        along = (dn * pre * stream).sum(1, keepdim=True) / (width * lr ** 2)
        total = total + (dn * pre - along * stream) / lr
    if not case["block"]:
        return out + [total] + ([(dn * unit).sum(0)] if pre is not None else [])
    out.append(case["scale"] * total)
    into = total if gate is None else total * gate
    if post is not None:
        along = (into * post * f).sum(1, keepdim=True) / (width * lf ** 2)
        out += [(into * post - along * f) / lf, (into * f / lf).sum(0)]
    else:
        out.append(into)
    if gate is not None:
        out.append((total * part).sum(0) if case["gate"] == "cols" else total * part)
    if pre is not None:
        out.append((dn * unit).sum(0))
    return out


def _exact_orth(case, s):
    # A step takes each singular value v to v (a + b v^2 + c v^4) and keeps the directions, so all of them multiply the matrix by
    # one polynomial of its product with itself, which is taken on that product's eigenvalues.
    g = s["g"].double()
    short = g.mT if case["tall"] else g
    square = (short @ short.mT.contiguous()).cpu()
    square = square / (square.diagonal(dim1=1, dim2=2).sum(1).sqrt() + _TINY)[:, None, None] ** 2
    values, vectors = torch.linalg.eigh(square)
    by, (a, b, c) = torch.ones_like(values), _STEP
    for _ in range(case["steps"]):
        factor = a + values * (b + c * values)
        by, values = by * factor, values * factor * factor
    size = torch.linalg.vector_norm(g, dim=(1, 2)).cpu() + _TINY
    x = ((vectors * (by / size[:, None])[:, None, :]) @ vectors.mT).to(g.device) @ short.contiguous()
    x = x.mT if case["tall"] else x
    return 0.99 * s["held"].double() - 0.02 * x if case["base"] else x


def _exact_int8(case, s):
    def whole(m):  # by the definition: 127 over the largest magnitude, and each product with it, rounded to 32 bits
        m = m.double()
        most = m.abs().max(1, keepdim=True).values
        by = torch.where(most > 0, (127.0 / most).float().double(), 0.0)
        return (m * by).float().double().round(), (most / 127.0).float().double()

    wq, w_scale = whole(s["w"]) if case["fresh"] else (s["wq"][:, :case["inner"]].double(), s["w_scale"].double()[:, None])
    xq, x_scale = whole(s["x"])
    y = x_scale * (xq @ wq.T) * w_scale.T
    if case["bias"]:
        y = y + s["bias_values"].double()
    if case["residual"]:
        y = y + s["residual_values"].double()
    return y


def exact(case, seed):
    return {"norm": _exact_norm, "orth": _exact_orth, "int8": _exact_int8}[case["op"]](case, prepare(case, seed))
