"""What the tests of the norms around a block, of orthogonalised updates and of products of eight bits share: the definitions in 64 bits,
inputs, the sizes at which the kernels can go wrong, and checks that take the operators as a `run` object, so that the CPU build of
the kernels and the GPU go through the same ones. `run` has the binding's functions on host tensors.

Tolerances follow from the arithmetic and were set before the first run; UNIT is one rounding to a result's type, and each rounding of a
float32 on the way is allowed two."""
import math

import torch

from local_cases import TINY, TYPES, UNIT, near, normal

ULP = 2.0 ** -23

# --------------------------------------------------------------------------------------------------- norms around a block

NORMS = [  # type, rows, cols, pad, first, block, post, gate, pre, scale
    ("f32", 1, 1, 0, 0, True, True, "cols", True, 1.0), ("bf16", 3, 5, 0, 0, True, True, "full", True, 0.5), ("f16", 2, 8, 0, 0, True, False, "none", True, 1.0),
    ("f32", 7, 9, 3, 1, True, True, "none", False, 1.25), ("bf16", 70, 16, 0, 0, True, True, "cols", True, 1.0), ("f16", 33, 33, 1, 3, True, False, "full", True, 1.0),
    ("f32", 5, 129, 0, 0, False, False, "none", True, 1.0), ("bf16", 9, 256, 8, 0, True, True, "cols", True, 1.0), ("f16", 3, 515, 6, 0, True, True, "full", True, -2.0),
    ("bf16", 2, 1001, 0, 5, True, True, "cols", True, 1.0), ("f32", 3, 2049, 0, 0, True, True, "full", True, 1.0), ("bf16", 2, 4100, 4, 2, True, True, "cols", True, 0.5),
    ("f16", 2, 8192, 0, 0, False, False, "none", True, 1.0), ("bf16", 2, 8200, 0, 0, True, True, "full", True, 1.0), ("f32", 3, 9001, 1, 0, True, False, "cols", True, 1.0),
    ("f16", 2, 9001, 0, 0, False, False, "none", True, 1.0), ("f32", 4, 8195, 0, 0, True, True, "cols", False, 1.0), ("f32", 4, 40, 0, 0, True, False, "cols", False, 1.0),
]
NORMS_LARGE = [  # for the GPU: many rows to a block, every group size
    ("bf16", 3001, 1001, 6, 0, True, True, "full", True, 1.0), ("f32", 4096, 256, 0, 0, True, True, "cols", True, 0.5), ("f16", 20000, 8, 0, 0, True, True, "cols", True, 1.0),
    ("bf16", 2500, 4096, 0, 0, True, True, "cols", True, 1.0), ("f32", 700, 8000, 0, 0, True, True, "full", True, 1.0), ("bf16", 150, 20000, 8, 0, True, True, "full", True, 1.0),
    ("f16", 1100, 600, 0, 0, True, False, "none", True, 1.0), ("f32", 9000, 24, 0, 1, True, True, "full", False, 1.0), ("bf16", 4097, 128, 0, 0, False, False, "none", True, 1.0),
    ("f16", 90, 30001, 0, 3, True, True, "cols", True, 0.5), ("f32", 3000, 1, 0, 0, True, True, "full", True, 1.0), ("bf16", 513, 2000, 0, 0, True, True, "none", True, 1.0),
]


def norm_inputs(kind, rows, cols, pad, first, block, post, gate, pre, seed=0):
    gen = torch.Generator().manual_seed(seed + rows * 11 + cols)
    kind = TYPES[kind]
    m = lambda s: normal(gen, rows, cols, sigma=s, kind=kind, pad=pad, first=first)  # noqa: E731
    vec = lambda: torch.randn(cols, generator=gen) * 0.2 + 1.0  # noqa: E731
    x, f = m(1.5), m(0.7) if block else None
    gates = {"none": lambda: None, "cols": lambda: vec() * 0.5, "full": lambda: m(0.6)}[gate]()
    return x, f, vec() if post else None, gates, vec() if pre else None, m(0.1) if pre else None, m(0.1) if block else None


def norm_exact(x, f, post, gate, pre, dh, dr, scale, eps):
    """All results in 64 bits, and for each what its sums' terms amount to, which bounds its roundings."""
    up = lambda t: None if t is None else t.double()  # noqa: E731
    x, f, post, gate, pre, dh, dr = map(up, (x, f, post, gate, pre, dh, dr))
    cols = x.shape[1]
    root = lambda v: 1.0 / torch.sqrt((v * v).mean(1, keepdim=True) + eps)  # noqa: E731
    size = lambda v: torch.linalg.vector_norm(v, dim=1, keepdim=True)  # noqa: E731
    out, most = {}, {}
    one = torch.ones(cols, dtype=torch.float64)
    g = one if gate is None else gate
    if f is None:
        r, m = x, x.abs()
    else:
        q = root(f) if post is not None else torch.ones(x.shape[0], 1, dtype=torch.float64)
        fn = f * q
        p = fn * (one if post is None else post)
        r, m = scale * x + g * p, (scale * x).abs() + (g * p).abs()
        out["r"], most["r"] = r, m
    # how much more r's roundings are than r: they go into its mean
    cond = float((size(m) / size(r).clamp(min=1e-30)).max()) if r.numel() else 1.0
    d, da = (torch.zeros_like(x) if dr is None else dr), (torch.zeros_like(x) if dr is None else dr.abs())
    if pre is not None:
        t = root(r)
        rn, rm = r * t, m * t
        out["h"], most["h"] = rn * pre, rm * pre.abs() + (rn * pre).abs() * cond
        if dh is not None:
            a = dh * pre
            d = d + t * (a - rn * (a * rn).mean(1, keepdim=True))
            da = da + t * (a.abs() + rm * (a.abs() * rm).mean(1, keepdim=True))
            out["dpre"], most["dpre"] = (dh * rn).sum(0), (dh.abs() * rm).sum(0)
    out["dx"], most["dx"] = (d, da) if f is None else (scale * d, abs(scale) * da)
    if f is not None:
        dp, dpa = d * g, da * g.abs()
        if post is not None:
            b, ba = dp * post, dpa * post.abs()
            out["df"] = q * (b - fn * (b * fn).mean(1, keepdim=True))
            most["df"] = q * (ba + fn.abs() * (ba * fn.abs()).mean(1, keepdim=True))
            out["dpost"], most["dpost"] = (dp * fn).sum(0), (dpa * fn.abs()).sum(0)
        else:
            out["df"], most["df"] = dp, dpa
        if gate is not None:
            out["dgate"], most["dgate"] = d * p, da * p.abs()
            if gate.dim() == 1:
                out["dgate"], most["dgate"] = out["dgate"].sum(0), most["dgate"].sum(0)
    return out, most, cond


def check_norm(run, kind, rows, cols, pad, first, block, post, gate, pre, scale, eps=1e-5):
    x, f, post, gate, pre, dh, dr = norm_inputs(kind, rows, cols, pad, first, block, post, gate, pre)
    kind = x.dtype
    want, most, cond = norm_exact(x, f, post, gate, pre, dh, dr, scale, eps)
    u, tiny = UNIT[kind], TINY[kind]
    r, h, rstd = run.residual_norm(x, f, post, gate, pre, scale, eps)
    assert (r is None) == (f is None) and (h is None) == (pre is None)
    # six roundings to r; to h the root's and two more, its own and what the root takes over from r's
    for got, name, n in ((r, "r", 6), (h, "h", 12)):
        if got is not None:
            assert got.dtype == kind
            near(got, want[name], u * want[name].abs() + n * ULP * most[name] + tiny)
    dx, df, dpost, dgate, dpre = run.residual_norm_backward(dh, dr, x, f, post, gate, pre, rstd, scale)
    # a mean: eight terms in a lane, six exchanges, sixteen wavefronts, and one term for every 8192 columns; the factors' ten or so and what the
    # roots take over, twice
    n = 56 + 16 * cond + 2 * cols / 8192
    for got, name in ((dx, "dx"), (df, "df"), (dgate, "dgate")):
        if got is not None and got.dim() == 2:
            assert got.dtype == kind
            near(got, want[name], u * want[name].abs() + n * ULP * most[name] + tiny)
    for got, name in ((dpost, "dpost"), (dgate, "dgate"), (dpre, "dpre")):
        if got is not None and got.dim() == 1:
            assert got.dtype == torch.float32
            near(got, want[name], (n + rows + 16) * ULP * most[name] + 2.0 ** -126)
    assert [t is None for t in (df, dpost, dgate, dpre)] == [t is None for t in (f, post, gate, pre)]


def check_norm_special(run):
    """Zero rows, rows of the greatest magnitudes, and rows with NaN, which stay in their row."""
    ones = torch.ones(64)
    for kind in TYPES.values():
        big = torch.finfo(kind).max
        x, f = torch.zeros(4, 64, dtype=kind), torch.zeros(4, 64, dtype=kind)
        x[1], f[2] = big, -big
        x[3, 7] = math.nan
        r, h, rstd = run.residual_norm(x, f, ones, None, ones, 1.0, 1e-6)
        assert not r[0].any() and not h[0].any()
        assert torch.equal(r[1], x[1]) and float((h[1].double() - 1).abs().max()) <= 2 * UNIT[kind] + 8 * ULP
        # (float16 has no greater square than eps in its smallest: the greatest row's norm is 1 all the same)
        assert float((r[2].double() + 1).abs().max()) <= 2 * UNIT[kind] + 8 * ULP
        assert bool(h[3].isnan().all()) and int(r[3].isnan().sum()) == 1
        dh = torch.ones(4, 64, dtype=kind)
        dx, df, dpost, _, dpre = run.residual_norm_backward(dh, None, x, f, ones, None, ones, rstd, 1.0)
        assert not dx[:3].isnan().any() and bool(dx[3].isnan().all())
        # all of a row's elements alike: nothing of a gradient without a part across the row is left
        assert float(dx[1].abs().max()) <= 64 * ULP
        assert bool(dpre.isnan().all()) and bool(dpost.isnan().any())


def check_norm_far(run):
    """Rows near the greatest numbers with small gains, and the least with large ones: no factor of h alone leaves the normal numbers by far."""
    for cols in (5, 64, 1001, 9001):
        gen = torch.Generator().manual_seed(cols)
        unit = torch.randn(4, cols, generator=gen).clamp(-3.0, 3.0)
        for kind in (torch.float32, torch.bfloat16):
            for size, gain in ((2.0 ** 125, 1e-3), (2.0 ** 120, 1e-4), (2.0 ** 126, 1e-12), (2.0 ** -100, 1e5)):
                x, pre = (unit * size).to(kind), torch.full((cols,), gain) * (1.0 + torch.rand(cols, generator=gen))
                for f in (None, torch.zeros(4, cols, dtype=kind)):
                    want, most, _ = norm_exact(x, f, None, None, pre, None, None, 1.0, 2.0 ** -240)
                    _, h, _ = run.residual_norm(x, f, None, None, pre, 1.0, 2.0 ** -240)
                    # as in check_norm: the root, which below the normal numbers has 21 bits, is within two of its twelve
                    near(h, want["h"], UNIT[kind] * want["h"].abs() + 12 * ULP * most["h"] + TINY[kind])


def check_norm_gradients(run):
    """Against differences of the forward call along each gradient, in float32; the third derivative and the results' roundings bound how
    far the quotient is off."""
    x, f, post, gate, pre, dh, dr = norm_inputs("f32", 5, 48, 0, 0, True, True, "full", True, seed=3)
    args, step = [x, f, post, gate, pre], 2.0 ** -7
    _, _, rstd = run.residual_norm(*args, 0.8, 1e-5)
    dx, df, dpost, dgate, dpre = run.residual_norm_backward(dh, dr, *args, rstd, 0.8)

    def value(a):
        r, h, _ = run.residual_norm(*a, 0.8, 1e-5)
        return float((r.double() * dr).sum() + (h.double() * dh).sum())

    weight = float(dr.abs().sum() + dh.abs().sum())
    for i, grad in enumerate((dx, df, dpost, dgate, dpre)):
        d = grad / grad.norm()
        plus, minus = ([v + s * step * d if j == i else v for j, v in enumerate(args)] for s in (1.0, -1.0))
        got, want = float((grad.double() * d).sum()), (value(plus) - value(minus)) / (2 * step)
        # results are below 16, their third derivatives along d below 64 max|d|^3
        room = weight * (step ** 2 * 64 * float(d.abs().max()) ** 3 / 6 + 16 * 2.0 ** -22 / step)
        assert abs(got - want) <= room < 0.1 * got


SUMS = [(1, 3), (70, 40), (200, 260), (530, 2050), (100, 9001)]  # rows, cols
SUMS_LARGE = [(3001, 1001), (5000, 520), (2100, 4096), (700, 8000), (1500, 9001), (263000, 5), (300001, 8)]  # blocks that take several sets of rows


def check_norm_sums(run, rows, cols):
    """Gradients summed over rows of whole numbers, where both norms are of rows of ones: every sum is exact, so no row may be missing or counted
    twice."""
    gen = torch.Generator().manual_seed(rows + cols)
    whole = lambda lo, hi, *shape: torch.randint(lo, hi + 1, shape, generator=gen).float()  # noqa: E731
    ones, eps = 2.0 * whole(0, 1, rows, cols) - 1.0, 2.0 ** -254
    dh, dr, full = whole(-8, 8, rows, cols), whole(-8, 8, rows, cols), whole(-2, 2, rows, cols)
    post, gate, kind = 2.0 ** whole(-2, 2, cols), whole(1, 5, cols), torch.bfloat16 if cols % 2 else torch.float32
    to = lambda *t: tuple(v.to(kind) for v in t)  # noqa: E731
    x, f, dr, full, dh = to(whole(-3, 3, rows, cols), ones, dr, full, dh)
    _, _, rstd = run.residual_norm(x, f, post, gate, None, 1.0, eps)
    assert bool((rstd == 1.0).all())
    _, _, dpost, dgate, _ = run.residual_norm_backward(None, dr, x, f, post, gate, None, rstd, 1.0)
    part = (dr.double() * f.double()).sum(0)
    assert torch.equal(dpost.double(), part * gate) and torch.equal(dgate.double(), part * post)
    _, _, dpost, dgate, _ = run.residual_norm_backward(None, dr, x, f, post, full, None, rstd, 1.0)
    assert torch.equal(dpost.double(), (dr.double() * full.double() * f.double()).sum(0))
    assert torch.equal(dgate.double(), dr.double() * f.double() * post)
    _, _, rstd = run.residual_norm(f, None, None, None, post, 1.0, eps)
    dpre = run.residual_norm_backward(dh, dr, f, None, None, None, post, rstd, 1.0)[4]
    assert torch.equal(dpre.double(), (dh.double() * f.double()).sum(0))


# --------------------------------------------------------------------------------------------------- orthogonalised updates

QUINTIC, CUBIC = (3.4445, -4.7750, 2.0315), (1.5, -0.5, 0.0)
UPDATES = [  # type, parties, rows, cols, base, steps, pad
    ("f32", 1, 1, 1, False, [QUINTIC] * 5, 0), ("bf16", 3, 1, 9, True, [QUINTIC] * 3, 0), ("f16", 2, 7, 3, False, [QUINTIC] * 5, 0),
    ("f32", 2, 16, 33, True, [QUINTIC] * 5, 3), ("bf16", 2, 70, 17, True, [CUBIC] * 4, 0), ("f16", 1, 33, 40, False, [QUINTIC], 1),
    ("f32", 1, 64, 64, False, [QUINTIC] * 2, 0), ("bf16", 1, 65, 70, True, [QUINTIC] * 2, 0), ("f32", 2, 300, 4, False, [QUINTIC] * 5, 0),
    ("f32", 1, 3, 600, True, [CUBIC] * 16, 5), ("f32", 1, 90, 66, False, [QUINTIC], 0),
    ("f32", 2, 9, 800, True, [QUINTIC] * 2, 0), ("f16", 1, 780, 16, False, [QUINTIC] * 5, 1), ("bf16", 1, 45, 300, True, [QUINTIC] * 2, 0),
    ("f32", 1, 290, 48, True, [CUBIC], 0), ("f16", 1, 100, 30, True, [QUINTIC] * 2, 0), ("f32", 1, 60, 52, False, [QUINTIC], 2),
    ("bf16", 1, 97, 99, True, [QUINTIC] * 2, 0), ("f32", 1, 130, 104, False, [QUINTIC], 0), ("f16", 1, 73, 72, True, [CUBIC] * 3, 0),
]
UPDATES_LARGE = [
    ("f32", 8, 16, 4096, True, [QUINTIC] * 5, 0), ("bf16", 7, 1001, 37, False, [QUINTIC] * 5, 0), ("f32", 64, 512, 64, True, [QUINTIC] * 5, 0),
    ("f16", 5, 128, 2000, True, [QUINTIC] * 5, 8), ("f32", 3, 3001, 100, False, [QUINTIC] * 5, 0), ("bf16", 2, 5, 100001, True, [QUINTIC] * 5, 0),
    ("f32", 300, 8, 64, False, [QUINTIC] * 5, 0), ("f16", 4, 20000, 24, True, [QUINTIC] * 3, 1), ("f32", 2, 128, 128, False, [CUBIC] * 12, 0),
    ("bf16", 3, 65, 4096, False, [QUINTIC], 0), ("f32", 9, 1000, 128, True, [QUINTIC] * 2, 0), ("f16", 6, 48, 777, False, [QUINTIC] * 4, 3),
]


def update_exact(g, base, keep, scale, steps, eps):
    x = g.double()
    x = x / (torch.linalg.vector_norm(x, dim=(1, 2), keepdim=True) + eps)
    tall = x.shape[1] > x.shape[2]
    x = x.mT if tall else x
    for a, b, c in steps:
        k = x @ x.mT.contiguous()
        x = a * x + (b * k + c * k @ k) @ x
    x = scale * (x.mT if tall else x)
    return x, x if base is None else keep * base.double() + x


def update_inputs(kind, parties, rows, cols, base, pad, seed=0):
    gen = torch.Generator().manual_seed(seed + rows * 13 + cols)
    kind, short = TYPES[kind], min(rows, cols)
    weak = torch.logspace(0, -3, short)  # directions down to a thousandth of the strongest
    g = torch.randn(parties, rows, cols, generator=gen) * (weak if cols == short else weak[:, None])
    wide = torch.zeros(parties, rows, cols + pad, dtype=kind)
    wide[:, :, :cols] = g.to(kind)
    held = torch.randn(parties, rows, cols, generator=gen).to(kind) if base else None
    return wide[:, :, :cols], held


def check_update(run, kind, parties, rows, cols, base, steps, pad, eps=1e-7):
    g, held = update_inputs(kind, parties, rows, cols, base, pad)
    x, want = update_exact(g, held, 0.9, -0.3, steps, eps)
    got = run.orthogonal_update(g, held, 0.9, -0.3, steps, eps)
    assert got.dtype == g.dtype and got.shape == g.shape
    # 64 bits on the way: 28000 of a rounding of K, of sums of 128, is 2^-31 of a matrix; then one rounding to float32 and one to the type
    room = (UNIT[g.dtype] + ULP) * want.abs() + 2.0 ** -31 * x.abs().amax((1, 2), keepdim=True) + TINY[g.dtype]
    near(got, want, room)


def check_update_special(run):
    """A matrix of zeros, one with NaN, one with an infinity, very large and very small ones: each by itself."""
    for kind in (torch.float32, torch.bfloat16):
        for rows, cols in ((5, 40), (40, 5), (70, 80)):
            gen = torch.Generator().manual_seed(rows)
            g = torch.randn(6, rows, cols, generator=gen)
            g[1], g[2, 3, 4], g[3, 0, 0] = 0.0, math.nan, math.inf
            g[4] *= 2.0 ** 100
            g[5] *= 2.0 ** -100
            g = g.to(kind)
            eps = 2.0 ** -140
            got = run.orthogonal_update(g, None, 1.0, 1.0, [QUINTIC] * 3, eps)
            x, want = update_exact(g, None, 1.0, 1.0, [QUINTIC] * 3, eps)
            assert not got[1].any() and bool(got[2].isnan().all()) and bool(got[3].isnan().all())
            fine = [0, 4, 5]
            near(got[fine], want[fine], (UNIT[kind] + ULP) * want[fine].abs() + 2.0 ** -31)


def check_update_orthogonal(run):
    """The classical cubic brings every singular value to 1."""
    g, _ = update_inputs("f32", 2, 12, 50, False, 0)
    x = run.orthogonal_update(g, None, 1.0, 1.0, [(1.875, -1.25, 0.375)] * 16, 1e-12).double()
    assert float((x @ x.mT - torch.eye(12, dtype=torch.float64)).abs().max()) < 50 * 2.0 ** -23


# Lists that raise directions by more than an adapter's gradient of a low rank bears at once: their steps are taken in parts
POLAR = (1.875, -1.25, 0.375)
LISTS = {"6": [QUINTIC] * 6, "8": [QUINTIC] * 8, "12": [QUINTIC] * 12, "16": [QUINTIC] * 16, "steep": [(6.0, -21.0, 16.0)] + [POLAR] * 9,
         "first": [(3000.0, 0.0, 0.0), (1e-3, 0.0, 0.0)] + [POLAR] * 2, "polar": [POLAR] * 16, "both": [QUINTIC] * 3 + [POLAR] * 13, "cubic": [CUBIC] * 16}
STEPS = [  # type, rows, cols, list, base
    ("f32", 16, 256, "16", False), ("f32", 900, 16, "12", True), ("f32", 3, 1, "16", False), ("f32", 1000, 7, "16", False), ("f32", 16, 800, "steep", True),
    ("f32", 20, 256, "16", False), ("f32", 256, 32, "12", False), ("f32", 48, 100, "8", True), ("f32", 90, 45, "16", False), ("f32", 64, 256, "8", False),
    ("f32", 200, 64, "16", True), ("f32", 70, 100, "12", False), ("f32", 128, 140, "8", False), ("f32", 140, 128, "16", False), ("bf16", 20, 70, "16", True),
    ("f16", 100, 66, "12", False), ("f32", 32, 256, "polar", False), ("f32", 60, 64, "both", False), ("f32", 64, 50, "steep", False),
    ("f32", 33, 40, "first", True), ("f32", 300, 4, "first", False), ("f32", 33, 40, "6", False), ("f32", 33, 100, "cubic", True), ("bf16", 97, 128, "6", False),
]


def low_ranks(kind, rows, cols, seed=0):
    """Matrices of rank 1 in whole numbers, of rank 3, of equal rows, and one whose directions go down to a thousandth of the strongest."""
    gen = torch.Generator().manual_seed(seed + rows * 23 + cols)
    n = lambda *s: torch.randn(*s, generator=gen)  # noqa: E731
    whole = torch.randint(-8, 9, (rows, 1), generator=gen) * torch.randint(-8, 9, (1, cols), generator=gen)
    whole[0, 0] = 1
    short = min(rows, cols)
    weak = torch.logspace(0, -3, short)
    full = n(rows, cols) * (weak if cols == short else weak[:, None])
    return torch.stack([whole.float(), n(rows, 3) @ n(3, cols), n(1, cols).expand(rows, cols), full]).to(TYPES[kind])


def update_longer(g, steps, eps):
    """X product by product in 80 bits, and for each matrix what the steps raise a direction by: the product of their greatest factors on the
    singular values, with zero, that there are."""
    import numpy as np
    out, raised = [], []
    for m in g:
        x = m.double().numpy().astype(np.longdouble)
        x = x / (np.sqrt((x * x).sum()) + np.longdouble(eps))
        tall = x.shape[0] > x.shape[1]
        x = x.T if tall else x
        values, most = np.append(np.linalg.svd(x.astype(np.float64), compute_uv=False), 0.0), 1.0
        for a, b, c in steps:
            factor = a + b * values ** 2 + c * values ** 4
            values, most = values * factor, most * max(1.0, float(abs(factor).max()))
            k = x @ x.T
            x = np.longdouble(a) * x + (np.longdouble(b) * k + np.longdouble(c) * (k @ k)) @ x
        out.append(torch.from_numpy((x.T if tall else x).astype(np.float64)))
        raised.append(most)
    return torch.stack(out), torch.tensor(raised, dtype=torch.float64)[:, None, None]


def check_update_steps(run, kind, rows, cols, name, base, eps=1e-7):
    g, steps, keep, scale = low_ranks(kind, rows, cols), LISTS[name], 0.9, -0.3
    held = torch.randn(g.shape, generator=torch.Generator().manual_seed(rows)).to(g.dtype) if base else None
    x, raised = update_longer(g, steps, eps)
    want = scale * x + (0.0 if held is None else keep * held.double())
    got = run.orthogonal_update(g, held, keep, scale, steps, eps)
    # As in check_update, and a rounding of 2^-53 in each of three products a step, of sums of min(rows, cols), which the steps raise; of what they
    # multiply, X's greatest column (or row)
    norm = torch.linalg.vector_norm(g.double(), dim=(1, 2), keepdim=True)
    wide = torch.linalg.vector_norm(g.double(), dim=1 if rows <= cols else 2).amax(1)[:, None, None] / norm
    room = 3 * len(steps) * min(rows, cols) * 2.0 ** -53 * raised * wide
    near(got, want, (UNIT[g.dtype] + ULP) * want.abs() + abs(scale) * (2.0 ** -31 * x.abs().amax((1, 2), keepdim=True) + room) + TINY[g.dtype])


def check_update_steps_special(run):
    """check_update_special's matrices, each by itself, with steps that are taken in parts, and rows that lie further apart."""
    for rows, cols in ((5, 40), (900, 6), (50, 24), (70, 80)):
        gen = torch.Generator().manual_seed(rows)
        wide = torch.randn(6, rows, cols + 3, generator=gen)
        g = wide[:, :, :cols]
        g[1], g[2, 3, 4], g[3, 0, 0] = 0.0, math.nan, math.inf
        g[4] *= 2.0 ** 100
        g[5] *= 2.0 ** -100
        steps, eps = LISTS["12"], 2.0 ** -140
        got = run.orthogonal_update(g, None, 1.0, 1.0, steps, eps)
        assert not got[1].any() and bool(got[2].isnan().all()) and bool(got[3].isnan().all())
        fine = [0, 4, 5]
        want, raised = update_longer(g[fine], steps, eps)
        # (what is not of a low rank has no directions that only roundings raise)
        near(got[fine], want, 2 * ULP * want.abs() + 2.0 ** -31)


def check_update_rounds_once(run):
    """Results next to a border between two numbers of 16 bits, which a rounding to 32 bits on the way would put on it; of every form of the products."""
    for kind in (torch.float16, torch.bfloat16):
        u = UNIT[kind]
        for rows, cols in ((5, 40), (40, 5), (5, 900), (900, 5), (20, 41), (41, 20), (39, 40), (60, 64), (64, 50), (70, 81), (81, 70), (100, 101), (101, 100)):
            g, base = torch.zeros(1, rows, cols, dtype=kind), torch.ones(1, rows, cols, dtype=kind)
            for keep, want in ((1 + u + 2.0 ** -40, 1 + 2 * u), (1 + u - 2.0 ** -40, 1), (1 + 3 * u - 2.0 ** -40, 1 + 2 * u), (-1 - 3 * u + 2.0 ** -40, -1 - 2 * u),
                               (-1 - u - 2.0 ** -40, -1 - 2 * u), (1 + u, 1), (1 + 3 * u, 1 + 4 * u)):
                got = run.orthogonal_update(g, base, keep, 1.0, [QUINTIC], 1e-7)
                assert bool((got.double() == want).all()), (kind, rows, cols, keep)
        # the greatest, the least, and what has no value
        base[0, 0, :6] = torch.tensor([torch.finfo(kind).max, torch.finfo(kind).smallest_normal * 2 * u, math.inf, -math.inf, math.nan, -0.0]).to(kind)
        got = run.orthogonal_update(g, base, 1.0, 1.0, [QUINTIC], 1e-7)
        assert torch.equal(got.nan_to_num(7.0), base.nan_to_num(7.0))
        got = run.orthogonal_update(g, base, 1.0 + 2.0 * u, 1.0, [QUINTIC], 1e-7)[0, 0, :5]
        assert float(got[0]) == math.inf and torch.equal(got[1:4], base[0, 0, 1:4]) and bool(got[4].isnan())


def check_update_zeros(run):
    """A matrix of zeros gives zeros with the least eps there is and whatever the steps raise, and leaves the others alone."""
    for rows, cols in ((5, 40), (900, 6), (20, 41), (70, 80)):
        g = torch.randn(3, rows, cols, generator=torch.Generator().manual_seed(rows))
        g[1] = 0.0
        for steps in ([QUINTIC] * 2, LISTS["8"], [(1e200, 0.0, 0.0), (1e-200, 0.0, 0.0)], [(1e200, 1e100, 0.0)] * 3):
            got = run.orthogonal_update(g, None, 1.0, 1.0, steps, 5e-324)
            assert not got[1].any()
            if steps[0] == QUINTIC:
                want, _ = update_longer(g[[0, 2]], steps, 0.0)
                near(got[[0, 2]], want, 2 * ULP * want.abs() + 2.0 ** -31)


# --------------------------------------------------------------------------------------------------- eight bits

INT8 = [  # type, rows, inner, outer, pad, bias, residual
    ("f32", 1, 1, 1, 0, False, False), ("bf16", 1, 130, 20, 0, True, False), ("f16", 3, 127, 33, 1, False, True), ("f32", 17, 128, 16, 0, True, True),
    ("bf16", 40, 33, 70, 0, False, False), ("f16", 65, 257, 65, 3, True, True), ("f32", 2, 1025, 130, 0, False, True), ("bf16", 130, 64, 40, 8, True, False),
    ("f16", 1, 2049, 7, 0, True, True), ("f32", 70, 300, 5, 1, False, False), ("bf16", 20, 700, 90, 0, True, True), ("bf16", 1, 9000, 3, 0, False, False),
    ("f16", 6, 2050, 20, 1, True, True), ("f32", 19, 2300, 18, 0, False, True), ("bf16", 33, 2048, 70, 0, True, False), ("f32", 2, 20000, 5, 0, True, False),
]
INT8_LARGE = [
    ("bf16", 1, 4096, 4096, 0, False, False), ("f16", 16, 4096, 515, 0, True, True), ("f32", 64, 1000, 1001, 1, True, False), ("f16", 3001, 1001, 515, 0, True, True),
    ("bf16", 300, 600, 2050, 0, False, True), ("f32", 1030, 2000, 1100, 0, False, False), ("bf16", 2100, 520, 2100, 8, True, True), ("f32", 33, 20000, 64, 0, True, True),
    ("f16", 5000, 20, 20, 0, False, False), ("bf16", 7, 130944, 9, 0, True, False), ("bf16", 257, 8192, 130, 0, False, False), ("f32", 129, 128, 5000, 3, True, True),
]


def eight_bits(x):
    """The definition, with its two roundings to float32: whole numbers and the rows' scales."""
    x = x.float()
    amax = x.abs().amax(1, keepdim=True)
    bad = ~amax.isfinite()
    first = torch.where(amax < 2.0 ** -100, 2.0 ** 64, 1.0)
    by = torch.where((amax > 0) & ~bad, torch.full_like(amax, 127.0) / (amax * first), 0.0)
    q = torch.where(bad | (amax == 0), 0.0, torch.round(x * first * by))
    return q, torch.where(bad, math.nan, amax / torch.full_like(amax, 127.0))[:, 0]


def check_quantize(run, kind, rows, cols, pad):
    gen = torch.Generator().manual_seed(rows * 17 + cols)
    x = normal(gen, rows, cols, kind=TYPES[kind], pad=pad)
    q, scale = run.quantize_rows(x)
    want, by = eight_bits(x)
    assert q.dtype == torch.int8 and q.shape == (rows, (cols + 127) // 128 * 128)
    assert torch.equal(q[:, :cols].float(), want) and not q[:, cols:].any() and torch.equal(scale, by)


def check_quantize_special(run):
    for kind in TYPES.values():
        f = torch.finfo(kind)
        x = torch.zeros(8, 40, dtype=kind)
        x[1], x[2, 3], x[3, 4], x[4], x[5] = 3.0, math.nan, -math.inf, f.max, f.smallest_normal
        x[5, 0], x[6], x[7, 39] = -f.smallest_normal, -f.max, f.smallest_normal * f.eps  # (the least there is)
        q, scale = run.quantize_rows(x)
        want, by = eight_bits(x)
        assert torch.equal(q[:, :40].float(), want) and torch.equal(scale.isnan(), by.isnan())
        assert torch.equal(scale.nan_to_num(), by.nan_to_num())
        assert not q[0].any() and float(scale[0]) == 0.0 and int(q[1, 0]) == 127 and int(q[6, 0]) == -127 and int(q[5, 0]) == -127 and int(q[7, 39]) == 127
        w, ws = run.quantize_rows(torch.ones(3, 40, dtype=kind))
        y = run.int8_forward(x, w, ws, None, None)
        assert bool(y[2].isnan().all()) and bool(y[3].isnan().all()) and not y[0].any() and int(y.isnan().sum()) == 6


def int8_inputs(kind, rows, inner, outer, pad, bias, residual):
    gen = torch.Generator().manual_seed(rows * 19 + inner)
    kind = TYPES[kind]
    x, w = normal(gen, rows, inner, kind=kind, pad=pad), normal(gen, outer, inner, sigma=inner ** -0.5, kind=kind)
    return x, w, torch.randn(outer, generator=gen) if bias else None, normal(gen, rows, outer, kind=kind, pad=pad) if residual else None


def check_int8(run, kind, rows, inner, outer, pad, bias, residual):
    x, w, bias, residual = int8_inputs(kind, rows, inner, outer, pad, bias, residual)
    wq, ws = run.quantize_rows(w)
    xw, xs = eight_bits(x)
    ww, _ = eight_bits(w)
    got = run.int8_forward(x, wq, ws, bias, residual)
    part = xs.double()[:, None] * ws.double() * (xw.double() @ ww.double().T)
    want, most = part, part.abs()
    if bias is not None:
        want, most = want + bias, most + bias.abs()
    if residual is not None:
        want, most = want + residual.double(), most + residual.double().abs()
    assert got.dtype == x.dtype
    # the sum's, the scales' and the products' roundings to float32, two additions, and one to the type
    near(got, want, UNIT[x.dtype] * want.abs() + 5 * ULP * most + TINY[x.dtype])
    xq, x_scale = run.quantize_rows(x)
    assert torch.equal(run.int8_product(xq, x_scale, wq, ws, inner, x.dtype, bias, residual), got)


def check_int8_limits(run):
    """The longest sum of the greatest numbers is exact."""
    cols = 130944
    x = torch.ones(2, cols)
    x[1] = -1.0
    w = torch.ones(2, cols)
    w[1, ::2] = -1.0
    wq, ws = run.quantize_rows(w)
    got = run.int8_forward(x, wq, ws, None, None)
    want = torch.tensor([[1.0, 0.0], [-1.0, 0.0]], dtype=torch.float64) * cols
    near(got, want, 5 * ULP * want.abs())


INT8_SCALES = [(2, 300, 40), (16, 2048, 20), (20, 2100, 18), (40, 300, 70)]
INT8_SCALES_LARGE = [(300, 600, 2050), (2050, 200, 2050), (4097, 300, 4097)]


def check_int8_scales(run, rows, inner, outer):
    """Scales whose product alone is below the least normal number, or above the greatest, where the results are ordinary: each sum is a whole
    number times both."""
    gen = torch.Generator().manual_seed(rows)
    for kind in (torch.float32, torch.bfloat16):
        x, w = torch.randn(rows, inner, generator=gen), torch.randn(outer, inner, generator=gen)
        x[0], w[0] = 1.0, 1.0
        x[1], w[1] = 0.0, 0.0
        x[1, :2], w[1, 0], w[1, 1] = 1.0, 1.0, -1.0  # (against each other a sum of zero)
        for by_x, by_w in ((2.0 ** -60, 2.0 ** -60), (2.0 ** -20, 2.0 ** -98), (2.0 ** 90, 2.0 ** -95), (2.0 ** 60, 2.0 ** 100)):
            wq, ws = run.quantize_rows((w * by_w).to(kind))
            xq, xs = eight_bits((x * by_x).to(kind))
            ww, _ = eight_bits((w * by_w).to(kind))
            got = run.int8_forward((x * by_x).to(kind), wq, ws, None, None)
            want = xs.double()[:, None] * ws.double() * (xq.double() @ ww.double().T)
            assert float(want[1, 1]) == 0.0 and float(got[1, 1]) == 0.0
            most, greatest = want.abs(), torch.finfo(kind).max
            want = torch.where(most > greatest, want.sign() * math.inf, want)
            clear = (most / greatest - 1.0).abs() > 2.0 ** -6  # (not within a rounding of the greatest number)
            room = torch.where(most > greatest, 0.0, UNIT[kind] * most + 5 * ULP * most + TINY[kind])
            near(torch.where(clear, got.double(), 0.0), torch.where(clear, want, 0.0), room)
    # a row whose scale is below the least number is zero whatever the weights are
    wq, ws = run.quantize_rows(torch.full((outer, inner), 2.0 ** 127))
    assert not run.int8_forward(torch.full((rows, inner), 2.0 ** -149), wq, ws, None, None).any()


INT8_WIDE = [  # more outputs than a common model's width: rows that the multiplying blocks bring to eight bits themselves, and one more
    ("bf16", 1, 130, 4100, 0, True, True), ("f32", 3, 2050, 4113, 1, False, False), ("f16", 4, 1001, 5000, 0, True, False), ("bf16", 5, 520, 4097, 0, False, True),
    ("f32", 16, 100, 4096, 0, True, False), ("f32", 4, 300, 8192, 0, False, True), ("bf16", 4, 140, 8193, 0, True, False), ("f16", 1, 300, 8193, 0, False, False),
]
INT8_WIDE_LARGE = [("bf16", 1, 4096, 32000, 0, False, False), ("f16", 2, 8192, 20001, 0, True, True), ("bf16", 4, 2048, 128000, 0, False, False)]

# --------------------------------------------------------------------------------------------------- each kernel form

def norm_forms(kind):
    """Every group size, with and without a vector across the row's end, by mode: rows that fill no block and rows that fill several."""
    for n, cols in enumerate((3, 8, 30, 64, 130, 512, 777, 1500, 2048, 3001, 4096, 5003, 8192, 8193, 9000)):
        for block, post, gate, pre in ((True, True, "cols", True), (True, True, "full", True), (False, False, "none", True), (True, n % 2 == 0, "none", n % 3 == 0)):
            yield (kind, 5 if n % 2 else 19, cols, n % 2, n % 3, block, post, gate, pre, 1.0 if not block else 0.75)


def update_forms(kind, tall):
    """Every number of tiles, filled and not, with loads of whole and of single elements, by one launch and by several."""
    for k in (1, 5, 16, 17, 24, 32, 33, 36, 48, 50, 64, 65, 72, 90, 96, 97, 100, 128):
        for length in ((k, 70, 800, 1100) if k <= 16 else (k, 140, 300)):
            if length >= k:
                rows, cols = (length, k) if tall else (k, length)
                yield (kind, 2 if k % 2 else 9, rows, cols, k % 3 == 0, [QUINTIC] * (1 + k % 3), k % 2)


def int8_forms(kind):
    """Rows that a block brings to eight bits itself, few rows, and tiles of three sizes."""
    for rows, inner, outer in ((1, 2048, 40), (2, 100, 17), (3, 4096, 33), (4, 8192, 20), (4, 8200, 20), (5, 2048, 40), (5, 8200, 20), (8, 4096, 40), (9, 3500, 40), (11, 300, 4097), (13, 70, 4096), (16, 2049, 4096), (17, 2048, 30), (32, 4100, 9),
                               (33, 2048, 30), (32, 2048, 4097), (8, 1900, 50), (70, 40, 70), (2050, 130, 2050), (4090, 200, 4093), (4097, 3000, 4097)):
        yield (kind, rows, inner, outer, 0, rows % 2 == 0, rows % 3 == 0)
