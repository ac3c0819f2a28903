"""What the tests of a party's local operators share: the definitions in 64 bits, inputs, the sizes at which the kernels can go
wrong, and checks that take the operators as a `run` object, so that the CPU build of the kernels and the GPU go through the same
ones. `run` has the binding's functions on host tensors.

Tolerances follow from the arithmetic and were set before the first run. u is half the distance between neighbours of a result's
type at 1, 2^-24 / 2^-11 / 2^-8 for float32 / float16 / bfloat16: one rounding to the type. A sum of n float32 terms is off by at most n
roundings of the sum of magnitudes; two ulp are allowed for each, which leaves room for how matrix instructions round."""
import math

import numpy as np
import torch

TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
UNIT = {t: torch.finfo(t).eps / 2 for t in TYPES.values()}
TINY = {torch.float32: 2.0 ** -126, torch.float16: 2.0 ** -24, torch.bfloat16: 2.0 ** -126}  # of a result's type


def philox(group, row, seed, offset):
    """The four words of one call, in Python integers (Salmon et al. 2011, ten rounds)."""
    c = [group, row, offset & 0xFFFFFFFF, offset >> 32]
    k = [seed & 0xFFFFFFFF, seed >> 32]
    for _ in range(10):
        x, y = c[0] * 0xD2511F53, c[2] * 0xCD9E8D57
        c = [(y >> 32) ^ c[1] ^ k[0], y & 0xFFFFFFFF, (x >> 32) ^ c[3] ^ k[1], x & 0xFFFFFFFF]
        k = [(k[0] + 0x9E3779B9) & 0xFFFFFFFF, (k[1] + 0xBB67AE85) & 0xFFFFFFFF]
    return c


def factor(rows, cols, p, seed, offset):
    """float64 factors of dropout."""
    t = round(65536 * p)
    out = np.zeros((rows, cols))
    for r in range(rows):
        for g in range((cols + 7) // 8):
            words = philox(g, r, seed, offset)
            for j in range(min(8, cols - 8 * g)):
                draw = words[j // 2] >> (16 * (j % 2)) & 0xFFFF
                out[r, 8 * g + j] = 65536.0 / (65536.0 - t) if draw >= t else 0.0
    return torch.from_numpy(out)


def near(got, want, room):
    """Infinities and NaN in the same places, the rest within `room`."""
    got, want = got.double(), want.double()
    assert got.shape == want.shape
    assert torch.equal(got.isnan(), want.isnan()) and torch.equal(got.isinf(), want.isinf())
    assert torch.equal(got[want.isinf()], want[want.isinf()])
    fine = want.isfinite()
    room = torch.as_tensor(room, dtype=torch.float64).expand(want.shape)[fine]
    off = (got - want)[fine].abs()
    assert bool((off <= room).all()), "off by %g where %g is allowed" % (float(off[off > room].max()), float(room[off > room].max()))


def normal(gen, *shape, sigma=1.0, kind=torch.float32, pad=0, first=0):
    """A matrix whose rows lie `pad` elements further apart than they are long, `first` elements into their array."""
    wide = (torch.randn(*shape[:-1], shape[-1] + pad + first, generator=gen) * sigma).to(kind)
    return wide[..., first:first + shape[-1]]


# --------------------------------------------------------------------------------------------------- dropout

DROPOUT = [  # type, rows, cols, pad, first, p, residual
    ("f32", 1, 1, 0, 0, 0.5, False), ("bf16", 1, 7, 0, 0, 0.3, True), ("f16", 3, 8, 0, 0, 0.5, False),
    ("bf16", 5, 33, 0, 0, 0.1, True), ("f32", 4, 40, 8, 0, 0.25, True), ("f16", 7, 64, 8, 0, 0.9, True),
    ("bf16", 3, 129, 3, 1, 0.5, False), ("f32", 2, 1000, 5, 3, 0.05, True), ("f16", 130, 24, 0, 0, 0.5, False),
    ("f32", 6, 48, 0, 0, 0.0, True), ("bf16", 6, 48, 0, 0, 1.0, True), ("f16", 6, 20, 0, 0, 1.0, False),
]


def check_dropout(run, kind, rows, cols, pad, first, p, residual, seed=2 ** 63 + 12345, offset=2 ** 40 + 7):
    gen = torch.Generator().manual_seed(rows * 1000 + cols)
    kind = TYPES[kind]
    x = normal(gen, rows, cols, kind=kind, pad=pad, first=first)
    res = normal(gen, rows, cols, kind=kind, pad=pad, first=first) if residual else None
    f = factor(rows, cols, p, seed, offset)
    scaled = torch.where(f > 0, x.double() * f, 0.0)
    want = scaled + (res.double() if residual else 0.0)
    got = run.dropout(x, p, seed, offset, residual=res)
    assert got.dtype == kind
    near(got, want, UNIT[kind] * want.abs() + 2.0 ** -22 * (scaled.abs() + want.abs()) + TINY[kind])
    if not residual:
        assert torch.equal(got == 0, (f == 0) | (x == 0))


def check_dropout_special(run):
    """Whatever a dropped element holds is gone; other seeds and offsets drop others; the share is about p."""
    x = torch.full((16, 64), math.nan)
    x[::2] = math.inf
    f = factor(16, 64, 0.5, 5, 0)
    got = run.dropout(x, 0.5, 5, 0)
    assert torch.equal(got == 0, f == 0) and bool(got[1::2][f[1::2] > 0].isnan().all()) and bool((got[::2][f[::2] > 0] == math.inf).all())
    ones = torch.ones(64, 256)
    masks = [run.dropout(ones, 0.25, s, o) for s, o in ((1, 0), (2, 0), (1, 1), (1 + 2 ** 32, 0), (1, 2 ** 32))]
    for i, m in enumerate(masks):
        assert abs(float((m == 0).float().mean()) - 0.25) < 6 * math.sqrt(0.25 * 0.75 / ones.numel())
        assert all(not torch.equal(m, o) for o in masks[:i])


# --------------------------------------------------------------------------------------------------- adapters

ADAPTERS = [  # type, rows, inner, outer, rank, parties, p, order, pad
    ("bf16", 1, 1, 1, 1, 1, 0.0, "sorted", 0), ("f32", 1, 40, 24, 4, 3, 0.0, "mixed", 0), ("f16", 2, 8, 130, 16, 2, 0.5, "mixed", 0),
    ("bf16", 17, 64, 64, 16, 4, 0.1, "mixed", 0), ("f32", 20, 33, 19, 5, 3, 0.2, "mixed", 3), ("bf16", 33, 72, 40, 17, 2, 0.1, "sorted", 8),
    ("f16", 40, 31, 70, 3, 9, 0.3, "none", 1), ("bf16", 70, 136, 136, 8, 64, 0.0, "mixed", 0), ("f32", 130, 16, 8, 2, 2, 0.1, "sorted", 0),
    ("f16", 5, 520, 24, 65, 2, 0.0, "mixed", 0), ("bf16", 131, 24, 16, 16, 3, 0.5, "one", 0), ("f32", 3, 12, 520, 128, 1, 0.0, "bad", 0),
]

ADAPTERS_LARGE = [  # for the GPU: several tiles, chunks and parts
    ("bf16", 300, 1032, 520, 16, 8, 0.1, "sorted", 0), ("f16", 257, 515, 1025, 24, 5, 0.2, "mixed", 1), ("f32", 400, 260, 300, 8, 3, 0.1, "mixed", 0),
    ("bf16", 1, 4096, 1024, 16, 8, 0.0, "sorted", 0), ("bf16", 64, 2048, 1024, 16, 64, 0.0, "mixed", 0), ("f32", 16, 1000, 600, 4, 16, 0.0, "mixed", 0),
    ("f16", 31, 2056, 264, 64, 4, 0.0, "mixed", 0), ("bf16", 600, 256, 264, 64, 1, 0.5, "one", 0),
]


def adapter_inputs(kind, rows, inner, outer, rank, parties, order, pad, seed=0):
    gen = torch.Generator().manual_seed(seed + rows * 7 + inner)
    kind = TYPES[kind]
    x, w = normal(gen, rows, inner, kind=kind, pad=pad), normal(gen, outer, inner, sigma=inner ** -0.5, kind=kind, pad=pad)
    a, b = normal(gen, parties, rank, inner, sigma=inner ** -0.5, kind=kind), normal(gen, parties, outer, rank, sigma=0.5, kind=kind)
    dy = normal(gen, rows, outer, kind=kind, pad=pad)
    scale = torch.rand(parties, generator=gen) + 0.5
    index = torch.randint(-1, parties, (rows,), generator=gen)
    if order == "sorted":
        index = index.clamp(min=0).sort().values
    elif order == "none":
        index[:] = -1
    elif order == "one":
        index[:] = parties - 1
    elif order == "bad":
        index[0], index[-1] = parties, -7
    return x, w, a.contiguous(), b.contiguous(), scale, index.to(torch.int32), dy


def adapter_exact(x, w, a, b, scale, index, dy, f, absolute=False):
    """Forward and backward in 64 bits; `absolute`: with every factor's magnitude, which bounds the sums."""
    t64 = (lambda v: v.double().abs()) if absolute else (lambda v: v.double())
    x, w, a, b, dy = (t64(v) for v in (x, w, a, b, dy))
    xd = torch.where(f > 0, x * f, 0.0)
    y, h, dx = x @ w.T, torch.zeros(x.shape[0], a.shape[1], dtype=torch.float64), dy @ w
    da, db = torch.zeros_like(a), torch.zeros_like(b)
    for t, p in enumerate(index.tolist()):
        if not 0 <= p < a.shape[0]:
            continue
        h[t] = scale[p].double() * (a[p] @ xd[t])
        y[t] += b[p] @ h[t]
        g = scale[p].double() * (b[p].T @ dy[t])
        dx[t] += torch.where(f[t] > 0, f[t] * (a[p].T @ g), 0.0)
        da[p] += torch.outer(g, xd[t])
        db[p] += torch.outer(dy[t], h[t])
    return y, h, dx, da, db


def check_adapters(run, kind, rows, inner, outer, rank, parties, p, order, pad, seed=77, offset=2 ** 35 + 1):
    x, w, a, b, scale, index, dy = adapter_inputs(kind, rows, inner, outer, rank, parties, order, pad)
    f = factor(rows, inner, p, seed, offset)
    want, most = (adapter_exact(x, w, a, b, scale, index, dy, f, absolute=m) for m in (False, True))
    y, h, status = run.adapter_forward(x, w, a, b, scale, index, p, seed, offset)
    assert status == (1 if order == "bad" else 0)
    assert y.dtype == x.dtype and h.dtype == torch.float32
    u, ulp = UNIT[x.dtype], 2.0 ** -23
    near(y, want[0], u * want[0].abs() + (inner + rank + 8) * ulp * most[0] + TINY[x.dtype])
    near(h, want[1], (inner + 8) * ulp * most[1])
    dx, da, db, status = run.adapter_backward(dy, x, w, a, b, scale, index, h, p, seed, offset)
    assert status == (1 if order == "bad" else 0)
    assert dx.dtype == x.dtype and da.dtype == torch.float32 and db.dtype == torch.float32
    near(dx, want[2], u * want[2].abs() + (outer + rank + 8) * ulp * most[2] + TINY[x.dtype])
    near(da, want[3], (outer + rows + 8) * ulp * most[3])
    near(db, want[4], (inner + rows + 8) * ulp * most[4])


def check_adapters_other_parties_infinities(run):
    """What another party's adapter holds does not reach a row, nor does what another row holds."""
    for kind in ("f32", "bf16"):
        x, w, a, b, scale, index, dy = adapter_inputs(kind, 40, 24, 20, 4, 3, "mixed", 0)
        index[:] = torch.arange(40) % 2  # party 2 has no row
        clean = run.adapter_forward(x, w, a, b, scale, index, 0.0, 0, 0)
        back = run.adapter_backward(dy, x, w, a, b, scale, index, clean[1], 0.0, 0, 0)
        a[1], b[1], a[2], b[2] = math.inf, math.nan, math.nan, math.inf
        x[3], dy[5] = math.nan, math.inf
        dirty = run.adapter_forward(x, w, a, b, scale, index, 0.0, 0, 0)
        mine = index == 0
        assert torch.equal(dirty[0][mine], clean[0][mine]) and torch.equal(dirty[1][mine], clean[1][mine])
        dirty_back = run.adapter_backward(dy, x, w, a, b, scale, index, clean[1], 0.0, 0, 0)
        assert torch.equal(dirty_back[0][mine], back[0][mine])
        assert torch.equal(dirty_back[1][0], back[1][0]) and torch.equal(dirty_back[2][0], back[2][0])
        assert not dirty_back[1][2].any() and not dirty_back[2][2].any()


# --------------------------------------------------------------------------------------------------- labels

LABELS = [  # type, rows, cols, pad, first, top, mask
    ("f32", 1, 1, 0, 0, 1, ""), ("f32", 70, 2, 0, 0, 2, ""), ("bf16", 5, 7, 0, 0, 3, "inf"), ("f16", 300, 32, 0, 0, 32, "low"),
    ("bf16", 6, 33, 0, 0, 5, ""), ("f32", 9, 100, 3, 1, 64, "inf"), ("f16", 3, 515, 1, 3, 20, "inf"), ("bf16", 2, 2048, 0, 0, 0, ""),
    ("f32", 2, 2049, 0, 0, 7, "low"), ("bf16", 1, 9000, 0, 5, 20, "inf"), ("f16", 3, 4101, 0, 0, 64, "ties"), ("bf16", 3, 5000, 0, 0, 10, "ties"),
    ("f32", 4, 64, 0, 0, 64, "ties"), ("bf16", 5, 2600, 0, 0, 0, "inf"),
]

LABELS_LARGE = [  # for the GPU: long rows in parts, many rows
    ("bf16", 1, 131072, 0, 0, 20, "inf"), ("f32", 17, 50001, 0, 0, 64, ""), ("f16", 64, 20003, 5, 1, 5, "inf"), ("bf16", 1500, 3000, 0, 0, 8, "ties"),
    ("f32", 5000, 2, 0, 0, 1, "low"), ("bf16", 1100, 2500, 1, 0, 0, ""),
]


def label_inputs(kind, rows, cols, pad, first, mask):
    gen = torch.Generator().manual_seed(cols * 3 + rows)
    kind = TYPES[kind]
    x = normal(gen, rows, cols, sigma=3.0, kind=kind, pad=pad, first=first)
    if mask == "ties":
        x.copy_((x.float().round().clamp(-2, 2) * 0.5).to(kind))
        x[0] = 1.0
        x[1, ::2] = -0.0
        x[1, 1::2] = 0.0
    elif mask:
        hide = torch.rand(rows, cols, generator=gen) < 0.5
        x[hide] = -math.inf if mask == "inf" else torch.finfo(kind).min
        x[-1] = -math.inf if mask == "inf" else torch.finfo(kind).min
    label = torch.randint(0, cols, (rows,), generator=gen)
    label[::5] = -1
    if rows > 2:
        label[2] = cols  # out of range
    return x, label.to(torch.int32), gen


def label_exact(x, label, top):
    x = x.double()
    some = ~(x == -math.inf).all(1)
    m = torch.where(some, x.amax(1), 0.0)
    lse = torch.where(some, m + torch.log(torch.exp(x - m[:, None]).sum(1)), -math.inf)
    lp = torch.where(some[:, None], x - lse[:, None], -math.inf)
    prob = torch.exp(lp)
    entropy = -torch.where(prob > 0, prob * lp, 0.0).sum(1)
    has = (label >= 0) & (label < x.shape[1])
    logp = torch.where(has, lp.gather(1, label.long().clamp(0, x.shape[1] - 1)[:, None])[:, 0], 0.0)
    order = np.lexsort((np.broadcast_to(np.arange(x.shape[1]), x.shape), -x.numpy()), axis=1)[:, :top]
    index = torch.from_numpy(order.copy())
    return logp, entropy, lse, lp.gather(1, index), index, lp, prob, has, some


def check_labels(run, kind, rows, cols, pad, first, top, mask):
    x, label, gen = label_inputs(kind, rows, cols, pad, first, mask)
    logp, entropy, lse, top_logp, index, lp, prob, has, some = label_exact(x, label, top)
    got = run.label_logprobs(x, label, top)
    assert got[5] == int(bool((~has & (label != -1)).any()))
    # a logarithm of the sum: one exponential's error, which grows with the distance from the maximum that the terms with
    # weight have, and the roundings of the sum over a lane's share
    size = torch.where(some, x.double().amax(1).abs(), 0.0)
    mean = torch.where(some, torch.where(prob > 0, prob * (lp - lp.amax(1, keepdim=True)).abs(), 0.0).sum(1), 0.0)
    room = 2.0 ** -22 * (8 + size + mean) + (cols / 64 + 32) * 2.0 ** -23
    finite = torch.where(logp.isfinite(), logp.abs(), 0.0)
    near(got[0], logp, room + 2.0 ** -22 * finite)
    near(got[1], entropy, room * (1 + mean))
    near(got[2], lse, room)
    if top:
        assert torch.equal(got[4].long(), index)
        near(got[3], top_logp, room[:, None] + 2.0 ** -22 * torch.where(top_logp.isfinite(), top_logp.abs(), 0.0))
    dlogp, dh = torch.randn(rows, generator=gen), torch.randn(rows, generator=gen)
    for with_top, with_entropy in ((True, True), (False, True), (False, False)):
        dtop = torch.randn(rows, top, generator=gen) if top and with_top else None
        dx = run.label_logprobs_backward(x, label, got[2], got[1], dlogp, dh if with_entropy else None, got[4] if dtop is not None else None, dtop)
        given = torch.where(has, dlogp, 0.0).double()
        one = torch.zeros(rows, cols, dtype=torch.float64)
        one[torch.arange(rows)[has], label[has].long()] += dlogp[has].double()
        if dtop is not None:
            one.scatter_add_(1, index, dtop.double())
            given = given + dtop.double().sum(1)
        d = dh.double() if with_entropy else torch.zeros(rows, dtype=torch.float64)
        safe = torch.where(prob > 0, lp, 0.0)
        want = prob * (-given[:, None] - d[:, None] * (safe + entropy[:, None])) + one
        want = torch.where(some[:, None], want, 0.0)
        weight = prob * (given.abs()[:, None] + d.abs()[:, None] * (safe.abs() + entropy[:, None] + 1))
        close = UNIT[x.dtype] * want.abs() + weight * (room[:, None] * 2 + 2.0 ** -21 * (8 + safe.abs())) + 2.0 ** -20 * one.abs() + TINY[x.dtype]
        if dtop is not None:  # their sum's own roundings
            close = close + (top + 2) * 2.0 ** -23 * (prob * dtop.abs().sum(1).double()[:, None] + one.abs())
        near(dx, want, torch.where(some[:, None], close, 0.0))


def check_labels_nan(run):
    """A NaN or +inf makes its own row NaN and no other; NaN is first among the alternatives, the lowest column first."""
    for cols in (5, 70, 3000):
        x = torch.randn(4, cols, generator=torch.Generator().manual_seed(cols))
        clean = run.label_logprobs(x, torch.zeros(4, dtype=torch.int32), 3)
        x[1, cols - 1], x[1, cols - 2], x[2, 1] = math.nan, math.nan, math.inf
        got = run.label_logprobs(x, torch.zeros(4, dtype=torch.int32), 3)
        for g, c in zip(got[:4], clean):
            assert torch.equal(g[0], c[0]) and torch.equal(g[3], c[3]) and bool(g[1:3].isnan().all())
        assert got[4][1, :2].tolist() == [cols - 2, cols - 1] and got[4][2, 0] == 1
        dx = run.label_logprobs_backward(x, torch.zeros(4, dtype=torch.int32), got[2], got[1], torch.ones(4), None, None, None)
        assert bool(dx[1:3].isnan().all()) and not bool(dx[[0, 3]].isnan().any())


# --------------------------------------------------------------------------------------------------- adapters, more than 256 rows

ADAPTERS_SHORT_SUMS = [  # sums of few terms, which leave their own roundings little room
    ("f16", 256, 1, 24, 1, 3, 0.0, "one", 0), ("f16", 300, 1, 24, 1, 3, 0.0, "one", 0), ("bf16", 500, 3, 70, 2, 300, 0.3, "mixed", 1),
    ("f32", 300, 1, 24, 1, 3, 0.0, "one", 0),
]


def check_adapters_cancelling(run, kind, rows):
    """W = -B A but for its rounding: what is left of y and dx shows how many bits of h and g the adapters' part takes."""
    inner, outer, rank = 2, 3, 2
    x, w, a, b, scale, index, dy = adapter_inputs(kind, rows, inner, outer, rank, 2, "one", 0)
    scale[:] = 1.0
    w.copy_((-(b[1].double() @ a[1].double())).to(w.dtype))
    f = factor(rows, inner, 0.0, 1, 0)
    want, most = (adapter_exact(x, w, a, b, scale, index, dy, f, absolute=m) for m in (False, True))
    u, ulp = UNIT[x.dtype], 2.0 ** -23
    y, h, _ = run.adapter_forward(x, w, a, b, scale, index, 0.0, 1, 0)
    near(y, want[0], u * want[0].abs() + (inner + rank + 8) * ulp * most[0] + TINY[x.dtype])
    dx, _, _, _ = run.adapter_backward(dy, x, w, a, b, scale, index, h, 0.0, 1, 0)
    near(dx, want[2], u * want[2].abs() + (outer + rank + 8) * ulp * most[2] + TINY[x.dtype])


def check_adapters_own_infinities(run, kind):
    """An infinity that a row's own adapter or its h or g holds reaches the results that it is a term of, as infinity or, against a
    zero, as NaN, however many rows come together. All else is small integers, whose sums are exact."""
    few = None
    for rows in (256, 257):
        inner, outer, rank, parties = 8, 16, 3, 2
        gen = torch.Generator().manual_seed(9)
        ints = lambda *s: torch.randint(-2, 3, s, generator=gen).to(TYPES[kind])  # noqa: E731
        w, a, b = ints(outer, inner), ints(parties, rank, inner), ints(parties, outer, rank)
        x, dy, index = ints(257, inner)[:rows], ints(257, outer)[:rows], (torch.arange(rows) % 3 - 1).to(torch.int32)
        b[1, 2, 0], b[1, 3, 1], a[1, 2, 4] = math.inf, -math.inf, math.inf  # a row's B, and its A, so its h
        scale = torch.tensor([1.0, 2.0])
        f = factor(rows, inner, 0.0, 1, 0)
        want = adapter_exact(x, w, a, b, scale, index, dy, f)
        y, h, _ = run.adapter_forward(x, w, a, b, scale, index, 0.0, 1, 0)
        near(y, want[0], 0.0)
        near(h, want[1], 0.0)
        dx, _, _, _ = run.adapter_backward(dy, x, w, a, b, scale, index, h, 0.0, 1, 0)
        near(dx, want[2], 0.0)
        if rows == 256:
            assert bool(y.isinf().any()) and bool(y.isnan().any()) and bool(dx.isinf().any() | dx.isnan().any())
            few = y, dx
        else:
            for got, was in zip((y, dx), few):
                assert torch.equal(got[:256].nan_to_num(7e3), was.nan_to_num(7e3))


# --------------------------------------------------------------------------------------------------- labels, far from zero

LABELS_FAR = [  # type, rows, cols, pad, first, top, shift of the logits, mask
    ("f32", 70, 2, 0, 0, 1, 0.0, "low"), ("f32", 5, 7, 1, 0, 2, 1e5, ""), ("f32", 9, 33, 0, 1, 3, 1e4, "low"), ("bf16", 9, 8, 0, 0, 1, 0.0, "low"),
    ("f16", 30, 100, 3, 0, 5, 3e4, "inf"), ("f32", 4, 512, 0, 0, 0, -1e5, ""), ("f32", 5, 515, 2, 0, 4, 1e6, "inf"), ("bf16", 3, 700, 0, 0, 0, 1e4, "low"),
    ("f32", 3, 2100, 0, 0, 9, 1e5, "low"), ("bf16", 2, 9000, 0, 0, 3, 0.0, "low"), ("f32", 2, 9000, 1, 1, 0, -1e4, ""), ("f16", 2, 33001, 0, 0, 2, 0.0, "low"),
    ("f32", 2, 40000, 0, 0, 0, 1e9, "low"), ("bf16", 1, 300001, 0, 0, 20, 0.0, ""),
]


def check_labels_far(run, kind, rows, cols, pad, first, top, shift, mask):
    """The gradient's accuracy does not depend on where a row's logits lie, as lse's does. A probability is off by its exponential, whose
    argument is rounded and multiplied, and by the sum of the row's; nothing grows with the maximum."""
    x, label, gen = label_inputs(kind, rows, cols, pad, first, "")
    x.copy_((x.float() + shift).to(x.dtype))
    if mask:
        value = -math.inf if mask == "inf" else torch.finfo(x.dtype).min
        x[torch.rand(rows, cols, generator=gen) < 0.5] = value
        x[-1] = value
    _, _, _, _, index, _, _, has, some = label_exact(x, label, top)
    away = torch.where(some[:, None], x.double() - torch.where(some, x.double().amax(1), 0.0)[:, None], -math.inf)  # (64 bits do not hold lse either)
    lp = torch.where(some[:, None], away - torch.exp(away).sum(1, keepdim=True).log(), -math.inf)
    prob = torch.exp(lp)
    entropy = -torch.where(prob > 0, prob * lp, 0.0).sum(1)
    got = run.label_logprobs(x, label, top)
    near(got[1], entropy, 2.0 ** -23 * (40 + 2 * entropy + cols / 64) * (1 + entropy))
    dlogp, dh = torch.randn(rows, generator=gen), torch.randn(rows, generator=gen)
    dtop = torch.randn(rows, top, generator=gen) if top else None
    given = torch.where(has, dlogp, 0.0).double()
    one = torch.zeros(rows, cols, dtype=torch.float64)
    one[torch.arange(rows)[has], label[has].long()] += dlogp[has].double()
    if top:
        one.scatter_add_(1, index, dtop.double())
        given = given + dtop.double().sum(1)
    safe = torch.where(prob > 0, lp, 0.0)
    mean = (prob * safe.abs()).sum(1, keepdim=True)
    for d in (torch.zeros(rows), dh):
        dx = run.label_logprobs_backward(x, label, got[2], got[1], dlogp, d if d is dh else None, index.to(torch.int32) if top else None, dtop)
        d = d.double()
        want = torch.where(some[:, None], prob * (-given[:, None] - d[:, None] * (safe + entropy[:, None])) + one, 0.0)
        ulp = 2.0 ** -23
        far = torch.where(prob > 0, (x.double() - got[2].double()[:, None]).abs(), 0.0)  # what the exponentials are taken of
        of_p = ulp * (40 + 2 * far + 2 * (prob * far).sum(1, keepdim=True) + cols / 64 + top)
        of_entropy = ulp * (40 + 2 * mean + cols / 64) * (1 + mean)
        weight = prob * (given.abs()[:, None] + (dtop.abs().double().sum(1, keepdim=True) if top else 0.0) + d.abs()[:, None] * (safe.abs() + entropy[:, None] + 1))
        room = UNIT[x.dtype] * want.abs() + weight * of_p + prob * d.abs()[:, None] * (of_p + of_entropy) + 2 * (top + 2) * ulp * one.abs() + TINY[x.dtype]
        near(dx, want, torch.where(some[:, None], room, 0.0))


def check_labels_far_columns(run):
    """Columns far below the maximum in float32: their exponentials are as exact as the near ones'. The maximum is 0, and so is lse, whose sum
    the others do not reach; x - lse is exact, and a column's gradient is off by one exponential and a few products."""
    gen = torch.Generator().manual_seed(11)
    x = -torch.rand(40, 100, generator=gen) * 55 - 25
    x[:, 3] = 0.0
    x[:, 70] = -math.inf
    label, given = torch.full((40,), -1, dtype=torch.int32), torch.randn(40, 2, generator=gen)
    label[::2] = 3
    got = run.label_logprobs(x, label, 2)
    assert not got[2].any() and bool((got[4][:, 0] == 3).all())
    dx = run.label_logprobs_backward(x, label, got[2], got[1], given[:, 0].contiguous(), None, got[4], torch.stack((given[:, 1], torch.zeros(40)), 1))
    want = -torch.exp(x.double()) * (torch.where(label >= 0, given[:, 0], 0.0) + given[:, 1])[:, None].double()
    others = torch.arange(100) != 3
    # 2 units of the exponential, its argument's rounding put back to 2^-24 of it, four products, the sum of what is given
    size = torch.exp(x.double()) * given.double().abs().sum(1, keepdim=True)
    near(dx[:, others], want[:, others], (8 * 2.0 ** -24 * size + 2.0 ** -149)[:, others])


# --------------------------------------------------------------------------------------------------- adapters, the forms for many rows

ADAPTERS_MANY = [  # more rows than k_few takes, by tiles of 64 x 64
    ("bf16", 300, 33, 19, 17, 3, 0.2, "mixed", 3), ("f16", 257, 70, 131, 1, 5, 0.1, "mixed", 1), ("f32", 333, 41, 70, 128, 2, 0.3, "mixed", 0),
    ("bf16", 500, 130, 65, 128, 9, 0.5, "sorted", 8), ("f16", 300, 64, 64, 16, 4, 0.1, "none", 0), ("f32", 270, 7, 8, 17, 3, 0.5, "bad", 1),
    ("bf16", 280, 5, 200, 16, 64, 0.1, "bad", 0), ("f16", 400, 600, 24, 17, 40, 0.05, "one", 0), ("f32", 300, 16, 24, 16, 2, 0.0, "mixed", 0),
    ("bf16", 300, 40, 40, 8, 2, 1.0, "mixed", 0),
]

ADAPTERS_TILES = [  # for the GPU: the larger tiles, forward where the outputs are many, backward and with dropout where the inputs are
    ("bf16", 2040, 70, 2040, 16, 5, 0.3, "mixed", 0), ("bf16", 2040, 2040, 70, 3, 5, 0.3, "mixed", 0), ("f16", 2040, 70, 2040, 33, 5, 0.3, "mixed", 1),
    ("f16", 2040, 2040, 70, 16, 5, 0.3, "mixed", 0), ("f16", 2040, 2040, 70, 5, 2, 0.0, "sorted", 0), ("bf16", 4090, 70, 4081, 16, 7, 0.3, "mixed", 0),
    ("bf16", 4090, 4081, 70, 24, 7, 0.3, "mixed", 0), ("bf16", 3900, 3841, 130, 16, 1, 0.0, "one", 0), ("f16", 4090, 70, 4081, 3, 300, 0.3, "mixed", 0),
    ("f16", 4090, 4081, 70, 16, 7, 0.3, "sorted", 0), ("f32", 4090, 33, 4081, 16, 7, 0.3, "mixed", 0), ("f32", 4090, 4081, 33, 5, 7, 0.3, "mixed", 0),
]


def factor_of_many(rows, cols, p, seed, offset):
    """As `factor`, with whole arrays of calls at a time."""
    u, low, t = np.uint64, np.uint64(0xFFFFFFFF), round(65536 * p)
    groups = (cols + 7) // 8
    c = list(np.broadcast_arrays(np.arange(groups, dtype=u)[None], np.arange(rows, dtype=u)[:, None], u(offset & 0xFFFFFFFF), u(offset >> 32)))
    k = [seed & 0xFFFFFFFF, seed >> 32]
    for _ in range(10):
        x, y = c[0] * u(0xD2511F53), c[2] * u(0xCD9E8D57)
        c = [(y >> u(32)) ^ c[1] ^ u(k[0]), y & low, (x >> u(32)) ^ c[3] ^ u(k[1]), x & low]
        k = [(k[0] + 0x9E3779B9) & 0xFFFFFFFF, (k[1] + 0xBB67AE85) & 0xFFFFFFFF]
    draws = np.stack([c[j // 2] >> u(16 * (j % 2)) & u(0xFFFF) for j in range(8)], -1).reshape(rows, groups * 8)[:, :cols]
    return torch.from_numpy(np.where(draws >= t, 65536.0 / max(65536.0 - t, 1.0), 0.0))


def adapter_exact_of_many(x, w, a, b, scale, index, dy, f, absolute=False):
    """As `adapter_exact`, party by party."""
    t64 = (lambda v: v.double().abs()) if absolute else (lambda v: v.double())
    x, w, a, b, dy = (t64(v) for v in (x, w, a, b, dy))
    xd = torch.where(f > 0, x * f, 0.0)
    y, h, dx = x @ w.T, torch.zeros(x.shape[0], a.shape[1], dtype=torch.float64), dy @ w
    da, db = torch.zeros_like(a), torch.zeros_like(b)
    for p in range(a.shape[0]):
        t = (index == p).nonzero()[:, 0]
        h[t] = scale[p].double() * (xd[t] @ a[p].T)
        y[t] += h[t] @ b[p].T
        g = scale[p].double() * (dy[t] @ b[p])
        dx[t] += f[t] * (g @ a[p])
        da[p], db[p] = g.T @ xd[t], dy[t].T @ h[t]
    return y, h, dx, da, db


def check_adapters_of_many(run, kind, rows, inner, outer, rank, parties, p, order, pad, seed=2 ** 40 + 3, offset=5):
    x, w, a, b, scale, index, dy = adapter_inputs(kind, rows, inner, outer, rank, parties, order, pad)
    f = factor_of_many(rows, inner, p, seed, offset)
    want, most = (adapter_exact_of_many(x, w, a, b, scale, index, dy, f, absolute=m) for m in (False, True))
    y, h, status = run.adapter_forward(x, w, a, b, scale, index, p, seed, offset)
    u, ulp = UNIT[x.dtype], 2.0 ** -23
    assert status == (1 if order == "bad" else 0)
    near(y, want[0], u * want[0].abs() + (inner + rank + 8) * ulp * most[0] + TINY[x.dtype])
    near(h, want[1], (inner + 8) * ulp * most[1])
    dx, da, db, status = run.adapter_backward(dy, x, w, a, b, scale, index, h, p, seed, offset)
    assert status == (1 if order == "bad" else 0)
    near(dx, want[2], u * want[2].abs() + (outer + rank + 8) * ulp * most[2] + TINY[x.dtype])
    near(da, want[3], (outer + rows + 8) * ulp * most[3])
    near(db, want[4], (inner + rows + 8) * ulp * most[4])


def check_factor_of_many():
    for rows, cols, p, seed, offset in ((7, 33, 0.3, 2 ** 63 + 5, 2 ** 40 + 9), (3, 8, 1.0, 1, 0), (2, 20, 0.0, 0, 3)):
        assert torch.equal(factor(rows, cols, p, seed, offset), factor_of_many(rows, cols, p, seed, offset))


def check_adapters_isolation(run, kind, rows):
    """What another party's adapter or another row holds does not reach a row, and rows keep their bits."""
    x, w, a, b, scale, index, dy = adapter_inputs(kind, rows, 24, 20, 4, 4, "mixed", 0)
    index[:] = torch.arange(rows) % 3 - 1  # parties 2 and 3 have no row
    clean = run.adapter_forward(x, w, a, b, scale, index, 0.25, 3, 0)
    back = run.adapter_backward(dy, x, w, a, b, scale, index, clean[1], 0.25, 3, 0)
    a[1], b[1], a[2], b[2], a[3], b[3] = math.inf, math.nan, math.nan, math.inf, -math.inf, -math.inf
    x[2], dy[5] = math.nan, math.inf  # rows of party 1
    dirty = run.adapter_forward(x, w, a, b, scale, index, 0.25, 3, 0)
    dirty_back = run.adapter_backward(dy, x, w, a, b, scale, index, clean[1], 0.25, 3, 0)
    mine = index < 1
    assert all(torch.equal(d[mine], c[mine]) for d, c in zip(dirty[:2], clean[:2])) and torch.equal(dirty_back[0][mine], back[0][mine])
    assert torch.equal(dirty_back[1][0], back[1][0]) and torch.equal(dirty_back[2][0], back[2][0])
    assert not dirty_back[1][2:].any() and not dirty_back[2][2:].any()


# what the sizes of the lists above leave of the kernels' forms, by type
ADAPTERS_FORMS = [(kind, rows, 70 + rank, 60, rank, 3, 0.2, "mixed", 1) for kind in TYPES for rows in (9, 25, 70) for rank in (7, 40, 100)]
ADAPTERS_FORMS += [("f16", 260, 90, 30, 100, 2, 0.1, "mixed", 0)]
LABELS_FORMS = [  # as LABELS_FAR
    ("f16", 3, 100, 0, 0, 0, 10.0, "inf"), ("f16", 2, 3000, 1, 0, 0, -10.0, "low"), ("f16", 2, 41001, 0, 1, 3, 0.0, ""), ("bf16", 2, 21000, 3, 0, 4, 0.0, "inf"),
    ("f32", 3, 6001, 0, 0, 3, 100.0, ""), ("f32", 2, 17000, 0, 0, 2, -1000.0, "low"),
]
