"""The kernels of the norms around a block, of orthogonalised updates and of products of eight bits, compiled for the CPU against a
stand-in for the HIP runtime (tests/emu), through the same C entry points, against the definitions in 64 bits. Buffers end at a guard
page, so that an access past an end faults."""
import ctypes as C
import os
import sys

import pytest
import torch

import block_cases as cases
from paper_2107_13797_amd import _cabi
from test_emu_local import NAMES, Buffer

pytestmark = pytest.mark.skipif(not os.path.exists("/opt/rocm/llvm/bin/clang++"), reason="no clang for the half types")
BAD = 2 ** 64 - 1


class Emulated:
    """The binding's functions on host tensors."""

    def __init__(self, lib):
        self.lib = lib

    def buf(self, t):
        return None if t is None else Buffer(self.lib, t)

    def new(self, *shape, kind=torch.float32):
        return self.buf(torch.full(shape, 9, dtype=kind))

    def workspace(self, nbytes):
        assert nbytes != BAD
        return self.buf(torch.full((nbytes,), 0xA5, dtype=torch.uint8)), nbytes

    @staticmethod
    def at(b):
        return None if b is None else b.p

    @staticmethod
    def ld(t):
        return 0 if t is None else t.stride(0) if t.shape[0] > 1 else t.shape[1]

    def norm_operands(self, x, f, post, gate, pre):
        full, by_cols = (gate, None) if gate is not None and gate.dim() == 2 else (None, gate)
        held = [self.buf(t) for t in (x, f, post, full, by_cols, pre)]
        px, pf, ppost, pg, pc, ppre = map(self.at, held)
        return held, (px, self.ld(x), pf, self.ld(f), ppost, pg, self.ld(full), pc, ppre)

    def residual_norm(self, x, f, post, gate, pre, scale, eps):
        (rows, cols), kind = x.shape, x.dtype
        held, operands = self.norm_operands(x, f, post, gate, pre)
        r, h = (None if t is None else self.new(rows, cols, kind=kind) for t in (f, pre))
        rstd = self.new(2, rows)
        assert self.lib.haflo_residual_norm(NAMES[kind], *operands, rows, cols, scale, eps, self.at(r), cols, self.at(h), cols, rstd.p, None) == 0
        return *(None if t is None else t.get() for t in (r, h)), rstd.get()

    def residual_norm_backward(self, dh, dr, x, f, post, gate, pre, rstd, scale):
        (rows, cols), kind = x.shape, x.dtype
        held, operands = self.norm_operands(x, f, post, gate, pre)
        bh, br, bs = (self.buf(t) for t in (dh, dr, rstd))
        dx, df = self.new(rows, cols, kind=kind), None if f is None else self.new(rows, cols, kind=kind)
        full = gate is not None and gate.dim() == 2
        dgate = None if gate is None else self.new(*gate.shape, kind=gate.dtype)
        dpost, dpre = (None if t is None else self.new(cols) for t in (post, pre))
        ws, nbytes = self.workspace(self.lib.haflo_residual_norm_workspace_bytes(NAMES[kind], rows, cols))
        assert self.lib.haflo_residual_norm_backward(
            NAMES[kind], self.at(bh), self.ld(dh), self.at(br), self.ld(dr), *operands, bs.p, rows, cols, scale, dx.p, cols, self.at(df), cols,
            self.at(dgate) if full else None, cols, None if full else self.at(dgate), self.at(dpost), self.at(dpre), ws.p, nbytes, None) == 0
        return tuple(None if t is None else t.get() for t in (dx, df, dpost, dgate, dpre))

    def orthogonal_update(self, g, base, keep, scale, steps, eps):
        bg, bb, out = self.buf(g), self.buf(base), self.new(*g.shape, kind=g.dtype)
        parties, rows, cols = g.shape
        ws, nbytes = self.workspace(self.lib.haflo_update_workspace_bytes(NAMES[g.dtype], parties, rows, cols))
        values = (C.c_double * (3 * len(steps)))(*(v for s in steps for v in s))
        assert self.lib.haflo_orthogonal_update(NAMES[g.dtype], bg.p, g.stride(1), g.stride(0), self.at(bb), cols, rows * cols, parties, rows, cols, values,
                                                len(steps), keep, scale, eps, out.p, cols, rows * cols, ws.p, nbytes, None) == 0
        return out.get()

    def quantize_rows(self, x):
        rows, cols = x.shape
        bx, q, scale = self.buf(x), self.new(rows, (cols + 127) // 128 * 128, kind=torch.int8), self.new(rows)
        assert self.lib.haflo_quantize_rows(NAMES[x.dtype], bx.p, self.ld(x), rows, cols, q.p, scale.p, None) == 0
        return q.get(), scale.get()

    def int8_forward(self, x, wq, ws, bias, residual):
        (rows, inner), outer, kind = x.shape, wq.shape[0], x.dtype
        held = [self.buf(t) for t in (x, wq, ws, bias, residual)]
        px, pw, ps, pb, pr = map(self.at, held)
        y, (room, nbytes) = self.new(rows, outer, kind=kind), self.workspace(self.lib.haflo_int8_workspace_bytes(NAMES[kind], rows, inner, outer))
        assert self.lib.haflo_int8_forward(NAMES[kind], px, self.ld(x), pw, ps, pb, pr, self.ld(residual), rows, inner, outer, y.p, outer, room.p,
                                           nbytes, None) == 0
        return y.get()

    def int8_product(self, xq, xs, wq, ws, inner, kind, bias, residual):
        rows, outer = xq.shape[0], wq.shape[0]
        held = [self.buf(t) for t in (xq, xs, wq, ws, bias, residual)]
        px, pxs, pw, ps, pb, pr = map(self.at, held)
        y = self.new(rows, outer, kind=kind)
        assert self.lib.haflo_int8_product(NAMES[kind], px, pxs, pw, ps, pb, pr, self.ld(residual), rows, inner, outer, y.p, outer, None) == 0
        return y.get()


@pytest.fixture(scope="module")
def run():
    sys.path.insert(0, os.path.join(os.path.dirname(__file__), "emu"))
    import build_emu_local
    lib = _cabi.bind(C.CDLL(build_emu_local.build()), prototypes=_cabi.LOCAL_PROTOTYPES)
    lib.hipemu_alloc.restype = C.c_void_p
    lib.hipemu_alloc.argtypes = [C.c_size_t]
    lib.hipemu_free.argtypes = [C.c_void_p]
    return Emulated(lib)


@pytest.mark.parametrize("case", cases.NORMS, ids=str)
def test_norm(run, case):
    cases.check_norm(run, *case)


def test_norm_special(run):
    cases.check_norm_special(run)


def test_norm_far(run):
    cases.check_norm_far(run)


@pytest.mark.parametrize("case", cases.SUMS, ids=str)
def test_norm_sums(run, case):
    cases.check_norm_sums(run, *case)


def test_norm_gradients(run):
    cases.check_norm_gradients(run)


@pytest.mark.parametrize("case", cases.UPDATES, ids=lambda c: "-".join(map(str, c[:5] + (len(c[5]),))))
def test_update(run, case):
    cases.check_update(run, *case)


@pytest.mark.parametrize("case", cases.STEPS, ids=str)
def test_update_steps(run, case):
    cases.check_update_steps(run, *case)


def test_update_steps_special(run):
    cases.check_update_steps_special(run)


def test_update_special(run):
    cases.check_update_special(run)


def test_update_rounds_once(run):
    cases.check_update_rounds_once(run)


def test_update_zeros(run):
    cases.check_update_zeros(run)


def test_update_orthogonal(run):
    cases.check_update_orthogonal(run)


@pytest.mark.parametrize("case", [c[:3] + (c[4],) for c in cases.INT8], ids=str)
def test_quantize(run, case):
    cases.check_quantize(run, *case)


def test_quantize_special(run):
    cases.check_quantize_special(run)


@pytest.mark.parametrize("case", cases.INT8, ids=str)
def test_int8(run, case):
    cases.check_int8(run, *case)


@pytest.mark.parametrize("case", cases.INT8_SCALES, ids=str)
def test_int8_scales(run, case):
    cases.check_int8_scales(run, *case)


@pytest.mark.parametrize("case", cases.INT8_WIDE, ids=str)
def test_int8_wide(run, case):
    cases.check_int8(run, *case)


def test_int8_limits(run):
    cases.check_int8_limits(run)


def test_in_place(run):
    """Each result over each input that it may lie over gives what it gives elsewhere, also where a vector goes across the row's end."""
    lib, kind = run.lib, torch.float16
    for rows, cols in ((3, 5), (2, 40), (2, 515), (2, 1001), (2, 9001)):
        x, f, post, gate, pre, dh, dr = cases.norm_inputs("f16", rows, cols, 0, 0, True, True, "full", True)
        want_r, want_h, rstd = run.residual_norm(x, f, post, gate, pre, 0.5, 1e-5)
        want = run.residual_norm_backward(dh, dr, x, f, post, gate, pre, rstd, 0.5)
        ws, nbytes = run.workspace(lib.haflo_residual_norm_workspace_bytes(NAMES[kind], rows, cols))
        for over_r, over_h in ((0, 1), (1, 0), (2, 1), (0, 2)):
            b = [run.buf(t) for t in (x, f, gate, post, pre, rstd)]
            px, pf, pg, ppost, ppre, ps = (t.p for t in b)
            r, h = b[over_r], b[over_h]
            assert lib.haflo_residual_norm(NAMES[kind], px, cols, pf, cols, ppost, pg, cols, None, ppre, rows, cols, 0.5, 1e-5, r.p, cols, h.p, cols, ps, None) == 0
            assert torch.equal(r.get(), want_r) and torch.equal(h.get(), want_h)
        for over in ((0, 1, 2), (1, 0, 4), (3, 4, 2), (2, 3, 1)):
            b = [run.buf(t) for t in (dh, dr, gate, x, f, post, pre, rstd)]
            ph, pr, pg, px, pf, ppost, ppre, ps = (t.p for t in b)
            dx, df, dg = (b[i] for i in over)
            vec = [run.new(cols), run.new(cols)]
            assert lib.haflo_residual_norm_backward(NAMES[kind], ph, cols, pr, cols, px, cols, pf, cols, ppost, pg, cols, None, ppre, ps, rows, cols, 0.5, dx.p, cols,
                                                    df.p, cols, dg.p, cols, None, vec[0].p, vec[1].p, ws.p, nbytes, None) == 0
            assert all(torch.equal(a, c) for a, c in zip((dx.get(), df.get(), vec[0].get(), dg.get(), vec[1].get()), want))
    for rows, cols in ((6, 50), (50, 6), (20, 900), (900, 20), (70, 75)):
        g, held = cases.update_inputs("f32", 2, rows, cols, True, 0)
        g = g.contiguous()
        want = run.orthogonal_update(g, held, 0.9, -0.3, [cases.QUINTIC] * 2, 1e-7)
        ws, nbytes = run.workspace(lib.haflo_update_workspace_bytes(0, 2, rows, cols))
        for over in (0, 1):
            b = [run.buf(g), run.buf(held)]
            assert lib.haflo_orthogonal_update(0, b[0].p, cols, rows * cols, b[1].p, cols, rows * cols, 2, rows, cols, (C.c_double * 6)(*cases.QUINTIC * 2), 2, 0.9,
                                               -0.3, 1e-7, b[over].p, cols, rows * cols, ws.p, nbytes, None) == 0
            assert torch.equal(b[over].get(), want)
    for rows in (2, 20):
        x, w, bias, residual = cases.int8_inputs("bf16", rows, 300, 33, 0, True, True)
        q, s = run.quantize_rows(w)
        want = run.int8_forward(x, q, s, bias, residual)
        b = [run.buf(t) for t in (x, q, s, bias, residual)]
        ws, nbytes = run.workspace(lib.haflo_int8_workspace_bytes(2, rows, 300, 33))
        assert lib.haflo_int8_forward(2, b[0].p, 300, b[1].p, b[2].p, b[3].p, b[4].p, 33, rows, 300, 33, b[4].p, 33, ws.p, nbytes, None) == 0
        assert torch.equal(b[4].get(), want)


OVER_X = [(kind, rows, width, outer) for kind in ("f32", "bf16") for rows in (1, 2, 8, 16, 17, 40) for width, outer in ((256, 256), (300, 45), (2048, 64))]


@pytest.mark.parametrize("case", OVER_X, ids=str)
def test_int8_over_its_rows(run, case):
    """A result over x, with x for a residual and without, is what it is elsewhere, whatever the number of rows; the workspace is then that of
    17 rows or more, and a call without it is refused."""
    kind, rows, width, outer = case
    lib = run.lib
    x, w, bias, _ = cases.int8_inputs(kind, rows, width, outer, 0, True, False)
    q, s = run.quantize_rows(w)
    number = NAMES[x.dtype]
    ws, nbytes = run.workspace(lib.haflo_int8_workspace_bytes(number, max(rows, 17), width, outer))
    for with_x in (False, True):
        want = run.int8_forward(x, q, s, bias, x[:, :outer] if with_x else None)
        b = [run.buf(t) for t in (x, q, s, bias)]
        px, pq, ps, pb = (v.p for v in b)
        call = lambda w, n: lib.haflo_int8_forward(number, px, width, pq, ps, pb, px if with_x else None, width, rows, width, outer, px, width, w, n, None)  # noqa: E731
        assert call(None, 0) == -1 and call(ws.p, nbytes // 32) == -1
        assert torch.equal(b[0].get(), x)
        assert call(ws.p, nbytes) == 0
        got = b[0].get()
        assert torch.equal(got[:, :outer], want) and torch.equal(got[:, outer:], x[:, outer:])


def test_update_interleaved(run):
    """Matrices whose rows lie between each other's, as in rows x parties x cols, also over the operands; rows that overlap are refused."""
    lib = run.lib
    values = (C.c_double * 3)(*cases.QUINTIC)
    for rows, cols in ((5, 40), (40, 5), (900, 16), (20, 30), (70, 66)):
        g, held = cases.update_inputs("f32", 3, rows, cols, True, 0)
        want = run.orthogonal_update(g, held, 0.9, -0.3, [cases.QUINTIC], 1e-7)
        ws, nbytes = run.workspace(lib.haflo_update_workspace_bytes(0, 3, rows, cols))
        between = lambda t: run.buf(t.transpose(0, 1).contiguous())  # noqa: E731
        for over in (None, 0, 1):
            b = [between(g), between(held)]
            out = run.new(rows, 3, cols) if over is None else b[over]
            call = lambda ldo, so: lib.haflo_orthogonal_update(0, b[0].p, 3 * cols, cols, b[1].p, 3 * cols, cols, 3, rows, cols, values, 1, 0.9, -0.3, 1e-7,  # noqa: E731
                                                               out.p, ldo, so, ws.p, nbytes, None)
            if over is None:
                assert call(3 * cols - 1, cols) == -1 and call(3 * cols, cols - 1) == -1 and call(3 * cols, 2 * cols) == -1
            assert call(3 * cols, cols) == 0
            assert torch.equal(out.get().transpose(0, 1), want)


def test_some_gradients(run):
    """Gradients that are not asked for change nothing about the others; what r has from elsewhere may be nothing."""
    lib = run.lib
    for cols in (40, 9000):
        x, f, post, gate, pre, dh, _ = cases.norm_inputs("f32", 3, cols, 0, 0, True, True, "cols", True)
        _, _, rstd = run.residual_norm(x, f, post, gate, pre, 1.0, 1e-5)
        want = run.residual_norm_backward(dh, torch.zeros_like(x), x, f, post, gate, pre, rstd, 1.0)
        b = [run.buf(t) for t in (dh, x, f, post, gate, pre, rstd)]
        ph, px, pf, ppost, pg, ppre, ps = (t.p for t in b)
        ws, nbytes = run.workspace(lib.haflo_residual_norm_workspace_bytes(0, 3, cols))
        for asked in ((1, 0, 0, 0, 0), (0, 1, 0, 0, 0), (0, 0, 1, 0, 0), (0, 0, 0, 1, 0), (0, 0, 0, 0, 1), (0, 0, 0, 0, 0), (1, 1, 1, 1, 1)):
            out = [run.new(*(x.shape if i < 2 else (cols,))) for i in range(5)]
            dx, df, dpost, dgate, dpre = (o.p if a else None for o, a in zip(out, asked))
            assert lib.haflo_residual_norm_backward(0, ph, cols, None, 0, px, cols, pf, cols, ppost, None, 0, pg, ppre, ps, 3, cols, 1.0, dx, cols, df, cols, None, 0,
                                                    dgate, dpost, dpre, ws.p, nbytes, None) == 0
            for o, a, w in zip(out, asked, want):
                assert torch.equal(o.get(), w) if a else bool((o.get() == 9).all())


def test_norm_least_eps_and_greatest_scale(run):
    """Roots' reciprocals and the scale are float32: what leaves them infinite is refused, and with the least eps a row of zeros gives zeros."""
    lib = run.lib
    b = run.buf(torch.zeros(256))
    p, q = b.p, b.p + 512
    for scale, eps, code in ((1.0, 2.0 ** -254, 0), (1.0, 2.0 ** -255, -1), (1.0, 5e-324, -1), (3.4028234663852886e38, 1e-6, 0), (-3.5e38, 1e-6, -1), (1e200, 1e-6, -1)):
        assert lib.haflo_residual_norm(0, p, 8, p, 8, p, None, 8, None, p, 2, 8, scale, eps, q, 8, q + 128, 8, q + 256, None) == code, (scale, eps)
        if eps == 1e-6:
            assert lib.haflo_residual_norm_backward(0, p, 8, None, 8, p, 8, p, 8, p, None, 8, None, p, p, 2, 8, scale, q, 8, None, 8, None, 8, None, None, None,
                                                    q + 128, 256, None) == code, scale
    for cols in (40, 9000):
        zero, ones = torch.zeros(2, cols), torch.ones(cols)
        r, h, rstd = run.residual_norm(zero, zero, ones, ones, ones, 1.0, 2.0 ** -254)
        assert not r.any() and not h.any() and bool((rstd == 2.0 ** 127).all())
        grads = run.residual_norm_backward(torch.full((2, cols), 2.0 ** -100), None, zero, zero, ones, 0.0 * ones, ones, rstd, 1.0)
        assert not any(bool(g.isnan().any()) for g in grads)


def test_nothing_to_do(run):
    """No rows, no matrices: gradients summed over rows are zeros, nothing else is touched."""
    lib = run.lib
    some = run.buf(torch.zeros(64))
    p = some.p
    assert lib.haflo_residual_norm(0, None, 8, None, 0, None, None, 0, None, p, 0, 8, 1.0, 1e-6, None, 0, None, 8, None, None) == 0
    vec = [run.new(70) for _ in range(3)]
    a, b, c = (v.p for v in vec)
    gains = run.buf(torch.ones(70))
    assert lib.haflo_residual_norm_backward(0, None, 70, None, 70, None, 70, p, 70, gains.p, None, 0, gains.p, gains.p, None, 0, 70, 1.0, None, 0, None, 0, None, 0, a, b, c,
                                            None, 0, None) == 0
    assert not any(v.get().any() for v in vec)
    assert lib.haflo_orthogonal_update(0, None, 8, 0, None, 0, 0, 0, 4, 8, (C.c_double * 3)(1, 1, 1), 1, 1.0, 1.0, 1e-7, None, 8, 0, None, 0, None) == 0
    assert lib.haflo_quantize_rows(0, None, 8, 0, 8, None, None, None) == 0
    assert lib.haflo_int8_forward(0, None, 8, None, None, None, None, 0, 0, 8, 4, None, 4, None, 0, None) == 0
    assert lib.haflo_int8_product(0, None, None, None, None, None, None, 0, 0, 8, 4, None, 4, None) == 0


def test_sizes_and_refusals(run):
    """Size queries, and arguments that are refused before any kernel starts."""
    lib, inf, nan = run.lib, float("inf"), float("nan")
    b = run.buf(torch.zeros(4096))
    p, q = b.p, b.p + 4096
    for kind in (0, 1, 2):
        assert lib.haflo_residual_norm_workspace_bytes(kind, 2 ** 31 - 1, 2 ** 31 - 1) < 2 ** 63 and lib.haflo_residual_norm_workspace_bytes(kind, 5, 1) > 0
        assert lib.haflo_update_workspace_bytes(kind, 4096, 128, 2 ** 26) < 2 ** 50 and lib.haflo_update_workspace_bytes(kind, 1, 2 ** 31 - 1, 1) < 2 ** 40
        assert lib.haflo_int8_workspace_bytes(kind, 2 ** 31 - 1, 130944, 2048) < 2 ** 50 and lib.haflo_int8_workspace_bytes(kind, 1, 64, 2 ** 31 - 1) != BAD
    for args in ((3, 1, 1), (0, 2 ** 31, 1), (0, 1, 0), (0, 1, 2 ** 31)):
        assert lib.haflo_residual_norm_workspace_bytes(*args) == BAD
    for args in ((3, 1, 4, 4), (0, 4097, 4, 4), (0, 1, 0, 4), (0, 1, 4, 0), (0, 1, 129, 129), (0, 1, 129, 2 ** 31), (0, 4096, 4, 2 ** 30)):
        assert lib.haflo_update_workspace_bytes(*args) == BAD
    for args in ((3, 1, 4, 4), (0, 2 ** 31, 4, 4), (0, 1, 0, 4), (0, 1, 4, 0), (0, 1, 130945, 4), (0, 1, 4, 2 ** 31), (0, 2 ** 22, 4, 2 ** 21)):
        assert lib.haflo_int8_workspace_bytes(*args) == BAD

    def norm(kind=0, x=p, ldx=8, f=p, ldf=8, post=p, gate=None, ldg=8, cols_gate=None, pre=p, rows=3, cols=8, scale=1.0, eps=1e-6, r=q, ldr=8, h=q + 2048, ldh=8, s=q + 1024):
        return lib.haflo_residual_norm(kind, x, ldx, f, ldf, post, gate, ldg, cols_gate, pre, rows, cols, scale, eps, r, ldr, h, ldh, s, None)

    assert norm() == 0
    for bad in (dict(kind=3), dict(x=None), dict(ldx=7), dict(ldf=7), dict(gate=p, cols_gate=p), dict(gate=p, ldg=7), dict(pre=None, f=None, post=None), dict(f=None),
                dict(f=None, post=None, scale=0.5), dict(f=None, post=None, cols_gate=p), dict(f=None, post=None, gate=p), dict(rows=2 ** 31), dict(cols=0),
                dict(scale=inf), dict(scale=nan), dict(eps=0.0), dict(eps=-1.0), dict(eps=inf), dict(eps=nan), dict(r=None), dict(ldr=7), dict(h=None), dict(ldh=7),
                dict(s=None), dict(r=p, ldr=9), dict(h=p, ldh=9), dict(r=q, h=q)):
        assert norm(**bad) == -1, bad

    def back(kind=0, dh=p, lddh=8, dr=p, lddr=8, x=p, f=p, post=p, gate=None, cols_gate=p, pre=p, s=p, rows=3, cols=8, scale=1.0, dx=q, lddx=8, df=q + 256, lddf=8, dg=None,
             lddg=8, dgc=q + 512, dpost=q + 768, dpre=q + 1024, ws=q + 1280, n=2048):
        return lib.haflo_residual_norm_backward(kind, dh, lddh, dr, lddr, x, 8, f, 8, post, gate, 8, cols_gate, pre, s, rows, cols, scale, dx, lddx, df, lddf, dg, lddg, dgc,
                                                dpost, dpre, ws, n, None)

    assert back() == 0
    for bad in (dict(kind=-1), dict(dh=None), dict(lddh=7), dict(lddr=7), dict(x=None), dict(s=None), dict(f=None), dict(post=None), dict(pre=None), dict(cols_gate=None),
                dict(dg=q), dict(gate=p, dgc=None), dict(lddx=7), dict(lddf=7), dict(scale=inf), dict(dx=p, lddx=9), dict(df=p, lddf=9), dict(dx=q, df=q), dict(ws=None),
                dict(ws=q + 1284), dict(n=16), dict(cols=0), dict(gate=p, cols_gate=None, dgc=None, dg=q + 256)):
        assert back(**bad) == -1, bad

    need = lib.haflo_update_workspace_bytes(0, 2, 20, 30)
    ws = run.buf(torch.zeros(need + 64, dtype=torch.uint8))

    def update(kind=0, g=p, ldg=30, sg=600, base=None, ldb=30, sb=600, parties=1, rows=20, cols=30, c=(1.0, 0.0, 0.0), steps=1, keep=1.0, scale=1.0, eps=1e-7, out=q, ldo=30,
               so=600, w=None, n=need):
        c = None if c is None else (C.c_double * len(c))(*c)
        return lib.haflo_orthogonal_update(kind, g, ldg, sg, base, ldb, sb, parties, rows, cols, c, steps, keep, scale, eps, out, ldo, so, ws.p if w is None else w, n, None)

    assert update() == 0
    for bad in (dict(kind=7), dict(g=None), dict(ldg=29), dict(base=p, ldb=29), dict(out=None), dict(ldo=29), dict(ldo=2 ** 33), dict(parties=2, so=599), dict(parties=4097),
                dict(rows=0), dict(rows=129, cols=129, ldg=129, ldo=129), dict(c=None), dict(steps=0), dict(steps=17, c=(0.0,) * 51), dict(c=(1.0, nan, 0.0)), dict(keep=inf),
                dict(scale=nan), dict(eps=0.0), dict(eps=inf), dict(out=p, ldo=31), dict(base=q, ldb=31, out=q), dict(n=need // 4), dict(w=ws.p + 8)):
        assert update(**bad) == -1, bad

    def quant(kind=0, x=p, ldx=8, rows=3, cols=8, to=q, s=q + 1024):
        return lib.haflo_quantize_rows(kind, x, ldx, rows, cols, to, s, None)

    assert quant() == 0
    for bad in (dict(kind=3), dict(x=None), dict(ldx=7), dict(to=None), dict(to=q + 8), dict(s=None), dict(cols=0), dict(cols=130945, ldx=130945), dict(rows=2 ** 31)):
        assert quant(**bad) == -1, bad

    def product(kind=0, xq=p, xs=p, wq=p, wsc=p, res=None, ldr=4, rows=3, inner=8, outer=4, y=q, ldy=4):
        return lib.haflo_int8_product(kind, xq, xs, wq, wsc, None, res, ldr, rows, inner, outer, y, ldy, None)

    assert product() == 0
    for bad in (dict(kind=3), dict(xq=None), dict(xq=p + 4), dict(xs=None), dict(wq=None), dict(wq=p + 8), dict(wsc=None), dict(res=p, ldr=3), dict(y=None), dict(ldy=3),
                dict(res=q, ldr=5), dict(inner=0), dict(outer=0)):
        assert product(**bad) == -1, bad

    def forward(x=p, ldx=8, rows=17, wq=p, y=q, ldy=4, w=q + 1024, n=4096):
        return lib.haflo_int8_forward(0, x, ldx, wq, p, None, None, 0, rows, 8, 4, y, ldy, w, n, None)

    assert forward() == 0
    for bad in (dict(x=None), dict(ldx=7), dict(wq=p + 8), dict(y=None), dict(ldy=3), dict(w=None), dict(w=q + 1028), dict(n=100)):
        assert forward(**bad) == -1, bad


def test_launches_in_turns(run):
    """The same sources with few lanes to a launch."""
    import build_emu_local
    lib = _cabi.bind(C.CDLL(build_emu_local.build(narrow=True)), prototypes=_cabi.LOCAL_PROTOTYPES)
    lib.hipemu_alloc.restype = C.c_void_p
    lib.hipemu_alloc.argtypes = [C.c_size_t]
    lib.hipemu_free.argtypes = [C.c_void_p]
    narrow = Emulated(lib)
    cases.check_int8(narrow, "bf16", 40, 100, 700, 0, True, True)
    cases.check_int8(narrow, "f32", 1, 130, 900, 0, True, False)
    cases.check_int8(narrow, "f16", 5, 2050, 600, 0, False, False)
    cases.check_quantize(narrow, "f32", 700, 260, 0)
    cases.check_update(narrow, "f32", 150, 2, 800, True, [cases.QUINTIC], 0)
    cases.check_update(narrow, "bf16", 3, 70, 66, True, [cases.QUINTIC] * 2, 0)
    cases.check_norm(narrow, "bf16", 2, 70000, 0, 0, True, True, "cols", True, 1.0)


def test_update_steps_in_place(run):
    """Steps that are taken in parts read G again before any result is written: over G and over the base the results are the same."""
    lib, steps = run.lib, cases.LISTS["8"]
    values = (C.c_double * 24)(*(v for s in steps for v in s))
    for rows, cols in ((6, 50), (50, 6), (16, 900), (20, 90), (90, 20), (70, 75)):
        g, held = cases.update_inputs("f32", 2, rows, cols, True, 0)
        want = run.orthogonal_update(g, held, 0.9, -0.3, steps, 1e-7)
        ws, nbytes = run.workspace(lib.haflo_update_workspace_bytes(0, 2, rows, cols))
        for over in (0, 1):
            b = [run.buf(g), run.buf(held)]
            assert lib.haflo_orthogonal_update(0, b[0].p, cols, rows * cols, b[1].p, cols, rows * cols, 2, rows, cols, values, 8, 0.9, -0.3, 1e-7, b[over].p, cols,
                                               rows * cols, ws.p, nbytes, None) == 0
            assert torch.equal(b[over].get(), want)


@pytest.mark.parametrize("kind", ["f32", "f16", "bf16"])
def test_norm_forms(run, kind):
    for case in cases.norm_forms(kind):
        if case[2] <= 1500 or (kind == "bf16" and case[2] % 4 != 1):
            cases.check_norm(run, *case)


@pytest.mark.parametrize("tall", [False, True])
@pytest.mark.parametrize("kind", ["f32", "f16", "bf16"])
def test_update_forms(run, kind, tall):
    for n, case in enumerate(cases.update_forms(kind, tall)):
        if n % 3 == ("f32", "f16", "bf16").index(kind) and case[1] * case[2] * case[3] < 2 ** 16:  # (each size once over the types, but the largest)
            cases.check_update(run, *case)


@pytest.mark.parametrize("kind", ["f32", "f16", "bf16"])
def test_int8_forms(run, kind):
    for case in cases.int8_forms(kind):
        if case[1] * case[2] * case[3] < 2 ** 23:
            cases.check_int8(run, *case)
