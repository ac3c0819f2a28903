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


def test_norm_gradients(run):
    cases.check_norm_gradients(run)


@pytest.mark.parametrize("case", cases.UPDATES, ids=lambda c: "-".join(map(str, c[:5] + (len(c[5]),))))
def test_update(run, case):
    cases.check_update(run, *case)


def test_update_special(run):
    cases.check_update_special(run)


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


def test_int8_limits(run):
    cases.check_int8_limits(run)
