"""The kernels of a party's local operators, compiled for the CPU against a stand-in for the HIP runtime (tests/emu), through the
same C entry points, against the definitions in 64 bits. Buffers end at a guard page, so that an access past an end faults."""
import ctypes as C
import os
import sys

import pytest
import torch

import local_cases as cases
from paper_2107_13797_amd import _cabi

pytestmark = pytest.mark.skipif(not os.path.exists("/opt/rocm/llvm/bin/clang++"), reason="no clang for the half types")
NAMES = {torch.float32: _cabi.TYPE_F32, torch.float16: _cabi.TYPE_F16, torch.bfloat16: _cabi.TYPE_BF16}


class Buffer:
    """A guarded copy of a host tensor with its strides, or of fresh memory."""

    def __init__(self, lib, t):
        self.lib, self.t = lib, t
        last = sum((n - 1) * s for n, s in zip(t.shape, t.stride())) + 1 if t.numel() else 0
        self.flat = torch.as_strided(t, (last,), (1,), t.storage_offset()).contiguous()
        # a slice keeps its distance from a 16-byte boundary
        self.skip = t.storage_offset() * t.element_size() % 16
        self.n = last * t.element_size()
        self.base = lib.hipemu_alloc(self.skip + max(self.n, 1))
        self.p = self.base + self.skip
        C.memmove(self.p, self.flat.data_ptr(), self.n)

    def get(self):
        out = torch.empty_like(self.flat)
        C.memmove(out.data_ptr(), self.p, self.n)
        return torch.as_strided(out, self.t.shape, self.t.stride()).clone()

    def __del__(self):
        self.lib.hipemu_free(self.base)


class Emulated:
    """The binding's functions on host tensors."""

    def __init__(self, lib):
        self.lib = lib

    def buf(self, t):
        return Buffer(self.lib, t)

    def ld(self, t):
        return t.stride(0) if t.shape[0] > 1 else t.shape[1]

    def workspace(self, nbytes):
        assert nbytes != 2 ** 64 - 1
        return self.buf(torch.full((nbytes,), 0xA5, dtype=torch.uint8)), nbytes

    def dropout(self, x, p, seed, offset, residual=None):
        y = self.buf(torch.full_like(x, 9.0))
        bx, br = self.buf(x), self.buf(residual) if residual is not None else None
        assert self.lib.haflo_dropout(NAMES[x.dtype], bx.p, self.ld(x), br.p if br else None, self.ld(residual) if br else 0, y.p,
                                      self.ld(y.t), *x.shape, p, seed, offset, None) == 0
        return y.get()

    def adapter_forward(self, x, w, a, b, scale, index, p, seed, offset):
        rows, inner, outer, parties, rank = *x.shape, w.shape[0], a.shape[0], a.shape[1]
        ws, nbytes = self.workspace(self.lib.haflo_adapter_workspace_bytes(NAMES[x.dtype], 0, rows, inner, outer, parties, rank))
        bufs = [self.buf(t) for t in (x, w, a, b, scale, index)]
        y, h, st = self.buf(torch.full((rows, outer), 9.0, dtype=x.dtype)), self.buf(torch.full((rows, rank), 9.0)), self.buf(torch.zeros(1, dtype=torch.int32))
        x_, w_, a_, b_, s_, i_ = (t.p for t in bufs)
        assert self.lib.haflo_adapter_forward(NAMES[x.dtype], x_, self.ld(x), w_, self.ld(w), a_, b_, s_, i_, rows, inner, outer, parties, rank,
                                              p, seed, offset, y.p, outer, h.p, st.p, ws.p, nbytes, None) == 0
        return y.get(), h.get(), int(st.get()[0])

    def adapter_backward(self, dy, x, w, a, b, scale, index, h, p, seed, offset):
        rows, inner, outer, parties, rank = *x.shape, w.shape[0], a.shape[0], a.shape[1]
        ws, nbytes = self.workspace(self.lib.haflo_adapter_workspace_bytes(NAMES[x.dtype], 1, rows, inner, outer, parties, rank))
        bufs = [self.buf(t) for t in (dy, x, w, a, b, scale, index, h)]
        d_, x_, w_, a_, b_, s_, i_, h_ = (t.p for t in bufs)
        dx, da, db = self.buf(torch.full((rows, inner), 9.0, dtype=x.dtype)), self.buf(torch.full(a.shape, 9.0)), self.buf(torch.full(b.shape, 9.0))
        st = self.buf(torch.zeros(1, dtype=torch.int32))
        assert self.lib.haflo_adapter_backward(NAMES[x.dtype], d_, self.ld(dy), x_, self.ld(x), w_, self.ld(w), a_, b_, s_, i_, h_, rows, inner,
                                               outer, parties, rank, p, seed, offset, dx.p, inner, da.p, db.p, st.p, ws.p, nbytes, None) == 0
        return dx.get(), da.get(), db.get(), int(st.get()[0])

    def label_logprobs(self, x, label, top):
        rows, cols = x.shape
        ws, nbytes = self.workspace(self.lib.haflo_label_workspace_bytes(NAMES[x.dtype], rows, cols, top))
        bx, bl, st = self.buf(x), self.buf(label), self.buf(torch.zeros(1, dtype=torch.int32))
        logp, entropy, lse = (self.buf(torch.full((rows,), 9.0)) for _ in range(3))
        tl, ti = self.buf(torch.full((rows, top), 9.0)), self.buf(torch.full((rows, top), -9, dtype=torch.int32))
        assert self.lib.haflo_label_logprobs(NAMES[x.dtype], bx.p, self.ld(x), bl.p, rows, cols, top, logp.p, entropy.p, lse.p, tl.p, ti.p,
                                             st.p, ws.p, nbytes, None) == 0
        return logp.get(), entropy.get(), lse.get(), tl.get(), ti.get(), int(st.get()[0])

    def label_logprobs_backward(self, x, label, lse, entropy, dlogp, dentropy, top_index, dtop):
        rows, cols = x.shape
        bufs = [self.buf(t) if t is not None else None for t in (x, label, lse, entropy, dlogp, dentropy, top_index, dtop)]
        x_, l_, s_, e_, d_, h_, i_, t_ = (t.p if t else None for t in bufs)
        top, dx = 0 if dtop is None else dtop.shape[1], self.buf(torch.full((rows, cols), 9.0, dtype=x.dtype))
        assert self.lib.haflo_label_logprobs_backward(NAMES[x.dtype], x_, self.ld(x), l_, s_, e_, d_, h_, i_, t_, rows, cols, top, dx.p, cols,
                                                      None) == 0
        return dx.get()


@pytest.fixture(scope="module")
def run():
    sys.path.insert(0, os.path.join(os.path.dirname(__file__), "emu"))
    import build_emu_local
    lib = _cabi.bind(C.CDLL(build_emu_local.build()), prototypes=_cabi.LOCAL_PROTOTYPES)
    lib.hipemu_alloc.restype = C.c_void_p
    lib.hipemu_alloc.argtypes = [C.c_size_t]
    lib.hipemu_free.argtypes = [C.c_void_p]
    return Emulated(lib)


@pytest.mark.parametrize("case", cases.DROPOUT, ids=str)
def test_dropout(run, case):
    cases.check_dropout(run, *case)


def test_dropout_special(run):
    cases.check_dropout_special(run)


@pytest.mark.parametrize("case", cases.ADAPTERS, ids=str)
def test_adapters(run, case):
    cases.check_adapters(run, *case)


def test_adapters_other_parties_infinities(run):
    cases.check_adapters_other_parties_infinities(run)


@pytest.mark.parametrize("case", cases.LABELS, ids=str)
def test_labels(run, case):
    cases.check_labels(run, *case)


def test_labels_nan(run):
    cases.check_labels_nan(run)


def test_sizes_and_refusals(run):
    """Size queries and calls without work or with arguments that are refused, none of which starts a kernel that reads."""
    lib, bad = run.lib, 2 ** 64 - 1
    for kind in (0, 1, 2):
        for rows in (0, 1, 2 ** 31 - 1):
            assert lib.haflo_label_workspace_bytes(kind, rows, 50000, 20) != bad
            assert lib.haflo_adapter_workspace_bytes(kind, 0, rows, 64, 64, 8, 16) != bad and lib.haflo_adapter_workspace_bytes(kind, 1, rows, 64, 64, 8, 16) != bad
    for args in ((3, 1, 8, 8, 1, 1), (0, 2 ** 31, 8, 8, 1, 1), (0, 1, 0, 8, 1, 1), (0, 1, 8, 0, 1, 1), (0, 1, 8, 8, 0, 1), (0, 1, 8, 8, 4097, 1), (0, 1, 8, 8, 1, 0),
                 (0, 1, 8, 8, 1, 129)):
        assert lib.haflo_adapter_workspace_bytes(args[0], 1, *args[1:]) == bad
    for args in ((3, 1, 8, 1), (0, 2 ** 31, 8, 1), (0, 1, 0, 0), (0, 1, 8, 9), (0, 1, 100, 65)):
        assert lib.haflo_label_workspace_bytes(*args) == bad
    some = run.buf(torch.zeros(64))
    p = some.p
    drop = lambda *a: lib.haflo_dropout(*a, None)  # noqa: E731
    assert drop(0, None, 8, None, 0, None, 8, 0, 8, 0.5, 1, 0) == 0
    assert drop(0, p, 7, None, 0, p, 8, 2, 8, 0.5, 1, 0) == -1 and drop(0, p, 8, None, 0, p, 7, 2, 8, 0.5, 1, 0) == -1
    assert drop(0, p, 8, p, 7, p, 8, 2, 8, 0.5, 1, 0) == -1 and drop(0, p, 8, None, 0, None, 8, 2, 8, 0.5, 1, 0) == -1
    assert drop(0, p, 8, None, 0, p, 8, 2, 8, 1.01, 1, 0) == -1 and drop(0, p, 8, None, 0, p, 8, 2, 8, float("nan"), 1, 0) == -1
    assert drop(4, p, 8, None, 0, p, 8, 2, 8, 0.5, 1, 0) == -1
    fwd = lambda rows, ldx=4, ws=p, n=256, index=p: lib.haflo_adapter_forward(0, p, ldx, p, 4, p, p, p, index, rows, 4, 4, 1, 1, 0.0, 0, 0, p, 4, p, None, ws, n, None)  # noqa: E731
    assert fwd(0, index=None) == 0 and fwd(2, ldx=3) == -1 and fwd(2, index=None) == -1
    assert lib.haflo_adapter_backward(0, p, 4, p, 4, p, 4, p, p, p, p, p, 2, 4, 4, 1, 1, 0.0, 0, 0, p, 4, p, p, None, p, 255, None) == -1
    assert lib.haflo_label_logprobs(0, p, 4, p, 0, 4, 0, None, None, None, None, None, None, None, 0, None) == 0
    assert lib.haflo_label_logprobs(0, p, 4, p, 1, 4, 1, p, p, p, None, None, None, None, 0, None) == -1
    assert lib.haflo_label_logprobs(0, p, 9000, p, 1, 9000, 0, p, p, p, None, None, None, None, 0, None) == -1  # needs a workspace
    assert lib.haflo_label_logprobs_backward(0, p, 4, p, p, p, p, None, None, p, 1, 4, 1, p, 4, None) == -1  # dtop without its columns


def test_no_rows(run):
    """A party without rows has zero gradients."""
    x, w, a, b, scale, index, dy = cases.adapter_inputs("f32", 4, 8, 6, 3, 2, "mixed", 0)
    none = slice(0, 0)
    _, da, db, status = run.adapter_backward(dy[none], x[none], w, a, b, scale, index[none], torch.zeros(0, 3), 0.0, 0, 0)
    assert not da.any() and not db.any() and status == 0


@pytest.mark.parametrize("case", cases.ADAPTERS_SHORT_SUMS, ids=str)
def test_adapters_short_sums(run, case):
    cases.check_adapters(run, *case)


@pytest.mark.parametrize("rows", [200, 300])
@pytest.mark.parametrize("kind", cases.TYPES)
def test_adapters_cancelling(run, kind, rows):
    cases.check_adapters_cancelling(run, kind, rows)


@pytest.mark.parametrize("kind", cases.TYPES)
def test_adapters_own_infinities(run, kind):
    cases.check_adapters_own_infinities(run, kind)


@pytest.mark.parametrize("case", cases.LABELS_FAR, ids=str)
def test_labels_far(run, case):
    cases.check_labels_far(run, *case)


def test_labels_far_columns(run):
    cases.check_labels_far_columns(run)


def test_in_place_refusals(run):
    """A result over an input whose rows lie at another distance would be written where other rows are still read."""
    lib, one, two = run.lib, run.buf(torch.zeros(64)), run.buf(torch.zeros(64))
    p, other = one.p, two.p
    drop = lambda x, ldx, r, ldr, y, ldy, rows: lib.haflo_dropout(0, x, ldx, r, ldr, y, ldy, rows, 8, 0.5, 1, 0, None)  # noqa: E731
    assert drop(p, 8, None, 0, p, 9, 3) == -1 and drop(p, 16, None, 0, p, 8, 3) == -1 and drop(other, 8, p, 12, p, 8, 3) == -1
    assert drop(p, 9, None, 0, p, 9, 3) == 0 and drop(other, 8, p, 9, p, 9, 3) == 0 and drop(p, 8, p, 8, p, 8, 3) == 0
    assert drop(p, 9, None, 0, p, 8, 1) == 0 and drop(p, 8, None, 0, other, 9, 3) == 0
    row = run.buf(torch.zeros(8))
    grad = lambda x, ld, dx, lddx, rows: lib.haflo_label_logprobs_backward(0, x, ld, row.p, row.p, row.p, row.p, None, None, None, rows, 8, 0, dx, lddx, None)  # noqa: E731
    assert grad(p, 8, p, 9, 3) == -1 and grad(p, 9, p, 8, 3) == -1
    assert grad(p, 9, p, 9, 3) == 0 and grad(p, 8, p, 9, 1) == 0


def test_workspace_alignment(run):
    """A workspace off a 16-byte boundary is refused, whatever it has room for."""
    lib = run.lib
    need = [lib.haflo_adapter_workspace_bytes(0, b, 300, 8, 8, 1, 4) for b in (0, 1)] + [lib.haflo_label_workspace_bytes(0, 1, 9000, 4)]
    some, ws = run.buf(torch.zeros(300 * 8)), run.buf(torch.zeros(max(need) + 16, dtype=torch.uint8))
    index, p = run.buf(torch.zeros(300, dtype=torch.int32)), some.p
    out = [run.buf(torch.zeros(300 * 8)) for _ in range(4)]
    for off in (0, 4, 8):
        args = (ws.p + off, need[0], None)
        got = [lib.haflo_adapter_forward(0, p, 8, p, 8, p, p, p, index.p, 300, 8, 8, 1, 4, 0.0, 0, 0, out[0].p, 8, out[1].p, None, *args)]
        args = (ws.p + off, need[1], None)
        got += [lib.haflo_adapter_backward(0, p, 8, p, 8, p, 8, p, p, p, index.p, p, 300, 8, 8, 1, 4, 0.0, 0, 0, out[0].p, 8, out[1].p, out[2].p, None, *args)]
        args = (ws.p + off, need[2], None)
        wide = run.buf(torch.zeros(9000))
        got += [lib.haflo_label_logprobs(0, wide.p, 9000, index.p, 1, 9000, 4, out[0].p, out[1].p, out[2].p, out[3].p, index.p, None, *args)]
        assert got == ([0, 0, 0] if off == 0 else [-1, -1, -1])


@pytest.fixture(scope="module")
def narrow():
    """The same sources with few lanes to a launch, so that ordinary sizes take several where the card's limit would be passed."""
    import build_emu_local
    lib = _cabi.bind(C.CDLL(build_emu_local.build(narrow=True)), prototypes=_cabi.LOCAL_PROTOTYPES)
    lib.hipemu_alloc.restype = C.c_void_p
    lib.hipemu_alloc.argtypes = [C.c_size_t]
    lib.hipemu_free.argtypes = [C.c_void_p]
    return Emulated(lib)


def test_launches_in_turns(run, narrow):
    cases.check_adapters(narrow, "f32", 2500, 7, 70, 2, 100, 0.1, "mixed", 1)
    cases.check_adapters(narrow, "bf16", 40, 16, 2100, 4, 2, 0.1, "mixed", 0)
    cases.check_labels(narrow, "bf16", 300, 40, 0, 0, 2, "inf")
    cases.check_labels(narrow, "f32", 200, 2100, 0, 0, 0, "inf")
    cases.check_labels(narrow, "f16", 100, 5130, 0, 0, 0, "")
    cases.check_dropout(narrow, "f16", 100, 2200, 0, 0, 0.5, True)


@pytest.mark.parametrize("case", cases.ADAPTERS_MANY, ids=str)
def test_adapters_many(run, case):
    cases.check_adapters_of_many(run, *case)


@pytest.mark.parametrize("rows", [40, 300])
@pytest.mark.parametrize("kind", cases.TYPES)
def test_adapters_isolation(run, kind, rows):
    cases.check_adapters_isolation(run, kind, rows)


def test_factor_of_many():
    cases.check_factor_of_many()


class Forms:
    """Which kernels calls of given sizes launch: entry points with addresses that nothing reads, as no kernel runs."""

    def __init__(self, lib):
        self.lib = lib
        lib.hipemu_launches.restype = C.c_char_p
        lib.hipemu_dry.argtypes = [C.c_int]

    def of(self, call):
        self.lib.hipemu_launches()
        self.lib.hipemu_dry(1)
        try:
            assert call() == 0
        finally:
            self.lib.hipemu_dry(0)
        return [n.strip("()") for n in self.lib.hipemu_launches().decode().split("\n") if n]

    def adapters(self, kind, rows, inner, outer, rank, parties, p, order, pad):
        t, a, big = NAMES[cases.TYPES[kind]], 2 ** 20, 2 ** 62
        fwd = lambda: self.lib.haflo_adapter_forward(t, a, inner + pad, a, inner + pad, a, a, a, a, rows, inner, outer, parties, rank, p, 0, 0, a, outer, a, None, a, big, None)  # noqa: E731
        bwd = lambda: self.lib.haflo_adapter_backward(t, a, outer + pad, a, inner + pad, a, inner + pad, a, a, a, a, a, rows, inner, outer, parties, rank, p, 0, 0, a, inner, a, a, None, a, big, None)  # noqa: E731
        return {(kind,) + (n,) for n in self.of(fwd) + self.of(bwd)}

    def labels(self, kind, rows, cols, top, backward):
        t, a = NAMES[cases.TYPES[kind]], 2 ** 20
        if backward:
            call = lambda: self.lib.haflo_label_logprobs_backward(t, a, cols, a, a, a, a, a, a if top else None, a if top else None, rows, cols, top, a, cols, None)  # noqa: E731
        else:
            call = lambda: self.lib.haflo_label_logprobs(t, a, cols, a, rows, cols, top, a, a, a, a, a, None, a, 2 ** 62, None)  # noqa: E731
        return {(kind, n) for n in self.of(call)}


def test_every_form_is_tested(run):
    """Each kernel form that some size selects is selected by a case that the GPU runs against the definition."""
    import test_gpu_local as gpu
    forms, listed = Forms(run.lib), lambda test: test.pytestmark[0].args[1]
    every, tested = set(), set()
    for kind in cases.TYPES:
        for rank in (1, 16, 17, 32, 33, 64, 65, 128):
            for p in (0.0, 0.1):
                for rows, inner, outer in ((1, 8, 8), (20, 8, 8), (40, 8, 8), (300, 8, 8), (300, 600, 600), (300, 513, 8), (2100, 2100, 2100), (8192, 4096, 4096), (70000, 32768, 32768)):
                    every |= forms.adapters(kind, rows, inner, outer, rank, 3, p, "", 0)
        for cols in (2, 33, 700, 1100, 2049, 3000, 6000, 9000, 17000, 30000, 50000):
            for rows in (1, 40, 2000, 9000):
                for top in (0, 2):
                    every |= forms.labels(kind, rows, cols, top, False) | forms.labels(kind, rows, cols, top, True)
    for case in cases.ADAPTERS + cases.ADAPTERS_LARGE + cases.ADAPTERS_SHORT_SUMS + cases.ADAPTERS_MANY + cases.ADAPTERS_TILES + cases.ADAPTERS_FORMS + listed(gpu.test_adapters_some_rows):
        tested |= forms.adapters(*case)
    for kind, rows in gpu.FAR_FORWARD:
        tested |= forms.adapters(kind, rows, 32768, 16, 2, 2, 0.0, "", 0)
    for kind, rows in gpu.FAR_GRADIENT:
        tested |= forms.adapters(kind, rows, 16, 32768, 2, 2, 0.5, "", 0)
    for kind, rows, cols, _, _, top, *_ in cases.LABELS + cases.LABELS_LARGE + cases.LABELS_FAR + cases.LABELS_FORMS + listed(gpu.test_labels_many_rows):
        tested |= forms.labels(kind, rows, cols, top, False) | forms.labels(kind, rows, cols, top, True) | forms.labels(kind, rows, cols, 0, True)
    assert not every - tested, sorted(every - tested)
    tiles = {(k, n) for k, n in every if n.startswith("k_project")}
    assert len(tiles) == 2 * 8 + 4, sorted(tiles)


@pytest.mark.parametrize("case", cases.ADAPTERS_FORMS, ids=str)
def test_adapters_forms(run, case):
    cases.check_adapters_of_many(run, *case)


@pytest.mark.parametrize("case", cases.LABELS_FORMS, ids=str)
def test_labels_forms(run, case):
    cases.check_labels_far(run, *case)


def test_sizes_past_64_bits(run):
    """Counts that each are in range, whose products a workspace's size does not hold, are refused rather than wrapped around."""
    size, most = run.lib.haflo_adapter_workspace_bytes, 2 ** 31 - 600
    for kind in (0, 1, 2):
        for backward in (0, 1):
            for rows, inner, outer in ((most, most, 64), (most, 64, most), (64, most, most), (2 ** 30, 2 ** 28, 2 ** 28)):
                assert size(kind, backward, rows, inner, outer, 4096, 128) == 2 ** 64 - 1
            for rows, inner, outer in ((most, 64, 64), (64, most, 64), (64, 64, most), (2 ** 20, 2 ** 20, 2 ** 20)):
                need = size(kind, backward, rows, inner, outer, 4096, 128)
                assert (2 * rows * inner if rows > 256 else 2 * outer * inner) <= need < 2 ** 63
