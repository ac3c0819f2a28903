"""The norms around a block, orthogonalised updates and products of eight bits on the GPU, through the binding, against the definitions
in 64 bits."""
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

import block_cases as cases  # noqa: E402
from test_gpu_local import back, dev  # noqa: E402


class Gpu:
    """The binding's functions on host tensors."""

    def __init__(self, api):
        self.api = api

    def residual_norm(self, x, f, post, gate, pre, scale, eps):
        return back(*self.api.haflo_residual_norm(*map(dev, (x, f, post, gate, pre)), scale, eps))

    def residual_norm_backward(self, dh, dr, x, f, post, gate, pre, rstd, scale):
        return back(*self.api.haflo_residual_norm_backward(*map(dev, (dh, dr, x, f, post, gate, pre, rstd)), scale))

    def orthogonal_update(self, g, base, keep, scale, steps, eps):
        return self.api.haflo_orthogonal_update(dev(g), dev(base), keep, scale, steps, eps).cpu()

    def quantize_rows(self, x):
        return back(*self.api.haflo_quantize_rows(dev(x)))

    def int8_forward(self, x, wq, ws, bias, residual):
        return self.api.haflo_int8_forward(*map(dev, (x, wq, ws, bias, residual))).cpu()

    def int8_product(self, xq, xs, wq, ws, inner, kind, bias, residual):
        return self.api.haflo_int8_product(*map(dev, (xq, xs, wq, ws)), inner, kind, dev(bias), dev(residual)).cpu()


@pytest.fixture(scope="module")
def api():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2107_13797_amd import api
    api.lib()
    return api


@pytest.fixture(scope="module")
def run(api):
    return Gpu(api)


@pytest.mark.parametrize("case", cases.NORMS + cases.NORMS_LARGE, ids=str)
def test_norm(run, case):
    cases.check_norm(run, *case)


def test_norm_special(run):
    cases.check_norm_special(run)


def test_norm_gradients(run):
    cases.check_norm_gradients(run)


@pytest.mark.parametrize("case", cases.UPDATES + cases.UPDATES_LARGE, ids=lambda c: "-".join(map(str, c[:5] + (len(c[5]),))))
def test_update(run, case):
    cases.check_update(run, *case)


def test_update_special(run):
    cases.check_update_special(run)


def test_update_orthogonal(run):
    cases.check_update_orthogonal(run)


@pytest.mark.parametrize("case", [c[:3] + (c[4],) for c in cases.INT8 + cases.INT8_LARGE], ids=str)
def test_quantize(run, case):
    cases.check_quantize(run, *case)


def test_quantize_special(run):
    cases.check_quantize_special(run)


@pytest.mark.parametrize("case", cases.INT8 + cases.INT8_LARGE, ids=str)
def test_int8(run, case):
    cases.check_int8(run, *case)


def test_int8_limits(run):
    cases.check_int8_limits(run)
