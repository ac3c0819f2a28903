"""CPU-only checks of the binding of the norms around a block, of orthogonalised updates and of products of eight bits."""
import pytest
import torch

from test_local_host import OnDevice


def _calls(api):
    """Each function with its tensors by name, and a call that takes them."""
    f, i8 = torch.zeros, torch.int8
    block = dict(x=f(3, 8), f=f(3, 8), post=f(8), gate=f(8), pre=f(8))
    weights = dict(wq=f(5, 128, dtype=i8), w_scale=f(5), bias=f(5), residual=f(3, 5), out=f(3, 5))
    return [
        (dict(block, out=f(3, 8), normed=f(3, 8)), lambda t: api.haflo_residual_norm(**t)),
        (dict(block, dh=f(3, 8), dr=f(3, 8), rstd=f(2, 3)), lambda t: api.haflo_residual_norm_backward(**t)),
        (dict(g=f(2, 4, 8), base=f(2, 4, 8), out=f(2, 4, 8)), lambda t: api.haflo_orthogonal_update(**t)),
        (dict(x=f(3, 8)), lambda t: api.haflo_quantize_rows(**t)),
        (dict(weights, xq=f(3, 128, dtype=i8), x_scale=f(3)), lambda t: api.haflo_int8_product(**t, cols=8)),
        (dict(weights, x=f(3, 8)), lambda t: api.haflo_int8_forward(**t)),
    ]


@pytest.fixture
def api(monkeypatch):
    from paper_2107_13797_amd import api
    reached = []

    class Library:
        def __getattr__(self, name):
            return lambda *args: reached.append((name, args)) or 0

    monkeypatch.setattr(api, "_lib", Library())
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 0, raising=False)
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda device: None, raising=False)
    api_reached = api
    api_reached.reached = reached
    yield api_reached
    del api_reached.reached


def test_operands_on_one_device(api):
    """Calls go to the current device's stream: an operand of another device is refused, whichever it is, and so is all of them there."""
    for number, (tensors, call) in enumerate(_calls(api)):
        call({n: OnDevice(t, 0) for n, t in tensors.items()})
        assert api.reached
        del api.reached[:]
        for odd in list(tensors) + [None]:
            with pytest.raises(api.HafloError, match="device"):
                call({n: OnDevice(t, 1 if odd in (n, None) else 0) for n, t in tensors.items()})
                pytest.fail("call %d took %s of another device" % (number, odd or "all"))
            assert not [n for n, _ in api.reached if not n.endswith("workspace_bytes")]


def test_arguments_reach_their_places(api):
    """What is given and what is not, by position, for calls of many arguments."""
    d = lambda *s, kind=torch.float32: OnDevice(torch.zeros(*s, dtype=kind), 0)  # noqa: E731
    x, f, gate, post, pre, dh, dr, rstd = d(3, 8), d(3, 8), d(3, 8), d(8), d(8), d(3, 8), d(3, 8), d(2, 3)
    at = lambda t: t.data_ptr()  # noqa: E731
    r, h, t = api.haflo_residual_norm(x, f, post, gate, pre, 0.5, 1e-3)
    name, a = api.reached[-1]
    assert name == "haflo_residual_norm" and a[:10] == (0, at(x), 8, at(f), 8, at(post), at(gate), 8, None, at(pre)) and a[10:14] == (3, 8, 0.5, 1e-3)
    assert a[14:19] == (at(r), 8, at(h), 8, at(t)) and t.shape == (2, 3)
    r, h, _ = api.haflo_residual_norm(x, pre=pre)
    assert r is None and api.reached[-1][1][3] is None and api.reached[-1][1][14] is None
    dx, df, dpost, dgate, dpre = api.haflo_residual_norm_backward(dh, dr, x, f, post, gate, pre, rstd, 0.5)
    a = api.reached[-1][1]
    assert a[1:5] == (at(dh), 8, at(dr), 8) and a[14] == at(rstd) and a[15:18] == (3, 8, 0.5) and a[18] == at(dx) and a[20] == at(df)
    assert a[22] == at(dgate) and a[24:27] == (None, at(dpost), at(dpre)) and dgate.shape == (3, 8)
    _, _, _, dgate, _ = api.haflo_residual_norm_backward(dh, None, x, f, post, pre, pre, rstd, 0.5, need_dx=False)
    a = api.reached[-1][1]
    assert a[3] is None and a[18] is None and a[22] is None and a[24] == at(dgate) and dgate.shape == (8,)


def test_distances(api):
    """Slices keep their distances between rows and between matrices."""
    wide = torch.zeros(3, 6, 20)
    g = OnDevice(wide[:, 1:5, 2:10], 0)
    out = api.haflo_orthogonal_update(g)
    a = api.reached[-1][1]
    assert a[1:4] == (g.data_ptr(), 20, 120) and a[4] is None and a[7:10] == (3, 4, 8) and list(a[10]) == [v for c in api.NEWTON_SCHULZ for v in c] and a[11] == 5
    assert a[15:18] == (out.data_ptr(), 8, 32)
    x = OnDevice(torch.zeros(4, 30)[:, 3:11], 0)
    q, s = api.haflo_quantize_rows(x)
    assert api.reached[-1][1][1:5] == (x.data_ptr(), 30, 4, 8) and q.shape == (4, 128) and s.shape == (4,)


def test_int8_workspace_over_its_rows(api):
    """Where the result lies over x, the binding asks for the workspace of 17 rows or more."""
    q, s = (OnDevice(torch.zeros(*n, dtype=t), 0) for n, t in (((8, 128), torch.int8), ((8,), torch.float32)))
    for rows, over, want in ((3, False, 3), (3, True, 17), (40, True, 40), (40, False, 40)):
        x = OnDevice(torch.zeros(rows, 8), 0)
        api.haflo_int8_forward(x, q, s, out=x if over else OnDevice(torch.zeros(rows, 8), 0))
        name, args = api.reached[-2]
        assert name == "haflo_int8_workspace_bytes" and args == (0, want, 8, 8)
