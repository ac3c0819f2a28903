"""CPU-only checks of the local operators' boundary: header, prototypes and library agree; the generator's published values."""
import ctypes as C
import os

import pytest
import torch

import local_cases as cases
from conftest import ROOT
from paper_2107_13797_amd import _cabi
from test_host_logic import declared_symbols


def test_header_prototypes_and_library_agree():
    names = declared_symbols("haflo_local.h")
    assert set(names) == set(_cabi.LOCAL_PROTOTYPES)
    path = os.path.join(ROOT, "paper_2107_13797_amd", "libhaflo.so")
    if not os.path.exists(path):
        from paper_2107_13797_amd import build
        build.build_library(verbose=False)
    lib = _cabi.bind(C.CDLL(path), prototypes=_cabi.LOCAL_PROTOTYPES)
    assert lib.haflo_label_workspace_bytes(9, 1, 1, 0) == 2 ** 64 - 1
    assert lib.haflo_dropout(0, None, 8, None, 0, None, 8, 4, 8, 0.5, 0, 0, None) == -1


def test_generator_known_answers():
    """The values that were published with Philox4x32-10 for counters and keys of zeros and of ones."""
    assert cases.philox(0, 0, 0, 0) == [0x6627E8D5, 0xE169C58D, 0xBC57AC4C, 0x9B00DBD8]
    ones = 0xFFFFFFFF
    assert cases.philox(ones, ones, 2 ** 64 - 1, 2 ** 64 - 1) == [0x408F276D, 0x41C83B0E, 0xA20BC7C6, 0x6D5451FD]


class OnDevice:
    """A host tensor that says it lies on a GPU."""
    is_cuda = True

    def __init__(self, t, device):
        self.t, self.device = t, torch.device("cuda", device)

    def get_device(self):
        return self.device.index

    def new_empty(self, *args, **kwargs):
        return OnDevice(self.t.new_empty(*args, **kwargs), self.device.index)

    def __getattr__(self, name):
        return getattr(self.t, name)


def _calls(api):
    """Each function with its tensors by name, and a call that takes them."""
    f, i = torch.zeros, torch.int32
    adapters = dict(x=f(3, 8), w=f(5, 8), a=f(2, 4, 8), b=f(2, 5, 4), scale=f(2), index=f(3, dtype=i), status=f(1, dtype=i))
    labels = dict(logits=f(3, 8), label=f(3, dtype=i))
    return [
        (dict(x=f(3, 8), residual=f(3, 8), out=f(3, 8)), lambda t: api.haflo_dropout(t.pop("x"), 0.5, 1, **t)),
        (adapters, lambda t: api.haflo_adapter_forward(**t)),
        (dict(adapters, dy=f(3, 5), h=f(3, 4)), lambda t: api.haflo_adapter_backward(**t)),
        (dict(labels, status=f(1, dtype=i)), lambda t: api.haflo_label_logprobs(**t, top=2)),
        (dict(labels, lse=f(3), entropy=f(3), dlogp=f(3), dentropy=f(3), top_index=f(3, 2, dtype=i), dtop=f(3, 2), out=f(3, 8)),
         lambda t: api.haflo_label_logprobs_backward(**t)),
    ]


def test_operands_on_one_device(monkeypatch):
    """Calls go to the current device's stream: an operand of another device is refused, whichever it is, and so is all of them there."""
    from paper_2107_13797_amd import api
    reached = []

    class Library:
        def __getattr__(self, name):
            return lambda *args: reached.append(name) or 0

    monkeypatch.setattr(api, "_lib", Library())
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 0, raising=False)
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda device: None, raising=False)
    for number, (tensors, call) in enumerate(_calls(api)):
        call({n: OnDevice(t, 0) for n, t in tensors.items()})
        assert reached
        del reached[:]
        for odd in list(tensors) + [None]:
            with pytest.raises(api.HafloError, match="device"):
                call({n: OnDevice(t, 1 if odd in (n, None) else 0) for n, t in tensors.items()})
                pytest.fail("call %d took %s of another device" % (number, odd or "all"))
            assert not [n for n in reached if not n.endswith("workspace_bytes")]


def test_status_type(monkeypatch):
    """Four bytes are written to the status: it has to be a 32-bit integer."""
    from paper_2107_13797_amd import api
    monkeypatch.setattr(api, "_lib", type("L", (), {"__getattr__": lambda s, n: lambda *a: 0})())
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 0, raising=False)
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda device: None, raising=False)
    for tensors, call in _calls(api):
        if "status" not in tensors:
            continue
        for bad in (torch.zeros(1, dtype=torch.int8), torch.zeros(0, dtype=torch.int32), torch.zeros(1)):
            with pytest.raises(api.HafloError):
                call({n: OnDevice(t, 0) for n, t in dict(tensors, status=bad).items()})
