"""CPU-only checks of the local operators' boundary: header, prototypes and library agree; the generator's published values."""
import ctypes as C
import os

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
