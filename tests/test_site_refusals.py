"""Arguments that the calls of the site norm, the residual tail and the 8-bit checkpoints refuse: each returns its
error before anything is launched, so these run without a GPU, with addresses that nothing reads."""
import ctypes
import os

import pytest

from paper_2111_07383_amd import _abi
from paper_2111_07383_amd import binding as B

pytestmark = pytest.mark.skipif(not os.path.exists(_abi.LIB_PATH), reason="libssconv.so not built")

P = ctypes.c_void_p(4096)   # an address for buffers that a refused call never touches
N = None
F = ((0, 3), (1, 2))


def fields(f):
    return ctypes.byref(B.make_fields(f))


def rows(data=4096, exps=None):
    return ctypes.byref(_abi.Rows(data, exps))


def refused(rc, code=_abi.E_INVALID):
    assert rc == code
    assert _abi.lib().ssconv_last_error()


def bad_lists():
    yield ((0, 0),)
    yield ((5, 1),)
    yield ((-1, 1),)
    yield ((0, 1025),)
    yield ((4, 113), (0, 8))      # 1025 channels


@pytest.mark.parametrize("f", bad_lists())
def test_field_lists(f):
    L = _abi.lib()
    assert L.ssconv_packed_blocks(fields(f)) == 0
    assert L.ssconv_site_norm_workspace_size(fields(f), 5) == 0
    assert L.ssconv_residual_workspace_size(fields(f), 5) == 0
    refused(L.ssconv_pack(fields(f), P, 0, 1, P, P, N))
    refused(L.ssconv_unpack(fields(f), P, P, 1, 0, P, N))
    refused(L.ssconv_site_norm_forward(fields(f), rows(), 0, 1, 1e-5, N, P, N, N, N))
    refused(L.ssconv_site_norm_backward(fields(f), rows(), P, N, 0, 1, 1e-5, N, P, N, N, 0, N))
    refused(L.ssconv_residual_forward(fields(f), P, P, 0, 1, 1e-5, N, N, N, P, P, N, N, N, N, N))
    refused(L.ssconv_residual_backward(fields(f), rows(), rows(), P, P, 0, 1, 1e-5, N, N, N, P, P, N, N, N, N, 0, N))
    with pytest.raises(ValueError):
        B.packed_blocks(f)


def test_gates_need_room():
    L = _abi.lib()
    eight = ((1, 1),) * 8                       # no entry left for the gates
    refused(L.ssconv_residual_forward(fields(eight), P, P, 0, 1, 1e-5, N, N, N, P, P, N, N, N, N, N))
    wide = ((1, 300),)                          # 900 channels and 300 gates
    refused(L.ssconv_residual_forward(fields(wide), P, P, 0, 1, 1e-5, N, N, N, P, P, N, N, N, N, N))
    assert L.ssconv_residual_workspace_size(fields(wide), 5) == 0
    assert L.ssconv_packed_blocks(fields(wide)) == 29
    assert L.ssconv_packed_blocks(fields(((0, 33), (1, 11), (0, 2)))) == 2 + 2 + 1
    with pytest.raises(ValueError):
        B.gate_fields(((0, 1),) * 9)


def test_types_sizes_and_eps():
    L = _abi.lib()
    refused(L.ssconv_pack(fields(F), P, 2, 1, P, P, N), _abi.E_DTYPE)
    refused(L.ssconv_unpack(fields(F), P, P, 1, -1, P, N), _abi.E_DTYPE)
    refused(L.ssconv_site_norm_forward(fields(F), rows(), 7, 1, 1e-5, N, P, N, N, N), _abi.E_DTYPE)
    refused(L.ssconv_site_norm_backward(fields(F), rows(), P, N, 7, 1, 1e-5, N, P, N, N, 0, N), _abi.E_DTYPE)
    refused(L.ssconv_residual_forward(fields(F), P, P, 2, 1, 1e-5, N, N, N, P, P, N, N, N, N, N), _abi.E_DTYPE)
    refused(L.ssconv_pack(fields(F), P, 0, -1, P, P, N))
    refused(L.ssconv_site_norm_forward(fields(F), rows(), 0, -1, 1e-5, N, P, N, N, N))
    for eps in (0.0, -1.0, float("nan"), float("inf"), 1e-60):   # 1e-60 is 0 in fp32
        refused(L.ssconv_site_norm_forward(fields(F), rows(), 0, 1, eps, N, P, N, N, N))
        refused(L.ssconv_site_norm_backward(fields(F), rows(), P, N, 0, 1, eps, N, P, N, N, 0, N))
        refused(L.ssconv_residual_forward(fields(F), P, P, 0, 1, eps, N, N, N, P, P, N, N, N, N, N))
        refused(L.ssconv_residual_backward(fields(F), rows(), rows(), P, P, 0, 1, eps, N, N, N, P, P, N, N, N, N, 0, N))


def test_missing_buffers():
    L = _abi.lib()
    refused(L.ssconv_pack(fields(F), N, 0, 1, P, P, N))
    refused(L.ssconv_pack(fields(F), P, 0, 1, N, P, N))
    refused(L.ssconv_pack(fields(F), P, 0, 1, P, N, N))
    refused(L.ssconv_unpack(fields(F), P, N, 1, 0, P, N))
    refused(L.ssconv_site_norm_forward(fields(F), rows(0), 0, 1, 1e-5, N, P, N, N, N))
    refused(L.ssconv_site_norm_forward(fields(F), N, 0, 1, 1e-5, N, P, N, N, N))
    refused(L.ssconv_site_norm_forward(fields(F), rows(), 0, 1, 1e-5, N, N, N, N, N))
    refused(L.ssconv_site_norm_forward(fields(F), rows(), 0, 1, 1e-5, N, P, P, N, N))          # half a checkpoint
    refused(L.ssconv_site_norm_forward(fields(F), rows(4096, 4096), 0, 1, 1e-5, N, P, P, P, N))  # of a checkpoint
    refused(L.ssconv_site_norm_backward(fields(F), rows(), N, N, 0, 1, 1e-5, N, P, N, N, 0, N))
    refused(L.ssconv_residual_forward(fields(F), P, N, 0, 1, 1e-5, N, N, N, P, P, N, N, N, N, N))
    refused(L.ssconv_residual_forward(fields(F), P, P, 0, 1, 1e-5, N, N, N, P, P, P, N, N, N, N))
    refused(L.ssconv_residual_forward(fields(F), P, P, 0, 1, 1e-5, N, N, P, P, N, N, N, N, N, N))   # gain_next alone
    for y, h in ((rows(4096, 4096), rows()), (rows(), rows(4096, 4096))):                       # one a checkpoint
        refused(L.ssconv_residual_backward(fields(F), y, h, P, P, 0, 1, 1e-5, N, N, N, P, P, N, N, N, N, 0, N))
    refused(L.ssconv_residual_backward(fields(F), rows(), N, P, P, 0, 1, 1e-5, N, N, N, P, P, N, N, N, N, 0, N))
    refused(L.ssconv_residual_backward(fields(F), rows(), rows(), P, N, 0, 1, 1e-5, N, N, P, P, P, N, N, N, N, 0, N))
    refused(L.ssconv_residual_backward(fields(F), rows(), rows(), P, N, 0, 1, 1e-5, N, N, N, P, P, N, N, P, P, 1 << 30, N))


def test_workspaces():
    L = _abi.lib()
    need = L.ssconv_site_norm_workspace_size(fields(F), 100)
    assert need > 0
    for ws, size in ((N, need), (P, need - 1), (ctypes.c_void_p(4096 + 128), need)):
        refused(L.ssconv_site_norm_backward(fields(F), rows(), P, N, 0, 100, 1e-5, N, P, P, ws, size, N))
    need = L.ssconv_residual_workspace_size(fields(F), 100)
    for out in ((P, N, N), (N, P, N), (N, N, P)):
        refused(L.ssconv_residual_backward(fields(F), rows(), rows(), P, P, 0, 100, 1e-5, N, N, N, P, P, *out, P,
                                           need - 1, N))


def test_empty_calls_do_nothing():
    L = _abi.lib()
    assert L.ssconv_pack(fields(F), N, 0, 0, N, N, N) == 0
    assert L.ssconv_unpack(fields(F), N, N, 0, 1, N, N) == 0
    assert L.ssconv_site_norm_forward(fields(F), rows(0), 0, 0, 1e-5, N, N, N, N, N) == 0
    assert L.ssconv_residual_forward(fields(F), N, N, 1, 0, 1e-5, N, N, N, N, N, N, N, N, N, N) == 0


def test_backward_packed():
    L = _abi.lib()
    refused(L.ssconv_backward_packed(fields(((0, 0),)), P, P, 0, 1e-5, N, P, 0, 4, N, P, N, N, P, N, P, 0, N))
    refused(L.ssconv_backward_packed(fields(F), P, P, 0, 1e-5, N, P, 0, 4, N, P, N, N, P, N, P, 0, N))   # no rule book
    refused(L.ssconv_backward_packed(fields(F), P, P, 1, 0.0, N, P, 0, 4, N, P, N, N, P, N, P, 0, N))    # eps
    refused(L.ssconv_backward_packed(fields(F), P, P, 0, 1e-5, P, P, 0, 4, N, P, N, N, P, N, P, 0, N))   # gain alone
    assert L.ssconv_backward_packed_workspace_size(N, 0, 4, 4) == 0
