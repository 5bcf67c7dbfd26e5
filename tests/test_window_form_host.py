"""CPU tests of how calls of attention in a window say that they are run: what is refused, and that pieces and workspaces agree."""
import ctypes as C

import pytest

import paper_2603_05503_amd as pkg
from paper_2603_05503_amd.layer_ops import _CWindow, _CWindowForm


def form(*sizes, window=(4, 0, 0, 1, 0)):
    w, f = _CWindow(*window), _CWindowForm()
    return pkg.load_library().calibatt_window_attn_form(*sizes, C.addressof(w), C.addressof(f)), f


def test_form_refusals():
    for sizes, status in (((0, 1, 1, 1, 1, 64), -2), ((1, 3, 2, 1, 1, 64), -2), ((1, 1, 1, 1, 1, 96), -3)):
        assert form(*sizes)[0] == status
    assert form(1, 1, 1, 1, 1, 64, window=(-2, 0, 0, 1, 0))[0] == -2
    lib, w = pkg.load_library(), _CWindow(4, 0, 0, 1, 0)
    assert lib.calibatt_window_attn_form(1, 1, 1, 1, 1, 64, C.addressof(w), None) == -1
    assert lib.calibatt_window_attn_form(1, 1, 1, 1, 1, 64, None, C.addressof(_CWindowForm())) == -1
    with pytest.raises(pkg.CalibattError):
        pkg.Window(-5).form(1, 1, 1, 1, 1, 64)


@pytest.mark.parametrize("sizes", [(1, 1, 1, 1, 1, 64), (16, 32, 8, 1, 65536, 128), (1, 4, 4, 3000, 3000, 128), (2, 2, 1, 300, 900, 64),
                                   (1, 40, 40, 32760, 32760, 128)])
def test_forms_and_workspaces_agree(sizes):
    B, Hq, Hkv, Nq, Nk, D = sizes
    for w in (pkg.Window(-1), pkg.Window(64, 3, 9), pkg.Window(2, -1, 300, 150)):
        f, (fwd, bwd) = w.form(*sizes), w.workspace_bytes(*sizes)
        assert f["forward"] == pkg.WINDOW_SHARED_ROWS if Hq // Hkv * Nq <= 32 else f["forward"] != pkg.WINDOW_SHARED_ROWS
        assert fwd == (f["forward_parts"] * B * Hq * Nq * (D + 2) * 4 if f["forward_parts"] > 1 else 0)
        assert min(f["dq_parts"], f["dkv_parts"], f["sink_parts"]) >= 1 and f["sink_blocks"] <= -(-Nk // 256)
        sums = B * Hq * Nq * 8 + (f["dq_parts"] > 1) * f["dq_parts"] * B * Hq * Nq * D * 4
        assert bwd >= sums + (f["dkv_parts"] > 1) * f["dkv_parts"] * B * Hkv * Nk * 2 * D * 4
