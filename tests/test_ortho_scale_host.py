"""CPU-only: the scales of orthogonal updates that are refused."""
import ctypes as C
import os

import pytest


@pytest.mark.parametrize("scale", [2.0 ** -81, -1e-30, 1e-45])
def test_scales_whose_bits_would_be_lost(scale):
    from paper_2103_07454_amd import evg, nn
    if not os.path.exists(evg.LIB_PATH):
        from paper_2103_07454_amd import build
        build.build_library()
    cfg, h = nn.OrthoConfig(2, 8, 8, 0, 0, 5, 3.4445, -4.7750, 2.0315, 0.9, 1, 1e-7, scale), C.c_void_p()
    assert nn.lib().evg_ortho_init(C.byref(h), C.byref(cfg), None) == 1 and h.value is None
    assert b"scale" in evg.lib().evg_error_text()
