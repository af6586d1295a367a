"""CPU-only checks of the operators' C ABI: a plain C header, every declared symbol, and refusals that come before the GPU is touched."""
import ctypes as C
import os
import re
import subprocess
import textwrap

import numpy as np
import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def nn():
    from paper_2103_07454_amd import evg, nn as m
    if not os.path.exists(evg.LIB_PATH):
        from paper_2103_07454_amd import build
        build.build_library()
    m.lib()
    return m


def test_header_compiles_as_c99(tmp_path):
    src = tmp_path / "use.c"
    src.write_text(textwrap.dedent("""
        #include "evg_nn.h"
        int main(void) {
          evg_clip_config a; evg_blocknorm_config b; evg_ffn_config c; evg_blocknorm_in i; evg_blocknorm_grads g; evg_mat m;
          (void)a; (void)b; (void)c; (void)i; (void)g; (void)m;
          (void)evg_clip_init; (void)evg_clip_run; (void)evg_clip_destroy; (void)evg_blocknorm_init; (void)evg_blocknorm_forward;
          (void)evg_blocknorm_backward; (void)evg_blocknorm_destroy; (void)evg_ffn_init; (void)evg_ffn_saved_bytes;
          (void)evg_ffn_forward; (void)evg_ffn_backward; (void)evg_ffn_destroy;
          return 0;
        }
    """))
    subprocess.run(["gcc", "-std=c99", "-Wall", "-Wextra", "-Werror", "-pedantic", "-I", os.path.join(ROOT, "include"), "-c", str(src),
                    "-o", str(tmp_path / "use.o")], check=True)


def test_exports_every_declared_symbol(nn):
    header = open(os.path.join(ROOT, "include", "evg_nn.h")).read()
    header = re.sub(r"/\*.*?\*/", "", header, flags=re.S)
    declared = set(re.findall(r"\b(evg_[a-z_]+)\s*\(", header))
    assert declared == set(nn.EXPORTS)
    for name in declared:
        assert getattr(nn.lib(), name) is not None


def refused(nn, init, cfg):
    from paper_2103_07454_amd import evg
    h = C.c_void_p()
    rc = getattr(nn.lib(), init)(C.byref(h), C.byref(cfg), None)
    assert h.value is None and evg.lib().evg_error_text()
    return rc


@pytest.mark.parametrize("change", [dict(P=0), dict(L=0), dict(grad_type=3), dict(out_type=1), dict(eps=-1.0), dict(eps=float("inf")),
                                    dict(nonfinite=2), dict(layer_numel=None)])
def test_clip_refuses(nn, change):
    n = np.array([10, 3], np.uint64)
    cfg = nn.ClipConfig(2, 2, n.ctypes.data_as(C.POINTER(C.c_uint64)), 0, 0, 1e-6, 0)
    for k, v in change.items():
        setattr(cfg, k, v)
    assert refused(nn, "evg_clip_init", cfg) == 1


@pytest.mark.parametrize("change", [dict(workers=0), dict(width=0), dict(width=16385), dict(type=3), dict(kind=2), dict(eps=-1.0),
                                    dict(eps=float("nan")), dict(residual_scale=float("nan")), dict(branch_scale=float("inf")),
                                    dict(workers=1 << 20, max_rows=1 << 20)])
def test_blocknorm_refuses(nn, change):
    cfg = nn.BlockNormConfig(2, 64, 8, 0, 0, 1e-5, 1.0, 1.0)
    for k, v in change.items():
        setattr(cfg, k, v)
    assert refused(nn, "evg_blocknorm_init", cfg) == 1


@pytest.mark.parametrize("change", [dict(workers=0), dict(workers=65536), dict(width=0), dict(width=(1 << 20) + 1), dict(hidden=0),
                                    dict(hidden=(1 << 20) + 1), dict(type=3), dict(activation=4), dict(max_rows=0x7FFFFFFF),
                                    dict(workers=65535, max_rows=0x7FFFFF00, hidden=1 << 20)])
def test_ffn_refuses(nn, change):
    cfg = nn.FFNConfig(1, 64, 64, 8, 0, 0, 1)
    for k, v in change.items():
        setattr(cfg, k, v)
    assert refused(nn, "evg_ffn_init", cfg) == 1


def test_null_handles(nn):
    l = nn.lib()
    m, i, g = C.byref(nn.Mat()), C.byref(nn.BlockNormIn()), C.byref(nn.BlockNormGrads())
    assert l.evg_clip_run(None, None, None, 1.0, 1.0, None) == 1
    assert l.evg_blocknorm_forward(None, i, m, m) == 1 and l.evg_blocknorm_backward(None, i, m, m, g) == 1
    assert l.evg_ffn_forward(None, 1, m, m, m, m, m, None) == 1
    assert l.evg_ffn_backward(None, 1, m, m, m, m, m, None, m, m, m, m) == 1
    assert l.evg_ffn_saved_bytes(None, 5) == 0
    assert l.evg_clip_destroy(None) == 0 and l.evg_blocknorm_destroy(None) == 0 and l.evg_ffn_destroy(None) == 0


def test_no_silent_fallback_without_gpu(nn):
    import torch
    if torch.cuda.is_available():
        pytest.skip("a GPU is present")
    for make in (lambda: nn.GradClip([4], 1), lambda: nn.BlockNorm(8, max_rows=1), lambda: nn.GatedFFN(8, 8, max_rows=1)):
        with pytest.raises(RuntimeError):
            make()


def test_reference_gradients_against_automatic_ones():
    """The formulas of tests/nn_reference.py, by which the kernels are judged, against differentiation by torch in 64 bits."""
    import torch
    import nn_reference as ref
    gen = torch.Generator().manual_seed(0)
    make = lambda *s: torch.randn(*s, generator=gen, dtype=torch.float64)
    T, D, F = 7, 12, 9
    for kind in ("silu", "gelu", "gelu_tanh", "relu"):
        v = [make(T, D).requires_grad_(), make(F, D).requires_grad_(), make(F, D).requires_grad_(), make(D, F).requires_grad_()]
        dy = make(T, D)
        got = ref.ffn(kind, torch.float32, *[t.detach() for t in v], dy)
        y = (ref.act(kind, v[0] @ v[1].t())[0] * (v[0] @ v[2].t())) @ v[3].t()
        for name, g in zip(("dx", "dw_gate", "dw_up", "dw_down"), torch.autograd.grad(y, v, dy)):
            assert torch.allclose(got[name][0], g, rtol=1e-10, atol=1e-12), (kind, name)
    for kind in ("rms", "layer"):
        t = dict(residual=make(T, D), branch=make(T, D), gate=make(3, D), post=make(D), pre=make(D))
        if kind == "layer":
            t.update(post_bias=make(D), pre_bias=make(D))
        do, dn = make(T, D), make(T, D)
        kw = dict(eps=1e-3, alpha=0.7, beta=1.3, gate_rows=3)
        got, size = ref.blocknorm(kind, dict(t, d_out=do, d_normed=dn), **kw)
        assert all((size[k] >= got[k].abs() * (1 - 1e-12)).all() for k in ("residual", "normed", "d_residual", "d_branch"))
        leaves = {k: x.clone().requires_grad_() for k, x in t.items()}
        out, _ = ref.blocknorm(kind, leaves, **kw)
        for name, g in zip(t, torch.autograd.grad([out["residual"], out["normed"]], list(leaves.values()), [do, dn])):
            assert torch.allclose(got["d_" + name], g, rtol=1e-9, atol=1e-11), (kind, name)
