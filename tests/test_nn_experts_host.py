"""CPU-only checks of the operators for tokens, experts and orthogonal updates: refusals that come before the GPU is touched, and the references that
the kernels are judged by."""
import ctypes as C
import os

import pytest
import torch

import nn_experts_reference as ref


@pytest.fixture(scope="module")
def nn():
    from paper_2103_07454_amd import evg, nn as m
    if not os.path.exists(evg.LIB_PATH):
        from paper_2103_07454_amd import build
        build.build_library()
    m.lib()
    return m


def refused(nn, init, cfg, change):
    from paper_2103_07454_amd import evg
    for k, v in change.items():
        setattr(cfg, k, v)
    h = C.c_void_p()
    rc = getattr(nn.lib(), init)(C.byref(h), C.byref(cfg), None)
    assert h.value is None and evg.lib().evg_error_text()
    return rc == 1


@pytest.mark.parametrize("change", [dict(workers=0), dict(workers=65536), dict(vocab=0), dict(vocab=(1 << 24) + 1), dict(width=0), dict(width=(1 << 20) + 1),
                                    dict(max_tokens=(1 << 26) + 1), dict(type=3), dict(scale=float("inf"))])
def test_embed_refuses(nn, change):
    assert refused(nn, "evg_embed_init", nn.EmbedConfig(2, 10, 8, 4, 0, 1.0, 1), change)


@pytest.mark.parametrize("change", [dict(workers=0), dict(experts=0), dict(experts=1025), dict(top=0), dict(top=9), dict(type=3), dict(workers=1 << 16, max_tokens=1 << 16)])
def test_router_refuses(nn, change):
    assert refused(nn, "evg_router_init", nn.RouterConfig(2, 8, 2, 4, 0, 0), change)


@pytest.mark.parametrize("change", [dict(workers=0), dict(workers=65536), dict(experts=0), dict(experts=1025), dict(top=0), dict(top=9), dict(width=0), dict(width=(1 << 20) + 1),
                                    dict(max_tokens=1 << 28), dict(capacity=1 << 29), dict(type=3), dict(workers=65535, max_tokens=1 << 27, top=1)])
def test_experts_refuses(nn, change):
    assert refused(nn, "evg_experts_init", nn.ExpertsConfig(2, 8, 2, 8, 4, 0, 0), change)


@pytest.mark.parametrize("change", [dict(matrices=0), dict(matrices=65536), dict(rows=0), dict(rows=65537), dict(cols=0), dict(rows=16385, cols=16385), dict(type=3), dict(out_type=1),
                                    dict(steps=0), dict(steps=65), dict(a=float("nan")), dict(a=3.5, b=0.0, c=0.0), dict(b=float("inf")), dict(momentum=float("nan")),
                                    dict(eps=-1.0), dict(eps=float("inf")), dict(scale=float("nan"))])
def test_ortho_refuses(nn, change):
    assert refused(nn, "evg_ortho_init", nn.OrthoConfig(2, 8, 8, 0, 0, 5, *ref.POLYNOMIAL, 0.9, 1, 1e-7, 1.0), change)


def test_null_handles(nn):
    l, m, i, p = nn.lib(), C.byref(nn.Mat()), C.byref(nn.Ids()), C.byref(nn.ExpertsPlan())
    assert l.evg_embed_forward(None, 1, i, m, m) == 1 and l.evg_embed_backward(None, 1, i, m, m, 0) == 1
    assert l.evg_router_forward(None, 1, m, None, None) == 1 and l.evg_router_backward(None, 1, None, m, None, m) == 1
    assert l.evg_experts_dispatch(None, 1, m, None, m, p) == 1 and l.evg_experts_combine(None, 1, m, None, p, m) == 1
    assert l.evg_experts_combine_backward(None, 1, m, m, None, p, m, None) == 1 and l.evg_experts_slots(None, 5) == 0
    assert l.evg_ortho_update(None, m, m, m, m) == 1
    for name in ("embed", "router", "experts", "ortho"):
        assert getattr(l, f"evg_{name}_destroy")(None) == 0
        assert getattr(l, f"evg_{name}_init")(None, None, None) == 1


def test_no_silent_fallback_without_gpu(nn):
    if torch.cuda.is_available():
        pytest.skip("a GPU is present")
    for make in (lambda: nn.Embedding(4, 4, max_tokens=1), lambda: nn.Router(4, 2, max_tokens=1), lambda: nn.ExpertSort(4, 2, 8, max_tokens=1), lambda: nn.Orthogonal(4, 4)):
        with pytest.raises(RuntimeError):
            make()


def test_reference_gradients_against_differentiation():
    gen = torch.Generator().manual_seed(0)
    make = lambda *s: torch.randn(*s, generator=gen, dtype=torch.float64)  # noqa: E731
    table, ids, dy = make(7, 5).requires_grad_(), torch.tensor([3, -1, 3, 6, 0, 9]), make(6, 5)
    y, _ = ref.embed(ids, table, 0.7, torch.float32)
    got, _ = ref.embed_backward(ids, dy, 7, 0.7, torch.float32)
    assert torch.allclose(got, torch.autograd.grad(y, table, dy)[0])

    logits = make(9, 6)
    logits[0], logits[1, :4] = -float("inf"), -float("inf")
    chosen = ref.choose(logits, 3)
    assert chosen[0].tolist() == [-1, -1, -1] and int((chosen[1] >= 0).sum()) == 2
    dw = make(9, 3)
    for over_chosen in (False, True):
        w, _, d, _ = ref.route(logits, chosen, over_chosen, dw, torch.float32)
        loss = lambda z: (ref.route(z, chosen, over_chosen)[0] * dw).sum()  # noqa: E731
        h = 1e-6
        for row in range(1, 9):
            for e in range(6):
                if logits[row, e] > -float("inf"):
                    z = torch.zeros_like(logits)
                    z[row, e] = h
                    assert abs(float(loss(logits + z) - loss(logits - z)) / (2 * h) - float(d[row, e])) < 1e-7

    x, weights, dy = make(9, 4), make(9, 3), make(9, 4)
    for capacity in (0, 2):
        slot, source, counts = ref.plan(chosen, 6, capacity)
        assert int(counts.sum()) == int((chosen >= 0).sum())
        rows = ref.dispatch(x, source, 3).requires_grad_()
        weights.requires_grad_()
        y, _ = ref.combine(rows, weights, slot, torch.float32)
        want = torch.autograd.grad(y, (rows, weights), dy)
        (d_rows, _), (d_weights, _) = ref.combine_backward(dy, rows.detach(), weights.detach(), slot, source, 3, torch.float32)
        assert torch.allclose(d_rows, want[0]) and torch.allclose(d_weights, want[1])
        # the rows' gradient back to the tokens is the sum over their slots
        leaf = x.clone().requires_grad_()
        back = torch.autograd.grad(ref.dispatch(leaf, source, 3), leaf, want[0])[0]
        assert torch.allclose(ref.combine(want[0], None, slot, torch.float32)[0], back)


def test_reference_update_against_singular_values():
    gen = torch.Generator().manual_seed(1)
    for r, c in ((5, 9), (9, 5), (6, 6), (1, 4)):
        u = torch.randn(r, c, generator=gen, dtype=torch.float64)
        left, s, right = torch.linalg.svd(u, full_matrices=False)
        s = s / (u.norm() + 1e-7)
        for _ in range(5):
            s = 3.4445 * s - 4.7750 * s ** 3 + 2.0315 * s ** 5
        got, bound = ref.orthogonal(u, torch.float32)
        assert torch.allclose(got, left @ torch.diag(s) @ right, atol=1e-10) and bound > 0
