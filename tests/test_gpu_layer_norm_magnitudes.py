"""Layer norm of features whose squares still fit float32 but whose cubes, or their root mean square's reciprocal's, do
not, against float64.  Run with -m gpu."""
import pytest
import torch

import training_reference as ref

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
F32, BF16 = torch.float32, torch.bfloat16


@pytest.fixture(scope="module")
def e2f():
    import paper_2501_19216_amd as m
    return m


@pytest.fixture(scope="module")
def ctx(e2f):
    c = e2f.e2f_create(0, 0)
    yield c
    c.close()


@pytest.mark.parametrize("L,C", [(0, 40), (1, 12), (2, 64), (3, 16), (4, 128), (5, 8), (6, 36)])
@pytest.mark.parametrize("t", [F32, BF16])
@pytest.mark.parametrize("power,eps", [(53, 1e-5), (42, 1e-5), (20, 0.0), (-20, 0.0), (-50, 0.0)])
def test_magnitudes(e2f, ctx, L, C, t, power, eps):
    n, K = 21, (L + 1) ** 2
    g = torch.Generator().manual_seed(L + C)
    x = (torch.randn(n, K, C, generator=g) * torch.exp(0.5 * torch.randn(n, 1, 1, generator=g)) * 2.0 ** power).to(t)
    w, b = 1 + 0.2 * torch.randn(L + 1, C, generator=g), 0.3 * torch.randn(C, generator=g)
    go = torch.randn(n, K, C, generator=g).to(t)
    shape = (n, K, C) if L else (n, C)
    kw = dict(lmax=L, weight=w.to(DEV), bias=b.to(DEV), eps=eps)
    want = ref.layer_norm(x, L, w, b, eps, False, go)
    ref.check(e2f.e2f_layer_norm_forward(ctx, x.view(shape).to(DEV), **kw).view(n, K, C), want["out"], "out")
    gx, gw, gb = e2f.e2f_layer_norm_backward(ctx, x.view(shape).to(DEV), go.view(shape).to(DEV), **kw)
    ref.check(gx.view(n, K, C), want["grad_x"], "grad_x")
    ref.check(gw, want["grad_w"], "grad_w")
    ref.check(gb, want["grad_b"], "grad_b")
