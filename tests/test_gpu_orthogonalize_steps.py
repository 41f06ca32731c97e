"""Orthogonalised updates of few steps and of none, of matrices of a workgroup and of tiled ones.  Run with -m gpu."""
import pytest
import torch

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
F32, BF16 = torch.float32, torch.bfloat16
# by a workgroup; by tiles of 64, wide and tall; by tiles of 128 (64 of them)
SIZES = [(24, 40, 1), (128, 100, 1), (150, 400, 1), (300, 70, 1), (400, 150, 1), (250, 250, 64)]


@pytest.fixture(scope="module")
def e2f():
    import paper_2501_19216_amd as m
    return m


@pytest.fixture(scope="module")
def ctx(e2f):
    c = e2f.e2f_create(0, 0)
    yield c
    c.close()


@pytest.mark.parametrize("r,c,n", SIZES)
@pytest.mark.parametrize("steps", [0, 1, 2])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
def test_a_value_that_is_not_finite_without_steps(e2f, ctx, r, c, n, steps, bad):
    """It makes its matrix NaN, whatever the number of steps, and leaves the others alone."""
    g = torch.Generator().manual_seed(r + c)
    grads = torch.randn(n + 2, r, c, generator=g).to(DEV)
    weights = torch.randn(n + 2, r, c, generator=g).to(DEV)
    kw = dict(steps=steps, scale=-0.5)
    for extra in ({}, dict(weights=[weights], decay=0.5)):
        clean = e2f.e2f_orthogonalize(ctx, [grads], **kw, **extra)[0]
        worse = grads.clone()
        worse[1, r - 1, c // 2] = bad
        got = e2f.e2f_orthogonalize(ctx, [worse], **kw, **extra)[0]
        assert bool(clean.isfinite().all()) and bool(got[1].isnan().all())
        assert torch.equal(got[0], clean[0]) and torch.equal(got[2:], clean[2:])
