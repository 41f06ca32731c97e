"""Orthogonalised updates entry by entry against float64, with bounds from the same arithmetic on the CPU, which see the
loss of any operand's low part (test_update_precision.py).  Run with -m gpu."""
import pytest
import torch

import training_reference as ref
import update_precision as up

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
F32, BF16 = torch.float32, torch.bfloat16
# matrices of a workgroup, tiles of 64 (with waves along the sums and without), tiles of 128 (of the triangle too: the
# last but one)
WORKGROUP = [(16, 16, 2), (17, 16, 1), (60, 40, 1), (64, 384, 1), (96, 224, 1), (140, 90, 1), (128, 128, 3)]
TILED = [(130, 200, 1), (200, 333, 2), (517, 200, 6), (257, 259, 1), (300, 1500, 1), (640, 640, 1), (250, 250, 64), (500, 380, 22),
         (510, 640, 64), (1270, 380, 30)]
EACH = [(4.0, -5.0, 2.0), (2.5, -3.0, 1.5)]  # of two steps, other than the default


@pytest.fixture(scope="module")
def e2f():
    import paper_2501_19216_amd as m
    return m


@pytest.fixture(scope="module")
def ctx(e2f):
    c = e2f.e2f_create(0, 0)
    yield c
    c.close()


def check(e2f, ctx, r, c, n, kind, gt=F32, wt=F32, moments=False, weights=False, coefs=(ref.MUON,) * 5, scale=1.0,
          decay=0.0, nesterov=True):
    grads = [up.matrix(r, c, i, kind).to(gt) for i in range(n)]
    kw = dict(steps=len(coefs), coefs=coefs, scale=scale, decay=decay, nesterov=nesterov, momentum=0.9)
    dev = lambda ts: None if ts is None else [t.to(DEV) for t in ts]  # noqa: E731
    m = [3 * up.matrix(r, c, 100 + i, kind) for i in range(n)] if moments else None
    w = [up.matrix(r, c, 200 + i, "plain").to(wt) for i in range(n)] if weights else None
    outs = [torch.empty(r, c, dtype=wt, device=DEV) for _ in range(n)]
    e2f.e2f_orthogonalize(ctx, dev(grads), outs=outs, moments=dev(m), weights=dev(w), **kw)
    for i in sorted({0, n // 2, n - 1}):
        want = up.expected(grads[i], m[i] if moments else None, w[i] if weights else None, 0.9, nesterov, coefs, scale,
                           decay, dtype=wt)
        up.check(outs[i], want, (r, c, kind, i))


@pytest.mark.parametrize("r,c,n", WORKGROUP + TILED)
@pytest.mark.parametrize("kind", ["plain", "mixed", "strong"])
def test_five_steps(e2f, ctx, r, c, n, kind):
    check(e2f, ctx, r, c, n, kind)


@pytest.mark.parametrize("r,c,n", WORKGROUP + TILED)
@pytest.mark.parametrize("coefs", [[], [ref.MUON], [ref.MUON] * 2, EACH], ids=["none", "one", "two", "each"])
@pytest.mark.parametrize("t", [F32, BF16])
def test_few_steps(e2f, ctx, r, c, n, coefs, t):
    """The last product straight behind the first matrix, both of the buffers that steps take in turn, coefficients of
    each step."""
    check(e2f, ctx, r, c, n, "strong", gt=t, coefs=coefs)
    check(e2f, ctx, r, c, n, "strong", wt=t, weights=True, coefs=coefs, scale=-0.3, decay=0.98)


@pytest.mark.parametrize("r,c,n", [(60, 40, 1), (128, 128, 3), (130, 200, 1), (400, 150, 1), (500, 380, 22)])
@pytest.mark.parametrize("nesterov", [False, True])
@pytest.mark.parametrize("wt", [F32, BF16])
def test_momentum_and_weights(e2f, ctx, r, c, n, nesterov, wt):
    check(e2f, ctx, r, c, n, "mixed", gt=BF16, wt=wt, moments=True, weights=True, scale=-0.2, decay=0.998, nesterov=nesterov)


def test_steps_that_converge(e2f, ctx):
    """Fifteen steps of the iteration that converges."""
    for r, c in ((30, 70), (128, 96), (150, 400)):
        check(e2f, ctx, r, c, 1, "plain", coefs=[(15 / 8, -10 / 8, 3 / 8)] * 15)
