"""Layer norm of irrep features and of rows, with all gradients, against float64.  Run with -m gpu."""
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


def data(n, L, C, t, seed, offset=0.7):
    g = torch.Generator().manual_seed(seed)
    x = (torch.randn(n, (L + 1) ** 2, C, generator=g) * torch.exp(0.5 * torch.randn(n, 1, 1, generator=g)) + offset).to(t)
    return x, 1 + 0.2 * torch.randn(L + 1, C, generator=g), 0.3 * torch.randn(C, generator=g), \
        torch.randn(n, (L + 1) ** 2, C, generator=g).to(t)


def run(e2f, ctx, x, L, w, b, g, silu=False, eps=1e-5):
    """x, g [n, K, C] on the CPU or the device."""
    n, K, C = x.shape
    kw = dict(lmax=L, weight=None if w is None else w.to(DEV), bias=None if b is None else b.to(DEV), eps=eps, silu=silu)
    xd, gd = x.to(DEV), g.to(DEV)
    if not L:
        xd, gd = xd[:, 0], gd[:, 0].contiguous()
    want = ref.layer_norm(x.cpu(), L, w, b, eps, silu, g.cpu())
    out = e2f.e2f_layer_norm_forward(ctx, xd, **kw)
    ref.check(out.view(n, K, C), want["out"], "out")
    gx, gw, gb = e2f.e2f_layer_norm_backward(ctx, xd, gd, **kw)
    ref.check(gx.view(n, K, C), want["grad_x"], "grad_x")
    ref.check(gw, want["grad_w"], "grad_w")
    ref.check(gb, want["grad_b"], "grad_b")
    return out, gx, gw, gb


@pytest.mark.parametrize("C", [1, 2, 3, 4, 7, 8, 31, 64, 100, 129, 256, 257, 500, 512, 513, 1000, 1024, 1025, 2049, 5001, 8192])
@pytest.mark.parametrize("t", [F32, BF16])
@pytest.mark.parametrize("silu", [False, True])
def test_rows(e2f, ctx, C, t, silu):
    n = 37 if C > 300 else 301
    x, w, b, g = data(n, 0, C, t, C)
    run(e2f, ctx, x, 0, w, b, g, silu)


@pytest.mark.parametrize("n", [1, 2, 3, 15, 16, 17, 511, 513, 4097, 20000])
@pytest.mark.parametrize("C", [12, 64, 130])
def test_numbers_of_rows(e2f, ctx, n, C):
    x, w, b, g = data(n, 0, C, F32, n + C)
    run(e2f, ctx, x, 0, w, b, g, True)


@pytest.mark.parametrize("L", [1, 2, 3, 4, 5, 6])
@pytest.mark.parametrize("C", [4, 12, 64, 128, 260, 516, 1024])
@pytest.mark.parametrize("t", [F32, BF16])
def test_degrees(e2f, ctx, L, C, t):
    x, w, b, g = data(23, L, C, t, L + C)
    run(e2f, ctx, x, L, w, b, g)


@pytest.mark.parametrize("L", [0, 2, 4])
def test_many_atoms(e2f, ctx, L):
    x, w, b, g = data(3001, L, 36, F32, L)
    run(e2f, ctx, x, L, w, b, g)


@pytest.mark.parametrize("L", [0, 3])
def test_without_weights(e2f, ctx, L):
    x, w, b, g = data(50, L, 20, F32, 3)
    run(e2f, ctx, x, L, None, None, g)
    run(e2f, ctx, x, L, w, None, g)
    run(e2f, ctx, x, L, None, b, g)


@pytest.mark.parametrize("offset", [100.0, -3e4])
@pytest.mark.parametrize("C", [64, 1000])
def test_rows_far_from_zero(e2f, ctx, offset, C):
    x, w, b, g = data(40, 0, C, F32, 5, offset)
    run(e2f, ctx, x, 0, w, b, g)


def test_constant_and_tiny_rows(e2f, ctx):
    """A variance of zero, of far less than eps, and of values whose squares underflow."""
    x, w, b, g = data(9, 0, 48, F32, 6)
    x[0] = 3.0
    x[1] = 0.0
    x[2] *= 1e-6
    x[3] *= 1e-25
    run(e2f, ctx, x, 0, w, b, g)
    run(e2f, ctx, x, 0, w, b, g, True)
    x, w, b, g = data(9, 2, 16, F32, 7)
    x[0, 1:] = 0.0
    x[1] = 0.0
    run(e2f, ctx, x, 2, w, b, g)


def test_activation_far_out(e2f, ctx):
    """Large weights: the activation's both ends, without overflow."""
    x, w, b, g = data(64, 0, 32, F32, 8)
    run(e2f, ctx, x, 0, 100 * w, b, g, True)
    out = e2f.e2f_layer_norm_forward(ctx, x[:, 0].to(DEV), weight=(1e30 * w).to(DEV), silu=True)
    assert not bool(out.isnan().any())


def test_values_that_are_not_finite_stay_in_their_rows(e2f, ctx):
    for L, C in ((0, 40), (2, 12), (4, 128)):
        x, w, b, g = data(20, L, C, F32, 9)
        clean = run(e2f, ctx, x, L, w, b, g)
        bad = x.clone()
        bad[3, 0, 5], bad[11, 0, 0] = float("nan"), float("inf")
        xd, gd = (t.to(DEV) if L else t[:, 0].contiguous().to(DEV) for t in (bad, g))
        kw = dict(lmax=L, weight=w.to(DEV), bias=b.to(DEV))
        out = e2f.e2f_layer_norm_forward(ctx, xd, **kw)
        gx, gw, gb = e2f.e2f_layer_norm_backward(ctx, xd, gd, **kw)
        rows = [i for i in range(20) if i not in (3, 11)]
        assert torch.equal(out[rows], clean[0][rows]) and torch.equal(gx[rows], clean[1][rows])
        first = (lambda t: t[:, 0]) if L else (lambda t: t)
        assert bool(first(out)[[3, 11]].isnan().all()) and bool(first(gx)[[3, 11]].isnan().all())
        if L:
            assert torch.equal(out[:, 1:], clean[0][:, 1:]) and torch.equal(gx[:, 1:], clean[1][:, 1:])


@pytest.mark.parametrize("t", [F32, BF16])
@pytest.mark.parametrize("L,C", [(0, 33), (0, 64), (0, 1030), (2, 16), (4, 64)])
def test_rows_further_apart_and_odd_addresses(e2f, ctx, t, L, C):
    n, K = 57, (L + 1) ** 2
    x, w, b, g = data(n, L, C, t, C)
    wide = torch.full((n, K * C + 7), float("nan"), dtype=t, device=DEV)
    wide[:, 3:3 + K * C] = x.flatten(1).to(DEV)
    view = wide[:, 3:3 + K * C]
    out = torch.empty(n * K * C + 1, dtype=t, device=DEV)[1:]
    kw = dict(lmax=L, weight=w.to(DEV), bias=b.to(DEV))
    shape = (n, K, C) if L else (n, C)
    xv, gd = (view.unflatten(1, (K, C)) if L else view), g.to(DEV).view(shape)
    got = e2f.e2f_layer_norm_forward(ctx, xv, out=out.view(shape), **kw)
    packed = x.to(DEV).view(shape)
    assert torch.equal(got, e2f.e2f_layer_norm_forward(ctx, packed, **kw))
    odd = torch.empty(n * K * C + 1, dtype=t, device=DEV)[1:].view(shape).copy_(gd)
    for p, q in zip(e2f.e2f_layer_norm_backward(ctx, xv, odd, **kw), e2f.e2f_layer_norm_backward(ctx, packed, gd, **kw)):
        assert torch.equal(p, q)


def test_parts_of_the_backward(e2f, ctx):
    x, w, b, g = data(100, 1, 8, F32, 2)
    kw = dict(lmax=1, weight=w.to(DEV), bias=b.to(DEV))
    gx, gw, gb = e2f.e2f_layer_norm_backward(ctx, x.to(DEV), g.to(DEV), **kw)
    only = e2f.e2f_layer_norm_backward(ctx, x.to(DEV), g.to(DEV), want_weights=False, **kw)
    assert torch.equal(only[0], gx) and only[1] is None and only[2] is None
    none, gw2, gb2 = e2f.e2f_layer_norm_backward(ctx, x.to(DEV), g.to(DEV), want_x=False, **kw)
    assert none is None and torch.equal(gw, gw2) and torch.equal(gb, gb2)


def test_no_rows(e2f, ctx):
    x = torch.empty(0, 4, 8, device=DEV)
    assert e2f.e2f_layer_norm_forward(ctx, x, lmax=1).shape == x.shape
    gx, gw, gb = e2f.e2f_layer_norm_backward(ctx, x, x, lmax=1)
    assert gx.shape == x.shape and bool((gw == 0).all()) and bool((gb == 0).all())


@pytest.mark.parametrize("L,silu", [(0, False), (0, True), (2, False)])
def test_gradients_against_differences(e2f, ctx, L, silu):
    """Central differences of float64 sums of the float32 forward: steps of 2^-7 of values near one leave 2^-14 of curvature
    and 2^-17 sqrt(size) of rounding."""
    n, C = 5, 12
    x, w, b, g = data(n, L, C, F32, 4)
    shape = (n, (L + 1) ** 2, C) if L else (n, C)
    p = dict(x=x.view(shape).to(DEV), weight=w.to(DEV), bias=b.to(DEV))
    gd = g.view(shape).to(DEV)
    f = lambda q: float((e2f.e2f_layer_norm_forward(ctx, q["x"], lmax=L, weight=q["weight"], bias=q["bias"], silu=silu).double() * gd).sum())  # noqa: E731
    grads = e2f.e2f_layer_norm_backward(ctx, p["x"], gd, lmax=L, weight=p["weight"], bias=p["bias"], silu=silu)
    gen = torch.Generator().manual_seed(1)
    for name, grad in zip(("x", "weight", "bias"), grads):
        for _ in range(4):
            v = torch.randn(p[name].shape, generator=gen).to(DEV)
            v = v / v.norm()
            h = 2.0 ** -7
            num = (f({**p, name: p[name] + h * v}) - f({**p, name: p[name] - h * v})) / (2 * h)
            scale = float(grad.double().norm())
            assert abs(num - float((grad.double() * v).sum())) <= 4e-3 * scale + 1e-3


def test_captured_and_replayed(e2f, ctx):
    x, w, b, g = (t.to(DEV) for t in data(700, 2, 24, F32, 1))
    ws = torch.empty(1 << 22, dtype=torch.uint8, device=DEV)
    kw = dict(lmax=2, weight=w, bias=b)
    with pytest.raises(ValueError):
        with torch.cuda.graph(torch.cuda.CUDAGraph()):
            e2f.e2f_layer_norm_backward(ctx, x, g, **kw)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = e2f.e2f_layer_norm_forward(ctx, x, **kw)
        grads = e2f.e2f_layer_norm_backward(ctx, x, g, workspace=ws, **kw)
    for k in range(4):
        x.mul_(-1.25).add_(0.1)
        g.mul_(1.5)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, e2f.e2f_layer_norm_forward(ctx, x, **kw))
        for p, q in zip(grads, e2f.e2f_layer_norm_backward(ctx, x, g, **kw)):
            assert torch.equal(p, q)


def test_on_another_stream(e2f, ctx):
    x, w, b, g = (t.to(DEV) for t in data(3000, 0, 64, F32, 1))
    x, g = x[:, 0], g[:, 0].contiguous()
    want = e2f.e2f_layer_norm_backward(ctx, x, g, weight=w, bias=b)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        got = e2f.e2f_layer_norm_backward(ctx, x, g, weight=w, bias=b)
    again = e2f.e2f_layer_norm_backward(ctx, x, g, weight=w, bias=b)
    torch.cuda.current_stream().wait_stream(s)
    for p, q, r in zip(want, got, again):
        assert torch.equal(p, q) and torch.equal(p, r)


def test_refused_by_the_binding(e2f, ctx):
    x, w, b, g = (t.to(DEV) for t in data(10, 0, 8, F32, 1))
    x, g = x[:, 0], g[:, 0]
    for bad in (lambda: e2f.e2f_layer_norm_forward(ctx, x.half()), lambda: e2f.e2f_layer_norm_forward(ctx, x.cpu()),
                lambda: e2f.e2f_layer_norm_forward(ctx, x, lmax=1), lambda: e2f.e2f_layer_norm_forward(ctx, x.t()),
                lambda: e2f.e2f_layer_norm_forward(ctx, x, weight=w[:, :7]),
                lambda: e2f.e2f_layer_norm_forward(ctx, x, bias=b.bfloat16()),
                lambda: e2f.e2f_layer_norm_forward(ctx, x, out=torch.empty(10, 9, device=DEV)),
                lambda: e2f.e2f_layer_norm_backward(ctx, x, g[:9]),
                lambda: e2f.e2f_layer_norm_backward(ctx, x, g.bfloat16()),
                lambda: e2f.e2f_layer_norm_backward(ctx, x, g, workspace=torch.empty(4096, device=DEV))):
        with pytest.raises(ValueError):
            bad()
    y = torch.zeros(4, 4, 8, device=DEV)
    for bad in (lambda: e2f.e2f_layer_norm_forward(ctx, y, lmax=1, silu=True),
                lambda: e2f.e2f_layer_norm_forward(ctx, x, eps=-1.0), lambda: e2f.e2f_layer_norm_forward(ctx, x, out=x),
                lambda: e2f.e2f_layer_norm_forward(ctx, torch.zeros(2, 9000, device=DEV))):
        with pytest.raises(e2f.E2FError):
            bad()
