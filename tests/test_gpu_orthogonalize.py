"""Orthogonalised updates of matrices against float64.  Run with -m gpu."""
import math

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


def matrix(r, c, seed, kind="mixed"):
    g = torch.Generator().manual_seed(seed)
    if kind == "plain":
        return torch.randn(r, c, generator=g)
    few = max(1, min(r, c) // 8)  # a few strong directions and noise
    return torch.randn(r, few, generator=g) @ torch.randn(few, c, generator=g) * few ** -0.5 + 0.1 * torch.randn(r, c, generator=g)


def close(got, want, x, room, scale, weight=None, decay=0.0):
    """The whole matrix's error: X's room and the roundings of the sum and of the type, in the Frobenius norm."""
    steps = ref.half_step(got.dtype) if got.dtype != F32 else 0.0
    size = abs(scale) * float(x.norm()) + (abs(decay) * float(weight.double().norm()) if weight is not None else 0.0)
    bound = abs(scale) * room + (2 * ref.U + 1.01 * steps) * size + 1e-30
    off = float((got.cpu().double() - want).norm())
    assert off <= bound, (off, bound, off / max(size, 1e-300))


def check(e2f, ctx, grads, **kw):
    """grads: CPU matrices [r, c]; kw of the call with CPU lists; only: the matrices that are looked at."""
    only = kw.pop("only", None)
    dev = lambda v: None if v is None else [t.to(DEV) for t in v]  # noqa: E731
    lists = {k: kw.pop(k) for k in ("moments", "weights") if k in kw}
    outs = kw.pop("outs", None)
    got_m = dev(lists.get("moments"))
    news = None if got_m is None else [torch.full_like(t, 9.0) for t in got_m]
    got = e2f.e2f_orthogonalize(ctx, dev(grads), outs=outs, moments=got_m, new_moments=news, weights=dev(lists.get("weights")), **kw)
    coefs = kw.get("coefs", ref.MUON)
    steps = kw.get("steps", 5)
    coefs = [coefs] * steps if not hasattr(coefs[0], "__len__") else coefs
    for i, g in enumerate(grads):
        if only is not None and i not in only:
            continue
        m, w = (lists[k][i] if k in lists else None for k in ("moments", "weights"))
        want, new, x, room = ref.orthogonalize(g, m, w, kw.get("momentum", 0.95), kw.get("nesterov", True), coefs,
                                               kw.get("scale", 1.0), kw.get("decay", 0.0), kw.get("eps", 1e-7))
        close(got[i], want, x, room, kw.get("scale", 1.0), w, kw.get("decay", 0.0))
        if m is not None:
            size = abs(kw.get("momentum", 0.95)) * m.double().abs() + g.double().abs()
            assert bool(((news[i].cpu().double() - new).abs() <= 2.01 * ref.U * size + 1e-45).all())
            assert torch.equal(got_m[i].cpu(), m)
    return got


@pytest.mark.parametrize("r,c", [(1, 1), (1, 2), (1, 50), (50, 1), (2, 2), (3, 5), (16, 16), (17, 16), (15, 40), (64, 64),
                                 (65, 63), (63, 200), (128, 128), (129, 128), (100, 300), (300, 100), (128, 500), (333, 200),
                                 (256, 256), (257, 259), (511, 130), (640, 640), (90, 220),
                                 (96, 224), (96, 225), (64, 384), (200, 33), (31, 512), (513, 32), (60, 257), (128, 129)])
@pytest.mark.parametrize("t", [F32, BF16])
def test_sizes(e2f, ctx, r, c, t):
    check(e2f, ctx, [matrix(r, c, r + c).to(t), matrix(r, c, 7, "plain").to(t)])


@pytest.mark.parametrize("r,c", [(1, 2000), (1200, 1100), (96, 5000), (3000, 40)])
def test_long_sides(e2f, ctx, r, c):
    check(e2f, ctx, [matrix(r, c, 5)])


@pytest.mark.parametrize("r,c,n", [(150, 200, 64), (300, 260, 60), (250, 250, 64), (500, 380, 22), (510, 640, 64), (1270, 380, 30)])
@pytest.mark.parametrize("t", [F32, BF16])
def test_many_large_matrices(e2f, ctx, r, c, n, t):
    """Enough of them that the products take their large tiles."""
    grads = [matrix(r, c, i).to(t) for i in range(n)]
    check(e2f, ctx, grads, weights=[matrix(r, c, 100 + i, "plain").to(t) for i in range(n)], scale=-0.3, decay=0.98,
          only=(0, 1, n // 2, n - 1))


@pytest.mark.parametrize("gt", [F32, BF16])
@pytest.mark.parametrize("wt", [F32, BF16])
@pytest.mark.parametrize("r,c", [(16, 16), (40, 100), (128, 128), (300, 70), (200, 333)])
@pytest.mark.parametrize("nesterov", [False, True])
def test_momentum_and_weights(e2f, ctx, gt, wt, r, c, nesterov):
    n = 3
    grads = [matrix(r, c, i).to(gt) for i in range(n)]
    check(e2f, ctx, grads, moments=[3 * matrix(r, c, 10 + i) for i in range(n)],
          weights=[matrix(r, c, 20 + i, "plain").to(wt) for i in range(n)], momentum=0.9, nesterov=nesterov, scale=-0.3,
          decay=0.98)


def test_in_place_and_weights_not_read(e2f, ctx):
    r, c = 48, 80
    g, m, w = (matrix(r, c, i).to(DEV) for i in range(3))
    kw = dict(scale=-0.1, decay=0.9)
    new = torch.empty_like(m)
    want = e2f.e2f_orthogonalize(ctx, [g], weights=[w], moments=[m], new_moments=[new], **kw)[0]
    w2, m2 = w.clone(), m.clone()
    got = e2f.e2f_orthogonalize(ctx, [g], outs=[w2], weights=[w2], moments=[m2], **kw)
    assert got[0] is w2 and torch.equal(w2, want) and torch.equal(m2, new)
    # without decay the weights are not looked at
    nan = torch.full_like(w, float("nan"))
    x = e2f.e2f_orthogonalize(ctx, [g], weights=[nan])[0]
    assert torch.equal(x, e2f.e2f_orthogonalize(ctx, [g])[0]) and bool(x.isfinite().all())


@pytest.mark.parametrize("coefs", [(1.5, -0.5, 0.0), (15 / 8, -10 / 8, 3 / 8)])
@pytest.mark.parametrize("r,c", [(30, 70), (128, 96), (150, 400)])
def test_steps_that_converge(e2f, ctx, coefs, r, c):
    """Twenty steps of the iterations that converge to the orthogonal factor, which is then known apart from them."""
    g = matrix(r, c, 3, "plain")
    got = check(e2f, ctx, [g], coefs=coefs, steps=30)[0].cpu().double()
    u, s, v = torch.linalg.svd(g.double(), full_matrices=False)
    assert float((got - u @ v).norm()) <= 1e-4 * math.sqrt(min(r, c))


@pytest.mark.parametrize("steps", [0, 1, 2, 7])
@pytest.mark.parametrize("r,c", [(20, 33), (140, 90)])
def test_numbers_of_steps(e2f, ctx, steps, r, c):
    check(e2f, ctx, [matrix(r, c, 2)], steps=steps)
    if steps:
        each = [(4.0 - 0.2 * k, -5.0 + 0.1 * k, 2.0) for k in range(steps)]
        if steps <= 2:
            check(e2f, ctx, [matrix(r, c, 2)], steps=steps, coefs=each)


def test_lists_of_stacks_and_sizes(e2f, ctx):
    """Stacks and matrices of several sizes in one call, more of one size than a launch holds."""
    g = torch.Generator().manual_seed(1)
    shapes = [(5, 12, 12), (8, 30), (3, 12, 12), (8, 30), (130, 12, 12), (67, 140, 130), (1, 70, 8), (0, 4, 4), (6, 6), (0, 5), (5, 0), (2, 0, 3)]
    grads = [torch.randn(*s, generator=g).to(DEV) for s in shapes]
    outs = e2f.e2f_orthogonalize(ctx, grads, scale=0.5)
    for x, o in zip(grads, outs):
        assert o.shape == x.shape
        one = [e2f.e2f_orthogonalize(ctx, [m], scale=0.5)[0] for m in (x if x.dim() == 3 else x[None])]
        # (of matrices beyond a workgroup's the order of the sums goes by how many there are)
        for i, (a, b) in enumerate(zip(one, o if o.dim() == 3 else o[None])):
            if min(x.shape[-2:]) <= 128:
                assert torch.equal(a, b)
            elif i % 16 == 0:
                want, _, xo, room = ref.orthogonalize((x if x.dim() == 3 else x[None])[i].cpu(), scale=0.5)
                close(a, want, xo, room, 0.5)
                close(b, want, xo, room, 0.5)
    want, _, x, room = ref.orthogonalize(grads[5][66].cpu(), scale=0.5)
    close(outs[5][66], want, x, room, 0.5)
    want, _, x, room = ref.orthogonalize(grads[4][129].cpu(), scale=0.5)
    close(outs[4][129], want, x, room, 0.5)
    assert e2f.e2f_orthogonalize(ctx, []) == []


@pytest.mark.parametrize("r,c", [(24, 40), (200, 140)])
def test_in_place_of_several_sizes(e2f, ctx, r, c):
    """Pieces of one buffer, matrices of several sizes, weights and momentum in place."""
    shapes = [(r, c), (3, 5, 7), (r, c), (12, 9)]
    sizes = [math.prod(s) for s in shapes]
    g = torch.Generator().manual_seed(r)
    flat = [torch.randn(sum(sizes), generator=g).to(DEV) for _ in range(3)]
    cut = lambda t: [x.view(s) for x, s in zip(t.split(sizes), shapes)]  # noqa: E731
    want = [t.clone() for t in flat]
    kw = dict(scale=-0.1, decay=0.5)
    for x, m, w in zip(cut(want[0]), cut(want[1]), cut(want[2])):
        e2f.e2f_orthogonalize(ctx, [x], outs=[w], weights=[w], moments=[m], **kw)
    grads, moments, weights = map(cut, flat)
    e2f.e2f_orthogonalize(ctx, grads, outs=weights, weights=weights, moments=moments, **kw)
    assert torch.equal(flat[0], want[0]) and torch.equal(flat[1], want[1])
    assert float((flat[2] - want[2]).norm()) <= 1e-4 * float(want[2].norm())


@pytest.mark.parametrize("r,c", [(24, 40), (200, 140)])
def test_scales_of_the_gradient(e2f, ctx, r, c):
    """Values near the ends of the type's range; zeros; one value."""
    for s in (1e-30, 1e30, 1e37):
        check(e2f, ctx, [matrix(r, c, 1) * s], eps=0.0)
    check(e2f, ctx, [matrix(r, c, 1) * 1e-8])
    zero = torch.zeros(r, c)
    assert bool((e2f.e2f_orthogonalize(ctx, [zero.to(DEV)])[0] == 0).all())
    one = zero.clone()
    one[3, 5] = -2.0
    check(e2f, ctx, [one])


@pytest.mark.parametrize("r,c", [(24, 40), (128, 128), (200, 140)])
@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
def test_values_that_are_not_finite_stay_in_their_matrix(e2f, ctx, r, c, bad):
    g = [matrix(r, c, i) for i in range(3)]
    clean = e2f.e2f_orthogonalize(ctx, [x.to(DEV) for x in g])
    g[1][2, 3] = bad
    got = e2f.e2f_orthogonalize(ctx, [x.to(DEV) for x in g])
    assert torch.equal(got[0], clean[0]) and torch.equal(got[2], clean[2]) and bool(got[1].isnan().all())


@pytest.mark.parametrize("t", [F32, BF16])
def test_odd_addresses(e2f, ctx, t):
    for r, c in ((33, 21), (70, 190)):
        g = matrix(r, c, 4).to(t)
        w = matrix(r, c, 6, "plain").to(t)
        odd = lambda x: torch.empty(x.numel() + 1, dtype=x.dtype, device=DEV)[1:].view(x.shape).copy_(x)  # noqa: E731
        out = odd(torch.full_like(w, 3.0))
        e2f.e2f_orthogonalize(ctx, [odd(g)], outs=[out], weights=[odd(w)], decay=0.5)
        assert torch.equal(out, e2f.e2f_orthogonalize(ctx, [g.to(DEV)], weights=[w.to(DEV)], decay=0.5)[0])


@pytest.mark.parametrize("r,c", [(40, 40), (150, 260)])
def test_captured_and_replayed(e2f, ctx, r, c):
    grads = [matrix(r, c, i).to(DEV) for i in range(4)]
    weights = [matrix(r, c, 9 + i).to(DEV) for i in range(4)]
    moments = [matrix(r, c, 19 + i).to(DEV) for i in range(4)]
    kw = dict(scale=-0.1, decay=0.99)
    w2, m2 = [w.clone() for w in weights], [m.clone() for m in moments]
    ws = torch.empty(1 << 24, dtype=torch.uint8, device=DEV)
    with pytest.raises(ValueError):
        with torch.cuda.graph(torch.cuda.CUDAGraph()):
            e2f.e2f_orthogonalize(ctx, grads, outs=weights, weights=weights, moments=moments, **kw)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        e2f.e2f_orthogonalize(ctx, grads, outs=weights, weights=weights, moments=moments, workspace=ws, **kw)
    for _ in range(4):
        graph.replay()
        torch.cuda.synchronize()
        e2f.e2f_orthogonalize(ctx, grads, outs=w2, weights=w2, moments=m2, **kw)
        assert all(torch.equal(a, b) for a, b in zip(weights + moments, w2 + m2))
        for x in grads:
            x.mul_(-0.7)


def test_same_bits_on_another_stream(e2f, ctx):
    g = [matrix(200, 300, i).to(DEV) for i in range(5)] + [matrix(64, 32, i).to(DEV) for i in range(5)]
    want = e2f.e2f_orthogonalize(ctx, g)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        got = e2f.e2f_orthogonalize(ctx, g)
    again = e2f.e2f_orthogonalize(ctx, g)
    torch.cuda.current_stream().wait_stream(s)
    assert all(torch.equal(a, b) and torch.equal(a, c) for a, b, c in zip(want, got, again))


def test_refused_by_the_binding(e2f, ctx):
    g = [torch.zeros(4, 6, device=DEV)]
    flat, other = torch.zeros(49, device=DEV), torch.zeros(5, 5, device=DEV)
    for bad in (lambda: e2f.e2f_orthogonalize(ctx, [g[0].half()]), lambda: e2f.e2f_orthogonalize(ctx, [g[0].t()]),
                lambda: e2f.e2f_orthogonalize(ctx, [g[0].cpu()]), lambda: e2f.e2f_orthogonalize(ctx, [g[0][0]]),
                lambda: e2f.e2f_orthogonalize(ctx, [g[0], g[0].bfloat16()]),
                lambda: e2f.e2f_orthogonalize(ctx, g, outs=[]), lambda: e2f.e2f_orthogonalize(ctx, g, outs=[torch.zeros(6, 4, device=DEV)]),
                lambda: e2f.e2f_orthogonalize(ctx, g, new_moments=[torch.zeros(4, 6, device=DEV)]),
                lambda: e2f.e2f_orthogonalize(ctx, g, moments=[g[0].bfloat16()]),
                lambda: e2f.e2f_orthogonalize(ctx, g, weights=[g[0].bfloat16()], outs=[torch.zeros(4, 6, device=DEV)]),
                # (of matrices of two sizes)
                lambda: e2f.e2f_orthogonalize(ctx, [flat[:24].view(4, 6), flat[24:].view(5, 5)], outs=[flat[20:44].view(4, 6), other]),
                lambda: e2f.e2f_orthogonalize(ctx, [g[0], other], outs=[flat[:24].view(4, 6), flat[23:48].view(5, 5)]),
                lambda: e2f.e2f_orthogonalize(ctx, g, coefs=(1.0, 2.0)), lambda: e2f.e2f_orthogonalize(ctx, g, coefs=[(1, 0, 0)] * 4)):
        with pytest.raises(ValueError):
            bad()
    for bad in (lambda: e2f.e2f_orthogonalize(ctx, g, outs=g), lambda: e2f.e2f_orthogonalize(ctx, g, decay=0.5),
                lambda: e2f.e2f_orthogonalize(ctx, g, steps=-1), lambda: e2f.e2f_orthogonalize(ctx, g, coefs=(9.0, 0.0, 0.0)),
                lambda: e2f.e2f_orthogonalize(ctx, [torch.zeros(200, 300, device=DEV)], workspace=torch.empty(256, dtype=torch.uint8, device=DEV))):
        with pytest.raises(e2f.E2FError):
            bad()
