"""The norms around a block, its gate and residual sum, and their gradients
against float64, elementwise within bounds on float32 arithmetic.  Run with
-m gpu."""
import math

import pytest
import torch

import block_reference as ref

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.fixture(scope="module")
def e2f():
    import paper_2501_19216_amd as m
    return m


@pytest.fixture(scope="module")
def ctx(e2f):
    c = e2f.e2f_create(0, 0)
    yield c
    c.close()


def inputs(n, L, C, gates, dtype, seed, post=True, scale=True, pre=True, block=True):
    g = torch.Generator().manual_seed(seed)
    K = (L + 1) ** 2
    r = lambda *s: torch.randn(*s, generator=g)  # noqa: E731
    v = dict(x=(2 * r(n, K, C)).to(dtype), block=(r(n, K, C) * torch.exp(r(n, 1, 1))).to(dtype) if block else None,
             gate=(2 * r(n, gates, C)).to(dtype) if gates else None, post_w=1 + 0.3 * r(L + 1, C) if post else None,
             res_scale=r(L + 1, C) if scale else None, pre_w=1 + 0.3 * r(L + 1, C) if pre else None)
    return v, r(n, K, C).to(dtype), r(n, K, C).to(dtype) if pre else None


def run(e2f, ctx, v, L, g_out=None, g_normed=None, eps=1e-5, back=True):
    d = {name: None if t is None else t.to(DEV) for name, t in v.items()}
    out, normed, rstd = e2f.e2f_block_norm_forward(ctx, d["x"], L, *list(d.values())[1:], eps=eps)
    got = {"normed": normed, "rstd": rstd}
    if d["block"] is not None:
        got["out"] = out
    if back:
        up = lambda t: None if t is None else t.to(DEV)  # noqa: E731
        names = ("grad_x", "grad_block", "grad_gate", "grad_post_w", "grad_scale", "grad_pre_w")
        got.update(zip(names, e2f.e2f_block_norm_backward(ctx, d["x"], rstd, L, *list(d.values())[1:], eps=eps,
                                                          grad_out=up(g_out), grad_normed=up(g_normed))))
    return got


def compare(got, want, dtype):
    for name, r in want.items():
        low = name in ("out", "normed", "grad_x", "grad_block", "grad_gate")
        ref.check(got[name], r, dtype if low else torch.float32, name)
    for name, t in got.items():
        assert (t is None) == (name not in want), name


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("L,C,gates,n", [
    (0, 4, 0, 1), (0, 4, 1, 700), (0, 8, 1, 3), (0, 100, 1, 65), (0, 256, 0, 33), (0, 516, 1, 9), (0, 1024, 1, 70),
    (1, 4, 2, 5), (1, 12, 1, 129), (1, 64, 2, 40), (1, 300, 1, 17), (1, 1024, 2, 6), (2, 16, 1, 32), (2, 48, 3, 77),
    (2, 128, 0, 30), (2, 1024, 3, 5), (3, 4, 4, 9), (3, 64, 4, 61), (3, 132, 1, 21), (3, 640, 4, 5),
    (4, 20, 5, 31), (4, 128, 5, 50), (4, 260, 1, 7), (4, 1024, 5, 3), (5, 32, 6, 19), (5, 96, 0, 25), (5, 520, 6, 3),
    (6, 4, 1, 13), (6, 64, 7, 29), (6, 128, 7, 10), (6, 512, 7, 3), (6, 1024, 1, 2)])
def test_shapes(e2f, ctx, L, C, gates, n, dtype):
    v, g_out, g_normed = inputs(n, L, C, gates, dtype, 1000 * L + C + n)
    got = run(e2f, ctx, v, L, g_out, g_normed)
    compare(got, ref.block_norm(**v, L=L, g_out=g_out, g_normed=g_normed, grads=True), dtype)


@pytest.mark.parametrize("L,C", [(0, 64), (2, 32), (4, 128), (4, 512)])
@pytest.mark.parametrize("kw", [dict(post=False, scale=False), dict(pre=False), dict(scale=False), dict(post=False),
                                dict(block=False, post=False, scale=False), dict(post=False, scale=False, pre=False)])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_parts_left_out(e2f, ctx, L, C, kw, dtype):
    gates = 0 if kw.get("block") is False else L + 1
    v, g_out, g_normed = inputs(37, L, C, gates, dtype, C + L, **kw)
    got = run(e2f, ctx, v, L, g_out, g_normed)
    compare(got, ref.block_norm(**v, L=L, g_out=g_out, g_normed=g_normed, grads=True), dtype)


@pytest.mark.parametrize("with_out,with_normed", [(True, False), (False, True), (False, False)])
def test_gradients_left_out(e2f, ctx, with_out, with_normed):
    v, g_out, g_normed = inputs(20, 2, 24, 3, torch.float32, 3)
    g_out, g_normed = g_out if with_out else None, g_normed if with_normed else None
    got = run(e2f, ctx, v, 2, g_out, g_normed)
    compare(got, ref.block_norm(**v, L=2, g_out=g_out, g_normed=g_normed, grads=True), torch.float32)


def test_two_dimensional_activations(e2f, ctx):
    v, g_out, g_normed = inputs(50, 0, 96, 1, torch.float32, 9)
    a = run(e2f, ctx, v, 0, g_out, g_normed)
    flat = {name: t if t is None or t.dim() < 3 else t[:, 0] for name, t in v.items()}
    b = run(e2f, ctx, flat, 0, g_out[:, 0], g_normed[:, 0])
    for name in a:
        assert torch.equal(a[name].reshape(-1), b[name].reshape(-1)), name


def test_no_atoms(e2f, ctx):
    v, g_out, g_normed = inputs(0, 2, 16, 1, torch.float32, 9)
    got = run(e2f, ctx, v, 2, g_out, g_normed)
    assert got["out"].numel() == 0
    for name in ("grad_post_w", "grad_scale", "grad_pre_w"):
        assert torch.all(got[name] == 0)


def test_zero_rows_large_rows_and_rows_not_finite(e2f, ctx):
    L, C, n = 2, 20, 12
    v, g_out, g_normed = inputs(n, L, C, 3, torch.float32, 5)
    v["block"][3] = 0.0
    v["x"][4], v["block"][4] = 0.0, 0.0  # rms = sqrt(eps)
    v["x"][5] *= 1e15                     # squares of 10^30
    v["gate"][6], v["gate"][7] = 90.0, -90.0  # gates wholly open and shut
    got = run(e2f, ctx, v, L, g_out, g_normed)
    compare(got, ref.block_norm(**v, L=L, g_out=g_out, g_normed=g_normed, grads=True), torch.float32)
    # what is not finite stays in its row (the weights' gradients sum over rows)
    for value in (math.inf, math.nan):
        bad = {name: None if t is None else t.clone() for name, t in v.items()}
        bad["block"][8, 3, 2] = value
        other = run(e2f, ctx, bad, L, g_out, g_normed)
        rows = torch.arange(n, device=DEV) != 8
        for name in ("out", "normed", "grad_x", "grad_block", "grad_gate", "rstd"):
            assert torch.equal(other[name][rows], got[name][rows]), name
        assert not torch.isfinite(other["out"][8]).all()


def test_addresses_of_any_alignment(e2f, ctx):
    # arrays that begin one element past an aligned address
    L, C, n = 1, 12, 30
    for dtype in (torch.float32, torch.bfloat16):
        v, g_out, g_normed = inputs(n, L, C, 2, dtype, 6)
        want = run(e2f, ctx, v, L, g_out, g_normed)

        def shifted(t):
            buf = torch.empty(t.numel() + 1, dtype=t.dtype, device=DEV)
            return buf[1:].copy_(t.reshape(-1)).view(t.shape)

        d = [None if t is None else shifted(t.to(DEV)) for t in v.values()]
        out, normed = (shifted(torch.zeros_like(v["x"])) for _ in range(2))
        out, normed, rstd = e2f.e2f_block_norm_forward(ctx, d[0], L, *d[1:], out=out, normed=normed)
        grads = e2f.e2f_block_norm_backward(ctx, d[0], rstd, L, *d[1:], grad_out=shifted(g_out.to(DEV)),
                                            grad_normed=shifted(g_normed.to(DEV)))
        for a, name in zip((out, normed, rstd, *grads), ("out", "normed", "rstd", "grad_x", "grad_block", "grad_gate",
                                                          "grad_post_w", "grad_scale", "grad_pre_w")):
            assert torch.equal(a, want[name]), name


@pytest.mark.parametrize("L,C", [(0, 256), (3, 64), (4, 128), (4, 512)])
def test_deterministic_captured_and_on_another_stream(e2f, ctx, L, C):
    n = 3000
    v, g_out, g_normed = inputs(n, L, C, L + 1, torch.float32, 8)
    d = [t.to(DEV) for t in v.values()]
    gs = dict(grad_out=g_out.to(DEV), grad_normed=g_normed.to(DEV))
    space = torch.empty(64 << 20, dtype=torch.uint8, device=DEV)

    def step():
        out, normed, rstd = e2f.e2f_block_norm_forward(ctx, d[0], L, *d[1:])
        return [out, normed, rstd, *e2f.e2f_block_norm_backward(ctx, d[0], rstd, L, *d[1:], workspace=space, **gs)]

    first = step()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        again = step()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(first, again))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step()
    for r in range(3):
        d[0].mul_(1.0 if r == 0 else 0.9)
        graph.replay()
        torch.cuda.synchronize()
        space.fill_(255)
        want = step()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, want)), r


def test_beyond_2_to_the_31_values(e2f, ctx):
    # offsets that pass 32 bits: the last rows of 2.2e9 bfloat16 values
    L, C = 6, 64
    n = 700000
    g = torch.Generator(device=DEV).manual_seed(2)
    x = torch.empty(n, 49, C, dtype=torch.bfloat16, device=DEV).normal_(generator=g)
    w = torch.rand(L + 1, C, device=DEV, generator=g) + 0.5
    _, normed, rstd = e2f.e2f_block_norm_forward(ctx, x, L, pre_w=w)
    gx, _, _, _, _, _ = e2f.e2f_block_norm_backward(ctx, x, rstd, L, pre_w=w, grad_normed=x, want_weights=False)
    last = x[-3:].cpu()
    want = ref.block_norm(last, L, pre_w=w.cpu(), g_normed=last, grads=True)
    ref.check(normed[-3:], want["normed"], torch.bfloat16, "normed")
    ref.check(gx[-3:], want["grad_x"], torch.bfloat16, "grad_x")


def test_gradients_against_differences(e2f, ctx):
    L, C, n = 2, 8, 6
    v, g_out, g_normed = inputs(n, L, C, 3, torch.float32, 12)
    got = run(e2f, ctx, v, L, g_out, g_normed)
    g = torch.Generator().manual_seed(1)

    def f(values):
        r = ref.block_norm(**values, L=L)
        return float((r["out"][0] * g_out.double()).sum() + (r["normed"][0] * g_normed.double()).sum())

    base = {name: t.double() for name, t in v.items()}
    h = 1e-5
    for name, out in (("x", "grad_x"), ("block", "grad_block"), ("gate", "grad_gate"), ("post_w", "grad_post_w"),
                      ("res_scale", "grad_scale"), ("pre_w", "grad_pre_w")):
        d = torch.randn(base[name].shape, generator=g, dtype=torch.float64)
        num = (f({**base, name: base[name] + h * d}) - f({**base, name: base[name] - h * d})) / (2 * h)
        mine = got[out].cpu().double()
        # differences: h^2 times a third derivative, and 2^-53 / h of the sum; float32: some 10^2 half steps
        assert abs(num - float((mine * d).sum())) <= float((mine.abs() * d.abs()).sum()) * (1e-6 + 1e-4), name
