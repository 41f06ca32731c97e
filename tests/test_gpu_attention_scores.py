"""Capped attention where scores are infinite, large, far apart or saturated, against float64.  Atoms at one point have
an envelope of 1 and, without radial functions, scores that are exact by their construction: what is left are the
roundings of the softmax itself, counted at each bound.  Run with -m gpu."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
U = 2.0 ** -24


@pytest.fixture(scope="module")
def e2f():
    import paper_2501_19216_amd as m
    return m


@pytest.fixture(scope="module")
def ctx(e2f):
    c = e2f.e2f_create(0, 0)
    yield c
    c.close()


def stars(receivers, degree):
    """Rows of `degree` edges from senders of their own, which come behind the receivers: edge e is sent by receivers + e."""
    E = receivers * degree
    rp = torch.cat([torch.arange(receivers + 1) * degree, torch.full((E,), E)])
    return receivers + E, rp.to(DEV), (receivers + torch.arange(E)).int().to(DEV)


def from_scores(x, receivers):
    """q [n, H, 1] of ones and k [n, H, 1] of the edges' scores x [E, H]."""
    H = x.shape[1]
    q = torch.ones(receivers + x.shape[0], H, 1, device=DEV)
    return q, torch.cat([torch.zeros(receivers, H), x]).view(-1, H, 1).to(DEV)


# a lane of eight heads takes every eighth edge, of four waves a row every 32nd: the first and last edges are single
# ones of their lanes, and 300 edges pass the 128 whose scores stay in the LDS
@pytest.mark.parametrize("receivers,degree", [(40, 1), (40, 5), (40, 8), (40, 64), (9, 200), (3, 300), (1, 3000)])
@pytest.mark.parametrize("H", [1, 8, 12])
def test_scores_of_minus_infinity(e2f, ctx, receivers, degree, H):
    g = torch.Generator().manual_seed(degree + H)
    n, rp, ci = stars(receivers, degree)
    x = torch.randn(receivers * degree, H, generator=g).view(receivers, degree, H)
    r = torch.arange(receivers)
    x[r % 5 == 0, 0] = -math.inf
    x[r % 5 == 1, -1] = -math.inf
    x[r % 5 == 2, degree // 2:] = -math.inf
    x[r % 5 == 3, :, 0] = -math.inf  # all of one head's, which leave the others alone
    x = x.reshape(-1, H)
    q, k = from_scores(x, receivers)
    pos = torch.zeros(n, 3, device=DEV)
    alpha, lse = e2f.e2f_attention_forward(ctx, pos, rp, ci, 5.0, q=q, k=k)
    s = x.double().view(receivers, degree, H)
    want, total = torch.softmax(s, 1), torch.logsumexp(s, 1)  # (NaN and -infinity where all are -infinity)
    got = alpha.cpu().double().view(receivers, degree, H)
    assert torch.equal(got.isnan(), want.isnan())
    assert torch.equal(lse.cpu().double()[:receivers] == -math.inf, total == -math.inf)
    fine = ~want.isnan()
    # exponentials of up to 10 and their sum, at most degree / 8 terms and eight more in a chain; lse's own rounding
    room = U * (degree / 4 + 80)
    assert torch.all((got - want)[fine].abs() <= room * want[fine] + 1e-37)
    assert torch.all(got[fine & (s == -math.inf)] == 0)
    some = total != -math.inf
    assert torch.all((lse.cpu().double()[:receivers] - total)[some].abs() <= room * (1 + total[some].abs()))


@pytest.mark.parametrize("receivers,degree", [(40, 5), (9, 200), (1, 3000)])
def test_gradients_beside_scores_of_minus_infinity(e2f, ctx, receivers, degree):
    # products that overflow: q and k are finite, so every gradient is, and that of such a score is 0
    g = torch.Generator().manual_seed(degree)
    n, rp, ci = stars(receivers, degree)
    E, H = receivers * degree, 4
    x = torch.randn(E, H, generator=g)
    x[::3] = -3e38
    q, k = from_scores(x, receivers)
    ga = torch.randn(E, H, generator=g).to(DEV)
    pos = torch.zeros(n, 3, device=DEV)
    alpha, lse = e2f.e2f_attention_forward(ctx, pos, rp, ci, 5.0, q=q, k=k, scale=16.0)
    t = e2f.e2f_transpose_graph(ctx, n, rp, ci)
    gq, gk, _, gp = e2f.e2f_attention_backward(ctx, pos, rp, ci, 5.0, alpha, lse, ga, *t, q=q, k=k, scale=16.0)
    assert torch.isfinite(alpha).all() and torch.all(alpha[::3] == 0)
    assert torch.isfinite(gk).all() and torch.all(gk[receivers::3] == 0) and torch.all(gp == 0)
    p = torch.softmax((16.0 * x.double()).masked_fill(x.double() < -1e38, -math.inf).view(receivers, degree, H), 1)
    a = ga.cpu().double().view(receivers, degree, H)
    D = (p * a).sum(1, keepdim=True)
    want = 16.0 * p * (a - D)
    # scores of up to 16 * 4, once rounded, in the weights and in lse; the sums of a row
    room = U * (degree / 4 + 80 + 4 * 64) * 16.0 * p * (a.abs() + (p * a.abs()).sum(1, keepdim=True)) + 1e-36
    got = gk[receivers:].cpu().double().view(receivers, degree, H)
    assert torch.all((got - want).abs() <= room)


# Roundings of a weight of few edges, in steps U of itself: the exponential 3 (the instruction's last place is two), a
# lane's sum of four 3, its rescaling to the row's maximum 4, sums over lanes and waves 8, the quotient's two
# factors 2, the exponential in front 3: 23, and the envelope of 1
FEW = 24


@pytest.mark.parametrize("offset", [0.0, 100.0, 1000.0, 10000.0, -10000.0])
@pytest.mark.parametrize("H,degree", [(1, 200), (8, 20), (8, 32), (12, 7), (3, 129)])
def test_one_offset_of_a_row_s_scores_does_not_change_its_weights(e2f, ctx, offset, H, degree):
    # scores offset + m / 64: exact, as are their differences, which are below 1/2 (the exponential's argument to
    # the base of two stays below 1, whose rounding is half a step of the result at most)
    receivers = 20
    g = torch.Generator().manual_seed(degree)
    n, rp, ci = stars(receivers, degree)
    x = offset + torch.randint(0, 32, (receivers * degree, H), generator=g) / 64
    q, k = from_scores(x, receivers)
    alpha, _ = e2f.e2f_attention_forward(ctx, torch.zeros(n, 3, device=DEV), rp, ci, 5.0, q=q, k=k)
    want = torch.softmax(x.double().view(receivers, degree, H), 1)
    got = alpha.cpu().double().view(receivers, degree, H)
    steps = float(((got - want).abs() / want).max()) / U
    print("%.1f steps" % steps)
    assert steps <= FEW + degree / 32


@pytest.mark.parametrize("H,degree", [(8, 20), (8, 32), (12, 7), (4, 60)])
def test_scores_far_below_the_largest_keep_their_digits(e2f, ctx, H, degree):
    # scores m / 64 down to -80: exact; a lane sees four edges at most, in one step. The exponential holds three
    # half steps however far its argument is
    receivers = 50
    g = torch.Generator().manual_seed(degree)
    n, rp, ci = stars(receivers, degree)
    x = -torch.randint(0, 80 * 64, (receivers * degree, H), generator=g) / 64
    q, k = from_scores(x, receivers)
    alpha, _ = e2f.e2f_attention_forward(ctx, torch.zeros(n, 3, device=DEV), rp, ci, 5.0, q=q, k=k)
    want = torch.softmax(x.double().view(receivers, degree, H), 1)
    got = alpha.cpu().double().view(receivers, degree, H)
    steps = float(((got - want).abs() / want).max()) / U
    print("%.1f steps" % steps)
    assert steps <= FEW


def test_capped_scores_alone(e2f, ctx):
    # one edge a row: lse is its score. cap 2^4, so that x / cap is exact; the hyperbolic tangent by exponentials: e to 3
    # half steps, 2 e / (1 - e^2) < 1.32 times that, a difference, a sum and two for the quotient, and the product
    # with cap: 9; by its series fewer
    receivers, H, cap = 4000, 8, 16.0
    g = torch.Generator().manual_seed(1)
    n, rp, ci = stars(receivers, 1)
    x = torch.exp(torch.rand(receivers, H, generator=g) * 14 - 8) * (torch.randint(0, 2, (receivers, H), generator=g) * 2 - 1)
    q, k = from_scores(x, receivers)
    alpha, lse = e2f.e2f_attention_forward(ctx, torch.zeros(n, 3, device=DEV), rp, ci, 5.0, q=q, k=k, cap=cap)
    want = cap * torch.tanh(x.double() / cap)
    steps = float(((lse[:receivers].cpu().double() - want).abs() / want.abs()).max()) / U
    print("%.1f steps" % steps)
    assert steps <= 9 and torch.all(alpha == 1.0)


def gradient_of_scores(x, env, ga, receivers, degree):
    """ds [receivers, degree, H] in float64, and what ten operations after the weights may add to it: those have FEW
    roundings and the envelope 20 steps of 1 (its argument's, its series' and its square's); the sum over the row
    degree / 4 more; the core, p and ds two each."""
    p = torch.softmax(x.double().view(receivers, degree, -1), 1)
    a = ga.cpu().double().view(receivers, degree, -1)
    e = env.double().view(receivers, degree, 1)
    D = (p * e * a).sum(1, keepdim=True)
    bD = U * ((p * a.abs() * ((FEW + degree / 4 + 12) * e + 20)).sum(1, keepdim=True) + 2 * D.abs())
    ds = p * (e * a - D)
    return p, ds, p * (U * (20 * a.abs() + 2 * (e * a - D).abs()) + bD) + U * (FEW + 8) * ds.abs() + 1e-36


@pytest.mark.parametrize("offset", [0.0, 100.0, 1000.0, 10000.0, -10000.0])
@pytest.mark.parametrize("H,degree", [(1, 200), (8, 20), (12, 7), (4, 60)])
@pytest.mark.parametrize("apart", [False, True])
def test_gradients_at_one_offset_of_a_row_s_scores(e2f, ctx, offset, H, degree, apart):
    # the gradient of an edge's k is that of its score; with `apart` the senders lie between the receiver and the
    # cutoff, some of them next to it, and every seventh beyond it
    receivers, rc = 20, 5.0
    g = torch.Generator().manual_seed(degree + H)
    n, rp, ci = stars(receivers, degree)
    E = receivers * degree
    x = offset + torch.randint(0, 32, (E, H), generator=g) / 64
    q, k = from_scores(x, receivers)
    pos, env, beyond = torch.zeros(n, 3), torch.ones(E), torch.zeros(E, dtype=torch.bool)
    if apart:
        d = (rc * (1 - torch.exp(-16 * torch.rand(E, generator=g)))).float()  # down to 10^-7 from the cutoff
        beyond = torch.arange(E) % 7 == 3
        d[beyond] = 5.5
        pos[receivers:, 0] = d
        env = torch.where(d < rc, torch.cos(math.pi / 2 * d.double() / rc) ** 2, 0.0)
    pos = pos.to(DEV)
    ga = torch.randn(E, H, generator=g).to(DEV)
    alpha, lse = e2f.e2f_attention_forward(ctx, pos, rp, ci, rc, q=q, k=k)
    t = e2f.e2f_transpose_graph(ctx, n, rp, ci)
    _, gk, _, _ = e2f.e2f_attention_backward(ctx, pos, rp, ci, rc, alpha, lse, ga, *t, q=q, k=k)
    p, want, room = gradient_of_scores(x, env, ga, receivers, degree)
    # without a weight p is exp(x - lse): half a step of lse and of the difference
    beyond = beyond.view(receivers, degree, 1)
    room = room + U * want.abs() * torch.where(beyond, 2 * lse.cpu().double()[:receivers, None].abs(), 0.0)
    got = gk[receivers:].cpu().double().view(receivers, degree, H)
    worst = float(((got - want).abs() / room).max())
    print("%.3f of the bound" % worst)
    assert worst <= 1.0


@pytest.mark.parametrize("cap", [1.0, 16.0])
@pytest.mark.parametrize("largest", [0.3, 2.0, 8.0, 30.0])
def test_gradients_of_capped_scores(e2f, ctx, cap, largest):
    # x / cap exact; 1 - tanh^2 as 4 e / (1 + e)^2: e to three half steps, its sum and square two, the quotient three
    # (by 1 - t^2 below 0.35: less). p holds cap times nine half steps of the score, twice (test_capped_scores_alone)
    receivers, degree, H = 30, 20, 8
    g = torch.Generator().manual_seed(int(cap + 10 * largest))
    n, rp, ci = stars(receivers, degree)
    E = receivers * degree
    x = torch.randint(-4096, 4097, (E, H), generator=g) * (cap * largest / 4096)
    q, k = from_scores(x, receivers)
    ga = torch.randn(E, H, generator=g).to(DEV)
    pos = torch.zeros(n, 3, device=DEV)
    alpha, lse = e2f.e2f_attention_forward(ctx, pos, rp, ci, 5.0, q=q, k=k, cap=cap)
    t = e2f.e2f_transpose_graph(ctx, n, rp, ci)
    _, gk, _, _ = e2f.e2f_attention_backward(ctx, pos, rp, ci, 5.0, alpha, lse, ga, *t, q=q, k=k, cap=cap)
    z = x.double() / cap
    e = torch.exp(-2 * z.abs())
    turn = (4 * e / (1 + e) ** 2).view(receivers, degree, H)
    p, ds, room = gradient_of_scores(cap * torch.tanh(z), torch.ones(E), ga, receivers, degree)
    a = ga.cpu().double().view(receivers, degree, H)
    pa = (p * a.abs()).sum(1, keepdim=True)
    room = room + U * 18 * cap * p * (a.abs() + 2 * pa)
    want = ds * turn
    got = gk[receivers:].cpu().double().view(receivers, degree, H)
    worst = float(((got - want).abs() / (room * turn + U * 12 * want.abs() + 1e-36)).max())
    print("%.3f of the bound" % worst)
    assert worst <= 1.0


def test_gradients_over_inputs_are_refused(e2f, ctx):
    # an array for everything that the backward reads and writes; nothing is launched where an output overlaps
    import ctypes
    n, H, dk, R, E = 10, 4, 8, 8, 30
    prm = e2f.AttentionParams(H, H, dk, R, 5.0, 0.3, 10.0, 0, 0, 0)
    need = ctypes.c_size_t(0)
    assert e2f.lib.e2f_attention_backward_workspace_size(ctx.handle, ctypes.byref(prm), n, E, ctypes.byref(need)) == 0
    size = dict(pos=12 * n, gid=4 * n, q=4 * n * H * dk, k=4 * n * H * dk, w=4 * H * R, rp=8 * (n + 1), ci=4 * E,
                rt=8 * (n + 1), ct=4 * E, pm=4 * E, alpha=4 * E * H, lse=4 * n * H, ga=4 * E * H)
    out = dict(gq=4 * n * H * dk, gk=4 * n * H * dk, gw=4 * H * R, gp=12 * n)
    space = torch.zeros((len(size) + len(out)) * 8192 + need.value, dtype=torch.uint8, device=DEV)
    base, at = {}, space.data_ptr()
    for name in (*size, *out):
        base[name] = at
        at += 8192
    base["ws"] = at

    def call(**kw):
        v = {**base, **kw}
        p = [v[x] for x in ("pos", "gid", "q", "k")] + [n] + [v[x] for x in ("w", "rp", "ci")] + [E]
        p += [v[x] for x in ("rt", "ct", "pm", "alpha", "lse", "ga", "gq", "gk", "gw", "gp", "ws")]
        return e2f.lib.e2f_attention_backward(ctx.handle, ctypes.byref(prm), *p, need.value, None)

    assert call() == e2f.E2F_OK  # (a graph without edges: rp is all 0)
    torch.cuda.synchronize()
    for o, mine in out.items():
        for i, its in size.items():
            for where in (base[i], base[i] + its - 4, base[i] - mine + 4):
                assert call(**{o: where}) == e2f.E2F_EINVAL, (o, i)
    assert call(gq=base["gk"] + 4 * n * H * dk - 4) == e2f.E2F_EINVAL
    assert call(gp=base["ws"] + 128) == e2f.E2F_EINVAL and call(ws=base["q"] // 256 * 256) == e2f.E2F_EINVAL
