"""What one graph's atoms hold does not reach another graph's outputs: a wave takes many rows after each other, with a
head group of any size.  Run with -m gpu."""
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


def step(e2f, ctx, pos, rp, ci, t, gid, q, k, w, ga, cap):
    kw = dict(q=q, k=k, rbf_w=w, scale=0.3, cap=cap, graph_id=gid)
    alpha, lse = e2f.e2f_attention_forward(ctx, pos, rp, ci, 6.0, **kw)
    gq, gk, _, gp = e2f.e2f_attention_backward(ctx, pos, rp, ci, 6.0, alpha, lse, ga, *t, **kw)
    return dict(alpha=alpha, lse=lse, grad_q=gq, grad_k=gk, grad_pos=gp)


# graphs of `size` atoms, every pair of a graph listed and each atom with the one behind it in the next graph; rows
# short (a wave a row) and of more than 256 edges (four waves); no whole number of graphs for a workgroup, so that a
# wave has rows of several
@pytest.mark.parametrize("n,size", [(7700, 11), (2709, 301)])
@pytest.mark.parametrize("H,Hk,dk,dtype", [(6, 6, 8, torch.float32), (6, 2, 20, torch.float32), (1, 1, 4, torch.float32),
                                           (3, 3, 8, torch.bfloat16), (7, 7, 5, torch.float32), (18, 18, 8, torch.float32),
                                           (8, 8, 16, torch.float32)])
@pytest.mark.parametrize("masked", [False, True])
def test_positions_that_are_not_finite(e2f, ctx, n, size, H, Hk, dk, dtype, masked):
    g = torch.Generator().manual_seed(n + H)
    atom = torch.arange(n)
    first = atom // size * size
    j = first[:, None] + torch.arange(size)
    keep = j != atom[:, None]
    ci = j[keep].view(n, size - 1)
    if masked:
        ci = torch.cat([ci, ((atom + size) % n)[:, None]], dim=1).sort(dim=1).values
    deg = ci.shape[1]
    rp, ci = (torch.arange(n + 1) * deg).to(DEV), ci.reshape(-1).int().to(DEV)
    gid = (atom // size).int().to(DEV) if masked else None
    pos = (torch.rand(n, 3, generator=g) * 5).to(DEV)
    q, k = (torch.randn(n, h, dk, generator=g).to(dtype).to(DEV) for h in (H, Hk))
    w, ga = torch.randn(H, 8, generator=g).to(DEV), torch.randn(n * deg, H, generator=g).to(DEV)
    t = e2f.e2f_transpose_graph(ctx, n, rp, ci)
    want = step(e2f, ctx, pos, rp, ci, t, gid, q, k, w, ga, 5.0)
    graph = atom // size
    for value in (math.inf, math.nan):
        bad = (graph % 5 == 0).to(DEV)  # the first graph and every fifth: the waves' rows lie among them
        pos2 = pos.clone()
        pos2[bad] = value
        got = step(e2f, ctx, pos2, rp, ci, t, gid, q, k, w, ga, 5.0)
        for name, v in got.items():
            rows = ~bad.repeat_interleave(deg) if name == "alpha" else ~bad
            # nothing that these rows are made of has changed: the same bits
            assert torch.equal(v[rows], want[name][rows]), name


@pytest.mark.parametrize("H,dk,R", [(4, 8, 8), (6, 0, 32), (6, 4, 2)])
@pytest.mark.parametrize("far", [1e15, 1e19, 1e20, 3e38])
def test_atoms_parked_far_away(e2f, ctx, H, dk, R, far):
    # finite positions whose distances' squares, or distances, are beyond float32: no envelope, no radial function and
    # no force, but a place among the scores
    n, degree = 300, 20
    g = torch.Generator().manual_seed(H)
    pos = torch.rand(n, 3, generator=g) * 6
    pos[::7] = torch.tensor([far, -far, 0.5 * far])
    pos[3::7, 1] = -far
    send = torch.stack([torch.randperm(n - 1, generator=g)[:degree].sort().values for _ in range(n)])
    send = send + (send >= torch.arange(n)[:, None])
    rp, ci = torch.arange(n + 1) * degree, send.reshape(-1).int()
    q, k = (torch.randn(n, H, dk, generator=g) if dk else None for _ in range(2))
    w, ga = torch.randn(H, R, generator=g), torch.randn(n * degree, H, generator=g)
    want = ref.attention(pos, rp, ci, 6.0, q, k, w, H, 0.4, 5.0, None, ga)
    up = lambda t: None if t is None else t.to(DEV)  # noqa: E731
    t = e2f.e2f_transpose_graph(ctx, n, up(rp), up(ci))
    kw = dict(q=up(q), k=up(k), rbf_w=up(w), scale=0.4, cap=5.0)
    alpha, lse = e2f.e2f_attention_forward(ctx, up(pos), up(rp), up(ci), 6.0, **kw)
    gq, gk, gw, gp = e2f.e2f_attention_backward(ctx, up(pos), up(rp), up(ci), 6.0, alpha, lse, up(ga), *t, **kw)
    got = dict(alpha=alpha, lse=lse, grad_w=gw, grad_pos=gp, **(dict(grad_q=gq, grad_k=gk) if dk else {}))
    for name, v in got.items():
        ref.check(v, want[name], name=name)


@pytest.mark.parametrize("H,Hk,dk,dtype", [(6, 6, 8, torch.float32), (6, 2, 20, torch.float32),
                                           (8, 8, 16, torch.bfloat16), (16, 4, 5, torch.bfloat16)])
@pytest.mark.parametrize("cap", [0.0, 5.0])
def test_features_and_gradients_that_are_not_finite(e2f, ctx, H, Hk, dk, dtype, cap):
    # graphs of eleven atoms without an edge between them: a wave's rows before hold NaN and infinities
    n, size = 7700, 11
    g = torch.Generator().manual_seed(H + dk)
    atom = torch.arange(n)
    j = (atom // size * size)[:, None] + torch.arange(size)
    ci = j[j != atom[:, None]].view(n, size - 1).reshape(-1).int().to(DEV)
    rp = (torch.arange(n + 1) * (size - 1)).to(DEV)
    pos = (torch.rand(n, 3, generator=g) * 5).to(DEV)
    q, k = (torch.randn(n, h, dk, generator=g).to(dtype).to(DEV) for h in (H, Hk))
    w, ga = torch.randn(H, 8, generator=g).to(DEV), torch.randn(ci.numel(), H, generator=g).to(DEV)
    t = e2f.e2f_transpose_graph(ctx, n, rp, ci)
    want = step(e2f, ctx, pos, rp, ci, t, None, q, k, w, ga, cap)
    bad = (atom // size % 5 == 0).to(DEV)
    for what in ("q", "k", "ga"):
        for value in (math.inf, -math.inf, math.nan):
            v = dict(q=q.clone(), k=k.clone(), ga=ga.clone())
            v[what][bad.repeat_interleave(size - 1) if what == "ga" else bad] = value
            got = step(e2f, ctx, pos, rp, ci, t, None, v["q"], v["k"], w, v["ga"], cap)
            for name, x in got.items():
                rows = ~bad.repeat_interleave(size - 1) if name == "alpha" else ~bad
                assert torch.equal(x[rows], want[name][rows]), (what, value, name)
