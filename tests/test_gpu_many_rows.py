"""Calls of more workgroups than one launch holds (2^32 threads), against float64 on rows at the start, about the
border and at the end.  Run with -m gpu."""
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
    torch.cuda.empty_cache()


def test_norm_of_many_rows(e2f, ctx):
    # 516 channels of bfloat16 take a workgroup a row: 2^24 of them are 2^32 threads (17 GB)
    n, C = 2 ** 24 + 5, 516
    g = torch.Generator(device=DEV).manual_seed(1)
    x = torch.empty(n, C, dtype=torch.bfloat16, device=DEV).normal_(generator=g)
    pre = 1 + torch.randn(1, C, device=DEV, generator=g)
    _, normed, rstd = e2f.e2f_block_norm_forward(ctx, x, 0, pre_w=pre)
    rows = torch.tensor([0, 1, 2 ** 23, 2 ** 24 - 2, 2 ** 24 - 1, 2 ** 24, 2 ** 24 + 1, n - 1], device=DEV)
    want = ref.block_norm(x[rows].cpu().view(-1, 1, C), 0, pre_w=pre.cpu())
    ref.check(normed[rows].view(-1, 1, C), want["normed"], torch.bfloat16, "normed")
    ref.check(rstd[rows], want["rstd"], name="rstd")
    # every row was written
    assert float(rstd[:, 1].min()) > 0.8 and float(rstd[:, 1].max()) < 1.3 and bool((rstd[:, 0] == 1).all())


@pytest.mark.parametrize("reverses", [True, False])
def test_attention_of_many_atoms(e2f, ctx, reverses):
    # a wave an atom, four a workgroup: 2^26 atoms are 2^32 threads. Edges among 24 of them, far apart in number
    n, H, dk, R = 2 ** 26 + 77, 2, 4, 4
    atoms = torch.cat([torch.arange(8), torch.arange(2 ** 26 - 4, 2 ** 26 + 4), torch.arange(n - 8, n)])
    m = len(atoms)
    g = torch.Generator().manual_seed(2)
    adjacent = ~torch.eye(m, dtype=torch.bool)
    if not reverses:
        adjacent &= torch.rand(m, m, generator=g) < 0.6
    recv, send = adjacent.nonzero().unbind(1)
    small = torch.cat([torch.zeros(1, dtype=torch.long), adjacent.sum(1).cumsum(0)])
    deg = torch.zeros(n, dtype=torch.long, device=DEV)
    deg[atoms.to(DEV)] = adjacent.sum(1).to(DEV)
    rp = torch.zeros(n + 1, dtype=torch.long, device=DEV)
    torch.cumsum(deg, 0, out=rp[1:])
    ci = atoms[send].int()
    p, q, k = torch.rand(m, 3, generator=g) * 4, torch.randn(m, H, dk, generator=g), torch.randn(m, H, dk, generator=g)
    w, ga = torch.randn(H, R, generator=g), torch.randn(len(send), H, generator=g)

    def spread(t):
        out = torch.zeros(n, *t.shape[1:], device=DEV)
        out[atoms.to(DEV)] = t.to(DEV)
        return out

    pos, q1, k1 = spread(p), spread(q), spread(k)
    kw = dict(q=q1, k=k1, rbf_w=w.to(DEV), scale=0.5, cap=5.0)
    alpha, lse = e2f.e2f_attention_forward(ctx, pos, rp, ci.to(DEV), 6.0, **kw)
    t = e2f.e2f_transpose_graph(ctx, n, rp, ci.to(DEV))
    gq, gk, gw, gp = e2f.e2f_attention_backward(ctx, pos, rp, ci.to(DEV), 6.0, alpha, lse, ga.to(DEV), *t, **kw)
    want = ref.attention(p, small, send.int(), 6.0, q, k, w, H, 0.5, 5.0, None, ga)
    ref.check(alpha, want["alpha"], name="alpha")
    ref.check(gw, want["grad_w"], name="grad_w")
    others = torch.ones(n, dtype=torch.bool, device=DEV)
    others[atoms.to(DEV)] = False
    for name, v, empty in (("lse", lse, -math.inf), ("grad_q", gq, 0.0), ("grad_k", gk, 0.0), ("grad_pos", gp, 0.0)):
        ref.check(v[atoms.to(DEV)], want[name], name=name)
        assert bool((v[others] == empty).all()), name
    order = torch.sort(ci.long(), stable=True).indices
    assert torch.equal(t[2].cpu().long(), order) and torch.equal(t[1].cpu().long(), atoms[recv][order])
    count = torch.zeros(n, dtype=torch.long, device=DEV)
    count[atoms.to(DEV)] = torch.bincount(send, minlength=m).to(DEV)
    assert bool((t[0][1:] == count.cumsum(0)).all()) and int(t[0][0]) == 0


def test_norm_over_many_values(e2f, ctx):
    # 192 times a tensor of 2^33 values, whose chunks are 2^17 workgroups: more than one launch's threads
    t = torch.full((2 ** 33,), 0.5, dtype=torch.bfloat16, device=DEV)
    sumsq, norm = e2f.e2f_grad_norm(ctx, [t] * 192)
    assert float(sumsq) == 192 * 2.0 ** 31  # (every partial sum is a whole number of quarters below 2^53)
    assert abs(float(norm) - math.sqrt(192 * 2.0 ** 31)) <= 2.0 ** -24 * math.sqrt(192 * 2.0 ** 31)
