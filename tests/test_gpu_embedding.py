"""Rows of a table by type and the table's gradient against float64.  Run with -m gpu."""
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


def data(n, V, C, seed, t=F32, index=torch.int32, skew=True, pad=0.0):
    g = torch.Generator().manual_seed(seed)
    table = torch.randn(V, C, generator=g).to(t)
    idx = torch.randint(0, V, (n,), generator=g)
    if skew:  # half of the rows have one type, a quarter another ..
        few = (-torch.log2(torch.rand(n, generator=g).clamp_min(1e-9))).long().clamp_max(V - 1)
        idx = torch.where(torch.rand(n, generator=g) < 0.7, few, idx)
    if pad:
        idx = torch.where(torch.rand(n, generator=g) < pad, torch.full_like(idx, -1), idx)
    return table, idx.to(index), g


def both(e2f, ctx, table, idx, go, L, scale, dt, gdt):
    """go [n, K, C] on the device."""
    V, C = table.shape
    K = (L + 1) ** 2
    out = e2f.e2f_embedding_forward(ctx, table.to(DEV), idx.to(DEV), lmax=L, scale=scale, dtype=dt)
    ref.check(out.view(-1, K, C), ref.embedding(table, idx, K, scale), "out")
    gt = e2f.e2f_embedding_backward(ctx, idx.to(DEV), go, V, lmax=L, scale=scale, dtype=gdt)
    want = ref.embedding_grad(go.view(-1, K, C)[:, 0].cpu(), idx, V, scale)
    ref.check(gt, want, "grad_table")
    absent = torch.bincount(idx.long()[(idx >= 0) & (idx < V)], minlength=V) == 0
    assert bool((gt.cpu()[absent] == 0).all())


@pytest.mark.parametrize("n", [0, 1, 2, 63, 64, 65, 1000, 8192, 8193, 40000])
@pytest.mark.parametrize("V,C", [(1, 1), (5, 16), (100, 64), (255, 7), (256, 128), (300, 36), (70000, 3)])
def test_sizes(e2f, ctx, n, V, C):
    table, idx, g = data(n, V, C, n + V)
    both(e2f, ctx, table, idx, torch.randn(n, 1, C, generator=g).to(DEV).view(n, C), 0, 1.5, F32, F32)


@pytest.mark.parametrize("L", [0, 1, 2, 4, 6])
@pytest.mark.parametrize("table_t,out_t", [(F32, F32), (F32, BF16), (BF16, F32), (BF16, BF16)])
@pytest.mark.parametrize("C", [5, 6, 20, 64, 136])
def test_degrees_and_types(e2f, ctx, L, table_t, out_t, C):
    n, V = 777, 30
    table, idx, g = data(n, V, C, L + C, table_t, torch.int64, pad=0.1)
    both(e2f, ctx, table, idx, torch.randn(n, (L + 1) ** 2, C, generator=g).to(out_t).to(DEV), L, 0.7, out_t, table_t)


@pytest.mark.parametrize("C", [1, 100, 255, 1024, 2000])
@pytest.mark.parametrize("t", [F32, BF16])
def test_wide_rows(e2f, ctx, C, t):
    table, idx, g = data(3000, 1000, C, C, t)
    both(e2f, ctx, table, idx, torch.randn(3000, C, generator=g).to(t).to(DEV), 0, C ** 0.5, t, t)


@pytest.mark.parametrize("n", [100, 20000, 300000])
@pytest.mark.parametrize("kind", ["one", "sorted", "reversed", "runs", "distinct"])
@pytest.mark.parametrize("few", [17, 260])
def test_orders(e2f, ctx, n, kind, few):
    """One type alone; sorted, falling and alternating types; runs that end where stretches do; every type once."""
    V = n if kind == "distinct" else few
    g = torch.Generator().manual_seed(n)
    i = torch.arange(n)
    idx = {"one": torch.full((n,), 11), "sorted": i * V // n, "reversed": (n - 1 - i) * V // n, "runs": i // 64 % V,
           "distinct": torch.randperm(n, generator=g)}[kind].int()
    table = torch.randn(V, 20, generator=g)
    both(e2f, ctx, table, idx, torch.randn(n, 20, generator=g).to(DEV), 0, 1.0, F32, F32)


@pytest.mark.parametrize("n,V,C", [(700, 2000003, 4), (20000, 2000003, 4), (6000001, 50, 2), (2500000, 300, 1)])
def test_large_tables_and_many_rows(e2f, ctx, n, V, C):
    """Types of three digits; more workgroups of the sort than one round of its scan."""
    g = torch.Generator(device=DEV).manual_seed(n)
    idx = torch.randint(0, V, (n,), device=DEV, generator=g)
    go = torch.randn(n, C, device=DEV, generator=g)
    gt = e2f.e2f_embedding_backward(ctx, idx, go, V)
    ref.check(gt, ref.embedding_grad(go.cpu(), idx.cpu(), V, 1.0), "grad_table")


def test_outside_of_the_table(e2f, ctx):
    """Rows with an index outside of the table: zeros forward, and no part in the gradient, whatever they hold."""
    for V, C, t in ((12, 24, torch.int32), (12, 24, torch.int64), (500, 24, torch.int32), (500, 24, torch.int64)):
        far = [-1, -2 ** 31, V, 2 ** 31 - 1] + ([2 ** 32 + 3, -2 ** 40, 2 ** 63 - 1] if t == torch.int64 else [])
        idx = torch.tensor([3, far[0], 0, 11, 11] + far + [3], dtype=t)
        g = torch.randn(len(idx), C)
        inside = (idx >= 0) & (idx < V)
        want = ref.embedding_grad(g, idx, V, 1.0)
        g[~inside] = float("nan")
        table = torch.randn(V, C)
        out = e2f.e2f_embedding_forward(ctx, table.to(DEV), idx.to(DEV))
        ref.check(out[:, None], ref.embedding(table, idx, 1, 1.0), "out")
        assert bool((out.cpu()[~inside] == 0).all())
        ref.check(e2f.e2f_embedding_backward(ctx, idx.to(DEV), g.to(DEV), V), want, "grad_table")
        none = torch.full((500,), -1, dtype=t, device=DEV)
        assert bool((e2f.e2f_embedding_backward(ctx, none, torch.full((500, C), float("nan"), device=DEV), V) == 0).all())


def test_values_that_are_not_finite(e2f, ctx):
    for V in (9, 300):
        check_not_finite(e2f, ctx, V)


def check_not_finite(e2f, ctx, V):
    table, idx, _ = data(400, V, 8, 1, skew=False)
    idx[7] = 4
    table[4, 3] = float("nan")
    table[5, 2] = float("inf")
    out = e2f.e2f_embedding_forward(ctx, table.to(DEV), idx.to(DEV), lmax=1).cpu()
    assert torch.equal(out[:, 0].isnan(), table[idx.long()].isnan()) and torch.equal(out[:, 0].isinf(), table[idx.long()].isinf())
    assert bool((out[:, 1:] == 0).all())
    g = torch.randn(400, 8)
    at = int((idx == 4).nonzero()[0])
    g[at, 1] = float("inf")
    gt = e2f.e2f_embedding_backward(ctx, idx.to(DEV), g.to(DEV), V).cpu()
    assert gt[4, 1] == float("inf") and int(gt.isfinite().sum()) == gt.numel() - 1


@pytest.mark.parametrize("t", [F32, BF16])
def test_rows_further_apart_and_odd_addresses(e2f, ctx, t):
    n, V, C, L = 300, 20, 12, 1
    table, idx, g = data(n, V, C, 5, t)
    wide = torch.full((n, 4 * C + 5), 7.0, dtype=t, device=DEV)
    out = wide[:, 1:1 + 4 * C].unflatten(1, (4, C))
    odd = torch.empty(V * C + 1, dtype=t, device=DEV)[1:].view(V, C).copy_(table)
    e2f.e2f_embedding_forward(ctx, odd, idx.to(DEV), lmax=L, out=out)
    ref.check(out, ref.embedding(table, idx, 4, 1.0), "out")
    assert bool((wide[:, 0] == 7).all()) and bool((wide[:, 1 + 4 * C:] == 7).all())
    go = torch.randn(n, 4 * C + 5, generator=g).to(t).to(DEV)[:, 3:3 + 4 * C].unflatten(1, (4, C))
    gt = torch.empty(V * C + 1, dtype=t, device=DEV)[1:].view(V, C)
    e2f.e2f_embedding_backward(ctx, idx.to(DEV), go, V, lmax=L, grad_table=gt)
    ref.check(gt, ref.embedding_grad(go[:, 0].cpu(), idx, V, 1.0), "grad_table")


@pytest.mark.parametrize("V", [200, 500])
def test_same_bits_every_time_and_on_another_stream(e2f, ctx, V):
    table, idx, g = data(50000, V, 32, 3)
    idx, go = idx.to(DEV), torch.randn(50000, 32, generator=g).to(DEV)
    first = e2f.e2f_embedding_backward(ctx, idx, go, V)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        other = e2f.e2f_embedding_backward(ctx, idx, go, V)
    for _ in range(3):
        assert torch.equal(e2f.e2f_embedding_backward(ctx, idx, go, V), first)
    torch.cuda.current_stream().wait_stream(s)
    assert torch.equal(other, first)


@pytest.mark.parametrize("n,V", [(500, 40), (30000, 40), (500, 400), (30000, 3000)])
def test_captured_and_replayed(e2f, ctx, n, V):
    table, idx, g = data(n, V, 16, n)
    table, idx, go = table.to(DEV), idx.to(DEV), torch.randn(n, 16, generator=g).to(DEV)
    out, gt = torch.empty(n, 16, device=DEV), torch.empty(V, 16, device=DEV)
    ws = torch.empty(1 << 24, dtype=torch.uint8, device=DEV)
    with pytest.raises(ValueError):
        with torch.cuda.graph(torch.cuda.CUDAGraph()):
            e2f.e2f_embedding_backward(ctx, idx, go, V, grad_table=gt)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        e2f.e2f_embedding_forward(ctx, table, idx, out=out)
        e2f.e2f_embedding_backward(ctx, idx, go, V, grad_table=gt, workspace=ws)
    for k in range(4):
        idx.copy_((idx + k) % V)
        go.mul_(-0.5)
        gt.fill_(3.0)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, e2f.e2f_embedding_forward(ctx, table, idx))
        assert torch.equal(gt, e2f.e2f_embedding_backward(ctx, idx, go, V))


def test_refused_by_the_binding(e2f, ctx):
    table, idx, _ = data(10, 5, 8, 1)
    table, idx = table.to(DEV), idx.to(DEV)
    go = torch.zeros(10, 8, device=DEV)
    for bad in (lambda: e2f.e2f_embedding_forward(ctx, table, idx.short()),
                lambda: e2f.e2f_embedding_forward(ctx, table, idx[None]),
                lambda: e2f.e2f_embedding_forward(ctx, table, idx.cpu()),
                lambda: e2f.e2f_embedding_forward(ctx, table.half(), idx),
                lambda: e2f.e2f_embedding_forward(ctx, table.t(), idx),
                lambda: e2f.e2f_embedding_forward(ctx, table, idx, dtype=torch.float16),
                lambda: e2f.e2f_embedding_forward(ctx, table, idx, out=torch.empty(9, 8, device=DEV)),
                lambda: e2f.e2f_embedding_forward(ctx, table, idx, lmax=1, out=torch.empty(10, 8, device=DEV)),
                lambda: e2f.e2f_embedding_forward(ctx, table, idx, out=torch.empty(8, 10, device=DEV).t()),
                lambda: e2f.e2f_embedding_backward(ctx, idx, go[:9], 5),
                lambda: e2f.e2f_embedding_backward(ctx, idx, go[:1].expand(10, 8), 5),
                lambda: e2f.e2f_embedding_backward(ctx, idx, go, 5, grad_table=torch.empty(6, 8, device=DEV)),
                lambda: e2f.e2f_embedding_backward(ctx, idx, go, 5, workspace=torch.empty(10 ** 6, device=DEV)),
                lambda: e2f.e2f_embedding_backward(ctx, idx, go, 2 ** 31)):
        with pytest.raises(ValueError):
            bad()
    with pytest.raises(e2f.E2FError):
        e2f.e2f_embedding_backward(ctx, idx, go, 300, workspace=torch.empty(256, dtype=torch.uint8, device=DEV))
    with pytest.raises(e2f.E2FError):
        e2f.e2f_embedding_forward(ctx, table, idx, scale=float("nan"))
