"""Embedding and layer norm of more than 2^32 bytes and 2^31 values: rows at the start, about the borders and at the end
against float64, and the gradients that sum over all rows.  Run with -m gpu."""
import pytest
import torch

import training_reference as ref

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF16 = torch.bfloat16


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


def some_rows(n, width):
    """The first, the last, and those about the values 2^31 and 2^32."""
    at = [0, 1, n - 2, n - 1] + [v // width + d for v in (2 ** 30, 2 ** 31, 2 ** 32) for d in (-1, 0, 1)]
    return torch.tensor(sorted({r for r in at if 0 <= r < n}), device=DEV)


def test_embedding(e2f, ctx):
    n, V, C = 2 ** 26 + 5, 7, 66
    g = torch.Generator(device=DEV).manual_seed(1)
    table = torch.randn(V, C, device=DEV, generator=g)
    idx = torch.randint(-1, V, (n,), device=DEV, generator=g, dtype=torch.int32)
    out = e2f.e2f_embedding_forward(ctx, table, idx, dtype=BF16)
    rows = some_rows(n, C)
    ref.check(out[rows][:, None], ref.embedding(table.cpu(), idx[rows].cpu(), 1, 1.0), "out")
    # every row: the rows of each type are one row over and over
    for v in range(-1, V):
        want = torch.zeros(C, dtype=BF16, device=DEV) if v < 0 else table[v].to(BF16)
        for s in range(0, n, 2 ** 24):
            piece = out[s:s + 2 ** 24]
            assert bool(((piece == want).all(1) | (idx[s:s + 2 ** 24] != v)).all())
    # the gradient of that output: as many times the row as the type has rows; its sums are of 10^7 equal values
    got = e2f.e2f_embedding_backward(ctx, idx, out, V, dtype=torch.float32)
    counts = torch.bincount(idx.long() + 1, minlength=V + 1)[1:].double()[:, None].cpu()
    value = counts * table.to(BF16).cpu().double()
    # (a stretch of up to 64 rows, 256 such parts of a workgroup, those of the workgroups in 1024 strides)
    ref.check(got, (value, ref.U * (64 + 256 + counts / 1024 / 64 + 20) * value.abs()), "grad_table")


def test_layer_norm(e2f, ctx):
    n, C = 2 ** 26 + 77, 34
    g = torch.Generator(device=DEV).manual_seed(2)
    x = torch.empty(n, C, dtype=BF16, device=DEV).normal_(generator=g)
    go = torch.empty(n, C, dtype=BF16, device=DEV).normal_(generator=g)
    w, b = 1 + torch.randn(C, device=DEV, generator=g), torch.randn(C, device=DEV, generator=g)
    out = e2f.e2f_layer_norm_forward(ctx, x, weight=w, bias=b)
    gx, gw, gb = e2f.e2f_layer_norm_backward(ctx, x, go, weight=w, bias=b)
    rows = some_rows(n, C)
    want = ref.layer_norm(x[rows].cpu()[:, None], 0, w.cpu()[None], b.cpu(), g=go[rows].cpu()[:, None])
    ref.check(out[rows][:, None], want["out"], "out")
    ref.check(gx[rows][:, None], want["grad_x"], "grad_x")
    sw, sb, aw, ab = (torch.zeros(C, dtype=torch.float64, device=DEV) for _ in range(4))
    for s in range(0, n, 2 ** 22):
        v, d = x[s:s + 2 ** 22].double(), go[s:s + 2 ** 22].double()
        v = v - v.mean(1, keepdim=True)
        h = v * (v.square().mean(1, keepdim=True) + 1e-5).rsqrt()
        sw += (d * h).sum(0)
        sb += d.sum(0)
        aw += (d * h).abs().sum(0)
        ab += d.abs().sum(0)
    # a thread's rows one after the other (1,024 workgroups of 32 side by side), 5 exchanges and 4 waves, then float64; and 50
    # roundings of each term
    count = n / 1024 / 32 + 100
    for got, value, size in ((gw, sw, aw), (gb, sb, ab)):
        assert bool(((got.double() - value).abs() <= ref.U * count * size).all())
