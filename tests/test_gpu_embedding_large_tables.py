"""The gradient of a table of more than 2^30 types, whose first and last places in the sorted order lie more than 2^31
values apart, against sums of float64.  Run with -m gpu."""
import pytest
import torch

import training_reference as ref

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.mark.parametrize("n", [1500, 5000])
def test_types_above_2_to_30(n):
    """Sorted by one workgroup and by several; types on both sides of the one whose place is 2^31 behind the table's
    first."""
    import paper_2501_19216_amd as e2f
    ctx = e2f.e2f_create(0, 0)
    V = 2 ** 30 + 2 ** 20 + 3
    border = 2 ** 31 - V
    assert border < V
    g = torch.Generator().manual_seed(n)
    some = torch.tensor([0, 1, border - 1, border, border + 1, 2 ** 30, V - 2, V - 1, -1, V])
    idx = torch.cat([some, torch.randint(0, V, (n // 2,), generator=g), some[torch.randint(0, 10, (n - 10 - n // 2,), generator=g)]])
    idx = idx[torch.randperm(n, generator=g)]
    go = torch.randn(n, 1, generator=g)
    got = e2f.e2f_embedding_backward(ctx, idx.int().to(DEV), go.to(DEV), V, dtype=torch.bfloat16)
    there = (idx >= 0) & (idx < V)
    types, short = idx[there].unique(return_inverse=True)
    want = ref.embedding_grad(go[there], short, len(types), 1.0)
    ref.check(got[types.to(DEV)], want, "grad_table")
    # nothing but these
    assert int(torch.count_nonzero(got)) == int(torch.count_nonzero(got[types.to(DEV)]))
    del got
    ctx.close()
    torch.cuda.empty_cache()
