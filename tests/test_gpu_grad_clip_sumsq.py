"""Gradient clipping whose sum of squares lies in one of its outputs is refused, and beside them is not.  Run with
-m gpu."""
import pytest
import torch

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


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_sum_of_squares_in_an_output(e2f, ctx, dtype):
    per = 64 // torch.finfo(dtype).bits  # values of 8 bytes
    flat = torch.ones(64 * per, dtype=dtype, device=DEV)
    other = torch.ones(100, device=DEV)
    places = flat.view(torch.float64)
    for place, fits in ((0, True), (15, True), (16, False), (20, False), (47, False), (48, True), (63, True)):
        places.fill_(4.0)  # (as sumsq: a norm of 2)
        grads = flat[16 * per:48 * per]
        if fits:
            e2f.e2f_grad_clip(ctx, [other, grads], places[place], 1.0)
        else:
            before = flat.clone()
            with pytest.raises(e2f.E2FError):
                e2f.e2f_grad_clip(ctx, [other, grads], places[place], 1.0)
            assert torch.equal(flat.view(torch.uint8), before.view(torch.uint8))  # nothing was written
    # as an input that is not written it may be anywhere
    places.fill_(4.0)
    e2f.e2f_grad_clip(ctx, [flat[:32 * per]], places[3], 1.0, outs=[torch.empty_like(flat[:32 * per])])
    with pytest.raises(e2f.E2FError):
        e2f.e2f_grad_clip(ctx, [torch.ones_like(flat)], places[63], 1.0, outs=[flat])
