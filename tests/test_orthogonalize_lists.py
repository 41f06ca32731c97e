"""CPU-only checks of e2f_orthogonalize's lists of several sizes: which outputs may lie over which inputs, and that
nothing is launched before every size is accepted.  The context has no device, so that the library checks its arguments
and goes no further."""
import ctypes

import pytest
import torch


@pytest.fixture(scope="module")
def e2f():
    import paper_2501_19216_amd as e
    return e


@pytest.fixture
def call(e2f, monkeypatch):
    """The binding with CPU tensors: "refused" where it or the library refuses, "accepted" where only the device is
    missing."""
    ctx = e2f.e2f_create(0, None)
    monkeypatch.setattr(e2f, "_stream", lambda device=None: ctypes.c_void_p(0))

    def run(grads, **kw):
        kw.setdefault("workspace", torch.empty(256, dtype=torch.uint8))
        try:
            e2f.e2f_orthogonalize(ctx, grads, **kw)
        except ValueError:
            return "refused"
        except e2f.E2FError as e:
            return "accepted" if e.status == e2f.E2F_EDEVICE else "refused"
    yield run
    ctx.close()


def test_outputs_over_tensors_of_another_size(call):
    a, b, c, d = (torch.zeros(240) for _ in range(4))
    two = lambda x, y: [x.view(8, 30), y.view(12, 20)]  # noqa: E731
    grads, other = two(a, b), two(c, d)
    e, f = torch.zeros(240), torch.zeros(240)
    assert call(grads, outs=other) == "accepted"
    # the other size's gradient, its own, the other size's weights and moments
    assert call(grads, outs=two(b, c)) == "refused"
    assert call(grads, outs=two(c, a)) == "refused"
    assert call(grads, outs=grads) == "refused"
    assert call(grads, outs=two(d, c), weights=two(c, d), decay=0.5) == "refused"
    assert call(grads, outs=two(c, e), weights=two(e, d), decay=0.5) == "refused"
    assert call(grads, outs=two(c, d), moments=two(d, e), new_moments=two(f, torch.zeros(240))) == "refused"
    assert call(grads, outs=two(c, d), moments=two(e, f), new_moments=two(f, e)) == "refused"
    assert call(grads, outs=two(c, d), moments=two(e, f), new_moments=two(e, b)) == "refused"
    assert call(grads, outs=two(c, d), moments=two(e, f), new_moments=two(e, d)) == "refused"
    # new moments where the weights are, and weights' outputs where the moments are
    assert call(grads, outs=two(c, d), weights=two(e, f), decay=0.5, moments=two(c, d), new_moments=two(e, f)) == "refused"
    # the tensors that they replace
    assert call(grads, outs=other, weights=other, decay=0.5) == "accepted"
    assert call(grads, outs=two(c, d), weights=two(c, d), decay=0.5) == "accepted"
    assert call(grads, outs=other, weights=other, decay=0.5, moments=two(e, f)) == "accepted"
    assert call(grads, outs=other, moments=two(e, f), new_moments=two(e, f)) == "accepted"
    # weights given twice: in place for both, or for one that the other still needs
    assert call(grads, outs=two(d, e), weights=two(c, c), decay=0.5) == "accepted"
    assert call(grads, outs=two(c, e), weights=two(c, c), decay=0.5) == "refused"
    # weights that are not read
    assert call(grads, outs=two(d, c), weights=two(c, d)) == "accepted"


class Counting:
    """The library, with the launching calls counted."""

    def __init__(self, lib):
        self.lib, self.launches = lib, 0

    def __getattr__(self, name):
        if name == "e2f_orthogonalize":
            self.launches += 1
        return getattr(self.lib, name)


def test_nothing_is_launched_before_every_size_is_accepted(call, e2f, monkeypatch):
    lib = Counting(e2f.lib)
    monkeypatch.setattr(e2f, "lib", lib)
    small, large, larger = torch.zeros(8, 30), torch.zeros(200, 300), torch.zeros(300, 400)

    def launches(grads, want, **kw):
        lib.launches = 0
        assert call(grads, outs=[torch.zeros_like(g) for g in grads], **kw) == want
        return lib.launches

    space = torch.empty((1 << 24) + 256, dtype=torch.uint8)
    space = space[-space.data_ptr() % 256:]
    assert launches([small, large, larger], "accepted", workspace=space) == 1  # (which says that there is no device)
    sizes = []
    for g in (large, larger):
        b = ctypes.c_size_t(0)
        prm = e2f.OrthogonalizeParams(*g.shape, 5, None, 1e-7, 0.95, 1, 1.0, 0.0, 0, 0)
        ctx = e2f.e2f_create(0, None)
        assert lib.e2f_orthogonalize_workspace_size(ctx.handle, ctypes.byref(prm), 1, ctypes.byref(b)) == e2f.E2F_OK
        ctx.close()
        sizes.append(b.value)
    assert 0 < sizes[0] < sizes[1]
    # enough for the first sizes only, in any order of them; not aligned; over a tensor of either size
    for grads in ([small, large, larger], [large, larger, small], [larger, small, large]):
        assert launches(grads, "accepted", workspace=space[:sizes[1]]) == 1
        for n in (0, 255, sizes[0] - 1, sizes[0], sizes[1] - 1):
            assert launches(grads, "refused", workspace=space[:n]) == 0, n
        assert launches(grads, "refused", workspace=space[8:]) == 0
    # matrices that fit a workgroup need none
    assert launches([small, torch.zeros(5, 5)], "accepted", workspace=space[:0]) == 1
    assert launches([small, torch.zeros(5, 5)], "accepted", workspace=space[8:]) == 1
    # a size that is too large behind one that is not
    huge = torch.zeros(1).expand(65537, 1)
    assert launches([small, torch.zeros(65537, 1)], "refused", workspace=space) == 0
    assert call([small, huge], workspace=space) == "refused"  # (not contiguous)


def test_a_workspace_over_a_tensor_of_any_size(call, e2f, monkeypatch):
    lib = Counting(e2f.lib)
    monkeypatch.setattr(e2f, "lib", lib)
    space = torch.empty((1 << 24) + 256, dtype=torch.uint8)
    space = space[-space.data_ptr() % 256:]
    small, large = torch.zeros(8, 30), torch.zeros(200, 300)
    at = space[1 << 20:(1 << 20) + 960].view(torch.float32).view(8, 30)
    new = lambda: [torch.zeros(8, 30), torch.zeros(200, 300)]  # noqa: E731
    for kw in (dict(outs=[at, new()[1]]), dict(outs=new(), moments=[at, new()[1]]),
               dict(outs=new(), weights=[at, new()[1]], decay=0.5)):
        for turn in (slice(None), slice(None, None, -1)):
            lists = {k: v[turn] if isinstance(v, list) else v for k, v in kw.items()}
            lib.launches = 0
            assert call([small, large][turn], workspace=space, **lists) == "refused", kw
            assert lib.launches == 0
    assert call([at, large], outs=new(), workspace=space) == "refused"
    # behind what the call needs of it
    behind = space[1 << 23:(1 << 23) + 960].view(torch.float32).view(8, 30)
    assert call([behind, large], outs=new(), workspace=space) == "accepted"
