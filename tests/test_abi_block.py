"""CPU-only checks of the boundary of the operators around the convolution:
arguments that are refused before any device work, sizes of workspaces."""
import ctypes

import pytest


@pytest.fixture(scope="module")
def e2f():
    import paper_2501_19216_amd as e
    return e


@pytest.fixture(scope="module")
def ctx(e2f):
    c = e2f.e2f_create(0, None)
    yield c
    c.close()


def at(address):
    return ctypes.c_void_p(address)


# never dereferenced: every call below ends before device work; 2^20 apart
A, B, C, D, E, F, G, H, I, J, K, M = (at((i + 1) << 20) for i in range(12))
BIG = 1 << 40


def attention_params(e2f, **kw):
    base = dict(heads=4, k_heads=2, dk=8, n_rbf=8, cutoff=5.0, scale=0.3, cap=10.0, dtype=0, ldq=0, ldk=0)
    base.update(kw)
    return e2f.AttentionParams(**base)


def test_attention_refusals(e2f, ctx):
    lib, EINVAL, EUNS, ECAP, EDEV = e2f.lib, e2f.E2F_EINVAL, e2f.E2F_EUNSUPPORTED, e2f.E2F_ECAPACITY, e2f.E2F_EDEVICE

    def fwd(prm=None, n=10, edges=30, handle=ctx.handle, pos=A, q=B, k=C, w=D, rp=E, ci=F, alpha=G, lse=H, none=False, **kw):
        prm = attention_params(e2f, **kw)
        return lib.e2f_attention_forward(handle, None if none else ctypes.byref(prm), pos, None, q, k, n, w, rp, ci,
                                         edges, alpha, lse, None)

    def bwd(n=10, edges=30, pos=A, q=B, k=C, w=D, rp=E, ci=F, alpha=G, lse=H, ga=I, rt=J, ct=K, pm=M, gq=A, gk=B, gw=C,
            gp=D, ws=E, size=BIG, **kw):
        return lib.e2f_attention_backward(ctx.handle, ctypes.byref(attention_params(e2f, **kw)), pos, None, q, k, n, w,
                                          rp, ci, edges, rt, ct, pm, alpha, lse, ga, gq, gk, gw, gp, ws, size, None)

    for call in (fwd, bwd):
        assert call() == EDEV  # valid, but the context has no device
        for kw in (dict(heads=0), dict(k_heads=0), dict(k_heads=3), dict(k_heads=8), dict(dk=-1), dict(n_rbf=1),
                   dict(n_rbf=-2), dict(cutoff=0.0), dict(cutoff=float("inf")), dict(scale=float("nan")),
                   dict(cap=-1.0), dict(cap=float("nan")), dict(cap=float("inf")), dict(dtype=2), dict(ldq=31),
                   dict(ldk=15), dict(ldq=-32), dict(n=-1), dict(edges=-1), dict(n=0), dict(pos=None), dict(q=None),
                   dict(k=None), dict(w=None), dict(rp=None), dict(ci=None), dict(alpha=None)):
            assert call(**kw) == EINVAL, kw
        for kw in (dict(heads=65, k_heads=65), dict(dk=257), dict(n_rbf=33), dict(edges=2 ** 31), dict(n=2 ** 31 - 1)):
            assert call(**kw) == EUNS, kw
        for kw in (dict(ldq=32, ldk=16), dict(ldq=4096), dict(cap=0.0), dict(dtype=1), dict(n_rbf=0, w=None, **(dict(gw=None) if call is bwd else {})),
                   dict(dk=0, q=None, k=None, **(dict(gq=None, gk=None) if call is bwd else {}))):
            assert call(**kw) == EDEV, kw
    assert fwd(handle=None) == EINVAL and fwd(none=True) == EINVAL
    assert fwd(lse=None) == EDEV  # not kept
    assert bwd(gq=None, gk=None, gw=None, gp=None) == EINVAL
    assert bwd(dk=0, q=None, k=None) == EINVAL and bwd(n_rbf=0) == EINVAL  # the gradient of what is not there
    assert bwd(lse=None) == EINVAL and bwd(ga=None) == EINVAL
    for kw in (dict(rt=None), dict(ct=None), dict(pm=None)):
        assert bwd(**kw) == EINVAL
        assert bwd(gk=None, gp=None, **kw) == EDEV
    b = ctypes.c_size_t(0)
    size = lib.e2f_attention_backward_workspace_size
    assert size(ctx.handle, ctypes.byref(attention_params(e2f)), 10, 30, ctypes.byref(b)) == e2f.E2F_OK
    assert b.value % 256 == 0
    assert bwd(size=b.value) == EDEV and bwd(size=b.value - 1) == ECAP and bwd(ws=None) == ECAP
    assert bwd(ws=at((1 << 20) + 128)) == EINVAL
    assert size(ctx.handle, ctypes.byref(attention_params(e2f)), 10, 30, None) == EINVAL
    assert size(ctx.handle, ctypes.byref(attention_params(e2f, heads=0)), 10, 30, ctypes.byref(b)) == EINVAL


def test_transpose_refusals(e2f, ctx):
    lib, EINVAL, EUNS, ECAP, EDEV = e2f.lib, e2f.E2F_EINVAL, e2f.E2F_EUNSUPPORTED, e2f.E2F_ECAPACITY, e2f.E2F_EDEVICE

    def call(n=10, edges=30, rp=A, ci=B, rt=C, ct=D, pm=E, ws=F, size=BIG, handle=ctx.handle):
        return lib.e2f_transpose_graph(handle, n, rp, ci, edges, rt, ct, pm, ws, size, None)

    assert call() == EDEV
    for kw in (dict(n=-1), dict(edges=-1), dict(n=0), dict(rp=None), dict(ci=None), dict(rt=None), dict(ct=None),
               dict(pm=None), dict(handle=None), dict(ws=at((1 << 20) + 8))):
        assert call(**kw) == EINVAL, kw
    assert call(edges=2 ** 31) == EUNS and call(n=2 ** 31 - 1) == EUNS
    assert call(edges=0, ci=None, ct=None, pm=None) == EDEV
    b = ctypes.c_size_t(0)
    assert lib.e2f_transpose_graph_workspace_size(ctx.handle, 10, 30, ctypes.byref(b)) == e2f.E2F_OK
    assert call(size=b.value) == EDEV and call(size=b.value - 1) == ECAP and call(ws=None) == ECAP
    assert lib.e2f_transpose_graph_workspace_size(ctx.handle, 10, 30, None) == EINVAL


def norm_params(e2f, **kw):
    base = dict(lmax=2, channels=16, gates=1, eps=1e-5, dtype=0, post_w=A.value, res_scale=B.value, pre_w=C.value)
    base.update(kw)
    return e2f.NormParams(**base)


def test_norm_refusals(e2f, ctx):
    lib, EINVAL, EUNS, ECAP, EDEV = e2f.lib, e2f.E2F_EINVAL, e2f.E2F_EUNSUPPORTED, e2f.E2F_ECAPACITY, e2f.E2F_EDEVICE
    n = 8
    row = 4 * 9 * 16

    def fwd(n=n, x=D, block=E, gate=F, out=G, normed=H, rstd=I, handle=ctx.handle, none=False, **kw):
        prm = norm_params(e2f, **kw)
        return lib.e2f_block_norm_forward(handle, None if none else ctypes.byref(prm), x, block, gate, n, out, normed,
                                          rstd, None)

    def bwd(n=n, x=D, block=E, gate=F, rstd=G, go=H, gn=I, gx=J, gb=K, gg=M, gp=at(13 << 20), gs=at(14 << 20),
            gw=at(15 << 20), ws=at(16 << 20), size=BIG, **kw):
        return lib.e2f_block_norm_backward(ctx.handle, ctypes.byref(norm_params(e2f, **kw)), x, block, gate, rstd, n,
                                           go, gn, gx, gb, gg, gp, gs, gw, ws, size, None)

    for call in (fwd, bwd):
        assert call() == EDEV
        for kw in (dict(n=-1), dict(lmax=-1), dict(gates=2), dict(gates=-1), dict(eps=-1.0), dict(eps=float("nan")),
                   dict(dtype=2), dict(x=None), dict(gate=None), dict(gates=0), dict(block=None)):
            assert call(**kw) == EINVAL, kw
        for kw in (dict(lmax=7), dict(channels=0), dict(channels=18), dict(channels=1028), dict(n=2 ** 31 - 1)):
            assert call(**kw) == EUNS, kw
        assert call(gates=3) == EDEV and call(dtype=1) == EDEV and call(eps=0.0) == EDEV
    assert fwd(handle=None) == EINVAL and fwd(none=True) == EINVAL
    assert fwd(out=None) == EINVAL and fwd(normed=None) == EINVAL and fwd(pre_w=None) == EINVAL
    assert fwd(normed=None, pre_w=None) == EDEV and fwd(rstd=None) == EDEV
    alone = dict(block=None, gate=None, gates=0, post_w=None, res_scale=None, out=None)
    assert fwd(**alone) == EDEV and fwd(**alone, pre_w=None, normed=None) == EINVAL
    assert fwd(**{**alone, "out": G}) == EINVAL and fwd(**{**alone, "post_w": A.value}) == EINVAL
    # outputs over inputs or each other
    for kw in (dict(out=D), dict(out=E), dict(normed=D), dict(normed=G), dict(out=at(D.value + n * row - 4)),
               dict(out=at(D.value - n * row + 4)), dict(normed=F), dict(rstd=D)):
        assert fwd(**kw) == EINVAL, kw
    assert fwd(out=at(D.value + n * row)) == EDEV
    assert bwd(gx=None, gb=None, gg=None, gp=None, gs=None, gw=None) == EINVAL
    assert bwd(rstd=None) == EINVAL
    assert bwd(gates=0, gate=None) == EINVAL and bwd(gates=0, gate=None, gg=None) == EDEV
    assert bwd(post_w=None) == EINVAL and bwd(post_w=None, gp=None) == EDEV
    assert bwd(res_scale=None) == EINVAL and bwd(res_scale=None, gs=None) == EDEV
    assert bwd(pre_w=None, gw=None) == EINVAL and bwd(pre_w=None, gw=None, gn=None) == EDEV
    assert bwd(pre_w=None, gn=None) == EINVAL
    assert bwd(go=None, gn=None) == EDEV
    for kw in (dict(gx=D), dict(gx=H), dict(gb=E), dict(gg=F), dict(gx=K), dict(gp=A), dict(gs=at(15 << 20)), dict(gb=I)):
        assert bwd(**kw) == EINVAL, kw
    b = ctypes.c_size_t(0)
    assert lib.e2f_block_norm_workspace_size(ctx.handle, ctypes.byref(norm_params(e2f)), n, ctypes.byref(b)) == e2f.E2F_OK
    assert bwd(size=b.value) == EDEV and bwd(size=b.value - 1) == ECAP and bwd(ws=at((16 << 20) + 64)) == EINVAL
    assert bwd(ws=None, size=0, gp=None, gs=None, gw=None) == EDEV  # only the weights' gradients need it
    assert lib.e2f_block_norm_workspace_size(ctx.handle, ctypes.byref(norm_params(e2f)), n, None) == EINVAL


def test_clip_refusals(e2f, ctx):
    lib, EINVAL, ECAP, EDEV = e2f.lib, e2f.E2F_EINVAL, e2f.E2F_ECAPACITY, e2f.E2F_EDEVICE
    p = lambda *v: (ctypes.c_void_p * len(v))(*v)  # noqa: E731
    sizes = lambda *v: (ctypes.c_int64 * len(v))(*v)  # noqa: E731
    types = lambda *v: (ctypes.c_int32 * len(v))(*v)  # noqa: E731
    a, b = 1 << 20, 2 << 20

    def norm(count=2, ts=p(a, b), ns=sizes(10, 20), ds=types(0, 1), sumsq=A, out=B, ws=C, size=BIG, handle=ctx.handle):
        return lib.e2f_grad_norm(handle, count, ts, ns, ds, sumsq, out, ws, size, None)

    def clip(count=2, ts=p(a, b), os=p(3 << 20, 4 << 20), ns=sizes(10, 20), ds=types(0, 1), sumsq=A, max_norm=1.0):
        return lib.e2f_grad_clip(ctx.handle, count, ts, os, ns, ds, sumsq, max_norm, None)

    for call in (norm, clip):
        assert call() == EDEV
        for kw in (dict(count=-1), dict(ts=None), dict(ns=None), dict(ds=None), dict(ns=sizes(10, -1)),
                   dict(ds=types(0, 2)), dict(ts=p(a, None)), dict(ts=p(a + 2, b)), dict(ts=p(a, b + 1))):
            assert call(**kw) == EINVAL, kw
        assert call(ts=p(a, b + 2)) == EDEV and call(ts=p(a + 4, b)) == EDEV
        assert call(ts=p(a, None), ns=sizes(10, 0), **(dict(os=p(3 << 20, None)) if call is clip else {})) == EDEV
    assert norm(handle=None) == EINVAL and norm(sumsq=None, out=None) == EINVAL
    assert norm(sumsq=None) == EDEV and norm(out=None) == EDEV
    size = ctypes.c_size_t(0)
    assert lib.e2f_grad_norm_workspace_size(ctx.handle, 2, sizes(10, 20), ctypes.byref(size)) == e2f.E2F_OK
    assert norm(size=size.value) == EDEV and norm(size=size.value - 1) == ECAP and norm(ws=at((1 << 20) + 8)) == EINVAL
    assert lib.e2f_grad_norm_workspace_size(ctx.handle, 2, sizes(10, -20), ctypes.byref(size)) == EINVAL
    for kw in (dict(sumsq=None), dict(max_norm=0.0), dict(max_norm=-1.0), dict(max_norm=float("nan")),
               dict(max_norm=float("inf")), dict(os=None), dict(os=p(3 << 20, None))):
        assert clip(**kw) == EINVAL, kw
    assert clip(os=p(a, b)) == EDEV  # in place
    assert clip(ts=p(a, a), os=p(3 << 20, 4 << 20)) == EDEV  # read twice
    assert clip(ts=p(a, a), os=p(a, a), ds=types(0, 0), ns=sizes(10, 10)) == EINVAL  # the same tensor twice, in place
    assert clip(ts=p(a, a), os=p(a, b)) == EINVAL  # read by one, written by the other
    assert clip(os=p(b, a)) == EINVAL and clip(os=p(a + 4, b)) == EINVAL and clip(os=p(3 << 20, 3 << 20)) == EINVAL
    assert clip(ts=p(a, a + 40), os=p(a, a + 40)) == EDEV  # neighbours
    assert clip(ts=p(a, a + 38), os=p(a, a + 38)) == EINVAL
