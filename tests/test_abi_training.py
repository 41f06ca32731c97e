"""CPU-only checks of the boundary of embedding, layer norm and orthogonalised updates: arguments that are refused
before any device work, sizes of workspaces, overlaps."""
import ctypes

import pytest

INF, NAN = float("inf"), float("nan")
BIG = 1 << 40


@pytest.fixture(scope="module")
def e2f():
    import paper_2501_19216_amd as e
    return e


@pytest.fixture(scope="module")
def ctx(e2f):
    c = e2f.e2f_create(0, None)
    yield c
    c.close()


def at(slot, offset=0):
    """Never dereferenced: 2^20 apart."""
    return ctypes.c_void_p((slot << 20) + offset)


def embedding(e2f, **kw):
    return e2f.EmbeddingParams(**{**dict(vocab=10, channels=8, lmax=1, scale=2.0, table_dtype=0, dtype=0, index_bytes=4,
                                         ld=0), **kw})


def test_embedding_refusals(e2f, ctx):
    lib, EINVAL, EUNS, ECAP, EDEV = e2f.lib, e2f.E2F_EINVAL, e2f.E2F_EUNSUPPORTED, e2f.E2F_ECAPACITY, e2f.E2F_EDEVICE

    def fwd(n=20, table=at(1), index=at(2), out=at(3), handle=ctx.handle, none=False, **kw):
        return lib.e2f_embedding_forward(handle, None if none else ctypes.byref(embedding(e2f, **kw)), table, index, n,
                                         out, None)

    def bwd(n=20, table=at(1), index=at(2), out=at(3), ws=at(4), size=BIG, handle=ctx.handle, none=False, **kw):
        return lib.e2f_embedding_backward(handle, None if none else ctypes.byref(embedding(e2f, **kw)), index, n, out,
                                          table, ws, size, None)

    for call in (fwd, bwd):
        assert call() == EDEV
        for kw in (dict(vocab=0), dict(vocab=-1), dict(channels=0), dict(lmax=-1), dict(scale=INF), dict(scale=NAN),
                   dict(table_dtype=2), dict(dtype=-1), dict(index_bytes=2), dict(ld=31), dict(ld=-32), dict(n=-1),
                   dict(index=None), dict(out=None), dict(table=None), dict(handle=None), dict(none=True),
                   dict(table=at(1, 2)), dict(out=at(3, 2)), dict(index=at(2, 4), index_bytes=8), dict(dtype=1, out=at(3, 1))):
            assert call(**kw) == EINVAL, kw
        for kw in (dict(channels=65537), dict(lmax=7), dict(n=2 ** 31 - 1), dict(vocab=2 ** 31 - 1), dict(ld=2 ** 41)):
            assert call(**kw) == EUNS, kw
        for kw in (dict(ld=32), dict(ld=1000), dict(index_bytes=8), dict(dtype=1, out=at(3, 2)), dict(table_dtype=1, table=at(1, 2)),
                   dict(scale=0.0), dict(n=0, index=None, out=None)):
            assert call(**kw) == EDEV, kw
    b = ctypes.c_size_t(0)
    size = lib.e2f_embedding_backward_workspace_size
    assert size(ctx.handle, ctypes.byref(embedding(e2f)), 20, ctypes.byref(b)) == e2f.E2F_OK and b.value % 256 == 0
    assert bwd(size=b.value) == EDEV and bwd(size=b.value - 1) == ECAP and bwd(ws=None) == ECAP
    assert bwd(ws=at(4, 128)) == EINVAL
    assert size(ctx.handle, ctypes.byref(embedding(e2f)), 20, None) == EINVAL
    assert size(ctx.handle, ctypes.byref(embedding(e2f, vocab=0)), 20, ctypes.byref(b)) == EINVAL
    # overlaps: the table's 320 bytes, the index's 80, out's 20 rows of 128
    assert fwd(out=at(1, 316)) == EINVAL and fwd(out=at(1, 320)) == EDEV
    assert fwd(out=at(2, 76)) == EINVAL and fwd(out=at(2, 80)) == EDEV and fwd(out=at(2, -2560)) == EDEV
    assert fwd(out=at(2, -2556)) == EINVAL
    assert bwd(table=at(3, 2556)) == EINVAL and bwd(table=at(3, 2560)) == EDEV
    assert bwd(table=at(3, 19 * 400 + 124), ld=100) == EINVAL and bwd(table=at(3, 19 * 400 + 128), ld=100) == EDEV
    assert bwd(table=at(4)) == EINVAL and bwd(ws=at(2)) == EINVAL and bwd(ws=at(3)) == EINVAL


def layer(e2f, **kw):
    return e2f.LayerNormParams(**{**dict(lmax=1, channels=8, eps=1e-5, silu=0, dtype=0, weight=at(1).value,
                                         bias=at(2).value, ldx=0), **kw})


def test_layer_norm_refusals(e2f, ctx):
    lib, EINVAL, EUNS, ECAP, EDEV = e2f.lib, e2f.E2F_EINVAL, e2f.E2F_EUNSUPPORTED, e2f.E2F_ECAPACITY, e2f.E2F_EDEVICE

    def fwd(n=20, x=at(3), out=at(4), handle=ctx.handle, none=False, **kw):
        return lib.e2f_layer_norm_forward(handle, None if none else ctypes.byref(layer(e2f, **kw)), x, n, out, None)

    def bwd(n=20, x=at(3), out=at(4), gx=at(5), gw=at(6), gb=at(7), ws=at(8), size=BIG, handle=ctx.handle, none=False,
            **kw):
        return lib.e2f_layer_norm_backward(handle, None if none else ctypes.byref(layer(e2f, **kw)), x, n, out, gx, gw,
                                           gb, ws, size, None)

    for call in (fwd, bwd):
        assert call() == EDEV
        for kw in (dict(lmax=-1), dict(channels=0), dict(eps=-1.0), dict(eps=NAN), dict(eps=INF), dict(silu=2),
                   dict(silu=1), dict(dtype=2), dict(ldx=31), dict(ldx=-1), dict(n=-1), dict(x=None), dict(out=None),
                   dict(handle=None), dict(none=True), dict(x=at(3, 2)), dict(weight=at(1, 2).value)):
            assert call(**kw) == EINVAL, kw
        for kw in (dict(lmax=7), dict(channels=6), dict(channels=1028), dict(lmax=0, channels=8193), dict(n=2 ** 31 - 1),
                   dict(ldx=2 ** 41)):
            assert call(**kw) == EUNS, kw
        for kw in (dict(lmax=0, silu=1), dict(lmax=0, channels=1), dict(lmax=0, channels=8191, n=1), dict(weight=None),
                   dict(bias=None), dict(ldx=32), dict(ldx=77), dict(eps=0.0), dict(dtype=1, x=at(3, 2)),
                   dict(n=0, x=None, out=None)):
            assert call(**kw) == EDEV, kw
    assert bwd(gx=None, gw=None, gb=None) == EINVAL
    assert bwd(gw=None, gb=None, ws=None, size=0) == EDEV and bwd(gx=None) == EDEV and bwd(gb=None, ws=None) == ECAP
    b = ctypes.c_size_t(0)
    size = lib.e2f_layer_norm_workspace_size
    assert size(ctx.handle, ctypes.byref(layer(e2f)), 20, ctypes.byref(b)) == e2f.E2F_OK and b.value % 256 == 0
    assert bwd(size=b.value) == EDEV and bwd(size=b.value - 1) == ECAP and bwd(ws=at(8, 64)) == EINVAL
    assert size(ctx.handle, ctypes.byref(layer(e2f)), 20, None) == EINVAL
    # overlaps: 20 rows of 128 bytes, weights of 64, biases of 32
    assert fwd(out=at(3, 2556)) == EINVAL and fwd(out=at(3, 2560)) == EDEV and fwd(out=at(3)) == EINVAL
    assert fwd(out=at(1, 60)) == EINVAL and fwd(out=at(1, 64)) == EDEV and fwd(out=at(2, 28)) == EINVAL
    assert fwd(out=at(3, 19 * 400 + 124), ldx=100) == EINVAL and fwd(out=at(3, 19 * 400 + 128), ldx=100) == EDEV
    assert bwd(gx=at(4)) == EINVAL and bwd(gx=at(3)) == EINVAL and bwd(gw=at(1)) == EINVAL and bwd(gb=at(2)) == EINVAL
    assert bwd(gw=at(5, 2556)) == EINVAL and bwd(gb=at(6, 60)) == EINVAL and bwd(ws=at(6)) == EINVAL


def ortho(e2f, coefs=None, **kw):
    return e2f.OrthogonalizeParams(**{**dict(rows=8, cols=16, steps=5, coefs=coefs, eps=1e-7, momentum=0.9, nesterov=1,
                                             scale=1.0, decay=0.5, grad_dtype=0, dtype=0), **kw})


def array_of(values):
    return (ctypes.c_void_p * len(values))(*[None if v is None else v.value for v in values])


def test_orthogonalize_refusals(e2f, ctx):
    lib, EINVAL, EUNS, ECAP, EDEV = e2f.lib, e2f.E2F_EINVAL, e2f.E2F_EUNSUPPORTED, e2f.E2F_ECAPACITY, e2f.E2F_EDEVICE
    base = dict(g=[at(1), at(2)], m=[at(3), at(4)], to=[at(5), at(6)], w=[at(7), at(8)], out=[at(9), at(10)])

    def call(count=2, ws=at(20), size=BIG, handle=ctx.handle, none=False, coefs=None, **kw):
        lists = [kw.pop(k, base[k]) for k in ("g", "m", "to", "w", "out")]
        c = None if coefs is None else (ctypes.c_float * len(coefs))(*coefs)
        prm = ortho(e2f, coefs=None if c is None else ctypes.addressof(c), **kw)
        return lib.e2f_orthogonalize(handle, None if none else ctypes.byref(prm), count,
                                     *(None if v is None else array_of(v) for v in lists), ws, size, None)

    assert call() == EDEV
    for kw in (dict(count=-1), dict(rows=-1), dict(cols=-1), dict(steps=-1), dict(eps=-1.0), dict(eps=NAN),
               dict(momentum=NAN), dict(scale=INF), dict(decay=NAN), dict(nesterov=2), dict(grad_dtype=2), dict(dtype=2),
               dict(handle=None), dict(none=True), dict(g=None), dict(out=None), dict(m=None), dict(to=None),
               dict(w=None), dict(g=[at(1), None]), dict(m=[None, at(4)]), dict(out=[at(9, 2), at(10)]),
               dict(to=[at(5), at(6, 1)])):
        assert call(**kw) == EINVAL, kw
    for kw in (dict(steps=65), dict(rows=65537), dict(cols=65537), dict(rows=65536, cols=32768)):
        assert call(**kw) == EUNS, kw
    # coefficients whose steps leave the singular values unbounded, or are no numbers
    for coefs in ([NAN, 0, 0], [0, INF, 0], [100, 0, 0], [3.0, 0, 0] * 5, [0, 5000, 0]):
        assert call(steps=len(coefs) // 3, coefs=coefs) == EINVAL, coefs
    for coefs in ([1.5, -0.5, 0] * 20, [15 / 8, -10 / 8, 3 / 8] * 7, [8.28, -23.6, 17.3, 4.1, -2.9, 0.55], [0, 0, 0], []):
        assert call(steps=len(coefs) // 3, coefs=coefs) == EDEV, coefs
    for kw in (dict(m=None, to=None), dict(w=None, decay=0.0), dict(count=0, g=None, out=None), dict(rows=0, g=None),
               dict(grad_dtype=1, g=[at(1, 2), at(2)]), dict(dtype=1, w=[at(7, 2), at(8)]), dict(steps=0), dict(steps=64),
               dict(momentum=-0.5), dict(eps=0.0)):
        assert call(**kw) == EDEV, kw
    b = ctypes.c_size_t(0)
    size = lib.e2f_orthogonalize_workspace_size
    big = dict(rows=200, cols=300)
    assert size(ctx.handle, ctypes.byref(ortho(e2f, **big)), 2, ctypes.byref(b)) == e2f.E2F_OK
    assert b.value > 0 and b.value % 256 == 0
    assert call(size=b.value, **big) == EDEV and call(size=b.value - 1, **big) == ECAP and call(ws=None, **big) == ECAP
    assert call(ws=at(20, 8), **big) == EINVAL
    assert call(ws=at(9), **big) == EINVAL and call(ws=at(1), **big) == EINVAL and call(ws=at(7), **big) == EINVAL
    assert size(ctx.handle, ctypes.byref(ortho(e2f)), 2, None) == EINVAL
    for kw in (dict(rows=0), {}):  # nothing to do, or all in a workgroup
        assert size(ctx.handle, ctypes.byref(ortho(e2f, **kw)), 2, ctypes.byref(b)) == e2f.E2F_OK and b.value == 0
        assert call(ws=None, size=0, **kw) == EDEV
    # overlaps: matrices of 512 bytes; an output may be the input that it replaces
    assert call(out=base["w"]) == EDEV and call(to=base["m"]) == EDEV and call(out=base["w"], to=base["m"]) == EDEV
    assert call(out=[at(8), at(7)]) == EINVAL and call(to=[at(4), at(3)]) == EINVAL  # each other's
    assert call(out=[at(7), at(7)], w=[at(7), at(7)]) == EINVAL
    for name in ("g", "m", "w"):
        first = base[name][1].value
        for out in ("to", "out"):
            for off, want in ((4, EINVAL), (508, EINVAL), (-508, EINVAL), (512, EDEV), (-512, EDEV)):
                assert call(**{out: [base[out][0], ctypes.c_void_p(first + off)]}) == want, (name, out, off)
    assert call(out=base["g"]) == EINVAL and call(out=base["to"]) == EINVAL and call(out=base["m"]) == EINVAL
    assert call(out=base["w"], decay=0.0) == EDEV  # (not read then)
    assert call(dtype=1, grad_dtype=1, out=[at(1, 256), at(10)]) == EDEV and call(out=[at(1, 256), at(10)]) == EINVAL
