"""CPU-only checks of the block's operators: outputs over inputs, over each other and over the workspace are refused
before any device work."""
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


def at(slot, offset=0):
    """Never dereferenced: 2^20 apart."""
    return ctypes.c_void_p((slot << 20) + offset)


n, EDGES, H, HK, DK = 10, 30, 4, 2, 8


def attention_params(e2f, **kw):
    return e2f.AttentionParams(**{**dict(heads=H, k_heads=HK, dk=DK, n_rbf=8, cutoff=5.0, scale=0.3, cap=10.0, dtype=0,
                                         ldq=0, ldk=0), **kw})


def test_attention_forward(e2f, ctx):
    base = dict(pos=at(1), gid=at(2), q=at(3), k=at(4), w=at(5), rp=at(6), ci=at(7), alpha=at(8), lse=at(9))

    def call(prm={}, **kw):
        v = {**base, **kw}
        return e2f.lib.e2f_attention_forward(ctx.handle, ctypes.byref(attention_params(e2f, **prm)), v["pos"], v["gid"],
                                             v["q"], v["k"], n, v["w"], v["rp"], v["ci"], EDGES, v["alpha"], v["lse"],
                                             None)

    assert call() == e2f.E2F_EDEVICE
    size = dict(pos=12 * n, gid=4 * n, q=4 * n * H * DK, k=4 * n * HK * DK, w=4 * H * 8, rp=8 * (n + 1), ci=4 * EDGES)
    out = dict(alpha=4 * EDGES * H, lse=4 * n * H)
    for o, mine in out.items():
        for i, its in size.items():
            first = base[i].value
            for where in (first, first + its - 4, first - mine + 4):
                assert call(**{o: ctypes.c_void_p(where)}) == e2f.E2F_EINVAL, (o, i)
            for where in (first + its, first - mine):
                assert call(**{o: ctypes.c_void_p(where)}) == e2f.E2F_EDEVICE, (o, i)
    assert call(lse=at(8, 4 * EDGES * H - 4)) == e2f.E2F_EINVAL and call(lse=at(8, 4 * EDGES * H)) == e2f.E2F_EDEVICE
    # columns of one projection: as far as the last atom's features
    wide = dict(ldq=100, ldk=100)
    end = 4 * (9 * 100 + H * DK)
    assert call(wide, alpha=at(3, end - 4)) == e2f.E2F_EINVAL and call(wide, alpha=at(3, end)) == e2f.E2F_EDEVICE
    assert call(dict(wide, dtype=1), alpha=at(3, end // 2)) == e2f.E2F_EDEVICE
    # what is not read may lie anywhere
    assert call(dict(dk=0), alpha=base["q"], lse=base["k"]) == e2f.E2F_EDEVICE


def test_transposed_graph(e2f, ctx):
    base = dict(rp=at(1), ci=at(2), rt=at(3), ct=at(4), pm=at(5), ws=at(6))

    def call(**kw):
        v = {**base, **kw}
        return e2f.lib.e2f_transpose_graph(ctx.handle, n, v["rp"], v["ci"], EDGES, v["rt"], v["ct"], v["pm"], v["ws"],
                                           1 << 19, None)

    assert call() == e2f.E2F_EDEVICE
    for kw in (dict(rt=at(1)), dict(ct=at(2)), dict(pm=at(2, 4 * EDGES - 4)), dict(ct=at(1, 8 * n + 4)), dict(pm=at(4)),
               dict(ct=at(3)), dict(ws=at(1)), dict(ws=at(3)), dict(ws=at(4)), dict(pm=at(6, 16)), dict(ci=at(6))):
        assert call(**kw) == e2f.E2F_EINVAL, kw
    for kw in (dict(ct=at(2, 4 * EDGES)), dict(pm=at(4, 4 * EDGES)), dict(ci=at(1, 8 * (n + 1)))):
        assert call(**kw) == e2f.E2F_EDEVICE, kw


def test_norms(e2f, ctx):
    L, C = 2, 16
    w = 4 * (L + 1) * C
    prm = e2f.NormParams(L, C, 1, 1e-5, 0, at(1).value, at(2).value, at(3).value)

    def fwd(out=at(7), normed=at(8), rstd=at(9)):
        return e2f.lib.e2f_block_norm_forward(ctx.handle, ctypes.byref(prm), at(4), at(5), at(6), n, out, normed, rstd,
                                              None)

    assert fwd() == e2f.E2F_EDEVICE
    for slot in (1, 2, 3):  # the weights are inputs too
        for name in ("out", "normed", "rstd"):
            assert fwd(**{name: at(slot)}) == e2f.E2F_EINVAL and fwd(**{name: at(slot, w - 4)}) == e2f.E2F_EINVAL
            assert fwd(**{name: at(slot, w)}) == e2f.E2F_EDEVICE
    need = ctypes.c_size_t(0)
    assert e2f.lib.e2f_block_norm_workspace_size(ctx.handle, ctypes.byref(prm), n, ctypes.byref(need)) == e2f.E2F_OK

    def bwd(ws=at(20), gx=at(13), gp=at(16)):
        return e2f.lib.e2f_block_norm_backward(ctx.handle, ctypes.byref(prm), at(4), at(5), at(6), at(9), n, at(10),
                                               at(11), gx, at(14), at(15), gp, at(17), at(18), ws, need.value, None)

    assert bwd() == e2f.E2F_EDEVICE
    for slot in (1, 2, 3, 4, 5, 6, 9, 10, 11, 13, 14, 15, 16, 17, 18):  # the workspace over any of them
        assert bwd(ws=at(slot)) == e2f.E2F_EINVAL, slot
    assert bwd(gx=at(20, need.value - 4)) == e2f.E2F_EINVAL and bwd(gx=at(20, need.value)) == e2f.E2F_EDEVICE
