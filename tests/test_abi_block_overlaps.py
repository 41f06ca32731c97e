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
