"""The calls on 8-bit block matrices and experts without a GPU: bad arguments are refused on the host, before any launch."""
import ctypes as C
import os

import pytest


@pytest.fixture(scope="module")
def mad():
    import paper_2106_10860_amd as m
    if not os.path.exists(m.LIB_PATH):
        from paper_2106_10860_amd.build import build
        build()
    return m


FAKE = 0x10000        # never dereferenced: every call below fails validation first, or has nothing to do


def refused(mad, status, expected, text=""):
    assert status == expected, mad.lib().maddness_last_error().decode()
    if text:
        assert text in mad.lib().maddness_last_error().decode()


def test_quantise_blocks_refuses(mad):
    base = dict(x=FAKE, dtype=2, count=1, rows=4, cols=200, ldx=200, stride_x=0, tile=1, source=None, source_rows=0, repeat=1, factors=None,
                q=FAKE, ldq=208, scale=FAKE, lds=4, qt=None, ldqt=0, scale_t=None, ldst=0, stream=None)

    def call(**kw):
        return mad.lib().maddness_quantise_blocks(*{**base, **kw}.values())

    inval, unsupported, align = mad.MADDNESS_E_INVAL, mad.MADDNESS_E_UNSUPPORTED, mad.MADDNESS_E_ALIGN
    for kw, status, text in (
            (dict(rows=-1), inval, "negative"), (dict(cols=1 << 31), unsupported, "cols"), (dict(count=-1), inval, "count"),
            (dict(count=70000), unsupported, "count"), (dict(tile=64), inval, "tile"), (dict(dtype=3), inval, "dtype"),
            (dict(x=None), inval, "NULL"), (dict(ldx=199), inval, "stride"), (dict(x=FAKE + 1), align, "element"), (dict(q=None), inval, "both"),
            (dict(scale=None), inval, "NULL"), (dict(ldq=192), inval, "ld"), (dict(ldq=200), align, "16"), (dict(q=FAKE + 8), align, "16"),
            (dict(lds=1), inval, "lds"), (dict(lds=6), align, "4"), (dict(scale=FAKE + 2), align, "4"), (dict(factors=FAKE), inval, "source"),
            (dict(source=FAKE, count=2), inval, "one matrix"), (dict(source=FAKE, source_rows=4, repeat=0), inval, "repeat"),
            (dict(source=FAKE, source_rows=1 << 20, repeat=1 << 20), unsupported, "repeat"), (dict(qt=FAKE, ldqt=16), inval, "qt"),
            (dict(source=FAKE + 2, source_rows=4), align, "4-byte")):
        refused(mad, call(**kw), status, text)
    for kw in (dict(rows=0), dict(cols=0, x=None), dict(count=0)):
        refused(mad, call(**kw), mad.MADDNESS_OK)


def test_block_product_refuses(mad):
    M, inval, unsupported, align = mad._BlockMatrix, mad.MADDNESS_E_INVAL, mad.MADDNESS_E_UNSUPPORTED, mad.MADDNESS_E_ALIGN

    def matrix(**kw):
        return M(**{**dict(data=FAKE, dtype=16, tile=1, rows=20, cols=300, ld=304, stride=0, scale=FAKE, lds=4, scale_stride=0), **kw})

    def call(A=None, B=None, by=0, groups=1, offsets=None, source=None, slots=0, repeat=1, out=FAKE, dtype=2, ldo=30, work=None, size=0):
        A, B = A or matrix(), B or matrix(rows=30, tile=128)
        return mad.lib().maddness_block_product(C.byref(A), C.byref(B), by, groups, offsets, source, slots, repeat, out, dtype, ldo, work, size, None)

    for kw, status, text in (
            (dict(by=3), inval, "by"), (dict(A=matrix(rows=-1)), inval, "negative"), (dict(A=matrix(cols=299)), inval, "columns"),
            (dict(A=matrix(tile=2)), inval, "tile"), (dict(A=matrix(ld=300)), align, "16"), (dict(A=matrix(ld=288)), inval, "ld"),
            (dict(A=matrix(data=FAKE + 4)), align, "16"), (dict(A=matrix(lds=2)), inval, "lds"), (dict(A=matrix(scale=None)), inval, "NULL"),
            (dict(B=matrix(rows=30, dtype=2)), unsupported, "E4M3"), (dict(A=matrix(dtype=3)), inval, "dtype"), (dict(dtype=16), inval, "out"),
            (dict(out=None), inval, "out"), (dict(ldo=29), inval, "out"), (dict(out=FAKE + 1), align, "out"), (dict(by=1, groups=0), inval, "groups"),
            (dict(by=1, groups=70000, offsets=FAKE), unsupported, "groups"), (dict(by=1, groups=3), inval, "offsets"),
            (dict(by=1, groups=3, offsets=FAKE + 2), align, "offsets"), (dict(by=2, groups=3, offsets=FAKE), inval, "tile 1"),
            (dict(source=FAKE, slots=5), inval, "source"), (dict(by=1, groups=3, offsets=FAKE, source=FAKE, slots=5, repeat=0), inval, "repeat"),
            (dict(by=1, groups=3, offsets=FAKE, source=FAKE, slots=-1), inval, "slots"), (dict(by=1, groups=3, offsets=FAKE, source=FAKE + 1, slots=5), align, "source"),
            (dict(by=1, groups=3, offsets=FAKE, source=FAKE, slots=5, repeat=1 << 30), unsupported, "repeat"),
            (dict(A=matrix(dtype=2), by=2, groups=3, offsets=FAKE), unsupported, "E4M3"),
            (dict(A=matrix(dtype=2, rows=500)), unsupported, "workspace"),
            (dict(A=matrix(dtype=2, rows=500), work=FAKE + 4, size=1 << 20), align, "workspace")):
        refused(mad, call(**kw), status, text)
    assert mad.lib().maddness_block_product(None, None, 0, 1, None, None, 0, 1, FAKE, 2, 30, None, 0, None) == inval
    refused(mad, call(A=matrix(rows=0)), mad.MADDNESS_OK)
    need = mad.lib().maddness_block_product_workspace
    assert need(500, 300, 0, 2) >= 500 * 304 + 500 * 4 and need(500, 300, 0, 16) == 0 and need(0, 300, 0, 2) == 0


def test_route_and_order_refuse(mad):
    L, inval, unsupported, align = mad.lib(), mad.MADDNESS_E_INVAL, mad.MADDNESS_E_UNSUPPORTED, mad.MADDNESS_E_ALIGN
    base = dict(logits=FAKE, dtype=0, T=5, E=64, ldl=64, bias=None, scores=0, groups=8, kept=4, k=6, renormalise=1, factor=1.0, ids=FAKE,
                weights=FAKE, stream=None)

    def route(**kw):
        return L.maddness_route(*{**base, **kw}.values())

    for kw, status, text in (
            (dict(T=-1), inval, "T"), (dict(E=0), unsupported, "E"), (dict(E=1025, ldl=1025), unsupported, "E"), (dict(scores=2), inval, "scores"),
            (dict(k=0), inval, "k"), (dict(k=65), inval, "k"), (dict(k=33), unsupported, "k"), (dict(dtype=3), inval, "dtype"), (dict(ldl=63), inval, "logits"),
            (dict(logits=FAKE + 2), align, "logits"), (dict(groups=7), inval, "groups"), (dict(kept=9), inval, "kept"), (dict(kept=0), inval, "kept"),
            (dict(E=1024, ldl=1024, groups=128), unsupported, "groups"), (dict(ids=None), inval, "ids"), (dict(bias=FAKE + 1), align, "bias")):
        refused(mad, route(**kw), status, text)
    refused(mad, route(T=0, ids=None), mad.MADDNESS_OK)

    def gradient(T=5, k=6, ids=FAKE, dw=FAKE, out=FAKE, ldd=64):
        return L.maddness_route_gradient(FAKE, 0, T, 64, 64, 0, k, 1, 1.0, ids, dw, out, ldd, None)

    refused(mad, gradient(k=65), inval)
    refused(mad, gradient(ids=None), inval, "ids")
    refused(mad, gradient(out=None), inval, "gradient")
    refused(mad, gradient(ldd=60), inval, "gradient")
    refused(mad, gradient(dw=FAKE + 2), align)

    assert L.maddness_order_capacity(10, 4, 128) == 10 + 4 * 127 and L.maddness_order_capacity(2, 64, 128) == 2 + 2 * 127
    need = L.maddness_order_workspace(10, 4)

    def order(slots=10, E=4, align=128, capacity=518, work=FAKE, size=need, offsets=FAKE, source=FAKE):
        return L.maddness_order(FAKE, slots, E, align, offsets, None, source, capacity, FAKE, work, size, None)

    refused(mad, order(slots=-1), inval)
    refused(mad, order(E=2000), unsupported, "E")
    refused(mad, order(align=0), inval, "align")
    refused(mad, order(capacity=517), inval, "capacity")
    refused(mad, order(size=need - 1), unsupported, "workspace")
    refused(mad, order(offsets=None), inval, "offsets")
    refused(mad, order(source=None), inval, "source")
    refused(mad, order(work=FAKE + 2), align)


def test_combine_refuses(mad):
    L, inval, align = mad.lib(), mad.MADDNESS_E_INVAL, mad.MADDNESS_E_ALIGN

    def combine(y=FAKE, rows=9, N=40, ldy=40, place=FAKE, weights=None, T=5, k=2, out=FAKE, dtype=2, ldo=40):
        return L.maddness_combine(y, 2, rows, N, ldy, place, weights, T, k, out, dtype, ldo, None)

    for kw, status in ((dict(k=0), inval), (dict(y=None), inval), (dict(ldy=39), inval), (dict(place=None), inval), (dict(out=None), inval),
                       (dict(ldo=39), inval), (dict(dtype=3), inval), (dict(place=FAKE + 2), align), (dict(weights=FAKE + 2), align), (dict(rows=-1), inval)):
        refused(mad, combine(**kw), status)
    refused(mad, combine(T=0), mad.MADDNESS_OK)
    assert L.maddness_combine_gradient(FAKE, 2, 40, FAKE, 2, 9, 40, 40, FAKE, 5, 2, None, None) == inval
    assert L.maddness_combine_gradient(FAKE, 2, 30, FAKE, 2, 9, 40, 40, FAKE, 5, 2, FAKE, None) == inval


def test_python_calls_refuse_host_tensors_and_wrong_types(mad):
    torch = pytest.importorskip("torch")
    x = torch.zeros(4, 32)
    for call in (lambda: mad.maddness_quantise_blocks(x), lambda: mad.maddness_route(x, 2), lambda: mad.BlockMatrix(x, x),
                 lambda: mad.maddness_block_product(x, x), lambda: mad.maddness_combine(x, torch.zeros(4, 1, dtype=torch.int32)),
                 lambda: mad.maddness_order(torch.zeros(4, dtype=torch.int32), 3)):
        with pytest.raises(TypeError):
            call()


def test_product_by_choice_refuses(mad):
    M, inval, unsupported, align = mad._BlockMatrix, mad.MADDNESS_E_INVAL, mad.MADDNESS_E_UNSUPPORTED, mad.MADDNESS_E_ALIGN
    A, B = (M(data=FAKE, dtype=16, tile=1, rows=rows, cols=300, ld=304, stride=0, scale=FAKE, lds=4, scale_stride=0) for rows in (20, 30))

    def call(groups=4, source=FAKE, slots=40, repeat=2, out=FAKE):
        return mad.lib().maddness_block_product(C.byref(A), C.byref(B), 4, groups, None, source, slots, repeat, out, 2, 30, None, 0, None)

    for kw, status, text in (
            (dict(slots=-1), inval, "slots"), (dict(slots=513, repeat=100), unsupported, "slots"), (dict(repeat=0), inval, "repeat"),
            (dict(slots=41), inval, "rows"), (dict(source=None), inval, "source"), (dict(source=FAKE + 2), align, "source"),
            (dict(groups=0), inval, "groups"), (dict(groups=70000), unsupported, "groups"), (dict(out=None), inval, "out")):
        refused(mad, call(**kw), status, text)
    refused(mad, call(slots=0, source=None), mad.MADDNESS_OK)
