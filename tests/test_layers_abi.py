"""The calls around exact layers without a GPU: bad arguments are refused on the host, before any launch."""
import ctypes as C
import math
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


def cases(mad, call, *rows):
    statuses = {"inval": mad.MADDNESS_E_INVAL, "unsupported": mad.MADDNESS_E_UNSUPPORTED, "align": mad.MADDNESS_E_ALIGN}
    for kw, status, text in rows:
        refused(mad, call(**kw), statuses[status], text)


def test_quantise_rows_refuses(mad):
    base = dict(x=FAKE, dtype=2, rows=4, cols=200, ldx=200, q=FAKE, ldq=208, scale=FAKE, stream=None)

    def call(**kw):
        return mad.lib().maddness_quantise_rows(*{**base, **kw}.values())

    cases(mad, call, (dict(rows=-1), "inval", "negative"), (dict(cols=1 << 31), "unsupported", "cols"), (dict(dtype=3), "inval", "dtype"), (dict(x=None), "inval", "NULL"),
          (dict(ldx=199), "inval", "stride"), (dict(x=FAKE + 1), "align", "element"), (dict(q=None), "inval", "NULL"), (dict(scale=None), "inval", "scale"),
          (dict(ldq=192), "inval", "ld"), (dict(ldq=200), "align", "16"), (dict(q=FAKE + 8), "align", "16"), (dict(scale=FAKE + 2), "align", "scale"))
    refused(mad, call(rows=0), mad.MADDNESS_OK)


def test_integer_product_refuses(mad):
    M = mad._IntegerMatrix

    def matrix(**kw):
        return M(**{**dict(data=FAKE, dtype=17, rows=20, cols=300, ld=304, scale=FAKE), **kw})

    def call(A=None, B=None, bias=None, out=FAKE, dtype=2, ldo=30, work=None, size=0):
        A, B = A or matrix(), B or matrix(rows=30)
        return mad.lib().maddness_integer_product(C.byref(A), C.byref(B), bias, out, dtype, ldo, work, size, None)

    deep = 131072
    cases(mad, call, (dict(A=matrix(rows=-1)), "inval", "negative"), (dict(A=matrix(cols=299)), "inval", "columns"), (dict(A=matrix(ld=300)), "align", "16"),
          (dict(A=matrix(ld=288)), "inval", "ld"), (dict(A=matrix(data=FAKE + 4)), "align", "16"), (dict(A=matrix(scale=None)), "inval", "scale"),
          (dict(A=matrix(cols=deep, ld=deep), B=matrix(rows=30, cols=deep, ld=deep)), "unsupported", "131071"), (dict(B=matrix(rows=30, dtype=2)), "unsupported", "I8"),
          (dict(A=matrix(dtype=3)), "inval", "dtype"), (dict(dtype=17), "inval", "out"), (dict(out=None), "inval", "out"), (dict(ldo=29), "inval", "out"),
          (dict(out=FAKE + 1), "align", "out"), (dict(bias=FAKE + 2), "align", "bias"), (dict(A=matrix(dtype=2, rows=500)), "unsupported", "workspace"),
          (dict(A=matrix(dtype=2, rows=500), work=FAKE + 4, size=1 << 20), "align", "workspace"))
    assert mad.lib().maddness_integer_product(None, None, None, FAKE, 2, 30, None, 0, None) == mad.MADDNESS_E_INVAL
    refused(mad, call(A=matrix(rows=0)), mad.MADDNESS_OK)
    refused(mad, call(B=matrix(rows=0), ldo=0), mad.MADDNESS_OK)
    need = mad.lib().maddness_integer_product_workspace
    assert need(500, 300, 2) >= 500 * 304 + 500 * 4 and need(500, 300, 17) == 0 and need(0, 300, 2) == 0 and need(5, 1 << 20, 2) == 0


def test_layer_norm_refuses(mad):
    L = mad.lib()
    base = dict(x=FAKE, dtype=2, rows=4, cols=200, ldx=200, weight=None, bias=None, pd=0, eps=1e-5, out=FAKE, od=2, ldo=200, scale=None, mean=None, rstd=None, stream=None)

    def call(**kw):
        return L.maddness_layer_norm(*{**base, **kw}.values())

    cases(mad, call, (dict(rows=-1), "inval", "rows"), (dict(cols=0), "inval", "mean"), (dict(cols=1 << 31), "unsupported", "cols"), (dict(dtype=17), "inval", "dtype"),
          (dict(x=None), "inval", "NULL"), (dict(ldx=199), "inval", "stride"), (dict(x=FAKE + 1), "align", "element"), (dict(weight=FAKE, pd=9), "inval", "weight"),
          (dict(weight=FAKE + 2), "align", "weight"), (dict(bias=FAKE + 1, pd=2), "align", "bias"), (dict(eps=-1e-9), "inval", "eps"), (dict(eps=math.nan), "inval", "eps"),
          (dict(eps=math.inf), "inval", "eps"), (dict(mean=FAKE), "inval", "together"), (dict(mean=FAKE, rstd=FAKE + 1), "align", "rstd"), (dict(scale=FAKE), "inval", "scale"),
          (dict(od=3), "inval", "out"), (dict(out=None), "inval", "out"), (dict(ldo=199), "inval", "out"), (dict(od=17, ldo=208), "inval", "scale"),
          (dict(od=17, scale=FAKE), "align", "16"))
    refused(mad, call(rows=0), mad.MADDNESS_OK)
    base = dict(g=FAKE, gd=2, ldg=200, x=FAKE, dtype=2, rows=4, cols=200, ldx=200, mean=FAKE, rstd=FAKE, weight=None, pd=0, dx=FAKE, ldd=200, dw=None, db=None, work=None, size=0,
                stream=None)

    def gradient(**kw):
        return L.maddness_layer_norm_gradient(*{**base, **kw}.values())

    need = L.maddness_layer_norm_gradient_workspace
    assert need(0, 10) == 0 and need(4, 0) == 0 and need(4, 200) >= 2 * 200 * 4
    cases(mad, gradient, (dict(cols=0), "inval", "mean"), (dict(g=None), "inval", "gradient"), (dict(gd=3), "inval", "gradient"), (dict(ldg=199), "inval", "gradient"),
          (dict(mean=None), "inval", "mean"), (dict(rstd=FAKE + 2), "align", "rstd"), (dict(weight=FAKE + 1), "align", "weight"), (dict(ldd=199), "inval", "dx"),
          (dict(dx=None), "inval", "both"), (dict(dw=FAKE), "inval", "together"), (dict(dw=FAKE, db=FAKE + 1), "align", "dbias"),
          (dict(dw=FAKE, db=FAKE), "unsupported", "workspace"), (dict(dw=FAKE, db=FAKE, work=FAKE + 8, size=1 << 24), "align", "workspace"),
          (dict(dw=FAKE, db=FAKE, work=FAKE, size=need(4, 200) - 1), "unsupported", "workspace"),
          (dict(cols=2**26 + 1, ldg=2**27, ldx=2**27, ldd=2**27, dw=FAKE, db=FAKE, work=FAKE, size=2**40), "unsupported", "2^26"))
    refused(mad, gradient(rows=0), mad.MADDNESS_OK)


def test_balance_refuses(mad):
    L = mad.lib()
    base = dict(logits=FAKE, dtype=0, T=5000, E=64, ldl=64, scores=0, ids=FAKE, k=2, factor=1.0, loss=FAKE, counts=FAKE, push=FAKE, work=FAKE, size=1 << 24, stream=None)

    def call(**kw):
        return L.maddness_balance(*{**base, **kw}.values())

    cases(mad, call, (dict(T=-1), "inval", "T"), (dict(E=0), "unsupported", "E"), (dict(E=1025, ldl=1025), "unsupported", "E"), (dict(scores=2), "inval", "scores"),
          (dict(dtype=3), "inval", "dtype"), (dict(ldl=63), "inval", "logits"), (dict(logits=FAKE + 2), "align", "logits"), (dict(k=0), "inval", "k"),
          (dict(T=1 << 30, k=4), "unsupported", "T k"), (dict(ids=None), "inval", "NULL"), (dict(loss=None), "inval", "NULL"), (dict(counts=FAKE + 1), "align", "counts"),
          (dict(push=FAKE + 2), "align", "push"), (dict(work=None), "unsupported", "workspace"), (dict(work=FAKE + 4), "align", "workspace"),
          (dict(size=L.maddness_balance_workspace(5000, 64) - 1), "unsupported", "workspace"))
    assert L.maddness_balance_workspace(-1, 64) == 0 and L.maddness_balance_workspace(5, 0) == 0 and L.maddness_balance_workspace(5, 2000) == 0
    base2 = dict(logits=FAKE, dtype=0, T=5, E=64, ldl=64, scores=0, push=FAKE, times=None, add=None, lda=0, out=FAKE, ldd=64, stream=None)

    def gradient(**kw):
        return L.maddness_balance_gradient(*{**base2, **kw}.values())

    cases(mad, gradient, (dict(push=None), "inval", "push"), (dict(times=FAKE + 1), "align", "loss_gradient"), (dict(add=FAKE, lda=63), "inval", "add"),
          (dict(add=FAKE + 2, lda=64), "align", "add"), (dict(out=None), "inval", "gradient"), (dict(ldd=63), "inval", "gradient"))
    refused(mad, gradient(T=0), mad.MADDNESS_OK)


def test_gradient_norm_and_clipping_refuse(mad):
    L = mad.lib()
    need = L.maddness_gradient_norm_workspace()
    assert need > 0

    def table(*rows):
        t = (mad._Tensor * max(len(rows), 1))()
        for i, r in enumerate(rows):
            t[i] = mad._Tensor(**{**dict(data=FAKE + 4096 * i, out=FAKE + 4096 * i, count=100, dtype=0, out_dtype=0), **r})
        return t, len(rows)

    def norm(*rows, n=None, out=FAKE, work=FAKE, size=need):
        t, count = table(*rows)
        return L.maddness_gradient_norm(t, count if n is None else n, out, work, size, None)

    def clip(*rows, top=1.0, out=FAKE, given=0, work=FAKE, size=need):
        t, count = table(*rows)
        return L.maddness_clip_gradients(t, count, top, out, given, work, size, None)

    inval, unsupported, align = mad.MADDNESS_E_INVAL, mad.MADDNESS_E_UNSUPPORTED, mad.MADDNESS_E_ALIGN
    for call in (norm, clip):
        refused(mad, call(dict(count=-1)), inval, "negative")
        refused(mad, call(dict(count=(1 << 40) + 1)), unsupported, "count")
        refused(mad, call(dict(), dict(dtype=3)), inval, "tensor 1")
        refused(mad, call(dict(data=None)), inval, "NULL")
        refused(mad, call(dict(data=FAKE + 2)), align, "tensor 0")
        refused(mad, call(dict(), out=None), inval, "norm")
        refused(mad, call(dict(), out=FAKE + 1), align, "norm")
        refused(mad, call(dict(), work=None), unsupported, "workspace")
        refused(mad, call(dict(), size=need - 1), unsupported, "workspace")
        refused(mad, call(dict(), work=FAKE + 4), align, "workspace")
    refused(mad, norm(dict(), n=-1), inval, "negative")
    assert L.maddness_gradient_norm(None, 2, FAKE, FAKE, need, None) == inval
    refused(mad, clip(dict(), top=-1.0), inval, "max_norm")
    refused(mad, clip(dict(), top=math.nan), inval, "max_norm")
    refused(mad, clip(dict(out=None)), inval, "NULL")
    refused(mad, clip(dict(out_dtype=4)), inval, "dtype")
    # what is written may not be anybody else's: the same tensor twice, overlapping ones, an output that covers another's input, other types in place
    refused(mad, clip(dict(), dict(data=FAKE, out=FAKE)), inval, "tensors 0 and 1 overlap")
    refused(mad, clip(dict(), dict(data=FAKE + 396, out=FAKE + 396)), inval, "overlap")
    refused(mad, clip(dict(out=FAKE + 4096 + 300), dict()), inval, "overlap")
    refused(mad, clip(dict(out=FAKE + 16)), inval, "overlap")
    refused(mad, clip(dict(out_dtype=2)), inval, "overlap")
    refused(mad, clip(dict(count=4000), dict(data=FAKE + 64, out=1 << 30), dict(data=FAKE + 40000, out=FAKE + 40000)), inval, "tensors 0 and 1")
    # the norm within what is read or written
    refused(mad, clip(dict(data=FAKE + 4096, out=FAKE + 8192), out=FAKE + 8192 + 396, given=1, work=None, size=0), inval, "norm lies within tensor 0")
    refused(mad, clip(dict(data=FAKE + 4096, out=FAKE + 8192), out=FAKE + 4096), inval, "norm lies within tensor 0")
    # nothing to do
    refused(mad, clip(given=1, work=None, size=0), mad.MADDNESS_OK)


def test_an_integer_matrix_is_checked_by_every_call(mad):
    """Its tensors can be replaced: what a call finds there is refused as by the constructor."""
    import torch
    W = mad.IntegerMatrix._made(torch.zeros((4, 32), dtype=torch.int8), torch.ones(4))
    with pytest.raises(TypeError, match="device tensors"):
        W._struct
    with pytest.raises(TypeError, match="device tensors"):
        mad.maddness_integer_product(torch.ones((3, 32)), W)
