"""Refusals of the entry points whose scales are found at run time: every
invalid argument is turned away on the host before anything is enqueued.  No
GPU is touched: the pointers are never read."""
import pytest

import paper_2408_13933_amd as mq

NZ = 256  # aligned, never dereferenced
INVALID, UNSUPPORTED = 1, 2
NAN = float("nan")


def quantize(**kw):
    a = dict(x=NZ, type=1, M=4, K=64, ldx=64, q=NZ, s=NZ, r=NZ)
    a.update(kw)
    return mq.lib().mq_quantize_tokens(a["x"], a["type"], a["M"], a["K"], a["ldx"], a["q"], a["s"],
                                       a["r"], None)


@pytest.mark.parametrize("kw", [
    dict(x=None), dict(q=None), dict(s=None), dict(type=-1), dict(type=3), dict(M=-1),
    dict(M=1 << 24), dict(K=0), dict(K=-5), dict(K=65537, ldx=1 << 17), dict(ldx=63),
    dict(ldx=1 << 40)])
def test_quantizer_refuses(kw):
    assert quantize(**kw) == INVALID


def product(**kw):
    a = dict(q=NZ, s=NZ, r=None, M=4, K=64, N=32, w=NZ, bits=8, ws=NZ, zp=None, b=None, y=NZ,
             type=0, wk=None, wkb=0, path=0)
    a.update(kw)
    return mq.lib().mq_qlinear_tokens(a["q"], a["s"], a["r"], a["M"], a["K"], a["N"], a["w"],
                                      a["bits"], a["ws"], a["zp"], a["b"], a["y"], a["type"],
                                      a["wk"], a["wkb"], a["path"], None)


def layer(**kw):
    a = dict(x=NZ, xt=2, ldx=64, M=4, K=64, N=32, w=NZ, bits=8, ws=NZ, zp=None, b=None, y=NZ,
             type=0, wk=NZ, wkb=1 << 20)
    a.update(kw)
    return mq.lib().mq_linear_tokens(a["x"], a["xt"], a["ldx"], a["M"], a["K"], a["N"], a["w"],
                                     a["bits"], a["ws"], a["zp"], a["b"], a["y"], a["type"],
                                     a["wk"], a["wkb"], None)


SHARED = [dict(w=None), dict(ws=None), dict(y=None), dict(type=3), dict(type=-1), dict(bits=5),
          dict(bits=16), dict(M=-1), dict(N=-1), dict(K=0), dict(K=65537), dict(K=63, bits=4),
          dict(wk=NZ + 16, wkb=1 << 20), dict(wkb=-1)]


@pytest.mark.parametrize("kw", SHARED + [
    dict(q=None), dict(s=None), dict(zp=NZ), dict(r=NZ), dict(path=-1), dict(path=4),
    dict(path=22), dict(path=1, M=17)])
def test_product_refuses(kw):
    assert product(**kw) == INVALID


@pytest.mark.parametrize("kw", SHARED + [
    dict(x=None), dict(xt=3), dict(xt=-1), dict(ldx=63), dict(ldx=1 << 40), dict(wk=None),
    dict(wkb=500), dict(M=1 << 24)])
def test_layer_refuses(kw):
    assert layer(**kw) == INVALID


def test_nothing_to_do():
    assert quantize(M=0, x=None, q=None, s=None) == 0
    for kw in (dict(M=0), dict(N=0)):
        assert product(q=None, w=None, y=None, **kw) == 0
        assert layer(x=None, w=None, y=None, wk=None, wkb=0, **kw) == 0


def test_layer_workspace():
    f = mq.mq_linear_tokens_workspace_bytes
    for args in ((-1, 64, 8, 8, 1), (1, 0, 8, 8, 1), (1, 64, -1, 8, 1), (1, 64, 8, 5, 1),
                 (1 << 24, 64, 8, 8, 1)):
        assert mq.lib().mq_linear_tokens_workspace_bytes(*args) == -1
        with pytest.raises(ValueError):
            f(*args)
    assert mq.lib().mq_linear_tokens_workspace_bytes(4, 64, 8, 8, 2) == -1
    # codes, scales and row sums; with a K split the parts too
    assert f(40, 4096, 256, 8, False) >= 40 * (4096 + 8)
    assert f(40, 16384, 256, 8) > f(40, 16384, 256, 8, False)
