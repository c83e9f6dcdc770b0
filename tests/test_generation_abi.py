"""Refusals of the text-generation entry points (paged key/value cache,
attention over it, sampling): every invalid argument is turned away on the host before
anything is enqueued.  No GPU is touched: the pointers are never read."""
import struct

import pytest

import paper_2408_13933_amd as mq

NZ = 256  # aligned, never dereferenced
INVALID, UNSUPPORTED = 1, 2


def _cache(**kw):
    a = dict(k=NZ, v=NZ, pages=8, page=16, G=2, D=64)
    a.update(kw)
    return struct.pack("qqqiii4x", a["k"] or 0, a["v"] or 0, a["pages"], a["page"], a["G"], a["D"])


def _batch(**kw):
    a = dict(starts=NZ, lens=NZ, table=NZ, B=3, ld=4)
    a.update(kw)
    return struct.pack("qqqqq", a["starts"] or 0, a["lens"] or 0, a["table"] or 0, a["B"], a["ld"])


def append(cache=None, batch=None, no_cache=False, no_batch=False, **kw):
    a = dict(q=NZ, ldq=512, k=NZ, ldk=128, v=NZ, ldv=128, T=5, H=8, aq=0.1, zq=0, aqo=0.1, zqo=0,
             ak=0.1, zk=0, ako=0.1, zko=0, angles=NZ, positions=100, q_out=NZ, ldo=512)
    a.update(kw)
    c = None if no_cache else cache or _cache()
    b = None if no_batch else batch or _batch()
    return mq.lib().mq_rope_append(a["q"], a["ldq"], a["k"], a["ldk"], a["v"], a["ldv"], a["T"],
                                   a["H"], a["aq"], a["zq"], a["aqo"], a["zqo"], a["ak"], a["zk"],
                                   a["ako"], a["zko"], a["angles"], a["positions"], c, b,
                                   a["q_out"], a["ldo"], None)


def attend(cache=None, batch=None, no_cache=False, no_batch=False, **kw):
    a = dict(q=NZ, ldq=512, T=5, H=8, qs=0.1, qz=0, ks=0.1, vs=0.1, vz=0, ls=0.125, window=0,
             sinks=0, os=0.1, oz=0, ob=8, y=NZ, ldy=512, max_len=0, ws=NZ, wsb=0)
    a.update(kw)
    c = None if no_cache else cache or _cache()
    b = None if no_batch else batch or _batch()
    return mq.lib().mq_paged_attn(a["q"], a["ldq"], a["T"], a["H"], a["qs"], a["qz"], c, a["ks"],
                                  a["vs"], a["vz"], b, a["ls"], a["window"], a["sinks"], a["os"],
                                  a["oz"], a["ob"], a["y"], a["ldy"], a["max_len"], a["ws"],
                                  a["wsb"], None)


CACHES = [dict(k=None), dict(v=None), dict(k=NZ + 8), dict(v=NZ + 4), dict(pages=-1),
          dict(pages=1 << 31), dict(page=8), dict(page=24), dict(page=0), dict(page=-16),
          dict(page=2048), dict(G=0), dict(G=3), dict(G=1025), dict(D=8), dict(D=24), dict(D=0),
          dict(D=272)]
BATCHES = [dict(starts=None), dict(lens=None), dict(table=None), dict(B=-1), dict(B=1 << 26),
           dict(ld=-1), dict(ld=(1 << 31) + 1), dict(B=1 << 20, ld=1 << 20)]


@pytest.mark.parametrize("call", [append, attend])
def test_cache_and_batch_are_checked(call):
    assert call(no_cache=True) == INVALID and call(no_batch=True) == INVALID
    for kw in CACHES:
        assert call(cache=_cache(**kw)) == INVALID, kw
    for kw in BATCHES:
        assert call(batch=_batch(**kw)) == INVALID, kw


@pytest.mark.parametrize("kw", [
    dict(q=None), dict(k=None), dict(v=None), dict(q_out=None), dict(T=-1), dict(T=1 << 26),
    dict(H=0), dict(H=7), dict(H=1026), dict(ldq=511), dict(ldk=127), dict(ldv=127), dict(ldo=511),
    dict(ldq=1 << 40), dict(aq=0.0), dict(aqo=-1.0), dict(ak=float("nan")), dict(ako=float("inf")),
    dict(zq=32768), dict(zqo=-32769), dict(zk=40000), dict(zko=128), dict(positions=-1),
    dict(T=(1 << 26) - 1, H=1024, ldq=1 << 16, ldo=1 << 16),
])
def test_append_refuses(kw):
    assert append(**kw) == INVALID


@pytest.mark.parametrize("kw", [
    dict(q=None), dict(y=None), dict(T=-1), dict(T=1 << 26), dict(H=0), dict(H=9), dict(ldq=511),
    dict(ldy=511), dict(ldy=1 << 40), dict(qs=0.0), dict(ks=float("nan")), dict(vs=-0.1),
    dict(ls=0.0), dict(os=float("inf")), dict(qs=1e20, ks=1e20), dict(qz=32768), dict(vz=-129),
    dict(oz=128), dict(ob=16, oz=32768), dict(ob=4), dict(ob=32), dict(window=-1), dict(sinks=-1),
    dict(max_len=-1), dict(wsb=-1), dict(ws=NZ + 16, wsb=4096),
])
def test_attend_refuses(kw):
    assert attend(**kw) == INVALID


def test_more_work_groups_than_a_launch_has():
    many = (1 << 26) - 1
    assert append(T=many) == UNSUPPORTED
    assert append(batch=_batch(B=many)) == UNSUPPORTED
    assert attend(batch=_batch(B=many)) == UNSUPPORTED
    wide = dict(H=1024, ldq=1 << 14, ldy=1 << 14)
    assert attend(T=1 << 20, cache=_cache(G=1024, D=16), **wide) == UNSUPPORTED


def test_nothing_to_do():
    """No rows or no sequences: valid, nothing is read or launched."""
    for call in (append, attend):
        assert call(T=0, q=None) == 0
        assert call(batch=_batch(B=0, starts=None, lens=None, table=None)) == 0


@pytest.mark.parametrize("args", [(-1, 1, 8, 2, 64, 1), (1, -1, 8, 2, 64, 1), (1, 1, 0, 2, 64, 1),
                                  (1, 1, 8, 3, 64, 1), (1, 1, 8, 0, 64, 1), (1, 1, 8, 2, 60, 1),
                                  (1, 1, 8, 2, 272, 1), (1, 1, 8, 2, 64, -1),
                                  (1 << 26, 1, 8, 2, 64, 1)])
def test_attention_workspace_refuses(args):
    assert mq.lib().mq_paged_attn_workspace_bytes(*args) == -1
    with pytest.raises(ValueError):
        mq.mq_paged_attn_workspace_bytes(*args)


def test_attention_workspace_is_bounded():
    for T, B, H, G, D, L in [(1, 1, 32, 4, 64, 1 << 20), (512, 512, 64, 8, 128, 1 << 17),
                             (4096, 1, 32, 4, 64, 4096), (1, 1, 8, 1, 256, 100), (0, 0, 8, 1, 64, 9)]:
        n = mq.mq_paged_attn_workspace_bytes(T, B, H, G, D, L)
        assert 0 <= n <= 64 << 20


def sample(**kw):
    a = dict(x=NZ, bits=32, M=4, V=1000, ld=1000, alpha=0.1, zp=0, t=NZ, k=NZ, p=NZ, mp=NZ, u=NZ,
             y=NZ, ws=NZ, wsb=1 << 20)
    a.update(kw)
    return mq.lib().mq_sample(a["x"], a["bits"], a["M"], a["V"], a["ld"], a["alpha"], a["zp"],
                              a["t"], a["k"], a["p"], a["mp"], a["u"], a["y"], a["ws"], a["wsb"],
                              None)


@pytest.mark.parametrize("kw", [
    dict(x=None), dict(u=None), dict(y=None), dict(ws=None), dict(ws=NZ + 8), dict(wsb=0),
    dict(wsb=-1), dict(wsb=500), dict(bits=8), dict(bits=0), dict(M=-1), dict(M=1 << 31), dict(V=0),
    dict(V=-3), dict(V=(1 << 22) + 1, ld=1 << 23), dict(ld=999), dict(ld=1 << 40),
    dict(bits=16, alpha=0.0), dict(bits=16, alpha=float("nan")), dict(bits=16, zp=40000),
])
def test_sample_refuses(kw):
    assert sample(**kw) == INVALID


def test_sample_nothing_to_do_and_workspace():
    assert sample(M=0, x=None, u=None, y=None, ws=None, wsb=0) == 0
    for args in ((-1, 10), (1, 0), (1, (1 << 22) + 1), (1 << 31, 10)):
        assert mq.lib().mq_sample_workspace_bytes(*args) == -1
        with pytest.raises(ValueError):
            mq.mq_sample_workspace_bytes(*args)
    assert mq.mq_sample_workspace_bytes(0, 10) == 0
    one = mq.mq_sample_workspace_bytes(1, 256000)
    assert 0 < one <= mq.mq_sample_workspace_bytes(512, 256000) <= 64 << 20
    assert sample(V=256000, ld=256000, M=3, wsb=one - 1) == INVALID


def test_binding_checks_tensors():
    import torch
    t = torch.zeros(4)
    for args in (dict(k_cache=t.view(1, 1, 2, 2)), dict(k_cache=t)):
        with pytest.raises(ValueError):
            mq.mq_paged_attn(t, 1.0, 0, args["k_cache"], 1.0, t, 1.0, 0, t, t, t, 1.0, 1.0, 0)
