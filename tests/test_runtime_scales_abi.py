"""Refusals of the entry points whose scales are found at run time: every
invalid argument is turned away on the host before anything is enqueued.  No
GPU is touched: the pointers are never read."""
import struct

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


def _cache(**kw):
    a = dict(k=NZ, v=NZ, ks=NZ, vs=NZ, pages=8, page=32, block=16, G=2, D=64)
    a.update(kw)
    return struct.pack("qqqqqiiii", *((a[n] or 0) for n in ("k", "v", "ks", "vs", "pages", "page",
                                                            "block", "G", "D")))


def _batch(**kw):
    a = dict(starts=NZ, lens=NZ, table=NZ, B=3, ld=4)
    a.update(kw)
    return struct.pack("qqqqq", a["starts"] or 0, a["lens"] or 0, a["table"] or 0, a["B"], a["ld"])


def append(cache=None, batch=None, no_cache=False, no_batch=False, **kw):
    a = dict(q=NZ, ldq=512, k=NZ, ldk=128, v=NZ, ldv=128, type=1, T=5, H=8, angles=NZ,
             positions=100, q_out=NZ, ldo=512)
    a.update(kw)
    c = None if no_cache else cache or _cache()
    b = None if no_batch else batch or _batch()
    return mq.lib().mq_rope_append_blocks(a["q"], a["ldq"], a["k"], a["ldk"], a["v"], a["ldv"],
                                          a["type"], a["T"], a["H"], a["angles"], a["positions"],
                                          c, b, a["q_out"], a["ldo"], None)


CACHES = [dict(k=None), dict(v=None), dict(ks=None), dict(vs=None), dict(k=NZ + 8), dict(v=NZ + 4),
          dict(pages=-1), dict(pages=1 << 31), dict(page=8, block=8), dict(page=24), dict(page=0),
          dict(page=2048), dict(block=8), dict(block=24), dict(block=64), dict(block=0),
          dict(block=-16), dict(G=0), dict(G=3), dict(G=1025), dict(D=8), dict(D=24), dict(D=0),
          dict(D=272)]
BATCHES = [dict(starts=None), dict(lens=None), dict(table=None), dict(B=-1), dict(B=1 << 26),
           dict(ld=-1), dict(ld=(1 << 31) + 1), dict(B=1 << 20, ld=1 << 20)]


def attend(cache=None, batch=None, no_cache=False, no_batch=False, **kw):
    a = dict(q=NZ, ldq=512, type=1, T=5, H=8, ls=0.125, window=0, sinks=0, y=NZ, ldy=512,
             max_len=0, ws=NZ, wsb=0)
    a.update(kw)
    c = None if no_cache else cache or _cache()
    b = None if no_batch else batch or _batch()
    return mq.lib().mq_paged_attn_blocks(a["q"], a["ldq"], a["type"], a["T"], a["H"], c, b, a["ls"],
                                         a["window"], a["sinks"], a["y"], a["ldy"], a["max_len"],
                                         a["ws"], a["wsb"], None)


CALLS = [append, attend]


@pytest.mark.parametrize("call", CALLS)
def test_cache_and_batch_are_checked(call):
    assert call(no_cache=True) == INVALID and call(no_batch=True) == INVALID
    for kw in CACHES:
        assert call(cache=_cache(**kw)) == INVALID, kw
    for kw in BATCHES:
        assert call(batch=_batch(**kw)) == INVALID, kw


@pytest.mark.parametrize("call", CALLS)
def test_no_rows_or_sequences(call):
    assert call(T=0, q=None) == 0
    assert call(batch=_batch(B=0, starts=None, lens=None, table=None)) == 0


@pytest.mark.parametrize("kw", [
    dict(q=None), dict(k=None), dict(v=None), dict(q_out=None), dict(T=-1), dict(T=1 << 26),
    dict(H=0), dict(H=7), dict(H=1026), dict(ldq=511), dict(ldk=127), dict(ldv=127), dict(ldo=511),
    dict(ldq=1 << 40), dict(type=3), dict(type=-1), dict(positions=-1), dict(angles=NZ + 8),
    dict(T=(1 << 26) - 1, H=1024, ldq=1 << 16, ldo=1 << 16)])
def test_append_refuses(kw):
    assert append(**kw) == INVALID


def test_more_work_groups_than_a_launch_has():
    many = (1 << 26) - 1
    assert append(T=many) == UNSUPPORTED
    assert append(batch=_batch(B=many)) == UNSUPPORTED
    assert attend(batch=_batch(B=many)) == UNSUPPORTED


@pytest.mark.parametrize("kw", [
    dict(q=None), dict(y=None), dict(T=-1), dict(T=1 << 26), dict(H=0), dict(H=9), dict(ldq=511),
    dict(ldy=511), dict(ldy=1 << 40), dict(type=3), dict(type=-1), dict(ls=-0.1), dict(ls=NAN),
    dict(ls=float("inf")), dict(window=-1), dict(sinks=-1), dict(max_len=-1), dict(wsb=-1),
    dict(ws=NZ + 16, wsb=4096)])
def test_attend_refuses(kw):
    assert attend(**kw) == INVALID


def test_attention_workspace():
    f = mq.mq_paged_attn_blocks_workspace_bytes
    for args in [(-1, 1, 8, 2, 64, 1), (1, -1, 8, 2, 64, 1), (1, 1, 0, 2, 64, 1),
                 (1, 1, 8, 3, 64, 1), (1, 1, 8, 2, 60, 1), (1, 1, 8, 2, 272, 1),
                 (1, 1, 8, 2, 64, -1), (1 << 26, 1, 8, 2, 64, 1)]:
        assert mq.lib().mq_paged_attn_blocks_workspace_bytes(*args) == -1
        with pytest.raises(ValueError):
            f(*args)
    for args in [(1, 1, 32, 4, 64, 1 << 20), (512, 512, 64, 8, 128, 1 << 17),
                 (4096, 1, 32, 4, 64, 4096), (1, 1, 8, 1, 256, 100), (0, 0, 8, 1, 64, 9)]:
        assert 0 <= f(*args) <= 64 << 20


def adjust(no_rules=False, **kw):
    a = dict(x=NZ, type=0, M=3, V=100, ld=100, h=NZ, hl=NZ, pl=NZ, ldh=8, cols=8, r=NZ, p=NZ, f=NZ,
             bs=NZ, bt=NZ, bv=NZ, bn=4, m=NZ, ldm=4)
    a.update(kw)
    rules = struct.pack("14q", *((a[n] or 0) for n in ("h", "hl", "pl", "ldh", "cols", "r", "p",
                                                       "f", "bs", "bt", "bv", "bn", "m", "ldm")))
    return mq.lib().mq_adjust_logits(a["x"], a["type"], a["M"], a["V"], a["ld"],
                                     None if no_rules else rules, None)


@pytest.mark.parametrize("kw", [
    dict(no_rules=True), dict(x=None), dict(type=3), dict(type=-1), dict(M=-1), dict(M=1 << 31),
    dict(V=0), dict(V=(1 << 22) + 1, ld=1 << 23, ldm=1 << 20), dict(ld=99), dict(ld=1 << 40),
    dict(hl=None), dict(cols=-1), dict(ldh=7), dict(ldh=1 << 40), dict(bt=None), dict(bv=None),
    dict(bn=-1), dict(bn=1 << 31), dict(ldm=3), dict(ldm=1 << 40)])
def test_adjust_refuses(kw):
    assert adjust(**kw) == INVALID


def test_adjust_nothing_to_do_and_too_much():
    assert adjust(M=0, x=None) == 0
    assert adjust(h=None, bs=None, m=None) == 0
    assert adjust(M=1 << 23) == UNSUPPORTED
    assert adjust(M=1 << 14, V=1 << 22, ld=1 << 22, ldm=1 << 17) == UNSUPPORTED
