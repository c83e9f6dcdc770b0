"""Penalties, biases and masks on logits against their definition, bit for bit;
with the draw of a token after them."""
import numpy as np
import pytest

from tests import runtime_scales as rs

pytestmark = pytest.mark.gpu

TYPES = ["float32", "bfloat16", "float16"]


def _cuda(a):
    import torch
    return None if a is None else torch.from_numpy(np.ascontiguousarray(a)).cuda()


def _inputs(rng, M, V, hist, nbias, mask, type, pad=0):
    import torch
    x = torch.from_numpy((rng.standard_normal((M, V + pad)) * 4).astype(np.float32))
    x = x.to(getattr(torch, type))
    d = {}
    if hist is not None:
        h = (V * rng.random((M, hist)) ** 3).astype(np.int32)
        h[rng.random((M, hist)) < 0.05] = -1
        h[rng.random((M, hist)) < 0.05] = V
        d["history"] = h
        lens = rng.integers(0, hist + 1, M).astype(np.int32)
        lens[0] = hist
        d["lens"] = lens
        d["prompts"] = (lens * rng.random(M)).astype(np.int32)
        d["repetition"] = rng.uniform(0.7, 1.6, M).astype(np.float32)
        d["presence"] = rng.uniform(-1, 1, M).astype(np.float32)
        d["frequency"] = rng.uniform(-0.2, 0.7, M).astype(np.float32)
        for k, v in (("repetition", 1), ("presence", 0), ("frequency", 0)):
            d[k][M // 2] = v  # a row without penalties
    if nbias is not None:
        n = rng.integers(0, nbias + 1, M)
        n[0] = nbias
        starts = np.concatenate(([0], np.cumsum(n))).astype(np.int32)
        words = rng.integers(-2, V + 2, starts[-1]).astype(np.int32)
        words[::3] = words[0] if len(words) else 0  # one word again and again
        d["bias"] = (starts, words, rng.standard_normal(starts[-1]).astype(np.float32))
    if mask:
        keep = rng.choice([0.0, 0.01, 0.5, 0.97, 1.0], (M, 1))
        bits = rng.random((M, -(-V // 32) * 32)) < keep
        d["mask"] = np.packbits(bits, axis=1, bitorder="little").view(np.int32)
    return x, d


def _call(x, d):
    import paper_2408_13933_amd as mq
    b = d.get("bias")
    return mq.mq_adjust_logits(
        x, history=_cuda(d.get("history")), hist_lens=_cuda(d.get("lens")),
        prompt_lens=_cuda(d.get("prompts")), repetition=_cuda(d.get("repetition")),
        presence=_cuda(d.get("presence")), frequency=_cuda(d.get("frequency")),
        bias=None if b is None else tuple(_cuda(a) for a in b), mask=_cuda(d.get("mask")))


def _check(x, d, V):
    import torch
    g = x.cuda()
    y = _call(g[:, :V], d)
    assert y.data_ptr() == g.data_ptr()
    want = torch.from_numpy(rs.adjust_logits(x[:, :V].float().numpy(), **d)).to(x.dtype)
    assert torch.equal(g[:, :V].cpu().float().nan_to_num(12345.0), want.float().nan_to_num(12345.0))
    assert torch.equal(g[:, V:].cpu(), x[:, V:])


@pytest.mark.parametrize("type", TYPES)
@pytest.mark.parametrize("M,V,pad", [(1, 1, 0), (3, 7, 1), (2, 4095, 0), (5, 4096, 8), (4, 4100, 3),
                                     (2, 32000, 0), (1, 70001, 0), (40, 500, 4)])
@pytest.mark.parametrize("hist,nbias,mask", [(50, None, False), (None, 9, False),
                                             (None, None, True), (301, 40, True), (1, 0, True),
                                             (0, 3, False), (4000, 600, True)])
def test_adjust(M, V, pad, hist, nbias, mask, type):
    rng = np.random.default_rng(M + V)
    x, d = _inputs(rng, M, V, hist, nbias, mask, type, pad)
    _check(x, d, V)


@pytest.mark.parametrize("type", TYPES)
@pytest.mark.parametrize("M,V", [(3, 9000), (2, 40), (70, 5003)])
@pytest.mark.parametrize("hist,nbias", [(16383, None), (16384, 5), (20000, 300), (40, 131070),
                                        (40, 131071), (None, 140000)])
def test_long_histories_and_bias_lists(M, V, hist, nbias, type):
    """Around the most words and entries that counts of a few bits hold; all of a
    row's history the same word."""
    rng = np.random.default_rng(V)
    M = M if (nbias or 0) < 1000 else 1
    x, d = _inputs(rng, M, V, hist, nbias, V > 9, type)
    if hist is not None:
        d["history"][0] = V // 2
        d["prompts"][0] = 0
    _check(x, d, V)


@pytest.mark.parametrize("left", ["prompts", "repetition", "presence", "frequency"])
def test_parts_left_out(left):
    x, d = _inputs(np.random.default_rng(1), 4, 3000, 400, None, False, "float32")
    del d[left]
    _check(x, d, 3000)


def test_special_logits_and_settings():
    """Infinities, NaN and zeros of both signs among penalized, biased and
    forbidden words; zero, infinite and NaN penalties; lengths past the row."""
    V = 5000
    x, d = _inputs(np.random.default_rng(2), 8, V, 2000, 50, True, "float32")
    for i, v in enumerate((np.inf, -np.inf, np.nan, 0.0, -0.0, 3e38, -3e38)):
        x[:, i::97] = float(v)
    d["lens"][1], d["lens"][2] = 2 ** 31 - 1, -5
    d["prompts"][3], d["prompts"][4] = 2 ** 31 - 1, -7
    d["repetition"][5], d["frequency"][6], d["presence"][7] = 0.0, np.inf, np.nan
    with np.errstate(all="ignore"):
        _check(x, d, V)


def test_bias_starts_out_of_range():
    x, d = _inputs(np.random.default_rng(3), 4, 100, None, 10, False, "float32")
    starts, words, values = d["bias"]
    d["bias"] = (np.array([-3, 4, 2, 5, 2 ** 30], np.int32), words, values)
    _check(x, d, 100)


@pytest.mark.parametrize("starts", [(2 ** 31 - 1, 2 ** 31 - 1, 2 ** 31 - 1, 0, 9),
                                    (-2 ** 31, -2 ** 31, 2 ** 31 - 1, -1, 2 ** 31 - 1)])
def test_bias_starts_at_the_ends_of_their_range(starts):
    x, d = _inputs(np.random.default_rng(7), 4, 100, 50, 10, False, "float32")
    d["bias"] = (np.array(starts, np.int64).astype(np.int32),) + d["bias"][1:]
    _check(x, d, 100)


@pytest.mark.parametrize("type", TYPES)
def test_largest_vocabulary_and_row_offsets(type):
    """2^22 words; rows that begin past 2^32 elements."""
    import torch

    import paper_2408_13933_amd as mq
    V = 1 << 22
    x, d = _inputs(np.random.default_rng(4), 1, V, 3000, 100, True, type)
    _check(x, d, V)
    if type != "bfloat16":
        return
    M, V, ld = 3, 1000, 1 << 31
    x, d = _inputs(np.random.default_rng(5), M, V, 300, 10, True, type)
    big = torch.zeros((M - 1) * ld + V, dtype=torch.bfloat16, device="cuda")
    view = big.as_strided((M, V), (ld, 1))
    view.copy_(x.cuda())
    _call(view, d)
    want = torch.from_numpy(rs.adjust_logits(x.float().numpy(), **d)).to(x.dtype)
    assert torch.equal(view.cpu(), want)


def test_captured_and_drawn_from():
    """Adjusting and drawing, eager, on another stream and captured: the same
    tokens, all allowed; a word that a penalty forbids is not drawn again."""
    import torch

    import paper_2408_13933_amd as mq
    M, V = 16, 3000
    x, d = _inputs(np.random.default_rng(6), M, V, 200, 20, True, "float32")
    d["mask"][:, 0] |= 3  # a word each at least
    src = x.cuda()
    buf = torch.empty_like(src)
    u = torch.rand(M, generator=torch.Generator().manual_seed(1)).cuda()
    args = {k: _cuda(d[v]) for k, v in (("history", "history"), ("hist_lens", "lens"),
                                        ("prompt_lens", "prompts"), ("repetition", "repetition"),
                                        ("presence", "presence"), ("frequency", "frequency"),
                                        ("mask", "mask"))}
    args["bias"] = tuple(_cuda(a) for a in d["bias"])
    out = torch.empty(M, dtype=torch.int32, device="cuda")
    ws = torch.empty(mq.mq_sample_workspace_bytes(M, V), dtype=torch.uint8, device="cuda")

    def go():
        buf.copy_(src)
        mq.mq_adjust_logits(buf, **args)
        mq.mq_sample(buf, u, out=out, workspace=ws)

    go()
    torch.cuda.synchronize()
    want, logits = out.clone(), buf.clone()
    bits = np.unpackbits(d["mask"].view(np.uint8), axis=1, bitorder="little")
    assert all(bits[m, t] for m, t in enumerate(want.cpu().numpy()))
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        go()
    torch.cuda.synchronize()
    assert torch.equal(out, want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        go()
    for _ in range(3):
        out.zero_(), buf.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want) and torch.equal(buf, logits)
        go()
        torch.cuda.synchronize()
        assert torch.equal(out, want)


def test_binding_refuses():
    import torch

    import paper_2408_13933_amd as mq
    x = torch.zeros(2, 100, device="cuda")
    i = dict(dtype=torch.int32, device="cuda")
    h, n, f = torch.zeros(2, 5, **i), torch.zeros(2, **i), torch.ones(2, device="cuda")
    ok = dict(logits=x, history=h, hist_lens=n, prompt_lens=n, repetition=f,
              bias=(torch.zeros(3, **i), torch.zeros(4, **i), torch.zeros(4, device="cuda")),
              mask=torch.zeros(2, 4, **i))
    mq.mq_adjust_logits(**ok)
    bad = [dict(logits=x.double()), dict(logits=x.cpu()), dict(logits=x[0]), dict(logits=x.t()),
           dict(history=h.long()), dict(history=h[0]), dict(history=h[:1]), dict(hist_lens=None),
           dict(hist_lens=n[:1]), dict(prompt_lens=f), dict(repetition=n), dict(presence=f[:1]),
           dict(frequency=f.double()), dict(mask=torch.zeros(2, 3, **i)),
           dict(mask=torch.zeros(2, 4, device="cuda")), dict(mask=torch.zeros(1, 4, **i)),
           dict(bias=(torch.zeros(2, **i), torch.zeros(4, **i), torch.zeros(4, device="cuda"))),
           dict(bias=(torch.zeros(3, **i), torch.zeros(4, **i), torch.zeros(3, device="cuda")))]
    for kw in bad:
        with pytest.raises(ValueError):
            mq.mq_adjust_logits(**{**ok, **kw})
