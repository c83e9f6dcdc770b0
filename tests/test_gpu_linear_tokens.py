"""The token quantizer and the products with a scale per token against their
definitions: codes, scales, sums and outputs bit for bit."""
import numpy as np
import pytest

from tests import runtime_scales as rs

pytestmark = pytest.mark.gpu

TYPES = ["float32", "bfloat16", "float16"]


def _dt(name):
    import torch
    return getattr(torch, name)


def _x(rng, M, K, type, ld=None):
    """Rows of a wider tensor on the GPU and as fp32 numbers."""
    import torch
    x = rng.standard_normal((M, ld or K)).astype(np.float32) * rng.uniform(0.1, 9, (M, 1))
    x[:, rng.integers(0, K)] *= 20
    t = torch.from_numpy(x.astype(np.float32)).to(_dt(type))
    return t.cuda()[:, :K], t[:, :K].float().numpy()


def _weights(rng, N, K, bits, asym):
    lo, hi = (-128, 127) if bits == 8 else (-8, 7)
    w = rng.integers(lo if asym else lo + 1, hi + 1, (N, K)).astype(np.int8)
    ws = rng.uniform(0.001, 0.1, N).astype(np.float32)
    zp = rng.integers(lo, hi + 1, N).astype(np.int32) if asym else None
    return w, ws, zp


def _cuda(a):
    import torch
    return None if a is None else torch.from_numpy(np.ascontiguousarray(a)).cuda()


def _check_quantizer(x, f):
    import torch

    import paper_2408_13933_amd as mq
    sums = torch.full((f.shape[0],), 7, dtype=torch.int32, device="cuda")
    c, s = mq.mq_quantize_tokens(x, rowsum=sums)
    wc, wscale, wsum = rs.quantize_tokens(f)
    assert np.array_equal(s.cpu().numpy(), wscale, equal_nan=True)
    assert np.array_equal(c.cpu().numpy(), wc)
    assert np.array_equal(sums.cpu().numpy(), wsum)
    c2, s2 = mq.mq_quantize_tokens(x)
    assert torch.equal(c, c2) and torch.equal(s.view(torch.int32), s2.view(torch.int32))


@pytest.mark.parametrize("type", TYPES)
@pytest.mark.parametrize("M,K,ld", [(1, 1, 1), (1, 8, 8), (3, 7, 7), (5, 512, 520), (9, 500, 501),
                                    (2, 520, 520), (70, 2048, 2048), (4, 2050, 2050),
                                    (3, 5632, 5632), (2, 8200, 8208), (1, 16384, 16384),
                                    (2, 16392, 16392), (1, 65536, 65536), (1100, 64, 64)])
def test_quantizer(M, K, ld, type):
    _check_quantizer(*_x(np.random.default_rng(M * K), M, K, type, ld))


@pytest.mark.parametrize("type", TYPES)
@pytest.mark.parametrize("K", [33, 512, 4096, 20000])
def test_quantizer_special_rows(K, type):
    """Rows of zeros, with infinities or NaN, of the type's ends, of ties."""
    import torch
    t = _dt(type)
    fi = torch.finfo(t)
    x = torch.zeros((9, K), dtype=t)
    x[1, K // 2] = float("inf")
    x[2, K - 1] = float("nan")
    x[3, 0] = -float("inf")
    x[4] = fi.max
    x[5] = -fi.tiny
    x[6, ::2] = fi.max
    x[6, 1::2] = -fi.max
    x[7] = torch.arange(K).remainder(255).sub(127).to(t) / 2  # halves of a unit scale
    x[7, 0] = 127.0
    x[8, K // 3] = fi.smallest_normal
    _check_quantizer(x.cuda(), x.float().numpy())


CASES = [  # M, K, N, bits, asym, bias
    (1, 16, 1, 8, False, False), (1, 2048, 257, 8, False, True), (1, 2048, 64, 4, True, False),
    (1, 5632, 130, 8, True, True), (1, 16384, 40, 8, False, False), (1, 65536, 9, 8, True, False),
    (1, 100, 33, 8, True, True), (1, 90, 7, 4, False, False), (1, 96, 5000, 4, True, True),
    (2, 64, 3, 8, True, False), (5, 2048, 100, 4, False, True), (16, 5632, 2048, 4, True, False),
    (16, 2048, 4100, 8, False, False), (3, 208, 31, 4, True, False), (7, 33, 50, 8, False, True),
    (17, 256, 65, 8, True, True), (33, 2048, 127, 8, False, False), (100, 1024, 300, 4, True, True),
    (64, 4096, 256, 8, True, False), (40, 16384, 256, 8, False, True), (300, 512, 513, 8, True, False),
    (129, 160, 1000, 4, False, False), (50, 77, 60, 8, True, True), (20, 65536, 70, 8, True, False),
]


@pytest.mark.parametrize("M,K,N,bits,asym,bias", CASES)
@pytest.mark.parametrize("type,out", [("float32", "float32"), ("bfloat16", "bfloat16"),
                                      ("float16", "float32"), ("float32", "float16")])
def test_linear(M, K, N, bits, asym, bias, type, out):
    import torch

    import paper_2408_13933_amd as mq
    rng = np.random.default_rng(M + K + N)
    x, f = _x(rng, M, K, type, K + 16)
    w, ws, zp = _weights(rng, N, K, bits, asym)
    b = rng.standard_normal(N).astype(np.float32) if bias else None
    c, s, sums = rs.quantize_tokens(f)
    want = torch.from_numpy(rs.linear(c, s, w, ws, zp, b)).to(_dt(out))
    gw = _cuda(w if bits == 8 else rs.pack4(w))
    args = (gw, bits, _cuda(ws))
    y = mq.mq_linear_tokens(x, *args, w_zp=_cuda(zp), bias=_cuda(b), out_dtype=_dt(out))
    assert y.dtype == _dt(out) and torch.equal(y.cpu(), want)
    # without a K split, and with a workspace that holds anything
    for splits in (False, True):
        n = mq.mq_linear_tokens_workspace_bytes(M, K, N, bits, splits)
        ws_t = torch.full((n,), 0x5a, dtype=torch.uint8, device="cuda")
        y = mq.mq_linear_tokens(x, *args, w_zp=_cuda(zp), bias=_cuda(b), out_dtype=_dt(out),
                                workspace=ws_t)
        assert torch.equal(y.cpu(), want)
    # on the codes
    y = mq.mq_qlinear_tokens(_cuda(c), _cuda(s), *args, w_zp=_cuda(zp), bias=_cuda(b),
                             a_rowsum=_cuda(sums) if asym else None, out_dtype=_dt(out))
    assert torch.equal(y.cpu(), want)


@pytest.mark.parametrize("bits,asym", [(8, False), (8, True), (4, False), (4, True)])
@pytest.mark.parametrize("out", TYPES)
def test_every_path_gives_the_same_bits(bits, asym, out):
    import torch

    import paper_2408_13933_amd as mq
    rng = np.random.default_rng(bits + asym)
    for M, K, N in ((16, 512, 300), (150, 640, 500), (260, 1024, 512)):
        c = rng.integers(-127, 128, (M, K)).astype(np.int8)
        s = rng.uniform(0.01, 2, M).astype(np.float32)
        s[M // 2] = np.nan
        w, ws, zp = _weights(rng, N, K, bits, asym)
        b = rng.standard_normal(N).astype(np.float32)
        want = torch.from_numpy(rs.linear(c, s, w, ws, zp, b)).to(_dt(out))
        paths = [mq.PATH_AUTO, mq.PATH_PREFILL, mq.PATH_GENERIC]
        paths += [mq.PATH_DECODE] if M <= 16 else []
        paths += [mq.prefill_tile_path(t) for t in range(mq.PREFILL_TILES)]
        for path in paths:
            y = mq.mq_qlinear_tokens(
                _cuda(c), _cuda(s), _cuda(w if bits == 8 else rs.pack4(w)), bits, _cuda(ws),
                w_zp=_cuda(zp), a_rowsum=_cuda(c.sum(1, dtype=np.int32)) if asym else None,
                bias=_cuda(b), out_dtype=_dt(out), path=path)
            ok = torch.equal(torch.nan_to_num(y.cpu().float(), 1e9),
                             torch.nan_to_num(want.float(), 1e9))
            assert ok, (M, path)


@pytest.mark.parametrize("bits,asym", [(8, False), (8, True), (4, False), (4, True)])
@pytest.mark.parametrize("N", [1, 9, 2050, 4095, 4096, 5000, 8191, 8192, 8200, 16383, 16384, 20001])
def test_few_tokens_of_every_width(N, bits, asym):
    """The kernels of 2 to 16 tokens against one thread per output, and the one that
    quantizes too with a workspace that held anything; rows of whole and half chunks."""
    import torch

    import paper_2408_13933_amd as mq
    rng = np.random.default_rng(N + bits)
    for M, K in ((2, 16), (16, 48), (5, 528), (16, 2048), (3, 8208), (16, 16400)):
        if N > 9000 and K > 9000:
            continue
        c = _cuda(rng.integers(-127, 128, (M, K)).astype(np.int8))
        w, ws, zp = _weights(rng, N, K, bits, asym)
        args = (_cuda(w if bits == 8 else rs.pack4(w)), bits, _cuda(ws))
        kw = dict(w_zp=_cuda(zp), bias=_cuda(rng.standard_normal(N).astype(np.float32)))
        sums = c.sum(1, dtype=torch.int32) if asym else None
        a = _cuda(rng.uniform(0.01, 2, M).astype(np.float32))
        y = [mq.mq_qlinear_tokens(c, a, *args, a_rowsum=sums, out_dtype=torch.float32, path=p, **kw)
             for p in (mq.PATH_GENERIC, mq.PATH_AUTO, mq.PATH_DECODE)]
        assert torch.equal(y[0], y[1]) and torch.equal(y[0], y[2]), (M, K)
        x = (c.float() * a[:, None]).to(torch.bfloat16)
        q, s = mq.mq_quantize_tokens(x)
        r = q.sum(1, dtype=torch.int32) if asym else None
        want = mq.mq_qlinear_tokens(q, s, *args, a_rowsum=r, out_dtype=torch.float16,
                                    path=mq.PATH_GENERIC, **kw)
        n = mq.mq_linear_tokens_workspace_bytes(M, K, N, bits)
        work = torch.full((n,), 0x7b, dtype=torch.uint8, device="cuda")
        got = mq.mq_linear_tokens(x, *args, out_dtype=torch.float16, workspace=work, **kw)
        assert torch.equal(got, want), (M, K)


def test_sums_at_the_ends_of_their_range():
    """K = 65536 with codes and zero-points at the ends: 127 * 255 * 65536 < 2^31."""
    import torch

    import paper_2408_13933_amd as mq
    K = 65536
    for M in (1, 3, 18):
        x = torch.full((M, K), 2.0).cuda()
        x[M // 2] = -2.0
        w = torch.full((5, K), 127, dtype=torch.int8).cuda()
        w[1:3] = -128
        ws = torch.full((5,), 0.5).cuda()
        zp = torch.tensor([-128, 127, 0, 3, 127], dtype=torch.int32).cuda()
        y = mq.mq_linear_tokens(x, w, 8, ws, w_zp=zp)
        c, s, _ = rs.quantize_tokens(x.cpu().numpy())
        want = rs.linear(c, s, w.cpu().numpy(), ws.cpu().numpy(), zp.cpu().numpy(), None)
        assert np.abs(rs.token_sums(c, w.cpu().numpy(), zp.cpu().numpy())).max() == 127 * 255 * K
        assert np.array_equal(y.cpu().numpy(), want)


def test_bad_rows_do_not_spread():
    import torch

    import paper_2408_13933_amd as mq
    rng = np.random.default_rng(4)
    for M in (1, 4, 40):
        x, f = _x(rng, M, 256, "bfloat16")
        x[M // 2, 3] = float("nan")
        w, ws, _ = _weights(rng, 70, 256, 8, False)
        y = mq.mq_linear_tokens(x, _cuda(w), 8, _cuda(ws), out_dtype=torch.float32).cpu()
        bad = torch.isnan(y).all(1)
        assert bad[M // 2] and bad.sum() == 1
        assert torch.isfinite(y[~bad]).all()


def test_layers_share_a_workspace_and_a_graph():
    """Layers of different sizes (some with a K split) one after another on one
    workspace, captured and replayed, on a stream of their own."""
    import torch

    import paper_2408_13933_amd as mq
    rng = np.random.default_rng(8)
    shapes = [(40, 16384, 256), (64, 4096, 256), (300, 512, 513), (1, 2048, 64), (9, 512, 100)]
    ws_t = torch.full((32 << 20,), 0x33, dtype=torch.uint8, device="cuda")
    layers = []
    for M, K, N in shapes:
        x, f = _x(rng, M, K, "float16")
        w, ws, zp = _weights(rng, N, K, 8, True)
        c, s, _ = rs.quantize_tokens(f)
        want = torch.from_numpy(rs.linear(c, s, w, ws, zp, None)).to(torch.float16)
        out = torch.empty((M, N), dtype=torch.float16, device="cuda")
        layers.append((x, _cuda(w), _cuda(ws), _cuda(zp), out, want))
    assert any(mq.mq_qlinear_workspace_bytes(*sh) > 0 for sh in shapes)

    def go():
        for x, w, ws, zp, out, _ in layers:
            mq.mq_linear_tokens(x, w, 8, ws, w_zp=zp, out=out, workspace=ws_t)

    def check():
        torch.cuda.synchronize()
        for *_, out, want in layers:
            assert torch.equal(out.cpu(), want)
            out.zero_()

    go()
    check()
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        go()
    check()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        go()
    for _ in range(3):
        graph.replay()
        check()
        go()
        check()


def test_binding_refuses():
    import torch

    import paper_2408_13933_amd as mq
    x = torch.zeros(4, 32, device="cuda")
    w = torch.zeros(8, 32, dtype=torch.int8, device="cuda")
    s = torch.ones(8, device="cuda")
    mq.mq_linear_tokens(x, w, 8, s)
    bad = [dict(x=x.double()), dict(x=x.cpu()), dict(x=x.t()), dict(x=x[0]), dict(w_q=w[:, :16]),
           dict(w_q=w.to(torch.uint8)), dict(w_scale=s[:7]), dict(w_scale=s.double()),
           dict(w_zp=s), dict(bias=s[:3]), dict(out=torch.zeros(4, 9, device="cuda")),
           dict(out=torch.zeros(4, 8, dtype=torch.int32, device="cuda")),
           dict(workspace=torch.zeros(9, device="cuda"))]
    for kw in bad:
        a = dict(x=x, w_q=w, w_bits=8, w_scale=s)
        a.update(kw)
        with pytest.raises(ValueError):
            mq.mq_linear_tokens(**a)
    small = torch.zeros(256, dtype=torch.uint8, device="cuda")
    with pytest.raises(mq.MQError):
        mq.mq_linear_tokens(x, w, 8, s, workspace=small)
    c, a = mq.mq_quantize_tokens(x)
    for kw in (dict(a_scale=a[:3]), dict(a_q=x), dict(w_zp=torch.zeros(8, dtype=torch.int32,
                                                                       device="cuda"))):
        d = dict(a_q=c, a_scale=a, w_q=w, w_bits=8, w_scale=s)
        d.update(kw)
        with pytest.raises((ValueError, mq.MQError)):
            mq.mq_qlinear_tokens(**d)
