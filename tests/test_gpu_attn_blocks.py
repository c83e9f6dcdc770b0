"""Attention over the cache with block scales against its definition in 64 bits,
within a bound that counts its roundings (runtime_scales.attn_bound)."""
import numpy as np
import pytest

from tests import generation as gen
from tests import runtime_scales as rs

pytestmark = pytest.mark.gpu

TYPES = ["float32", "bfloat16", "float16"]
HALF = {"float32": 2.0 ** -24, "bfloat16": 2.0 ** -8, "float16": 2.0 ** -11}


def _pool(rng, n, G, page, D, block):
    """Codes and scales as an append makes them of normal values."""
    out = []
    for _ in range(2):
        x = rng.standard_normal((n, G, page // block, block, D)).astype(np.float32)
        x *= rng.uniform(0.3, 2.0, (n, G, page // block, 1, 1)).astype(np.float32)
        s = rs.scale_of(np.abs(x).max((3, 4)))
        c = np.rint(x / s[..., None, None]).astype(np.int8)
        out += [c.reshape(n, G, page, D), s]
    return out


def _queries(rng, T, cols, type, pad, spread=1.0):
    import torch
    x = rng.standard_normal((T, cols + pad)) * spread * rng.uniform(0.2, 2, (T, 1))
    x = torch.from_numpy(x.astype(np.float32)).to(getattr(torch, type))
    return x.cuda()[:, :cols], x[:, :cols].float().numpy()


def _put(cache, batch):
    import torch
    kc, ks, vc, vs = cache
    return ([torch.from_numpy(np.ascontiguousarray(a)).cuda()
             for a in (kc, ks, rs.v_layout(vc), vs)],
            [torch.from_numpy(np.ascontiguousarray(a)).cuda() for a in batch])


def _compare(got, q, cache, batch, scale, type, D, window, sinks):
    import torch
    want, size, most, count = rs.attn_blocks(q, *cache, *batch, scale, window, sinks)
    T, H = size.shape
    vs = cache[3]
    vs = vs[np.isfinite(vs) & (vs > 0)]
    rel, small = rs.attn_bound(size, most, count, D, 32 if type == "float32" else 16,
                               np.abs(np.log2(vs)).max())
    # (a context is a mean of values, whatever the weights are)
    far = 127 * float(vs.max())
    tol = np.minimum(rel, 2 * far * (1 + 2.0 ** -10)) + small * far
    want, got = want.reshape(T, H, D), got.astype(np.float64).reshape(T, H, D)
    tol = np.broadcast_to(tol[:, :, None], want.shape)
    # past the type's largest number the nearest one is infinite (from half a step
    # above it on; fp16 contexts of scales up to 2^30 get there)
    top = float(torch.finfo(getattr(torch, type)).max) * (1 + HALF[type] / 2)
    far = np.abs(want) > top + tol
    assert (got[far] == np.sign(want[far]) * np.inf).all()
    near = np.abs(want) < top - tol
    assert np.isfinite(got[near]).all()
    tol = tol + HALF[type] * (np.abs(want) + tol) + (2.0 ** -25 if type == "float16" else 0.0)
    err = np.abs(got[near] - want[near])
    assert (err <= tol[near]).all(), ((err / tol[near]).max(), np.argwhere(err > tol[near])[:3])


def _check(rng, H, G, D, page, block, new, lens, type, window=0, sinks=0, pad=0, spread=1.0,
           pages=None, edit=None, max_len=0, ws=None, splits=True):
    import torch

    import paper_2408_13933_amd as mq
    starts, lens, pg, pool = gen.batch(rng, new, lens, page)
    pg = pg if pages is None else pages(pg, pool)
    T = int(starts[-1])
    q, qf = _queries(rng, T + 2, H * D, type, pad, spread)
    cache = _pool(rng, pool, G, page, D, block)
    batch = (starts, lens, pg)
    if edit:
        edit(cache, batch, page, block)
    g, i = _put(cache, batch)
    out = torch.full((T + 2, H * D + pad), 7.0, dtype=q.dtype, device="cuda")[:, :H * D]
    scale = float(np.float32(D ** -0.5))
    if not splits:
        ws = torch.empty(0, dtype=torch.uint8, device="cuda")
    mq.mq_paged_attn_blocks(q, *g, *i, scale, window=window, sinks=sinks, max_len=max_len, out=out,
                            workspace=ws)
    got = out.float().cpu().numpy()
    assert (got[T:] == 7).all()  # rows of nobody
    _compare(got[:T], qf[:T], cache, batch, scale, type, D, window, sinks)
    return got[:T]


SHAPES = [(4, 2, 64, 16, 16), (8, 1, 256, 64, 32), (3, 3, 80, 32, 16), (2, 1, 16, 128, 128),
          (8, 4, 128, 64, 64), (1, 1, 48, 1024, 512), (32, 2, 32, 256, 16), (2, 2, 144, 128, 64),
          (4, 1, 176, 32, 32), (6, 2, 208, 16, 16), (2, 1, 240, 64, 16), (4, 4, 96, 64, 32)]


@pytest.mark.parametrize("H,G,D,page,block", SHAPES)
@pytest.mark.parametrize("type", TYPES)
def test_one_token_each(H, G, D, page, block, type):
    rng = np.random.default_rng(D + page)
    lens = [1, 2, 15, 16, 17, 63, 64, 65, 127, 300, 1000] + list(rng.integers(1, 700, 4))
    _check(rng, H, G, D, page, block, [1] * len(lens), lens, type)


@pytest.mark.parametrize("H,G,D,page,block", SHAPES)
@pytest.mark.parametrize("type,pad", [("float32", 1), ("bfloat16", 0), ("float16", 3),
                                      ("bfloat16", 8)])
def test_chunks_and_prompts(H, G, D, page, block, type, pad):
    rng = np.random.default_rng(D * page)
    new = [1, 17, 0, 33, 100, 64]
    lens = [200, 17, 5, 350, 100, 129]
    _check(rng, H, G, D, page, block, new, lens, type, pad=pad)


@pytest.mark.parametrize("type", TYPES)
@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 1), (7, 0), (64, 3), (100, 64), (300, 5),
                                          (5000, 4), (2 ** 31, 2 ** 40), (70, 1000)])
@pytest.mark.parametrize("new", [1, 50])
def test_windows(window, sinks, new, type):
    rng = np.random.default_rng(window + sinks)
    lens = [new, new + 63, 400, 1111]
    _check(rng, 4, 2, 64, 32, 16, [new] * 4, lens, type, window=window, sinks=sinks)


@pytest.mark.parametrize("type", TYPES)
@pytest.mark.parametrize("H,G,D", [(8, 1, 256), (4, 2, 64)])
def test_long_sequences_split(H, G, D, type):
    """With the keys in many parts, in few and in one."""
    rng = np.random.default_rng(11)
    import torch
    for ws in (None, torch.empty(40000, dtype=torch.uint8, device="cuda")):
        _check(rng, H, G, D, 128, 64, [1, 2], [20011, 3000], type, ws=ws)
    _check(rng, H, G, D, 128, 64, [1, 2], [20011, 3000], type, splits=False)
    _check(rng, H, G, D, 128, 64, [40, 2], [5000, 3000], type, max_len=5000)


@pytest.mark.parametrize("D", range(16, 257, 16))
@pytest.mark.parametrize("type", TYPES)
def test_every_head_size_in_parts(D, type):
    """Workspaces that held anything; tiles of many rows, of one to sixteen left over,
    and rows of their own."""
    import torch

    import paper_2408_13933_amd as mq
    for H, new, lens in ((8, [1, 17, 33, 20], [200, 317, 1350, 64]), (2, [1, 2, 8], [3000, 700, 9])):
        n = mq.mq_paged_attn_blocks_workspace_bytes(sum(new) + 2, len(new), H, 1, D, 3008)
        ws = torch.full((n // 4,), float("nan"), device="cuda").view(torch.uint8)
        _check(np.random.default_rng(D), H, 1, D, 64, 32, new, lens, type, ws=ws)


@pytest.mark.parametrize("B", [64, 65, 130, 256, 257, 400])
@pytest.mark.parametrize("H,G,D,type", [(4, 2, 64, "bfloat16"), (2, 2, 32, "float32"),
                                        (8, 1, 144, "float16")])
def test_many_sequences(B, H, G, D, type):
    """Of all lengths, some without new tokens or with several; one long."""
    rng = np.random.default_rng(B)
    new = rng.choice([0, 1, 1, 1, 1, 1, 2, 3], B)
    lens = rng.integers(4, 200, B)
    _check(rng, H, G, D, 16, 16, list(new), list(lens), type)
    _check(rng, H, G, D, 16, 16, list(new), list(lens), type, window=50, sinks=3)
    lens[B // 2] = 9000
    _check(rng, H, G, D, 16, 16, list(new), list(lens), type)


@pytest.mark.parametrize("B", [65, 300])
@pytest.mark.parametrize("type", ["float32", "float16"])
def test_many_prompts(B, type):
    """Tiles of many sequences, with none to forty new tokens each."""
    rng = np.random.default_rng(B)
    new = rng.integers(0, 41, B)
    lens = new + rng.integers(0, 150, B)
    _check(rng, 2, 1, 32, 16, 16, list(new), list(lens), type)
    _check(rng, 2, 1, 32, 16, 16, list(new), list(lens), type, window=30, sinks=2)


def test_sharp_and_flat_logits():
    for spread in (0.0, 1e-20, 30.0, 200.0):
        _check(np.random.default_rng(3), 4, 2, 64, 32, 16, [1, 20], [900, 300], "float32",
               spread=spread)
        _check(np.random.default_rng(4), 4, 2, 64, 32, 16, [1, 20], [900, 300], "bfloat16",
               spread=spread)


@pytest.mark.parametrize("type,spread", [("float32", 1e5), ("float32", 1e7), ("float32", 1e20),
                                         ("bfloat16", 1e5), ("bfloat16", 1e12),
                                         ("float16", 5000.0)])
@pytest.mark.parametrize("D", [32, 96, 256])
def test_huge_logits(type, spread, D):
    """Maxima whose last place is larger than a weight's range (one key has all the
    weight, as far as 32 bits tell)."""
    for new in (1, 40):
        _check(np.random.default_rng(5), 4, 2, D, 32, 16, [new, new], [900, 70], type,
               spread=spread)


@pytest.mark.parametrize("new", [1, 40])
def test_pages_out_of_range_and_short_lists(new):
    def pages(pg, pool):
        pg = pg.copy()
        pg[0, 0], pg[1, 1], pg[2, 2] = -1, pool, 2 ** 31 - 1
        pg[3, :] = -7
        return np.ascontiguousarray(pg[:, :9])
    rng = np.random.default_rng(5)
    got = _check(rng, 4, 2, 64, 16, 16, [new] * 6, [150, 100, 200, 60, 40, 20 if new > 1 else 0],
                 "bfloat16", pages=pages)
    assert (got[3 * new:4 * new] == 0).all()  # a sequence without any place


@pytest.mark.parametrize("type", TYPES)
@pytest.mark.parametrize("new,window", [(1, 0), (30, 0), (1, 20), (30, 20)])
def test_unseen_places_hold_anything(new, window, type):
    """Codes past the last token, scales of blocks that no row sees or that have
    no tokens: NaN, infinities, zeros."""
    def edit(cache, batch, page, block):
        kc, ks, vc, vs = cache
        starts, lens, pg = batch
        used = np.zeros(ks.shape, bool)
        for b, n in enumerate(lens):
            first = n - (starts[b + 1] - starts[b])
            for p in range(int(n)):
                if window == 0 or p > first - window or p < 2:
                    used[pg[b, p // page], :, p % page // block] = True
            if n % block:
                e = int(n - 1)
                kc[pg[b, e // page], :, e % page + 1:e % page + block - e % block] = 127
                vc[pg[b, e // page], :, e % page + 1:e % page + block - e % block] = -128
        bad = np.array([np.nan, np.inf, 0.0, -1.0, 3e38], np.float32)
        for s in (ks, vs):
            s[~used] = np.resize(bad, (~used).sum())
    rng = np.random.default_rng(6)
    _check(rng, 4, 2, 64, 64, 16, [new] * 4, [new, 100, 333, 64], type, edit=edit, window=window,
           sinks=2 if window else 0)


@pytest.mark.parametrize("type", TYPES)
@pytest.mark.parametrize("new", [1, 40])
def test_scales_of_every_size(new, type):
    """Value scales over 60 binary orders, blocks of zeros, key scales that differ."""
    def edit(cache, batch, page, block):
        kc, ks, vc, vs = cache
        r = np.random.default_rng(1)
        vs *= (2.0 ** r.integers(-30, 31, vs.shape)).astype(np.float32)
        ks *= r.uniform(0.01, 3, ks.shape).astype(np.float32)
        vc[:, :, :block] = 0
        vs[:, :, 0] = rs.scale_of(0.0)
    _check(np.random.default_rng(7), 4, 2, 64, 64, 16, [new] * 3, [new, 100, 700], type, edit=edit)


@pytest.mark.parametrize("type", TYPES)
def test_bad_queries_do_not_spread(type):
    import torch

    import paper_2408_13933_amd as mq
    rng = np.random.default_rng(8)
    for new in (1, 5, 60):
        H, G, D = 4, 2, 64
        starts, lens, pg, pool = gen.batch(rng, [new] * 3, [200, 70, 90], 16)
        q, _ = _queries(rng, 3 * new, H * D, type, 0)
        g, i = _put(_pool(rng, pool, G, 16, D, 16), (starts, lens, pg))
        g[0][:, 0, :, 100 - 64] = -5  # every product with the infinity is -infinity
        good = mq.mq_paged_attn_blocks(q, *g, *i, 0.125)
        q2 = q.clone()
        q2[new, 3], q2[0, 100] = float("nan"), float("inf")
        y = mq.mq_paged_attn_blocks(q2, *g, *i, 0.125).view(-1, H, D)
        nan = torch.isnan(y)
        assert nan[new, 0].all() and nan[0, 1].all() and nan.sum() == 2 * D
        assert torch.equal(y[~nan], good.view(-1, H, D)[~nan])


@pytest.mark.parametrize("type", ["float32", "bfloat16"])
def test_offsets_past_32_bits(type):
    """A pool of more than 2^32 codes with the sequence's pages at its end."""
    import torch

    import paper_2408_13933_amd as mq
    G, D, page, block, n = 8, 256, 1024, 1024, 2100
    rng = np.random.default_rng(9)
    small = _pool(rng, 3, G, page, D, block)
    g, _ = _put(small, [])
    big = []
    for a in g:
        t = torch.zeros((n,) + tuple(a.shape[1:]), dtype=a.dtype, device="cuda")
        t[n - 3:] = a
        big.append(t)
    assert big[0].numel() > 2 ** 32
    for new in (1, 30):
        q, qf = _queries(rng, new, 16 * D, type, 0)
        batch = [np.array(a, np.int32) for a in ([0, new], [2500], [[2, 0, 1]])]
        at = [torch.from_numpy(a).cuda() for a in batch]
        at[2] += n - 3
        y = mq.mq_paged_attn_blocks(q, *big, *at, 1 / 16)
        _compare(y.float().cpu().numpy(), qf, small, batch, 1 / 16, type, D, 0, 0)
        # appending there too
        k = torch.randn(new, G * D, device="cuda").to(q.dtype)
        want = [a.clone() for a in g]
        lo = [b.to(torch.int32) for b in at]
        mq.mq_rope_append_blocks(q, k, k, *big, *lo)
        lo[2] = lo[2] - (n - 3)
        mq.mq_rope_append_blocks(q, k, k, *want, *lo)
        for a, b in zip(big, want):
            assert torch.equal(a[n - 3:], b) and not a[:n - 3:97].any()
        small = [a.cpu().numpy() for a in want]
        small[2] = rs.v_rows(small[2])
        g = want


def test_captured_and_on_another_stream():
    """Graphs of append and attention with a workspace of their own each, replayed
    with eager calls between."""
    import torch

    import paper_2408_13933_amd as mq
    rng = np.random.default_rng(10)
    H, G, D, page = 8, 2, 64, 32
    runs = []
    for new, L in ((1, 3000), (70, 500)):
        starts, lens, pg, pool = gen.batch(rng, [new] * 2, [L, L - 20], page)
        g, i = _put(_pool(rng, pool, G, page, D, 16), (starts, lens, pg))
        x = [torch.randn(2 * new, c * D, device="cuda").to(torch.bfloat16) for c in (H, G, G)]
        n = mq.mq_paged_attn_blocks_workspace_bytes(2 * new, 2, H, G, D, L)
        ws = torch.empty(max(n, 256), dtype=torch.uint8, device="cuda")
        out = torch.empty_like(x[0])
        rot = torch.empty_like(x[0])
        table = mq.mq_rope_table(L, D)

        def go(g=g, i=i, x=x, ws=ws, out=out, rot=rot, table=table, L=L):
            mq.mq_rope_append_blocks(*x, *g, *i, table=table, out=rot)
            mq.mq_paged_attn_blocks(rot, *g, *i, 0.125, max_len=L, out=out, workspace=ws)
        go()
        torch.cuda.synchronize()
        runs.append((go, out, out.clone()))
    stream = torch.cuda.Stream()
    graphs = []
    for go, out, want in runs:
        stream.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(stream):
            go()
        torch.cuda.synchronize()
        assert torch.equal(out, want)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            go()
        graphs.append(graph)
    for _ in range(3):
        for (go, out, want), graph in zip(runs, graphs):
            out.zero_()
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(out, want)
            out.zero_()
            go()
            torch.cuda.synchronize()
            assert torch.equal(out, want)


def test_binding_refuses():
    import torch

    import paper_2408_13933_amd as mq
    rng = np.random.default_rng(12)
    starts, lens, pg, pool = gen.batch(rng, [1, 1], [20, 30], 32)
    g, i = _put(_pool(rng, pool, 2, 32, 64, 16), (starts, lens, pg))
    q = torch.zeros(2, 256, device="cuda", dtype=torch.float16)
    names = ("k_cache", "k_scale", "v_cache", "v_scale", "starts", "lens", "pages")
    ok = dict(zip(names, g + i), q=q, logit_scale=0.125)
    mq.mq_paged_attn_blocks(**ok)
    bad = [dict(q=q.double()), dict(q=q.cpu()), dict(q=q[:, :100]), dict(q=q[0]),
           dict(k_cache=g[0].float()), dict(k_cache=g[0][0]), dict(v_cache=g[2].view(pool, 2, 64, 32)),
           dict(k_scale=g[1][:, :, :1].contiguous()), dict(v_scale=g[3].double()),
           dict(k_scale=g[1].cpu()), dict(starts=i[0].long()), dict(lens=i[1][:1]),
           dict(pages=i[2].cpu()), dict(out=q.float()), dict(workspace=q)]
    for kw in bad:
        with pytest.raises(ValueError):
            mq.mq_paged_attn_blocks(**{**ok, **kw})
    for kw in (dict(logit_scale=-1.0), dict(window=-1), dict(sinks=-1), dict(max_len=-1)):
        with pytest.raises(mq.MQError):
            mq.mq_paged_attn_blocks(**{**ok, **kw})
    x = q[:, :128].contiguous()
    for kw in (dict(k=x.float()), dict(v=x[:, :64]), dict(table=q), dict(out=q.float())):
        a = {**dict(zip(names, g + i)), "q": q, "k": x, "v": x, **kw}
        with pytest.raises(ValueError):
            mq.mq_rope_append_blocks(**a)
