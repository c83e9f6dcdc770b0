"""Appending to the cache with block scales against its definition: queries,
codes and scales bit for bit."""
import numpy as np
import pytest

from tests import generation as gen
from tests import runtime_scales as rs

pytestmark = pytest.mark.gpu

TYPES = ["float32", "bfloat16", "float16"]


def _pool(rng, n, G, page, D, block):
    kc = rng.integers(-127, 128, (n, G, page, D)).astype(np.int8)
    vc = rng.integers(-127, 128, (n, G, page, D)).astype(np.int8)
    ks = rng.uniform(0.005, 0.02, (n, G, page // block)).astype(np.float32)
    vs = rng.uniform(0.005, 0.02, (n, G, page // block)).astype(np.float32)
    return kc, ks, vc, vs


def _rows(rng, T, cols, type, pad):
    import torch
    x = torch.from_numpy(rng.standard_normal((T, cols + pad)).astype(np.float32))
    x = x.to(getattr(torch, type))
    return x.cuda()[:, :cols], x[:, :cols].float().numpy()


def _check(rng, H, G, D, page, block, new, lens, type, pad=0, angles=True, edit=None, pages=None,
           twice=False):
    import torch

    import paper_2408_13933_amd as mq
    starts, lens, pg, pool = gen.batch(rng, new, lens, page)
    pg = pg if pages is None else pages(pg, pool)
    T = int(starts[-1]) + 2  # two rows of nobody
    q, qf = _rows(rng, T, H * D, type, pad)
    k, kf = _rows(rng, T, G * D, type, pad)
    v, vf = _rows(rng, T, G * D, type, pad)
    if edit:
        edit(k, kf), edit(v, vf)
    kc, ks, vc, vs = _pool(rng, pool, G, page, D, block)
    P = max(list(lens) + [1]) - (angles == "short")
    table = mq.mq_rope_table(P, D) if angles and P > 0 else None
    ang = None if table is None else table.cpu().numpy().reshape(P, D // 2, 2)
    g = [torch.from_numpy(a).cuda() for a in (kc, ks, rs.v_layout(vc), vs)]
    i = [torch.from_numpy(np.ascontiguousarray(a)).cuda() for a in (starts, lens, pg)]
    out = torch.full((T, H * D), 7.0, dtype=q.dtype, device="cuda")
    want = np.full((T, H * D), 7.0, np.float32)
    for _ in range(1 + twice):
        mq.mq_rope_append_blocks(q, k, v, *g, *i, table=table, out=out)
        rs.append_blocks(qf, kf, vf, kc, ks, vc, vs, starts, lens, pg, ang, want)
    assert torch.equal(out.cpu(), torch.from_numpy(want).to(q.dtype))
    assert np.array_equal(g[1].cpu().numpy(), ks, equal_nan=True)
    assert np.array_equal(g[3].cpu().numpy(), vs, equal_nan=True)
    assert np.array_equal(g[0].cpu().numpy(), kc)
    assert np.array_equal(rs.v_rows(g[2].cpu().numpy()), vc)


SHAPES = [(4, 2, 64, 16, 16), (8, 1, 256, 64, 32), (3, 3, 80, 32, 16), (2, 1, 16, 128, 128),
          (8, 4, 128, 64, 64), (1, 1, 48, 1024, 512), (5, 5, 32, 256, 16), (2, 2, 256, 128, 128)]


@pytest.mark.parametrize("H,G,D,page,block", SHAPES)
@pytest.mark.parametrize("type", TYPES)
def test_one_token_each(H, G, D, page, block, type):
    rng = np.random.default_rng(D + page)
    lens = list(rng.integers(1, 300, 9)) + [1, block, block + 1, page, page + 1]
    _check(rng, H, G, D, page, block, [1] * len(lens), lens, type, twice=True)


@pytest.mark.parametrize("H,G,D,page,block", SHAPES)
@pytest.mark.parametrize("type,pad", [("float32", 1), ("bfloat16", 0), ("float16", 2),
                                      ("bfloat16", 4), ("bfloat16", 3)])
def test_chunks_and_prompts(H, G, D, page, block, type, pad):
    """Chunks that begin and end anywhere in a block, whole prompts, nothing."""
    rng = np.random.default_rng(D * page)
    new = [1, 15, 16, 17, 0, 40, 300, 2 * block, block - 1, 700]
    lens = [n + int(rng.integers(0, 100)) for n in new]
    lens[6], lens[7], lens[9] = 300, 3 * block, 700
    _check(rng, H, G, D, page, block, new, lens, type, pad=pad)


@pytest.mark.parametrize("type", TYPES)
@pytest.mark.parametrize("angles", [False, "short"])
def test_without_angles_and_past_them(type, angles):
    rng = np.random.default_rng(3)
    _check(rng, 4, 2, 64, 32, 16, [1, 20, 5], [40, 40, 5], type, angles=angles)


def test_lengths_and_pages_out_of_range():
    """Lengths below the new tokens (negative positions) and of zero, page
    entries that name no page, lists that are too short."""
    def pages(pg, pool):
        pg = pg.copy()
        pg[0, 0], pg[1, 1], pg[2, 0] = -1, pool, 2 ** 31 - 1
        return np.ascontiguousarray(pg[:, :3])
    rng = np.random.default_rng(5)
    _check(rng, 4, 2, 64, 16, 16, [3, 30, 9, 40, 1, 7, 2], [3, 50, 9, 100, 0, 4, -5], "bfloat16",
           pages=pages)


@pytest.mark.parametrize("type", TYPES)
def test_special_values(type):
    """Infinities, NaN, zeros, the type's ends."""
    import torch

    def edit(x, f):
        fi = torch.finfo(x.dtype)
        for r, val in ((0, float("nan")), (1, float("inf")), (2, fi.max), (3, fi.tiny), (20, -float("inf"))):
            f[r, 5] = val
            x[r, 5] = val
        x[40:60] = 0.0
        f[40:60] = 0.0
        x[60:64] = float("nan")
        f[60:64] = np.nan
    rng = np.random.default_rng(6)
    _check(rng, 2, 2, 64, 16, 16, [1, 1, 1, 1, 30, 40, 30], [9, 3, 20, 17, 30, 45, 31], type,
           edit=edit, angles=False)
    _check(rng, 2, 2, 64, 16, 16, [1, 1, 1, 1, 30, 40, 30], [9, 3, 20, 17, 30, 45, 31], type,
           edit=edit)


@pytest.mark.parametrize("scale", [0.0, -1.0, float("nan"), float("inf"), 1e-30, 1e30])
def test_a_block_of_unusable_scale(scale):
    """Scales that no append made: not positive and finite counts as 0."""
    import torch

    import paper_2408_13933_amd as mq
    rng = np.random.default_rng(7)
    kc, ks, vc, vs = _pool(rng, 1, 1, 16, 32, 16)
    ks[...] = vs[...] = scale
    x = rng.standard_normal((2, 32)).astype(np.float32)
    g = [torch.from_numpy(a).cuda() for a in (kc, ks, rs.v_layout(vc), vs)]
    starts, lens, pg = (np.array(a, np.int32) for a in ([0, 2], [7], [[0]]))
    i = [torch.from_numpy(a).cuda() for a in (starts, lens, pg)]
    t = torch.from_numpy(x).cuda()
    mq.mq_rope_append_blocks(t, t, t, *g, *i)
    rs.append_blocks(x, x, x, kc, ks, vc, vs, starts, lens, pg, None, x.copy())
    assert np.array_equal(g[0].cpu().numpy(), kc) and np.array_equal(g[1].cpu().numpy(), ks)
    assert np.array_equal(rs.v_rows(g[2].cpu().numpy()), vc)
    assert np.array_equal(g[3].cpu().numpy(), vs)


def test_token_by_token_holds_the_values():
    """A block filled one token at a time: every value is within half a step of
    its block's scale for each time the scale grew, and once for itself."""
    import torch

    import paper_2408_13933_amd as mq
    rng = np.random.default_rng(8)
    G, D, page, n = 2, 64, 32, 32
    x = (rng.standard_normal((n, G * D)) * np.linspace(0.2, 3, n)[:, None]).astype(np.float32)
    g = [torch.from_numpy(a).cuda() for a in (lambda p: (p[0], p[1], rs.v_layout(p[2]), p[3]))(
        _pool(rng, 2, G, page, D, 16))]
    pg = torch.tensor([[1]], dtype=torch.int32).cuda()
    starts = torch.tensor([0, 1], dtype=torch.int32).cuda()
    grew = np.zeros((G, 2))
    before = None
    for t in range(n):
        r = torch.from_numpy(x[t:t + 1]).cuda()
        mq.mq_rope_append_blocks(r, r, r, *g, starts, torch.tensor([t + 1], dtype=torch.int32).cuda(),
                                 pg)
        s = g[1].cpu().numpy()[1]
        if before is not None:
            grew += s != before
        before = s.copy()
    for codes, s in ((g[0].cpu().numpy(), g[1]), (rs.v_rows(g[2].cpu().numpy()), g[3])):
        s = s.cpu().numpy()[1]
        for h in range(G):
            for b in range(2):
                got = codes[1, h, 16 * b:16 * b + 16] * s[h, b]
                want = x[16 * b:16 * b + 16, h * D:(h + 1) * D]
                # (fp32 roundings of inverse and product: 2^-22 of 127 steps)
                assert np.abs(got - want).max() <= s[h, b] * (0.5 * (1 + grew[h, b]) + 1e-4)
