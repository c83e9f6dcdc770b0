"""mq_sample against the plain form of generation.py (Python integers for the
weights and their sums): tokens equal.  The weights are evaluated within 2^-46,
so a token could differ only where u times the total falls within about 2^-40
of a border; equal weights give exact borders on both sides."""
import numpy as np
import pytest

from tests import generation as gen

pytestmark = pytest.mark.gpu
INF = np.inf


def _mq():
    import paper_2408_13933_amd as mq
    return mq


def _run(x, u, t=None, k=None, p=None, floor=None, alpha=1.0, zp=0, ld=None, workspace=None):
    mq = _mq()
    import torch

    def dev(a, dt):
        return None if a is None else torch.from_numpy(np.asarray(a, dt)).cuda()

    x = np.asarray(x)
    g = torch.from_numpy(np.ascontiguousarray(x)).cuda()
    if ld:
        w = torch.zeros((x.shape[0], ld + 1), dtype=g.dtype, device="cuda")
        w[:, 1:1 + x.shape[1]] = g
        g = w[:, 1:1 + x.shape[1]]
    ws = None if workspace is None else torch.empty(workspace, dtype=torch.uint8, device="cuda")
    y = mq.mq_sample(g, dev(u, np.float32), dev(t, np.float32), dev(k, np.int32),
                     dev(p, np.float32), dev(floor, np.float32), alpha, zp, workspace=ws)
    torch.cuda.synchronize()
    real = x.astype(np.float64)
    if x.dtype == np.int16:
        real = gen.f32(alpha) * (real - zp)

    def one(a, m, dt, off):
        return off if a is None else float(np.asarray(a, dt)[m])

    want = [gen.sample_row(real[m], one(u, m, np.float32, 0), one(t, m, np.float32, 1.0),
                           int(one(k, m, np.int32, 0)), one(p, m, np.float32, 1.0),
                           one(floor, m, np.float32, 0.0)) for m in range(len(x))]
    assert y.cpu().numpy().tolist() == want
    return want


SETTINGS = [dict(), dict(k=1), dict(k=50), dict(p=0.9), dict(p=0.3), dict(floor=0.05),
            dict(k=20, p=0.8), dict(k=200, p=0.95, floor=0.02), dict(p=0.9, floor=0.3),
            dict(t=0.0), dict(t=0.3, k=9), dict(t=1.7, p=0.95)]


def _settings(names, M, rng):
    """Every row its own settings, drawn from SETTINGS."""
    rows = [SETTINGS[i] for i in rng.integers(0, len(SETTINGS), M)]
    off = dict(t=1.0, k=0, p=1.0, floor=0.0)
    return {n: [r.get(n, off[n]) for r in rows] for n in names}


@pytest.mark.parametrize("V", [1, 2, 63, 64, 65, 1000, 2048, 2049, 5000, 32000, 50257])
def test_settings_over_sizes(V):
    rng = np.random.default_rng(V)
    M = 24
    x = (rng.standard_normal((M, V)) * 2.5).astype(np.float32)
    u = rng.random(M)
    for kw in SETTINGS[:9] if V < 3000 else SETTINGS[2:9:2]:
        _run(x, u, **{n: [v] * M for n, v in kw.items()})
    _run(x, u, **_settings(("t", "k", "p", "floor"), M, rng))


@pytest.mark.parametrize("V", [1, 100, 2500, 32000])
def test_codes(V):
    """16-bit codes: many ties at the same code."""
    rng = np.random.default_rng(V)
    M = 16
    for std in (3000, 3, 0.3):
        x = np.clip(np.rint(rng.standard_normal((M, V)) * std), -32768, 32767).astype(np.int16)
        _run(x, rng.random(M), alpha=6e-4, zp=-77, **_settings(("t", "k", "p", "floor"), M, rng))


@pytest.mark.parametrize("V", [40, 3000, 9000])
def test_ties_go_to_the_lowest_index(V):
    """All equal, two values, a tie group cut by top_k and by top_p."""
    rng = np.random.default_rng(V)
    u = [0.0, 0.25, 0.5, 0.999, 1.0 - 2.0 ** -24]
    flat = np.zeros((5, V), np.float32)
    for kw in (dict(), dict(k=[7] * 5), dict(p=[0.5] * 5), dict(k=[30] * 5, p=[0.34] * 5),
               dict(floor=[1.0] * 5), dict(t=[0.0] * 5)):
        _run(flat, u, **kw)
    two = np.where(rng.random((5, V)) < 0.3, 1.0, 0.5).astype(np.float32)
    for k in (3, V // 3, V // 2, V - 1, V, V + 1):
        _run(two, u, k=[k] * 5)
    for p in (0.1, 0.4, 0.6, 0.9):
        _run(two, u, p=[p] * 5)
        _run(two, u, k=[V // 2 + 1] * 5, p=[p] * 5)
    zeros = np.where(rng.random((5, V)) < 0.5, 0.0, -0.0).astype(np.float32)  # -0 equals 0
    _run(zeros, u, k=[5] * 5)


def test_infinities_and_nan():
    V = 3000
    rng = np.random.default_rng(1)
    x = (rng.standard_normal((12, V)) * 3).astype(np.float32)
    x[0] = -INF                         # nothing can be drawn
    x[1] = np.nan
    x[2, :] = -INF
    x[2, 2999] = -3.0                   # one word left
    x[3, ::2] = -INF                    # masked by a grammar
    x[4, 5:2990] = np.nan
    x[5, [17, 900]] = INF               # only these have weight
    x[6, 100] = 3e38
    x[7, :] = -3e38
    x[7, 8] = -2.9e38
    x[8] = 1e-42                        # subnormal
    x[8, 7] = 2e-42
    x[9, :50] = -INF
    u = rng.random(12)
    for kw in (dict(), dict(k=[4] * 12), dict(p=[0.7] * 12), dict(floor=[0.1] * 12),
               dict(t=[0.0] * 12), dict(k=[2999] * 12, p=[0.99] * 12)):
        got = _run(x, u, **kw)
        assert got[0] == got[1] == -1 and got[2] == 2999


def test_settings_at_their_ends():
    V = 700
    rng = np.random.default_rng(2)
    x = (rng.standard_normal((8, V)) * 2).astype(np.float32)
    u = [0.0, -0.5, 1.0, 2.0, np.nan, 0.3, 0.6, 0.9999999]
    for kw in (dict(t=[0.0, -1.0, np.nan, 1e-30, 1e30, INF, 1e-6, 1.0]),
               dict(k=[0, -5, V, V + 1, 2 ** 31 - 1, 1, 2, V - 1]),
               dict(p=[0.0, -1.0, 1.0, 2.0, np.nan, 1e-30, 0.9999999, 0.5]),
               dict(floor=[0.0, -1.0, 1.0, 5.0, 1e-30, 0.999, 1e-6, np.nan])):
        _run(x, u, **kw)


def test_what_the_lists_do_not_hold():
    """Large top_k, flat rows with top_p, likely words crowded into one
    stretch or one lane's places: the whole row is looked at."""
    V, M = 20000, 6
    rng = np.random.default_rng(3)
    x = (rng.standard_normal((M, V)) * 0.5).astype(np.float32)
    u = rng.random(M)
    _run(x, u, k=[9000] * M)
    _run(x, u, k=[15000] * M, p=[0.9] * M)
    _run(x, u, p=[0.9] * M)
    x[:, 4000:4500] += 6.0
    x[:, 64 * np.arange(100)] += 5.0
    _run(x, u, k=[400] * M)
    _run(x, u, k=[700] * M, p=[0.8] * M, floor=[0.001] * M)
    _run(np.sort(x, axis=1), u, k=[100] * M)
    _run(np.sort(x, axis=1), u, p=[0.8] * M)


@pytest.mark.parametrize("dtype", [np.float32, np.int16])
def test_strided_rows_and_turns(dtype):
    """Rows with a stride and an odd start; a workspace for one row, for a
    few and for all."""
    mq = _mq()
    rng = np.random.default_rng(4)
    M, V = 9, 4099
    x = (rng.standard_normal((M, V)) * (2 if dtype == np.float32 else 4000)).astype(dtype)
    kw = _settings(("t", "k", "p", "floor"), M, rng)
    one = mq.mq_sample_workspace_bytes(1, V)
    got = [_run(x, rng.random(M) * 0 + 0.37, alpha=5e-4, ld=V + 11, workspace=ws, **kw)
           for ws in (one, 2 * one + 300, mq.mq_sample_workspace_bytes(M, V))]
    assert got[0] == got[1] == got[2]


def test_large_vocabulary():
    rng = np.random.default_rng(5)
    M, V = 6, 256000
    x = (rng.standard_normal((M, V)) * 2.5).astype(np.float32)
    _run(x, rng.random(M), t=[0.8, 1.0, 0.0, 1.2, 0.9, 1.0], k=[50, 0, 0, 1000, 0, 0],
         p=[0.95, 0.9, 1.0, 1.0, 0.7, 1.0], floor=[0, 0, 0, 0, 0.05, 0.1])


def test_frequencies():
    """Draws over a grid of u hit each kept word as often as its weight says."""
    mq = _mq()
    import torch
    V, M = 300, 4096
    rng = np.random.default_rng(6)
    row = (rng.standard_normal(V) * 2).astype(np.float32)
    u = ((np.arange(M) + 0.5) / M).astype(np.float32)
    x = torch.from_numpy(row).cuda().repeat(M, 1)
    k = torch.full((M,), 20, dtype=torch.int32, device="cuda")
    y = mq.mq_sample(x, torch.from_numpy(u).cuda(), top_k=k).cpu().numpy()
    w = np.exp(row.astype(np.float64) - row.max())
    keep = np.argsort(-row, kind="stable")[:20]
    prob = np.zeros(V)
    prob[keep] = w[keep] / w[keep].sum()
    count = np.bincount(y, minlength=V)
    # a grid of M points puts M * prob, give or take one, into an interval
    assert (np.abs(count - M * prob) <= 1 + 1e-3).all()


@pytest.mark.parametrize("dtype", ["float32", "int16"])
def test_rows_past_32_bits(dtype):
    """Rows whose offsets in words need more than 32 bits."""
    mq = _mq()
    import torch
    M, V, ld = 4, 5000, 1_500_000_000
    g = torch.Generator(device="cuda").manual_seed(4)
    x = torch.randint(-3000, 3001, (M, V), generator=g, device="cuda").to(getattr(torch, dtype))
    w = torch.empty((M, ld), dtype=x.dtype, device="cuda")[:, :V]
    w.copy_(x)
    u = torch.rand(M, generator=g, device="cuda")
    t = torch.full((M,), 900.0, device="cuda")
    kw = dict(temperature=t, top_p=torch.tensor([1.0, 0.9, 0.5, 1.0], device="cuda"),
              top_k=torch.tensor([0, 0, 700, 20], dtype=torch.int32, device="cuda"))
    want = mq.mq_sample(x, u, **kw)
    assert torch.equal(mq.mq_sample(w, u, **kw), want)
    assert len(set(want.tolist())) == M
