"""mq_paged_attn's codes where no rounding tie is near: equal to the plain
form's, without a step's allowance.

exp and the fp64 sums are evaluated within 2^-46, so a code may differ only
* where y / out_scale lies within SLACK of a half: y = v_scale num / den with
  |num| <= 255 den, num and den within 2^-46 (each of den's size), on both
  sides: 4 * 2^-46 * 255 * v_scale / out_scale steps;
* in a row with weights that lie within NEAR of a half: 32512 * 2^-46 < 2^-31 on
  both sides; each may move by 1, num / den by 255 over a den of at least 32512.
"""
import numpy as np
import pytest

from tests import generation as gen

pytestmark = pytest.mark.gpu

NEAR = 2.0 ** -30
VF = (0.031, 5)


def _near_ties(q, fq, k_cache, k_scale, starts, lens, pages, logit_scale, window, sinks):
    """Weights near a half, per row and head [T][H]."""
    _, G, page, D = k_cache.shape
    T, H = q.shape[0], q.shape[1] // D
    sigma = gen.f32(fq[0]) * gen.f32(k_scale) * gen.f32(logit_scale)
    near = np.zeros((T, H), np.int64)
    for b in range(len(lens)):
        pos = np.arange(int(lens[b]))
        for h in range(H):
            keys = k_cache[pages[b, pos // page], h // (H // G), pos % page].astype(np.float64)
            for t in range(starts[b], starts[b + 1]):
                at = int(lens[b]) - int(starts[b + 1]) + t
                see = (pos <= at) & ((window == 0) | (pos > at - window) | (pos < sinks))
                c = keys[see] @ (q[t, h * D:(h + 1) * D].astype(np.float64) - fq[1])
                for i in np.unique(pos[see] // gen.BLOCK):
                    x = c[pos[see] // gen.BLOCK == i]
                    w = gen.ONE * np.exp(sigma * (x - x.max()))
                    near[t, h] += (np.abs(w - np.floor(w) - 0.5) < NEAR).sum()
    return near


def _case(rng, H, G, D, page, new, lens, out_bits=16, q_zp=321, window=0, sinks=0, q_std=3000,
          k_std=30, logit_scale=None, parts=True):
    import torch

    import paper_2408_13933_amd as mq
    starts, lens, pages, pool = gen.batch(rng, new, lens, page)
    T = int(starts[-1])
    fq, k_scale, out_zp = (4.0e-4, q_zp), 0.05, -11
    q = np.clip(np.rint(rng.standard_normal((T, H * D)) * q_std) + q_zp, -32768, 32767)
    q = q.astype(np.int16)
    kc = np.clip(np.rint(rng.standard_normal((pool, G, page, D)) * k_std) + 9, -128, 127)
    kc = kc.astype(np.int8)
    vc = rng.integers(-128, 128, (pool, G, D, page)).astype(np.int8)
    logit_scale = D ** -0.5 if logit_scale is None else logit_scale
    out_scale = 0.03 if out_bits == 8 else 1.2e-4
    dev = [torch.from_numpy(np.ascontiguousarray(a)).cuda() for a in (q, kc, vc, starts, lens, pages)]
    gq, gkc, gvc, gst, gle, gpg = dev
    n = mq.mq_paged_attn_workspace_bytes(T, len(lens), H, G, D, int(lens.max()))
    ws = torch.empty(n if parts else 0, dtype=torch.uint8, device="cuda")
    y = mq.mq_paged_attn(gq, *fq, gkc, k_scale, gvc, *VF, gst, gle, gpg, logit_scale, out_scale,
                         out_zp, out_bits, window=window, sinks=sinks, workspace=ws,
                         max_len=int(lens.max()))
    got = y.cpu().numpy()
    real = gen.paged_attn(q, fq, kc, k_scale, vc, VF, starts, lens, pages, logit_scale, window,
                          sinks)
    want = gen.code(real, out_scale, out_zp, out_bits)
    bad = np.nonzero(got != want)
    if len(bad[0]) == 0:
        return
    near = _near_ties(q, fq, kc, k_scale, starts, lens, pages, logit_scale, window, sinks)
    steps = 255 * VF[0] / out_scale
    slack = steps * (2.0 ** -44 + near[bad[0], bad[1] // D] / gen.ONE)
    v = real[bad] / gen.f32(out_scale)
    # the code of some value within the slack
    lo, hi = (gen.code((v + s) * gen.f32(out_scale), out_scale, out_zp, out_bits)
              for s in (-slack, slack))
    assert ((got[bad] >= lo) & (got[bad] <= hi)).all(), (len(bad[0]), near.sum())


HEADS = [(32, 4, 64), (8, 1, 256), (3, 3, 80), (6, 2, 16), (5, 1, 48), (8, 2, 128), (7, 1, 192),
         (40, 1, 32)]


@pytest.mark.parametrize("H,G,D", HEADS)
@pytest.mark.parametrize("out_bits", [8, 16])
def test_single_tokens(H, G, D, out_bits):
    rng = np.random.default_rng(H + D + out_bits)
    lens = [1, 2, 16, 17, 127, 128, 129, 300, 777]
    for parts in (True, False):
        _case(rng, H, G, D, 32, [1] * len(lens), lens, out_bits=out_bits, parts=parts)


@pytest.mark.parametrize("H,G,D", HEADS)
@pytest.mark.parametrize("out_bits", [8, 16])
def test_chunks(H, G, D, out_bits):
    rng = np.random.default_rng(H + D + out_bits + 1)
    for parts in (True, False):
        _case(rng, H, G, D, 16, [70, 1, 0, 33, 5], [70, 260, 50, 133, 6], out_bits=out_bits,
              parts=parts)


@pytest.mark.parametrize("L", [3000, 9000, 40000])
def test_long_rows_in_parts(L):
    """Joins of up to 8, 64 and 256 parts; sharp and nearly flat logits."""
    rng = np.random.default_rng(L)
    for q_std in (3000, 200):
        _case(rng, 2, 1, 64, 64, [1, 1], [L, L // 3], q_std=q_std)


@pytest.mark.parametrize("window,sinks", [(1, 0), (5, 3), (130, 0), (200, 140), (64, 1000)])
def test_windows(window, sinks):
    rng = np.random.default_rng(window + sinks)
    _case(rng, 4, 2, 64, 16, [1, 40, 3, 1], [700, 500, 3, 129], window=window, sinks=sinks)


@pytest.mark.parametrize("q_zp", [-32768, -900, 0, 128, 32767])
def test_query_zero_points(q_zp):
    rng = np.random.default_rng(abs(q_zp))
    _case(rng, 4, 2, 64, 16, [30, 1], [200, 140], q_zp=q_zp, q_std=25000, logit_scale=0.01)
