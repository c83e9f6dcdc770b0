"""What tells a right attention over the cache with block scales from a wrong one: the
known answers against plausible wrong ones, the spread of errors with one fp16 term."""
import numpy as np
import pytest

from tests import attn_answers as aa
from tests import runtime_scales as rs

TYPES = ["float32", "bfloat16", "float16"]


@pytest.mark.parametrize("type", TYPES)
@pytest.mark.parametrize("keys,low", [(1, False), (2, False), (1, True)])
def test_known_answers_refuse_wrong_ones(keys, low, type):
    k = aa.Known(1, 32, 3, 20, keys, low)
    assert not k.off(k.want, type).any()
    kc, ks, vc, vs = k.cache
    # the definition in 64 bits, logits around 2^26
    y, size, most, count = rs.attn_blocks(k.q, *k.cache, *k.batch, k.scale)
    assert not k.off(y, type).any()
    # zeros, the mean of all values, another key's value (codes differ by a step or more)
    flat, _, _, _ = rs.attn_blocks(0 * k.q, *k.cache, *k.batch, k.scale)
    other = np.roll(k.want, 1, 0)
    for wrong in (np.zeros_like(y), flat, other.reshape(y.shape)):
        assert k.off(wrong, type).mean() > 0.9


@pytest.mark.parametrize("D,new,L", [(64, 1, 700), (144, 3, 400), (256, 1, 3000), (256, 2, 20011)])
def test_one_term_is_told_from_two(D, new, L):
    q, cache, batch, scale = aa.spread_inputs(D, new, L)
    want, _, most, _ = rs.attn_blocks(q, *cache, *batch, scale)
    unit = aa.noise(q, *cache, *batch, scale)
    got = {t: aa.spread(aa.emulate(q, *cache, *batch, scale, *t), want, unit)
           for t in ((2, 2), (1, 2), (2, 1))}
    assert got[2, 2] < aa.SPREAD / 2
    assert got[1, 2] > 2 * aa.SPREAD and got[2, 1] > 2 * aa.SPREAD, got


@pytest.mark.parametrize("type", TYPES)
def test_wide_rows_need_their_small_elements(type):
    w = aa.Wide(type, 40)
    large = np.where(np.abs(w.q) < 2.0 ** (w.top - 20), 0, w.q)
    flat, _, _, _ = rs.attn_blocks(large, *w.cache, *w.batch, w.scale)
    assert (np.abs(flat - w.want) > w.tolerance(type)).mean() > 0.3
