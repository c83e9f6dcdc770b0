"""What tells a right attention over the cache with block scales from a wrong one: the
known answers against plausible wrong ones."""
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
