"""Attention over the cache with block scales for batches of sequences with one new token
and others with many: the kernel of few rows with several tiles of a sequence, whole and
in parts, and the tiles' kernel with sequences of a row."""
import numpy as np
import pytest

from tests.test_gpu_attn_blocks import TYPES, _check

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("B,chunk", [(64, 200), (256, 333), (300, 200)])
@pytest.mark.parametrize("H,G,D", [(8, 2, 64), (4, 1, 144)])
@pytest.mark.parametrize("type", ["float32", "bfloat16"])
def test_chunks_among_single_tokens(B, chunk, H, G, D, type):
    rng = np.random.default_rng(B + chunk + D)
    new, lens = np.ones(B, np.int64), rng.integers(1, 150, B)
    for b, n in ((B // 3, chunk), (B - 1, 17), (0, 0)):
        new[b] = n
        lens[b] = n + 900
    args = (H, G, D, 32, 16, list(new), list(lens), type)
    _check(rng, *args)
    _check(rng, *args, window=60, sinks=5)
    _check(rng, *args, splits=False)


@pytest.mark.parametrize("type", TYPES)
def test_one_chunk_and_a_long_sequence_in_parts(type):
    rng = np.random.default_rng(3)
    for new, lens in (([1, 20, 1, 1, 1], [9000, 3000, 5, 700, 1]),
                      ([40, 1, 1, 1, 1, 1, 1, 1], [2000, 64, 65, 9000, 1, 16, 17, 300])):
        _check(rng, 2, 1, 64, 64, 32, new, lens, type)
        _check(rng, 2, 1, 256, 64, 32, new, lens, type, window=2500)
