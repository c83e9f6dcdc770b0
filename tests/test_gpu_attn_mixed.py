"""Attention over the cache with block scales for batches of sequences with one new token
and others with many: the kernel of few rows with several tiles of a sequence, whole and
in parts, and the tiles' kernel with sequences of a row."""
import numpy as np
import pytest

from tests.test_gpu_attn_blocks import TYPES, _check, _compare, _pool, _put, _queries

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


def test_millions_of_sequences():
    """2^22 sequences, five of them with a token each: 2^23 work-groups, below the 2^24 that
    are refused."""
    import torch

    import paper_2408_13933_amd as mq
    B, H, G, D, page, at = 1 << 22, 4, 2, 16, 16, [0, 7, 1 << 20, (1 << 22) - 2, (1 << 22) - 1]
    rng = np.random.default_rng(1)
    cache = _pool(rng, 5, G, page, D, 16)
    new = np.zeros(B, np.int32)
    new[at] = 1
    batch = [np.concatenate(([0], np.cumsum(new))).astype(np.int32), new * 11,
             np.zeros((B, 1), np.int32)]
    batch[2][at, 0] = [4, 0, 3, 1, 2]
    q, qf = _queries(rng, 5, H * D, "float32", 0)
    g, i = _put(cache, batch)
    y = mq.mq_paged_attn_blocks(q, *g, *i, 0.25)
    few = [np.arange(6, dtype=np.int32), batch[1][at], batch[2][at]]
    _compare(y.cpu().numpy(), qf, cache, few, 0.25, "float32", D, 0, 0)
    big = [torch.zeros(2 * B + 1, dtype=torch.int32, device="cuda"),
           torch.zeros(2 * B, dtype=torch.int32, device="cuda"),
           torch.zeros((2 * B, 1), dtype=torch.int32, device="cuda")]
    with pytest.raises(mq.MQError):
        mq.mq_paged_attn_blocks(q, *g, *big, 0.25)
