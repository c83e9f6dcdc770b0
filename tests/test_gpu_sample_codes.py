"""mq_sample on rows of 16-bit codes whose cut lies among the lowest codes:
masked words (codes have no -infinity, so a mask writes -32768) and flat rows
at the bottom of the range, found over the whole row; flat rows of either type
whose cut is among the listed words.  Tokens equal the plain form's
(tests/generation.py, Python integers)."""
import numpy as np
import pytest

from tests.test_gpu_sample import _run

pytestmark = pytest.mark.gpu

LOW = -32768
U = [0.0, 0.11, 0.37, 0.5, 0.83, 0.999]


def _rows(M, V, words):
    """M rows of -32768 but for `words`, {index: code}."""
    x = np.full((M, V), LOW, np.int16)
    for i, c in words.items():
        x[:, i] = c
    return x


@pytest.mark.parametrize("V", [65, 1500, 5000, 32000])
@pytest.mark.parametrize("top", [500, -3, -32000, 32767])
def test_more_wanted_than_allowed(V, top):
    """Three allowed words, the rest masked, top_k above three: the masked
    words of the lowest index fill it up."""
    x = _rows(len(U), V, {5: top, V // 2: top - 100, V - 1: top - 400})
    M = len(U)
    for alpha, t in ((6e-4, 1.0), (1e-5, 1.0), (6e-4, 1e3)):
        for kw in (dict(k=[50] * M), dict(k=[50] * M, p=[0.9] * M),
                   dict(k=[50] * M, p=[0.99] * M, floor=[1e-9] * M), dict(k=[3] * M),
                   dict(k=[4] * M), dict(k=[V - 1] * M), dict(p=[0.97] * M)):
            _run(x, U, t=[t] * M, alpha=alpha, zp=11, **kw)


def test_mass_among_masked_words():
    """31000 masked words with a good half of the mass, top_p's cut in them."""
    rng = np.random.default_rng(1)
    M, V = len(U), 32000
    x = np.full((M, V), LOW, np.int16)
    for m in range(M):
        at = rng.permutation(V)[:1000]
        x[m, at] = np.rint(-15000 + 300 * rng.standard_normal(1000))
    for t in (2.0, 3.0, 50.0):
        for p in (0.95, 0.6):
            _run(x, U, t=[t] * M, p=[p] * M, alpha=6e-4)
        _run(x, U, t=[t] * M, k=[15000] * M, alpha=6e-4)
        _run(x, U, t=[t] * M, k=[25000] * M, p=[0.9] * M, floor=[1e-12] * M, alpha=6e-4)


@pytest.mark.parametrize("bits", [10, 11, 12, 13, 14, 15])
def test_widths_of_the_range(bits):
    """The row's largest code 2^bits and some above the lowest, so that the
    last bin of the search is of every width and cut at every place."""
    rng = np.random.default_rng(bits)
    over = [0, 1, 2, 3, 5, 31, 32, 33, 63, 64, 500, 1000, 1023]
    V, M = 9000, len(over)
    x = np.full((M, V), LOW, np.int32)
    for m, o in enumerate(over):
        x[m, rng.permutation(V)[:40]] += rng.integers(0, 1 << bits, 40)
        x[m, rng.permutation(V)[:3000]] += rng.integers(0, 70, 3000)
        x[m, 1234] = LOW + (1 << bits) + o
    x = x.astype(np.int16)
    u = rng.random(M)
    # the lowest words weigh about e^-3 of the first
    alpha = 3.0 / (1 << bits)
    for kw in (dict(p=[0.97] * M), dict(p=[0.9] * M), dict(k=[7000] * M),
               dict(k=[8999] * M, p=[0.99] * M), dict(k=[200] * M)):
        _run(x, u, alpha=alpha, **kw)


@pytest.mark.parametrize("dtype", [np.float32, np.int16])
def test_flat_rows_whose_lists_hold_the_cut(dtype):
    """top_k within the listed words of a row so flat that more of them share
    one distance bin than there is room for."""
    rng = np.random.default_rng(2)
    M, V = len(U), 100000
    x = rng.standard_normal((M, V)) * (2 if dtype == np.float32 else 4000)
    x = x.astype(dtype)
    x[1, rng.permutation(V)[:900]] = x[1].max()  # more equal words than there is room for
    for kw in (dict(k=[300] * M), dict(k=[500] * M, p=[0.4] * M),
               dict(k=[550] * M, p=[0.9] * M, floor=[0.5] * M), dict(p=[0.002] * M)):
        _run(x, U, t=[3e4] * M, alpha=1e-3, **kw)
