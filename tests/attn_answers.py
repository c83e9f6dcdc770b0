"""Inputs of the attention over the cache with block scales whose answers are known
without a softmax."""
import numpy as np

from tests import generation as gen

HALF = {"float32": 2.0 ** -24, "bfloat16": 2.0 ** -8, "float16": 2.0 ** -11}
f4 = np.float32


class Known:
    """Rows of queries with one channel that is not 0, a power of two, over keys of one
    scale, a power of two: every logit but for its last factor is exact, and in this
    channel `keys` keys hold the code that wins by far (for rows of a negative query
    others do).  low: every key's code is negative in every channel, so that the
    winner's logit is too.  Value scales are powers of two, of one size where several keys
    win.  want: the mean of the winners' values, [T][H][D]; size: of their magnitudes."""
    H, G, page, block, scale = 4, 2, 32, 16, 0.125

    def __init__(self, seed, D, new, exponent, keys=1, low=False):
        rng = np.random.default_rng(seed)
        H, G, page, block = self.H, self.G, self.page, self.block
        starts, lens, pages, pool = gen.batch(rng, [new, new], [4000, 70], page)
        lo, hi = (-120, -20) if low else (-100, 100)
        kc = rng.integers(lo, hi, (pool, G, page, D), endpoint=True).astype(np.int8)
        vc = rng.integers(-127, 127, (pool, G, page, D), endpoint=True).astype(np.int8)
        shape = (pool, G, page // block)
        ks = np.full(shape, 2.0 ** exponent, f4)
        vs = (2.0 ** rng.integers(-3, 4, shape)).astype(f4) if keys == 1 else np.full(shape, 0.25, f4)
        T = int(starts[-1])
        self.q = np.zeros((T, H, D), f4)
        self.want, self.size = np.zeros((T, H, D)), np.zeros((T, H, D))
        for b in range(2):
            first = int(lens[b]) - new  # (every row of the sequence sees it and those before)
            for g in range(G):
                win = {}
                for d in range(D):
                    at = rng.choice(first + 1, 2 * keys, replace=False)
                    for i, p in enumerate(at):
                        code = -4 if low else 127 if i < keys else -127
                        if not low or i < keys:
                            kc[pages[b, p // page], g, p % page, d] = code
                    win[d] = at[:keys], at[keys:]
                for t in range(starts[b], starts[b + 1]):
                    for h in range(g * (H // G), (g + 1) * (H // G)):
                        d, minus = int(rng.integers(D)), not low and rng.random() < 0.5
                        self.q[t, h, d] = -8.0 if minus else 8.0
                        at = win[d][1 if minus else 0]
                        pg, slot = pages[b, at // page], at % page
                        v = vc[pg, g, slot] * vs[pg, g, slot // block].astype(np.float64)[:, None]
                        self.want[t, h], self.size[t, h] = v.mean(0), np.abs(v).mean(0)
        self.q = self.q.reshape(T, H * D)
        self.cache, self.batch = (kc, ks, vc, vs), (starts, lens, pages)

    def tolerance(self, type):
        """The winners' weights are equal and all others below 2^-60 of them.  The weight takes
        its exp2 (2^-22) and its rounding (half a step of fp16, 2^-11, of two fp16 numbers
        2^-22), the value scale its logarithm of at most 3, where the last place is 2^-22,
        and that one's exp2 (2^-22 in all: 2^-21), sum, quotient and product 2^-24 each:
        below 2^-20, and 2^-11 for 16 bits.  Then the result's own rounding."""
        rel = 2.0 ** -20 + (0.0 if type == "float32" else 2.0 ** -11)
        return rel * self.size + HALF[type] * (np.abs(self.want) + rel * self.size)

    def off(self, got, type):
        """Outputs that are further from the answer than the tolerance."""
        err = np.abs(got.astype(np.float64).reshape(self.want.shape) - self.want)
        return ~(err <= self.tolerance(type))
