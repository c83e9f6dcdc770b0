"""Inputs of the attention over the cache with block scales whose answers are known
without a softmax, and a measure of its errors that tells one fp16 term of queries or
weights from two."""
import numpy as np

from tests import generation as gen
from tests import runtime_scales as rs

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


def noise(q, kc, ks, vc, vs, starts, lens, pages, logit_scale):
    """Of every output sqrt(sum w^2 (v - y)^2) in 64 bits: what independent relative errors
    of the weights with a standard deviation of 1 would put it off by."""
    n_pages, G, page, D = kc.shape
    block = page // ks.shape[2]
    T, H = q.shape[0], q.shape[1] // D
    out = np.zeros((T, H, D))
    for b in range(len(lens)):
        pos = np.arange(int(lens[b]))
        pg, slot = pages[b, pos // page], pos % page
        for h in range(H):
            g = h // (H // G)
            k = kc[pg, g, slot] * ks[pg, g, slot // block].astype(np.float64)[:, None]
            v = vc[pg, g, slot] * vs[pg, g, slot // block].astype(np.float64)[:, None]
            for t in range(starts[b], starts[b + 1]):
                n = int(lens[b]) - int(starts[b + 1]) + t + 1
                x = k[:n] @ q[t, h * D:(h + 1) * D].astype(np.float64) * logit_scale
                w = np.exp(x - x.max())
                w /= w.sum()
                y = w @ v[:n]
                out[t, h] = np.sqrt((w * w) @ (v[:n] - y) ** 2)
    return out.reshape(T, H * D)


# A weight's relative error in a call of fp32 has a standard deviation below 4 * 10^-6, for
# logits that stay below 20: four roundings of numbers below 32 in the exponent (half a last
# place, 2^-20, evenly spread, times ln 2: 3.8e-7 each), a sum of up to 256 products of 16
# or 32 at a time in fp32 (16 roundings of sums below 20: 2^-20 / sqrt(3) each, 2.2e-6
# together), exp2, two fp16 terms of the weight and of each query (2^-22 and less).  With
# one term of the weight alone it is that of fp16, 2^-11 / sqrt(3) times the root mean square
# of 1 / mantissa, 0.74: 2.1e-4; with one term of the queries the logit's, as much times
# its spread.
SPREAD = 2.0 ** -16


def spread(got, want, unit):
    """Root mean square of the errors in units of `noise`, of rows that see several keys."""
    there = unit > 0
    e = (got.astype(np.float64) - want)[there] / unit[there]
    return float(np.sqrt(np.mean(e * e)))


def emulate(q, kc, ks, vc, vs, starts, lens, pages, logit_scale, q_terms=2, w_terms=2):
    """Contexts [T][H * D] of fp32 queries by the steps of the call, with so many fp16 terms
    of queries and of weights."""
    def terms(x, n):
        hi = x.astype(np.float16).astype(f4)
        return hi if n == 1 else hi + (x - hi).astype(np.float16).astype(f4)
    n_pages, G, page, D = kc.shape
    block = page // ks.shape[2]
    T, H = q.shape[0], q.shape[1] // D
    out = np.zeros((T, H, D), f4)
    for b in range(len(lens)):
        pos = np.arange(int(lens[b]))
        pg, slot = pages[b, pos // page], pos % page
        for h in range(H):
            g = h // (H // G)
            sk, sv = ks[pg, g, slot // block], vs[pg, g, slot // block]
            k, v = kc[pg, g, slot].astype(f4), vc[pg, g, slot].astype(np.float64)
            lv = np.log2(sv)
            for t in range(starts[b], starts[b + 1]):
                n = int(lens[b]) - int(starts[b + 1]) + t + 1
                r = q[t, h * D:(h + 1) * D]
                e = int(np.frexp(np.abs(r).max())[1]) - 1
                c = k[:n] @ terms(r * f4(2.0 ** (14 - e)), q_terms)
                a = f4(logit_scale * np.log2(np.e)) * f4(2.0 ** (e - 14)) * sk[:n]
                x = c * a + lv[:n]
                w = np.exp2(x - x.max() + f4(8))
                y = terms(w, w_terms).astype(np.float64) @ v[:n]
                out[t, h] = y / (w / sv[:n]).astype(np.float64).sum()
    return out.reshape(T, H * D)


def spread_inputs(D, new, L, H=2, G=1, page=32, block=16):
    """fp32 queries and a cache of normal values: (q, cache, batch, logit scale)."""
    rng = np.random.default_rng(D + new + L)
    batch = gen.batch(rng, [new, new], [L, L // 2 + 7], page)
    batch, pool = batch[:3], batch[3]
    cache = []
    for _ in range(2):
        x = rng.standard_normal((pool, G, page // block, block, D)).astype(f4)
        x *= rng.uniform(0.3, 2.0, (pool, G, page // block, 1, 1)).astype(f4)
        s = rs.scale_of(np.abs(x).max((3, 4)))
        cache += [np.rint(x / s[..., None, None]).astype(np.int8).reshape(pool, G, page, D), s]
    T = int(batch[0][-1])
    q = (rng.standard_normal((T, H * D)) * rng.uniform(0.5, 1.5, (T, 1))).astype(f4)
    return q, cache, batch, float(f4(D ** -0.5))


class Wide:
    """Rows of `type` with one channel of 2^top, where every code is 0, beside elements
    around 2^(top - 30), that make logits of the size of 1."""
    D, H = 32, 2

    def __init__(self, type, new):
        import torch
        self.top = 15 if type == "float16" else 20
        q, self.cache, self.batch, self.scale = spread_inputs(self.D, new, 400, self.H)
        small = 2.0 ** (self.top - 30)
        q = (q * small).astype(f4)
        q.reshape(-1, self.H, self.D)[..., 5] = 2.0 ** self.top
        self.q = torch.from_numpy(q).to(getattr(torch, type)).float().numpy()
        self.cache[0][..., 5] = 0
        self.cache[1] *= f4(1 / small)
        self.want, self.size, self.most, self.count = rs.attn_blocks(
            self.q, *self.cache, *self.batch, self.scale)

    def tolerance(self, type):
        """The row's largest element lies in [2^14, 2^15) as fp16, where a step of the least
        ones is 2^-24: an element is off by half of it, 2^-25 * 2^(top - 14).  A logit is by as
        much times the sum of its keys' magnitudes, a weight by exp of that, in numerator and
        denominator; then runtime_scales.attn_bound.  The largest weight is 2^8 at least, so
        that those too small for fp16 are short of 2^-33 of it."""
        kc, ks, _, vs = self.cache
        key = (np.abs(kc.astype(np.float64)).sum(3) * np.repeat(ks, 16, 2)).max()
        off = 2.0 ** (self.top - 39) * key * self.scale
        rel, _ = rs.attn_bound(self.size, self.most, self.count, self.D,
                               32 if type == "float32" else 16, np.abs(np.log2(vs)).max())
        tol = self.size * np.expm1(2 * off) + rel * np.exp(2 * off)
        tol = (tol + self.count * 2.0 ** -33 * 127 * vs.max())[:, :, None]
        want = np.abs(self.want.reshape(tol.shape[:2] + (self.D,)))
        return (tol + HALF[type] * (want + tol)).reshape(self.want.shape)
