"""Plain forms of the operators whose scales are found at run time, written from
their definitions with numpy.  What a definition rounds to fp32 is rounded to
fp32 here, so that codes and scales are compared bit for bit."""
import numpy as np

TINY = 2.0 ** -60
f4 = np.float32


def scale_of(most):
    return f4(np.maximum(f4(most), f4(TINY))) / f4(127.0)


def quantize_tokens(x):
    """Codes, scales and row sums of fp32 rows."""
    most = np.abs(x).max(1)
    bad = ~np.isfinite(most)
    s = scale_of(np.where(bad, 0, most))
    with np.errstate(invalid="ignore", over="ignore"):
        c = np.rint(x * (f4(1.0) / s)[:, None])
    c = np.where(bad[:, None], 0, c).astype(np.int8)
    return c, np.where(bad, f4(np.nan), s), c.sum(1, dtype=np.int32)


def token_sums(codes, w, zp):
    """Exact integer sums of a product with int8 weights [N][K]."""
    w = w.astype(np.float64) - (0 if zp is None else zp.astype(np.float64)[:, None])
    return np.rint(codes.astype(np.float64) @ w.T).astype(np.int64)


def linear(codes, a_scale, w, w_scale, zp, bias):
    """fp32 outputs, each step rounded once."""
    y = token_sums(codes, w, zp).astype(f4) * w_scale[None, :] * a_scale[:, None]
    return y if bias is None else y + bias[None, :]


def unpack4(w):
    """int8 weights [N][K] of packed ones [N][K/2]."""
    out = np.empty((w.shape[0], 2 * w.shape[1]), np.int8)
    out[:, 0::2] = (w << 4).astype(np.uint8).view(np.int8) >> 4
    out[:, 1::2] = w.view(np.int8) >> 4
    return out


def pack4(w):
    u = w.view(np.uint8) & 15
    return np.ascontiguousarray(u[:, 0::2] | (u[:, 1::2] << 4))


# ---------------------------------------------------------------------------
# The cache with block scales.  Token-major arrays: keys and values as
# [pages][G][page][D] codes; the values' own layout by v_layout/v_rows.

def v_layout(v):
    """[pages][G][page][D] to the cache's [pages][G][page / 16][D][16]."""
    n, G, page, D = v.shape
    return np.ascontiguousarray(v.reshape(n, G, page // 16, 16, D).swapaxes(3, 4))


def v_rows(v):
    n, G, g, D, _ = v.shape
    return np.ascontiguousarray(v.swapaxes(3, 4).reshape(n, G, g * 16, D))


def place(pages, n_pages, page, b, pos):
    if pos < 0 or pos // page >= pages.shape[1]:
        return None
    at = int(pages[b, pos // page])
    return (at, pos % page) if 0 <= at < n_pages else None


def rotate(x, heads, angle):
    """One token's fp32 values by cos/sin pairs [D/2][2] (None: not) in fp64,
    rounded to fp32."""
    u = x.astype(np.float64).reshape(heads, 2, -1)
    if angle is None:
        return x.reshape(heads, -1)
    c, s = angle[:, 0], angle[:, 1]
    with np.errstate(invalid="ignore", over="ignore"):
        return np.concatenate((u[:, 0] * c - u[:, 1] * s, u[:, 1] * c + u[:, 0] * s),
                              axis=1).astype(f4)


def _finite_max(x):
    a = np.abs(x[np.isfinite(x)])
    return a.max() if a.size else f4(0)


def _block_codes(x, s):
    with np.errstate(invalid="ignore", over="ignore"):
        c = np.rint(np.clip(x * (f4(1.0) / s), f4(-127), f4(127)))
    return np.where(np.isnan(x), 0, c).astype(np.int8)


def append_blocks(q, k, v, kc, ks, vc, vs, starts, lens, pages, angles, out):
    """fp32 rows q, k, v; updates the codes [pages][G][page][D], the scales
    [pages][G][page / block] and the queries' rows of out in place."""
    n_pages, G, page, D = kc.shape
    block = page // ks.shape[2]
    for b in range(len(lens)):
        s0, s1, n = int(starts[b]), int(starts[b + 1]), int(lens[b])
        toks = [(t, n - s1 + t) for t in range(s0, s1)]
        toks = [(t, p) for t, p in toks if p >= 0 and (angles is None or p < len(angles))]
        new = {}
        for t, p in toks:
            ang = None if angles is None else angles[p]
            out[t] = rotate(q[t], q.shape[1] // D, ang).reshape(-1)
            new[p] = rotate(k[t], G, ang), v[t].reshape(G, D)
        for i in sorted({p // block for p in new}):
            at = place(pages, n_pages, page, b, i * block)
            if at is None:
                continue
            pg, slot = at
            ps = [p for p in new if p // block == i]
            lo = min(ps) - i * block
            for which, codes, scales in ((0, kc, ks), (1, vc, vs)):
                x = np.stack([new[p][which] for p in ps])  # [tokens][G][D]
                for g in range(G):
                    old = scales[pg, g, slot // block] if lo else f4(0)
                    if not (old > 0 and np.isfinite(old)):
                        old = f4(0)
                    s = np.maximum(old, scale_of(_finite_max(x[:, g])))
                    before = scales[pg, g, slot // block]
                    if lo and not before == s:
                        c = codes[pg, g, slot:slot + lo]
                        c[...] = np.rint(c.astype(f4) * (old / s)).astype(np.int8)
                    scales[pg, g, slot // block] = s
                    codes[pg, g, slot + lo:slot + lo + len(ps)] = _block_codes(x[:, g], s)


def attn_blocks(q, kc, ks, vc, vs, starts, lens, pages, logit_scale, window=0, sinks=0):
    """The rows' contexts [T][H * D] in fp64 and what bounds their rounding
    errors, per row and head: the largest over channels of sum w |v|, over keys of
    sum |q k| logit_scale, the keys seen (0: none)."""
    n_pages, G, page, D = kc.shape
    block = page // ks.shape[2]
    T, H = q.shape[0], q.shape[1] // D
    y, size, most, count = np.zeros((T, H, D)), np.zeros((T, H)), np.zeros((T, H)), np.zeros((T, H))
    for b in range(len(lens)):
        n = min(int(lens[b]), pages.shape[1] * page)
        pos = [p for p in range(n) if place(pages, n_pages, page, b, p) is not None]
        pos = np.array(pos, dtype=np.int64)
        pg, slot = pages[b, pos // page], pos % page
        at = np.arange(starts[b], starts[b + 1]) + int(lens[b]) - int(starts[b + 1])
        for h in range(H):
            g = h // (H // G)
            # (scales of what no row sees may be anything)
            with np.errstate(invalid="ignore", over="ignore"):
                k = kc[pg, g, slot] * ks[pg, g, slot // block].astype(np.float64)[:, None]
                v = vc[pg, g, slot] * vs[pg, g, slot // block].astype(np.float64)[:, None]
            for t in range(starts[b], starts[b + 1]):
                p = at[t - starts[b]]
                see = pos <= p
                if window > 0:
                    see &= (pos > p - window) | (pos < sinks)
                if not see.any():
                    continue
                r = q[t, h * D:(h + 1) * D].astype(np.float64)
                x = k[see] @ r * logit_scale
                w = np.exp(x - x.max())
                w /= w.sum()
                y[t, h] = w @ v[see]
                size[t, h] = (w @ np.abs(v[see])).max()
                most[t, h] = (np.abs(k[see]) @ np.abs(r)).max() * logit_scale
                count[t, h] = see.sum()
    return y.reshape(T, H * D), size, most, count


def attn_bound(size, most, count, D, bits, vs_log2):
    """How far a context of attn_blocks may be off before its last rounding, per
    row and head.  With u = 2^-24 and logits in log2 units, X = most * log2(e):
    a logit is the sum of at most D products in fp32 (D u X, as much again for
    the order inside an instruction's sums; fp32 queries are short of 2^-22 X), its
    factor has three roundings (4 u X), the exponent adds log2 of the value scale
    and the maximum (numbers up to X + |log2 vs| + 8: four roundings); a weight
    takes its exp2 (2^-22) and its rounding (2^-11 for 16-bit types, else 2^-22);
    numerator and denominator each sum `count` terms over steps of 64 ((count /
    16 + 64) u); every relative error of a weight counts in both: weights w r with r
    from 2^-e to 2^e have a mean R of that range, and sum w (r / R - 1) v is at most
    2^(2 e) - 1 of sum w |v| (from e = 400 on, where 64 bits may not hold the other
    weights, nothing is said).  Weights too
    small for fp16 are short of 2^-25 of 2^1 at least (the largest is >= 2): count
    * 2^-26 of the values."""
    u, X = 2.0 ** -24, most * 1.4426950408889634
    logit = (2 * D * u + 2.0 ** -22 + 4 * u) * X + 4 * u * (X + vs_log2 + 8)
    weight = 2.0 ** -22 + (2.0 ** -11 if bits == 16 else 2.0 ** -22)
    rel = np.exp2(np.minimum(2 * logit, 999)) - 1 + 2 * (weight + (count / 16 + 64) * u)
    return np.where(logit < 400, size * rel * 1.01, np.inf), count * 2.0 ** -26


def adjust_logits(x, history=None, lens=None, prompts=None, repetition=None, presence=None,
                  frequency=None, bias=None, mask=None):
    """fp32 logits [M][V] changed step by step, each rounded to fp32."""
    x = x.astype(f4).copy()
    M, V = x.shape
    for m in range(M):
        if history is not None:
            words = history[m, :max(0, min(int(lens[m]), history.shape[1]))]
            p = max(0, int(prompts[m])) if prompts is not None else 0
            drawn = words[p:]
            r = f4(1) if repetition is None else repetition[m]
            for w in np.unique(words[(words >= 0) & (words < V)]):
                x[m, w] = x[m, w] / r if x[m, w] > 0 else x[m, w] * r
                n = int((drawn == w).sum())
                if n:
                    f = f4(0) if frequency is None else frequency[m]
                    x[m, w] = x[m, w] - f * f4(n)
                    x[m, w] = x[m, w] - (f4(0) if presence is None else presence[m])
        if bias is not None:
            starts, words, values = bias
            last = {}
            for i in range(max(0, starts[m]), min(starts[m + 1], len(words))):
                if 0 <= words[i] < V:
                    last[words[i]] = values[i]
            for w, v in last.items():
                x[m, w] = x[m, w] + v
        if mask is not None:
            bits = np.unpackbits(np.ascontiguousarray(mask[m]).view(np.uint8), bitorder="little")
            x[m, bits[:V] == 0] = -np.inf
    return x
