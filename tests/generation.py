"""Plain 64-bit forms of the operators of text generation (the paged
key/value cache, attention over it, sampling), written from their
definitions with numpy, one sequence, head and row at a time."""
import numpy as np

BLOCK, ONE = 128, 32512


def f32(v):
    return np.float64(np.float32(v))


def code(v, scale, zp, bits):
    half = 1 << (bits - 1)
    return np.clip(np.rint(np.clip(v / f32(scale), -2.0 ** 40, 2.0 ** 40)) + zp, -half, half - 1)


def place(pages, n_pages, page, b, pos):
    """(page index, slot) of a position of sequence b, or None."""
    if pos < 0 or pos // page >= pages.shape[1]:
        return None
    at = int(pages[b, pos // page])
    return (at, pos % page) if 0 <= at < n_pages else None


def rotate(x, heads, scale, zp, angle):
    """One token's real values, rotated by cos/sin pairs [D/2][2] (or not)."""
    u = (f32(scale) * (x.astype(np.float64) - zp)).reshape(heads, 2, -1)
    if angle is None:
        return u.reshape(heads, -1)
    c, s = angle[:, 0], angle[:, 1]
    return np.concatenate((u[:, 0] * c - u[:, 1] * s, u[:, 1] * c + u[:, 0] * s), axis=1)


def rope_append(q, k, v, fq, fqo, fk, fko, k_cache, v_cache, starts, lens, pages, angles, out):
    """Updates k_cache, v_cache and out in place."""
    n_pages, G, page, D = k_cache.shape
    for b in range(len(lens)):
        for t in range(starts[b], starts[b + 1]):
            pos = int(lens[b]) - int(starts[b + 1]) + t
            if pos < 0 or (angles is not None and pos >= len(angles)):
                continue
            ang = None if angles is None else angles[pos]
            out[t] = code(rotate(q[t], q.shape[1] // D, *fq, ang), *fqo, 16).reshape(-1)
            at = place(pages, n_pages, page, b, pos)
            if at is not None:
                k_cache[at[0], :, at[1]] = code(rotate(k[t], G, *fk, ang), *fko, 8)
                v_cache[at[0], :, :, at[1]] = v[t].reshape(G, D)


def paged_attn(q, fq, k_cache, k_scale, v_cache, fv, starts, lens, pages, logit_scale,
               window=0, sinks=0):
    """The rows' contexts as real values [T][H * D] before their code, and the
    smallest weight sum of a block behind each (0: nothing seen)."""
    n_pages, G, page, D = k_cache.shape
    T, H = q.shape[0], q.shape[1] // D
    sigma = f32(fq[0]) * f32(k_scale) * f32(logit_scale)
    y = np.zeros((T, H, D))
    for b in range(len(lens)):
        n = min(int(lens[b]), pages.shape[1] * page)
        pos = [p for p in range(n) if place(pages, n_pages, page, b, p) is not None]
        pos = np.array(pos, dtype=np.int64)
        pg, slot = pages[b, pos // page], pos % page
        for h in range(H):
            keys = k_cache[pg, h // (H // G), slot].astype(np.float64)
            vals = v_cache[pg, h // (H // G), :, slot].astype(np.float64) - fv[1]
            for t in range(starts[b], starts[b + 1]):
                at = int(lens[b]) - int(starts[b + 1]) + t
                see = pos <= at
                if window > 0:
                    see &= (pos > at - window) | (pos < sinks)
                if not see.any():
                    continue
                c = keys[see] @ (q[t, h * D:(h + 1) * D].astype(np.float64) - fq[1])
                top, num, den = c.max(), np.zeros(D), 0.0
                blocks = pos[see] // BLOCK
                for i in np.unique(blocks):
                    m = blocks == i
                    w = np.rint(ONE * np.exp(sigma * (c[m] - c[m].max())))
                    f = np.exp(sigma * (c[m].max() - top))
                    num += f * (w @ vals[see][m])
                    den += f * w.sum()
                y[t, h] = f32(fv[0]) * num / den
    return y.reshape(T, H * D)


def assert_codes(got, real, scale, zp, bits, slack):
    """Codes of real values: equal, but for one step in at most one of a
    thousand where the value lies within ``slack`` (in steps) of a rounding tie."""
    want = code(real, scale, zp, bits)
    bad = np.nonzero(got != want)
    if len(bad[0]) == 0:
        return
    assert len(bad[0]) <= 1e-3 * want.size, (len(bad[0]), want.size)
    v = real[bad] / f32(scale)
    tie = np.abs(v - np.floor(v) - 0.5)
    assert (np.abs(got[bad].astype(np.int64) - want[bad]) <= 1).all() and (tie <= slack).all(), \
        (len(bad[0]), np.abs(got[bad].astype(np.int64) - want[bad]).max(), tie.max())


def batch(rng, new, lens, page, spare=3, first=0):
    """starts, lens and a page list over a pool of shuffled pages; returns
    also the pool's size.  Unused entries hold page ``first``."""
    need = [-(-max(n, 0) // page) for n in lens]
    pool = sum(need) + spare
    perm = rng.permutation(pool).astype(np.int32)
    pages = np.full((len(lens), max(need + [1])), first, np.int32)
    at = 0
    for b, n in enumerate(need):
        pages[b, :n] = perm[at:at + n]
        at += n
    starts = np.concatenate(([0], np.cumsum(new))).astype(np.int32)
    return starts, np.array(lens, np.int32), pages, pool


def sample_row(x, u, t=1.0, k=0, p=1.0, floor=0.0):
    """One row's token: x real logits (fp64), the settings as in mq_sample;
    Python integers for the weights and their sums."""
    idx = [i for i in range(len(x)) if x[i] > -np.inf]
    if not idx:
        return -1
    order = sorted(idx, key=lambda i: (-x[i], i))
    top = x[order[0]]
    if not t > 0:
        return order[0]
    if 0 < k < len(order):
        order = order[:k]

    def weight(i):
        if x[i] == top:
            return 1 << 40
        return 0 if np.isinf(top) else int(np.rint(np.exp((x[i] - top) / t) * 2.0 ** 40))

    w = {i: weight(i) for i in order}
    if p < 1:
        total, before, kept = float(sum(w.values())), 0, []
        for i in order:
            if kept and not float(before) < p * total:
                break
            kept.append(i)
            before += w[i]
        order = kept
    if floor > 0:
        order = [i for i in order if float(w[i]) >= min(floor, 1.0) * 2.0 ** 40]
    total = sum(w[i] for i in order)
    r = min(int(np.floor(min(max(u, 0.0), 1.0) * float(total))) if u == u else 0, total - 1)
    run = 0
    for i in sorted(order):
        run += w[i]
        if run > r:
            return i
