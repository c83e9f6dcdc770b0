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
