"""Plain statements of the operators around the products, in 64 bits, and the bounds that binary32 arithmetic keeps to.

u = 2^-24 is half a step of binary32.  A sum of n terms formed in any order is off by at most (n - 1) u times the sum of the
terms' sizes, each further operation by u; the store in half adds 2^-11 of the value, or 2^-25 where it is subnormal.
"""
import numpy as np

U = 2.0 ** -24
HALF = 2.0 ** -11
TINY = 2.0 ** -25


def store_bound(value, dtype):
    return np.abs(value) * HALF + TINY if np.dtype(dtype) == np.float16 else np.zeros_like(value)


def norm(x, r, gamma, eps):
    """(h, v, s): the sum, the weighted sum and the tokens' factors for x, r [.., K, N]."""
    h = x.astype(np.float64) + (0 if r is None else r.astype(np.float64))
    v = h * (1.0 if gamma is None else gamma.astype(np.float64)[:, None])
    return h, v, 1.0 / np.sqrt((h * h).mean(axis=-2) + eps)


def check_norm(y, scale, h_out, x, r, gamma, eps):
    """Results of a call against the formulas; y int8 with scale, or floating."""
    K = x.shape[-2]
    h, v, s = norm(x, r, gamma, eps)
    if h_out is not None:   # one rounding of the binary32 sum
        assert np.array_equal(h_out, (x.astype(np.float32) + (0 if r is None else r.astype(np.float32))).astype(x.dtype))
    # s: the sum of K squares of rounded sums, the mean and the addition of eps are under a square root, which halves their error
    s_bound = (K / 2 + 6) * U
    if y.dtype != np.int8:
        want = v * s[..., None, :]
        # below 2^-126 binary32 is spaced 2^-149: the product v is then off by up to 2^-150 whatever its size, which s multiplies, and
        # so is the result, which is v times s
        bound = np.abs(want) * (s_bound + 4 * U) + store_bound(want, y.dtype) + 2.0 ** -150 * (1 + s[..., None, :])
        assert (np.abs(y.astype(np.float64) - want) <= bound * 1.001).all(), np.max(np.abs(y - want) / np.maximum(bound, 1e-300))
        return
    top = np.abs(v).max(axis=-2)
    zero = top < 2.0 ** -100
    steps = v * np.where(zero, 0.0, 127.0 / np.where(zero, 1.0, top))[..., None, :]
    # six roundings (sum and product of v and of the largest one, the quotient, the last product) move a value of at most 127 steps
    assert (np.abs(y.astype(np.float64) - steps) <= 0.5 + 127 * 6 * U * 1.001).all(), np.max(np.abs(y - steps))
    want = np.where(zero, 0.0, top * s / 127.0)
    assert (np.abs(scale.astype(np.float64) - want) <= want * (s_bound + 8 * U) * 1.001).all()


def dequantize(c, row, col):
    return c.astype(np.float64) * (1.0 if col is None else col.astype(np.float64)[..., None, :]) * (1.0 if row is None else row.astype(np.float64)[:, None])


def check_dequantize(y, c, row, col):
    want = dequantize(c, row, col)
    assert (np.abs(y.astype(np.float64) - want) <= np.abs(want) * 3 * U * 1.001 + store_bound(want, y.dtype)).all()


def adapters(x, down, up, index, alpha, c, row, col):
    """(y, size): the result and the sum of the sizes of the terms it is made of.  x [b, K, N], index [b, N]."""
    x64, c64 = x.astype(np.float64), c.astype(np.float64)
    if x.dtype == np.int8:
        c64 = dequantize(c, row, col)
        x64 = dequantize(x, None, col)
    y, size = c64.copy(), np.abs(c64)
    for b in range(x.shape[0]):
        for a in range(down.shape[0]):
            at = np.nonzero(index[b] == a)[0]
            if len(at):
                f = 1.0 if alpha is None else float(alpha[a])
                d, p = down[a].astype(np.float64), up[a].astype(np.float64)
                y[b][:, at] += f * (p @ (d @ x64[b][:, at]))
                size[b][:, at] += abs(f) * (np.abs(p) @ (np.abs(d) @ np.abs(x64[b][:, at])))
    return y, size


def check_adapters(y, x, down, up, index, alpha, c, row, col):
    want, size = adapters(x, down, up, index, alpha, c, row, col)
    # K and rank terms to a sum, factors and additions; t may be held to 22 bits (4 u), which the 16 cover
    bound = size * (x.shape[-2] + down.shape[1] + 16) * U + store_bound(want, y.dtype)
    off = np.abs(y.astype(np.float64) - want)
    assert (off <= bound * 1.001).all(), (np.max(off / np.maximum(bound, 1e-300)), np.argwhere(off > bound)[:4])
