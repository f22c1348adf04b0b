"""Float64 numpy restatement of the rollout-side operators: drawing a token from a row of logits, rounding to 8-bit floating
point with a scale per block of 128, and the matrix product of such matrices.  Test infrastructure: plain and slow."""
import numpy as np

MAX8 = {"e4m3": 448.0, "e5m2": 57344.0}


def sample_row(z, u, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0, K=0):
    """One row.  Returns dict(id, logp, top_ids[K], top_p[K], kept (number of tokens), margin): ``margin`` is the smallest distance,
    relative to the whole mass, of a decision (the draw, the top_p cut) from flipping; None for a row without a distribution."""
    z = np.asarray(z, np.float64)
    V = z.size
    if np.isnan(z).any() or z.max() == np.inf or z.max() == -np.inf:
        return None
    tau, k = float(temperature), int(top_k)
    if tau == 0.0:
        tau, k = 1.0, 1
    order = np.argsort(-z, kind="stable")
    with np.errstate(over="ignore"):
        w = np.exp((z[order] - z[order[0]]) / tau)
    w[w < 2.0 ** -1000] = 0.0
    n = int(np.isfinite(z).sum())
    if 0 < k < V:
        n = min(n, k)
    margin = np.inf
    cs = np.cumsum(w[:n])
    m = n
    if top_p < 1.0:
        reach = cs >= top_p * cs[-1]
        m = max(1, int(np.argmax(reach)) + 1) if reach.any() else n
        margin = np.abs(cs - top_p * cs[-1]).min() / cs[-1]
    if min_p > 0.0:
        m = min(m, int((w[:n] >= min_p).sum()))
    by_id = np.zeros(V)
    by_id[order[:m]] = w[:m]
    c = np.cumsum(by_id)
    a = int(np.argmax(c > u * c[-1]))
    margin = min(margin, np.abs(c[by_id > 0] / c[-1] - u).min())
    with np.errstate(divide="ignore"):
        logp = (z[a] - z[order[0]]) / tau - np.log(c[-1])
    return dict(id=a, logp=logp, top_ids=order[:K], top_p=by_id[order[:K]] / c[-1], kept=m, margin=margin)


def round8(y, fmt):
    """float64 -> the nearest value of the 8-bit type, ties to even, beyond the largest: the largest."""
    bits, low = (3, -6) if fmt == "e4m3" else (2, -14)
    with np.errstate(divide="ignore"):
        e = np.floor(np.log2(np.abs(y), where=y != 0, out=np.full(y.shape, -1000.0)))
    e = np.where(np.abs(y) >= np.exp2(e + 1), e + 1, np.where(np.abs(y) < np.exp2(e), e - 1, e))      # log2 next to a power of two
    step = np.exp2(np.maximum(e, low) - bits)
    return np.clip(np.rint(y / step) * step, -MAX8[fmt], MAX8[fmt])


def quantize(x, fmt, block_rows):
    """(values, scales, quotients) of x [rows, cols] float64: blocks of block_rows x 128, scale = max(amax, 2^-100) / largest value."""
    rows, cols = x.shape
    nr, nk = -(-rows // block_rows), -(-cols // 128)
    pad = np.zeros((nr * block_rows, nk * 128))
    pad[:rows, :cols] = np.abs(x)
    amax = np.maximum(pad.reshape(nr, block_rows, nk, 128).max(axis=(1, 3)), 2.0 ** -100)
    wide = spread(amax, rows, cols, block_rows)
    y = x * MAX8[fmt] / wide
    return round8(y, fmt), amax / MAX8[fmt], y


def spread(scale, rows, cols, block_rows):
    return np.repeat(np.repeat(scale, block_rows, 0)[:rows], 128, 1)[:, :cols]


def product(a, sa, a_block_rows, b, sb, b_block_rows):
    """(C, S): the product of the scaled matrices and the sum of the magnitudes of its terms (for error bounds)."""
    A, B = a * spread(sa, *a.shape, a_block_rows), b * spread(sb, *b.shape, b_block_rows)
    return A @ B.T, np.abs(A) @ np.abs(B).T
