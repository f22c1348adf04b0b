"""Float64 numpy restatement of the losses against a reference policy (log-probabilities of tokens, the clipped policy loss with a KL
term, the loss over pairs of sequences) and of the 4-bit weights and their product.  Test infrastructure: plain and slow."""
import numpy as np


def log_softmax(z):
    m = z.max(axis=1, keepdims=True)
    return z - m - np.log(np.exp(z - m).sum(axis=1, keepdims=True))


def token_logp(z, ids):
    with np.errstate(divide="ignore"):
        return log_softmax(z)[np.arange(len(ids)), ids]


def logp_gradient(z, ids, c):
    """sum_t c_t logp_t differentiated by z."""
    d = -np.exp(log_softmax(z)) * c[:, None]
    d[np.arange(len(ids)), ids] += c
    return d


def _xlog(p, l):
    """p * l where p > 0, else 0."""
    out = np.zeros(np.broadcast(p, l).shape)
    np.multiply(p, l, out=out, where=p > 0)
    return out


def policy_kl(z, ids, mu_logp, adv, valid, form, beta, eps_low, eps_high, y=None, ref_logp=None, scale=None):
    """dict(loss, kl, mask, dlogits, r, spread); form "pi_ref", "ref_pi" or "k3".  ``spread``: largest |log pi_j - log rho_j| of the row over
    entries with probability (the size of the terms of its KL)."""
    T, V = z.shape
    n = int(valid.sum())
    s = scale if scale else (1.0 / n if n else 0.0)
    out = dict(kl=np.zeros(T), mask=np.zeros(T, np.uint8), dlogits=np.zeros((T, V)), r=np.zeros(T), spread=np.zeros(T), terms=np.zeros(T))
    loss = 0.0
    for t in np.flatnonzero(valid):
        l = log_softmax(z[t:t + 1])[0]
        p, a, A = np.exp(l), ids[t], adv[t]
        r = np.exp(l[a] - mu_logp[t])
        M = 0 if (A > 0 and r > 1 + eps_high) or (A < 0 and r < 1 - eps_low) else 1
        hot = np.zeros(V)
        hot[a] = 1.0
        g = s * M * r * A
        d = g * (p - hot)
        if form == "k3":
            x = ref_logp[t] - l[a]
            kl = np.expm1(x) - x
            d += s * beta * (1 - np.exp(x)) * (hot - p)
        else:
            q = log_softmax(y[t:t + 1])[0]
            with np.errstate(invalid="ignore"):
                dl = l - q
            if form == "pi_ref":
                kl = _xlog(p, dl).sum()
                d += s * beta * (_xlog(p, dl) - p * kl)
                out["spread"][t] = np.abs(dl[p > 0]).max()
            else:
                kl = _xlog(np.exp(q), -dl).sum()
                d += s * beta * (p - np.exp(q))
                out["spread"][t] = np.abs(dl[np.exp(q) > 0]).max()
        sur = min(r * A, np.clip(r, 1 - eps_low, 1 + eps_high) * A)
        out["terms"][t] = s * (beta * kl - sur)
        loss += out["terms"][t]
        out["kl"][t], out["mask"][t], out["dlogits"][t], out["r"][t] = kl, M, d, r
    out["loss"] = loss
    return out


def preference(z, ids, cu, valid, kind, beta, smoothing=0.0, margin=0.0, average=False, ref_logp=None, scale=None):
    """dict(loss, reward, logp, dlogits, coef)."""
    T, V = z.shape
    P = (len(cu) - 1) // 2
    inside = np.zeros(T, bool)
    inside[cu[0]:cu[-1]] = True
    use = inside & valid
    logp = np.zeros(T)
    logp[use] = token_logp(z[use], ids[use])
    ratio = logp - (0 if ref_logp is None else ref_logp)
    loss, n, reward, coef = 0.0, 0, np.zeros(2 * P), np.zeros(T)
    for p in range(P):
        rows = [[t for t in range(cu[2 * p + k], cu[2 * p + k + 1]) if use[t]] for k in (0, 1)]
        if not rows[0] or not rows[1]:
            continue
        w = [beta / (len(rs) if average else 1.0) for rs in rows]
        R = [w[k] * sum(ratio[t] for t in rows[k]) for k in (0, 1)]
        h = R[0] - R[1] - margin
        if kind == "sigmoid":
            L = (1 - smoothing) * np.logaddexp(0, -h) + smoothing * np.logaddexp(0, h)
            dh = 1 / (1 + np.exp(-h)) - (1 - smoothing)
        elif kind == "ipo":
            L = (h / beta - 1 / (2 * beta)) ** 2
            dh = 2 * (h / beta - 1 / (2 * beta)) / beta
        else:
            L = max(0.0, 1 - h)
            dh = -1.0 if h < 1 else 0.0
        loss, n = loss + L, n + 1
        reward[2 * p:2 * p + 2] = R
        coef[rows[0]], coef[rows[1]] = dh * w[0], -dh * w[1]
    s = scale if scale else (1.0 / n if n else 0.0)
    d = np.zeros((T, V))
    d[use] = logp_gradient(z[use], ids[use], s * coef[use])
    return dict(loss=s * loss, reward=reward, logp=logp, dlogits=d, coef=s * coef)


def round_bits(x, bits):
    """float64 -> so many significant bits, ties to even."""
    m, e = np.frexp(x)
    return np.ldexp(np.rint(m * 2.0 ** bits), e - bits)


def int4_quantize(x, group):
    """(codes 0 .. 15 [rows, cols], scales, values in 64 bits) of x [rows, cols] float64."""
    rows, cols = x.shape
    n = -(-cols // group)
    pad = np.zeros((rows, n * group))
    pad[:, :cols] = x
    scale = round_bits(np.maximum(np.abs(pad).reshape(rows, n, group).max(axis=2), 2.0 ** -100) / 7, 8)
    wide = np.repeat(scale, group, 1)[:, :cols]
    code = np.clip(np.rint(x / wide), -7, 7)
    return (code + 8).astype(np.uint8), scale, code * wide


def unpack(q, cols):
    out = np.empty((q.shape[0], 2 * q.shape[1]), np.uint8)
    out[:, 0::2], out[:, 1::2] = q & 15, q >> 4
    return out[:, :cols]


def pack(codes):
    rows, cols = codes.shape
    wide = np.zeros((rows, cols + cols % 2), np.uint8)
    wide[:, :cols] = codes
    return wide[:, 0::2] | (wide[:, 1::2] << 4)


def int4_product(x, codes, scale, group):
    """(y, sum of the magnitudes of its terms)."""
    w = (codes.astype(np.float64) - 8) * np.repeat(scale, group, 1)[:, :codes.shape[1]]
    return x @ w.T, np.abs(x) @ np.abs(w).T
