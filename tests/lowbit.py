"""Operators on eight-bit operands and draws, written out in 64 bits from their definitions (numpy only)."""
import numpy as np
import torch

BLOCK = 128


def as_float64(t):
    """Values of a torch tensor of any of the operators' types."""
    if t.dtype in (torch.float8_e4m3fn, torch.float8_e8m0fnu):
        t = t.cpu().float()
    return t.cpu().double().numpy()


def round_e4m3(v):
    """Nearest value with three mantissa bits, ties to even; below 2^-6 steps of 2^-9; nan stays."""
    v = np.asarray(v, np.float64)
    a = np.abs(v)
    with np.errstate(all="ignore"):
        _, e = np.frexp(np.where(np.isfinite(a), a, 0.0))
        step = np.ldexp(1.0, np.maximum(e - 1, -6) - 3)
        return np.where(np.isfinite(v), np.rint(v / step) * step, np.nan)


def blocks_of(n):
    return -(-n // BLOCK)


def block_amax(x, block_rows):
    rows, cols = x.shape
    a = np.where(np.isfinite(x), np.abs(x), 0.0)
    out = np.zeros((-(-rows // block_rows), blocks_of(cols)))
    for i in range(out.shape[0]):
        for j in range(out.shape[1]):
            part = a[i * block_rows:(i + 1) * block_rows, j * BLOCK:(j + 1) * BLOCK]
            out[i, j] = part.max() if part.size else 0.0
    return out


def scale_e8m0(amax):
    """Smallest 2^e, e >= -127, with amax / 2^e <= 448, found by trying."""
    s = np.full(amax.shape, 2.0 ** -127)
    while True:
        low = amax > 448.0 * s
        if not low.any():
            return s
        s = np.where(low, 2.0 * s, s)


def quantize(x, block_rows, scale):
    """(q as values, scales) of a float64 matrix that holds values of a 32- or 16-bit type."""
    rows, cols = x.shape
    amax = block_amax(x, block_rows)
    if scale == "e8m0":
        s = scale_e8m0(amax)
        per = np.repeat(np.repeat(s, block_rows, 0)[:rows], BLOCK, 1)[:, :cols]
        with np.errstate(all="ignore"):
            return round_e4m3(x / per), s
    a = np.maximum(amax.astype(np.float32), np.float32(2.0 ** -100))
    s, inv = a / np.float32(448), np.float32(448) / a  # (numpy divides and multiplies fp32 with one rounding)
    per = np.repeat(np.repeat(inv, block_rows, 0)[:rows], BLOCK, 1)[:, :cols]
    with np.errstate(all="ignore"):
        v = x.astype(np.float32) * per
    return round_e4m3(np.where(np.isfinite(x), v, np.nan)), s.astype(np.float64)


def matmul(a, sa, b, sb):
    """(sums, sums of magnitudes), float64: operands as values, scales as values."""
    k = a.shape[1]
    rows = np.repeat(sb, BLOCK, 0)[:b.shape[0]]
    wide = lambda s: np.repeat(s, BLOCK, 1)[:, :k]  # noqa: E731
    av, bv = a * wide(sa), b * wide(rows)
    return av @ bv.T, np.abs(av) @ np.abs(bv).T


def distribution(x, t=1.0, top_k=0, top_p=1.0, min_p=0.0):
    """Weights of one row in the order of the indices, zero where a candidate does not stay. Settings as fp32 holds them."""
    t, top_p, min_p = (float(np.float32(v)) for v in (t, top_p, min_p))
    x = np.where(np.isnan(x), -np.inf, np.asarray(x, np.float64))
    w = np.zeros(len(x))
    if not len(x) or x.max() == -np.inf:
        return w
    best = x.max()
    if not t > 0:
        w[int(np.argmax(x))] = 1.0
        return w
    with np.errstate(all="ignore"):
        raw = np.where(x == best, 1.0, np.exp((x - best) / t))
    raw = np.where(np.isnan(raw), 0.0, raw)
    order = sorted(np.nonzero(raw > 0)[0], key=lambda j: (-x[j], j))
    if top_k > 0:
        order = order[:top_k]
    if top_p < 1:
        part, total, n = 0.0, float(np.sum(raw[order])), 0
        while n < len(order) and (n == 0 or part < max(top_p, 0.0) * total):
            part += raw[order[n]]
            n += 1
        order = order[:n]
    stays = [j for j in order if raw[j] >= min(min_p, 1.0)]
    w[stays] = raw[stays]
    return w


def check_draws(x, u, idx, logp, **settings):
    """Every draw is where the definition puts it. A weight is held to 2^-s with s >= 62 - bits of the length (52 at most),
    each off by half of that: a border is off by no more than len * 2^-s, and 64-bit sums lose far less."""
    w = distribution(x, **settings)
    cum = np.cumsum(w)
    if not cum.size or cum[-1] == 0:
        assert (np.asarray(idx) == -1).all() and (np.asarray(logp) == -np.inf).all()
        return
    total = cum[-1]
    tol = len(x) * 2.0 ** -min(52, 62 - len(x).bit_length()) + total * len(x) * 2.0 ** -52
    for q, (uq, j, lp) in enumerate(zip(np.asarray(u, np.float64), idx, logp)):
        assert 0 <= j < len(x), (q, j)
        target = min(max(uq, 0.0), 1 - 2.0 ** -24) * total
        assert w[j] > 0, (q, j, "does not stay")
        assert cum[j] - w[j] - tol <= target <= cum[j] + tol, (q, j, cum[j] - w[j], target, cum[j])
        want = np.log(w[j] / total)
        # one rounding to fp32, beside what the weights' rounding moves the sum by
        assert abs(lp - want) <= 2.0 ** -24 * abs(want) + 2 * tol / total + 1e-12, (q, lp, want)
