"""The operators on frozen rows in 64 bits, from their definition (numpy; no code of the library)."""
import numpy as np

GRID = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def row_bytes(dim):
    return 4 if dim <= 8 else 8 if dim <= 16 else -(-dim // 32) * 16


def quantize(x):
    """(codes, scales) of the float32 rows x, and the float64 values they stand for."""
    x = np.asarray(x, dtype=np.float64)
    n, dim = x.shape
    blocks = -(-dim // 32)
    padded = np.zeros((n, 32 * blocks))
    padded[:, :dim] = x
    b = padded.reshape(n, blocks, 32)
    finite = np.isfinite(b).all(axis=2)
    most = np.abs(np.where(finite[:, :, None], b, 0.0)).max(axis=2)
    exponent = np.where(most > 0, np.frexp(most)[1] - 1 - 2, -127)
    exponent = np.clip(exponent, -127, 127)
    y = np.where(finite[:, :, None], b, 0.0) / np.exp2(exponent.astype(np.float64))[:, :, None]
    # the nearest magnitude; of two equally near ones the one with an even number
    off = np.abs(np.abs(y)[..., None] - GRID)
    order = np.array([0, 2, 4, 6, 1, 3, 5, 7])
    number = order[np.argmin(off[..., order], axis=-1)]
    code = (number | np.where(np.signbit(y), 8, 0)).astype(np.uint8)
    code[~finite] = 0
    scales = np.where(finite, exponent + 127, 255).astype(np.uint8)
    flat = code.reshape(n, -1)[:, :2 * row_bytes(dim)]
    codes = (flat[:, 0::2] | flat[:, 1::2] << 4).astype(np.uint8)
    return codes, scales, values(codes, scales, dim)


def values(codes, scales, dim):
    flat = np.stack((codes & 15, codes >> 4), axis=2).reshape(codes.shape[0], -1)
    v = np.where(flat & 8, -1.0, 1.0) * GRID[flat & 7]
    s = np.where(scales == 255, np.nan, np.exp2(scales.astype(np.float64) - 127))
    return v[:, :dim] * np.repeat(s, 32, axis=1)[:, :dim]


def scores(q, r, scale, bias=None):
    with np.errstate(invalid="ignore"):
        s = np.float64(np.float32(scale)) * (q @ r.T)
    if bias is not None:
        bias = np.asarray(bias, dtype=np.float64)
        out = ~np.isfinite(bias)
        s = s + np.where(out, 0.0, bias)
        s[:, out] = -np.inf
    return s


def log_probs(q, r, scale, bias=None, given=None):
    """lse, entropy, logp (of `given`), and the scores."""
    s = scores(q, r, scale, bias)
    n = s.shape[1]
    with np.errstate(all="ignore"):
        most = s.max(axis=1, initial=-np.inf, keepdims=True)
        most = np.where(np.isneginf(most), 0.0, most)
        lse = (most + np.log(np.exp(s - most).sum(axis=1, keepdims=True)))
        logp = s - lse
        p = np.where(np.isneginf(s), 0.0, np.exp(logp))
        entropy = -np.where(p == 0, 0.0, p * logp).sum(axis=1)
        out = {"scores": s, "lse": lse[:, 0], "entropy": entropy}
        if given is not None:
            v = np.take_along_axis(s, np.clip(given, 0, max(n - 1, 0)).astype(np.int64), axis=1) if n else np.zeros(given.shape)
            v = np.where(np.isneginf(v), v, v - lse)
            out["logp"] = np.where(given < 0, 0.0, np.where(given >= n, np.nan, v))
    return out


def query_gradient(q, r, scale, bias, given, u, h):
    """d (sum(u * logp) + sum(h * entropy)) / dq."""
    out = log_probs(q, r, scale, bias)
    s, (m, n) = out["scores"], out["scores"].shape
    with np.errstate(all="ignore"):
        logp = np.where(np.isneginf(s), 0.0, s - out["lse"][:, None])
        p = np.where(np.isneginf(s), 0.0, np.exp(logp))
    c = np.zeros((m, n))
    if h is not None:
        c -= np.asarray(h, dtype=np.float64)[:, None] * p * (logp + out["entropy"][:, None])
    if given is not None:
        for i in range(m):
            for j, g in enumerate(given[i]):
                if 0 <= g < n and not np.isneginf(s[i, g]):
                    c[i] -= float(u[i, j]) * p[i]
                    c[i, g] += float(u[i, j])
    kept = r if bias is None else np.where(np.isfinite(np.asarray(bias, dtype=np.float64))[:, None], r, 0.0)
    return np.float64(np.float32(scale)) * (c @ kept)
