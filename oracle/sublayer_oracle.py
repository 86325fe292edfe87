"""Plain float64 numpy of the operators around the pool layer: the norm in front of it, the balance loss over sequences, 8-bit values
with block scales and the experts on them.  Written from the definitions, one at a time, without blocking or fusion; it imports
nothing from the package."""
import numpy as np

E4M3_MAX = 448.0


# ---------------------------------------------------------------------------- norm
def rmsnorm(x, residual, weight, eps):
    """(h, y): h = x + residual, y = h / sqrt(mean(h^2) + eps) * weight."""
    h = np.asarray(x, np.float64)
    if residual is not None:
        h = h + np.asarray(residual, np.float64)
    s = 1.0 / np.sqrt(np.mean(h * h, axis=1, keepdims=True) + eps)
    return h, h * s * np.asarray(weight, np.float64)


def rmsnorm_bwd(h, weight, dy, dh, eps):
    """(dx, d_weight) of y = h s w with s = (mean h^2 + eps)^(-1/2): ds/dh_j = -s^3 h_j / d."""
    h, w, dy = (np.asarray(a, np.float64) for a in (h, weight, dy))
    s = 1.0 / np.sqrt(np.mean(h * h, axis=1, keepdims=True) + eps)
    g = w * dy
    dx = s * g - h * s ** 3 * np.mean(g * h, axis=1, keepdims=True)
    if dh is not None:
        dx = dx + np.asarray(dh, np.float64)
    return dx, np.sum(dy * h * s, axis=0)


# ---------------------------------------------------------------------------- balance loss over sequences
def seq_balance_loss(logits, topk_idx, offsets, alpha, router, sigma, c, eps):
    """(counts, loss, d_logits, d_sigma) of alpha / B' sum_b sum_i f_{b,i} P_{b,i}, sequence by sequence and token by token."""
    z = np.asarray(logits, np.float64)
    T, E = z.shape
    k = topk_idx.shape[1]
    B = len(offsets) - 1
    used = sum(1 for b in range(B) if offsets[b + 1] > offsets[b])
    counts = np.zeros((B, E), np.int64)
    loss, d_sigma, dz = 0.0, 0.0, np.zeros_like(z)
    for b in range(B):
        t0, t1 = offsets[b], offsets[b + 1]
        if t1 <= t0:
            continue
        for t in range(t0, t1):
            for j in range(k):
                counts[b, topk_idx[t, j]] += 1
        f = E * counts[b] / (k * (t1 - t0))
        coef = alpha * f / (used * (t1 - t0))           # d loss / d score, the same for every token of the sequence
        for t in range(t0, t1):
            if router == "softmax":
                p = np.exp(z[t] - z[t].max())
                p /= p.sum()
                loss += coef @ p
                dz[t] = p * (coef - coef @ p)
            else:
                n = np.sqrt(z[t] @ z[t])
                if n > 0:                               # logits that are all zero have no direction: nothing, also with eps = 0
                    s = sigma * c * np.maximum(z[t], 0.0) / (n + eps)
                    loss += coef @ s
                    d_sigma += coef @ s / sigma
                    gz = np.where(z[t] > 0, coef * sigma * c, 0.0)
                    dz[t] = gz / (n + eps) - z[t] * (gz @ z[t]) / (n * (n + eps) ** 2)
    return counts, loss, dz, d_sigma


# ---------------------------------------------------------------------------- 8-bit values with block scales
def e4m3_values():
    """Value of each of the 256 bytes: sign, 4 exponent bits (bias 7), 3 fraction bits; 0x7f and 0xff are NaN."""
    v = np.zeros(256)
    for b in range(256):
        e, m = (b >> 3) & 15, b & 7
        v[b] = (1 + m / 8.0) * 2.0 ** (e - 7) if e else m / 8.0 * 2.0 ** -6
        if b & 0x7f == 0x7f:
            v[b] = np.nan
        if b & 0x80:
            v[b] = -v[b]
    return v


def to_e4m3(v):
    """Nearest e4m3 byte of every value (|v| <= 448), ties to the even fraction, by comparison with the whole grid."""
    grid = e4m3_values()[:127]                          # the non-negative values, ascending; the byte's last bit says even or odd
    a = np.abs(np.asarray(v, np.float64))
    hi = np.clip(np.searchsorted(grid, a), 1, 126)
    lo = hi - 1
    dl, dh = a - grid[lo], grid[hi] - a
    code = np.where(dl < dh, lo, np.where(dh < dl, hi, np.where(lo % 2 == 0, lo, hi)))
    return (code + np.where(np.signbit(v), 128, 0)).astype(np.uint8)


def mx8_scale_bytes(rows, cols):
    return (-(-cols // 128), rows, 4)


def to_mx8(v):
    """(bytes [rows, cols], scale bytes [ceil(cols/128), rows, 4]) of a matrix, block by block."""
    v = np.asarray(v, np.float64)
    rows, cols = v.shape
    q = np.zeros((rows, cols), np.uint8)
    s = np.full(mx8_scale_bytes(rows, cols), 127, np.uint8)
    for b in range(cols // 32):
        blk = v[:, 32 * b:32 * b + 32]
        with np.errstate(invalid="ignore"):
            amax = np.max(np.abs(blk), axis=1)
        bad = ~np.isfinite(amax)
        amax = np.where(bad, 0.0, amax)
        e = np.full(rows, -127)
        while (amax > E4M3_MAX * 2.0 ** e).any():
            e = np.where(amax > E4M3_MAX * 2.0 ** e, e + 1, e)
        with np.errstate(invalid="ignore"):
            code = to_e4m3(np.where(bad[:, None], 0.0, blk) / (2.0 ** e)[:, None])
        q[:, 32 * b:32 * b + 32] = np.where(bad[:, None], 0x7f, code)
        s[b // 4, :, b % 4] = np.where(bad, 255, e + 127)
    return q, s


def from_mx8(q, s):
    """The values that the bytes stand for."""
    rows, cols = q.shape
    e = np.transpose(s, (1, 0, 2)).reshape(rows, -1)[:, :cols // 32].astype(np.int64) - 127
    scale = np.where(e == 128, np.nan, 2.0 ** np.minimum(e, 127))
    return e4m3_values()[q] * np.repeat(scale, 32, axis=1)


# ---------------------------------------------------------------------------- experts
def expert_h(x, offsets, w_gate_up):
    """H = silu(X W_gate^T) * (X W_up^T) of the rows in group order, not rounded."""
    S, (E, f2, _) = x.shape[0], w_gate_up.shape
    h = np.zeros((S, f2 // 2))
    for e in range(E):
        r = slice(offsets[e], offsets[e + 1])
        ab = x[r] @ w_gate_up[e].T
        a, b = ab[:, :f2 // 2], ab[:, f2 // 2:]
        h[r] = a / (1.0 + np.exp(-a)) * b
    return h


def expert_y(h, offsets, w_down):
    y = np.zeros((h.shape[0], w_down.shape[1]))
    for e in range(w_down.shape[0]):
        r = slice(offsets[e], offsets[e + 1])
        y[r] = h[r] @ w_down[e].T
    return y
