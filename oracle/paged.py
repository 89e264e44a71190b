"""64-bit reference of the paged key-value cache's operators and of the 4-bit projection (numpy, plain loops)."""
import numpy as np


def rows_of(lens, start):
    """[(sequence, position)] of every row of the batch, in row order; rows of nobody are None."""
    out = [None] * int(start[-1])
    for b in range(len(lens)):
        for t in range(int(start[b]), int(start[b + 1])):
            out[t] = (b, int(lens[b]) - (int(start[b + 1]) - t))
    return out


def rotate(x, pos, theta, dim):
    """x [heads][dh] at position pos: pairs (i, i + dim / 2) turned by pos * theta^(-2 i / dim)."""
    x = np.array(x, np.float64)
    h = dim // 2
    # angles in the host's long double, taken to one turn there: a double's last bit is 4e-7 rad at 2e9 tokens
    ang = np.longdouble(pos) * np.longdouble(theta) ** (np.arange(h).astype(np.longdouble) * -2 / dim)
    ang = np.remainder(ang, 2 * np.longdouble("3.14159265358979323846264338327950288")).astype(np.float64)
    c, s = np.cos(ang), np.sin(ang)
    a, b = x[..., :h].copy(), x[..., h:dim].copy()
    x[..., :h], x[..., h:dim] = a * c - b * s, b * c + a * s
    return x


def attend(q, keys, values, seen, scale):
    """q [group][dh] over keys, values [n][dh] where `seen` [n]: (out [group][dh], lse [group])."""
    k, v = keys[seen].astype(np.float64), values[seen].astype(np.float64)
    if not seen.any():
        return np.zeros(q.shape), np.full(len(q), -np.inf)
    with np.errstate(all="ignore"):
        z = scale * (q.astype(np.float64) @ k.T)
        top = z.max(axis=1, keepdims=True)
        p = np.exp(z - top)
        total = p.sum(axis=1, keepdims=True)
        return (p / total) @ v, (top + np.log(total))[:, 0]


def dequantize(q, scale, zero):
    """w [N][K] in 64 bits of bytes q [N][K / 2], scale [N][groups] and zero [N][groups] or None."""
    n, groups = scale.shape
    w = np.stack([q & 15, q >> 4], axis=-1).reshape(n, groups, -1).astype(np.float64)
    z = 8.0 if zero is None else (zero & 15).astype(np.float64)[..., None]
    return ((w - z) * scale.astype(np.float64)[..., None]).reshape(n, -1)
