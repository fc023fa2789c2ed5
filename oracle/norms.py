"""Group normalisation with an activation (forward and backward), and tensors held in 8 bits, from their definitions in float64:
the oracle of fdg_gn_* and fdg_ckpt_* (include/fdg_ops.h).  Tensors are [N, pixels, C]; no code is shared with the library."""
import numpy as np

CKPT_BLOCK = 32


# ---- group norm ------------------------------------------------------------------------------------------------------

def _by_group(t, groups):
    """[N, pixels, C] -> [N, groups, pixels * channels of a group]."""
    n, p, c = t.shape
    return t.reshape(n, p, groups, c // groups).transpose(0, 2, 1, 3).reshape(n, groups, -1)


def _by_pixel(t, groups, c):
    n = t.shape[0]
    return t.reshape(n, groups, -1, c // groups).transpose(0, 2, 1, 3).reshape(n, -1, c)


def activation(z, act):
    if act == "relu":
        return np.maximum(z, 0.0)
    if act == "silu":
        with np.errstate(over="ignore"):
            return z / (1.0 + np.exp(-z))
    return z


def activation_slope(z, act):
    if act == "relu":
        return (z > 0).astype(np.float64)
    if act == "silu":
        with np.errstate(over="ignore"):
            s = 1.0 / (1.0 + np.exp(-z))
        return s * (1.0 + z * (1.0 - s))
    return np.ones_like(z)


def groupnorm_stats(x, groups, eps):
    """mean, rstd [N, groups]; biased variance."""
    g = _by_group(x, groups)
    mean = g.mean(-1)
    var = ((g - mean[..., None]) ** 2).mean(-1)
    return mean, 1.0 / np.sqrt(var + eps)


def groupnorm_xhat(x, stats, groups):
    mean, rstd = stats
    return _by_pixel((_by_group(x, groups) - mean[..., None]) * rstd[..., None], groups, x.shape[-1])


def groupnorm_forward(x, groups, gamma, beta, eps, act="none", res=None):
    """(y, z, (mean, rstd))."""
    stats = groupnorm_stats(x, groups, eps)
    z = groupnorm_xhat(x, stats, groups) * gamma + beta
    if res is not None:
        z = z + res
    return activation(z, act), z, stats


def groupnorm_backward(dz, x, stats, groups, gamma, res=None):
    """(dx, dgamma, dbeta) from the gradient dz of the normalisation's output (the activation's slope already applied)."""
    xhat = groupnorm_xhat(x, stats, groups)
    h, hx = _by_group(dz * gamma, groups), _by_group(xhat, groups)
    d = stats[1][..., None] * (h - h.mean(-1, keepdims=True) - hx * (h * hx).mean(-1, keepdims=True))
    dx = _by_pixel(d, groups, x.shape[-1])
    return dx if res is None else dx + res, (dz * xhat).sum((0, 1)), dz.sum((0, 1))


# ---- 8 bits ------------------------------------------------------------------------------------------------------------

def ckpt_encode(x):
    """(codes int8 [rows, C], scale bytes uint8 [rows, blocks]) of a [rows, C] array, block by block."""
    rows, c = x.shape
    blocks = -(-c // CKPT_BLOCK)
    codes = np.zeros((rows, c), np.int8)
    scales = np.zeros((rows, blocks), np.uint8)
    for r in range(rows):
        for b in range(blocks):
            v = np.asarray(x[r, b * CKPT_BLOCK:(b + 1) * CKPT_BLOCK], np.float64)
            if not np.isfinite(v).all():
                scales[r, b] = 255
                continue
            top = np.abs(v).max()
            e = -126
            if top > 0:
                e = max(int(np.floor(np.log2(top))) - 9, -126)
                while np.rint(np.ldexp(top, -e)) > 127 and e < 121:
                    e += 1
            codes[r, b * CKPT_BLOCK:(b + 1) * CKPT_BLOCK] = np.clip(np.rint(np.ldexp(v, -e)), -127, 127)
            scales[r, b] = e + 127
    return codes, scales


def ckpt_decode(codes, scales):
    rows, c = codes.shape
    step = np.where(scales == 255, np.nan, np.ldexp(1.0, scales.astype(np.int64) - 127))
    return codes.astype(np.float64) * np.repeat(step, CKPT_BLOCK, 1)[:, :c]
