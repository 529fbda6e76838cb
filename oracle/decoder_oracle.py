"""64-bit definitions of the 4-bit decoder operators (numpy, CPU): E2M1 quantisation, the norm with the residual's addition, products, cached attention."""
import numpy as np

LEVELS = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def e2m1_code(x):
    """Nearest level of |x| (ties to the even code, above 6 saturates), sign in bit 3."""
    a = np.abs(x)
    middle = (LEVELS[1:] + LEVELS[:-1]) / 2
    low = np.searchsorted(middle, a, "left")
    tie = (low < 7) & (a == middle[np.minimum(low, 6)]) & (low % 2 == 1)
    return ((low + tie) | (np.signbit(x).astype(np.int64) << 3)).astype(np.uint8)


def e2m1_value(code):
    return np.where(code & 8, -1.0, 1.0) * LEVELS[code & 7]


def group_exponent(x):
    """Smallest e >= -120 with max |x| <= 7 * 2^e over the last axis (found by comparisons: no logarithm decides)."""
    most = np.abs(x).max(-1)
    e = np.where(most == 0, -120, np.maximum(np.frexp(most)[1].astype(np.int64) - 6, -120))
    for _ in range(8):
        e += most > 7.0 * np.exp2(e)
    return e


def quantise_groups(x):
    """Rows [..., cols] -> codes [..., cols], exponents [..., cols / 32], values."""
    g = x.reshape(x.shape[:-1] + (x.shape[-1] // 32, 32))
    e = group_exponent(g)
    code = e2m1_code(g / np.exp2(e)[..., None])
    return code.reshape(x.shape), e, (e2m1_value(code) * np.exp2(e)[..., None]).reshape(x.shape)


def bf16(x):
    """Nearest bf16, ties to even, of numbers that fp32 holds exactly or that are rounded to fp32 first."""
    b = np.ascontiguousarray(np.asarray(x, np.float32)).view(np.uint32).astype(np.uint64)
    b = (b + 0x7fff + ((b >> 16) & 1)) & 0xffff0000
    return b.astype(np.uint32).view(np.float32).astype(np.float64)


def quantise_vectors(v):
    """Vectors [..., D] -> codes, scale [..., 1], values: s = max(bf16(max |v| / 6), 2^-120)."""
    s = np.maximum(bf16(np.abs(v).max(-1, keepdims=True).astype(np.float32) / np.float32(6)), 2.0 ** -120)
    code = e2m1_code(v / s)
    return code, s, e2m1_value(code) * s


def rmsnorm_residual(x, r, gain, eps):
    h = (0 if x is None else x) + (0 if r is None else r)
    y = h / np.sqrt((h ** 2).mean(-1, keepdims=True) + eps)
    return h, y if gain is None else y * gain


def attention(q, k, v, scale, seen):
    """q [n][H][D], k, v [keys][KV][D], seen [n]: (output, sum_j p_j |v_j|, largest scale * sum |q||k| of a visible key), a row without keys zero."""
    n, H, D = q.shape
    group = H // k.shape[1]
    out, spread, size = np.zeros((n, H, D)), np.zeros((n, H, D)), np.zeros((n, H))
    for i in range(n):
        c = min(int(seen[i]), k.shape[0])
        if c <= 0:
            continue
        for h in range(H):
            kk, vv = k[:c, h // group], v[:c, h // group]
            x = scale * (kk @ q[i, h])
            p = np.exp(x - x.max())
            p /= p.sum()
            out[i, h], spread[i, h] = p @ vv, p @ np.abs(vv)
            size[i, h] = abs(scale) * (np.abs(kk) @ np.abs(q[i, h])).max()
    return out, spread, size
