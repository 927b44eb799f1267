"""fp64 definitions of 8-bit rows and of the query / key norm with rotation over several axes (NumPy; test infrastructure, no code shared
with the HIP path).  Matrices are plain arrays; an element is its e4m3 value times its block's power of two."""
import numpy as np


def _e4m3_table():
    t = np.empty(256)
    for b in range(256):
        sign, e, m = -1.0 if b & 0x80 else 1.0, (b >> 3) & 15, b & 7
        if e == 15 and m == 7:
            t[b] = np.nan
        elif e:
            t[b] = sign * (1 + m / 8) * 2.0 ** (e - 7)
        else:
            t[b] = sign * m * 2.0 ** -9
    return t


E4M3 = _e4m3_table()
_POSITIVE = E4M3[:127]                 # 0 .. 448, increasing


def to_e4m3(v):
    """Bytes of the nearest e4m3 value, ties to the even one; v within [-448, 448] or NaN (0x7f)."""
    a = np.abs(v)
    finite = np.where(np.isnan(v), 0.0, a)
    hi = np.clip(np.searchsorted(_POSITIVE, finite), 0, 126)
    lo = np.maximum(hi - 1, 0)
    up, down = _POSITIVE[hi] - finite, finite - _POSITIVE[lo]
    b = np.where(up < down, hi, np.where(down < up, lo, np.where(hi % 2 == 0, hi, lo)))
    b = np.where(_POSITIVE[hi] == finite, hi, b)
    return np.where(np.isnan(v), 0x7F, b | np.where(np.signbit(v), 0x80, 0)).astype(np.uint8)


def scale_byte(big):
    """Exponent byte for the largest finite magnitude of a block: smallest e >= -127 with big <= 448 * 2^e."""
    e = np.full(np.shape(big), -127)
    for k in range(-127, 121):
        e = np.where(big > 448.0 * 2.0 ** k, k + 1, e)
    return (e + 127).astype(np.uint8)


def blocks(K):
    return -(-K // 128)


def quantize(x):
    """x [R, K] (fp64) -> bytes [R, 128 nb] with zeros behind column K, exponent bytes [R, nb]."""
    R, K = x.shape
    nb = blocks(K)
    p = np.zeros((R, nb * 128))
    p[:, :K] = x
    p = p.reshape(R, nb, 128)
    finite = np.isfinite(p)
    s = scale_byte(np.where(finite, np.abs(p), 0.0).max(-1))
    with np.errstate(invalid="ignore"):
        v = np.where(finite, p, np.nan) / 2.0 ** (s[..., None].astype(np.float64) - 127)
    return to_e4m3(v).reshape(R, nb * 128), s


def dequantize(data, scale, K):
    nb = blocks(K)
    s = np.where(scale[:, :nb] == 255, np.nan, 2.0 ** (scale[:, :nb].astype(np.float64) - 127))
    return (E4M3[data[:, :128 * nb]].reshape(len(data), nb, 128) * s[..., None]).reshape(len(data), -1)[:, :K]


def gelu(x):
    with np.errstate(over="ignore"):
        return x / (1 + np.exp(-2 * np.sqrt(2 / np.pi) * (x + 0.044715 * x ** 3)))


def linear(a, w, bias=None, act=False):
    y = a @ w.T
    if bias is not None:
        y = y + bias
    return gelu(y) if act else y


def layer_norm(x, eps=1e-6):
    d = x - x.mean(-1, keepdims=True)
    return d / np.sqrt((d * d).mean(-1, keepdims=True) + eps)


def mlp(x, shift, scale, w1, b1, w2, b2):
    """w1, w2: values of the 8-bit weights."""
    h = layer_norm(x) * (1 + scale) + shift
    h = dequantize(*quantize(h), h.shape[1])
    u = linear(h, w1, b1, True)
    u = dequantize(*quantize(u), u.shape[1])
    return linear(u, w2, b2)


def rope_factors(places, axis_dim, origin=(0, 0, 0), step=(1, 1, 1), theta=10000.0):
    out = []
    for n, d, o, s in zip(places, axis_dim, origin, step):
        angle = (o + s * np.arange(n, dtype=np.float64))[:, None] * theta ** (-np.arange(0, d, 2, dtype=np.float64) / max(d, 1))
        out.append(np.stack([np.cos(angle), np.sin(angle)], -1).reshape(-1, 2))
    return np.concatenate(out) if out else np.zeros((0, 2))


def qk_norm_rope(x, places, axis_dim, norm, gamma, beta, eps, rotate=True, **angles):
    """x [n, H, D] -> the same; norm: "none", "layer", "rms"."""
    n, H, D = x.shape
    if norm == "layer":
        y = layer_norm(x, eps)
    elif norm == "rms":
        y = x / np.sqrt((x * x).mean(-1, keepdims=True) + eps)
    else:
        y = x.copy()
    if gamma is not None:
        y = y * gamma
    if beta is not None:
        y = y + beta
    if not rotate:
        return y
    theta, origin, step = angles.get("theta", 10000.0), angles.get("origin", (0, 0, 0)), angles.get("step", (1, 1, 1))
    T, Y, X = places
    for token in range(n):
        g = token % (T * Y * X)
        place = (g // (Y * X), g // X % Y, g % X)
        first = 0
        for a in range(3):
            for i in range(axis_dim[a] // 2):
                angle = (origin[a] + step[a] * place[a]) * theta ** (-2 * i / axis_dim[a])
                c, s = np.cos(angle), np.sin(angle)
                u, v = y[token, :, first + 2 * i].copy(), y[token, :, first + 2 * i + 1].copy()
                y[token, :, first + 2 * i] = u * c - v * s
                y[token, :, first + 2 * i + 1] = u * s + v * c
            first += axis_dim[a]
    return y
