"""The AdamW step in float32, operation for operation as it is stated, and moments in 8 bits.

Blocks of 128 elements have a power of two each, 2^(s - 127): m in e4m3, u = sqrt(v) without a sign in four bits of exponent
and four of mantissa.  A code is floor(|x| / step + r / 65536), step the code's spacing at |x| and r 16 random bits.
"""
import numpy as np

from oracle import philox

F = np.float32
# bits of the mantissa, largest number, code of a NaN
KINDS = {"m": (3, 448.0, 0x7F), "u": (4, 480.0, 0xFF)}


def constants(lr, beta1, beta2, eps, weight_decay, t):
    b1, b2, lr = F(beta1), F(beta2), F(lr)
    return dict(b1=b1, c1=F(1) - b1, b2=b2, c2=F(1) - b2, eps=F(eps), decay=F(1) - lr * F(weight_decay),
                step=F(float(lr) / (1 - float(b1) ** t)), r=F(1 / np.sqrt(1 - float(b2) ** t)))


def step(p, g, m, v, k, scale=None):
    """(p, m, v, sqrt(v)) after one step; float32 arrays, every operation rounded."""
    with np.errstate(all="ignore"):
        if scale is not None:
            g = g * F(scale)
        p = p * k["decay"]
        m = k["b1"] * m + k["c1"] * g
        v = k["b2"] * v + k["c2"] * (g * g)
        u = np.sqrt(v)
        p = p - (k["step"] * m) / (u * k["r"] + k["eps"])
    return p, m, v, u


def encode(x, kind, random):
    """(codes, scale bytes) of x (a multiple of 128 of them); random: 16 bits each."""
    bits, top, nan = KINDS[kind]
    a = np.abs(x.astype(np.float64)).reshape(-1, 128)
    finite = np.isfinite(a)
    a = np.where(finite, a, 0)
    big = a.max(1)
    e = np.frexp(np.where(big > 0, big, 1) / top)[1] - 1
    e = np.where(np.ldexp(top, e) >= big, e, e + 1)
    e = np.where(big > 0, np.maximum(e, -126), -126)
    t = a * np.exp2(-e.astype(np.float64))[:, None]
    field = np.where(t > 0, np.maximum(np.frexp(t)[1] - 1, -6), -6)
    spacing = np.exp2(field - float(bits))
    q = np.floor(np.floor(t / spacing * 65536) / 65536 + random.reshape(-1, 128) / 65536).astype(np.int64)
    # of q spacings: the leading one's place carries into the exponent's field by itself
    code = ((field + 6) << bits) + q
    if kind == "u":
        code = np.where(a > 0, np.maximum(code, 1), code)
    code = np.where(finite, code, nan)
    if kind == "m":
        code = code | np.where(np.signbit(x.reshape(-1, 128)), 0x80, 0)
    return code.astype(np.uint8).reshape(-1), (e + 127).astype(np.uint8)


def decode(codes, scales, kind):
    """float32 values."""
    bits, _, nan = KINDS[kind]
    c = codes.astype(np.int64).reshape(-1, 128)
    sign = (c & 0x80) != 0 if kind == "m" else np.zeros_like(c, bool)
    c = c & 0x7F if kind == "m" else c
    field, m = c >> bits, c & ((1 << bits) - 1)
    v = np.where(field == 0, m, m + (1 << bits)) * np.exp2(np.maximum(field - 1, 0) - 6.0 - bits)
    v = v * np.exp2(np.clip(scales.astype(np.float64), 1, 247) - 127)[:, None]
    v = np.where(c == nan, np.nan, v)
    with np.errstate(over="ignore"):
        return np.where(sign, -v, v).astype(F).reshape(-1)


def step8(p, g, state, k, seed, t, tensor_id, scale=None):
    """(p, state) after one step; state: (codes of m, codes of u, scales [blocks, 2]); p, g flat."""
    n = p.size
    m, u = decode(state[0], state[2][:, 0], "m")[:n], decode(state[1], state[2][:, 1], "u")[:n]
    p, m, _, u = step(p, g, m, u * u, k, scale)
    whole = -(-n // 128) * 128
    words = philox.noise_words(seed, t, tensor_id, np.arange(whole, dtype=np.uint64)).astype(np.int64)
    pad = lambda x: np.concatenate([x, np.zeros(whole - n, F)])  # noqa: E731
    cm, sm = encode(pad(m), "m", words & 0xFFFF)
    cu, su = encode(pad(u), "u", words >> 16)
    return p, (cm, cu, np.stack([sm, su], 1))
