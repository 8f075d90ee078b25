"""Plain forms of the 8- and 4-bit formats in 64 bits (numpy), for the tests.  Not collected by pytest (no test_ prefix)."""
import numpy as np

E2M1 = np.array([0, 0.5, 1, 1.5, 2, 3, 4, 6, -0.0, -0.5, -1, -1.5, -2, -3, -4, -6])
# all e4m3 values: sign, four bits of exponent (bias 7, 0: subnormal), three of fraction; 0x7f and 0xff are NaN
E4M3 = np.array([(-1 if c & 128 else 1) * (np.nan if c & 127 == 127 else (c & 7) * 2.0 ** -9 if (c >> 3) & 15 == 0
                                          else (8 + (c & 7)) * 2.0 ** (((c >> 3) & 15) - 10)) for c in range(256)])


def scale_values(b):
    return np.where(b == 255, np.nan, 2.0 ** (b.astype(np.float64) - 127))


def scale_bytes(amax, top):
    """The smallest power of two s with amax <= top * s, as its byte; 0 for 0, 255 for infinity and NaN."""
    out = np.zeros(amax.shape, np.uint8)
    for i, a in np.ndenumerate(amax):
        if not np.isfinite(a):
            out[i] = 255
            continue
        e = 0
        if a > 0:
            e = max(0, int(np.floor(np.log2(a / top))) + 126)
            while a > top * 2.0 ** (e - 127):
                e += 1
        out[i] = e
    return out


def values4(W4, scales):
    """[C, D / 2] codes and [C, D / 32] scale bytes -> [C, D]."""
    codes = np.stack((W4 & 15, W4 >> 4), 2).reshape(W4.shape[0], -1)
    return E2M1[codes] * np.repeat(scale_values(scales), 32, 1)


def values8(q, scales):
    return E4M3[q] * np.repeat(scale_values(scales), 32, 1)


def quantize4(w):
    """Codes and scale bytes of [C, D] values: the nearest code, the even one of two that are equally near."""
    blocks = w.reshape(w.shape[0], -1, 32)
    s = scale_bytes(np.abs(blocks).max(2), 6.0)
    with np.errstate(invalid="ignore"):
        v = (blocks / scale_values(s)[:, :, None]).reshape(w.shape)
    a = np.abs(v)
    code = np.zeros(w.shape, np.uint8)
    for k, (edge, even_below) in enumerate([(0.25, 1), (0.75, 0), (1.25, 1), (1.75, 0), (2.5, 1), (3.5, 0), (5.0, 1)]):
        code[(a > edge) if even_below else (a >= edge)] = k + 1
    code |= np.where(np.signbit(w), 8, 0).astype(np.uint8)
    return code[:, 0::2] | (code[:, 1::2] << 4), s
