"""The packed 4-bit format from its definition, in Python and numpy doubles (shared by the tests of the 4-bit calls; no code
of the library)."""
import numpy as np

MAGNITUDES = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])
VALUES = np.concatenate([MAGNITUDES, -MAGNITUDES])


def nearest_code(v):
    """Code of the nearest magnitude, ties to the even code: v >= 0, any array."""
    d = np.abs(v[..., None] - MAGNITUDES)
    best = d.min(-1, keepdims=True)
    near = d == best                                     # one code, or two neighbours
    first = near.argmax(-1)
    two = near.sum(-1) == 2
    return np.where(two & (first % 2 == 1), first + 1, first)


def quantise(x):
    """x float64 [n][K] -> codes uint8 [n][Kp] and scale bytes uint8 [n][Kp/32], Kp = K rounded up to whole blocks."""
    n, K = x.shape
    Kp = -(-K // 32) * 32
    b = np.zeros((n, Kp))
    b[:, :K] = x
    b = b.reshape(n, Kp // 32, 32)
    bad = ~np.isfinite(b).all(-1)
    top = np.where(bad, 1.0, np.abs(np.where(np.isfinite(b), b, 0)).max(-1))
    e = np.maximum(np.floor(np.log2(np.where(top > 0, top, 2.0 ** -149))).astype(int) - 2, -127)
    # log2 of a double next to a power of two may be off: put it right against the powers themselves
    e = np.where((top >= 2.0 ** (e + 3.0)) & (top > 0), e + 1, e)
    e = np.maximum(np.where((top < 2.0 ** (e + 2.0)) & (e > -127), e - 1, e), -127)
    v = np.where(bad[..., None], 0.0, b) / (2.0 ** e)[..., None]
    code = nearest_code(np.abs(v)) + 8 * (np.signbit(v) & ~bad[..., None])
    byte = np.where(bad, 255, e + 127)
    return code.reshape(n, Kp).astype(np.uint8), byte.astype(np.uint8)


def scale_index(rows, K):
    """[rows][ceil(K/128)*4] positions of the scale bytes, by the layout's formula."""
    kt = -(-K // 128)
    r = np.arange(rows)[:, None]
    b = np.arange(kt * 4)[None]
    return ((r // 128) * kt + b // 4) * 512 + (r % 32) * 16 + (r % 128) // 32 * 4 + b % 4


def pack(x):
    """x -> data uint8 [n][Kp/2], scales uint8 [tiles*512]; bytes of rows that fill the last tile are 255 (they must not matter)."""
    n, K = x.shape
    code, byte = quantise(x)
    data = code[:, 0::2] | (code[:, 1::2] << 4)
    scales = np.full(-(-n // 128) * (-(-K // 128)) * 512, 255, np.uint8)
    full = np.full((n, -(-K // 128) * 4), 127, np.uint8)
    full[:, :byte.shape[1]] = byte
    scales[scale_index(n, K)] = full
    return np.ascontiguousarray(data), scales


def values(code, byte, K):
    n = code.shape[0]
    s = np.where(byte == 255, np.nan, 2.0 ** (byte.astype(float) - 127))
    return (VALUES[code].reshape(n, byte.shape[1], 32) * s[..., None]).reshape(n, code.shape[1])[:, :K]


def rounded(x):
    """The values that x stands for once packed."""
    return values(*quantise(x), x.shape[1])
