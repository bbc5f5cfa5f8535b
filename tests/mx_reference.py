"""Pages whose elements share a power of two by blocks of 32, in 64 bits.

An element is a code of `bits` bits after the leading one, with the lowest exponent
`low`: e4m3 has 3 and -6 (values up to 448), e2m1 has 1 and 0 (up to 6)."""
import numpy as np

KINDS = {"mx8": (3, -6, 448.0), "mx4": (1, 0, 6.0)}


def values(kind):
    """What the codes 0, 1, 2, ... stand for, the sign apart; e4m3's last is NaN."""
    bits, low, most = KINDS[kind]
    got = []
    for code in range(1 << (7 if kind == "mx8" else 3)):
        e, m = code >> bits, code & ((1 << bits) - 1)
        got.append(m * 2.0 ** (low - bits) if e == 0 else (1 + m * 2.0 ** -bits) * 2.0 ** (low + e - 1))
    if kind == "mx8":
        got[-1] = np.nan
    assert got[-2 if kind == "mx8" else -1] == most
    return np.array(got)


def powers_of(blocks, kind):
    """The bytes of blocks (..., 32): the first power that is enough, going up."""
    a = np.abs(blocks).max(-1)
    finite = np.isfinite(blocks).all(-1)
    e = np.where(a == 0, -127, np.maximum(np.frexp(np.where(finite, a, 1.0))[1] - 12, -127))    # too small, or the least there is
    for _ in range(16):
        e = np.where(finite & (a > KINDS[kind][2] * 2.0 ** e), e + 1, e)
    assert (~finite | (a <= KINDS[kind][2] * 2.0 ** e)).all()
    return np.where(finite, e + 127, 255).astype(np.uint8)


def nearest(x, kind):
    """The codes of the values nearest to x, of two as near the even one, signs in the top bit."""
    table = values(kind)
    table = table[np.isfinite(table)]
    off = np.abs(np.abs(x)[..., None] - table)
    best = off.min(-1, keepdims=True)
    at = (off == best)
    code = at.argmax(-1)                                    # the lower of two
    code = np.where(at.sum(-1) > 1, code + (code & 1), code)
    return np.where(np.signbit(x), code + (128 if kind == "mx8" else 8), code).astype(np.uint8)


def pack(x, kind):
    """(elements, powers) of rows x (..., D): elements as bytes, two to one where they have 4 bits."""
    blocks = x.reshape(-1, 32)
    p = powers_of(blocks, kind)
    bad = p == 255
    u = np.where(bad[:, None], 0.0, blocks) / 2.0 ** (p.astype(np.float64) - 127)[:, None]
    code = nearest(u, kind)
    code[bad] = 0
    code = code.reshape(x.shape)
    if kind == "mx4":
        code = code[..., ::2] | code[..., 1::2] << 4
    return code, p.reshape(*x.shape[:-1], -1)


def unpack(code, powers, kind):
    """What the elements stand for."""
    if kind == "mx4":
        code = np.stack([code & 15, code >> 4], -1).reshape(*code.shape[:-1], -1)
    sign = 128 if kind == "mx8" else 8
    x = values(kind)[code & (sign - 1)] * np.where(code & sign, -1.0, 1.0)
    by = np.where(powers == 255, np.nan, 2.0 ** (powers.astype(np.float64) - 127))
    return x * np.repeat(by, 32, -1)
