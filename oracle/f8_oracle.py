"""Plain CPU oracle of the operators with 8-bit matrices in blocks of 128 (include/ckpt_train.h): conversion to the bit in f32 arithmetic as the header defines it, everything else in 64 bits. Shares nothing with the library."""
import numpy as np

E4M3, E5M2 = 3, 4
MOST = {E4M3: 448.0, E5M2: 57344.0}
HALF_STEP = {E4M3: 2.0 ** -4, E5M2: 2.0 ** -3}                # of a value that is not subnormal, relative to it, at most
HALF_SMALLEST = {E4M3: 2.0 ** -10, E5M2: 2.0 ** -17}          # of a subnormal one, in units of the scale


def _table(fmt):
    """The value of every code."""
    fraction_bits, bias = (3, 7) if fmt == E4M3 else (2, 15)
    code = np.arange(256)
    e, f = (code & 0x7F) >> fraction_bits, code & ((1 << fraction_bits) - 1)
    v = np.where(e == 0, f * 2.0 ** (1 - bias - fraction_bits), (1 + f / 2 ** fraction_bits) * 2.0 ** (e - bias))
    if fmt == E4M3:
        v[(code & 0x7F) == 0x7F] = np.nan
    else:
        v[(code & 0x7F) == 0x7C] = np.inf
        v[(code & 0x7F) > 0x7C] = np.nan
    return np.where(code & 0x80, -v, v)


TABLE = {f: _table(f) for f in (E4M3, E5M2)}


def nearest_codes(y, fmt):
    """Codes of values up to the largest (and what rounds to it), ties to the even code; NaN: the code 0x7F."""
    finite = TABLE[fmt][: 0x7F if fmt == E4M3 else 0x7C]
    a = np.abs(np.nan_to_num(y.astype(np.float64), nan=0.0, posinf=0.0, neginf=0.0))
    above = np.clip(np.searchsorted(finite, a, side="left"), 1, len(finite) - 1)      # finite[above - 1] <= a <= finite[above]
    middle = (finite[above - 1] + finite[above]) / 2
    code = np.where((a > middle) | ((a == middle) & (above % 2 == 0)), above, above - 1)
    code = np.where(np.isnan(y), 0x7F, code)
    return (code | np.where(np.signbit(y), 0x80, 0)).astype(np.uint8)


def padded(n):
    return -(-n // 128) * 128


def quantize(x, fmt, block_rows=1):
    """(codes in rows of a multiple of 128, scales [blocks of columns, rows / block_rows]) of an f32 matrix."""
    x = np.asarray(x, np.float32)
    rows, cols = x.shape
    full = np.zeros((-(-rows // block_rows) * block_rows, padded(cols)), np.float32)
    full[:rows, :cols] = x
    blocks = full.reshape(-1, block_rows, full.shape[1] // 128, 128)
    amax = np.abs(blocks).max((1, 3))                     # NaN where there is one
    with np.errstate(all="ignore"):
        most = np.float32(MOST[fmt])
        scale = np.maximum(amax / most, np.float32(2.0 ** -126))
        inverse = np.minimum(np.where(amax == 0, np.inf, most / amax).astype(np.float32), np.float32(2.0 ** 126))
        bad = ~np.isfinite(amax)
        scale[bad] = inverse[bad] = np.nan
        y = blocks * inverse[:, None, :, None]
    codes = nearest_codes(y, fmt).reshape(full.shape)[:rows]
    codes[:, cols:] = 0
    return codes, np.ascontiguousarray(scale.T)


def values(codes, scales, fmt, cols, block_rows=1):
    rows = codes.shape[0]
    scale = np.repeat(np.repeat(scales.astype(np.float64).T, block_rows, 0)[:rows], 128, 1)
    return (TABLE[fmt][codes] * scale[:, : codes.shape[1]])[:, :cols]


def _sigmoid(z):
    return np.where(z >= 0, 1 / (1 + np.exp(-np.abs(z))), np.exp(-np.abs(z)) / (1 + np.exp(-np.abs(z))))


def gate(name, g):
    """(act(g), act'(g), z, dz/dg) in 64 bits, act(g) = g / (1 + exp(-z))."""
    g = np.asarray(g, np.float64)
    k = 2 * np.sqrt(2 / np.pi)
    z, dz = (g, np.ones_like(g)) if name == "silu" else (k * (g + 0.044715 * g ** 3), k * (1 + 3 * 0.044715 * g * g))
    s = _sigmoid(z)
    return g * s, s + g * s * _sigmoid(-z) * dz, z, dz


# f32 sums of a block by the matrix cores, then of the blocks: every rounding is at most 2^-24 of the sum of the magnitudes, and there are no more than so many of them on the way of a product.
def sum_error(a, b):
    """Bound of a product's f32 error, for each element."""
    k = a.shape[1]
    return (min(k, 128) + -(-k // 128) + 4) * 2.0 ** -24 * (np.abs(a) @ np.abs(b).T)


def forward(x, wg, wu, name):
    """{"gate", "up", "h"}: (value, bound of the f32 error)."""
    g, u = x @ wg.T, x @ wu.T
    eg, eu = sum_error(x, wg), sum_error(x, wu)
    act, slope, z, dz = gate(name, g)
    # exp(-z): z and its product with log2(e) are each rounded a few times, relative to |z|; the rest is some ten roundings; |act'| is at most 1.13
    e_act = 1.13 * eg + np.abs(act) * (4 * np.abs(z) + 10) * 2.0 ** -24
    return {"gate": (g, eg), "up": (u, eu), "h": (act * u, e_act * (np.abs(u) + eu) + np.abs(act) * eu + np.abs(act * u) * 2.0 ** -23)}


def backward(dy, wd, g, u, name):
    """{"dgate", "dup", "h"}: (value, bound of the f32 error) from the values of gate and up as they are held."""
    dh, e = dy @ wd.T, sum_error(dy, wd)
    act, slope, z, dz = gate(name, g)
    s = _sigmoid(z)
    rounding = (4 * np.abs(z) + 16) * 2.0 ** -24
    e_slope = (s + np.abs(act * dz)) * rounding          # 1 - s is off by s's error, which may be all that is left of it
    e_act = np.abs(act) * rounding
    return {"dgate": (dh * u * slope, np.abs(u) * (e * (np.abs(slope) + e_slope) + np.abs(dh) * e_slope) + np.abs(dh * u * slope) * 2.0 ** -22),
            "dup": (dh * act, e * (np.abs(act) + e_act) + np.abs(dh) * e_act + np.abs(dh * act) * 2.0 ** -23),
            "h": (act * u, e_act * np.abs(u) + np.abs(act * u) * 2.0 ** -23)}


def wrong_rounding(codes, scales, exact, error, fmt):
    """What is wrong with codes and scales (block_rows 1) as the rounding of values within `error` of `exact`; None if nothing is."""
    rows, cols = exact.shape
    if codes.shape != (rows, padded(cols)) or scales.shape != (padded(cols) // 128, rows):
        return "shape"
    if np.any(codes[:, cols:]):
        return "padding"

    def blocks(v):
        full = np.zeros((rows, padded(cols)))
        full[:, :cols] = v
        return full.reshape(rows, -1, 128).max(2)
    amax, most_error = blocks(np.abs(exact)), blocks(error)
    off = np.abs(np.maximum(amax / MOST[fmt], 2.0 ** -126) - scales.T)
    if np.any(off > (most_error + amax * 2.0 ** -23) / MOST[fmt]):
        return "scale"
    got = values(codes, scales, fmt, cols)
    scale = np.repeat(scales.T.astype(np.float64), 128, 1)[:, :cols]
    # half a step of the value that was rounded; the product with the inverse of the scale and the scale itself are off by a few roundings
    allowed = np.maximum(HALF_STEP[fmt] * (np.abs(exact) + error), HALF_SMALLEST[fmt] * scale) * (1 + 2.0 ** -20) + error + np.abs(exact) * 2.0 ** -22
    if np.any(np.abs(got - exact) > allowed):
        return "code"
    return None
