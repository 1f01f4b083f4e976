"""CPU oracle for the operators of a training step (numpy). TEST INFRASTRUCTURE ONLY, shares nothing with the library.

The definitions are those of include/ckpt_train.h: block-scaled 4-bit and 8-bit formats by search in the table of the
format's values, stochastic rounding from the same counter-based random bits, the product of decoded matrices in
float64, the AdamW step with moments in float32 operation by operation and the rest in float64.
"""
import numpy as np

from oracle.proxy_oracle import bf16_bits, bf16_to_f64, mix

MXFP4, MXFP8 = 1, 2
U64 = (1 << 64) - 1

# values of the codes without sign, in code order
FP4 = np.array([0, 0.5, 1, 1.5, 2, 3, 4, 6])
FP8 = np.array([(m / 8 if e == 0 else 1 + m / 8) * 2.0 ** (max(e, 1) - 7) for e in range(16) for m in range(8)][:127])      # the last one is 448
GRID = {MXFP4: FP4, MXFP8: FP8}
SIGN = {MXFP4: 8, MXFP8: 128}


def scale_bytes(blocks, fmt):
    """blocks: [..., 32] float64 -> biased exponents; 255 where something is not finite."""
    top = GRID[fmt][-1]
    out = np.zeros(blocks.shape[:-1], np.int64)
    amax = np.abs(blocks).max(-1)
    bad = ~np.isfinite(blocks).all(-1)
    powers = top * 2.0 ** np.arange(-127.0, 128.0)          # what fits under each exponent
    out = np.searchsorted(powers, np.where(bad, 0, amax), side="left")
    return np.where(bad, 255, out).astype(np.uint8)


def blocks_of(x):
    rows, cols = x.shape
    nb = -(-cols // 32)
    b = np.zeros((rows, nb * 32))
    b[:, :cols] = x
    return b.reshape(rows, nb, 32)


def bits16(key, rows, cols):
    """[rows, cols] random sixteen-bit numbers; every row begins with a group of four of its own."""
    groups = -(-cols // 4)
    with np.errstate(over="ignore"):
        r = mix(np.uint64(key & U64) + np.arange(rows * groups, dtype=np.uint64))
    return np.stack([(r >> np.uint64(16 * j)) & np.uint64(0xFFFF) for j in range(4)], -1).astype(np.int64).reshape(rows, 4 * groups)[:, :cols]


def element_codes(y, fmt, random=None, nonzero=False):
    """Codes of scaled values |y| <= the format's largest, sign included. NaN: 0x7F in 8 bits, 0 in 4."""
    grid, a = GRID[fmt], np.abs(y)
    nan = np.isnan(y)
    a = np.where(nan, 0, a)
    below = np.searchsorted(grid, a, side="right") - 1       # the code at or under a
    above = np.minimum(below + 1, len(grid) - 1)
    lo, hi = grid[below], grid[above]
    if random is None:
        up = (a - lo > hi - a) | ((a - lo == hi - a) & (below % 2 == 1) & (hi > lo))
    else:
        step = np.where(hi > lo, hi - lo, 1)
        up = np.floor((a - lo) / step * 65536) + random >= 65536        # the distance in 2^16ths of a step, cut
    code = np.where(up, above, below)
    if nonzero:
        code = np.where((a > 0) & (code == 0), 1, code)
    code = np.where(nan, 0x7F if fmt == MXFP8 else 0, code)
    return (code + np.where(np.signbit(y), SIGN[fmt], 0)).astype(np.uint8)


def quantize(x, fmt, key=None, nonzero=False):
    """x: [rows, cols] values (float32 or less) -> codes [rows, cols], one a byte, and scale bytes [rows, ceil(cols / 32)]. key: stochastic."""
    x = np.asarray(x, np.float64)
    rows, cols = x.shape
    b = blocks_of(x)
    byte = scale_bytes(b, fmt)
    inverse = np.where(byte == 255, np.nan, 2.0 ** (127.0 - byte.astype(np.float64)))
    with np.errstate(invalid="ignore"):
        y = (b * inverse[..., None]).reshape(rows, -1)[:, :cols]
    return element_codes(y, fmt, None if key is None else bits16(key, rows, cols), nonzero), byte


def values(codes, byte, fmt):
    grid = np.append(GRID[fmt], np.nan) if fmt == MXFP8 else GRID[fmt]
    v = grid[codes & (SIGN[fmt] - 1)] * np.where(codes & SIGN[fmt], -1.0, 1.0)
    scale = np.where(byte == 255, np.nan, 2.0 ** (byte.astype(np.float64) - 127))
    return v * np.repeat(scale, 32, axis=1)[:, : codes.shape[1]]


def pack_rows(codes, byte, fmt, code_pitch, scale_pitch):
    """Codes and scales as they lie in memory, rows filled up with zeros."""
    rows, cols = codes.shape
    c, s = np.zeros((rows, code_pitch), np.uint8), np.zeros((rows, scale_pitch), np.uint8)
    if fmt == MXFP4:
        even = np.zeros((rows, 2 * code_pitch), np.uint8)
        even[:, :cols] = codes
        c[:] = even[:, 0::2] | (even[:, 1::2] << 4)
    else:
        c[:, :cols] = codes
    s[:, : byte.shape[1]] = byte
    return c, s


def gemm(a, b, c=None):
    """A [M, K], B [N, K] values -> (A B^T (+ C), the sum of the products' magnitudes) in float64."""
    return a @ b.T + (0 if c is None else c), np.abs(a) @ np.abs(b).T


def half_bits(x32, dtype):
    return bf16_bits(x32) if dtype == "bf16" else np.asarray(x32, np.float32).astype(np.float16).view(np.uint16)


def half_values(bits, dtype):
    return bf16_to_f64(bits) if dtype == "bf16" else np.asarray(bits, np.uint16).view(np.float16).astype(np.float64)


def moments(m, v, g, scale, beta1, beta2):
    """float32 in, float32 out, every operation rounded."""
    f = np.float32
    with np.errstate(over="ignore", invalid="ignore"):
        g = (np.asarray(g, f) * f(scale)).astype(f)
        m = np.asarray(m, f) * f(beta1) + g * f(1.0 - beta1)
        v = np.asarray(v, f) * f(beta2) + (g * g) * f(1.0 - beta2)
    return m, v


def adamw(master, m, v, lr, beta1, beta2, eps, step, weight_decay):
    """(new master, the update's size) in float64 from the step's new moments."""
    m, v = np.asarray(m, np.float64), np.asarray(v, np.float64)
    update = lr * (m / (1 - beta1 ** step)) / (np.sqrt(v / (1 - beta2 ** step)) + eps)
    return np.asarray(master, np.float64) * (1 - lr * weight_decay) - update, np.abs(update)


def step_bits16(seed, step, first_block, numel):
    """Random numbers of one tensor's elements: those of m, those of v."""
    with np.errstate(over="ignore"):
        key = int(mix(mix(np.uint64(seed & U64)) + np.uint64(step)))
    r = bits16(key + 8 * first_block, 1, -(-numel // 4) * 4).reshape(-1, 4)
    return r.reshape(1, -1)[:, :numel], r[:, ::-1].reshape(1, -1)[:, :numel]


def moment8(x, random=None, nonzero=False):
    """A flat f32 moment in 8 bits with given random numbers [1, n]."""
    b = blocks_of(np.asarray(x, np.float64).reshape(1, -1))
    byte = scale_bytes(b, MXFP8)
    inverse = np.where(byte == 255, np.nan, 2.0 ** (127.0 - byte.astype(np.float64)))
    with np.errstate(invalid="ignore"):
        y = (b * inverse[..., None]).reshape(1, -1)[:, : x.size]
    return element_codes(y, MXFP8, random, nonzero).reshape(-1), byte.reshape(-1)
