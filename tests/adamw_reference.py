"""AdamW with 8-bit or 32-bit states, plainly, in numpy: the update in 64 bits
and the held form of m and v (the format is stated in include/mtdao.h)."""
import numpy as np

BLOCK = 256
U64 = np.uint64


def _table(exponent_bits, mantissa_bits, top):
    """The non-negative values of a small floating format, ascending, up to top."""
    bias = (1 << (exponent_bits - 1)) - 1
    vals = []
    for e in range(1 << exponent_bits):
        for f in range(1 << mantissa_bits):
            part = f / (1 << mantissa_bits)
            vals.append(part * 2.0 ** (1 - bias) if e == 0 else (1 + part) * 2.0 ** (e - bias))
    return np.array([v for v in vals if v <= top])


FORMATS = {"m": (_table(4, 3, 448.0), 7, 20), "v": (_table(5, 2, 57344.0), 14, 21)}


def state_offsets(numels):
    at, offs = 0, []
    for k in numels:
        offs.append(at)
        at += -(-k // BLOCK) * BLOCK
    return offs, at


def splitmix(z):
    with np.errstate(over="ignore"):
        z = (z ^ (z >> U64(30))) * U64(0xBF58476D1CE4E5B9)
        z = (z ^ (z >> U64(27))) * U64(0x94D049BB133111EB)
        return z ^ (z >> U64(31))


def words(seed, t, replica, n):
    """(low, high) 32-bit random words of the n elements of a replica's state vector."""
    golden = 0x9E3779B97F4A7C15
    with np.errstate(over="ignore"):
        key = splitmix(np.array([(seed + golden * (t + 1)) % (1 << 64)], U64))
        counter = (U64(replica) << U64(32)) + np.arange(n // 8, dtype=U64)
        z = splitmix(key + counter * U64(golden))
        odd = np.array([pow(0x9E3779B1, i + 1, 1 << 32) for i in range(8)], np.uint32)
        low = (z & U64(0xFFFFFFFF)).astype(np.uint32)[:, None] * odd
        high = (z >> U64(32)).astype(np.uint32)[:, None] * odd
    return low.reshape(-1), high.reshape(-1)


def nearest(values, table):
    """Round to the nearest entry, ties to the even one; larger than all: the largest."""
    a = np.minimum(np.abs(values), table[-1])
    hi = np.clip(np.searchsorted(table, a), 1, len(table) - 1)
    lo = hi - 1
    down, up = a - table[lo], table[hi] - a
    pick = np.where((up < down) | ((up == down) & (hi % 2 == 0)), hi, lo)
    return np.copysign(table[pick], values)


def block_scales(x, top):
    """Power of two of each block: its largest magnitude is in [2^top, 2^(top+1)) of it."""
    largest = np.abs(x.astype(np.float64)).reshape(-1, BLOCK).max(1)
    _, e = np.frexp(largest)
    return np.where(largest < 2.0 ** -110, 0.0, np.ldexp(1.0, e - 1 - top))


def scaled(x, name):
    """(values in units of their block's scale, scales), fp32 arithmetic."""
    _, top, _ = FORMATS[name]
    scale = block_scales(x, top)
    per = np.repeat(scale, BLOCK)
    with np.errstate(divide="ignore", invalid="ignore"):
        y = np.where(per > 0, x.astype(np.float64) / per, 0.0).astype(np.float32)
    if name == "v":
        y = np.where(per > 0, np.maximum(y, np.float32(2.0 ** -16)), y)
    return y, scale.astype(np.float32)


def hold(x, name, word=None):
    """(codes' values, scales) of an fp32 state vector; word: None for nearest."""
    table, _, drop = FORMATS[name]
    y, scale = scaled(x, name)
    if word is not None:
        by = (word >> np.uint32(32 - drop)).astype(np.int64) - (1 << (drop - 1))
        bits = (y.view(np.uint32).astype(np.int64) + by) & 0xFFFFFFFF
        y = np.where(np.abs(y) < 2.0 ** -30, np.float32(0), bits.astype(np.uint32).view(np.float32))
    return nearest(y.astype(np.float64), table), scale


def ema32(beta, s, target):
    """beta s + (1 - beta) target in fp32, each operation rounded."""
    b, c = np.float32(beta), np.float32(1.0 - beta)
    return (s * b) + (target * c)


def update64(p, g, m, v, t, lr, wd, betas, eps):
    """(p, m, v) after a step, in 64 bits."""
    p, g, m, v = (np.asarray(a, np.float64) for a in (p, g, m, v))
    m = betas[0] * m + (1 - betas[0]) * g
    v = betas[1] * v + (1 - betas[1]) * g * g
    hat = (m / (1 - betas[0] ** (t + 1))) / (np.sqrt(v / (1 - betas[1] ** (t + 1))) + eps)
    return p * (1 - lr * wd) - lr * hat, m, v
