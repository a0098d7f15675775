"""AdamW written from its formulas with numpy: in 64 bits, and in fp32 with one rounding for every operation (what m, v and the codes
of states in 8 bits are defined by).  Shares no code with the library."""
import numpy as np

BLOCK = 256
f32 = np.float32
TOP_M, TOP_V, LEAST = f32(448.0), f32(57344.0), f32(2.0 ** -110)


def step64(p, g, m, v, *, lr, beta1, beta2, eps, step, decay, k=1.0):
    """p', m', v' in 64 bits, and how far fp32 may be from p' (all arguments exact in 64 bits)."""
    p, g, m, v = (np.asarray(a, np.float64) for a in (p, g, m, v))
    g = k * g
    m2, v2 = beta1 * m + (1 - beta1) * g, beta2 * v + (1 - beta2) * g * g
    d = np.sqrt(v2) / np.sqrt(1 - beta2 ** step) + eps
    a = lr / (1 - beta1 ** step)
    p2 = p - (lr * decay * p + a * m2 / d)
    # Roundings of 2^-24 each.  m': 3 and those of b1, w1 and k g, of the parts that may cancel.  d: v' 5 and b2, w2, k g twice, halved
    # by the root; the root 2, r2 3, the product, eps and the sum: 13.  Quotient 4 (two units in the last place), a 3, product 1: 26 of the whole
    # term, where its parts do not cancel, and 2 more for m's.  rate p: 3,
    # the sum 1; the difference 1 of p'.
    term = a * (np.abs(beta1 * m) + np.abs((1 - beta1) * g)) / d
    slack = 2.0 ** -24 * (np.abs(p2) + 5 * np.abs(lr * decay * p) + 28 * term) + 1e-44
    return p2, m2, v2, slack


def moments32(g, m, v, *, beta1, beta2, k=1.0):
    """m', v' rounded operation by operation."""
    g = f32(k) * np.asarray(g, f32)
    m2 = f32(beta1) * m + f32(1 - beta1) * g
    v2 = f32(beta2) * v + (f32(1 - beta2) * g) * g
    assert m2.dtype == v2.dtype == f32
    return m2, v2


def philox(c0, c1, c2, c3, key):
    """Philox4x32-10 of arrays of 32-bit numbers held in 64 bits: four words."""
    u = np.uint64
    low, shift = u(0xFFFFFFFF), u(32)
    c = [np.asarray(x, u) for x in (c0, c1, c2, c3)]
    k = [key & 0xFFFFFFFF, key >> 32 & 0xFFFFFFFF]
    for _ in range(10):
        p0, p1 = u(0xD2511F53) * c[0], u(0xCD9E8D57) * c[2]
        c = [p1 >> shift ^ c[1] ^ u(k[0]), p1 & low, p0 >> shift ^ c[3] ^ u(k[1]), p0 & low]
        k = [(k[0] + 0x9E3779B9) & 0xFFFFFFFF, (k[1] + 0xBB67AE85) & 0xFFFFFFFF]
    return c


def draws(first_block, count, seed, step):
    """The 16-bit draws of the elements of `count` blocks."""
    q = np.arange(32 * count, dtype=np.uint64) + np.uint64(32 * first_block)
    words = philox(q & np.uint64(0xFFFFFFFF), q >> np.uint64(32), np.full_like(q, 0xFFFFFFFF), np.full_like(q, step), seed)
    h = np.zeros((count, BLOCK), np.uint32)
    lane = 4 * np.arange(32)
    for s in range(8):
        h[:, (s // 4) * 128 + lane + s % 4] = (words[s // 2] >> np.uint64(16 * (s % 2)) & np.uint64(0xFFFF)).reshape(count, 32)
    return h


def values_of(fraction_bits, exponent_bits):
    """The values of the codes 0 .. 2^(bits) - 1 of a float without sign."""
    bias = 2 ** (exponent_bits - 1) - 1
    out = []
    for code in range(2 ** (fraction_bits + exponent_bits)):
        e, f = code >> fraction_bits, code % 2 ** fraction_bits
        out.append((f if e == 0 else f + 2 ** fraction_bits) * 2.0 ** (max(e, 1) - bias - fraction_bits))
    return np.array(out)


E4M3, E5M2 = values_of(3, 4)[:0x7F], values_of(2, 5)[:0x7C]


def decode(codes, table, scale):
    """fp32 values of codes with (for e4m3) a sign."""
    sign = np.where(codes & 0x80, f32(-1), f32(1))
    return sign * table.astype(f32)[codes & 0x7F] * f32(scale)


def pack(x, top, table, h):
    """Scale and codes of a block's magnitudes: the lower neighbour's code, and one more where what is above it asks for it."""
    most = x.max()
    if not most >= LEAST:
        return f32(0), np.zeros(x.size, np.uint8)
    y = (x * (top / most)).astype(np.float64)
    low = np.searchsorted(table, y, side="right") - 1
    low = np.minimum(low, table.size - 2)
    share = (y - table[low]) / (table[low + 1] - table[low])
    return most / top, (low + (share + (h + 0.5) / 65536 >= 1)).astype(np.uint8)


def swapped(h):
    return (h & 0xFF) << 8 | h >> 8


def step8(p, g, m, v, scales, first_block, *, seed, step, beta1, beta2, k=1.0, **rest):
    """A tensor's step with states in 8 bits: p' and its slack as step64, codes of m and v, scales [blocks, 2]."""
    n = len(g)
    m2c, v2c, s2 = np.zeros(n, np.uint8), np.zeros(n, np.uint8), np.zeros_like(scales)
    wide_m, wide_v = np.zeros(n, f32), np.zeros(n, f32)
    blocks = -(-n // BLOCK)
    all_draws = draws(first_block, blocks, seed, step)
    for b in range(blocks):
        at = slice(b * BLOCK, min(n, (b + 1) * BLOCK))
        wide_m[at], wide_v[at] = decode(m[at], E4M3, scales[b, 0]), decode(v[at], E5M2, scales[b, 1])
        m2, v2 = moments32(g[at], wide_m[at], wide_v[at], beta1=beta1, beta2=beta2, k=k)
        h = all_draws[b, :m2.size]
        s2[b, 0], codes = pack(np.abs(m2), TOP_M, E4M3, h)
        m2c[at] = codes | np.where(np.signbit(m2), 0x80, 0).astype(np.uint8)
        s2[b, 1], codes = pack(v2, TOP_V, E5M2, swapped(h))
        above = (v2 >= f32(2.0 ** -128)) & (v2.max() >= LEAST)
        v2c[at] = np.where((codes == 0) & above, 1, codes)
    p2, _, _, slack = step64(p, g, wide_m, wide_v, beta1=beta1, beta2=beta2, step=step, k=k, **rest)
    return p2, slack, m2c, v2c, s2
