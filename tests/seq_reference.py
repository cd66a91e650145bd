"""Plain 64-bit forms of the behaviour-sequence operators and of AdamW, token by token, and the 8-bit states' rounding
in numpy's IEEE binary32 and integers."""
import numpy as np

EPS = {"f32": 2.0 ** -24, "f16": 2.0 ** -11, "bf16": 2.0 ** -8}     # half a unit in the last place, relative
TINY = {"f32": 2.0 ** -150, "f16": 2.0 ** -25, "bf16": 2.0 ** -134}  # ... of the subnormal numbers, absolute


def embed(table, ids, scale, padding_id=-1):
    table, ids = np.asarray(table, np.float64), np.asarray(ids)
    held = (ids >= 0) & (ids < len(table)) & ((ids != padding_id) | (padding_id < 0))
    out = np.zeros((len(ids), table.shape[1]))
    out[held] = table[ids[held]] * scale
    return out


def embed_grad(dout, ids, num_rows, scale, padding_id=-1):
    """The gradient and, for bounds, the sums of magnitudes and the rows' token counts."""
    dout, ids = np.asarray(dout, np.float64), np.asarray(ids)
    held = (ids >= 0) & (ids < num_rows) & ((ids != padding_id) | (padding_id < 0))
    grad, mag = np.zeros((num_rows, dout.shape[1])), np.zeros((num_rows, dout.shape[1]))
    np.add.at(grad, ids[held], dout[held])
    np.add.at(mag, ids[held], np.abs(dout[held]))
    return grad * scale, mag * abs(scale), np.bincount(ids[held], minlength=num_rows)[:num_rows]


def gates(gate):
    gate = np.asarray(gate, np.float64)
    e = np.exp(-np.abs(gate))
    a = np.where(gate >= 0, 1 / (1 + e), e / (1 + e))
    return a, np.where(gate >= 0, e / (1 + e), 1 / (1 + e))


def recur(x, gate, offsets, h0=None):
    """h, h_last and the states before each token; a token whose gate is +inf keeps the state whatever x is."""
    x = np.asarray(x, np.float64)
    a, keep = gates(gate)
    seqs, dim = len(offsets) - 1, x.shape[1]
    h, before, last = np.zeros_like(x), np.zeros_like(x), np.zeros((seqs, dim))
    for s in range(seqs):
        state = np.zeros(dim) if h0 is None else np.asarray(h0[s], np.float64)
        for t in range(offsets[s], offsets[s + 1]):
            before[t] = state
            state = a[t] * state + np.where(keep[t] > 0, keep[t] * np.where(keep[t] > 0, x[t], 0.0), 0.0)
            h[t] = state
        last[s] = state
    return h, last, before


def recur_grad(x, gate, offsets, dh, dlast, h0=None):
    x = np.asarray(x, np.float64)
    a, keep = gates(gate)
    _, _, before = recur(x, gate, offsets, h0)
    seqs, dim = len(offsets) - 1, x.shape[1]
    dx, dg, d0 = np.zeros_like(x), np.zeros_like(x), np.zeros((seqs, dim))
    for s in range(seqs):
        c = np.zeros(dim) if dlast is None else np.asarray(dlast[s], np.float64)
        for t in range(offsets[s + 1] - 1, offsets[s] - 1, -1):
            e = c + (0.0 if dh is None else np.asarray(dh[t], np.float64))
            dx[t] = keep[t] * e
            held = np.where(keep[t] > 0, x[t], 0.0)
            dg[t] = np.where(keep[t] > 0, a[t] * keep[t] * (before[t] - held) * e, 0.0)
            c = a[t] * e
        d0[s] = c
    return dx, dg, d0


def adamw(p, g, m, v, t, lr, b1, b2, eps, wd):
    """The new p, m and v, and the magnitude of the step without the cancellation in m."""
    p, g, m, v = (np.asarray(z, np.float64) for z in (p, g, m, v))
    v = b2 * v + (1 - b2) * g * g
    size = lr / (1 - b1 ** t) / (np.sqrt(v / (1 - b2 ** t)) + eps)
    reach = size * (b1 * np.abs(m) + (1 - b1) * np.abs(g))
    m = b1 * m + (1 - b1) * g
    return p * (1 - lr * wd) - size * m, m, v, reach


M32 = 0xFFFFFFFF


def mix(x):
    x = np.asarray(x, np.uint64) & np.uint64(M32)
    for shift, factor in ((16, 0x6A09E667), (15, 0xBB67AE85), (16, 1)):
        x = x ^ (x >> np.uint64(shift))
        x = (x * np.uint64(factor)) & np.uint64(M32)
    return x


def random_bits(count, seed, step, tensor):
    """(for m, for v): 20 random bits an element, the low 4 zero."""
    key = int(mix((seed + step * 0x9E3779B1 + tensor * 0xC2B2AE35) & M32))
    i = np.arange(count, dtype=np.uint64)
    r = mix(((i & np.uint64(M32)) * np.uint64(0x9E3779B1) + (i >> np.uint64(32)) + np.uint64(key)) & np.uint64(M32))
    return ((r & np.uint64(0xFFFF)) << np.uint64(4)).astype(np.int64), ((r >> np.uint64(16)) << np.uint64(4)).astype(np.int64)


def decode(codes):
    """e4m3 values: 4 bits of exponent (bias 7), 3 of mantissa, no infinities."""
    c = np.asarray(codes, np.int64)
    e, f = (c >> 3) & 15, c & 7
    mag = np.where(e > 0, (8 + f) * 2.0 ** (e - 10.0), f * 2.0 ** -9)
    return np.where(c & 128, -mag, mag)


def store8(x, rnd, keep_small):
    """float32 values of one tensor to codes and the blocks' scales, each operation in binary32."""
    n, f = len(x), np.float32
    y = np.zeros(-(-n // 256) * 256, f)
    y[:n] = x
    y = y.reshape(-1, 256)
    r = np.zeros(y.size, np.int64)
    r[:n] = rnd
    r = r.reshape(y.shape)
    top = np.abs(y).max(1)
    held = top > f(2.0 ** -100)
    with np.errstate(divide="ignore"):
        inv, scale = np.where(held, (f(1) / top) * f(448), f(0)), np.where(held, top * (f(1) / f(448)), f(0))
    z = np.minimum(np.abs(y) * inv[:, None], f(448))
    normal = ((z.view(np.int32).astype(np.int64) + r) >> 20) - (120 << 3)
    small = np.floor(z * f(512) + r.astype(f) * f(2.0 ** -20)).astype(np.int64)
    codes = np.where(z >= f(2.0 ** -6), normal, small)
    if keep_small:
        codes = np.where((z > 0) & (codes < 1), 1, codes)
    codes = codes | np.where(y < 0, 128, 0)
    return codes.reshape(-1)[:n].astype(np.uint8), scale
