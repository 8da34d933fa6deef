"""fp64 reference of the paged operators: rotation, FP4 storage, page layout,
attention.  NumPy only; test infrastructure, written from the definitions in
include/hermes.h."""
import numpy as np

LEVELS = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def bf16_bits(x):
    """fp64 -> fp32 -> bf16, to nearest even, as uint16 patterns."""
    u = np.asarray(x, np.float64).astype(np.float32).view(np.uint32).astype(np.uint64)
    return ((u + 0x7FFF + ((u >> 16) & 1)) >> 16).astype(np.uint16)


def bf16_value(bits):
    return (np.asarray(bits, np.uint16).astype(np.uint32) << 16).view(np.float32).astype(np.float64)


def sections(d, axes, section=(0, 0, 0)):
    """Axis of every frequency pair."""
    if axes != 3:
        return np.zeros(d // 2, int)
    if not any(section):
        t = d // 8
        h = (d // 2 - t) // 2
        section = (t, h, d // 2 - t - h)
    return np.repeat(np.arange(3), section)


def rotate(x, rope, theta=1.0e6, section=(0, 0, 0)):
    """x [n][heads][d] (fp64) at positions rope [n] or [3][n]; bf16 patterns."""
    d = x.shape[-1]
    rope = np.atleast_2d(np.asarray(rope, np.int64))
    axis = sections(d, rope.shape[0], section)
    angle = rope[axis].T * theta ** (-2.0 * np.arange(d // 2) / d)
    c, s = np.cos(angle)[:, None], np.sin(angle)[:, None]
    a, b = x[..., : d // 2], x[..., d // 2:]
    return bf16_bits(np.concatenate([a * c - b * s, b * c + a * s], -1))


def fp4(bits):
    """(codes, scale bytes) of bf16 patterns [.., d]."""
    x = bf16_value(bits)
    b = x.reshape(x.shape[:-1] + (x.shape[-1] // 32, 32))
    amax = np.abs(b).max(-1)
    finite = np.isfinite(amax)
    e = np.full(amax.shape, -119)
    for k in range(-119, 125):            # the least e with amax <= 7 * 2^e, at most 125
        e = np.where(finite & (amax > 7.0 * 2.0 ** k), k + 1, e)
    with np.errstate(invalid="ignore"):
        y = b / (2.0 ** e)[..., None]
        gap = np.abs(np.abs(y)[..., None] - LEVELS)
        order = np.array([0, 2, 4, 6, 1, 3, 5, 7])            # of equal gaps the even code
        code = order[np.argmin(np.where(np.isnan(gap), np.inf, gap)[..., order], -1)]
    code = (code + 8 * np.signbit(b)).astype(np.uint8)
    return code.reshape(x.shape), np.where(finite, e + 127, 255).astype(np.uint8)


def fp4_value(code, scale):
    v = np.where(code >= 8, -LEVELS[code & 7], LEVELS[code & 7])
    s = np.where(scale == 255, np.nan, 2.0 ** (scale.astype(np.float64) - 127))
    return (v.reshape(v.shape[:-1] + (v.shape[-1] // 32, 32)) * s[..., None]).reshape(v.shape)


def stored(bits, fmt):
    """What bf16 patterns read back as (fp64)."""
    return bf16_value(bits) if fmt == "bf16" else fp4_value(*fp4(bits))


def block_bytes(d, page, fmt):
    return 2 * page * (2 * d if fmt == "bf16" else d // 2 + d // 32)


def store(pages, table, k, v, page, fmt, first=0):
    """Stores k, v (patterns [n][hkv][d]) as tokens first .. first + n - 1 of the sequence
    whose page ids are `table`, in pages uint8 [n_pages][hkv * block_bytes]."""
    n, hkv, d = k.shape
    if n == 0:
        return
    size, s = block_bytes(d, page, fmt), d // 16
    t = first + np.arange(n)
    pid, r = np.asarray(table)[t // page][:, None, None], (t % page)[:, None]
    head, chan, blk = np.arange(hkv)[None, :, None], np.arange(d)[None], np.arange(d // 32)[None]
    at_k = r * d + chan                                                      # elements of the block's K
    at_v = r // 4 * (4 * d) + chan // s * (4 * s) + r % 4 * s + chan % s      # and V
    if fmt == "bf16":
        words = pages.view(np.uint16).reshape(len(pages), hkv, size // 2)
        words[pid, head, at_k[:, None]] = k
        words[pid, head, page * d + at_v[:, None]] = v
        return
    blocks = pages.reshape(len(pages), hkv, size)
    half = page * d // 2
    for x, at, start in ((k, at_k, 0), (v, at_v, half)):
        code, _ = fp4(x)
        blocks[pid, head, start + (at[:, 0::2] // 2)[:, None]] = code[..., 0::2] | (code[..., 1::2] << 4)
    blocks[pid, head, 2 * half + (r * (d // 32) + blk)[:, None]] = fp4(k)[1]
    blocks[pid, head, 2 * half + page * (d // 32) + (r // 4 * (d // 8) + blk * 4 + r % 4)[:, None]] = fp4(v)[1]


def attend(q, k, v, scale):
    """Rows q [n][hq][d] as the last n tokens over k, v [T][hkv][d] (fp64).  Returns O, lse,
    and for error bounds sum p |v| and the largest sum |q_c k_c| * scale a row."""
    n, hq, d = q.shape
    T, hkv = k.shape[:2]
    out, lse = np.zeros((n, hq, d)), np.full((n, hq), -np.inf)
    mag, dots = np.zeros((n, hq, d)), np.zeros((n, hq))
    seen = np.arange(T)[None] <= np.arange(T - n, T)[:, None]
    some = seen.any(1)
    if not some.any():
        return out, lse, mag, dots
    seen = seen[some]
    for h in range(hq):
        kk, vv = k[:, h // (hq // hkv)], v[:, h // (hq // hkv)]
        x = np.where(seen, q[some, h] @ kk.T * scale, -np.inf)
        top = x.max(1, keepdims=True)
        p = np.exp(x - top)
        z = p.sum(1, keepdims=True)
        lse[some, h] = (top + np.log(z))[:, 0]
        out[some, h], mag[some, h] = p / z @ vv, p / z @ np.abs(vv)
        dots[some, h] = np.where(seen, np.abs(q[some, h]) @ np.abs(kk).T * scale, 0).max(1)
    return out, lse, mag, dots
