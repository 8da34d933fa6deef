"""fp64 reference of what stands around a generated token: products with weights in 4
bits, the choice over beams and vocabulary, the reordering of pages.  NumPy only; test
infrastructure, written from the definitions in include/hermes.h."""
import numpy as np

from oracle import pages_oracle as pages


def _padded(x, rows, cols):
    out = np.zeros((rows, cols), x.dtype)
    out[:x.shape[0], :x.shape[1]] = x
    return out


def pack(bits):
    """Memory of a weight whose bf16 patterns are [n_out][n_in], as uint8."""
    n, k = bits.shape
    N, K = -(-n // 16), -(-k // 128)
    code, scale = pages.fp4(_padded(bits, 16 * N, 128 * K))
    byte = (code[:, 0::2] | (code[:, 1::2] << 4)).reshape(N, 16, K, 4, 4, 4)         # [.., n, .., block, lane / 16, byte]
    codes = byte.transpose(0, 2, 4, 1, 3, 5)
    scales = np.full((N, -(-K // 4), 16, 4, 4), 8, np.uint8)
    for kt in range(K):
        scales[:, kt // 4, :, kt % 4] = scale.reshape(N, 16, K, 4)[:, :, kt]
    return codes.reshape(-1), scales


def unused_scales(n, k):
    """Scale bytes that no tile has (those behind the last of its four)."""
    N, K = -(-n // 16), -(-k // 128)
    m = np.zeros((N, -(-K // 4), 16, 4, 4), bool)
    if K % 4:
        m[:, -1, :, K % 4:] = True
    return m


def weight(bits):
    """What a weight stands for, fp64 [n_out][n_in]."""
    n, k = bits.shape
    return pages.fp4_value(*pages.fp4(_padded(bits, n, -(-k // 32) * 32)))[:, :k]


def product(x, w, bias=None, add=None):
    """x [m][k] and w [n][k] fp64.  The result, and the sum of its terms' magnitudes."""
    out, mag = x @ w.T, np.abs(x) @ np.abs(w).T
    for extra in (bias, add):
        if extra is not None:
            out, mag = out + extra, mag + np.abs(extra)
    return out, mag


def values(logits, score, done=None, pad=0):
    """Value of every continuation [beams][vocab] (-infinity: none) of one sequence."""
    beams, vocab = logits.shape
    out = np.full((beams, vocab), -np.inf)
    for b in range(beams):
        if not np.isfinite(score[b]):
            continue
        if done is not None and done[b]:
            out[b, pad] = score[b]
            continue
        x = logits[b].astype(np.float64)
        if np.isnan(x).any() or (x == np.inf).any() or (x == -np.inf).all():
            continue
        top = x.max()
        with np.errstate(under="ignore"):
            out[b] = (np.float64(score[b]) - (top + np.log(np.exp(x - top).sum()))) + x
    return out


def select(value, keep):
    """The first `keep` (value, beam, token) of values [beams][vocab], best first."""
    flat = value.reshape(-1)
    order = np.argsort(-flat, kind="stable")
    order = order[flat[order] > -np.inf][:keep]
    return flat[order], order // value.shape[1], order % value.shape[1]


BAD_ID, BAD_LENGTH, BAD_PARENT, NO_ROOM = 1, 2, 8, 16


def reorder(tables, kv_len, parent, room, grow, page, n_pages):
    """One group: tables [beams][max_pages], kv_len [beams], parent [beams], room (first,
    pages).  The new tables and lengths, the copies (from, to, rows), and the status bits."""
    beams, most = tables.shape
    out, lens = np.full_like(tables, -1), np.zeros_like(kv_len)
    bits = 0
    first, size = int(room[0]), int(room[1])
    if first < 0 or size < 0 or size > 65536 or first + size > n_pages:
        first = size = 0
        bits |= BAD_ID
    par = []
    for j in range(beams):
        p = int(parent[j])
        if p < -1 or p >= beams:
            p = -1
            bits |= BAD_PARENT
        n = int(kv_len[p]) if p >= 0 else 0
        if n < 0 or n > most * page:
            n = 0
            bits |= BAD_LENGTH
        par.append(p)
        lens[j] = n
        out[j, :n // page] = tables[p, :n // page]
    own = set(range(first, first + size))
    held = {int(x) for j in range(beams) for x in out[j, :lens[j] // page]}
    last = [int(tables[par[j], lens[j] // page]) if lens[j] % page else None for j in range(beams)]
    kept = [last[j] in own and last[j] not in held and last[j] not in last[:j] for j in range(beams)]
    free = sorted(own - held - {last[j] for j in range(beams) if kept[j]}, reverse=True)
    copies = []
    for j in range(beams):
        if par[j] < 0:
            continue
        n = int(lens[j])
        want = -(-(n + grow) // page)
        if want > most:
            bits |= NO_ROOM
        for e in range(n // page, min(want, most)):
            if e == n // page and kept[j]:
                out[j, e] = last[j]
            elif free:
                out[j, e] = free.pop()
                if e == n // page and n % page:
                    if 0 <= last[j] < n_pages:
                        copies.append((last[j], int(out[j, e]), -(-(n % page) // 4) * 4))
                    else:
                        bits |= BAD_ID
            else:
                bits |= NO_ROOM
    return out, lens, copies, bits


def copy_rows(memory, heads, d, page, fmt, source, target, rows):
    """Copies the first `rows` rows (a multiple of four) of a page to another."""
    size = pages.block_bytes(d, page, fmt)
    parts = [2 * d, 2 * d] if fmt == "bf16" else [d // 2, d // 2, d // 32, d // 32]
    a, b = memory[source].reshape(heads, size).copy(), memory[target].reshape(heads, size)
    at = 0
    for row in parts:
        b[:, at:at + rows * row] = a[:, at:at + rows * row]
        at += page * row
