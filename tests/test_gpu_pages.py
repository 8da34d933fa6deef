"""Pages on the device against the fp64 reference (oracle/pages_oracle.py).

What is stored, and the rotated queries, are exact: rotation in fp64 leaves about
2^-44 of doubt before a rounding to 2^-9, and storing is exact arithmetic on what was
rounded.  Attention is bound row by row (see _bounds)."""
import numpy as np
import pytest
import torch

from oracle import pages_oracle as orc
from paper_2601_14724_amd import hermes as H

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def dev(x, dtype=None):
    if x.dtype == np.uint16:
        return torch.from_numpy(x.view(np.int16)).to(DEV).view(torch.bfloat16)
    return torch.from_numpy(np.ascontiguousarray(x)).to(DEV) if dtype is None else torch.tensor(x, dtype=dtype, device=DEV)


def bits(t):
    return t.contiguous().view(torch.int16).cpu().numpy().view(np.uint16)


def f64(t):
    return t.double().cpu().numpy()


def fmt_of(name):
    return H.PAGE_FP4 if name == "fp4" else H.PAGE_BF16


def i32(x):
    return torch.tensor(np.asarray(x), dtype=torch.int32, device=DEV)


class Setup:
    """Sequences of given lengths and rows in shuffled pages whose memory is 0xFF (NaN as
    bf16, as an FP4 scale) wherever nothing is stored, and their tables (-1 past the end)."""

    def __init__(self, heads, fmt, page, rows, lens, seed=0, fill=True, spare=0, scale=1.0, axes=1, behind=0, **pool):
        self.hq, self.hkv, self.d = heads
        self.fmt, self.page, self.rows, self.lens = fmt, page, rows, lens
        rng = self.rng = np.random.default_rng(seed)
        need = [-(-t // page) for t in lens]
        self.n_pages = sum(need) + 2
        ids = rng.permutation(self.n_pages)
        self.tables = np.full((len(lens), max(max(need), 1) + spare), -1, np.int32)
        at = 0
        for b, n in enumerate(need):
            self.tables[b, :n] = ids[at:at + n]
            at += n
        self.pages = np.full((self.n_pages, self.hkv * orc.block_bytes(self.d, page, fmt)), 0xFF, np.uint8)
        self.k = [orc.bf16_bits(rng.standard_normal((t, self.hkv, self.d)) * scale) for t in lens]
        self.v = [orc.bf16_bits(rng.standard_normal((t, self.hkv, self.d))) for t in lens]
        if fill:
            for b in range(len(lens)):
                orc.store(self.pages, self.tables[b], self.k[b], self.v[b], page, fmt)
        self.start = np.concatenate([[0], np.cumsum(rows)]).astype(np.int32)
        self.n = int(self.start[-1]) + behind
        self.q = orc.bf16_bits(rng.standard_normal((self.n, self.hq, self.d)) * scale)
        self.pool = H.KVPages(*heads, self.n_pages, page_rows=page, fmt=fmt_of(fmt), pages=dev(self.pages), rope_axes=axes,
                              **pool)
        one = all(r == 1 for r in rows) and behind == 0
        self.batch = H.PageBatch(i32(self.tables), i32(lens), None if one else i32(self.start), n_rows=self.n)

    def hints(self, max_rows, max_len):
        self.batch._batch.max_rows, self.batch._batch.max_len = max_rows, max_len
        return self

    def check_attend(self, out, lse, only=None, scale=None):
        for b, (r, t) in enumerate(zip(self.rows, self.lens)):
            if r == 0 or (only is not None and b not in only):
                continue
            sl = slice(self.start[b], self.start[b + 1])
            k, v = orc.stored(self.k[b], self.fmt), orc.stored(self.v[b], self.fmt)
            _bounds(out[sl], None if lse is None else lse[sl], orc.bf16_value(self.q[sl]), k, v,
                    scale or self.d ** -0.5, f"sequence {b}")


def _bounds(out, lse, q, k, v, scale, what):
    """|O - O_ref| <= 2^-8 sum p|v| (P as bf16) + 2^-8 |O| (its own rounding) + e sum p|v|,
    |lse - ref| <= e, where e holds fp32: a score's error is at most d 2^-24 sum |q_c k_c|
    scale (a sum of d products in any order) and 2^-22 of its size (its scaling and the
    maximum's subtraction, log2 domain), twice for numerator and denominator; 2^-21 for an
    exp2; and T 2^-24 for a sum of T terms."""
    want, wlse, mag, dots = orc.attend(q, k, v, scale)
    T, d = k.shape[0], q.shape[-1]
    e = 2 * (d * 2.0 ** -24 + 2.0 ** -22) * dots + 2.0 ** -21 + T * 2.0 ** -24
    tol = (2.0 ** -8 + e[..., None]) * mag + 2.0 ** -8 * np.abs(want) + 2.0 ** -120
    err = np.abs(f64(out) - want)
    assert np.isfinite(f64(out)).all(), what
    assert (err <= tol).all(), f"{what}: O off by {(err / tol).max():.2f} of its bound"
    if lse is not None:
        got = f64(lse)
        empty = np.isneginf(wlse)
        assert (np.isneginf(got) == empty).all(), what
        gap = np.abs(np.where(empty, 0, got) - np.where(empty, 0, wlse))
        assert (gap <= e + 2.0 ** -23 * np.abs(np.where(empty, 0, wlse))).all(), f"{what}: lse off by {gap.max()}"


# ------------------------------------------------------------------ append, read
APPENDS = [
    ((14, 2, 64), "fp4", 16, [1, 1, 1], [1, 17, 40], 1),
    ((28, 4, 128), "fp4", 64, [5, 0, 33, 1], [5, 9, 100, 64], 1),
    ((8, 8, 128), "bf16", 32, [7, 64], [40, 64], 1),
    ((7, 1, 64), "bf16", 256, [3], [259], 1),
    ((3, 3, 64), "fp4", 128, [10, 2], [130, 2], 3),
    ((12, 6, 128), "fp4", 32, [9], [33], 3),
    ((2, 1, 128), "bf16", 16, [4, 6], [2, 5], 3),        # more rows than the length: the first are not stored
    ((4, 2, 64), "fp4", 16, [1 + 5 * (b % 3) for b in range(130)], [12 + b for b in range(130)], 1),
    ((9, 9, 128), "bf16", 32, [0, 700, 0, 420, 3], [0, 900, 5, 420, 64], 1),
]


@pytest.mark.parametrize("heads,fmt,page,rows,lens,axes", APPENDS)
@pytest.mark.parametrize("fused", [False, True])
def test_append_and_read(heads, fmt, page, rows, lens, axes, fused):
    s = Setup(heads, fmt, page, rows, lens, seed=7, fill=False, axes=axes, behind=3)
    hq, hkv, d = heads
    rng = np.random.default_rng(8)
    k, v = (orc.bf16_bits(rng.standard_normal((s.n, hkv, d)) * np.exp2(rng.integers(-9, 9, (s.n, hkv, 1)))) for _ in "kv")
    rope = rng.integers(0, 300_000, s.n if axes == 1 else (3, s.n)).astype(np.int32)
    q_, k_, v_ = dev(s.q), dev(k), dev(v)
    if fused:      # parts of one projection's output
        both = torch.cat([x.flatten(1) for x in (q_, k_, v_)], 1)
        q_, k_, v_ = (x.unflatten(1, (-1, d)) for x in both.split([hq * d, hkv * d, hkv * d], 1))
        assert not q_.is_contiguous() or s.n == 1
    q_out = torch.full((s.n, hq, d), 7.0, dtype=torch.bfloat16, device=DEV)
    s.pool.append(s.batch, k_, v_, q=q_, rope=i32(rope), q_out=q_out)
    m = s.start[-1]
    turned = orc.rotate(orc.bf16_value(s.q), rope)
    assert (bits(q_out)[:m] == turned[:m]).all()
    assert (q_out[m:] == 7.0).all()                        # rows of no sequence
    kr = orc.rotate(orc.bf16_value(k), rope)
    want_k, want_v = np.zeros((s.n, hkv, d)), np.zeros((s.n, hkv, d))
    for b, (r, t) in enumerate(zip(rows, lens)):
        skip = max(0, r - t)
        sl = slice(s.start[b] + skip, s.start[b + 1])
        orc.store(s.pages, s.tables[b], kr[sl], v[sl], page, fmt, first=t - r + skip)
        want_k[sl], want_v[sl] = orc.stored(kr[sl], fmt), orc.stored(v[sl], fmt)
    assert (s.pool.pages.cpu().numpy() == s.pages).all()   # every byte, those nothing was stored in too
    kb, vb = (torch.full((s.n, hkv, d), 7.0, dtype=torch.bfloat16, device=DEV) for _ in "kv")
    s.pool.read(s.batch, kb, vb)
    assert (f64(kb)[:m] == want_k[:m]).all() and (f64(vb)[:m] == want_v[:m]).all()
    assert (kb[m:] == 7.0).all() and (vb[m:] == 7.0).all()
    assert s.pool.faults() == 0


def test_append_without_rotation_in_place_and_far_positions():
    s = Setup((4, 2, 64), "bf16", 16, [6], [6], fill=False)
    k, v = s.k[0], s.v[0]
    s.pool.append(s.batch, dev(k), dev(v))
    kb, vb = s.pool.read(s.batch)
    assert (bits(kb) == k).all() and (bits(vb) == v).all()
    rope = np.array([0, -5, 2 ** 31 - 1, 2 ** 20, 1, 10 ** 9], np.int32)
    q = dev(s.q)
    assert s.pool.append(s.batch, dev(k), dev(v), q=q, rope=i32(rope), q_out=q).data_ptr() == q.data_ptr()
    # 2^31 positions: an angle's own rounding (2^-23) may turn a bf16 value by one step
    near = rope < 2 ** 29
    assert (bits(q)[near] == orc.rotate(orc.bf16_value(s.q), rope)[near]).all()
    gap = np.abs(f64(q) - orc.bf16_value(orc.rotate(orc.bf16_value(s.q), rope)))
    assert (gap <= 2.0 ** -7 * np.abs(f64(q)) + 2.0 ** -20).all()


def test_fp4_of_special_values():
    hkv, d = 1, 64
    rows = np.zeros((9, hkv, d))
    rows[1, 0, 0], rows[2, 0, 40] = 2.0 ** 127 * 1.99, -2.0 ** -126
    rows[3, 0] = np.linspace(-7, 7, 64)
    rows[4, 0, :8] = [6, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5]
    rows[5, 0, 5] = 2.0 ** -119
    rows[6, 0, 33], rows[7, 0, 1] = np.inf, np.nan          # their block of 32 alone
    rows[6, 0, :32] = rows[7, 0, 32:] = 1.5
    rows[8] = 2.0 ** -133                                  # subnormal
    x = orc.bf16_bits(rows)
    pool = H.KVPages(1, 1, d, 1, page_rows=16, fmt=H.PAGE_FP4)
    batch = H.PageBatch(i32([[0]]), i32([9]), i32([0, 9]), n_rows=9)
    pool.append(batch, dev(x), dev(x[::-1].copy()))
    k, v = (f64(t) for t in pool.read(batch))
    want = orc.stored(x, "fp4")
    assert np.isnan(want[6, 0, 32:]).all() and np.isnan(want[7, 0, :32]).all() and np.isnan(want).sum() == 64
    assert np.array_equal(k, want, equal_nan=True) and np.array_equal(v, want[::-1], equal_nan=True)


# ----------------------------------------------------------------------- attend
HEADS = [(14, 2, 64), (28, 4, 128), (4, 4, 128), (2, 1, 64), (64, 1, 128), (33, 3, 64)]
SHAPES = [
    ([1], [1]),
    ([1, 1, 1, 1], [513, 0, 31, 2000]),
    ([3, 0, 17, 5, 40], [3, 12, 700, 2, 41]),              # none, all of it, more than the length
    ([130, 1], [130, 333]),
    ([300], [1111]),
    ([9, 4], [999, 70]),
    ([18, 1, 16], [2100, 129, 16]),
]


@pytest.mark.parametrize("heads", HEADS, ids=lambda h: "x".join(map(str, h)))
@pytest.mark.parametrize("fmt,page", [("fp4", 16), ("fp4", 64), ("bf16", 32), ("bf16", 256)])
@pytest.mark.parametrize("rows,lens", SHAPES, ids=lambda x: "-".join(map(str, x)))
def test_attend(heads, fmt, page, rows, lens):
    s = Setup(heads, fmt, page, rows, lens, seed=3, spare=3)
    lse = torch.full((s.n, s.hq), 5.0, device=DEV)
    for max_rows, max_len in ((max(rows), max(lens)), (0, 0)):
        s.hints(max_rows, max_len)
        out = s.pool.attend(s.batch, dev(s.q), lse=lse)
        s.check_attend(out, lse)
    assert s.pool.faults() == 0


@pytest.mark.parametrize("max_rows,max_len", [(1, 1), (1, 10 ** 6), (2, 129), (400, 64), (16, 1000)])
@pytest.mark.parametrize("d", [64, 128])
def test_attend_does_not_depend_on_the_hints(max_rows, max_len, d):
    """Hints below and above the truth choose other cuts, not other results."""
    s = Setup((6, 2, d), "fp4", 32, [70, 1, 9], [900, 1700, 5], seed=5).hints(max_rows, max_len)
    lse = torch.empty((s.n, s.hq), device=DEV)
    s.check_attend(s.pool.attend(s.batch, dev(s.q), lse=lse), lse)


@pytest.mark.parametrize("fmt", ["fp4", "bf16"])
def test_attend_sharp_scores(fmt):
    """Scores of some hundreds: the running maximum moves, and most of P underflows."""
    s = Setup((8, 2, 128), fmt, 64, [1, 50], [3000, 1500], seed=9, scale=6.0)
    lse = torch.empty((s.n, s.hq), device=DEV)
    s.check_attend(s.pool.attend(s.batch, dev(s.q), lse=lse), lse)


@pytest.mark.parametrize("max_rows", [1, 3, 40])
def test_attend_many_sequences(max_rows):
    """More sequences than lanes, some without rows, some without tokens."""
    rows, lens = [b * 7 % 4 for b in range(150)], [b * 37 % 400 for b in range(150)]
    s = Setup((8, 2, 64), "fp4", 16, rows, lens, seed=10).hints(max_rows, 5000)
    lse = torch.empty((s.n, s.hq), device=DEV)
    s.check_attend(s.pool.attend(s.batch, dev(s.q), lse=lse), lse)


def test_attend_scale_strides_and_rows_behind():
    s = Setup((6, 3, 64), "fp4", 16, [2, 3], [50, 77], behind=4, sm_scale=0.31)
    wide = torch.zeros((s.n, 6 * 64 + 40), dtype=torch.bfloat16, device=DEV)
    q = wide[:, 8:8 + 6 * 64].unflatten(1, (6, 64))
    q.copy_(dev(s.q))
    out = torch.full((s.n, 6, 64), 3.0, dtype=torch.bfloat16, device=DEV)
    lse = torch.full((s.n, 6), 3.0, device=DEV)
    for hints in ((3, 77), (0, 0)):
        s.hints(*hints)
        out[:5], lse[:5] = 0, 0
        s.pool.attend(s.batch, q, out=out, lse=lse)
        s.check_attend(out, lse, scale=0.31)
        assert (out[5:] == 3.0).all() and (lse[5:] == 3.0).all()


@pytest.mark.parametrize("d,fmt", [(64, "fp4"), (128, "bf16")])
def test_rows_before_the_first_start(d, fmt):
    """row_start[0] > 0: the rows before it are no sequence's, and stay as they are."""
    s = Setup((4, 2, d), fmt, 16, [3, 2], [40, 7], behind=7)
    start = s.start + 4
    batch = H.PageBatch(i32(s.tables), i32([40, 7]), i32(start), n_rows=s.n)
    out = torch.full((s.n, 4, d), 3.0, dtype=torch.bfloat16, device=DEV)
    kb, vb = (torch.full((s.n, 2, d), 3.0, dtype=torch.bfloat16, device=DEV) for _ in "kv")
    s.pool.attend(batch, dev(s.q), out=out)
    s.pool.read(batch, kb, vb)
    for x in (out, kb, vb):
        assert (x[:4] == 3.0).all() and (x[9:] == 3.0).all()
    s.q = s.q[4:]
    s.check_attend(out[4:], None)
    for b, (r, t) in enumerate(zip(s.rows, s.lens)):
        assert (f64(kb)[start[b]:start[b + 1]] == orc.stored(s.k[b], fmt)[t - r:]).all()
    assert s.pool.faults() == 0


def test_attend_long_split():
    """One token over a long sequence: many ranges, joined."""
    s = Setup((14, 2, 64), "fp4", 64, [1, 1], [20011, 1], seed=11).hints(1, 20011)
    lse = torch.empty((2, 14), device=DEV)
    first = s.pool.attend(s.batch, dev(s.q), lse=lse)
    s.check_attend(first, lse)
    for _ in range(3):                                     # the same bits every time
        assert torch.equal(s.pool.attend(s.batch, dev(s.q)), first)


def test_sequences_share_pages():
    s = Setup((4, 2, 64), "fp4", 32, [1, 1], [100, 100], seed=12)
    s.k[1], s.v[1] = s.k[0], s.v[0]
    tables = np.repeat(s.tables[:1], 2, 0)
    batch = H.PageBatch(i32(tables), i32([100, 100]))
    s.check_attend(s.pool.attend(batch, dev(s.q)), None)


def test_pool_beyond_4_gib():
    page, heads = 256, (2, 1, 128)
    size = orc.block_bytes(128, page, "bf16")
    n_pages = (5 << 30) // size
    pool = H.KVPages(*heads, n_pages, page_rows=page, fmt=H.PAGE_BF16)
    table = np.array([[n_pages - 1, 3, n_pages - 2]], np.int32)
    rng = np.random.default_rng(13)
    k, v = (orc.bf16_bits(rng.standard_normal((700, 1, 128))) for _ in "kv")
    batch = H.PageBatch(i32(table), i32([700]), i32([0, 700]), n_rows=700)
    pool.append(batch, dev(k), dev(v))
    kb, vb = pool.read(batch)
    assert (bits(kb) == k).all() and (bits(vb) == v).all()
    q = orc.bf16_bits(rng.standard_normal((1, 2, 128)))
    out = pool.attend(H.PageBatch(i32(table), i32([700])), dev(q))
    _bounds(out, None, orc.bf16_value(q), orc.bf16_value(k), orc.bf16_value(v), 128 ** -0.5, "high pages")


# ------------------------------------------------------- what the device refuses
def test_bad_ids_lengths_and_starts_are_noted():
    s = Setup((4, 2, 64), "fp4", 16, [2, 2, 2], [40, 40, 40], seed=14)
    before = s.pool.pages.clone()
    tables = s.tables.copy()
    tables[0, 2], tables[1, 0] = s.n_pages, -7            # of sequence 0 the last page, of 1 the first
    k = dev(orc.bf16_bits(np.ones((6, 2, 64))))
    batch = H.PageBatch(i32(tables), i32([40, 40, 40]), i32(s.start), n_rows=6)
    s.pool.append(batch, k, k)
    assert s.pool.faults() == H.PAGE_BAD_ID and s.pool.faults() == 0
    changed = (s.pool.pages != before).any(1).cpu().numpy()
    assert set(np.flatnonzero(changed)) == {tables[1, 2], tables[2, 2]}
    s.pool.pages.copy_(before)
    lse = torch.empty((6, 4), device=DEV)
    out = s.pool.attend(batch, dev(s.q), lse=lse)
    assert s.pool.faults() == H.PAGE_BAD_ID
    s.k[0][32:], s.v[0][32:], s.k[1][:16], s.v[1][:16] = 0, 0, 0, 0      # read as zeros
    s.check_attend(out, lse)
    kb, _ = s.pool.read(batch)
    assert (kb[:2] == 0).all() and s.pool.faults() == H.PAGE_BAD_ID

    for lens in ([-1, 40, 40], [16 * s.tables.shape[1] + 1, 40, 40]):
        batch = H.PageBatch(i32(s.tables), i32(lens), i32(s.start), n_rows=6)
        out = s.pool.attend(batch, dev(s.q), lse=lse)
        assert s.pool.faults() == H.PAGE_BAD_LENGTH
        assert (out[:2] == 0).all() and torch.isneginf(lse[:2]).all()
        s.pool.append(batch, k, k)
        assert s.pool.faults() == H.PAGE_BAD_LENGTH
        s.pool.pages.copy_(before)
    for start in ([0, 2, 1, 6], [0, 2, 4, 900], [-3, 2, 4, 6]):
        batch = H.PageBatch(i32(s.tables), i32([40, 40, 40]), i32(start), n_rows=6)
        s.pool.attend(batch, dev(s.q))
        assert s.pool.faults() == H.PAGE_BAD_ROWS
        s.pool.append(batch, k, k)
        s.pool.read(batch)
        s.pool.faults()
    torch.cuda.synchronize()


def test_the_binding_refuses():
    s = Setup((4, 2, 64), "fp4", 16, [2], [20])
    q, k = dev(s.q), dev(s.k[0][:2])
    for call in (lambda: s.pool.attend(s.batch, q[:1]), lambda: s.pool.attend(s.batch, q.float()),
                 lambda: s.pool.attend(s.batch, q.cpu()), lambda: s.pool.append(s.batch, k, k.transpose(1, 2)),
                 lambda: s.pool.append(s.batch, k, k, q=q, rope=i32([1])), lambda: s.pool.read(s.batch, k=q),
                 lambda: s.pool.attend(s.batch, q, lse=torch.empty(2, 4)),
                 lambda: H.PageBatch(i32(s.tables), i32([1, 2])), lambda: H.PageBatch(i32(s.tables), i32([1]), i32([0, 1])),
                 lambda: H.KVPages(4, 2, 64, 3, pages=s.pool.pages)):
        with pytest.raises(ValueError):
            call()
    with pytest.raises(H.HermesError):
        s.pool.append(s.batch, k, k, q=q)                  # queries without positions
    with pytest.raises(H.HermesError):
        H.KVPages(4, 2, 64, 3, page_rows=24)
    empty = H.PageBatch(i32(np.zeros((0, 1))), i32(np.zeros(0)))
    assert s.pool.attend(empty, q[:0]).shape == (0, 4, 64)


# ------------------------------------------------- streams, graphs, used together
def test_two_streams_at_once():
    a = Setup((14, 2, 64), "fp4", 64, [1], [9000], seed=20).hints(1, 9000)
    b = Setup((28, 4, 128), "bf16", 32, [20], [2500], seed=21).hints(20, 2500)
    want = [s.pool.attend(s.batch, dev(s.q)) for s in (a, b)]
    qs, streams = [dev(s.q) for s in (a, b)], [torch.cuda.Stream() for _ in "ab"]
    torch.cuda.synchronize()
    got = [[], []]
    for _ in range(5):
        for i, s in enumerate((a, b)):
            with torch.cuda.stream(streams[i]):
                got[i].append(s.pool.attend(s.batch, qs[i]))
    torch.cuda.synchronize()
    for i in range(2):
        assert all(torch.equal(x, want[i]) for x in got[i])


@pytest.mark.parametrize("fmt,first", [("fp4", [30, 500, 1]), ("bf16", [30, 500, 1]), ("fp4", [9000, 4000, 1])])
def test_captured_decoding(fmt, first):
    """A captured token (append, then attend) replayed while lengths, positions and inputs
    move on, against the same calls made eagerly; short sequences without cuts, and long ones
    with."""
    steps = 5
    s = Setup((14, 2, 64), fmt, 16, [1] * 3, [t + steps for t in first], seed=22, fill=False)
    for b, t in enumerate(first):
        orc.store(s.pages, s.tables[b], s.k[b][:t], s.v[b][:t], 16, fmt)
    s.pool.pages.copy_(dev(s.pages))
    eager = H.KVPages(14, 2, 64, s.n_pages, page_rows=16, fmt=fmt_of(fmt), pages=dev(s.pages))
    rng = np.random.default_rng(23)
    ins = [[dev(orc.bf16_bits(rng.standard_normal((3, h, 64)))) for h in (14, 2, 2)] for _ in range(steps)]
    q, k, v = (x.clone() for x in ins[0])
    kv_len, rope, out = i32(first), i32(first), torch.empty_like(q)
    batch = H.PageBatch(i32(s.tables), kv_len, max_len=max(first) + steps)
    kv_len += 1

    def token(pool, batch):
        pool.attend(batch, pool.append(batch, k, v, q=q, rope=rope), out=out)

    graph = torch.cuda.CUDAGraph()
    before = s.pool.pages.clone()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        token(s.pool, batch)
    torch.cuda.current_stream().wait_stream(side)
    with torch.cuda.graph(graph):
        token(s.pool, batch)
    s.pool.pages.copy_(before)
    for i in range(steps):
        for x, y in zip((q, k, v), ins[i]):
            x.copy_(y)
        graph.replay()
        got = out.clone()
        token(eager, batch)
        assert torch.equal(got, out), f"step {i}"
        assert torch.equal(s.pool.pages, eager.pages)
        kv_len += 1
        rope += 1
        torch.cuda.synchronize()


@pytest.mark.parametrize("fmt,axes", [("fp4", 1), ("bf16", 1), ("fp4", 3)])
def test_stream_then_answer(fmt, axes):
    """The path as it is used: chunks enter a context and are cut back, the compact caches
    of all layers (of different lengths) are packed, a question is rotated and appended
    to every layer's pages and attends, then tokens one by one, against the reference
    over the context's own caches."""
    L, hq, hkv, d, page, budgets = 3, 6, 2, 64, 16, [40, 55, 90]
    rng = np.random.default_rng(24)
    rnd = lambda *shape: orc.bf16_bits(rng.standard_normal(shape))
    kv = H.HermesKV(L, hq, hkv, d, budgets, max_chunk=48, rope_axes=axes)
    at = 0
    for n in (48, 31, 17):
        pos = np.arange(at, at + n, dtype=np.int32)
        thw = i32(np.stack([pos, pos % 7, pos % 5])) if axes == 3 else None
        kv.append(dev(rnd(L, n, hq, d)), dev(rnd(L, n, hkv, d)), dev(rnd(L, n, hkv, d)), i32(pos), rope_thw=thw)
        if at == 0:
            pool = H.KVPages(hq, hkv, d, 40, page_rows=page, fmt=fmt_of(fmt), rope_axes=axes)
            tables, kv_len = i32(rng.permutation(40)[:30].reshape(L, 10)), i32([0] * L)
            with pytest.raises(H.HermesError) as e:         # between append and compress
                kv.pack(pool, tables, kv_len)
            assert e.value.code == H.ESTATE
        kv.compress()
        at += n
    kv.pack(pool, tables, kv_len)
    lens = kv_len.cpu().tolist()
    assert lens == [kv.length(l) for l in range(L)] == budgets
    k, v = ([bits(kv.view(l)[i]) for l in range(L)] for i in range(2))
    start = np.concatenate([[0], np.cumsum(lens)])
    kb, vb = pool.read(H.PageBatch(tables, kv_len, i32(start), n_rows=int(start[-1])))
    for l in range(L):
        assert (f64(kb)[start[l]:start[l + 1]] == orc.stored(k[l], fmt)).all()
        assert (f64(vb)[start[l]:start[l + 1]] == orc.stored(v[l], fmt)).all()

    kv.profile(True)
    kv.pack(pool, tables[1], kv_len[1:2], layer=1)         # one layer again
    assert kv.profile_read(H.K_PACK)[1] == 1
    with pytest.raises(H.HermesError) as e:
        kv.pack(pool, tables[:, :2].contiguous(), kv_len)
    assert e.value.code == H.ECAPACITY
    with pytest.raises(H.HermesError):
        kv.pack(H.KVPages(hq, 1, d, 4), tables, kv_len)
    for n in (13, 1, 1, 1):
        kv_len += n
        pos = np.tile(np.arange(at, at + n, dtype=np.int32), L)
        rope = np.stack([pos, pos, pos]) if axes == 3 else pos
        q, kn, vn = rnd(L * n, hq, d), rnd(L * n, hkv, d), rnd(L * n, hkv, d)
        rows = None if n == 1 else i32(np.arange(L + 1) * n)
        batch = H.PageBatch(tables, kv_len, rows, n_rows=L * n, max_rows=n)
        lse = torch.empty((L * n, hq), device=DEV)
        turned = pool.append(batch, dev(kn), dev(vn), q=dev(q), rope=i32(rope))
        out = pool.attend(batch, turned, lse=lse)
        qr, kr = orc.rotate(orc.bf16_value(q), rope), orc.rotate(orc.bf16_value(kn), rope)
        for l in range(L):
            sl = slice(l * n, (l + 1) * n)
            k[l], v[l] = np.concatenate([k[l], kr[sl]]), np.concatenate([v[l], vn[sl]])
            _bounds(out[sl], lse[sl], orc.bf16_value(qr[sl]), orc.stored(k[l], fmt), orc.stored(v[l], fmt), d ** -0.5,
                    f"layer {l}")
        at += n
    assert pool.faults() == 0
    kv.close()


def test_pack_an_empty_cache():
    kv = H.HermesKV(2, 4, 2, 64, [20, 20], max_chunk=8)
    pool = H.KVPages(4, 2, 64, 2, page_rows=16)
    kv_len = i32([9, 9])
    kv.pack(pool, i32([[0], [1]]), kv_len)
    assert kv_len.tolist() == [0, 0]
    out = pool.attend(H.PageBatch(i32([[0], [1]]), kv_len), torch.ones((2, 4, 64), dtype=torch.bfloat16, device=DEV))
    assert (out == 0).all()
    kv.close()
