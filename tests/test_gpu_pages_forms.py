"""Pages on the device: calls that test_gpu_pages.py leaves out, against the same reference
and with the same bounds."""
import numpy as np
import pytest
import torch

from paper_2601_14724_amd import hermes as H
from oracle import pages_oracle as orc
from test_gpu_pages import DEV, Setup, bits, dev, f64, fmt_of, i32

pytestmark = pytest.mark.gpu


def cut(s):
    """Whether the host plans s's attention with cuts (which need a workspace)."""
    return H.lib.hermes_page_workspace_bytes(s.pool._ref, s.batch._ref) > 0


@pytest.mark.parametrize("heads,fmt", [((8, 2, 64), "fp4"), ((8, 2, 128), "bf16")])
def test_starts_that_fall_give_a_row_to_one_sequence(heads, fmt):
    """With cuts, a start that falls counts as the greatest before it."""
    rng = np.random.default_rng(30)
    start = np.concatenate([[0], np.cumsum(rng.integers(0, 4, 150))]).astype(np.int32)
    for b in (3, 20, 64, 65, 100, 128, 149):
        start[b] = max(0, start[b] - int(rng.integers(1, 9)))
    start[70] = -5
    kept = np.maximum.accumulate(np.maximum(start, 0))
    rows, lens = np.diff(kept).tolist(), [int(x) for x in rng.integers(20, 400, 150)]
    s = Setup(heads, fmt, 16, rows, lens, seed=31, spare=9)
    batch = H.PageBatch(i32(s.tables), i32(lens), i32(start), n_rows=s.n)
    lse = torch.empty((s.n, s.hq), device=DEV)
    s.check_attend(s.pool.attend(batch, dev(s.q), lse=lse), lse)
    assert s.pool.faults() == H.PAGE_BAD_ROWS


def test_rows_are_stored_where_there_are_too_many_to_attend():
    """2^14 + 1 rows of one KV head with 2^16 query heads: stored and read back, refused by attend."""
    n, page = (1 << 14) + 1, 256
    pool = H.KVPages(1 << 16, 1, 64, 65, page_rows=page, fmt=H.PAGE_BF16)
    batch = H.PageBatch(i32(np.arange(65)[None]), i32([n]), i32([0, n]), n_rows=n)
    rng = np.random.default_rng(32)
    k, v = (orc.bf16_bits(rng.standard_normal((n, 1, 64))) for _ in "kv")
    pool.append(batch, dev(k), dev(v))
    kb, vb = pool.read(batch)
    assert (bits(kb) == k).all() and (bits(vb) == v).all()
    none = torch.empty(1, dtype=torch.bfloat16, device=DEV)     # (never read)
    with pytest.raises(H.HermesError) as e:
        pool._run(H.lib.hermes_page_attend, "hermes_page_attend", pool._ref, batch._ref, none.data_ptr(), 1 << 22,
                  none.data_ptr(), None, None, 0)
    assert e.value.code == H.EINVAL


# ------------------------------------------------------------- kinds of launches
@pytest.mark.parametrize("rows", [1, 4])                 # up to 16 and up to 32 packed rows
@pytest.mark.parametrize("heads", [(14, 2, 64), (14, 2, 128)], ids=lambda h: "x".join(map(str, h)))
@pytest.mark.parametrize("fmt,page", [("fp4", 64), ("fp4", 16), ("bf16", 32)])
def test_attend_many_short_items(fmt, page, heads, rows):
    """512 (sequence, KV head) pairs and more without cuts: workgroups of four waves."""
    rng = np.random.default_rng(33)
    lens = [int(x) for x in rng.integers(0, 200, 262)]
    lens[5], lens[6], lens[261] = 0, 1, 500
    counts = [1] * 262 if rows == 1 else [int(x) for x in rng.integers(0, rows + 1, 262)]
    s = Setup(heads, fmt, page, counts, lens, seed=34).hints(rows, 500)
    assert not cut(s)
    lse = torch.empty((s.n, s.hq), device=DEV)
    s.check_attend(s.pool.attend(s.batch, dev(s.q), lse=lse), lse)
    assert s.pool.faults() == 0


@pytest.mark.parametrize("max_rows", [1, 8])
@pytest.mark.parametrize("fmt", ["fp4", "bf16"])
def test_attend_few_rows_of_many_sequences_with_cuts(fmt, max_rows):
    """Cuts of 16- and 32-row items, over sequences past the first 64, some without rows or tokens."""
    rows, lens = [b * 7 % 4 for b in range(150)], [b * 37 % 400 for b in range(150)]
    lens[40], lens[149] = 3000, 2100
    s = Setup((8, 2, 64), fmt, 16, rows, lens, seed=35, spare=200).hints(max_rows, 5000)
    assert cut(s)
    lse = torch.empty((s.n, s.hq), device=DEV)
    s.check_attend(s.pool.attend(s.batch, dev(s.q), lse=lse), lse)


@pytest.mark.parametrize("heads", [(65, 65, 64), (140, 70, 128)], ids=lambda h: "x".join(map(str, h)))
@pytest.mark.parametrize("rows,max_rows", [([1, 1, 1], 1), ([20, 0, 3], 20), ([90, 1, 40], 0)])
def test_attend_more_kv_heads_than_lanes(heads, rows, max_rows):
    s = Setup(heads, "fp4", 32, rows, [500, 90, 900], seed=36, spare=300).hints(max_rows, 0)
    s.batch._batch.max_rows = max_rows
    assert cut(s)
    lse = torch.empty((s.n, s.hq), device=DEV)
    s.check_attend(s.pool.attend(s.batch, dev(s.q), lse=lse), lse)


# ----------------------------------------------------------------- pack, rotation
@pytest.mark.parametrize("fmt,page", [("fp4", 16), ("fp4", 64), ("bf16", 32)])
@pytest.mark.parametrize("hkv,d", [(4, 128), (3, 128), (1, 128), (9, 128), (2, 64), (9, 64)])
def test_pack_stores_every_byte(hkv, d, fmt, page):
    """All layers at once, of lengths that end inside a page and inside four rows, one empty."""
    lens = [130, 1, 0, 64, 259, 7]
    rng = np.random.default_rng(37)
    rnd = lambda n: orc.bf16_bits(rng.standard_normal((n, hkv, d)) * np.exp2(rng.integers(-9, 9, (n, hkv, d // 32))).repeat(32, 2))
    k, v = ([rnd(n) for n in lens] for _ in "kv")
    k[0][3, 0, :32], v[0][5, hkv - 1, 32:64] = 0, 0x0001           # a block of zeros, one of subnormals
    kv = H.HermesKV(len(lens), 2 * hkv, hkv, d, [max(n, 1) for n in lens], max_chunk=4,
                    init=[(dev(a), dev(b), i32(np.arange(len(a)))) for a, b in zip(k, v)])
    need = [-(-n // page) for n in lens]
    n_pages = sum(need) + 2
    ids = iter(rng.permutation(n_pages))
    tables = np.full((len(lens), max(need) + 1), -1, np.int32)
    for b, n in enumerate(need):
        tables[b, :n] = [next(ids) for _ in range(n)]
    want = np.full((n_pages, hkv * orc.block_bytes(d, page, fmt)), 0xFF, np.uint8)
    pool = H.KVPages(2 * hkv, hkv, d, n_pages, page_rows=page, fmt=fmt_of(fmt), pages=dev(want.copy()))
    kv_len = i32([-3] * len(lens))
    kv.pack(pool, i32(tables), kv_len)
    for b in range(len(lens)):
        orc.store(want, tables[b], k[b], v[b], page, fmt)
    assert kv_len.tolist() == lens
    assert (pool.pages.cpu().numpy() == want).all()
    assert pool.faults() == 0
    kv.close()


@pytest.mark.parametrize("d,theta,section", [(64, 1.0e4, (0, 0, 0)), (128, 5.0e5, (0, 0, 0)), (128, 1.0e6, (16, 24, 24)),
                                             (64, 1.0e4, (32, 0, 0)), (64, 1.0e6, (0, 1, 31))])
def test_append_sections_and_bases(d, theta, section):
    """Three axes with given sections, and other bases than 10^6 (also with one axis)."""
    for axes in (1, 3):
        s = Setup((6, 3, d), "bf16", 16, [20, 5], [30, 5], seed=38, fill=False, axes=axes, rope_theta=theta,
                  mrope_section=section if axes == 3 else (0, 0, 0))
        rng = np.random.default_rng(39)
        k, v = (orc.bf16_bits(rng.standard_normal((25, 3, d))) for _ in "kv")
        rope = rng.integers(0, 30_000, 25 if axes == 1 else (3, 25)).astype(np.int32)
        q = s.pool.append(s.batch, dev(k), dev(v), q=dev(s.q), rope=i32(rope))
        turn = lambda x: orc.rotate(orc.bf16_value(x), rope, theta, section)
        assert (bits(q) == turn(s.q)).all()
        kb, vb = s.pool.read(s.batch)
        assert (bits(kb) == turn(k)).all() and (bits(vb) == v).all()
