"""Pages on the device: calls that test_gpu_pages.py leaves out, against the same reference
and with the same bounds."""
import numpy as np
import pytest
import torch

from paper_2601_14724_amd import hermes as H
from oracle import pages_oracle as orc
from test_gpu_pages import DEV, Setup, bits, dev, i32

pytestmark = pytest.mark.gpu


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
