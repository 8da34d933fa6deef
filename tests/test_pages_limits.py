"""Sizes that the pages' calls take or refuse, and the cut of an attention call, worked out
on the host (no device)."""
import ctypes

import pytest

from paper_2601_14724_amd import hermes as H
from test_pages_host import _attend, _batch, _pool, _read


def _bytes(pool, batch):
    return H.lib.hermes_page_workspace_bytes(ctypes.byref(pool), ctypes.byref(batch))


def test_limits_of_attention_are_attentions_alone():
    """2^25 rows of 28 + 4 heads are too many to attend in one call, not to be read (or
    appended).  (A read of neither K nor V is checked and does nothing.)"""
    pool = _pool(n_q_heads=28, n_kv_heads=4, head_dim=128)
    most = _batch(n_rows=1 << 25)
    assert _read(pool, most, None, None) == H.OK
    assert _attend(pool, most, qs=28 * 128) == H.EINVAL and _bytes(pool, most) == 0
    wide = _pool(n_q_heads=1 << 16, n_kv_heads=1)
    b = _batch(n_seqs=1, n_rows=1 << 14, max_pages=1)
    assert _read(wide, b, None, None) == H.OK and _attend(wide, b, qs=1 << 22) == H.EINVAL
    for over in (dict(n_rows=(1 << 25) + 1), dict(n_seqs=(1 << 22) + 1), dict(max_pages=1 << 26)):
        assert _read(pool, _batch(**over), None, None) == H.EINVAL


def test_the_cost_limit_is_the_headers():
    pool = _pool(n_q_heads=28, n_kv_heads=4, head_dim=128)
    for n_rows in range(1 << 20, 1 << 25, 1 << 20):
        for max_pages in (1, 1000, 1 << 20):
            b = _batch(n_seqs=5, n_rows=n_rows, max_pages=max_pages, max_rows=0, max_len=0)
            cost = (n_rows * 28 / 16 + 5 * 4) * 7 * (max_pages * 32 + 1024 + n_rows)
            assert (_bytes(pool, b) > 0) == (cost <= 4e15), (n_rows, max_pages)


def test_a_row_a_sequence_needs_no_hint():
    """Without row starts every sequence has one row, whatever max_rows says."""
    pool = _pool(n_q_heads=28, n_kv_heads=4, head_dim=128)
    for seqs in (1, 3, 28, 256):
        for pages in (1, 20, 300):
            got = {_bytes(pool, _batch(n_seqs=seqs, n_rows=seqs, row_start=None, max_rows=m, max_len=0, max_pages=pages))
                   for m in (0, 1, 2, seqs, 1000)}
            assert len(got) == 1, (seqs, pages, got)


@pytest.mark.parametrize("over,code", [(dict(head_dim=96), H.ENOTSUP), (dict(head_dim=256), H.ENOTSUP), (dict(page_rows=24), H.EINVAL),
                                       (dict(n_kv_heads=3), H.EINVAL), (dict(fmt=2), H.EINVAL), (dict(n_pages=0), H.EINVAL),
                                       (dict(sm_scale=1e-40), H.EINVAL)], ids=str)
def test_the_binding_says_why_a_pool_is_refused(over, code):
    with pytest.raises(H.HermesError) as e:
        H.KVPages(**(dict(n_q_heads=4, n_kv_heads=2, head_dim=64, n_pages=3) | over))
    assert e.value.code == code
