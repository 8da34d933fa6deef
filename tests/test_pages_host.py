"""Pages without a device: the refusals of the C ABI, sizes, and pins of the fp64
reference (quantiser, layout, attention)."""
import ctypes
import itertools

import numpy as np
import pytest
import torch

from oracle import pages_oracle as orc
from paper_2601_14724_amd import hermes as H

FAKE = 0x100000   # aligned, never dereferenced: every call below fails validation first


def _pool(**over):
    p = H.PagePoolStruct()
    p.n_q_heads, p.n_kv_heads, p.head_dim, p.format = 4, 2, 64, H.PAGE_FP4
    p.page_rows, p.n_pages, p.pages = 32, 10, FAKE
    for k, v in over.items():
        if k == "mrope_section":
            for i in range(3):
                p.mrope_section[i] = v[i]
        else:
            setattr(p, k, v)
    return p


def _batch(**over):
    b = H.PageBatchStruct()
    b.n_seqs, b.n_rows, b.max_rows, b.max_len, b.max_pages = 3, 20, 10, 100, 8
    b.row_start, b.kv_len, b.tables = FAKE, FAKE, FAKE
    for k, v in over.items():
        setattr(b, k, v)
    return b


def _append(pool, batch, q=FAKE, qs=256, k=FAKE, ks=128, v=FAKE, vs=128, rope=FAKE, out=FAKE + 4096):
    return H.lib.hermes_page_append(ctypes.byref(pool) if pool else None, ctypes.byref(batch) if batch else None,
                                    q, qs, k, ks, v, vs, rope, out, None)


def _attend(pool, batch, q=FAKE, qs=256, out=FAKE, lse=None, ws=FAKE, nbytes=1 << 40):
    return H.lib.hermes_page_attend(ctypes.byref(pool) if pool else None, ctypes.byref(batch) if batch else None,
                                    q, qs, out, lse, ws, nbytes, None)


def _read(pool, batch, k=FAKE, v=FAKE):
    return H.lib.hermes_page_read(ctypes.byref(pool) if pool else None, ctypes.byref(batch) if batch else None, k, v, None)


BAD_POOLS = [dict(n_kv_heads=0), dict(n_q_heads=5), dict(n_q_heads=1), dict(format=2), dict(format=-1),
             dict(page_rows=8), dict(page_rows=48), dict(page_rows=512), dict(n_pages=0), dict(pages=None),
             dict(pages=FAKE + 8), dict(status=FAKE + 2), dict(sm_scale=float("inf")), dict(sm_scale=1e-40), dict(sm_scale=1e39),
             dict(rope_theta=float("nan")), dict(rope_axes=2), dict(rope_axes=3, mrope_section=(1, 2, 3)),
             dict(rope_axes=3, mrope_section=(-1, 17, 16)), dict(n_q_heads=1 << 17, n_kv_heads=1)]
BAD_BATCHES = [dict(n_seqs=-1), dict(n_rows=-1), dict(max_rows=-1), dict(max_len=-1), dict(max_pages=0),
               dict(row_start=None), dict(row_start=FAKE + 2), dict(kv_len=None), dict(kv_len=FAKE + 1),
               dict(tables=None), dict(tables=FAKE + 2), dict(max_pages=1 << 26), dict(n_seqs=1 << 24),
               dict(n_rows=(1 << 30) + 1)]


@pytest.mark.parametrize("over", BAD_POOLS, ids=str)
def test_bad_pools_are_refused(over):
    for call in (_append, _attend, _read):
        assert call(_pool(**over), _batch()) == H.EINVAL


@pytest.mark.parametrize("over", BAD_BATCHES, ids=str)
def test_bad_batches_are_refused(over):
    for call in (_append, _attend, _read):
        assert call(_pool(), _batch(**over)) == H.EINVAL


def test_more_rows_than_a_launch_holds_are_refused():
    """A row takes a wave, and a launch's threads are counted in 32 bits: 2^26 rows are 2^32."""
    for call in (_append, _attend, _read):
        assert call(_pool(), _batch(n_rows=1 << 26)) == H.EINVAL
        assert call(_pool(), _batch(n_rows=(1 << 25) + 1)) == H.EINVAL
    most = _batch(n_rows=1 << 25, max_rows=0, max_len=0)     # (no hints, so that cuts are planned for)
    assert H.lib.hermes_page_workspace_bytes(ctypes.byref(_pool()), ctypes.byref(most)) > 0


def test_null_structs_and_head_dims_are_refused():
    for call in (_append, _attend, _read):
        assert call(None, _batch()) == H.EINVAL
        assert call(_pool(), None) == H.EINVAL
        assert call(_pool(head_dim=96), _batch()) == H.ENOTSUP
        assert call(_pool(head_dim=256), _batch()) == H.ENOTSUP
    assert H.lib.hermes_page_bytes(None) == 0
    assert H.lib.hermes_page_bytes(ctypes.byref(_pool(head_dim=96))) == 0


def test_bad_append_arguments_are_refused():
    p, b = _pool(), _batch()
    for over in (dict(k=None), dict(v=None), dict(k=FAKE + 8), dict(v=FAKE + 2), dict(q=FAKE + 8), dict(out=None),
                 dict(q=None), dict(rope=None), dict(rope=FAKE + 1), dict(qs=248), dict(ks=120), dict(vs=132),
                 dict(qs=260), dict(out=FAKE + 8), dict(out=FAKE, qs=512)):
        assert _append(p, b, **over) == H.EINVAL, over


def test_bad_attend_and_read_arguments_are_refused():
    p, b = _pool(), _batch(max_len=0, max_pages=100)     # (long enough to be cut, so a workspace is needed)
    for over in (dict(q=None), dict(q=FAKE + 2), dict(qs=200), dict(qs=257), dict(out=None), dict(out=FAKE + 4),
                 dict(lse=FAKE + 2), dict(ws=None), dict(ws=FAKE + 8)):
        assert _attend(p, b, **over) == H.EINVAL, over
    need = H.lib.hermes_page_workspace_bytes(ctypes.byref(p), ctypes.byref(b))
    assert need > 0 and _attend(p, b, nbytes=need - 1) == H.ECAPACITY
    assert _read(p, b, k=FAKE + 8) == H.EINVAL and _read(p, b, v=FAKE + 2) == H.EINVAL


def test_a_batch_on_two_devices_is_refused(monkeypatch):
    """(shapes and types are checked elsewhere; the "meta" device stands in for a second one)"""
    monkeypatch.setattr(H, "_need", lambda *a: None)
    here, there = [lambda *s, d=d: torch.empty(s, dtype=torch.int32, device=d) for d in ("cpu", "meta")]
    H.PageBatch(here(3, 8), here(3), here(4), n_rows=5)
    for tables, lens, starts in ((there(3, 8), here(3), here(4)), (here(3, 8), there(3), here(4)),
                                 (here(3, 8), here(3), there(4))):
        with pytest.raises(ValueError, match="device"):
            H.PageBatch(tables, lens, starts, n_rows=5)


def test_empty_batches_do_nothing():
    for over in (dict(n_seqs=0, n_rows=0, row_start=None), dict(n_rows=0), dict(n_seqs=0, row_start=FAKE)):
        for call in (_append, _attend, _read):
            assert call(_pool(), _batch(kv_len=None, tables=None, max_pages=0, **over)) == H.OK
    assert _read(_pool(), _batch(), k=None, v=None) == H.OK


def test_pack_refuses_a_null_context():
    assert H.lib.hermes_page_pack(None, 0, ctypes.byref(_pool()), FAKE, 4, FAKE, None) == H.EINVAL


@pytest.mark.parametrize("d,page,fmt", itertools.product((64, 128), (16, 32, 64, 128, 256), ("bf16", "fp4")))
def test_page_bytes(d, page, fmt):
    p = _pool(head_dim=d, page_rows=page, format=H.PAGE_FP4 if fmt == "fp4" else H.PAGE_BF16)
    assert H.lib.hermes_page_bytes(ctypes.byref(p)) == 2 * orc.block_bytes(d, page, fmt)


def test_workspace_is_bounded_by_the_hints():
    """A batch that fills the device by itself needs none; without a hint the table's
    capacity counts."""
    p = _pool(n_q_heads=28, n_kv_heads=4, head_dim=128)
    need = lambda **o: H.lib.hermes_page_workspace_bytes(ctypes.byref(p), ctypes.byref(_batch(**o)))
    assert need(n_seqs=1000, n_rows=1000, max_rows=1, row_start=None) == 0
    one = need(n_seqs=1, n_rows=1, max_rows=1, row_start=None, max_len=6144, max_pages=1000)
    assert 0 < one <= need(n_seqs=1, n_rows=1, max_rows=1, row_start=None, max_len=0, max_pages=1000)
    assert need(n_seqs=1, n_rows=1, max_rows=1, row_start=None, max_len=100, max_pages=1000) == 0


# ---------------------------------------------------------------- the reference
def test_quantiser_takes_the_nearest_code_and_the_least_scale():
    rng = np.random.default_rng(1)
    x = orc.bf16_bits(rng.standard_normal((200, 64)) * np.exp2(rng.integers(-60, 60, (200, 1))))
    code, scale = orc.fp4(x)
    val, true = orc.fp4_value(code, scale), orc.bf16_value(x)
    step = 2.0 ** (scale.astype(float) - 127)
    amax = np.abs(true).reshape(200, 2, 32).max(-1)
    assert (amax <= 7 * step).all() and (amax > 3.5 * step).all()
    grid = np.concatenate([-orc.LEVELS, orc.LEVELS])[None, None] * step.repeat(32, 1)[..., None]
    assert (np.abs(val - true) == np.abs(grid - true[..., None]).min(-1)).all()
    assert (np.abs(val - true).reshape(200, 2, 32).max(-1) <= step).all()     # half of the widest step


def test_quantiser_by_hand():
    row = np.zeros(32)
    row[:12] = [6, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5, -0.25, -0.75, -5, 0.26]
    code, scale = orc.fp4(orc.bf16_bits(row)[None])
    assert scale[0, 0] == 127
    assert orc.fp4_value(code, scale)[0, :12].tolist() == [6, 0, 1, 1, 2, 2, 4, 4, 0, -1, -4, 0.5]
    for top, want in ((7.0, 0), (7.03125, 1), (3.5, -1), (3.515625, 0), (2.0 ** 127, 125), (2.0 ** -126, -119), (0, -119)):
        row = np.zeros(32)
        row[3] = top
        assert orc.fp4(orc.bf16_bits(row)[None])[1][0, 0] == want + 127


def test_rotation_turns_pairs_and_keeps_lengths():
    x = np.random.default_rng(2).standard_normal((5, 2, 64))
    same = orc.rotate(x, np.zeros(5, int))
    assert (same == orc.bf16_bits(x)).all()
    y = orc.bf16_value(orc.rotate(x, [1, 10, 1000, 10 ** 6, -7]))
    n = lambda z: np.hypot(z[..., :32], z[..., 32:])
    assert np.abs(n(y) - n(x)).max() <= 2.0 ** -8 * np.abs(n(x)).max() * 2
    three = orc.rotate(x, np.tile([3, 5, 8, 2, 1], (3, 1)))
    assert (three == orc.rotate(x, [3, 5, 8, 2, 1])).all()


def test_reference_attention_matches_a_plain_softmax():
    rng = np.random.default_rng(3)
    q, k, v = rng.standard_normal((3, 4, 64)), rng.standard_normal((7, 2, 64)), rng.standard_normal((7, 2, 64))
    out, lse, mag, _ = orc.attend(q, k, v, 0.125)
    x = k[:6, 1] @ q[1, 3] * 0.125
    p = np.exp(x) / np.exp(x).sum()
    assert np.allclose(out[1, 3], p @ v[:6, 1], rtol=0, atol=1e-14)
    assert abs(lse[1, 3] - np.log(np.exp(x).sum())) < 1e-14
    out, lse, _, _ = orc.attend(q, k[:1], v[:1], 0.125)     # three rows, one token
    assert (out[:2] == 0).all() and np.isneginf(lse[:2]).all() and np.allclose(out[2], v[0].repeat(2, 0))
