"""What stands around a generated token, without a device: the refusals of the C ABI and of
the binding, sizes, and pins of the fp64 reference."""
import ctypes

import numpy as np
import pytest
import torch

from oracle import pages_oracle as pages
from oracle import tokens_oracle as orc
from paper_2601_14724_amd import hermes as H

FAKE = 0x100000   # aligned, never dereferenced: every call below fails validation first
FAR = 1 << 40


# --------------------------------------------------------------------- weights
def _weight(n_out=100, n_in=200, data=FAKE):
    return H.WeightStruct(n_out, n_in, data)


def _product(w=None, x=FAR, xs=200, rows=4, bias=None, add=None, out=2 * FAR, kind=H.BF16, ws=None, nbytes=0):
    return H.lib.hermes_weight_product(ctypes.byref(w or _weight()), x, xs, rows, bias, add, out, kind, ws, nbytes, None)


@pytest.mark.parametrize("n,k", [(1, 1), (16, 128), (17, 129), (1003, 2236), (4608, 3584), (131072, 513)])
def test_weight_bytes(n, k):
    codes, scales = -(-n // 16) * -(-k // 128) * 1024, -(-n // 16) * -(-k // 512) * 256
    assert H.lib.hermes_weight_bytes(ctypes.byref(_weight(n, k, None))) == codes + scales


@pytest.mark.parametrize("over", [dict(n_out=0), dict(n_in=0), dict(n_out=-3), dict(n_out=(1 << 24) + 1), dict(n_in=(1 << 20) + 1)],
                         ids=str)
def test_bad_weights_are_refused(over):
    w = _weight(**over)
    assert H.lib.hermes_weight_bytes(ctypes.byref(w)) == 0
    assert H.lib.hermes_weight_pack(ctypes.byref(w), FAR, 1 << 21, None) == H.EINVAL
    assert _product(w, xs=1 << 21) == H.EINVAL


def test_bad_pack_arguments_are_refused():
    pack = lambda w, dense, stride: H.lib.hermes_weight_pack(w and ctypes.byref(w), dense, stride, None)
    assert pack(None, FAR, 200) == H.EINVAL
    for args in ((_weight(data=None), FAR, 200), (_weight(data=FAKE + 8), FAR, 200), (_weight(), None, 200),
                 (_weight(), FAR + 1, 200), (_weight(), FAR, 199), (_weight(), FAR, 1 << 40), (_weight(), FAKE, 200),
                 (_weight(), FAKE - 100, 200)):
        assert pack(*args) == H.EINVAL, args[1:]


def test_bad_product_arguments_are_refused():
    for over in (dict(w=_weight(data=None)), dict(w=_weight(data=FAKE + 4)), dict(x=None), dict(x=FAR + 8), dict(xs=192),
                 dict(xs=204), dict(xs=(1 << 24) + 8), dict(rows=-1), dict(rows=(1 << 20) + 1), dict(out=None), dict(out=2 * FAR + 8),
                 dict(bias=FAKE + 1), dict(add=FAKE + 1), dict(kind=2), dict(kind=-1),
                 dict(out=FAR), dict(out=FAR + 3 * 400), dict(bias=2 * FAR + 790), dict(add=2 * FAR + 2),
                 dict(add=2 * FAR, kind=H.FP32), dict(out=FAKE + 16)):
        assert _product(**over) == H.EINVAL, over
    assert H.lib.hermes_weight_product(None, FAR, 200, 4, None, None, 2 * FAR, 0, None, 0, None) == H.EINVAL


def test_products_that_are_cut_need_a_workspace():
    """Where a long sum has few outputs, workgroups share the inputs; else none is needed."""
    need = lambda n, k, rows: H.lib.hermes_weight_workspace_bytes(ctypes.byref(_weight(n, k)), rows)
    for n, k, rows in ((1152, 896, 1), (4608, 3584, 16), (14336, 3584, 64), (131072, 3584, 8), (1024, 14336, 8)):
        assert need(n, k, rows) == 0
    bytes_ = need(1000, 14336, 64)
    assert bytes_ > 0 and bytes_ % (64 * 64 * 63) == 0           # whole parts: fp32, 64 rows of 63 tiles of 16
    assert need(1000, 14336, 0) == 0 and need(0, 14336, 64) == 0 and need(1000, 14336, -1) == 0
    long = dict(w=_weight(1000, 14336), xs=14336, rows=64)
    assert _product(**long) == H.EINVAL and _product(**long, ws=FAKE + 8, nbytes=bytes_) == H.EINVAL
    assert _product(**long, ws=FAKE, nbytes=bytes_ - 1) == H.ECAPACITY


def test_a_product_of_no_rows_does_nothing():
    assert _product(rows=0, x=None, out=None) == H.OK


# ----------------------------------------------------------------------- beams
def _beam(**over):
    c = H.BeamConfig(2, 4, 1000, 8, H.BF16, 2, 2)
    for k, v in over.items():
        setattr(c, k, v)
    return c


def _select(cfg=None, logits=FAR, stride=1000, score=FAKE, done=None, outs=(2 * FAR, 3 * FAR, 4 * FAR, 5 * FAR), ws=6 * FAR,
            nbytes=1 << 30):
    return H.lib.hermes_beam_select(ctypes.byref(cfg or _beam()), logits, stride, score, done, *outs, ws, nbytes, None)


BAD_BEAMS = [dict(n_seqs=-1), dict(n_beams=0), dict(n_beams=65), dict(n_vocab=0), dict(n_keep=0), dict(n_keep=65),
             dict(n_seqs=1 << 14), dict(n_vocab=1 << 29), dict(logits_type=2), dict(end_token=-2), dict(end_token=1000),
             dict(pad_token=-1), dict(pad_token=1000)]


@pytest.mark.parametrize("over", BAD_BEAMS, ids=str)
def test_bad_beam_configs_are_refused(over):
    assert H.lib.hermes_beam_workspace_bytes(ctypes.byref(_beam(**over))) == 0
    assert _select(_beam(**over), stride=1 << 30) == H.EINVAL


def test_bad_select_arguments_are_refused():
    none_of = lambda i: tuple(None if j == i else (2 + j) * FAR for j in range(4))
    for over in (dict(logits=None), dict(logits=FAR + 1), dict(stride=999), dict(stride=1 << 40), dict(score=None),
                 dict(score=FAKE + 2), dict(done=FAKE + 1), dict(outs=none_of(0)), dict(outs=none_of(1)), dict(outs=none_of(2)),
                 dict(outs=(2 * FAR + 1, 3 * FAR, 4 * FAR, None)), dict(outs=(2 * FAR, 2 * FAR + 60, 4 * FAR, None)),
                 dict(outs=(FAKE + 4, 3 * FAR, 4 * FAR, None)), dict(outs=(FAR + 8000, 3 * FAR, 4 * FAR, None)),
                 dict(done=3 * FAR), dict(ws=None), dict(ws=6 * FAR + 8)):
        assert _select(**over) == H.EINVAL, over
    need = H.lib.hermes_beam_workspace_bytes(ctypes.byref(_beam()))
    assert need > 0 and _select(nbytes=need - 1) == H.ECAPACITY
    assert _select(_beam(logits_type=H.FP32), logits=FAR + 2) == H.EINVAL
    assert H.lib.hermes_beam_select(None, FAR, 1000, FAKE, None, 2 * FAR, 3 * FAR, 4 * FAR, None, FAR, 1 << 30, None) == H.EINVAL


def test_a_choice_of_no_sequences_does_nothing():
    assert _select(_beam(n_seqs=0), logits=None, score=None, outs=(None,) * 4, ws=None) == H.OK
    assert H.lib.hermes_beam_workspace_bytes(ctypes.byref(_beam(n_seqs=0))) == 0


def test_the_binding_refuses_other_logits():
    score = torch.zeros(2, 3)
    for logits in (torch.zeros(2, 3, 10), torch.zeros(2, 3, 10, dtype=torch.float16), torch.zeros(6, 10), None):
        with pytest.raises(ValueError, match="logits"):
            H.beam_select(logits, score, 4)


def test_the_binding_refuses_other_weights():
    for dense in (torch.zeros(3, 4), torch.zeros(3, 4, dtype=torch.bfloat16), torch.zeros(3, dtype=torch.bfloat16), None):
        with pytest.raises(ValueError, match="dense"):
            H.PackedWeight(dense)


# --------------------------------------------------------------------- reorder
def _pool(**over):
    p = H.PagePoolStruct()
    p.n_q_heads, p.n_kv_heads, p.head_dim, p.format = 4, 2, 64, H.PAGE_FP4
    p.page_rows, p.n_pages, p.pages = 32, 10, FAKE
    for k, v in over.items():
        setattr(p, k, v)
    return p


def _beams(**over):
    b = H.PageBeamsStruct(6, 3, 4, 8, 1, FAR, 2 * FAR, 3 * FAR, 4 * FAR, 5 * FAR, 6 * FAR)
    for k, v in over.items():
        setattr(b, k, v)
    return b


def _reorder(pool, beams):
    return H.lib.hermes_page_reorder(ctypes.byref(pool) if pool else None, ctypes.byref(beams) if beams else None, None)


@pytest.mark.parametrize("over", [dict(n_groups=-1), dict(n_seqs=0), dict(n_seqs=4), dict(n_beams=0), dict(n_beams=65),
                                  dict(max_pages=0), dict(max_pages=1 << 26), dict(grow=-1), dict(grow=(1 << 20) + 1),
                                  dict(n_groups=3 << 20), dict(parent=None), dict(room=None), dict(tables=None),
                                  dict(kv_len=None), dict(tables_out=None), dict(kv_len_out=None), dict(parent=FAR + 2),
                                  dict(tables_out=3 * FAR), dict(tables_out=3 * FAR + 6 * 4 * 8 * 4 - 4),
                                  dict(kv_len_out=4 * FAR), dict(kv_len_out=5 * FAR + 4), dict(kv_len_out=FAR),
                                  dict(tables_out=2 * FAR)], ids=str)
def test_bad_reorders_are_refused(over):
    assert _reorder(_pool(), _beams(**over)) == H.EINVAL


def test_reorders_of_bad_pools_are_refused():
    assert _reorder(None, _beams()) == H.EINVAL and _reorder(_pool(), None) == H.EINVAL
    assert _reorder(_pool(head_dim=96), _beams()) == H.ENOTSUP
    assert _reorder(_pool(page_rows=48), _beams()) == H.EINVAL and _reorder(_pool(pages=None), _beams()) == H.EINVAL


def test_a_reorder_of_no_groups_does_nothing():
    assert _reorder(_pool(), _beams(n_groups=0, n_seqs=0, tables=None, parent=None)) == H.OK


# ---------------------------------------------------------------- the reference
def test_weight_memory_by_hand():
    """One value in a weight of zeros: its code and its scale lie where the layout says."""
    for n, k in ((0, 0), (5, 33), (15, 127), (16, 128), (20, 700)):
        bits = np.zeros((21, 800), np.uint16)
        bits[n, k] = pages.bf16_bits(-1.5)
        codes, scales = orc.pack(bits)
        lane = 16 * (k % 32 // 8) + n % 16
        at = ((n // 16 * 7 + k // 128) * 64 + lane) * 16 + 4 * (k % 128 // 32) + k % 8 // 2
        # 1.5 = 6 x 2^-2: code 7, with the sign 15
        assert codes[at] == 15 << (4 * (k % 2)) and codes.sum() == codes[at]
        assert scales[n // 16, k // 512, n % 16, k // 128 % 4, k % 128 // 32] == 127 - 2 and (scales != 8).sum() == 1


def test_reference_product_of_one_row():
    w = np.zeros((3, 40))
    w[1, 39], w[2, 0] = 2.0, -3.0
    out, mag = orc.product(np.arange(40.0)[None], w, bias=np.array([1.0, 0, 0]), add=np.array([[0, 0, 5.0]]))
    assert out.tolist() == [[1.0, 78.0, 5.0]] and mag.tolist() == [[1.0, 78.0, 5.0]]


def whole_numbers(m, n, k, device="cpu", seed=0):
    """x [m][k], w [n][k] (fp64) of whole numbers, w as 4 bits hold them: a 6 in every 32 inputs makes their scale 1.
    Sums of up to 2^18 terms stay below 2^24, so that fp32 holds every one of them, in any order and cut."""
    g = torch.Generator(device=device).manual_seed(1000 * seed + m + n + k)
    level = torch.tensor([0, 1, 2, 3, 4, 6, -1, -2, -3, -4, -6], dtype=torch.float64, device=device)
    w = level[torch.randint(0, 11, (n, k), generator=g, device=device)]
    w[:, ::32] = 6
    w[::2, ::32] = -6
    x = torch.randint(1, 8, (m, k), generator=g, device=device).double()
    x[torch.rand((m, k), generator=g, device=device) < 0.5] *= -1
    return x, w


@pytest.mark.parametrize("m,n,k", [(9, 1000, 14336), (1, 300, 20000), (33, 33, 2565)])
def test_whole_numbers_show_what_a_product_leaves_out(m, n, k):
    """What exact tests of long products see: a piece of eight inputs, or the last few, left out or taken twice; and
    parts of a sum that are rounded to bf16."""
    x, w = whole_numbers(m, n, k)
    bits = pages.bf16_bits(w[:40].numpy().astype(np.float32))
    assert (orc.weight(bits) == w[:40].numpy()).all()
    want = x @ w.T
    assert 300 < want.abs().max() < 2 ** 24 and (want.float().double() == want).all()
    for i in range(0, k, 8):
        assert (x[:, i:i + 8] @ w[:, i:i + 8].T != 0).any()
    halves = [(x[:, a:b] @ w[:, a:b].T).bfloat16().double() for a, b in ((0, k // 256 * 128), (k // 256 * 128, k))]
    assert (halves[0] + halves[1] != want).any()


def test_reference_choice_by_hand():
    logits = np.log(np.array([[0.5, 0.25, 0.25], [0.125, 0.125, 0.75]]))
    v, parent, token = orc.select(orc.values(logits, np.array([-1.0, -1.0])), 4)
    assert parent.tolist() == [1, 0, 0, 0] and token.tolist() == [2, 0, 1, 2]
    assert np.allclose(v, -1 + np.log([0.75, 0.5, 0.25, 0.25]))
    v, parent, token = orc.select(orc.values(logits, np.array([-1.0, -1.2]), done=[0, 1], pad=1), 2)
    assert parent.tolist() == [1, 0] and token.tolist() == [1, 0] and v[0] == -1.2
    bad = logits.copy()
    bad[1, 0] = np.inf
    assert (orc.select(orc.values(bad, np.array([0.0, 5.0])), 9)[1] == 0).all()
    assert len(orc.select(orc.values(np.full((1, 3), -np.inf), np.zeros(1)), 2)[0]) == 0


def test_reference_reorder_by_hand():
    """Two rows a page.  Both beams go on from beam 0, which has three rows: its full page 0 is
    shared, its own page 11 kept by the first child and copied to the lowest free page for the second."""
    tables = np.array([[0, 11, -1], [0, 10, 13]], np.int32)
    out, lens, copies, bits = orc.reorder(tables, np.array([3, 5], np.int32), [0, 0], (10, 4), 2, 2, 14)
    assert out.tolist() == [[0, 11, 10], [0, 12, 13]] and lens.tolist() == [3, 3] and copies == [(11, 12, 4)] and bits == 0
    out, _, copies, bits = orc.reorder(tables, np.array([3, 5], np.int32), [1, -1], (12, 1), 0, 2, 14)
    assert out.tolist() == [[0, 10, 12], [-1] * 3] and copies == [(13, 12, 4)] and bits == 0
    out, _, copies, bits = orc.reorder(tables, np.array([3, 5], np.int32), [0, 0], (12, 1), 1, 2, 14)
    assert out.tolist() == [[0, 12, -1], [0, -1, -1]] and copies == [(11, 12, 4)] and bits == orc.NO_ROOM
