"""What stands around a generated token on the device, against the fp64 reference
(oracle/tokens_oracle.py).

What a weight stands for is exact, and so are the reordered tables and pages.  A product's
result is off by what its sums round: of n terms, in any order, n additions of up to
2^-23 of the terms' magnitudes (an addition may truncate), and half a step of the output.  A
choice is compared as test_tokens_bounds.check_choice says."""
import ctypes

import numpy as np
import pytest
import torch

from oracle import pages_oracle as pages
from oracle import tokens_oracle as orc
from paper_2601_14724_amd import hermes as H
from tests.test_tokens_bounds import DOUBT, beams_of, check_choice
from tests.test_tokens_host import whole_numbers

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def bf16(bits):
    return torch.from_numpy(np.ascontiguousarray(bits).view(np.int16)).to(DEV).view(torch.bfloat16)


def i32(x):
    return torch.tensor(np.asarray(x), dtype=torch.int32, device=DEV)


def rows_apart(bits, stride, fill=0x7FC0):
    """bf16 rows `stride` apart, NaN between them."""
    full = np.full((bits.shape[0], stride), fill, np.uint16)
    full[:, :bits.shape[1]] = bits
    return bf16(full)[:, :bits.shape[1]]


# --------------------------------------------------------------------- weights
def weight_bits(n, k, seed, scale=0.05):
    rng = np.random.default_rng(seed)
    return pages.bf16_bits(rng.standard_normal((n, k)) * scale * np.exp2(rng.integers(-3, 4, (n, 1))))


@pytest.mark.parametrize("n,k,stride", [(1, 1, 1), (16, 128, 128), (17, 129, 131), (40, 700, 700), (33, 1025, 1040), (5, 31, 33)])
def test_a_packed_weight_is_the_definition_s(n, k, stride):
    bits = weight_bits(n, k, 1)
    bits[0, :min(k, 32)] = 0
    if n > 4 and k > 40:
        bits[3, 32:64] = pages.bf16_bits(2.0 ** -126)
        bits[4, 40] = 0x7F80            # an infinity: a block of NaN
    w = H.PackedWeight(rows_apart(bits, stride))
    codes, scales = orc.pack(bits)
    got = w.data.cpu().numpy()
    got_codes, got_scales = got[:codes.size], got[codes.size:].reshape(scales.shape)
    used = ~orc.unused_scales(n, k)
    assert (got_scales == scales)[used].all()
    if n > 4 and k > 40:
        assert (scales == 255).sum() == 1
        bits[4, 32:64] = 0                # (the codes of a block of NaN may be any)
        codes2, _ = orc.pack(bits)
        lane = (0, [4, 20, 36, 52], slice(4, 8))      # output 4, inputs 32 to 63 of the first tile
        got_codes = got_codes.copy()
        got_codes.reshape(-1, 64, 16)[lane] = 0
        codes2.reshape(-1, 64, 16)[lane] = 0
        codes = codes2
    # (a code of zero may keep its sign)
    low, high = got_codes & 15, got_codes >> 4
    assert (np.where(low == 8, 0, low) == np.where(codes & 15 == 8, 0, codes & 15)).all()
    assert (np.where(high == 8, 0, high) == np.where(codes >> 4 == 8, 0, codes >> 4)).all()


def check_product(m, n, k, out, bias=False, add=False, stride=None, in_place=False, seed=0):
    rng = np.random.default_rng(seed)
    wb = weight_bits(n, k, seed + 1)
    xb = pages.bf16_bits(rng.standard_normal((m, k)))
    bb = pages.bf16_bits(rng.standard_normal(n)) if bias else None
    ab = pages.bf16_bits(rng.standard_normal((m, n)) * 3) if add else None
    w = H.PackedWeight(bf16(wb))
    x = rows_apart(xb, stride or -(-k // 8) * 8)
    kind = torch.bfloat16 if out == "bf16" else torch.float32
    extra = dict(bias=bf16(bb) if bias else None, add=bf16(ab) if add else None)
    if in_place:
        got = w.product(x, out=extra["add"], **extra)
        assert got is extra["add"]
    else:
        got = w.product(x, dtype=kind, **extra)
    assert got.dtype == kind and got.shape == (m, n)
    v = pages.bf16_value
    want, mag = orc.product(v(xb), orc.weight(wb), None if bb is None else v(bb), None if ab is None else v(ab))
    half = np.abs(want) * (2.0 ** -9 if out == "bf16" else 2.0 ** -24)
    sums = (k + 2) * 2.0 ** -23 * mag
    err = np.abs(got.double().cpu().numpy() - want)
    # the sum's error may carry the rounding to the next step: 2^-8 of the sum's error is far below `sums`
    assert (err <= sums * (1 + 2.0 ** -8) + half * 2 + 1e-30).all(), (err / (sums + half)).max()


@pytest.mark.parametrize("m", [1, 2, 5, 16, 17, 31, 33, 64, 65, 130])
def test_products_of_any_number_of_rows(m):
    check_product(m, 83, 300, "bf16", bias=True, seed=m)


@pytest.mark.parametrize("n", [1, 3, 16, 17, 64, 129, 1000])
@pytest.mark.parametrize("k", [1, 7, 8, 33, 127, 128, 129, 511, 513, 1100])
def test_products_of_any_size(n, k):
    check_product(3, n, k, "fp32", seed=n + k)


@pytest.mark.parametrize("m,n,k", [(1, 1152, 896), (16, 4608, 3584), (5, 1003, 2236), (64, 2048, 3584), (8, 40000, 512),
                                   (1, 300, 20000), (40, 5000, 1000), (4, 20001, 1153)])
@pytest.mark.parametrize("out", ["bf16", "fp32"])
def test_products_of_a_model_s_sizes(m, n, k, out):
    check_product(m, n, k, out, bias=n < 5000, add=n < 2000)


@pytest.mark.parametrize("m,n,k", [(16, 64, 5120), (9, 1000, 14336), (13, 4608, 8000), (32, 250, 5200), (17, 2048, 6001),
                                   (64, 64, 2560), (64, 1000, 8001), (33, 4000, 2700), (65, 130, 4000), (130, 20, 9000)])
@pytest.mark.parametrize("out", ["bf16", "fp32"])
def test_products_whose_inputs_are_shared_by_workgroups(m, n, k, out):
    assert H.lib.hermes_weight_workspace_bytes(ctypes.byref(H.WeightStruct(n, k, None)), m) > 0
    check_product(m, n, k, out, bias=True, add=n < 2000, seed=m)


@pytest.mark.parametrize("m,n,k", [(9, 16390, 200), (16, 33000, 130), (13, 66001, 64), (17, 16500, 1153), (32, 32800, 40),
                                   (30, 65600, 129), (33, 17000, 515), (64, 40001, 250), (48, 65540, 127), (100, 9001, 700),
                                   (200, 4610, 385), (16, 1000, 384), (64, 129, 257), (130, 65, 300), (24, 9000, 1531), (64, 1, 1), (5, 20010, 384),
                                   (8, 40, 129)])
@pytest.mark.parametrize("out", ["bf16", "fp32"])
def test_products_whose_rows_are_shared_by_waves(m, n, k, out):
    check_product(m, n, k, out, bias=True, add=n < 10000, seed=n)


# Every cut of the inputs and outputs that a product can have, with odd last tiles: up to 4, 8, 16, 32 and 64 rows;
# one, two and four tiles of outputs a wave; inputs shared by one to eight waves, and by workgroups; rows shared by waves.
WHOLE = [(1, 33, 5), (4, 5265, 5), (1, 33, 133), (4, 7985, 133), (1, 33, 515), (1, 14385, 1153), (1, 33, 903), (3, 2077, 5127),
         (1, 67185, 1300), (1, 25585, 1300), (2, 25585, 2565), (1, 16465, 1300), (3, 16477, 1531), (5, 33, 515), (7, 1037, 600),
         (5, 33, 903), (8, 2065, 1531), (5, 67185, 515), (5, 25585, 515), (7, 47985, 600), (5, 3185, 515), (7, 7997, 600),
         (5, 3185, 903), (8, 5265, 1153), (5, 67185, 1300), (5, 25585, 1300), (8, 25585, 1531), (5, 5265, 1300), (7, 9757, 2700),
         (5, 33, 5), (7, 9597, 300), (9, 33, 515), (16, 989, 600), (9, 33, 903), (13, 3025, 903), (9, 33, 5127), (9, 317, 20000),
         (5, 47985, 5), (7, 47985, 300), (9, 3185, 515), (16, 3197, 600), (9, 3185, 903), (9, 3185, 2565), (9, 1025, 5127),
         (9, 2045, 9005), (5, 67185, 5), (13, 131197, 300), (9, 5265, 515), (13, 5277, 600), (9, 5265, 903), (9, 14397, 2700),
         (9, 2065, 5127), (16, 4945, 5127), (17, 33, 5), (24, 2045, 300), (17, 33, 515), (17, 977, 600), (17, 33, 903),
         (17, 1025, 1531), (17, 33, 5127), (32, 305, 9005), (17, 47985, 5), (24, 47997, 903), (17, 3185, 515), (24, 3185, 600),
         (17, 3185, 903), (32, 3185, 2003), (17, 1025, 5127), (24, 1025, 14336), (17, 67185, 5), (17, 131197, 515), (17, 5265, 515),
         (17, 7997, 600), (17, 5265, 903), (24, 9597, 2003), (17, 2065, 5127), (24, 3025, 14336), (33, 33, 5), (33, 4945, 300),
         (33, 33, 515), (64, 1037, 1531), (33, 33, 2565), (33, 977, 2700), (65, 16465, 5), (33, 47985, 1531), (33, 3185, 515),
         (65, 3197, 1531), (33, 1025, 2565), (65, 2033, 5127), (33, 67185, 5), (130, 131185, 133), (33, 5265, 515), (50, 9745, 2565),
         (33, 2065, 2565), (50, 7997, 2565), (9, 1000, 14336), (1, 300, 20000), (13, 4608, 8000), (16, 4608, 3584),
         (64, 14336, 3584), (4, 1152, 18944)]


@pytest.mark.parametrize("m,n,k", WHOLE)
def test_products_of_whole_numbers_are_exact(m, n, k):
    """Sums that fp32 holds whatever their order: equal bit for bit, in bf16 after the one rounding."""
    x, w = whole_numbers(m, n, k, DEV)
    packed = H.PackedWeight(w.to(torch.bfloat16))
    rows = torch.full((m, -(-k // 8) * 8 + 8), float("nan"), dtype=torch.bfloat16, device=DEV)[:, :k]
    rows.copy_(x)
    want = torch.mm(x, w.T.contiguous())
    assert torch.equal(packed.product(rows, dtype=torch.float32).double(), want)
    bias = torch.arange(n, device=DEV) % 199 - 99.0
    add = (torch.arange(m * n, device=DEV) % 251 - 125.0).view(m, n)
    want += bias + add
    extra = dict(bias=bias.to(torch.bfloat16), add=add.to(torch.bfloat16))
    assert torch.equal(packed.product(rows, dtype=torch.float32, **extra).double(), want)
    assert torch.equal(packed.product(rows, **extra), want.to(torch.bfloat16))


@pytest.mark.parametrize("n", [50, 64])
def test_a_residual_is_added_in_place(n):
    check_product(9, n, 200, "bf16", bias=True, add=True, stride=264, in_place=True)


def test_products_of_strided_rows_and_of_empty_ones():
    check_product(7, 40, 256, "bf16", stride=1024)
    w = H.PackedWeight(bf16(weight_bits(20, 64, 1)))
    assert w.product(torch.empty(0, 64, dtype=torch.bfloat16, device=DEV)).shape == (0, 20)


def test_products_refuse_other_tensors():
    w = H.PackedWeight(bf16(weight_bits(20, 60, 1)))
    x = torch.zeros(4, 64, dtype=torch.bfloat16, device=DEV)
    w.product(x[:, :60])
    w.product(torch.zeros(1, 60, dtype=torch.bfloat16, device=DEV))       # (one row lies nowhere apart)
    row = torch.zeros(4, 20, dtype=torch.bfloat16, device=DEV)
    for bad in (x, x[:, :60].contiguous(), x[:, :60].float(), x[:, :60].cpu(), torch.zeros(60, 4, device=DEV).to(x.dtype).T):
        with pytest.raises(ValueError):
            w.product(bad)
    for extra in (dict(bias=row[0].float()), dict(bias=row), dict(add=row[:2]), dict(add=row.T), dict(out=row[:3]), dict(out=row.half()),
                  dict(dtype=torch.float16), dict(bias=row[0].cpu())):
        with pytest.raises(ValueError):
            w.product(x[:, :60], **extra)
    for bad in (torch.zeros(4, 72, dtype=torch.bfloat16, device=DEV)[:, 4:64], x[:1, :60].expand(4, 60)):   # misaligned; one row
        with pytest.raises(H.HermesError):
            w.product(bad)
    room = torch.zeros(400, dtype=torch.bfloat16, device=DEV)
    with pytest.raises(H.HermesError):
        w.product(room[:256].view(4, 64)[:, :60], out=room[200:280].view(4, 20))


def test_a_weight_s_columns_come_back_exactly():
    """x of unit rows: what the weight stands for, bit for bit; and an input's NaN stays in its row."""
    n, k = 70, 300
    wb = weight_bits(n, k, 5)
    w = H.PackedWeight(bf16(wb))
    eye = torch.eye(k, dtype=torch.bfloat16, device=DEV)
    x = torch.zeros(k, 304, dtype=torch.bfloat16, device=DEV)[:, :k]
    x.copy_(eye)
    assert (w.product(x, dtype=torch.float32).T.double().cpu().numpy() == orc.weight(wb)).all()
    x[7, 299] = float("nan")
    got = w.product(x, dtype=torch.float32)
    assert torch.isnan(got[7]).all() and not torch.isnan(got[:7]).any() and not torch.isnan(got[8:]).any()


def test_a_block_with_an_infinity_makes_its_output_nan():
    wb = weight_bits(40, 300, 6)
    wb[7, 130], wb[33, 299] = 0x7F80, 0x7FC0
    x = torch.randn(3, 304, device=DEV).to(torch.bfloat16)[:, :300]
    bad = torch.isnan(H.PackedWeight(bf16(wb)).product(x))
    assert bad[:, [7, 33]].all() and bad.sum() == 6


def test_an_infinite_input_does_as_the_sum_does():
    """(padded inputs and other tiles add nothing to it)"""
    wb = np.zeros((20, 140), np.uint16)
    wb[:, 139] = pages.bf16_bits(np.arange(20) % 3 - 1.0)
    x = torch.zeros(2, 144, dtype=torch.bfloat16, device=DEV)[:, :140]
    x[1, 139] = float("inf")
    got = H.PackedWeight(bf16(wb)).product(x, dtype=torch.float32).cpu().numpy()
    with np.errstate(invalid="ignore"):
        want = np.float32(np.inf) * (np.arange(20) % 3 - 1.0).astype(np.float32)
    assert (got[0] == 0).all() and np.array_equal(got[1], want, equal_nan=True)


def test_the_same_call_gives_the_same_bits():
    w = H.PackedWeight(bf16(weight_bits(5000, 1000, 7)))
    x = torch.randn(33, 1000, device=DEV).to(torch.bfloat16)
    first = w.product(x, dtype=torch.float32)
    logits = first.view(3, 11, 5000)
    chosen = H.beam_select(logits, torch.zeros(3, 11, device=DEV), 22)
    for _ in range(5):
        assert torch.equal(w.product(x, dtype=torch.float32), first)
        assert all(torch.equal(a, b) for a, b in zip(H.beam_select(logits, torch.zeros(3, 11, device=DEV), 22), chosen))


def test_a_weight_of_more_than_4_gib():
    """Its last outputs, whose codes and scales lie past 2^32 bytes; the others are zeros."""
    n, k = 2 ** 21 + 19, 4224
    dense = torch.zeros(n, k, dtype=torch.bfloat16, device=DEV)
    wb = weight_bits(40, k, 8)
    dense[-40:] = bf16(wb)
    w = H.PackedWeight(dense)
    del dense
    assert w.data.numel() > 2 ** 32
    xb = pages.bf16_bits(np.random.default_rng(9).standard_normal((2, k)))
    got = w.product(bf16(xb), dtype=torch.float32)
    assert (got[:, :-40] == 0).all()
    want, mag = orc.product(pages.bf16_value(xb), orc.weight(wb))
    err = np.abs(got[:, -40:].double().cpu().numpy() - want)
    assert (err <= (k + 2) * 2.0 ** -23 * mag + 2.0 ** -24 * np.abs(want)).all()


def test_a_product_writes_its_outputs_only():
    w = H.PackedWeight(bf16(weight_bits(37, 100, 2)))
    for kind in (torch.bfloat16, torch.float32):
        room = torch.full((8 * 37 + 64,), 7.0, dtype=kind, device=DEV)
        out = room[16:16 + 5 * 37].view(5, 37)
        w.product(torch.zeros(5, 104, dtype=torch.bfloat16, device=DEV)[:, :100], out=out)
        assert (out == 0).all() and (room[:16] == 7).all() and (room[16 + 5 * 37:] == 7).all()


# ----------------------------------------------------------------------- beams
def logits_of(rng, seqs, beams, vocab, kind, spread=3.0):
    x = (spread * rng.standard_normal((seqs, beams, vocab))).astype(np.float32)
    return pages.bf16_value(pages.bf16_bits(x)).astype(np.float32) if kind == "bf16" else x


def device_logits(x, kind, pad=0, offset=0):
    """x in rows `pad` longer, NaN between them, from `offset` elements into an allocation."""
    seqs, beams, vocab = x.shape
    dtype = torch.bfloat16 if kind == "bf16" else torch.float32
    room = torch.full((offset + seqs * beams * (vocab + pad),), float("nan"), dtype=dtype, device=DEV)
    rows = room[offset:].view(seqs, beams, vocab + pad)[..., :vocab]
    rows.copy_(torch.from_numpy(x).to(DEV))
    return rows


def choose(x, score, keep, kind="bf16", done=None, end=-1, pad_token=0, pad=0, offset=0):
    got = H.beam_select(device_logits(x, kind, pad, offset), torch.from_numpy(score).to(DEV), keep,
                        done=None if done is None else i32(done), end_token=end, pad_token=pad_token)
    got = [t.cpu().numpy() for t in got]
    check_choice(x, score, done, keep, end, pad_token, got)
    return got


@pytest.mark.parametrize("kind", ["bf16", "fp32"])
@pytest.mark.parametrize("seqs,beams,vocab,keep,pad,offset", [
    (1, 1, 1, 1, 0, 0), (1, 1, 2, 3, 0, 0), (2, 3, 511, 6, 1, 0), (3, 4, 512, 8, 0, 1), (1, 5, 513, 10, 3, 3),
    (5, 2, 1000, 2, 24, 0), (1, 64, 700, 64, 0, 0), (2, 8, 4099, 64, 5, 7), (1, 4, 32000, 4, 0, 0), (3, 5, 49999, 10, 17, 0),
    (4, 16, 20000, 32, 0, 0), (1, 2, 262144, 4, 0, 0), (40, 1, 100, 1, 0, 0), (700, 3, 130, 6, 1, 0)])
def test_choices_of_any_size(seqs, beams, vocab, keep, pad, offset, kind):
    rng = np.random.default_rng(vocab + beams)
    choose(logits_of(rng, seqs, beams, vocab, kind), -10 * rng.random((seqs, beams)).astype(np.float32), keep, kind, pad=pad,
           offset=offset)


@pytest.mark.parametrize("kind", ["bf16", "fp32"])
def test_done_beams_go_on_with_the_pad_token(kind):
    rng = np.random.default_rng(1)
    x = logits_of(rng, 4, 6, 3000, kind)
    x[0, 2] = np.nan                     # (what a done beam's logits hold does not matter)
    done = (rng.random((4, 6)) < 0.5).astype(np.int32) * 7
    done[0, 2] = done[3] = 1
    score = -4 * rng.random((4, 6)).astype(np.float32)
    got = choose(x, score, 12, kind, done=done, end=5, pad_token=1501)
    assert (got[1][3, :6] == np.argsort(-score[3], kind="stable")).all() and (got[2][3, :6] == 1501).all()
    assert (got[1][3, 6:] == -1).all()


def test_ties_go_to_the_lower_beam_and_token():
    score = np.zeros((1, 3), np.float32)
    got = choose(np.zeros((1, 3, 5000), np.float32), score, 64)
    assert (got[1] == 0).all() and (got[2][0] == np.arange(64)).all()
    got = choose(np.tile(np.float32([0, 1, 1, 0]), (1, 3, 400)), score, 10)
    assert (got[1] == 0).all() and got[2][0].tolist() == [1, 2, 5, 6, 9, 10, 13, 14, 17, 18]
    x = np.zeros((1, 3, 5000), np.float32)
    x[:, :, 4999] = 2
    got = choose(x, score, 5)
    assert got[1][0].tolist() == [0, 1, 2, 0, 0] and got[2][0].tolist() == [4999, 4999, 4999, 0, 1]


@pytest.mark.parametrize("kind", ["bf16", "fp32"])
@pytest.mark.parametrize("distinct", [False, True])
def test_more_candidates_than_the_list_holds(kind, distinct):
    """All but every 1024th run of 16 tokens reach any bound that a group of low ones sets."""
    vocab, rng = 64 * 512, np.random.default_rng(3)
    x = 5 + (logits_of(rng, 1, 2, vocab, kind, 0.5) if distinct else np.zeros((1, 2, vocab), np.float32))
    if kind == "bf16":
        x = pages.bf16_value(pages.bf16_bits(x)).astype(np.float32)
    x[0, :, np.arange(vocab) % 1024 < 16] = -20
    choose(x, np.float32([[-1, -1.5]]), 64, kind)


@pytest.mark.parametrize("kind", ["bf16", "fp32"])
def test_rising_and_falling_logits(kind):
    x = np.linspace(-30, 30, 20000, dtype=np.float32)
    x = np.stack([x, x[::-1], np.roll(x, 777)])[None]
    if kind == "bf16":
        x = pages.bf16_value(pages.bf16_bits(x)).astype(np.float32)
    choose(x, np.float32([[0, -1e-3, -0.5]]), 64, kind)


def test_masked_tokens_and_rows_that_offer_nothing():
    rng = np.random.default_rng(4)
    x = logits_of(rng, 3, 5, 2000, "fp32")
    x[0, :, 50:] = -np.inf                       # few tokens allowed
    x[0, 1] = -np.inf                            # none
    x[0, 2, 7] = np.nan
    x[0, 3, 1999] = np.inf
    x[1, :, :] = -np.inf
    x[1, 4, 1234] = -3
    x[2, 0, 5] = 3e38                            # far from the others, not infinite
    x[2, 1, 5] = -3e38
    score = np.float32([[0, 0, 0, 0, -np.inf], [0, 0, np.nan, 0, -2], [0, 0, np.inf, -1, -1e30]])
    got = choose(x, score, 60, "fp32")
    assert (got[1][0, :50] == 0).all() and (got[1][0, 50:] == -1).all()
    assert got[0][1, 0] == -2 and got[2][1, 0] == 1234 and (got[1][1, 1:] == -1).all()
    assert set(got[1][2]) <= {0, 1, 3, 4}


@pytest.mark.parametrize("kind", ["bf16", "fp32"])
@pytest.mark.parametrize("vocab", [49999, 152064])
def test_a_nan_before_a_wave_s_first_finite_step_is_not_lost(vocab, kind):
    """Vocabularies of which a wave takes several steps.  Beams with NaN: all that a lane holds of the first
    step, the first chunk, among masked tokens alone, with the sign set, in the last step of all.  None of them offers a token."""
    rng = np.random.default_rng(vocab)
    x = logits_of(rng, 2, 6, vocab, kind)
    for s in range(2):
        x[s, 0, :8] = np.nan
        x[s, 1, 512 * s:512 * s + 512] = np.nan
        x[s, 2, :4096] = -np.inf
        x[s, 2, 77 + 1000 * s] = np.nan
        x[s, 3, :8] = -np.float32(np.nan)
        x[s, 3, 8:2048] = -np.inf
        x[s, 4, vocab - 1 - 700 * s] = np.nan
    score = np.float32([[0, 0, 0, 0, 0, -9]] * 2)
    got = choose(x, score, 12, kind)
    assert (got[1] == 5).all()


@pytest.mark.parametrize("kind", ["bf16", "fp32"])
@pytest.mark.parametrize("allowed", [0, 5])
def test_tokens_masked_by_the_lowest_value(kind, allowed):
    """Finite, so they are chosen where nothing else is left: whole rows of ties."""
    lowest = float(torch.finfo(torch.bfloat16 if kind == "bf16" else torch.float32).min)
    x = np.full((2, 3, 40000), lowest, np.float32)
    rng = np.random.default_rng(5)
    for i in range(allowed):
        x[:, :, 7000 * i + 11] = pages.bf16_value(pages.bf16_bits(rng.standard_normal((2, 3)))).astype(np.float32)
    got = H.beam_select(device_logits(x, kind), torch.tensor([[0.0, -1, -2]] * 2, device=DEV), 32)
    parent, token = got[1].cpu().numpy(), got[2].cpu().numpy()
    free = [7000 * i + 11 for i in range(allowed)]
    for s in range(2):
        best = sorted(zip(parent[s, :3 * allowed], token[s, :3 * allowed]))
        assert best == [(b, t) for b in range(3) for t in free]
        # (a value of that size is the same for all tokens of the lowest logit, of every beam)
        rest = [t for t in range(40) if t not in free][:32 - 3 * allowed]
        assert (parent[s, 3 * allowed:] == 0).all() and token[s, 3 * allowed:].tolist() == rest


def test_rows_that_lie_gibibytes_apart():
    stride = 2 ** 30 + 24
    room = torch.empty(3 * stride + 1000, dtype=torch.bfloat16, device=DEV)
    rows = room.as_strided((2, 2, 1000), (2 * stride, stride, 1))
    x = logits_of(np.random.default_rng(6), 2, 2, 1000, "bf16")
    rows.copy_(torch.from_numpy(x).to(DEV))
    got = [t.cpu().numpy() for t in H.beam_select(rows, torch.zeros(2, 2, device=DEV), 5)]
    check_choice(x, np.zeros((2, 2), np.float32), None, 5, -1, 0, got)


@pytest.mark.parametrize("kind", ["bf16", "fp32"])
@pytest.mark.parametrize("seqs,beams,vocab,keep", [(2, 16, 500, 32), (1, 5, 512, 64), (3, 16, 150, 32), (1, 63, 300, 64), (2, 33, 512, 64),
                                                   (1, 16, 1000, 64), (2, 7, 541, 14), (4, 16, 997, 32), (5, 14, 543, 28),
                                                   (3, 1, 288, 2), (2, 3, 278, 6), (1, 6, 873, 12)])
def test_choices_of_more_than_there_are_chunks(seqs, beams, vocab, keep, kind):
    rng = np.random.default_rng(beams + vocab)
    x = logits_of(rng, seqs, beams, vocab, kind)
    score = -rng.random((seqs, beams)).astype(np.float32)
    done = (rng.random((seqs, beams)) < 0.3).astype(np.int32)
    choose(x, score, keep, kind)
    choose(x, score, keep, kind, done=done, end=2, pad_token=2)
    x[:, 1:, 4:] = -np.inf                          # most threads have nothing
    x[:, 0, :vocab // 2] = -np.inf
    choose(x, score, keep, kind, done=done, end=2, pad_token=2)
    x[:] = 0                                        # all alike
    choose(x, np.zeros_like(score), keep, kind)
    x[:, beams // 2] = np.nan
    choose(x, np.zeros_like(score), keep, kind)


def test_choices_of_few_tokens_leave_no_rest():
    got = choose(np.float32([[[1, 2, 3], [3, 2, 1]]]), np.zeros((1, 2), np.float32), 9, "fp32", end=0)
    assert got[1][0].tolist() == [0, 1, 0, 1, 0, 1, -1, -1, -1] and got[2][0].tolist() == [2, 0, 1, 1, 0, 2, -1, -1, -1]
    assert got[3][0].tolist() == [0, 1, 0, 0, 1, 0, 0, 0, 0]


def test_scores_of_steep_and_flat_rows():
    """ln sum exp where a peak comes late, where two values are all that a row holds, and where it rises slowly."""
    for kind in ("bf16", "fp32"):
        x = np.zeros((1, 2, 131072), np.float32)
        x[0, 0, ::2] = -5
        x[0, 0, 70000] = 6
        x[0, 1] = np.linspace(-20, 0, 131072)
        if kind == "bf16":
            x = pages.bf16_value(pages.bf16_bits(x)).astype(np.float32)
        dev_x, score = device_logits(x, kind), torch.zeros(1, 2, device=DEV)
        got = H.beam_select(dev_x, score, 64)
        for b in range(2):
            row = x[0, b].astype(np.float64)
            lse = row.max() + np.log(np.exp(row - row.max()).sum())
            mine = (got[1][0] == b).nonzero()[:, 0]
            for i in mine.tolist():
                # rounded once to fp32: half a step of it
                true = row[int(got[2][0, i])] - lse
                assert abs(float(got[0][0, i]) - true) <= 2.0 ** -24 * abs(true) + DOUBT


@pytest.mark.parametrize("n,parts,bound", [(2 ** 17, 64, DOUBT), (2 ** 20, 64, DOUBT), (2 ** 25, 64, 1.5e-6), (2 ** 25 + 77, 1, 1.5e-6)])
def test_scores_of_two_values_whose_differences_round(n, parts, bound):
    """ln sum exp of rows of a few peaks (the first token of every part) and one other value, so far below that its
    difference to the peak and that one's octaves round, alike for all: nothing averages it out.  A term t below is off by half an ulp
    of t, half an ulp of t log2 e times ln 2, an ulp of the exponential and three additions:
      4 to 8      2^-22 + 2^-21 ln 2 + 2^-23 + 3 x 2^-24 = 8.7e-7
      8 to 11     2^-21 + 2^-21 ln 2 + ..                = 1.11e-6
      11.1 to 16  2^-21 + 2^-20 ln 2 + ..                = 1.44e-6
      16 to 22.2  2^-20 + 2^-20 ln 2 + ..                = 1.92e-6
    of its share, T e^-t / (1 + T e^-t) of a peak and T others.  A wave takes T tokens, and has a greatest of its own: T is
    2^14 for 2^20 tokens (at 8 a share of 0.85: 9.4e-7; at 11.1 of 0.2) and 2^24 for the most that there may be (at 11.1 of
    1: 1.44e-6; at 16 of 0.66: 1.26e-6).  The score is chosen so that the value is close to 0, and its rounding far below that."""
    rng = np.random.default_rng(n)
    rows, share = 4, -(-n // parts)
    peak = rng.uniform(0, 6, 100000).astype(np.float32)
    x = (peak - rng.uniform(4, 20, len(peak))).astype(np.float32)
    far = x.astype(np.float64) - peak
    octaves = ((x - peak).astype(np.float64) * 1.4426950408889634).astype(np.float32)
    weight = share * np.exp(far) / (1 + share * np.exp(far))
    off = (octaves * np.log(2) - far) * weight                # of the subtraction and the argument alone
    pick = np.concatenate([np.argsort(off)[:rows // 2], np.argsort(-off)[:rows // 2]])
    peak, x = peak[pick], x[pick]
    logits = torch.from_numpy(x).to(DEV)[:, None].repeat(1, n)
    logits[:, ::share] = torch.from_numpy(peak).to(DEV)[:, None]
    p = peak.astype(np.float64)
    lse = p + np.log(parts + (n - parts) * np.exp(x - p))
    score = (lse - p).astype(np.float32)
    got = H.beam_select(logits.view(rows, 1, n), torch.from_numpy(score).to(DEV).view(rows, 1), 1)
    assert (got[2] == 0).all()
    value = got[0].cpu().numpy()[:, 0].astype(np.float64)
    assert (np.abs(value - ((score - lse) + p)) <= bound).all()


def test_strides_that_are_no_rows_are_refused():
    x = torch.zeros(2, 3, 100, device=DEV)
    score = torch.zeros(2, 3, device=DEV)
    H.beam_select(x[:, :, :50], score, 2)
    for bad in (x.transpose(0, 1)[:, :2].expand(3, 2, 100).transpose(0, 1)[:, [2, 0, 1]][:, :, ::2], x[..., ::2],
                torch.zeros(4, 3, 100, device=DEV)[::2]):
        with pytest.raises(ValueError):
            H.beam_select(bad, score, 2)
    with pytest.raises(ValueError):
        H.beam_select(x, score.double(), 2)
    with pytest.raises(ValueError):
        H.beam_select(x, score, 2, done=score)
    with pytest.raises(H.HermesError):
        H.beam_select(x, score, 65)
    with pytest.raises(H.HermesError):
        H.beam_select(torch.zeros(1, 1, 100, device=DEV).expand(2, 3, 100), score, 2)


# --------------------------------------------------------------------- reorder
@pytest.mark.parametrize("layers,seqs,beams,most,size,grow,heads,d,page,fmt,bad", [
    (0, 1, 1, 1, 3, 1, 1, 64, 16, "fp4", False),
    (1, 1, 4, 9, 60, 1, 2, 64, 64, "fp4", False),
    (3, 2, 5, 7, 50, 1, 2, 128, 16, "bf16", False),
    (28, 4, 4, 40, 200, 1, 4, 128, 32, "fp4", False),
    (2, 3, 64, 6, 500, 33, 1, 64, 16, "bf16", False),
    (1, 2, 3, 300, 5000, 700, 1, 64, 16, "fp4", False),
    (0, 300, 8, 4, 20, 1, 1, 128, 128, "fp4", False),
    (2, 2, 8, 3, 70, 300, 1, 64, 256, "bf16", False),
    (5, 3, 6, 8, 60, 20, 1, 64, 16, "fp4", True),
])
def test_reordered_tables_and_pages_are_the_definition_s(layers, seqs, beams, most, size, grow, heads, d, page, fmt, bad):
    rng = np.random.default_rng(layers * 10 + beams)
    groups = max(layers, 1) * seqs
    n_pages, room, tables, kv_len, parent = beams_of(rng, groups, seqs, beams, most, page, size, bad)
    memory = rng.integers(0, 255, (n_pages, heads * pages.block_bytes(d, page, fmt))).astype(np.uint8)
    lead = (layers, seqs) if layers else (seqs,)
    pool = H.KVPages(heads, heads, d, n_pages, page_rows=page, fmt=H.PAGE_FP4 if fmt == "fp4" else H.PAGE_BF16,
                     pages=torch.from_numpy(memory.copy()).to(DEV))
    got, lens = pool.reorder(i32(tables.reshape(lead + (beams, most))), i32(kv_len.reshape(lead + (beams,))), i32(parent),
                             i32(room.reshape(lead + (2,))), grow=grow)
    assert got.shape == lead + (beams, most) and lens.shape == lead + (beams,)
    got, lens = got.cpu().numpy().reshape(tables.shape), lens.cpu().numpy().reshape(kv_len.shape)
    bits = 0
    for g in range(groups):
        want, n, copies, b = orc.reorder(tables[g], kv_len[g], parent[g % seqs], room[g], grow, page, n_pages)
        assert (got[g] == want).all() and (lens[g] == n).all(), f"group {g}"
        for c in copies:
            orc.copy_rows(memory, heads, d, page, fmt, *c)
        bits |= b
    assert pool.faults() == bits
    if not bad:
        assert (pool.pages.cpu().numpy() == memory).all()


def test_a_shared_prompt_is_forked_without_writing_to_it():
    """All beams begin with one prompt outside their room: each gets a copy of its last page."""
    rng = np.random.default_rng(9)
    memory = rng.integers(0, 255, (12, 2 * pages.block_bytes(64, 16, "fp4"))).astype(np.uint8)
    pool = H.KVPages(2, 2, 64, 12, page_rows=16, pages=torch.from_numpy(memory.copy()).to(DEV))
    tables = i32([[[3, 1, 2, -1]] * 4])
    out, lens = pool.reorder(tables, i32([[38] * 4]), i32([[0] * 4]), i32([[6, 6]]))
    assert out.tolist() == [[[3, 1, x, -1] for x in (6, 7, 8, 9)]] and lens.tolist() == [[38] * 4] and pool.faults() == 0
    for t in (6, 7, 8, 9):
        orc.copy_rows(memory, 2, 64, 16, "fp4", 2, t, 8)
    assert (pool.pages.cpu().numpy() == memory).all()


def test_pages_past_4_gib_are_copied():
    n_pages = 2 ** 32 // (4 * pages.block_bytes(128, 64, "fp4")) + 40
    pool = H.KVPages(4, 4, 128, n_pages, page_rows=64)
    pool.pages[-30:] = torch.randint(0, 255, (30, pool.page_bytes), dtype=torch.uint8, device=DEV)
    memory = pool.pages[-30:].cpu().numpy()
    first = n_pages - 30
    out, _ = pool.reorder(i32([[[first + 3], [first + 4]]]), i32([[50, 41]]), i32([[1, 1]]), i32([[first, 20]]))
    assert out.tolist() == [[[first + 4], [first]]] and pool.faults() == 0
    orc.copy_rows(memory, 4, 128, 64, "fp4", 4, 0, 44)
    assert (pool.pages[-30:].cpu().numpy() == memory).all()


def test_reorder_refuses_other_tensors():
    pool = H.KVPages(2, 2, 64, 12, page_rows=16)
    t, n, p, r = i32(np.zeros((2, 3, 4))), i32(np.zeros((2, 3))), i32(np.zeros((2, 3))), i32(np.zeros((2, 2)))
    pool.reorder(t, n, p, r)
    for args in ((t[0], n, p, r), (t, n[:1], p, r), (t, n, p[:1], r), (t, n, p, r[:1]), (t.long(), n, p, r), (t, n.cpu(), p, r),
                 (t.transpose(0, 1).contiguous().transpose(0, 1), n, p, r)):
        with pytest.raises(ValueError):
            pool.reorder(*args)
    with pytest.raises(H.HermesError):
        pool.reorder(t, n, p, r, tables_out=t)
    with pytest.raises(H.HermesError):
        pool.reorder(t, n, p, r, grow=-1)


def test_numbers_past_32_bits_are_refused():
    """(their low halves are those of good calls)"""
    far = 2 ** 32
    logits, score = torch.zeros(1, 2, 100, device=DEV), torch.zeros(1, 2, device=DEV)
    pool = H.KVPages(2, 2, 64, 12, page_rows=16)
    t, n, p, r = i32(np.zeros((2, 3, 4))), i32(np.zeros((2, 3))), i32(np.zeros((2, 3))), i32([[0, 3], [3, 3]])
    w = H.PackedWeight(bf16(weight_bits(1, 8, 1)))
    row = torch.zeros(1, 8, dtype=torch.bfloat16, device=DEV)
    long = torch.empty(far + 16, dtype=torch.bfloat16, device=DEV)
    for call in (lambda: H.beam_select(logits, score, 2, end_token=far + 5), lambda: H.beam_select(logits, score, 2, end_token=-far + 5),
                 lambda: H.beam_select(logits, score, 2, pad_token=far + 5), lambda: H.beam_select(logits, score, far + 2),
                 lambda: H.beam_select(long.view(1, 1, -1), score[:, :1].contiguous(), 2),
                 lambda: H.PackedWeight(long.view(-1, 1)), lambda: w.product(row.expand(far + 1, 8)),
                 lambda: pool.reorder(t, n, p, r, grow=far + 1), lambda: pool.reorder(t, n, p, r, grow=1 - far)):
        with pytest.raises(H.HermesError):
            call()


# --------------------------------------------------------------- as they are used
class Model:
    """Two layers of one head group, products in 4 bits, and beams over their pages."""
    HQ, HKV, D, E, V, L, PAGE = 4, 2, 64, 256, 1000, 2, 16

    def __init__(self, seqs, beams, fmt, steps, prompt=21, seed=0):
        g = torch.Generator(device=DEV).manual_seed(seed)
        rand = lambda *s, scale=1.0: (torch.randn(s, generator=g, device=DEV) * scale).to(torch.bfloat16)
        self.seqs, self.beams, self.n = seqs, beams, seqs * beams
        self.embed = rand(self.V, self.E)
        width = (self.HQ + 2 * self.HKV) * self.D
        self.qkv = [H.PackedWeight(rand(width, self.E, scale=0.08)) for _ in range(self.L)]
        self.bias = [rand(width, scale=0.3) for _ in range(self.L)]
        self.proj = [H.PackedWeight(rand(self.E, self.HQ * self.D, scale=0.08)) for _ in range(self.L)]
        self.head = H.PackedWeight(rand(self.V, self.E, scale=0.1))
        most = -(-(prompt + steps + 1) // self.PAGE)
        groups = self.L * seqs
        shared = most                                       # the prompt's pages, a layer's after the other's
        room = beams * (most + 2)
        self.n_pages = self.L * shared + groups * room
        self.pool = H.KVPages(self.HQ, self.HKV, self.D, self.n_pages, page_rows=self.PAGE,
                              fmt=H.PAGE_FP4 if fmt == "fp4" else H.PAGE_BF16)
        tables = np.full((self.L, seqs, beams, most), -1, np.int32)
        have = -(-prompt // self.PAGE)
        for i in range(self.L):
            tables[i, :, :, :have] = i * shared + np.arange(have)
        at = self.L * shared + room * np.arange(groups).reshape(self.L, seqs)
        self.room = i32(np.stack([at, np.full_like(at, room)], -1))
        self.tables, self.kv_len = i32(tables), i32(np.full((self.L, seqs, beams), prompt))
        # a prompt in every layer's pages
        for i in range(self.L):
            k, v = rand(prompt, self.HKV, self.D), rand(prompt, self.HKV, self.D)
            b = H.PageBatch(i32(tables[i, :1, 0]), i32([prompt]), row_start=i32([0, prompt]), n_rows=prompt)
            self.pool.append(b, k, v, rope=torch.arange(prompt, dtype=torch.int32, device=DEV))

    def token(self, ids, tables, kv_len):
        """Logits of one token a beam, whose pages have room for it; kv_len counts it."""
        x = self.embed[ids.long().reshape(-1)]
        rope = (kv_len[0].reshape(-1) - 1).to(torch.int32)
        for i in range(self.L):
            y = self.qkv[i].product(x, bias=self.bias[i])
            q, k, v = (t.unflatten(1, (-1, self.D)) for t in y.split([self.HQ * self.D, self.HKV * self.D, self.HKV * self.D], 1))
            batch = H.PageBatch(tables[i].flatten(0, 1), kv_len[i].reshape(-1))
            q = self.pool.append(batch, k, v, q=q, rope=rope)
            x = self.proj[i].product(self.pool.attend(batch, q).flatten(1), add=x)
        return self.head.product(x, dtype=torch.float32).unflatten(0, (self.seqs, self.beams))


def generate(model, steps, step):
    """Beams over `steps` tokens; step(ids, score, done, tables, kv_len) -> the next of all, the parents."""
    ids = torch.arange(model.n, dtype=torch.int32, device=DEV).view(model.seqs, model.beams)
    score = torch.zeros(model.seqs, model.beams, device=DEV)
    done = torch.zeros(model.seqs, model.beams, dtype=torch.int32, device=DEV)
    first = torch.arange(model.beams, dtype=torch.int32, device=DEV).expand(model.seqs, -1).contiguous()
    tables, kv_len = model.pool.reorder(model.tables, model.kv_len, first, model.room)
    history = ids.unsqueeze(-1).cpu()
    for _ in range(steps):
        ids, score, done, tables, kv_len, parent = step(ids, score, done, tables, kv_len)
        history = torch.cat([history.gather(1, parent.cpu().long().unsqueeze(-1).expand(-1, -1, history.shape[-1])),
                             ids.cpu().unsqueeze(-1)], -1)
    return history, score, tables, kv_len


@pytest.mark.parametrize("fmt", ["fp4", "bf16"])
@pytest.mark.parametrize("seqs,beams", [(1, 1), (2, 3), (1, 8)])
def test_beams_hold_what_their_own_tokens_alone_would_have_stored(seqs, beams, fmt):
    """Beam search over projections, pages, logits, choices and reorders; then every final beam's
    tokens again, in pages of its own that are never reordered: the rows in its pages
    and its last logits are the same bit for bit, and its score is the sum of theirs."""
    steps = 40
    m = Model(seqs, beams, fmt, steps)

    def step(ids, score, done, tables, kv_len):
        kv_len = kv_len + 1
        logits = m.token(ids, tables, kv_len)
        score, parent, ids, done = H.beam_select(logits, score, beams, done=done)
        tables, kv_len = m.pool.reorder(tables, kv_len, parent, m.room)
        step.logits, step.parent = logits, parent
        return ids, score, done, tables, kv_len, parent

    history, score, tables, kv_len = generate(m, steps, step)
    assert m.pool.faults() == 0
    alone = Model(seqs, beams, fmt, steps)
    first = torch.arange(beams, dtype=torch.int32, device=DEV).expand(seqs, -1).contiguous()
    own, lens = alone.pool.reorder(alone.tables, alone.kv_len, first, alone.room, grow=steps)
    total = torch.zeros(seqs, beams, dtype=torch.float64)
    for t in range(steps):
        lens = lens + 1
        logits = alone.token(history[..., t].to(DEV), own, lens)
        x = logits.double().cpu()
        total += (x - x.logsumexp(-1, keepdim=True)).gather(-1, history[..., t + 1:t + 2].long())[..., 0]
    assert torch.equal(logits, step.logits.gather(1, step.parent.long().unsqueeze(-1).expand(-1, -1, m.V)))
    assert torch.equal(lens, kv_len)
    for i in range(m.L):
        n = int(lens[0, 0, 0])
        rows = []
        for pool, tab in ((m.pool, tables), (alone.pool, own)):
            start = torch.arange(0, n * m.n + 1, n, dtype=torch.int32, device=DEV)
            rows.append(pool.read(H.PageBatch(tab[i].flatten(0, 1), lens[i].reshape(-1), start, n_rows=n * m.n)))
        assert torch.equal(rows[0][0], rows[1][0]) and torch.equal(rows[0][1], rows[1][1])
    # a score is rounded to fp32 at each step
    bound = steps * (2.0 ** -24 * float(total.abs().max()) + DOUBT)
    assert (total - score.double().cpu()).abs().max() <= bound


def test_a_captured_step_replays_as_the_eager_one():
    seqs, beams, steps = 2, 4, 24
    runs = []
    for captured in (False, True):
        m = Model(seqs, beams, "fp4", steps, seed=3)
        ids = torch.arange(m.n, dtype=torch.int32, device=DEV).view(seqs, beams)
        score = torch.zeros(seqs, beams, device=DEV)
        done = torch.zeros(seqs, beams, dtype=torch.int32, device=DEV)
        first = torch.arange(beams, dtype=torch.int32, device=DEV).expand(seqs, -1).contiguous()
        tables, kv_len = m.pool.reorder(m.tables, m.kv_len, first, m.room)
        start = [t.clone() for t in (ids, score, done, tables, kv_len)]
        state = [t.clone() for t in start]
        parent = torch.zeros_like(ids)

        def step():
            ids, score, done, tables, kv_len = state
            grown = kv_len + 1
            new = H.beam_select(m.token(ids, tables, grown), score, beams, done=done, end_token=17, pad_token=17)
            t, n = m.pool.reorder(tables, grown, new[1], m.room)
            parent.copy_(new[1])
            for old, x in zip(state, (new[2], new[0], new[3], t, n)):
                old.copy_(x)

        graph = None
        if captured:
            side = torch.cuda.Stream()
            side.wait_stream(torch.cuda.current_stream())
            with torch.cuda.stream(side):
                step()
            torch.cuda.current_stream().wait_stream(side)
            for old, x in zip(state, start):
                old.copy_(x)
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph):
                step()
        seen = []
        for i in range(steps):
            graph.replay() if captured else step()
            if i % 5 == 0:
                torch.cuda.synchronize()
                (torch.ones(1000, device=DEV) * i).sum()          # (other work between replays)
            seen.append([t.clone() for t in state] + [parent.clone()])
        assert m.pool.faults() == 0
        runs.append(seen)
    for a, b in zip(*runs):
        assert all(torch.equal(x, y) for x, y in zip(a, b))


def test_calls_on_two_streams_at_once():
    """Two streams, each with inputs of its own made there: the results of one after the other."""
    def work(seed):
        g = torch.Generator(device=DEV).manual_seed(seed)
        w = H.PackedWeight((torch.randn(1000, 512, generator=g, device=DEV) * 0.1).to(torch.bfloat16))
        x = torch.randn(8, 512, generator=g, device=DEV).to(torch.bfloat16)
        out = []
        for _ in range(20):
            logits = w.product(x, dtype=torch.float32).view(2, 4, 1000)
            out.append(H.beam_select(logits, torch.zeros(2, 4, device=DEV), 8))
        return out
    want = [work(s) for s in (1, 2)]
    torch.cuda.synchronize()
    streams, got = [torch.cuda.Stream(), torch.cuda.Stream()], []
    for s, stream in zip((1, 2), streams):
        with torch.cuda.stream(stream):
            got.append(work(s))
    torch.cuda.synchronize()
    for a, b in zip(want, got):
        for x, y in zip(a, b):
            assert all(torch.equal(p, q) for p, q in zip(x, y))


@pytest.mark.parametrize("captured", [False, True])
def test_calls_in_turn_on_two_streams_that_overlap(captured):
    """Products whose inputs workgroups share (through a workspace), choices and reorders, issued in turn on two streams
    that both wait until all is issued; then as two graphs replayed at once, three times."""
    n, k, m, steps = 1000, 14336, 64, 12
    assert H.lib.hermes_weight_workspace_bytes(ctypes.byref(H.WeightStruct(n, k, None)), m) > 0
    sides = []
    for seed in (1, 2):
        x, w = whole_numbers(m, n, k, DEV, seed)
        rng = np.random.default_rng(seed)
        n_pages, room, tables, kv_len, parent = beams_of(rng, 6, 3, 4, 5, 16, 40, False)
        memory = torch.from_numpy(rng.integers(0, 255, (n_pages, 2 * pages.block_bytes(64, 16, "fp4"))).astype(np.uint8)).to(DEV)
        sides.append(dict(w=H.PackedWeight(w.to(torch.bfloat16)), x=x.to(torch.bfloat16), want=torch.mm(x, w.T.contiguous()).float(),
                          score=torch.zeros(8, 8, device=DEV), memory=memory,
                          pool=H.KVPages(2, 2, 64, n_pages, page_rows=16, pages=memory.clone()),
                          reorder=[i32(t) for t in (tables.reshape(2, 3, 4, 5), kv_len.reshape(2, 3, 4), parent, room.reshape(2, 3, 2))]))

    def step(s):
        logits = s["w"].product(s["x"], dtype=torch.float32)
        return logits, *H.beam_select(logits.view(8, 8, n), s["score"], 16), *s["pool"].reorder(*s["reorder"]), s["pool"].pages.clone()
    for s in sides:
        s["alone"] = step(s)
        assert torch.equal(s["alone"][0], s["want"])
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    got = [[], []]
    if captured:
        graphs = []
        for s, side, out in zip(sides, streams, got):
            graphs.append(torch.cuda.CUDAGraph())
            with torch.cuda.graph(graphs[-1], stream=side):
                out.extend(step(s) for _ in range(steps))
    for again in range(3 if captured else 1):
        for s in sides:
            s["pool"].pages.copy_(s["memory"])
        torch.cuda.synchronize()
        for side in streams:
            with torch.cuda.stream(side):
                torch.cuda._sleep(20_000_000)
        if captured:
            for side, graph in zip(streams, graphs):
                with torch.cuda.stream(side):
                    graph.replay()
        else:
            for _ in range(steps):
                for s, side, out in zip(sides, streams, got):
                    with torch.cuda.stream(side):
                        out.append(step(s))
        torch.cuda.synchronize()
        for s, out in zip(sides, got):
            assert len(out) == steps and s["pool"].faults() == 0
            for results in out:
                assert all(torch.equal(a, b) for a, b in zip(results, s["alone"]))
