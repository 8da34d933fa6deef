"""Kernels around a generated token on the CPU (tests/cpu_waves): which memory they touch,
and, where no matrix instruction is involved, what they give, also of tables, lengths,
parents and rooms that do not fit."""
import subprocess

import numpy as np
import pytest

from oracle import pages_oracle as pages
from oracle import tokens_oracle as orc
from tests.test_pages_bounds import compiled


def run(exe, args, *arrays):
    res = subprocess.run([exe] + [str(int(x)) for x in args], input=b"".join(np.ascontiguousarray(x).tobytes() for x in arrays),
                         capture_output=True, timeout=100)
    assert res.returncode == 0, res.stderr[-500:]
    return res.stdout


def cut(data, *shapes):
    out = []
    for dtype, shape in shapes:
        n = int(np.prod(shape)) * np.dtype(dtype).itemsize
        out.append(np.frombuffer(data[:n], dtype).reshape(shape))
        data = data[n:]
    assert not data
    return out


@pytest.fixture(scope="module")
def reorder(tmp_path_factory):
    return compiled(tmp_path_factory, "reorder", "-O1")


def beams_of(rng, groups, seqs, beams, most, page, size, bad):
    """Tables whose entries lie in the group's room or outside, lengths, parents, rooms."""
    n_pages = 5 + groups * size
    room = np.stack([5 + size * np.arange(groups), np.full(groups, size)], 1).astype(np.int32)
    tables = np.where(rng.random((groups, beams, most)) < 0.6,
                      room[:, :1, None] + rng.integers(0, size, (groups, beams, most)),
                      rng.integers(0, 5, (groups, beams, most))).astype(np.int32)
    kv_len = rng.integers(0, most * page + 1, (groups, beams)).astype(np.int32)
    parent = rng.integers(-1 if bad else 0, beams, (seqs, beams)).astype(np.int32)
    if bad:
        tables[rng.random(tables.shape) < 0.1] = n_pages + 7
        tables[rng.random(tables.shape) < 0.1] = -2 ** 31
        kv_len[rng.random(kv_len.shape) < 0.1] = -5
        kv_len[rng.random(kv_len.shape) < 0.1] = most * page + 1
        parent[rng.random(parent.shape) < 0.1] = beams
        parent[rng.random(parent.shape) < 0.1] = -2
        room[rng.random(groups) < 0.2, 0] = n_pages - 1
        room[rng.random(groups) < 0.1, 1] = -1
        room[rng.random(groups) < 0.1, 1] = 2 ** 31 - 1
    return n_pages, room, tables, kv_len, parent


@pytest.mark.parametrize("groups,seqs,beams,most,size,grow,heads,d,page,fmt,shares,bad", [
    (1, 1, 1, 1, 3, 0, 1, 64, 16, "fp4", 1, False),
    (1, 1, 1, 1, 3, 1, 1, 64, 16, "bf16", 1, False),
    (4, 2, 5, 7, 40, 1, 2, 64, 16, "fp4", 3, False),
    (2, 1, 64, 3, 70, 17, 1, 128, 16, "fp4", 2, False),       # more asked for than there is
    (3, 3, 4, 70, 300, 0, 1, 64, 32, "bf16", 1, False),
    (6, 2, 7, 5, 33, 3, 1, 64, 16, "fp4", 2, True),
    (12, 3, 3, 2, 9, 40, 2, 64, 16, "fp4", 1, True),
    (2, 2, 2, 130, 2500, 2000, 1, 64, 16, "fp4", 1, True),
])
def test_reorder_stays_in_bounds_and_gives_the_definition(reorder, groups, seqs, beams, most, size, grow, heads, d, page, fmt,
                                                          shares, bad):
    rng = np.random.default_rng(groups * 100 + beams)
    n_pages, room, tables, kv_len, parent = beams_of(rng, groups, seqs, beams, most, page, size, bad)
    block = pages.block_bytes(d, page, fmt)
    memory = rng.integers(0, 255, (n_pages, heads * block)).astype(np.uint8)
    row, scale = (2 * d, 0) if fmt == "bf16" else (d // 2, d // 32)
    out = run(reorder, (groups, seqs, beams, most, grow, page.bit_length() - 1, n_pages, heads, row, scale, shares),
              parent, room, tables, kv_len, memory)
    got, lens, after, status = cut(out, (np.int32, tables.shape), (np.int32, kv_len.shape), (np.uint8, memory.shape),
                                   (np.int32, (1,)))
    bits = 0
    for g in range(groups):
        want, n, copies, b = orc.reorder(tables[g], kv_len[g], parent[g % seqs], room[g], grow, page, n_pages)
        assert (got[g] == want).all() and (lens[g] == n).all(), f"group {g}"
        for c in copies:
            orc.copy_rows(memory, heads, d, page, fmt, *c)
        bits |= b
    assert status[0] == bits
    if not bad:                      # (bad tables may name pages of other groups' rooms)
        assert (after == memory).all()


@pytest.fixture(scope="module")
def beams(tmp_path_factory):
    return compiled(tmp_path_factory, "beams", "-O1")


# ln sum exp, term by term relative to its exponential: one ulp of the hardware's exponential (2^-23), half an
# ulp of its argument (2^-21 below 16 octaves, 2^-20 below 32: what lies further down adds less than 2^-11 of a
# row of 2^20), times ln 2, and three additions in fp32 (3 x 2^-24): 9.6e-7.
DOUBT = 1e-6


def check_choice(logits, score, done, keep, end, pad, got, doubt=DOUBT):
    """got (score, parent, token, done) [seqs][keep] of logits [seqs][beams][vocab] against the
    definition.  Where two values differ by less than `doubt` either order passes."""
    for s in range(logits.shape[0]):
        value = orc.values(logits[s], score[s], None if done is None else done[s], pad)
        want, parent, token = orc.select(value, keep)
        n = len(want)
        g_score, g_parent, g_token, g_done = (x[s] for x in got)
        assert (g_parent[n:] == -1).all() and (g_token[n:] == -1).all() and np.isneginf(g_score[n:]).all()
        assert (g_done[n:] == 0).all()
        mine = value[g_parent[:n], g_token[:n]]
        assert (np.abs(mine - want) <= doubt).all()
        # a score is a value rounded once
        assert (np.abs(g_score[:n].astype(np.float64) - mine) <= doubt + 2.0 ** -24 * np.abs(mine)).all()
        assert len({*zip(g_parent[:n].tolist(), g_token[:n].tolist())}) == n
        flat = np.sort(value.reshape(-1))[::-1][:keep + 1]
        flat = flat[flat > -np.inf]
        gap = np.abs(np.diff(flat))
        if not ((gap > 0) & (gap < doubt)).any():          # (equal ones have their order)
            assert (g_parent[:n] == parent).all() and (g_token[:n] == token).all()
        ended = g_token[:n] == end
        if done is not None:
            ended = ended | (done[s][g_parent[:n]] != 0)
        assert (g_done[:n] == ended).all()


@pytest.mark.parametrize("seqs,n_beams,vocab,keep,fp32,pad,with_done,per", [
    (1, 1, 1, 1, False, 0, False, 1),
    (2, 3, 513, 7, False, 1, True, 1),
    (1, 2, 1500, 64, True, 3, False, 2),
    (2, 2, 40, 64, True, 0, True, 1),
    (1, 6, 500, 64, False, 0, True, 1),        # fewer chunks than choices, more tokens than the list holds
    (2, 16, 260, 32, True, 5, False, 1),
])
def test_beam_select_stays_in_bounds_and_gives_the_definition(beams, seqs, n_beams, vocab, keep, fp32, pad, with_done, per):
    rng = np.random.default_rng(vocab)
    x = (3 * rng.standard_normal((seqs * n_beams, vocab))).astype(np.float32)
    if not fp32:
        x = pages.bf16_value(pages.bf16_bits(x)).astype(np.float32)
    x[rng.random(x.shape) < 0.05] = -np.inf
    score = -rng.random((seqs, n_beams)).astype(np.float32)
    done = (rng.random((seqs, n_beams)) < 0.4).astype(np.int32) if with_done else None
    stride = vocab + pad
    rows = np.full((seqs * n_beams, stride), np.nan, np.float32)
    rows[:, :vocab] = x
    rows = rows.reshape(-1)[:(seqs * n_beams - 1) * stride + vocab]
    end, end_pad = (2, 2) if vocab > 2 else (0, 0)
    out = run(beams, (seqs, n_beams, vocab, keep, fp32, stride, end, end_pad, with_done, per),
              rows if fp32 else pages.bf16_bits(rows), score, *([done] if with_done else []))
    k = (seqs, keep)
    got = cut(out, (np.float32, k), (np.int32, k), (np.int32, k), (np.int32, k))
    check_choice(x.reshape(seqs, n_beams, vocab), score, done, keep, end, end_pad, got)


def _nan_rows(n_beams, vocab, where):
    """Logits of one sequence, whose first beam has a NaN in the first steps of a wave."""
    x = (3 * np.random.default_rng(vocab).standard_normal((n_beams, vocab))).astype(np.float32)
    if where == "eight":                     # all that a lane holds
        x[0, :8] = np.nan
    elif where == "chunk":
        x[0, :512] = np.nan
    elif where == "masked":                  # beside masked tokens alone
        x[0, :2048] = -np.inf
        x[0, 77] = np.nan
    else:                                    # a NaN with the sign set, which orders below all
        x[0, :8] = -np.float32(np.nan)
        x[0, 8:512] = -np.inf
    return x


@pytest.mark.parametrize("where", ["eight", "chunk", "masked", "negative"])
@pytest.mark.parametrize("vocab,per", [(1500, 2), (2300, 5), (4196, 8), (6000, 16)])
@pytest.mark.parametrize("fp32", [True, False])
def test_a_nan_in_a_wave_s_first_steps_is_not_lost(beams, vocab, per, fp32, where):
    """A beam one of whose logits is NaN offers nothing, whatever follows it."""
    x = _nan_rows(2, vocab, where)
    if not fp32:
        x = pages.bf16_value(pages.bf16_bits(x)).astype(np.float32)
    assert np.isnan(x[0]).any()
    score = np.float32([[0, -5]])
    out = run(beams, (1, 2, vocab, 4, fp32, vocab, 2, 2, False, per), x if fp32 else pages.bf16_bits(x), score)
    got = cut(out, (np.float32, (1, 4)), (np.int32, (1, 4)), (np.int32, (1, 4)), (np.int32, (1, 4)))
    assert got[1].tolist() == [[1] * 4]
    check_choice(x[None], score, None, 4, 2, 2, got)


@pytest.fixture(scope="module")
def weights(tmp_path_factory):
    return compiled(tmp_path_factory, "weights", "-O1")


@pytest.mark.parametrize("n,k,m,row_quads,tiles,bias,add,fp32", [
    (1, 1, 9, 4, 1, 0, 0, 0),
    (70, 515, 16, 4, 1, 1, 1, 0),
    (150, 1290, 13, 4, 2, 0, 1, 1),
    (257, 256, 12, 4, 4, 0, 0, 0),
    (65, 1153, 17, 8, 1, 1, 0, 1),
    (129, 383, 32, 8, 2, 0, 1, 0),
    (300, 130, 31, 8, 4, 1, 0, 0),
    (65, 641, 33, 16, 1, 1, 1, 0),
    (100, 7, 64, 16, 2, 0, 1, 1),
    (258, 385, 70, 16, 4, 1, 0, 0),
])
def test_products_of_shared_rows_stay_in_bounds(weights, n, k, m, row_quads, tiles, bias, add, fp32):
    assert run(weights, (n, k, m, row_quads, tiles, 1, bias, add, fp32, 1, 1)) == b"done\n"


@pytest.mark.parametrize("n,k,m,row_quads,tiles,split,bias,add,fp32,parts", [
    (1, 1, 1, 1, 1, 1, 0, 0, 0, 1),
    (17, 129, 3, 1, 1, 8, 1, 1, 1, 1),
    (40, 1300, 7, 2, 2, 4, 0, 1, 0, 1),
    (100, 515, 13, 4, 4, 2, 1, 0, 0, 1),
    (33, 640, 17, 8, 2, 1, 1, 0, 1, 1),
    (70, 1025, 65, 16, 1, 4, 0, 1, 0, 1),
    (70, 1025, 65, 16, 4, 4, 1, 1, 0, 2),
    (35, 1290, 20, 8, 2, 2, 0, 1, 1, 5),
])
def test_products_stay_in_bounds(weights, n, k, m, row_quads, tiles, split, bias, add, fp32, parts):
    assert run(weights, (n, k, m, row_quads, tiles, split, bias, add, fp32, parts, 0)) == b"done\n"
