"""Which memory the pages' kernels touch: their sources compiled for the host
(tests/cpu_waves), in memory that ends where their inputs end."""
import os
import subprocess

import pytest

from paper_2601_14724_amd import build
from paper_2601_14724_amd import hermes as H

HERE = os.path.join(os.path.dirname(os.path.abspath(__file__)), "cpu_waves")
CLANG = os.path.join(os.path.dirname(os.path.realpath(build.HIPCC)), "..", "llvm", "bin", "clang++")


def compiled(tmp_path_factory, name, *options):
    exe = str(tmp_path_factory.mktemp("cpu_waves") / name)
    subprocess.run([CLANG, "-std=c++20", "-w", "-pthread", "-D__HIP__", f"-I{HERE}", f"-I{build.CSRC}",
                    f"-I{build.INCLUDE}", *options, os.path.join(HERE, name + ".cpp"), "-o", exe], check=True, timeout=120)
    return exe


@pytest.fixture(scope="module")
def append_rows(tmp_path_factory):
    return compiled(tmp_path_factory, "append_rows")


@pytest.mark.parametrize("share", [1, 4])
@pytest.mark.parametrize("axes", [1, 3])
@pytest.mark.parametrize("first", [0, 16])
@pytest.mark.parametrize("seqs", [3, 64, 130])      # starts held by the lanes, and searched in memory
def test_append_reads_only_rows_of_sequences(append_rows, seqs, first, axes, share):
    res = subprocess.run([append_rows, str(seqs), str(first), str(axes), str(share)], capture_output=True, text=True,
                         timeout=60)
    assert res.returncode == 0 and res.stdout == "done\n"


@pytest.fixture(scope="module")
def walk_items(tmp_path_factory):
    return compiled(tmp_path_factory, "walk_items")


@pytest.mark.parametrize("seqs,rows,heads,length,ends", [
    (70, 512, 16, 5000, 128),
    (130, 37, 7, 900, 128),
    (32768, 512, 1024, 2 ** 25 - 768, 1),   # taken as they are, the starts ask for a cost of 2^64 + 2^32
])
def test_starts_that_fall_stay_in_bounds(walk_items, seqs, rows, heads, length, ends):
    res = subprocess.run([walk_items] + [str(x) for x in (seqs, rows, heads, length, ends)], capture_output=True, text=True,
                         timeout=100)
    assert res.returncode == 0 and res.stdout == f"in bounds, status {H.PAGE_BAD_ROWS}\n"


def test_plans_of_any_size_are_counted_without_overflow(tmp_path_factory):
    exe = compiled(tmp_path_factory, "plans", "-O1", "-fsanitize=signed-integer-overflow,float-cast-overflow",
                   "-fno-sanitize-recover=all")
    res = subprocess.run([exe], capture_output=True, text=True, timeout=100)
    assert res.returncode == 0 and res.stdout == "good, many taken\n", res.stderr
