"""Which memory the pages' kernels touch: their sources compiled for the host
(tests/cpu_waves), in memory that ends where their inputs end."""
import os
import subprocess

import pytest

from paper_2601_14724_amd import build

HERE = os.path.join(os.path.dirname(os.path.abspath(__file__)), "cpu_waves")
CLANG = os.path.join(os.path.dirname(os.path.realpath(build.HIPCC)), "..", "llvm", "bin", "clang++")


def compiled(tmp_path_factory, name):
    exe = str(tmp_path_factory.mktemp("cpu_waves") / name)
    subprocess.run([CLANG, "-std=c++20", "-O1", "-w", "-pthread", "-D__HIP__", f"-I{HERE}", f"-I{build.CSRC}",
                    f"-I{build.INCLUDE}", os.path.join(HERE, name + ".cpp"), "-o", exe], check=True, timeout=120)
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
