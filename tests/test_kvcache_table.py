"""Entries of a page table behind a sequence's length are never read, on the CPU: the kernels read entries ahead of their use, up to the
last that ``table_of`` names."""

import os
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def kv_table(tmp_path_factory):
    exe = str(tmp_path_factory.mktemp("kv_table") / "kv_table")
    subprocess.check_call(["hipcc", "--offload-arch=gfx950", "-O1", "-std=c++17", "-I", os.path.join(ROOT, "include"),
                           "-I", os.path.join(ROOT, "paper_2606_22327_amd", "csrc"), "-x", "hip",
                           os.path.join(ROOT, "tests", "native", "kv_table_main.cpp"), "-o", exe])
    return exe


@pytest.mark.parametrize("page", [1, 16, 256])
def test_entries_behind_the_length_are_not_read(kv_table, page):
    width, lens = 40, [0, 1, page - 1, page, page + 1, 17 * page, 40 * page - 1, 40 * page]
    out = subprocess.run([kv_table, str(page.bit_length() - 1), str(width), *map(str, lens)], capture_output=True, text=True,
                         check=True).stdout.splitlines()
    got = [tuple(map(int, x.split())) for x in out]
    assert got == [(max(-(-n // page) - 1, 0), int(n > 0)) for n in lens]
