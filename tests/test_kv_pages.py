"""Pages of committed lengths up to the end of 32 bits: the arithmetic of commit and truncate (csrc/kv_pages.h) in a C++ program that ends where a sum leaves 32 bits, against
Python's whole numbers; and on the GPU, where lengths that do not fit are flagged and left alone."""
import itertools
import os
import shutil
import subprocess

import numpy as np
import pytest
import torch

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2605_08151_amd", "csrc")
TOP, LOW = 2 ** 31 - 1, -2 ** 31

PROGRAM = r"""
#include <cstdio>
#include "kv_pages.h"

int main()
{
    int from, to, c, P;
    while (std::scanf("%d %d %d %d", &from, &to, &c, &P) == 4) {
        const int n = specv::kv_rows(from, to);
        const bool fits = specv::kv_length_fits(n, c);
        std::printf("%d %d %d\n", n, (int)fits, fits ? specv::pages_of(c + n, P) : -1);
    }
}
"""


def test_pages_and_lengths_are_those_of_whole_numbers(tmp_path):
    if shutil.which("g++") is None:
        pytest.skip("needs g++")
    (tmp_path / "pages.cpp").write_text(PROGRAM)
    subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-fsanitize=undefined", "-fno-sanitize-recover=all", "-I", CSRC, str(tmp_path / "pages.cpp"), "-o", str(tmp_path / "pages")],
                   check=True)
    offsets = [LOW, LOW + 7, -3, 0, 1, 5, 1000, TOP - 16, TOP]
    cases = list(itertools.product(offsets, offsets, [LOW, -1, 0, 1, 15, 16, 17, 10 ** 6, TOP - 1000, TOP - 16, TOP - 5, TOP - 1, TOP], [1, 7, 16, 128, TOP]))
    out = subprocess.run([str(tmp_path / "pages")], input="\n".join(" ".join(map(str, c)) for c in cases), capture_output=True, text=True, check=True).stdout.splitlines()
    assert len(out) == len(cases)
    for (from_, to, c, P), line in zip(cases, out):
        n = to - from_ if 1 <= to - from_ <= TOP else 0
        fits = n >= 1 and c >= 0 and c + n <= TOP
        assert line == "%d %d %d" % (n, fits, -(-(c + n) // P) if fits else -1), (from_, to, c, P)


def _state(lens):
    i32 = lambda a: torch.from_numpy(np.ascontiguousarray(a, dtype=np.int32)).cuda()           # noqa: E731
    B = len(lens)
    return i32, dict(table=i32(np.arange(B * 4).reshape(B, 4)), lens=i32(lens), free=i32(np.full(40, -1)), count=i32([3]), status=i32([0]))


# lengths at the end of 32 bits, between two ordinary ones of 4 pages
FAR = [TOP, TOP - 1, TOP - 5, TOP - 16, TOP - 30]


@pytest.mark.gpu
@pytest.mark.parametrize("far", FAR)
def test_commit_leaves_lengths_that_pass_32_bits(far):
    from paper_2605_08151_amd import binding as sv
    i32, s = _state([40, far, 40])
    n = 20
    sv.spec_kv_commit(s["table"], s["lens"], i32([0, n, 2 * n, 3 * n]), i32([3, 3, 3]), s["free"], s["count"], 16, s["status"])
    fits = far + n <= TOP
    assert int(s["status"]) == (0 if fits else sv.FLAG_BAD_LENGTH)
    assert s["lens"].tolist() == [44, far + 4 if fits else far, 44]
    assert s["table"].tolist() == [[0, 1, 2, -1], [4, 5, 6, 7], [8, 9, 10, -1]] and int(s["count"]) == 5 and s["free"][3:5].tolist() == [3, 11]


@pytest.mark.gpu
@pytest.mark.parametrize("far", FAR)
@pytest.mark.parametrize("keep", [20, TOP - 40, TOP])
def test_truncate_of_lengths_at_the_end_of_32_bits(far, keep):
    from paper_2605_08151_amd import binding as sv
    i32, s = _state([60, far, 60])
    sv.spec_kv_truncate(s["table"], s["lens"], i32([40, keep, 48]), s["free"], s["count"], 16, s["status"])
    assert int(s["status"]) == 0 and s["lens"].tolist() == [40, min(far, keep), 48]
    held = [4, 5, -1, -1] if keep == 20 else [4, 5, 6, 7]
    freed = [3] + ([6, 7] if keep == 20 else []) + [11]
    assert s["table"].tolist() == [[0, 1, 2, -1], held, [8, 9, 10, -1]]
    assert int(s["count"]) == 3 + len(freed) and s["free"][3:3 + len(freed)].tolist() == freed


@pytest.mark.gpu
@pytest.mark.parametrize("far", [62, 10 ** 6] + FAR)
def test_a_path_behind_the_page_table_moves_nothing(far):
    """Accepted nodes 0, 2, 3 of a tree: their rows move to the front, unless the length puts them behind the table."""
    from paper_2605_08151_amd import binding as sv
    i32, s = _state([30, far, 40])
    cache = [torch.arange(12 * 16 * 8, device="cuda").remainder(251).to(torch.bfloat16).view(12, 1, 16, 8) for _ in range(2)]
    before = cache[0].clone()
    path = i32(np.tile([0, 2, 3, 0, 0], (3, 1)))
    sv.spec_kv_commit_tree(*cache, s["table"], s["lens"], i32([0, 5, 10, 15]), i32([2, 2, 2]), path, s["free"], s["count"], s["status"])
    fits = far + 5 <= TOP
    assert int(s["status"]) == (sv.FLAG_BAD_PAGE if fits else sv.FLAG_BAD_LENGTH)
    assert s["lens"].tolist() == [33, far + 3 if fits else far, 43]
    want = before.clone()
    for page0, c in ((0, 30), (8, 40)):
        for k, src in ((1, 2), (2, 3)):
            want[page0 + (c + k) // 16, 0, (c + k) % 16] = before[page0 + (c + src) // 16, 0, (c + src) % 16]
    for got in cache:
        assert torch.equal(got, want)
