"""Which requests the attention kernels compute, on the CPU: a C++ program runs the kernels' own rule (csrc/attn_request.h), built so that arithmetic beyond 32 bits ends it,
over offsets and lengths of every size, against Python's whole numbers.  No device code runs."""
import itertools
import os
import shutil
import subprocess

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2605_08151_amd", "csrc")

PROGRAM = r"""
#include <cstdio>
#include "attn_request.h"

int main()
{
    int r0, end, c, M, q, kv;
    while (std::scanf("%d %d %d %d %d %d", &r0, &end, &c, &M, &q, &kv) == 6) {
        const int n = specv::attn_request_rows(r0, end);
        std::printf("%d %d\n", n, (int)specv::attn_request_fits(r0, n, c, M, q, kv));
    }
}
"""
TOP, LOW = 2 ** 31 - 1, -2 ** 31


@pytest.fixture(scope="module")
def rule(tmp_path_factory):
    if shutil.which("g++") is None:
        pytest.skip("needs g++")
    d = tmp_path_factory.mktemp("request")
    (d / "rule.cpp").write_text(PROGRAM)
    subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-fsanitize=undefined", "-fno-sanitize-recover=all", "-I", CSRC, str(d / "rule.cpp"), "-o", str(d / "rule")], check=True)

    def run(cases):
        text = "\n".join(" ".join(map(str, c)) for c in cases)
        out = subprocess.run([str(d / "rule")], input=text, capture_output=True, text=True, check=True).stdout
        return [tuple(map(int, line.split())) for line in out.splitlines()]
    return run


def test_what_fits_is_what_fits_in_whole_numbers(rule):
    offsets = [LOW, LOW + 1, -5, -1, 0, 1, 4, 9, 10, 11, TOP - 1, TOP]
    lengths = [LOW, -1, 0, 1, 95, 96, 99, 100, 101, 10 ** 6, TOP - 4, TOP - 1, TOP]
    bounds = [(10, 4, 100), (10, 128, 100), (TOP, 128, TOP), (1, 1, 1), (10, 9, 3)]
    cases = [(r0, end, c, *b) for (r0, end, c), b in itertools.product(itertools.product(offsets, offsets, lengths), bounds)]
    got = rule(cases)
    assert len(got) == len(cases)
    for (r0, end, c, M, q, kv), (n, fits) in zip(cases, got):
        rows = end - r0
        want = r0 >= 0 and 1 <= rows <= q and end <= M and c >= 0 and c + rows <= kv
        assert bool(fits) == want, (r0, end, c, M, q, kv)
        assert n == (rows if r0 >= 0 and rows > 0 else 0)


def test_no_kernel_has_a_rule_of_its_own():
    for name in ("verify_attn.hip", "verify_attn_quant.hip"):
        text = open(os.path.join(CSRC, name)).read()
        assert "attn_request_fits(" in text and "attn_request_rows(" in text, name
        assert "c + n <= p.max_kv_len" not in text and "r0 + n <= p.M" not in text, name
