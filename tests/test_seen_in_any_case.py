"""Which entries of its row's table a query over chosen pages reads for the pages that it sees in any case, as hx_attend_top's kernel works it out, on the host."""
import os
import subprocess

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2605_16637_amd", "csrc")

PROGRAM = r"""
#include "hx_kv_span.hpp"
#include <stdio.h>
// each line: own n_pages n_first n_last -> all from to fixed, the entries that a workgroup of `threads` reads
int main(void)
{
    int own, n_pages, n_first, n_last;
    while (scanf("%d %d %d %d", &own, &n_pages, &n_first, &n_last) == 4) {
        const HxSeen s = hx_seen_in_any_case(own, n_pages, n_first, n_last);
        printf("%d %d %d %d", s.all, s.from, s.to, s.fixed);
        if (!s.all)
            for (int i = 0; i < s.fixed; ++i) printf(" %d", s.entry(i));
        printf("\n");
    }
    return 0;
}
"""


@pytest.fixture(scope="module")
def seen(tmp_path_factory):
    d = tmp_path_factory.mktemp("seen")
    (d / "a.cpp").write_text(PROGRAM)
    subprocess.check_call(["g++", "-std=c++17", "-Wall", "-Werror", "-fsanitize=undefined", "-fno-sanitize-recover=all", "-I", CSRC, "-o", str(d / "a"), str(d / "a.cpp")])

    def ask(cases):
        text = subprocess.check_output([str(d / "a")], input="\n".join(" ".join(map(str, c)) for c in cases), text=True)
        return [tuple(map(int, line.split())) for line in text.splitlines()]
    return ask


def test_entries_lie_in_the_row(seen):
    """Own pages of 0 and more, fewer and more than are seen; first and last ones that a short row has not."""
    cases = [(own, n_pages, first, last) for n_pages in (1, 2, 3, 4, 7, 12, 40, 4096) for first in (0, 1, 2, 4, 6, 11, 4095) for last in (1, 2, 3, 5, 12, 4096)
             if first + last <= n_pages for own in (0, 1, 2, 3, 6, 7, 8, 11, 12, 13, 39, 40, 300, 4095, 4096, 4097, 2 ** 31 - 1)]
    got = seen(cases)
    assert len(got) == len(cases) > 500
    for (own, n_pages, first, last), (all_seen, lo, hi, fixed, *entries) in zip(cases, got):
        assert bool(all_seen) == (own + 1 <= n_pages)
        want = [] if all_seen else [*range(first), *range(own - last + 1, own + 1)]
        assert entries == want and fixed == len(want), (own, n_pages, first, last)
        assert all(0 <= e <= own for e in entries)
        if not all_seen:
            assert (lo, hi) == (first, own - last + 1) and 0 <= lo <= hi <= own
