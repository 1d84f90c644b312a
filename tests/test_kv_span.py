"""Which entries of a row hx_kv_free gives back, as its kernel works it out, on the host."""
import os
import subprocess

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2605_16637_amd", "csrc")
LOW, HIGH = -2 ** 31, 2 ** 31 - 1

PROGRAM = r"""
#include "hx_kv_span.hpp"
#include <stdio.h>
// each line: first last len shift -> lo hi, how many entries a workgroup of 256 visits (16 rounds at most), the least and the largest of them
int main(void)
{
    int first, last, len, shift;
    while (scanf("%d %d %d %d", &first, &last, &len, &shift) == 4) {
        const HxSpan s = hx_filled_within(first, last, len, shift);
        long long n = 0, least = -1, most = -1;
        for (unsigned t = 0; t < 256; ++t) {
            int rounds = 0;
            for (uint32_t b = s.lo + t; b < s.hi && rounds < 16; b += 256, ++rounds) {
                const long long at = (int)b;          // as an offset into the row
                if (n == 0 || at < least) least = at;
                if (n == 0 || at > most) most = at;
                ++n;
            }
        }
        printf("%u %u %lld %lld %lld\n", s.lo, s.hi, n, least, most);
    }
    return 0;
}
"""


@pytest.fixture(scope="module")
def spans(tmp_path_factory):
    d = tmp_path_factory.mktemp("span")
    (d / "a.cpp").write_text(PROGRAM)
    subprocess.check_call(["g++", "-std=c++17", "-Wall", "-Werror", "-fsanitize=undefined", "-fno-sanitize-recover=all", "-I", CSRC, "-o", str(d / "a"), str(d / "a.cpp")])

    def ask(cases):
        text = subprocess.check_output([str(d / "a")], input="\n".join(" ".join(map(str, c)) for c in cases), text=True)
        return [tuple(map(int, line.split())) for line in text.splitlines()]
    return ask


@pytest.mark.parametrize("shift", [0, 1, 4, 10])
def test_entries_within_bounds(spans, shift):
    T = 1 << shift
    cases = [(first, last, n, shift) for n in (0, 1, T - 1, T, T + 1, 5 * T + 3, 700) for first in (LOW, -1, 0, 1, T, 2 * T - 1, n - 1, n, n + 1, HIGH - 255, HIGH)
             for last in (LOW, -1, 0, 1, T, 3 * T + 1, n - 1, n, n + 1, HIGH)]
    for (first, last, n, _), (lo, hi, count, least, most) in zip(cases, spans(cases)):
        want = [b for b in range(n // T) if b * T >= first and (b + 1) * T <= min(last, n)]
        assert count == len(want) and (not want or (least, most) == (want[0], want[-1])), (first, last, n)


@pytest.mark.parametrize("shift", [0, 4])
def test_rows_of_the_greatest_length(spans, shift):
    """The last entries of a row whose positions fill an int; a bound beyond them gives back nothing."""
    T, n = 1 << shift, HIGH
    cases = [(first, last, n, shift) for first in (n - 300 * T, n - 1, n) for last in (LOW, 0, n - 1, n)]
    for (first, last, _, _), (lo, hi, count, least, most) in zip(cases, spans(cases)):
        a, b = -(-first // T), max(last, 0) // T
        assert count == max(0, b - a) and (count == 0 or (least, most) == (a, b - 1)), (first, last)
