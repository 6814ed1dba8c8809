"""How the paged attention cuts keys among workgroups, at the limits of its sizes: the functions of
csrc/paged_cut.h, compiled for the host."""
import os
import subprocess

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))),
                    "paper_2601_03700_amd", "csrc")
MOST = 2 ** 31 - 1 - 1023           # tokens that a sequence may have
BLOCK = 64
SIZES = sorted({n for k in (0, 1, 31, 63, 64, 65, 127, 128, 1000, 16384, 40000, 2 ** 20 + 7,
                            2 ** 30, 2 ** 31 - 2 ** 26, MOST) for n in (k - 1, k, k + 1)
                if 0 <= n <= MOST} | {512 * 4194301})


def host(d, lines, asked):
    """Output lines of a program that includes the header, for lines of input."""
    src = ["#include <cstdio>", '#include "paged_cut.h"', "int main() {", *lines, "}"]
    (d / "cut.cpp").write_text("\n".join(src))
    # an overflow of int ends the program
    subprocess.run(["g++", "-std=c++17", "-O1", "-fsanitize=undefined", "-fno-sanitize-recover=all",
                    "-I", CSRC, "-o", str(d / "cut"), str(d / "cut.cpp")], check=True)
    r = subprocess.run([str(d / "cut")], input="\n".join(" ".join(map(str, a)) for a in asked),
                       capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
    return [tuple(map(int, line.split())) for line in r.stdout.splitlines()]


@pytest.fixture(scope="module")
def cuts(tmp_path_factory):
    """{(n, parts): [(begin, end), ...]}"""
    asked = [(n, parts) for n in SIZES for parts in range(1, 33)]
    out = iter(host(tmp_path_factory.mktemp("cut"), [
        'int n, parts; while (std::scanf("%d %d", &n, &parts) == 2) for (int p = 0; p < parts; ++p) {',
        f"const adept::KeyRange r = adept::part_of_keys(n, parts, p, {BLOCK});",
        'std::printf("%d %d\\n", r.begin, r.end); }'], asked))
    return {key: [next(out) for _ in range(key[1])] for key in asked}


@pytest.mark.parametrize("n", SIZES)
def test_parts_take_each_key_once(cuts, n):
    for parts in range(1, 33):
        at = 0
        for begin, end in cuts[n, parts]:
            assert begin == at and begin <= end <= n
            assert begin % BLOCK == 0 or begin == end == n
            at = end
        assert at == n
        # a part looks up to two blocks past its end
        assert max(e for _, e in cuts[n, parts]) + 3 * BLOCK < 2 ** 31


@pytest.mark.parametrize("entries", [1, 2, 40, 1023, 1024])
def test_stretches_of_single_entries(tmp_path, entries):
    """Entries of up to the most tokens, and as few stretches wanted as one: each unit is taken
    once, by at most wanted + entries stretches."""
    unit = 128
    most = -(-MOST // unit)
    asked = [(u * entries, want, least, u) for u in (0, 1, 2, 31, 1000, 2 ** 18, most - 1, most)
             for want in (1, 2, 3, 64, 2048) for least in (1, 2, 4)]
    out = host(tmp_path, [
        'long long sum; int want, least, units;',
        'while (std::scanf("%lld %d %d %d", &sum, &want, &least, &units) == 4) {',
        "const int cut = adept::stretch_units(sum, want, least);",
        'std::printf("%d %d\\n", cut, adept::stretches(units, cut)); }'], asked)
    assert len(out) == len(asked)
    for (_, want, least, units), (cut, parts) in zip(asked, out):
        assert cut >= least and parts >= 1
        assert (parts - 1) * cut < max(units, 1) <= max(parts * cut, 1)
        assert parts * entries <= want + entries
