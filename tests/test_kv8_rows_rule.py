"""Which rows an append of the 8-bit cache reads and writes queries of (csrc/kv8_rows.h), on the host: those of
the sequences and no others, each once, in groups of one and of four."""
import subprocess

import pytest

from paper_2609_09338_amd import build

PROGRAM = r"""
#include <cstdio>
#include "kv8_rows.h"
// per line: total, cu_first, cu_end, per, groups launched -> rows read (least, most), rows written as a list
int main() {
  int total, a, b, per, groups;
  while (std::scanf("%d %d %d %d %d", &total, &a, &b, &per, &groups) == 5) {
    const osp::QueryRows q = osp::query_rows(total, a, b);
    int least = 1 << 30, most = -1;
    char sep = ' ';
    for (int i = 0; i < groups; ++i) {
      if (!osp::group_has_rows(q, i, per)) continue;
      for (int r = 0; r < per; ++r) {
        const int row = i * per + r, at = osp::row_read(q, row);
        if (at < least) least = at;
        if (at > most) most = at;
        if (osp::has_row(q, row)) { std::printf("%c%d", sep, row); sep = ','; }
      }
    }
    std::printf(" | %d %d\n", least, most);
  }
}
"""


@pytest.fixture(scope="module")
def walk(tmp_path_factory):
    d = tmp_path_factory.mktemp("kv8_rows")
    (d / "main.cpp").write_text(PROGRAM)
    exe = str(d / "rule")
    subprocess.run(["g++", "-std=c++17", "-I", build.CSRC, str(d / "main.cpp"), "-o", exe], check=True)

    def ask(cases):
        text = "\n".join(" ".join(map(str, c)) for c in cases)
        out = []
        for line in subprocess.run([exe], input=text, capture_output=True, text=True, check=True).stdout.splitlines():
            rows, span = line.split("|")
            out.append(([int(x) for x in rows.split(",") if x.strip()], tuple(int(x) for x in span.split())))
        return out
    return ask


def test_rows_outside_the_sequences_are_neither_read_nor_written(walk):
    cases = [(total, a, b, per, (total + per - 1) // per)
             for total in (1, 4, 7, 34, 70) for a in (0, 1, 2, 3, 5, 33) for b in (0, 1, 6, 34, 70, 90) for per in (1, 4) if a <= b]
    for (total, a, b, per, _), (rows, span) in zip(cases, walk(cases)):
        want = list(range(a, min(b, total)))
        assert rows == want, (total, a, b, per)
        assert not want or (span[0] >= want[0] and span[1] <= want[-1]), (total, a, b, per, span)
        assert want or span == (1 << 30, -1)


def test_without_row_offsets_every_row_is_formed(walk):
    for n in (1, 5, 64):
        for per in (1, 4):
            assert walk([(n, 0, n, per, (n + per - 1) // per)])[0][0] == list(range(n))


def test_a_count_that_begins_below_zero_begins_at_the_first_row(walk):
    assert walk([(9, -3, 5, 4, 3)])[0] == ([0, 1, 2, 3, 4], (0, 4))
