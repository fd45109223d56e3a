"""What attention's kernels work out from a call's sizes, in a program of its own that ends where 32 bits do not hold a result.
No kernel runs."""
import os
import subprocess

import pytest

HERE = os.path.dirname(os.path.abspath(__file__))
MOST = 2 ** 31 - 64


@pytest.fixture(scope="module")
def sizes(tmp_path_factory):
    """Answers of attention_sizes.cpp, a line of numbers for each line asked."""
    from paper_2310_05674_b200 import build
    exe = str(tmp_path_factory.mktemp("sizes") / "attention_sizes")
    subprocess.check_call(["g++", "-std=c++17", "-fsanitize=signed-integer-overflow", "-fsanitize-undefined-trap-on-error",
                           "-I", build.CSRC, os.path.join(HERE, "attention_sizes.cpp"), "-o", exe])

    def ask(lines):
        out = subprocess.run([exe], input="\n".join(lines), capture_output=True, text=True, check=True).stdout
        rows = [[int(v) for v in line.split()] for line in out.splitlines()]
        assert len(rows) == len(lines)
        return rows
    return ask


@pytest.mark.parametrize("pages,page", [(1, 1), (5, 16), (1 << 24, 1 << 20), (2048, 1 << 20), (2047, 1 << 20), (1 << 24, 127),
                                        (1 << 24, 128), (1 << 24, 129), (33554431, 64)])
def test_steps_of_a_paged_sequence(sizes, pages, page):
    """Whatever a length says, it is taken as the nearest that the table holds, and its last step ends within 31 bits."""
    most = min(pages * page, MOST)
    lengths = [-2 ** 31, -1, 0, 1, 63, 64, 65, most - 65, most - 64, most - 63, most - 1, most, most + 1, MOST - 1, MOST, MOST + 1,
               2 ** 31 - 2, 2 ** 31 - 1]
    lengths = [n for n in lengths if -2 ** 31 <= n < 2 ** 31]
    for n, (keys, steps, last) in zip(lengths, sizes(["paged %d %d %d" % (n, pages, page) for n in lengths])):
        assert keys == max(0, min(n, most)), n
        assert steps == -(-keys // 64) and last == 64 * steps - 1, n


@pytest.mark.parametrize("lq,lk", [(1, 1), (5, 5), (3, 9), (9, 3), (0, 4), (4, 0), (2 ** 30, 2 ** 30), (2 ** 30, 0), (0, 2 ** 30), (1, 2 ** 30),
                                   (2 ** 30, 1), (2 ** 30, 2 ** 30 - 5)])
def test_what_a_query_sees(sizes, lq, lk):
    """At a text's ends, and for the rows of its last tile that lie behind it (up to 255 of queries, 127 of keys)."""
    ends = {0, 1, 2, 5, lq - 1, lq, lq + 255, lk - 1, lk, lk + 127}
    for causal in (0, 1):
        for prefix in sorted({0, min(2, lk), lk}):
            def ask(what, rows):
                return zip(rows, sizes(["%s %d %d %d %d %d" % (what, causal, lq, lk, prefix, i) for i in rows]))
            for i, (at, seen) in ask("query", sorted(i for i in ends if 0 <= i < lq + 256)):
                assert at == i + lk - lq
                assert seen == (max(0, min(lk, max(prefix, at + 1))) if causal else lk), (causal, prefix, i)
            for i, (first,) in ask("key", sorted(i for i in ends if 0 <= i < lk + 128)):
                assert first == (0 if not causal or i < prefix else max(0, i - (lk - lq))), (causal, prefix, i)
