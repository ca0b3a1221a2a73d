"""The paged cache's arithmetic on lengths, starts and pages (csrc/kv8_plan.hpp), walked on the host: whatever the arrays hold, rows and
positions stay inside the call, every new token's page is counted, and the chunks of the attention cover every cached token."""
import os
import random
import subprocess

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2502_15779_amd", "csrc")

SOURCE = r"""
#include "kv8_plan.hpp"
#include <cstdio>
#include <vector>
using namespace rcp;
int main()
{
    int kind, n, rows, width, shift, chunks;
    while (scanf("%d %d %d %d %d %d", &kind, &n, &rows, &width, &shift, &chunks) == 6) {
        std::vector<int> lengths(n), starts(n + 1);
        for (int& v : lengths) if (scanf("%d", &v) != 1) return 1;
        for (int& v : starts) if (scanf("%d", &v) != 1) return 1;
        const int* at = kind == 0 ? nullptr : starts.data();
        long long pages = 0;
        for (int b = 0; b < n; ++b) {
            const Kv8Run r = kv8_run(at, lengths.data(), b, rows);
            const Kv8Pages p = kv8_pages(r, width << shift, shift);
            printf("%d %d %d %d %d %d ", r.first, r.count, r.pos, r.length, p.first_page, p.pages);
            pages += p.pages;
        }
        long long total = 0;
        for (int v : lengths) total += kv8_clamp(v, 0, width << shift);
        const int C = kv8_chunk_tokens(static_cast<int>(total), n, chunks);
        long long sum = 0;
        for (int v : lengths) sum += kv8_chunks(kv8_clamp(v, 0, width << shift), C);
        printf("| %lld %lld %d %lld |", pages, kv8_most_pages(rows, n, shift), C, sum);
        if (kind != 0)
            for (int t = 0; t < rows; ++t) printf(" %d", kv8_sequence_of(at, n, t, rows));
        printf("\n");
    }
}
"""


@pytest.fixture(scope="module")
def walk(tmp_path_factory):
    d = tmp_path_factory.mktemp("kv8")
    (d / "plan.cpp").write_text(SOURCE)
    exe = str(d / "plan")
    subprocess.run(["g++", "-O1", "-std=c++17", "-Wall", "-Werror", "-fsanitize=undefined", "-fno-sanitize-recover", "-I", CSRC, str(d / "plan.cpp"),
                    "-o", exe], check=True)

    def run(kind, lengths, starts, rows, width, shift, chunks):
        n = len(lengths)
        text = " ".join(map(str, [kind, n, rows, width, shift, chunks] + list(lengths) + list(starts or [0] * (n + 1))))
        out = subprocess.run([exe], input=text, capture_output=True, text=True, check=True).stdout
        runs, sums, owner = (list(map(int, p.split())) for p in out.split("|"))
        return [runs[6 * b:6 * b + 6] for b in range(n)], sums, owner
    return run


def test_runs_of_ordinary_calls(walk):
    # (first row, count, position of the first, length, first page, pages)
    runs, sums, owner = walk(1, [40, 7, 0, 65], [2, 10, 17, 17, 18], 20, 5, 4, 16)
    assert runs == [[2, 8, 32, 40, 2, 1], [10, 7, 0, 7, 0, 1], [17, 0, 0, 0, 0, 0], [17, 1, 64, 65, 4, 1]]
    assert owner == [-1, -1] + [0] * 8 + [1] * 7 + [3] + [-1, -1]
    runs, _, _ = walk(0, [40, 0, 81], None, 3, 5, 4, 16)
    assert runs == [[0, 1, 39, 40, 2, 1], [1, 1, -1, 0, 0, 0], [2, 1, 80, 81, 0, 0]]   # empty; beyond the table
    runs, _, _ = walk(1, [5, 90], [0, 9, 29], 29, 5, 4, 16)                            # more new tokens than the length; past the end
    assert runs == [[0, 9, -4, 5, 0, 1], [9, 20, 70, 90, 4, 1]]


def test_no_contents_leave_the_call(walk):
    rng = random.Random(5)
    wild = [-2 ** 31, -1, 0, 1, 5, 63, 2 ** 24, 2 ** 24 + 1, 2 ** 31 - 1]
    for _ in range(60):
        n, rows, shift, width = rng.randint(1, 9), rng.randint(1, 40), rng.randint(4, 7), rng.randint(1, 6)
        lengths = [rng.choice(wild + [rng.randint(0, 200)]) for _ in range(n)]
        starts = [rng.choice(wild + [rng.randint(-3, 50)]) for _ in range(n + 1)]
        runs, _, owner = walk(1, lengths, starts, rows, width, shift, 2 * n)
        for first, count, pos, length, page, pages in runs:
            assert 0 <= first and 0 <= count and first + count <= rows and 0 <= length and pos == length - count
            assert 0 <= page and 0 <= pages and page + pages <= width
        for t, b in enumerate(owner):
            assert b == -1 or runs[b][0] <= t < runs[b][0] + runs[b][1]


def test_pages_and_chunks_fit_what_the_host_provides(walk):
    rng = random.Random(6)
    for _ in range(60):
        n, shift = rng.randint(1, 40), rng.randint(4, 7)
        width = rng.randint(1, 40)
        new = [rng.choice([0, 1, 1, 2, rng.randint(0, 300)]) for _ in range(n)]
        lengths = [m + rng.choice([0, rng.randint(0, 3000)]) for m in new]
        starts = [0]
        for m in new:
            starts.append(starts[-1] + m)
        chunks = rng.choice([2 * n, 2 * n + 1, 4 * n + 100])
        runs, (pages, most, C, cut), owner = walk(1, lengths, starts, max(starts[-1], 1), width, shift, chunks)
        assert pages <= most and cut <= chunks and C % 64 == 0 and C >= 64
        for (first, count, pos, length, page, pages), m in zip(runs, new):
            touched = {p >> shift for p in range(max(pos, 0), min(length, width << shift))} if m else set()
            assert sorted(touched) == list(range(page, page + pages))
        assert owner[:starts[-1]] == [b for b, m in enumerate(new) for _ in range(m)]
