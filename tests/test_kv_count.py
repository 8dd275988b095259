"""The number that holds a reserve's pages and copies (csrc/kv_count.hpp), at its bounds: compiled for the host."""
import shutil
import subprocess

import pytest

from paper_2609_36601_amd.build import CSRC
from tests.test_kv_abi import all_calls, lib, pool, table  # noqa: F401

# sums of n sequences that copy a page and take `fresh` new ones each, and of one more without a copy
PROGRAM = r"""
#include <cstdio>
#include <cstdlib>
#include "kv_count.hpp"
int main(int argc, char** argv) {
  for (int i = 1; i + 1 < argc; i += 2) {
    const int64_t n = atoll(argv[i]);
    const int32_t fresh = atoi(argv[i + 1]);
    int64_t sum = 0;
    for (int64_t b = 0; b < n; ++b) sum += saki::kv_count(true, fresh);
    sum += saki::kv_count(false, 5);
    printf("%lld %lld\n", (long long)saki::kv_count_pages(sum), (long long)saki::kv_count_copies(sum));
  }
}
"""


@pytest.mark.skipif(shutil.which("g++") is None, reason="needs a host compiler")
def test_sums_hold_every_copy(tmp_path):
    src = tmp_path / "count.cpp"
    src.write_text(PROGRAM)
    subprocess.run(["g++", "-O1", "-std=c++17", "-I", CSRC, str(src), "-o", str(tmp_path / "count")], check=True)
    cases = [(0, 0), (1, 3), (2**23 - 1, 0), (2**23, 0), (2**23 + 1, 1), (2**24, 0), (2**24, 2**13)]
    out = subprocess.run([str(tmp_path / "count"), *[str(x) for c in cases for x in c]], check=True, capture_output=True,
                         text=True).stdout.split()
    for i, (n, fresh) in enumerate(cases):
        assert (int(out[2 * i]), int(out[2 * i + 1])) == (n * (fresh + 1) + 5, n)


def test_tables_beyond_the_count_are_refused(lib):  # noqa: F811
    big = dict(n_seq=2**24, max_pages=2**14, page_size=8)
    for name, st in all_calls(lib, table(**big), pool()):
        assert st == 2, name
    assert lib.saki_kv_commit(table(**big), 64, None, None, None) == 2
    assert lib.saki_kv_fork(table(**big), 1, 64, 64, None, None) == 2
