"""Where the write path into pages puts a sequence's rows (host code, no GPU): by the length that the device holds, not by the host's bound of
it; a length that names no row of the table drops them."""
import os
import subprocess

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
SOURCE = r"""
#include <climits>
#include <cstdio>
#include "akvq_kernels.h"
using namespace akvq;
#define CHECK(c) do { if (!(c)) { std::printf("%d %d %d %d: %s\n", len, bound, first, end, #c); return 1; } } while (0)
int main() {
  const int ints[] = {INT_MIN, -40, -1, 0, 1, 31, 32, 95, 96, 97, 127, 128, 129, 1 << 25, 1 << 30, INT_MAX};
  for (int len : ints) for (int bound : {0, 1, 96, 128}) for (int first : ints) for (int end : ints) for (int most : {1, 50}) {
    PagedArgs a{};
    a.row_cap = 128; a.max_len = bound; a.n_rows = 97; a.max_rows = most;
    const ChunkSpan s = append_span(len, first, end, a), read = chunk_span(len, first, end, a);
    CHECK(s.rows >= 0 && s.rows <= most && s.first >= 0 && s.first + s.rows <= a.n_rows);
    if (len < 0 || len >= a.row_cap) CHECK(s.rows == 0);
    else CHECK(s.len == len && s.first == read.first && s.rows == read.rows);
    CHECK(read.len >= 0 && read.len <= bound);
  }
  std::puts("ok");
}
"""


def test_rows_go_where_the_length_says(tmp_path):
    (tmp_path / "span.cpp").write_text(SOURCE)
    subprocess.run(["g++", "-O1", "-std=c++17", "-D__HIP_PLATFORM_AMD__", "-I/opt/rocm/include", "-I" + os.path.join(ROOT, "paper_2501_15021_amd", "csrc"),
                    str(tmp_path / "span.cpp"), "-o", str(tmp_path / "span")], check=True, capture_output=True)
    done = subprocess.run([str(tmp_path / "span")], capture_output=True, text=True)
    assert done.returncode == 0 and done.stdout.strip() == "ok", done.stdout
