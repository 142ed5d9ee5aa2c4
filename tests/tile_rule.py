"""The rule that picks how many rows a workgroup of akvq_paged_attention takes, as the host code has it (csrc/akvq_kernels.h), for tests that are
meant for one of the tiles."""
import functools
import os
import subprocess
import tempfile

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
SOURCE = r"""
#include <cstdio>
#include "akvq_kernels.h"
int main() {
  long units, tokens, R, len;
  while (std::scanf("%ld %ld %ld %ld", &units, &tokens, &R, &len) == 4)
    std::printf("%ld %.9g %.9g\n", akvq::paged_tile_rows(units, tokens, R, len), akvq::paged_tile_cost(32, units, tokens, R, len),
                akvq::paged_tile_cost(akvq::kPagedManyRows, units, tokens, R, len));
}
"""


@functools.lru_cache(None)
def _program():
    path = tempfile.TemporaryDirectory()
    with open(os.path.join(path.name, "rule.cpp"), "w") as f:
        f.write(SOURCE)
    exe = os.path.join(path.name, "rule")
    subprocess.run(["g++", "-O1", "-std=c++17", "-D__HIP_PLATFORM_AMD__", "-I/opt/rocm/include", "-I" + os.path.join(ROOT, "paper_2501_15021_amd", "csrc"),
                    os.path.join(path.name, "rule.cpp"), "-o", exe], check=True, capture_output=True)
    return path, exe


def tiles(shapes):
    """For every (sequences x KV heads, tokens of the longest chunk, heads a KV head, bound of the cached rows): rows of a workgroup, and
    what the rule reckons for tiles of 32 and of 256, in us."""
    text = "\n".join(" ".join(str(int(x)) for x in s) for s in shapes)
    out = subprocess.run([_program()[1]], input=text, check=True, capture_output=True, text=True).stdout
    return [(int(t), float(a), float(b)) for t, a, b in (line.split() for line in out.splitlines())]


def tile_of(s, max_rows):
    """Of a call with these paged_inputs.Sequences."""
    rows = min(max_rows, s.x.shape[0])
    return tiles([(s.cache.B * s.Hkv, rows, s.Hq // s.Hkv, min(s.cache.max_len, s.cache.max_pages * s.cache.page_rows))])[0][0]
