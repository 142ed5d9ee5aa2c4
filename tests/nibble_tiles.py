"""The rule that picks how many rows a workgroup of attention over 4-bit codes takes, as the host code has it (csrc/akvq_kernels.h), for tests that are meant
for one of the tiles."""
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
  int G;
  while (std::scanf("%ld %ld %ld %ld %d", &units, &tokens, &R, &len, &G) == 5) {
    const akvq::PagedKind kind = {4, G};
    std::printf("%ld %d %.9g %.9g\n", akvq::paged_tile_rows(units, tokens, R, len, kind), akvq::paged_splits(units, tokens, R, len, kind),
                akvq::paged_tile_cost(32, units, tokens, R, len, kind), akvq::paged_tile_cost(akvq::kPagedManyRows, units, tokens, R, len, kind));
  }
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
    """For every (sequences x KV heads, tokens of the longest chunk, heads a KV head, bound of the cached rows, G): rows of a workgroup, splits of the
    keys, and what the rule reckons for tiles of 32 and of 256, in us."""
    text = "\n".join(" ".join(str(int(x)) for x in s) for s in shapes)
    out = subprocess.run([_program()[1]], input=text, check=True, capture_output=True, text=True).stdout
    return [(int(t), int(n), float(a), float(b)) for t, n, a, b in (line.split() for line in out.splitlines())]


def tile_of(s, max_rows):
    """Of a call with these sequences: 8 is a tile of 16 of which no workgroup has more than eight rows."""
    rows, R = min(max_rows, s.x.shape[0]), s.Hq // s.Hkv
    tile = tiles([(s.cache.B * s.Hkv, rows, R, min(s.cache.max_len, s.cache.max_pages * s.cache.page_rows), s.G)])[0][0]
    return 8 if tile == 16 and rows * R <= 8 else tile
