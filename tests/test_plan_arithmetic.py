"""Index arithmetic of the plan of a given choice up to its largest sizes: pieces of the kernel's and the launch's source,
compiled for the host with checks of signed overflow."""
import os
import re
import subprocess

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2406_00023_b200", "csrc")


def source():
    with open(os.path.join(CSRC, "sort.cu")) as f:
        return f.read()


def compiled(code, tmp_path):
    src, exe = tmp_path / "t.cpp", tmp_path / "t"
    src.write_text(code)
    subprocess.check_call(["g++", "-O1", "-std=c++17", "-fsanitize=signed-integer-overflow", "-fno-sanitize-recover=all", "-Wno-unknown-pragmas",
                           "-o", str(exe), str(src)])
    return lambda *args: subprocess.run([str(exe), *map(str, args)], capture_output=True, text=True, timeout=300)


FILL = """
#include <algorithm>
#include <cstdio>
#include <cstdlib>
#include <vector>
using std::max; using std::min;
struct Dim { int x; } gridDim, blockIdx;
struct Shape { int align, E, n_rows; };
static long long lowest, highest, rows, sum;                     // of the rows written; sum: of their numbers
struct Slot {
  long long at;
  void operator=(int) { lowest = min(lowest, at); highest = max(highest, at); ++rows; sum += at; }
};
struct Rows {
  Slot operator[](long long i) const { return {i}; }
  void four(long long i) const { for (int u = 0; u < 4; ++u) Slot{i + u} = -1; }
} row_token;
// arguments: CTAs, warps of a CTA, align, n_rows, then start and used of every expert
int main(int, char** a) {
  gridDim.x = atoi(a[1]);
  const int warps = atoi(a[2]);
  Shape s{atoi(a[3]), 0, atoi(a[4])};
  std::vector<int> start, used;
  for (char** q = a + 5; q[0]; q += 2) { start.push_back(atoi(q[0])); used.push_back(atoi(q[1])); }
  s.E = (int)start.size();
  lowest = 1ll << 62; highest = -1;
  for (blockIdx.x = 0; blockIdx.x < gridDim.x; ++blockIdx.x)
    for (int warp = 0; warp < warps; ++warp)
      for (int lane = 0; lane < 32; ++lane) {
        %s
      }
  printf("%%lld %%lld %%lld %%lld", lowest, highest, rows, sum);
}
"""


@pytest.fixture(scope="module")
def fill(tmp_path_factory):
    src = source()
    piece = src[src.index("const int first = s.align > 1"):src.index("if (blockIdx.x == 0 && tid == 0) {\n    int end")]
    piece, n = re.subn(r"\*reinterpret_cast<int4\*>\(row_token \+ r\) = make_int4\(-1, -1, -1, -1\);", "row_token.four(r);", piece)
    assert n == 1 and piece.count("row_token") == 3
    return compiled(FILL % piece, tmp_path_factory.mktemp("fill"))


TOP = 2 ** 31 - 65537                                       # the most rows that a configuration may have


@pytest.mark.parametrize("ctas, warps, align, n_rows, experts", [
    (1, 4, 1, 128, [(0, 60), (60, 60)]), (1, 16, 8, 1024 + 7 * 3, [(0, 1), (8, 0), (8, 1000)]), (16, 16, 128, 4 * 256, [(0, 256), (256, 0), (512, 3), (768, 129)]),
    (144, 16, 1, 300000, [(0, 299999)]), (144, 16, 1000, 200000, [(0, 5), (1000, 0), (1000, 100001)]),
    # as many rows as there may be: none, a few, all without a token; behind one expert, and behind the first of two
    (144, 16, 1, TOP, [(0, TOP)]), (144, 16, 1, TOP, [(0, 7), (7, TOP - 7)]), (144, 16, 1, TOP, [(0, TOP - 1001)]), (144, 16, 1, TOP, [(0, TOP - 300000)]),
    (144, 16, 1, TOP - 3, [(0, TOP - 3)]), (144, 16, 1, TOP, [(0, 0)]), (144, 16, 128, TOP // 128 * 128, [(0, 70000)]),
    (144, 16, 1024, TOP, [(0, 100), (1024, TOP - 2050)]), (1, 16, 1, TOP, [(0, TOP - 5)])], ids=str)
def test_rows_without_a_token_are_filled_and_no_others(fill, ctas, warps, align, n_rows, experts):
    r = fill(ctas, warps, align, n_rows, *[v for e in experts for v in e])
    assert r.returncode == 0, r.stderr
    gaps = [(lo + used, experts[i + 1][0] if i + 1 < len(experts) else n_rows) for i, (lo, used) in enumerate(experts)]
    gaps = [(a, b) for a, b in (gaps if align > 1 else gaps[-1:]) if a < b]
    lowest, highest, rows, total = map(int, r.stdout.split())
    assert rows == sum(b - a for a, b in gaps) and total == sum((a + b - 1) * (b - a) // 2 for a, b in gaps)
    if gaps:
        assert (lowest, highest) == (gaps[0][0], gaps[-1][1] - 1)


SPLIT = """
#include <algorithm>
#include <cstdio>
#include <cstdlib>
%s
%s
int main(int, char** a) {
  const PlanSplit p = plan_split(atoi(a[1]), atoi(a[2]), atoi(a[3]));
  printf("%%d %%d %%d", p.warps, p.ncta, p.nclusters);
}
"""


@pytest.fixture(scope="module")
def split(tmp_path_factory):
    src = source()
    rule = src[src.index("struct PlanSplit"):src.index("// The widest cluster of the plan's kernel")]
    return compiled(SPLIT % ("\n".join(re.findall(r"constexpr int SORT_.*", src)), rule), tmp_path_factory.mktemp("split"))


@pytest.mark.parametrize("widest", [1, 2, 4, 8, 16])
def test_the_plan_keeps_to_the_clusters_that_a_device_takes(split, widest):
    """No cluster wider than the device takes, whatever the batch; threads enough for two experts each; on a whole GPU one cluster
    up to 65536 pairs and up to 18 of 8 CTAs above."""
    for pairs in (0, 1, 512, 513, 1024, 1025, 4096, 4097, 8193, 65536, 65537, 200000, 600000, TOP):
        for E in (1, 64, 257, 1024):
            r = split(pairs, E, widest)
            assert r.returncode == 0, r.stderr
            warps, ncta, nclusters = map(int, r.stdout.split())
            assert 1 <= ncta <= widest and 4 <= warps <= 16 and 64 * warps >= E and 1 <= nclusters <= 18
            assert ncta == 8 or nclusters == 1
            assert (nclusters > 1) == (pairs > 65536 and widest >= 8)
            if ncta > 1 or pairs > 512:
                assert warps == 16
            if widest == 16 and pairs <= 65536:
                assert ncta == min(16, max(1, 1 << max(0, (pairs - 1) // 512).bit_length()))
