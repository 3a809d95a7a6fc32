"""The selective layer's host arithmetic, on the CPU."""
import os
import subprocess

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")


def output_of(tmp_path, code):
    """What a program with the library's host code prints, line by line."""
    src, exe = tmp_path / "program.cpp", str(tmp_path / "program")
    src.write_text(code)
    r = subprocess.run([HIPCC, "-std=c++17", "--offload-arch=gfx950", "-w", "-I", os.path.join(ROOT, "include"),
                        "-I", os.path.join(ROOT, "paper_1404_1521_amd", "csrc"), "-x", "hip", str(src), "-o", exe],
                       capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
    return subprocess.run([exe], capture_output=True, text=True, check=True).stdout.split("\n")[:-1]


def test_places_of_equal_sequences(tmp_path):
    """The first sequence that starts at a token or later, up to the most tokens of a call."""
    lines = output_of(tmp_path, """
#include <cstdio>
#include "operators.h"
int main() {
  const int sizes[] = {1, 2, 3, 7, 64, 1 << 20, (1 << 30) - 1, 1 << 30, 2147483647};
  for (int T : sizes) {
    const int places[] = {0, 1, T / 2, T - 1, T, (1 << 30) - 1, 1 << 30, (1 << 30) + 1, 2147483647};
    for (int lo : places) std::printf("%d %d %d\\n", lo, T, pg::first_equal(lo, T));
  }
  std::printf("5 0 %d\\n", pg::first_equal(5, 0));
}
""")
    assert len(lines) == 82
    for line in lines:
        lo, T, got = map(int, line.split())
        assert got == (-(-lo // T) if T else 0), (lo, T, got)


def test_groups_go_by_the_longest_sequence_there_may_be(tmp_path):
    """Where offsets may hold one sequence of hundreds of ranges, groups of them are put
    together, however many other sequences there are; where none can have many, none are."""
    lines = output_of(tmp_path, """
#include <cstdio>
#include "selective_plan.h"
int main() {
  const struct { bool offsets; int tokens, nseq, D, N, heads; } calls[] = {
    {true, 16384, 1, 64, 16, 1}, {true, 16384, 33, 64, 16, 1}, {true, 16384, 700, 256, 8, 2}, {true, 9000, 9000, 40, 32, 1},
    {false, 16384, 1, 64, 16, 1}, {false, 16384, 4, 64, 16, 1}, {false, 16384, 32, 64, 16, 1},
    {true, 4097, 1, 2048, 16, 1}, {true, 32768, 8, 2048, 16, 1}, {true, 100, 3, 64, 16, 1}};
  for (const auto& c : calls) {
    const pg::Packed s{c.offsets ? &c : nullptr, nullptr, 8, c.tokens, c.nseq};
    const pg::SelPlan p = pg::selective_plan(s, c.D, c.N, c.heads, pg::SelSpace{});
    std::printf("%d %d\\n", p.ranges, p.groups);
  }
}
""")
    plans = [tuple(map(int, line.split())) for line in lines]
    for i, (ranges, groups) in enumerate(plans):
        assert groups == (-(-ranges // 16) if i < 6 else 0), (i, ranges, groups)
    assert [r for r, _ in plans[:2]] == [1024, 1024]
