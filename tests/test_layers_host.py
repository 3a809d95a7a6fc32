"""The selective layer's host arithmetic, on the CPU."""
import os
import subprocess

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")


def test_places_of_equal_sequences(tmp_path):
    """The first sequence that starts at a token or later, up to the most tokens of a call."""
    src = tmp_path / "places.cpp"
    src.write_text("""
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
    exe = str(tmp_path / "places")
    r = subprocess.run([HIPCC, "-std=c++17", "--offload-arch=gfx950", "-w", "-I", os.path.join(ROOT, "include"),
                        "-I", os.path.join(ROOT, "paper_1404_1521_amd", "csrc"), "-x", "hip", str(src), "-o", exe],
                       capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
    lines = subprocess.run([exe], capture_output=True, text=True, check=True).stdout.split("\n")[:-1]
    assert len(lines) == 82
    for line in lines:
        lo, T, got = map(int, line.split())
        assert got == (-(-lo // T) if T else 0), (lo, T, got)
