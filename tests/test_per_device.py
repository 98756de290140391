"""What the library asks a device once is kept for that device alone."""
import os
import re
import subprocess

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2608_23805_gb300", "csrc")

PROGRAM = r"""
#include <cstdio>
#include "per_device.h"
int main() {
  static msi::PerDevice<4> kept;
  int asked = 0, fail = 0;
  auto get = [&](int dev, int key) {
    int v = -1;
    const int e = kept.get(dev, key, &v, [&](int* n) { ++asked; *n = 100 * dev + key; return fail; });
    printf("%d %d %d\n", e, v, asked);
  };
  get(0, 3); get(1, 3); get(0, 3); get(1, 3); get(1, 0); get(0, 0); get(0, 0);
  get(64, 2); get(64, 2); get(-1, 1);      // not kept
  fail = 7; get(2, 1); fail = 0; get(2, 1); get(2, 1);  // an error is not kept
}
"""


def test_kept_by_device(tmp_path):
    src = tmp_path / "p.cpp"
    src.write_text(PROGRAM)
    subprocess.run(["g++", "-std=c++17", "-Wall", "-Werror", "-I", CSRC, str(src), "-o", str(tmp_path / "p")], check=True)
    out = subprocess.run([str(tmp_path / "p")], check=True, capture_output=True, text=True).stdout.split("\n")
    assert [tuple(map(int, l.split())) for l in out if l] == [
        (0, 3, 1), (0, 103, 2), (0, 3, 2), (0, 103, 2), (0, 100, 3), (0, 0, 4), (0, 0, 4),
        (0, 6402, 5), (0, 6402, 6), (0, -99, 7), (7, 201, 8), (0, 201, 9), (0, 201, 9)]


def test_sampling_keeps_no_residency_of_its_own():
    with open(os.path.join(CSRC, "sample.cu")) as f:
        text = re.sub(r"//[^\n]*", "", f.read())
    assert not re.search(r"static\s+std::atomic<int>", text) and re.search(r"static PerDevice<", text)
    assert re.search(r"at_once\.get\(dev,", text)
