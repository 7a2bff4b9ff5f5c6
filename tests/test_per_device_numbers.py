"""A number that was found on one device (how many clusters of a kernel fit) says nothing of another.  The
helper that keeps them is plain C++ and runs here against a fake of the question; no GPU is used."""
import os
import re
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2607_17572_gb300", "csrc")

PROGRAM = r"""
#include <cstdio>
#include <thread>
#include <vector>
#include "per_device.cuh"

#define EXPECT(c) do { if (!(c)) { std::printf("line %d: %s\n", __LINE__, #c); return 1; } } while (0)
enum Status { ok = 0, failed = 7 };

int main() {
  {  // each device's own number, asked once
    jagg::NumberPerDevice numbers;
    int calls[80] = {};
    for (int dev : {0, 1, 0, 63, 1, 63, 5}) {
      int n = -1;
      EXPECT(numbers.get(dev, &n, [&](int* v) { ++calls[dev]; *v = 100 + dev; return ok; }) == ok);
      EXPECT(n == 100 + dev);
    }
    EXPECT(calls[0] == 1 && calls[1] == 1 && calls[5] == 1 && calls[63] == 1);
    for (int dev : {64, -1, 64}) {  // not kept
      int n = -1;
      EXPECT(numbers.get(dev, &n, [&](int* v) { ++calls[70]; *v = 9; return ok; }) == ok && n == 9);
    }
    EXPECT(calls[70] == 3);
  }
  {  // a failure is returned, not kept, and leaves the caller's number
    jagg::NumberPerDevice numbers;
    int n = 3;
    EXPECT(numbers.get(2, &n, [](int* v) { *v = 50; return failed; }) == failed && n == 3);
    EXPECT(numbers.get(2, &n, [](int* v) { *v = 60; return ok; }) == ok && n == 60);
    EXPECT(numbers.get(2, &n, [](int* v) { *v = 70; return ok; }) == ok && n == 60);
  }
  for (int round = 0; round < 200; ++round) {
    jagg::NumberPerDevice numbers;
    std::atomic<int> bad{0};
    std::vector<std::thread> ts;
    for (int t = 0; t < 8; ++t)
      ts.emplace_back([&, t] {
        const int dev = t & 3;
        int n = 0;
        numbers.get(dev, &n, [&](int* v) { *v = 10 + dev; return ok; });
        if (n != 10 + dev) ++bad;
      });
    for (auto& t : ts) t.join();
    EXPECT(bad == 0);
  }
  return 0;
}
"""


def test_number_per_device(tmp_path):
    cxx = shutil.which("g++") or shutil.which("c++")
    if not cxx:
        pytest.skip("no host compiler")
    src, exe = tmp_path / "t.cc", tmp_path / "t"
    src.write_text(PROGRAM)
    subprocess.run([cxx, "-std=c++17", "-O1", "-pthread", "-I", CSRC, str(src), "-o", str(exe)], check=True)
    r = subprocess.run([str(exe)], capture_output=True, text=True, timeout=60)
    assert r.returncode == 0, r.stdout


def test_the_clusters_that_fit_are_asked_for_each_device():
    text = open(os.path.join(CSRC, "gemm_fp8.cu")).read()
    assert len(re.findall(r"\bcudaOccupancyMaxActiveClusters\s*\(", text)) == 1
    assert re.search(r"static NumberPerDevice known\[F_MAX_SPLITS \+ 1\];", text)
