"""Kernel attributes are set once for every device, not once a process: the helper, compiled by itself, and its use."""
import os
import re
import subprocess

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2609_34977_gb300", "csrc")

PROGRAM = r"""
#include "device_once.h"
#include <stdio.h>
#include <thread>
#include <vector>
int main() {
  spd::DeviceOnce once;
  int calls[70] = {};
  auto set = [&](int d, int rc) { return once.run(d, [&] { ++calls[d < 0 ? 69 : d]; return rc; }); };
  for (int k = 0; k < 3; ++k) for (int d : {0, 1, 63}) if (set(d, 0)) return 1;
  if (calls[0] != 1 || calls[1] != 1 || calls[63] != 1) return 2;
  if (set(5, 7) != 7 || set(5, 7) != 7 || set(5, 0) || set(5, 7) || calls[5] != 3) return 3;   // tried again after a failure
  if (set(64, 0) || set(64, 0) || set(-1, 0) || calls[64] != 2 || calls[69] != 1) return 4;   // beyond the table: every time
  spd::DeviceOnce shared;
  std::atomic<int> done{0}, early{0};
  std::vector<std::thread> t;
  for (int k = 0; k < 16; ++k)
    t.emplace_back([&] {
      for (int i = 0; i < 1000; ++i) {
        shared.run(3, [&] { done = 1; return 0; });
        if (!done) ++early;   // came back before the set-up was done
      }
    });
  for (auto& x : t) x.join();
  return early ? 5 : 0;
}
"""


def test_set_up_runs_once_for_every_device(tmp_path):
    src, exe = tmp_path / "once.cc", tmp_path / "once"
    src.write_text(PROGRAM)
    subprocess.run(["g++", "-std=c++17", "-O2", "-pthread", "-I", CSRC, str(src), "-o", str(exe)], check=True)
    assert subprocess.run([str(exe)]).returncode == 0


def test_attributes_of_the_answers_kernels_are_set_for_the_device_of_the_call():
    # before an attribute is set stands the device's flag, or no flag at all; never one of the process
    for name in ("tree.cu", "weights.cu", "logits.cu", "cache.cu", "attention.cu"):
        lines = open(os.path.join(CSRC, name)).read().split("\n")
        for i, line in enumerate(lines):
            if "cudaFuncSetAttribute(" in line:
                before = "\n".join(lines[max(0, i - 12):i])
                assert not re.search(r"static (bool|std::once_flag)", before), (name, i + 1)
