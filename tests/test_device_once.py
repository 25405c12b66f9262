"""What has to be done once on every device is done on every device, not once in the process."""
import os
import re
import subprocess

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2307_09782_b200", "csrc")


def test_device_once(tmp_path):
    src, exe = tmp_path / "t.cpp", tmp_path / "t"
    src.write_text('''
#include "device_once.h"
int main() {
  zq::DeviceOnce a, b;
  int calls = 0, fails = 1;
  auto good = [&] { ++calls; return true; };
  for (int round = 0; round < 3; ++round)
    for (int dev = 0; dev < 64; ++dev)
      if (!a.run(dev, good)) return 1;
  if (calls != 64) return 2;               // once per device
  if (!b.run(0, good) || calls != 65) return 3;  // each for itself
  auto late = [&] { ++calls; return fails-- <= 0; };
  if (b.run(1, late) || !b.run(1, late) || !b.run(1, late) || calls != 67) return 4;  // a failure is tried again, a success not
  if (!a.run(64, good) || !a.run(64, good) || calls != 69) return 5;                  // beyond what it can note: every time
  if (a.run(-1, [] { return false; })) return 6;
  return 0;
}''')
    subprocess.run(["g++", "-std=c++17", "-Wall", "-Werror", "-I", CSRC, str(src), "-o", str(exe)], check=True)
    subprocess.run([str(exe)], check=True)


def test_kernel_attributes_are_set_per_device():
    for name in os.listdir(CSRC):
        if name.endswith((".cu", ".cuh")):
            text = open(os.path.join(CSRC, name)).read()
            assert len(re.findall(r"cudaFuncSetAttribute\(", text)) == (1 if name == "zq_common.cuh" else 0), name
            for call in re.findall(r"allow_shared_memory\(\w+", text):
                assert call == "allow_shared_memory(once" or name == "zq_common.cuh"
