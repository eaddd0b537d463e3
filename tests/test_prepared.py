"""What a kernel needs once on each device is done once, however many kernels and devices there are: the set that
remembers it, compiled by itself for the host."""
import os
import subprocess

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2608_26004_gb300", "csrc")

PROGRAM = r"""
#include <cstdio>
#include <thread>
#include <vector>

#include "prepared.h"

int main() {
  static asymspec_impl::Prepared all;
  static char kernels[300];
  int calls = 0, failed = 0;
  for (int round = 0; round < 3; ++round)
    for (int device = 0; device < 8; ++device)
      for (char& k : kernels)
        if (all.once(&k, device, [&] { return ++calls, 0; }) != 0) return 1;
  // what failed is tried again, and its error returned
  static char other;
  for (int i = 0; i < 3; ++i)
    if (all.once(&other, 0, [&] { return ++failed, i < 2 ? 7 : 0; }) != (i < 2 ? 7 : 0)) return 2;
  if (all.once(&other, 0, [] { return 9; }) != 0) return 3;
  // threads that meet at a kernel's first call
  static asymspec_impl::Prepared shared;
  std::atomic<int> together{0};
  std::vector<std::thread> threads;
  for (int t = 0; t < 8; ++t)
    threads.emplace_back([&] {
      for (int device = 0; device < 8; ++device)
        for (char& k : kernels) shared.once(&k, device, [&] { return ++together, 0; });
    });
  for (std::thread& t : threads) t.join();
  std::printf("%d %d %d\n", calls, failed, together.load());
  return 0;
}
"""


def test_each_kernel_and_device_once(tmp_path):
    source, program = tmp_path / "prepared.cc", tmp_path / "prepared"
    source.write_text(PROGRAM)
    subprocess.run(["g++", "-std=c++17", "-O1", "-pthread", "-I" + CSRC, str(source), "-o", str(program)], check=True)
    done = subprocess.run([str(program)], capture_output=True, text=True, timeout=60)
    assert done.returncode == 0 and done.stdout.split() == ["2400", "3", "2400"]
