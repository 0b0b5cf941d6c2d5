"""The note of how much shared memory a kernel has been allowed, under threads that want different sizes at once (no GPU: the
setting call is a fake)."""
import os
import shutil
import subprocess

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2605_25655_b200", "csrc")

PROGRAM = r"""
#include <chrono>
#include <cstdio>
#include <thread>
#include "smem_opt_in.cuh"
using thinfer::SmemAllowance;
static std::atomic<int> allowed{0}, inside{0}, failed{0};
static std::atomic<bool> slow{false};
static bool allow(int bytes) {            // the device: the last setting holds
  allowed = bytes;
  ++inside;
  if (slow && bytes == 2000)              // the larger size: another setting gets every chance to come in between
    for (int i = 0; i < 200 && inside < 2; ++i) std::this_thread::sleep_for(std::chrono::milliseconds(1));
  return true;
}
int main() {
  {  // a smaller size is set while a larger one is on its way; a third in between follows
    static SmemAllowance a;
    slow = true;
    std::thread big([] { a.ensure(3, 2000, allow); });
    while (inside == 0) std::this_thread::yield();
    std::thread small([] { a.ensure(3, 1000, allow); });
    big.join();
    small.join();
    slow = false;
    if (!a.ensure(3, 1500, allow) || allowed < 1500) { std::printf("1500 bytes of %d\n", allowed.load()); return 1; }
  }
  for (int round = 0; round < 300; ++round) {   // eight threads, sizes in different orders, on two devices
    SmemAllowance a;
    std::atomic<int> on[2] = {{0}, {0}};
    std::thread t[8];
    for (int k = 0; k < 8; ++k)
      t[k] = std::thread([&, k] {
        for (int i = 0; i < 20; ++i) {
          const int dev = (i + k) & 1, want = 1 + (i * 7 + k * 13) % 101;
          const bool ok = a.ensure(dev, want, [&](int n) { on[dev] = n; return true; });
          if (!ok || on[dev] < want) ++failed;
        }
      });
    for (auto& x : t) x.join();
  }
  SmemAllowance b;                          // a refusal is not noted, a device beyond the table is asked every time
  int asked = 0;
  if (b.ensure(0, 10, [&](int) { ++asked; return false; }) || !b.ensure(0, 10, [&](int) { ++asked; return true; }) || asked != 2) return 2;
  for (int i = 0; i < 2; ++i) b.ensure(64, 5, [&](int) { ++asked; return true; });
  if (asked != 4) return 3;
  std::printf("%d\n", failed.load());
  return failed ? 4 : 0;
}
"""


def test_a_smaller_size_never_takes_back_a_larger_one(tmp_path):
    cxx = shutil.which(os.environ.get("CXX", "g++"))
    if cxx is None:
        pytest.skip("no host compiler")
    src, exe = tmp_path / "opt.cpp", tmp_path / "opt"
    src.write_text(PROGRAM)
    subprocess.run([cxx, "-std=c++17", "-O1", "-pthread", "-I", CSRC, str(src), "-o", str(exe)], check=True, timeout=300)
    got = subprocess.run([str(exe)], capture_output=True, text=True, timeout=120)
    assert got.returncode == 0, (got.returncode, got.stdout)
