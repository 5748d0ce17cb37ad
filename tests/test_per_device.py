"""What the library finds out once for each device (per_device.h), on the host with devices that are only numbers."""
import os
import shutil
import subprocess

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2608_07974_gb300", "csrc")

PROGRAM = r"""
#include "per_device.h"
#include <cstdio>
#include <thread>
#include <vector>
#define CHECK(x) if (!(x)) { std::printf("line %d: %s\n", __LINE__, #x); return 1; }
struct Value { int dev = -1; };
int main() {
  static zl::PerDevice<Value> all;
  // a device's value is its own, and found out once however many threads ask first
  static std::atomic<int> made[3];
  std::vector<std::thread> threads;
  std::atomic<int> wrong{0};
  for (int i = 0; i < 24; ++i)
    threads.emplace_back([&, i] {
      const int dev = i % 3;
      const Value* v = all.get(dev, [&](Value& x) {
        made[dev]++;
        std::this_thread::sleep_for(std::chrono::milliseconds(20));
        x.dev = dev;
        return true;
      });
      if (!v || v->dev != dev) wrong++;
    });
  for (auto& t : threads) t.join();
  CHECK(wrong == 0);
  for (auto& m : made) CHECK(m == 1);
  // a failure is not kept
  int tries = 0;
  auto second = [&](Value& x) { x.dev = 7; return ++tries > 1; };
  CHECK(all.get(7, second) == nullptr);
  CHECK(all.get(7, second) && all.get(7, second)->dev == 7 && tries == 2);
  // numbers that are no device
  CHECK(all.get(-1, second) == nullptr && all.get(64, second) == nullptr && tries == 2);
  std::puts("ok");
}
"""


def test_every_device_is_asked_once(tmp_path):
    cxx = shutil.which("g++")
    if not cxx:
        pytest.skip("no g++")
    src, exe = tmp_path / "per_device.cpp", tmp_path / "per_device"
    src.write_text(PROGRAM)
    r = subprocess.run([cxx, "-std=c++17", "-O1", "-pthread", "-I", CSRC, str(src), "-o", str(exe)], capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
    r = subprocess.run([str(exe)], capture_output=True, text=True, timeout=60)
    assert r.returncode == 0 and "ok" in r.stdout, r.stdout + r.stderr
