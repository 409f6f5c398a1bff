"""The host code that prepares a kernel once on every device (csrc/device_once.hpp), built as plain C++: the second
device that a process uses is prepared as the first one was."""
import os
import subprocess

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
PROGRAM = r"""
#include "device_once.hpp"
#include <cstdio>
#include <thread>
#include <vector>
int main() {
  hyenand::DeviceOnce once;
  int runs = 0, fail = 0;
  auto on = [&](int device) { return once(device, [&] { ++runs; return fail; }); };
  auto expect = [&](const char* what, int got_runs, int device, int got) {
    runs = 0;
    const int e = on(device);
    if (runs != got_runs || e != got) { std::printf("%s: %d runs, result %d\n", what, runs, e); std::exit(1); }
  };
  expect("first device", 1, 0, 0);
  expect("first device again", 0, 0, 0);
  expect("second device", 1, 1, 0);
  expect("last device of the mask", 1, 63, 0);
  expect("both again", 0, 1, 0);
  fail = 7;
  expect("a failure is told", 1, 2, 7);
  expect("and told again", 1, 2, 7);
  expect("of its device alone", 0, 0, 0);
  fail = 0;
  expect("and tried again", 1, 2, 0);
  expect("until it succeeds", 0, 2, 0);
  expect("devices beyond the mask: each time", 1, 64, 0);
  expect("devices beyond the mask: each time", 1, 64, 0);
  std::atomic<int> many{0};
  hyenand::DeviceOnce shared;
  std::vector<std::thread> threads;
  for (int i = 0; i < 8; ++i)
    threads.emplace_back([&, i] { for (int k = 0; k < 1000; ++k) if (shared(i % 4, [&] { ++many; return 0; })) std::exit(2); });
  for (auto& t : threads) t.join();
  if (many < 4 || many > 8) { std::printf("%d runs on four devices\n", many.load()); return 3; }
  return 0;
}
"""


def test_once_on_every_device(tmp_path):
    src, exe = tmp_path / "once.cpp", tmp_path / "once"
    src.write_text("#include <cstdlib>\n" + PROGRAM)
    subprocess.run(["g++", "-O1", "-std=c++17", "-Wall", "-Werror", "-pthread", "-I",
                    os.path.join(ROOT, "paper_2607_19378_amd", "csrc"), "-o", str(exe), str(src)], check=True)
    run = subprocess.run([str(exe)], capture_output=True, text=True, timeout=60)
    assert run.returncode == 0, run.stdout


def test_no_attribute_is_set_for_the_first_device_alone():
    """Every dynamic LDS limit goes through it."""
    csrc = os.path.join(ROOT, "paper_2607_19378_amd", "csrc")
    users = [f for f in sorted(os.listdir(csrc)) if f.endswith((".hip", ".hpp")) and "hipFuncSetAttribute(" in open(os.path.join(csrc, f)).read()]
    assert users == ["kernels.hpp"]
