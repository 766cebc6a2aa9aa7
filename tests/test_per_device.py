"""What the library looks up once per device (csrc/per_device.h), from many host threads at once: compiled by the host compiler
with its thread sanitizer, no device needed."""
import os
import shutil
import subprocess

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2511_04063_b200", "csrc")
PROGRAM = r"""
#include "per_device.h"
#include <cstdio>
#include <thread>
#include <vector>
struct Found { int index = 0, sms = 0; const int* status = nullptr; long rest[13] = {}; };
int main() {
  static const int word = 0;
  std::atomic<int> wrong{0}, asked{0};
  for (int round = 0; round < 40; ++round) {
    dq::PerDevice<Found> known;
    std::atomic<int> waiting{0};
    std::vector<std::thread> threads;
    for (int t = 0; t < 8; ++t)
      threads.emplace_back([&] {
        waiting.fetch_add(1, std::memory_order_relaxed);
        while (waiting.load(std::memory_order_relaxed) < 8) {}
        for (int device = 0; device < dq::MAX_DEVICES; ++device) {
          Found f;
          const int error = known.get(device, f, [&](Found& v) {
            asked.fetch_add(1, std::memory_order_relaxed);
            v.index = device; v.sms = 148; v.status = &word;
            for (long& r : v.rest) r = device + 1;
            return 0;
          });
          bool right = error == 0 && f.index == device && f.sms == 148 && f.status == &word;
          for (long r : f.rest) right = right && r == device + 1;
          if (!right) wrong.fetch_add(1, std::memory_order_relaxed);
        }
      });
    for (auto& t : threads) t.join();
  }
  dq::PerDevice<Found> known;      // an error is handed on and not kept
  Found f;
  if (known.get(3, f, [](Found&) { return 5; }) != 5 || known.get(3, f, [](Found& v) { v.sms = 1; return 0; }) != 0 || f.sms != 1 ||
      known.get(3, f, [](Found&) { return 5; }) != 0)
    wrong.fetch_add(1, std::memory_order_relaxed);
  std::printf("wrong %d asked %d\n", wrong.load(), asked.load());
  return wrong.load() != 0;
}
"""


@pytest.mark.parametrize("sanitizer", [[], ["-fsanitize=thread"]])
def test_first_calls_of_many_threads_see_whole_values(tmp_path, sanitizer):
    source, binary = tmp_path / "threads.cpp", tmp_path / "threads"
    source.write_text(PROGRAM)
    for compiler in (os.environ.get("CXX"), "g++"):          # (not every compiler comes with the sanitizer)
        if not compiler or not shutil.which(compiler):
            continue
        built = subprocess.run([compiler, "-O2", "-std=c++17", "-pthread", "-I", CSRC, *sanitizer, str(source), "-o", str(binary)],
                               capture_output=True, text=True)
        if built.returncode == 0:
            break
    if built.returncode != 0 and "tsan" in built.stderr:
        pytest.skip("no compiler with a thread sanitizer")
    assert built.returncode == 0, built.stderr
    # (the sanitizer wants its addresses where they are without randomisation)
    fixed = [shutil.which("setarch"), "-R"] if shutil.which("setarch") and sanitizer else []
    ran = subprocess.run([*fixed, str(binary)], capture_output=True, text=True, timeout=300)
    if sanitizer and "unexpected memory mapping" in ran.stderr:
        pytest.skip("the thread sanitizer does not run under this kernel")
    assert ran.returncode == 0, ran.stdout + ran.stderr[-3000:]
    assert "wrong 0 asked %d\n" % (40 * 64) in ran.stdout
