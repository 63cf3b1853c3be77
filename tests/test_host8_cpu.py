"""Host-side arithmetic of the 8-bit layers (csrc/ff_host.h), compiled alone."""

import os
import shutil
import subprocess

import pytest

from .conftest import ROOT

CSRC = os.path.join(ROOT, "paper_2607_27842_gb300", "csrc")


def run_cpp(tmp_path, body):
    if shutil.which("g++") is None:
        pytest.skip("no g++")
    src, exe = tmp_path / "t.cpp", tmp_path / "t"
    src.write_text('#include <cstdio>\n#include <vector>\n#include "ff_host.h"\n' + body)
    subprocess.run(["g++", "-std=c++17", "-O1", "-fsanitize=undefined", "-fno-sanitize-recover", "-pthread", "-I", CSRC, str(src),
                    "-o", str(exe)], check=True)
    return subprocess.run([str(exe)], check=True, capture_output=True, text=True).stdout.split()


# sizes up to the largest dimension the operators take (2^31 - 256), and steps whose
# multiples pass 2^31 behind it
@pytest.mark.parametrize("total,step", [(1, 16384), (16384, 16384), (16385, 16384), (0x7fffc000, 16384), (0x7fffc001, 16384),
                                        (0x7fffff00, 16384), (0x7fffff00, 65535 * 128)])
def test_runs_cover_everything_once(tmp_path, total, step):
    out = run_cpp(tmp_path, """
int main() {
  long long end = 0, n = 0, bad = 0;
  ff::for_runs(%dll, %dll, [&](long long at, long long k) {
    bad += at != end || k < 1 || k > %dll;
    end = at + k;
    return ++n > 1000000 ? 1 : 0;
  });
  printf("%%lld %%lld %%lld", end, n, bad);
}""" % (total, step, step))
    assert [int(v) for v in out] == [total, -(-total // step), 0]


def test_runs_stop_at_the_first_failure(tmp_path):
    out = run_cpp(tmp_path, """
int main() {
  int n = 0;
  const int r = ff::for_runs(100, 10, [&](long long, long long) { return ++n == 3 ? 7 : 0; });
  printf("%d %d", n, r);
}""")
    assert out == ["3", "7"]


def test_every_device_is_prepared_once(tmp_path):
    """Each device has its value made on its own first call, by one of several threads;
    a preparation that failed is tried again."""
    out = run_cpp(tmp_path, """
#include <thread>
int main() {
  static ff::PerDevice<int> d;
  std::atomic<int> made[3] = {};
  auto get = [&](int dev, int* v) { return d.get(dev, v, [&](int& x) { x = 100 + dev; return ++made[dev] == 1 && dev == 2 ? 5 : 0; }); };
  int v = -1, failed = get(2, &v);
  printf("%d %d ", failed, v);
  std::vector<std::thread> t;
  std::atomic<int> wrong{0};
  for (int i = 0; i < 8; ++i)
    t.emplace_back([&] { for (int k = 0; k < 300; ++k) { int x = 0; if (get(k % 3, &x) || x != 100 + k % 3) ++wrong; } });
  for (auto& x : t) x.join();
  printf("%d %d %d %d", wrong.load(), made[0].load(), made[1].load(), made[2].load());
}""")
    assert out == ["5", "-1", "0", "1", "1", "2"]
