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
