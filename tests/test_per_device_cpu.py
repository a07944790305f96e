"""What the library keeps once for each device (kernel attributes, cluster
counts): compiled for the host with devices that are only numbers."""

import os
import re
import shutil
import subprocess

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2404_08573_gb300", "csrc")

MAIN = r"""
#include <cstdio>
#include "ff_per_device.h"
enum Err { OK = 0, FAILED = 7 };
int main() {
  ff::PerDevice<int> kept;
  int made = 0, v = -1;
  auto value = [&](int x) { return [&, x](int* p) { ++made; *p = x; return OK; }; };
  auto failure = [&](int* p) { ++made; *p = 99; return FAILED; };
  auto say = [&](Err e) { std::printf("%d:%d:%d ", (int)e, v, made); };
  say(kept.get(0, &v, value(10)));   // made
  say(kept.get(1, &v, value(11)));   // another device: made again
  say(kept.get(0, &v, value(12)));   // kept
  say(kept.get(1, &v, value(13)));   // kept
  say(kept.get(2, &v, failure));     // not kept, the value untouched
  say(kept.get(2, &v, value(14)));   // made
  say(kept.get(2, &v, failure));     // kept
  say(kept.get(1000, &v, value(15))); // beyond the table: made every time
  say(kept.get(1000, &v, value(16)));
}
"""


@pytest.mark.skipif(not shutil.which("g++"), reason="no host compiler")
def test_kept_for_each_device_and_no_failure_kept(tmp_path):
    src, exe = tmp_path / "main.cpp", tmp_path / "main"
    src.write_text(MAIN)
    subprocess.run(["g++", "-std=c++17", "-Wall", "-Werror", "-I", CSRC, str(src), "-o", str(exe), "-pthread"], check=True)
    out = subprocess.run([str(exe)], capture_output=True, text=True, check=True).stdout.split()
    assert out == ["0:10:1", "0:11:2", "0:10:2", "0:11:2", "7:11:3", "0:14:4", "0:14:4", "0:15:5", "0:16:6"]


def test_no_attribute_is_set_once_per_process():
    for name in sorted(os.listdir(CSRC)):
        text = open(os.path.join(CSRC, name)).read()
        assert not re.search(r"static (const )?\w+ \w+ =\s*\[?[^;]{0,80}cudaFuncSetAttribute", text), name
        assert not re.search(r"static const int \w+ = \[\][^;]*cuda", text), name
