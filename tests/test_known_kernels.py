"""What a thread remembers of the kernels that it has launched (csrc/rt_known.h): all that the library has, on several devices, and never an endless search."""
import os
import subprocess

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

PROGRAM = r"""
#include <cstdio>
#include <initializer_list>
#include "rt_known.h"

static char code[1 << 20];                                          // addresses as kernels have them: 16, 128 or 4096 bytes apart

int main() {
  for (int apart : {16, 128, 4096}) {
    static rt::KnownKernels k;
    k = rt::KnownKernels();
    for (int i = 0; i < 240; ++i)
      for (int dev = 0; dev < 3; ++dev) {
        rt::KnownKernels::Entry* e = k.at(code + i * apart, dev);
        if (e->fn) return 1;                                        // not there yet
        k.put(e, code + i * apart, dev, 1000 * dev + i);
      }
    for (int i = 0; i < 240; ++i)
      for (int dev = 0; dev < 3; ++dev) {
        const rt::KnownKernels::Entry* e = k.at(code + i * apart, dev);
        if (e->fn != code + i * apart || e->dev != dev || e->bytes != 1000 * dev + i) return 2;
      }
    for (int i = 0; i < 2000; ++i) {                                // more than it holds: those are not remembered
      rt::KnownKernels::Entry* e = k.at(code + 500000 + 8 * i, 7);
      if (!e->fn) k.put(e, code + 500000 + 8 * i, 7, 1);
    }
    if (k.used != rt::KnownKernels::kMost || k.at(code, 9)->fn) return 3;
    for (int i = 0; i < 240; ++i) if (k.at(code + i * apart, 1)->bytes != 1000 + i) return 4;
  }
  puts("ok");
}
"""


def test_every_kernel_is_remembered(tmp_path):
    src, exe = tmp_path / "known.cpp", tmp_path / "known"
    src.write_text(PROGRAM)
    subprocess.run(["g++", "-std=c++17", "-O1", "-I", os.path.join(ROOT, "paper_2604_21215_b200", "csrc"), "-o", str(exe), str(src)], check=True)
    r = subprocess.run([str(exe)], capture_output=True, text=True, timeout=60)
    assert r.returncode == 0 and r.stdout.split() == ["ok"], r.returncode
