"""A kernel's one-time setup (its shared-memory limit) is each device's own: the
flags that say where it has been done, and that each launch site uses them."""
import os
import shutil
import subprocess

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2606_12950_gb300", "csrc")

PROGRAM = r"""
#include "device_flags.h"
#include <initializer_list>
int main()
{
    static kvp::DeviceFlags f;
    for (int d : {0, 1, 5, 63, 64, 1000, -1})
        if (f.has(d)) return 1;
    f.set(1);
    f.set(63);
    f.set(64);   // more than it has flags for: never set, the setup is done again
    f.set(-1);
    for (int d = -2; d < 200; ++d)
        if (f.has(d) != (d == 1 || d == 63)) return 2;
    f.set(0);
    return f.has(0) && f.has(1) && !f.has(2) ? 0 : 3;
}
"""


def test_flags_of_devices(tmp_path):
    gxx = shutil.which("g++")
    if gxx is None:
        pytest.skip("no g++")
    src, exe = tmp_path / "flags.cpp", tmp_path / "flags"
    src.write_text(PROGRAM)
    subprocess.run([gxx, "-std=c++17", "-I", CSRC, "-o", str(exe), str(src)], check=True)
    assert subprocess.run([str(exe)]).returncode == 0


def test_every_attribute_is_set_under_a_devices_flag():
    found = 0
    for name in sorted(os.listdir(CSRC)):
        with open(os.path.join(CSRC, name)) as f:
            text = f.read()
        if "cudaFuncSetAttribute(" not in text:
            continue
        found += 1
        assert text.count("static DeviceFlags") + text.count("static kvp::DeviceFlags") >= 1, name
        assert "atomic<bool> attr_set" not in text, name
    assert found >= 2
