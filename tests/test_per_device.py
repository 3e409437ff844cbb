"""What is done once a device is done on each device: a process may use several."""
import os
import re
import subprocess

CSRC = os.path.join(os.path.dirname(__file__), "..", "paper_2110_06037_gb300", "csrc")

PROGRAM = r"""
#include <cassert>
#include <initializer_list>
#include "per_device.h"
int main() {
    sn::PerDevice a, b;
    int calls = 0;
    auto good = [&] { ++calls; return 0; };
    auto bad = [&] { ++calls; return 7; };
    assert(a.once(0, good) == 0 && a.once(0, good) == 0 && calls == 1);   // once on device 0
    assert(a.once(1, good) == 0 && calls == 2);                           // and once on device 1
    assert(a.once(63, good) == 0 && a.once(63, good) == 0 && calls == 3);
    assert(b.once(0, good) == 0 && calls == 4);                           // of its own
    assert(b.once(2, bad) == 7 && b.once(2, bad) == 7 && calls == 6);     // what failed is tried again
    assert(b.once(2, good) == 0 && b.once(2, bad) == 0 && calls == 7);
    for (int dev : {64, 65, -1}) assert(a.once(dev, good) == 0 && a.once(dev, good) == 0);
    assert(calls == 13);                                                  // no record of such a device: every time
}
"""


def test_once_a_device(tmp_path):
    src, exe = tmp_path / "t.cpp", tmp_path / "t"
    src.write_text(PROGRAM)
    subprocess.run(["g++", "-std=c++17", "-I", CSRC, str(src), "-o", str(exe)], check=True)
    subprocess.run([str(exe)], check=True)


def test_the_block_operators_set_no_attribute_once_a_process():
    """Their front end calls them on the device of the tensors, whichever that is."""
    seen = 0
    for name in ("kernels_norm.cu", "kernels_q4.cu", "q4_few.cuh", "kernels_q4_tc.cu", "kernels_ssm.cu", "kernels_ssm_tc.cu"):
        text = re.sub(r"//[^\n]*", "", open(os.path.join(CSRC, name)).read())
        assert "cudaFuncSetAttribute" not in text and not re.search(r"static (bool|size_t|int) \w+ *=", text), name
        seen += len(re.findall(r"allow_smem\(", text))
    assert seen >= 4
