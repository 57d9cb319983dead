"""csrc/per_device.h, compiled for the host: what is asked of the driver is kept per device, and a failed question is not kept."""
import os
import subprocess

from paper_2406_11257_b200 import build

PROGRAM = r"""
#include "per_device.h"
#include <cstdio>
static excp::PerDevice<9> room;
static unsigned asked = 0;
static void show(int device, unsigned key, unsigned answer) {
    const unsigned n = room.get(device, key, [&] { ++asked; return answer; });
    std::printf("%u %u\n", n, asked);
}
int main() {
    show(0, 4, 132);        // asked
    show(0, 4, 7);          // kept
    show(1, 4, 96);         // another device has its own
    show(0, 8, 128);        // and another key
    show(0, 4, 7);
    show(2, 4, 0);          // failed
    show(2, 4, 140);        // asked again
    show(2, 4, 0);
    show(64, 4, 5);         // past the last device: never kept
    show(64, 4, 6);
}
"""


def test_numbers_are_kept_per_device(tmp_path):
    (tmp_path / "main.cpp").write_text(PROGRAM)
    exe = str(tmp_path / "main")
    subprocess.check_call([os.environ.get("CXX", "g++"), "-std=c++17", "-Wall", "-Werror", "-I" + build.CSRC, str(tmp_path / "main.cpp"), "-o", exe])
    lines = [tuple(map(int, l.split())) for l in subprocess.check_output([exe], text=True).splitlines()]
    assert lines == [(132, 1), (132, 1), (96, 2), (128, 3), (132, 3), (0, 4), (140, 5), (140, 5), (5, 6), (6, 7)]


def test_the_product_asks_per_device():
    """No count of its own that all devices share; plans are kept per device."""
    text = open(os.path.join(build.CSRC, "product.cu")).read()
    assert "PerDevice<" in text and "known[MAX_SPLIT + 1]" not in text
