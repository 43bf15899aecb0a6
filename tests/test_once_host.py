"""Set-up that kernels need once per device (csrc/once.cuh, compiled here by itself), from several threads: none of them goes on before it is done."""
import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_1707_04585_b200", "csrc")

PROGRAM = r"""
#include "once.cuh"
#include <stdio.h>
#include <chrono>
#include <thread>
#include <vector>

// set() as cudaFuncSetAttribute: what it sets holds from some time after its start
static std::atomic<int> limit{0}, calls{0}, early{0};
static bool set() { calls++; std::this_thread::sleep_for(std::chrono::milliseconds(30)); limit = 227; return true; }

int main() {
    static OncePerDevice once;
    std::vector<std::thread> all;
    for (int i = 0; i < 8; i++) all.emplace_back([i] {
        std::this_thread::sleep_for(std::chrono::milliseconds(4 * i));       // the later ones while the first one's call is under way
        if (!once.ensure(0, set) || limit != 227) early++;                   // a launch in here would fail
    });
    for (auto &t : all) t.join();
    const int first = calls;
    for (int i = 0; i < 10; i++) once.ensure(0, set);
    static OncePerDevice again;
    int tries = 0;
    const bool a = again.ensure(3, [&] { tries++; return false; }), b = again.ensure(3, [&] { tries++; return true; }), c = again.ensure(3, [&] { tries++; return false; });
    const bool d = again.ensure(4, [&] { tries++; return true; });           // another device
    const bool e = again.ensure(64, [&] { tries++; return true; }) && again.ensure(64, [&] { tries++; return true; });         // beyond what is remembered: every time
    printf("%d %d %d %d %d %d %d %d %d\n", (int)early, calls == first, first >= 1, a, b, c, d, e, tries);
    return 0;
}
"""


def test_no_thread_goes_on_before_the_set_up_is_done(tmp_path):
    if shutil.which("g++") is None:
        pytest.skip("no g++")
    src, exe = tmp_path / "once.cpp", tmp_path / "once"
    src.write_text(PROGRAM)
    subprocess.run(["g++", "-std=c++17", "-O1", "-pthread", "-I", CSRC, "-x", "c++", str(src), "-o", str(exe)], check=True)
    out = subprocess.run([str(exe)], check=True, capture_output=True, text=True).stdout.split()
    assert [int(v) for v in out] == [0, 1, 1, 0, 1, 1, 1, 1, 5]
