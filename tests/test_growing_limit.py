"""The limit on a kernel's shared memory that several threads raise on their first calls (csrc/grow.h), compiled by itself and without a GPU."""
import os
import subprocess

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

PROGRAM = r"""
#include <chrono>
#include <cstdio>
#include <thread>
#include <vector>
#include "grow.h"

static void nap(int ms) { std::this_thread::sleep_for(std::chrono::milliseconds(ms)); }

int main()
{
    // the larger request sets the limit and is slow to return; the smaller one comes meanwhile
    {
        wcc::GrowingLimit g;
        std::atomic<int> limit{0}, calls{0};
        std::thread large([&] { if (!g.raise(110, [&](int n) { ++calls; limit = n; nap(200); return true; })) std::printf("refused "); });
        while (!calls) nap(1);
        std::thread small([&] { if (!g.raise(60, [&](int n) { ++calls; limit = n; return true; })) std::printf("refused "); });
        large.join();
        small.join();
        const bool known = g.raise(110, [&](int) { return false; });      // no further setting: it is known
        std::printf("%d %d ", limit.load(), (int)known);
    }
    // any order, many threads: whoever returns finds the limit at what it asked for, then and later
    {
        int bad = 0;
        for (int round = 0; round < 50; ++round) {
            wcc::GrowingLimit g;
            std::atomic<int> limit{0}, low{0};
            std::vector<std::thread> all;
            for (int i = 0; i < 8; ++i)
                all.emplace_back([&, i] {
                    for (int k = 0; k < 20; ++k) {
                        const int want = 1 + (i * 37 + k * 11) % 101;
                        g.raise(want, [&](int n) { limit = n; std::this_thread::yield(); return true; });
                        if (limit < want) ++low;
                    }
                });
            for (auto& t : all) t.join();
            bad += low;
        }
        std::printf("%d ", bad);
    }
    // a setting that fails is not recorded
    {
        wcc::GrowingLimit g;
        const bool first = g.raise(10, [](int) { return false; }), second = g.raise(10, [](int) { return true; });
        std::printf("%d %d\n", (int)first, (int)second);
    }
}
"""


def test_the_limit_only_grows(tmp_path):
    src, exe = tmp_path / "grow.cpp", tmp_path / "grow"
    src.write_text(PROGRAM)
    subprocess.check_call(["g++", "-std=c++17", "-O1", "-pthread", "-I", os.path.join(ROOT, "paper_2205_12268_b200", "csrc"), str(src), "-o", str(exe)])
    out = subprocess.run([str(exe)], capture_output=True, text=True, timeout=60)
    assert out.returncode == 0 and out.stdout.split() == ["110", "1", "0", "0", "1"], out.stdout


def test_kernels_limits_are_raised_through_it():
    text = open(os.path.join(ROOT, "paper_2205_12268_b200", "csrc", "common.cuh")).read()
    body = text[text.index("static wcc_status allow_smem"):]
    assert "GrowingLimit" in body[:body.index("\n}\n")]
