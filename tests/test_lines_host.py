"""What the products' warps read of lines off 16-byte boundaries, on the host: every unit that a lane asks for holds an element that is there, and every
element that is there is in a unit that some lane asks for, at its place."""
import os
import subprocess

import pytest

from paper_2607_19058_gb300 import _build

PROGRAM = r"""
#include <cstdio>
#include <cstdlib>
#include <map>

#include "skew_lines.h"

using namespace skew;

static uint16_t memory[1 << 16];
static long reads = 0;

static int fail(const char *what, int from, int lane, int64_t lines, int64_t elements) {
    std::printf("%s: lines from %d on, lane %d, of %ld lines of %ld elements\n", what, from, lane, long(lines), long(elements));
    return 1;
}

// One warp's lines of the stages of a tile whose operand has `outer` lines (MAJOR) of the summed index `summed`, or `summed` lines of `outer` elements; the tile
// starts at l0 of `outer`.
template <bool MAJOR, int N>
int warp(int start, int64_t ld, int64_t l0, int64_t outer, int64_t summed, int from) {
    const uint16_t *const p = memory + 8192 + start;
    const int64_t rows = MAJOR ? outer : summed, columns = MAJOR ? summed : outer;
    for (int64_t s0 = 0; s0 < summed; s0 += 64) {
        std::map<uint32_t, uintptr_t> got;
        for (int lane = 0; lane < 32; ++lane) {
            Lines<MAJOR, N> lines(p, ld, l0, outer, 0, summed, from, lane);
            for (int64_t s = 0; s < s0; s += 64) lines.next();
            bool ok = true;
            lines.units(lane, [&](uint32_t to, const char *at, bool there) {
                if (!there) return;
                ++reads;
                const uintptr_t a = reinterpret_cast<uintptr_t>(at);
                if (a % 16 || to % 16 || to >= uint32_t(N) * kRawLine) ok = false;
                bool holds = false;  // an element that is there
                for (int64_t i = 0; i < 8; ++i) {
                    const int64_t e = int64_t(a / 2) + i - int64_t(reinterpret_cast<uintptr_t>(p) / 2);
                    if (e >= 0 && e / ld < rows && e % ld < columns) holds = true;
                }
                if (!holds) ok = false;
                got[to] = a;
            });
            if (!ok) return fail("a unit without an element", from, lane, rows, columns);
        }
        for (int i = 0; i < N; ++i)
            for (int j = 0; j < 64; ++j) {
                const int line = from + i;
                const int64_t row = MAJOR ? l0 + line : s0 + line % 64, column = MAJOR ? s0 + j : l0 + line / 64 * 64 + j;
                if (row >= rows || column >= columns) continue;
                const uintptr_t first = reinterpret_cast<uintptr_t>(p + row * ld + column - j), a = first + 2 * j;
                const auto it = got.find(uint32_t(i * kRawLine + (a / 16 - first / 16) * 16));
                if (it == got.end() || it->second != a / 16 * 16) return fail("an element that no lane reads", from, i, rows, columns);
            }
    }
    return 0;
}

template <bool MAJOR, int N>
int all() {
    const int64_t summed[] = {1, 2, 7, 8, 57, 63, 64, 65, 127, 130};
    for (int64_t outer = 1; outer <= 260; outer += outer < 40 ? 1 : outer < 250 ? 7 : 1)
        for (int64_t k : summed)
            for (int64_t more : {0, 1, 2, 5, 8}) {
                const int64_t ld = (MAJOR ? k : outer) + more;
                if (ld * (MAJOR ? outer : k) > 32768) continue;
                for (int start : {0, 1, 3, 7})
                    for (int64_t l0 : {0, 128})
                        for (int from = 0; from < kOperandLines; from += N)
                            if (int rc = warp<MAJOR, N>(start, ld, l0, outer, k, from)) return rc;
            }
    return 0;
}

int main(int, char **which) {
    int rc = 0;
    switch (std::atoi(which[1])) {
        case 0: rc = all<true, 16>(); break;
        case 1: rc = all<true, 32>(); break;
        case 2: rc = all<false, 16>(); break;
        case 3: rc = all<false, 32>(); break;
    }
    if (!rc) std::printf("%ld\n", reads);
    return rc;
}
"""


@pytest.fixture(scope="module")
def program(tmp_path_factory):
    d = tmp_path_factory.mktemp("lines")
    src, exe = d / "lines.cpp", d / "lines"
    src.write_text(PROGRAM)
    subprocess.check_call(["g++", "-O1", "-std=c++17", "-I", _build.CSRC, str(src), "-o", str(exe)])
    return str(exe)


@pytest.mark.parametrize("which", range(4), ids=["along-16", "along-32", "across-16", "across-32"])
def test_every_unit_that_is_read_holds_an_element(program, which):
    r = subprocess.run([program, str(which)], capture_output=True, text=True)
    assert r.returncode == 0, r.stdout
    assert int(r.stdout) > 10000
