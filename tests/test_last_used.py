"""The plans that a thread keeps (csrc/last_used.hpp), compiled for the host: as many as there is room for, whichever sizes they belong to."""
import os
import shutil
import subprocess

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2305_13525_amd", "csrc")
SOURCE = r"""
#include <cstdio>
#include "last_used.hpp"

static int made = 0;
template <int N>
static int64_t ask(axo::LastUsed<int64_t, N>& kept, int64_t a, int64_t b, int64_t c) {
    return kept.get(a, b, c, [&] { ++made; return a * 1000003 + b * 1009 + c; });
}
#define CHECK(x) if (!(x)) return std::printf("line %d: " #x "\n", __LINE__), 1

int main() {
    {   // a block's two problems, and those of eight blocks of other widths: multiples of 128, asked for in turn
        axo::LastUsed<int64_t, 16> kept;
        for (int turn = 0; turn < 3; ++turn)
            for (int64_t w = 1; w <= 8; ++w) {
                CHECK(ask(kept, 4096, 128 * w, 512 * w) == 4096 * 1000003LL + 128 * w * 1009 + 512 * w);
                CHECK(ask(kept, 4096, 512 * w, 128 * w) == 4096 * 1000003LL + 512 * w * 1009 + 128 * w);
            }
        CHECK(made == 16);
        ask(kept, 1, 128, 512);  // the seventeenth takes the first one's place and nobody else's
        CHECK(made == 17);
        ask(kept, 4096, 512, 128);
        CHECK(made == 17);
        ask(kept, 4096, 128, 512);
        CHECK(made == 18);
    }
    {   // empty sizes and minus ones are sizes like any other; nothing is found where nothing was made
        axo::LastUsed<int64_t, 2> kept;
        made = 0;
        CHECK(ask(kept, 0, 0, 0) == 0 && ask(kept, -1, -1, -1) == -1001013 && made == 2);
    }
    {   // what was there stays if a new value cannot be made
        axo::LastUsed<int64_t, 1> kept;
        made = 0;
        ask(kept, 1, 2, 3);
        try {
            kept.get(4, 5, 6, []() -> int64_t { throw 1; });
            CHECK(false);
        } catch (int) {
        }
        CHECK(ask(kept, 1, 2, 3) == 1000003 + 2018 + 3 && made == 1);
    }
    return 0;
}
"""


def test_last_used(tmp_path):
    cxx = shutil.which("g++") or shutil.which("c++")
    if cxx is None:
        pytest.skip("no C++ compiler")
    (tmp_path / "t.cpp").write_text(SOURCE)
    subprocess.run([cxx, "-std=c++17", "-O1", "-Wall", "-Werror", "-I", CSRC, str(tmp_path / "t.cpp"), "-o", str(tmp_path / "t")], check=True)
    r = subprocess.run([str(tmp_path / "t")], stdout=subprocess.PIPE, text=True, timeout=60)
    assert r.returncode == 0, r.stdout
