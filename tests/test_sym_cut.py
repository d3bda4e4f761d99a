"""How the tiles of a symmetric product are dealt out (csrc/sym_cut.hpp), compiled on its own: every step of every tile is some workgroup's, once, and no two parts leave
their sums in one place."""
import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CODE = r"""
#include <cstdio>
#include <cstdlib>
#include <set>
#include <vector>
#include "sym_cut.hpp"

#define CHECK(x) do { if (!(x)) { std::printf("%s: %ld rows, %ld steps, %ld units\n", #x, s, steps, units); std::exit(1); } } while (0)

static void check(long s, long steps, long units, axo::SymPlan plan, const axo::SymCut& c, long tiles) {
    CHECK(c.steps == steps && c.whole + c.cut == tiles && plan.workgroups >= 1 && plan.workgroups <= 2 * units);
    std::vector<std::vector<char>> done(tiles, std::vector<char>(steps, 0));
    std::vector<int> parts(tiles, 0), last(tiles, -1);
    std::set<int> slots;
    long most = 0, all = 0;
    for (int id = 0; id < plan.workgroups; ++id) {
        axo::SymWalk walk(c, id, plan.workgroups);
        axo::SymPart p;
        long mine = 0;
        while (walk.next(c, p)) {
            CHECK(p.tile >= 0 && p.tile < tiles && p.count >= 1 && p.from >= 0 && p.from + p.count <= steps);
            for (int i = p.from; i < p.from + p.count; ++i) CHECK(!done[p.tile][i]++);
            mine += p.count;
            ++parts[p.tile];
            if (p.cut < 0) { CHECK(p.count == steps); continue; }
            CHECK(p.cut < c.cut && p.tile == c.whole + p.cut && p.parts == c.parts_of(p.cut) && p.parts <= 20);
            CHECK(p.slot >= 0 && p.slot < c.slots() && slots.insert(p.slot).second);
            // the parts of a tile are numbered in the order of their steps
            int number = -1;
            for (int i = 0; i < p.parts; ++i)
                if (c.slot_of(p.cut, i) == p.slot) number = i;
            CHECK(number >= 0);
            if (number == 0) CHECK(p.from == 0);
            if (number == p.parts - 1) CHECK(p.from + p.count == steps);
        }
        most = mine > most ? mine : most;
        all += mine;
    }
    for (long t = 0; t < tiles; ++t) {
        for (char d : done[t]) CHECK(d == 1);
        CHECK(parts[t] == (t < c.whole ? 1 : c.parts_of((int)(t - c.whole))));
    }
    CHECK(all == tiles * steps);
}

static long halves = 0;
static void check(long s, long steps, long units, axo::SymPlan plan) {
    if (plan.size == axo::SYM_HALF) {  // 256 x 128 tiles of which the i-th 256 rows have 2 i + 1, and the diagonal's others
        const long n = (s + 255) / 256;
        long diagonal = 0;
        for (long i = 0; i < n; ++i) diagonal += i * 256 + 128 < s;
        check(s, steps, units, plan, plan.cut, n * n);
        check(s, steps, units, plan, plan.diagonal, diagonal);
        CHECK(plan.counters() == plan.cut.cut + plan.diagonal.cut);
        CHECK(plan.partial_floats() == plan.diagonal.slots() * 128L * 128 && plan.cut.cut == 0);
        ++halves;
        return;
    }
    const long n = (s + plan.size - 1) / plan.size;
    check(s, steps, units, plan, plan.cut, n * (n + 1) / 2);
}

int main() {
    long n = 0;
    for (long units : {256, 7}) {
        for (long s : {1, 64, 128, 192, 576, 640, 1024, 1088, 1536, 2048, 2112, 3904, 4032, 4096, 4160, 5696})
            for (long steps : {1, 2, 3, 7, 9, 16, 17, 32, 33, 64, 100, 255, 256}) {
                if (units == 7 && s > 1100) continue;
                const axo::SymPlan plan = axo::sym_plan(s, steps, units);
                check(s, steps, units, plan);
                CHECK(plan.counters() <= axo::SYM_MOST_CUT);
                ++n;
            }
        for (long cut = 1; cut < units; cut += units > 100 ? 5 : 1)  // slices and rests of any proportion, whether they are planned or not
            for (long steps : {1, 2, 5, 16, 33, 64}) {
                const long s = 64, most = units, q = most / cut, each = (cut * steps + most - 1) / most, helpers = most - q * cut, rest = steps - q * each;
                if (helpers == 0 || rest <= 0) continue;
                const long further = cut > helpers ? (cut - helpers) * rest : 0, share = further > 0 ? (further + helpers - 1) / helpers : 1;
                if (q + (further > 0 ? rest / share + 2 : 1) > 16) continue;
                long side = 1;
                while (side * (side + 1) / 2 < cut) ++side;
                if (side * (side + 1) / 2 != cut) continue;
                axo::SymPlan plan;
                plan.size = 1;
                plan.workgroups = (int)most;
                plan.cut = {(int)steps, 0, (int)cut, (int)q, (int)each, (int)rest, (int)helpers, (int)share};
                check(side, steps, units, plan);
                (void)s;
                ++n;
            }
    }
    std::printf("%ld plans, %ld with tiles of 256 x 128\n", n, halves);
    return n > 200 && halves > 0 ? 0 : 2;
}
"""


def test_every_step_once(tmp_path):
    cxx = shutil.which("g++") or shutil.which("clang++")
    if not cxx:
        pytest.skip("no C++ compiler")
    (tmp_path / "t.cpp").write_text(CODE)
    subprocess.run([cxx, "-std=c++17", "-O1", "-I" + os.path.join(ROOT, "paper_2305_13525_amd", "csrc"), str(tmp_path / "t.cpp"), "-o", str(tmp_path / "t")], check=True)
    r = subprocess.run([str(tmp_path / "t")], stdout=subprocess.PIPE, text=True, timeout=120)
    assert r.returncode == 0, r.stdout
