"""Sizes for every way in which the symmetric products of the orthogonalised update are dealt out, and what tells on the host that they still are."""
import os
import shutil
import subprocess

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

# What a plan is called: rows of its tiles (SYM_HALF: 256 x 128 ones), workgroups' whole tiles (none, one, many), and how those that are left are cut: not, into equal slices, with a rest that
# goes to a helper of its own, or with rests of which helpers share further ones.
PLANS = r"""
#include <cstdio>
#include <cstring>
#include <set>
#include <string>
#include "sym_cut.hpp"

static const char* cut_of(const axo::SymCut& c) { return !c.cut ? "whole" : c.rest == 0 ? "slices" : c.helpers == c.cut ? "own" : "shared"; }
static std::string name(long s, long steps) {
    const axo::SymPlan p = axo::sym_plan(s, steps, 256);
    const bool half = p.size == axo::SYM_HALF;
    const std::string tiles = p.cut.whole == 0 ? "none" : p.cut.whole <= p.workgroups ? "one" : "many";
    return (half ? std::string("half") : std::to_string(p.size)) + " " + tiles + " " + cut_of(half ? p.diagonal : p.cut);
}
int main(int argc, char** argv) {
    if (argc == 2) {  // every name in a range of sizes
        std::set<std::string> all;
        const std::string most = argv[1];
        for (long s = 64; s <= 9216; s += 64)
            for (long l = s; l <= 40960; l += l < 4096 ? 64 : l < 12288 ? 256 : 1024) all.insert(name(s, l / 64));
        for (const std::string& n : all) std::printf("%s\n", n.c_str());
        return 0;
    }
    long s, l;
    while (std::scanf("%ld %ld", &s, &l) == 2) std::printf("%s,%s\n", name(s, l / 64).c_str(), name(s, s / 64).c_str());
}
"""

# padded sizes s <= l -> the plan of the Gram matrix, that of its polynomial
SYMMETRIC = [((192, 192), "32 one whole", "32 one whole"), ((192, 2432), "32 none own", "32 one whole"), ((256, 2560), "32 none slices", "32 one whole"),
             ((1024, 1024), "64 one whole", "64 one whole"), ((768, 2304), "64 none slices", "32 one whole"), ((1024, 4096), "64 none own", "64 one whole"),
             ((1600, 9472), "64 none shared", "64 one whole"),
             ((2048, 2048), "128 one whole", "128 one whole"), ((1536, 6144), "128 none slices", "64 one whole"), ((1472, 6400), "128 none own", "64 one whole"),
             ((2304, 5888), "128 none shared", "128 one whole"), ((2880, 2880), "128 one slices", "128 one slices"), ((2944, 2944), "128 one own", "128 one own"),
             ((3520, 3520), "128 many whole", "128 many whole"), ((4224, 4224), "128 many slices", "128 many slices"), ((4160, 4160), "128 many own", "128 many own"),
             ((4032, 4032), "half one own", "half one own"), ((4096, 4096), "half one slices", "half one slices"),
             ((4544, 4544), "256 one whole", "256 one whole"), ((3520, 4864), "256 none slices", "128 many whole"), ((3008, 8192), "256 none own", "128 one own"),
             ((4544, 5056), "256 none shared", "256 one whole"), ((5760, 5760), "256 one slices", "256 one slices"), ((5696, 5696), "256 one own", "256 one own"),
             ((6976, 6976), "256 one shared", "256 one shared"), ((7488, 7488), "256 many whole", "256 many whole"), ((8000, 8000), "256 many slices", "256 many slices"),
             ((8000, 8256), "256 many own", "256 many slices"), ((9024, 9024), "256 many shared", "256 many shared")]

# padded sizes s <= l whose product Q X, or X Q of a tall X, runs on 64 x 128 tiles: a round of them, more 64 x 64 ones
OBLONG = [(1024, 1280), (1024, 1216), (1088, 1152)]


def weights_of(s, l):
    """A wide and a tall weight, ragged, that are padded to these sizes."""
    return (s - 29, l - 13), (l - 13, s - 29)


class Plans:
    """The plans of sym_cut.hpp, compiled on its own."""

    def __init__(self, folder):
        cxx = shutil.which("g++") or shutil.which("clang++")
        if not cxx:
            import pytest

            pytest.skip("no C++ compiler")
        source, self.program = os.path.join(str(folder), "plans.cpp"), os.path.join(str(folder), "plans")
        with open(source, "w") as f:
            f.write(PLANS)
        subprocess.run([cxx, "-std=c++17", "-O2", "-I" + os.path.join(ROOT, "paper_2305_13525_amd", "csrc"), source, "-o", self.program], check=True)

    def of(self, sizes):
        """(name of the Gram matrix's plan, of the polynomial's) for each s, l."""
        r = subprocess.run([self.program], input="\n".join(f"{s} {l}" for s, l in sizes), stdout=subprocess.PIPE, text=True, check=True, timeout=120)
        return [tuple(line.split(",")) for line in r.stdout.splitlines()]

    def names(self):
        return set(subprocess.run([self.program, "all"], stdout=subprocess.PIPE, text=True, check=True, timeout=120).stdout.splitlines())
