"""How the linear layers' work is laid out for a plan, asked of the rules that the
library itself compiles (mtn_linear.h), in a program built by g++."""
import os
import shutil
import subprocess
import tempfile

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

PROGRAM = r"""
#include "mtn_linear.h"
#include <cstdio>
#include <vector>
using namespace mtn;
// n_cu dtype hq hkv d n_seq, then tokens per sequence
int main() {
    long n_cu, dtype, hq, hkv, d, n_seq;
    while (std::scanf("%ld %ld %ld %ld %ld %ld", &n_cu, &dtype, &hq, &hkv, &d, &n_seq) == 6) {
        std::vector<long> n(n_seq);
        long T = 0, most = 0, items = 0, longest = 0;
        for (long &x : n) {
            if (std::scanf("%ld", &x) != 1) return 1;
            T += x;
            most = std::max(most, x);
        }
        const long len = linear_segment(n_seq, T, hq, hkv, n_cu);
        for (long x : n) {
            items += len ? (x + len - 1) / len : 1;
            longest = std::max(longest, len ? std::min(len, x) : x);
        }
        std::printf("%ld %ld %ld\n", len, items, longest);
    }
}
"""


class Rules:
    def __init__(self):
        self.dir = tempfile.mkdtemp()
        src, self.exe = os.path.join(self.dir, "rules.cpp"), os.path.join(self.dir, "rules")
        with open(src, "w") as f:
            f.write(PROGRAM)
        subprocess.run(["g++", "-std=c++17", "-O1", "-D__HIP_PLATFORM_AMD__", "-I/opt/rocm/include",
                        "-I" + os.path.join(ROOT, "paper_2607_02640_amd", "csrc"), src, "-o", self.exe], check=True)

    def ask(self, plans):
        """plans: (n_cu, dtype, hq, hkv, d, tokens per sequence); a list of what the
        program prints for each."""
        text = "".join(f"{c} {t} {hq} {hkv} {d} {len(n)} {' '.join(map(str, n))}\n" for c, t, hq, hkv, d, n in plans)
        out = subprocess.run([self.exe], input=text, capture_output=True, text=True, check=True).stdout
        return [tuple(int(x) for x in line.split()) for line in out.splitlines()]

    def close(self):
        shutil.rmtree(self.dir)
