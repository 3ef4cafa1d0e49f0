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
        const int tile = linear_tile(dtype, longest), parts = linear_parts(items * hkv, hq / hkv, tile, n_cu);
        std::printf("%ld %ld %d %ld %d\n", len, items, tile, hq / hkv / parts, linear_slices(n_seq * hkv, d, n_cu));
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
        program prints for each: tokens of a segment (0: none), items, tokens of a tile,
        query heads of a chunk workgroup, slices of a state in the single-token form."""
        text = "".join(f"{c} {t} {hq} {hkv} {d} {len(n)} {' '.join(map(str, n))}\n" for c, t, hq, hkv, d, n in plans)
        out = subprocess.run([self.exe], input=text, capture_output=True, text=True, check=True).stdout
        return [tuple(int(x) for x in line.split()) for line in out.splitlines()]

    def close(self):
        shutil.rmtree(self.dir)


# Plans whose layout the tests pin for 256 compute units, and run on a device that has
# them: (dtype, query heads, KV heads, head dim, tokens of each sequence, then tokens of
# a tile, query heads of a workgroup and whether sequences are cut)
N_CU = 256


def ragged(n, lo, hi):
    return [lo + i * 37 % (hi - lo + 1) for i in range(n)]


CHUNKS = [
    # a workgroup for every query head of a KV head
    *[("bf16", 4 * g, 4, d, ragged(70, 30, 93), 64, g, False) for g in (2, 4, 8) for d in (64, 128)],
    *[("bf16", 4 * g, 4, d, ragged(70, 1, 32), 32, g, False) for g in (2, 4, 8) for d in (64, 128)],
    *[("f32", 4 * g, 4, d, ragged(70, 1, 70), 32, g, False) for g in (2, 4, 8) for d in (64, 128)],
    # ... for half of them
    *[("bf16", 4 * g, 4, d, ragged(34, 17, 100), 64, g // 2, False) for g in (4, 8) for d in (64, 128)],
    *[("bf16", 4 * g, 4, d, ragged(17, 2, 32), 32, g // 2, False) for g in (4, 8) for d in (64, 128)],
    *[("f32", 4 * g, 4, d, ragged(17, 2, 80), 32, g // 2, False) for g in (4, 8) for d in (64, 128)],
    # segments, several heads each
    *[("bf16", 32, 4, d, [4101, 1, 233], 64, 4, True) for d in (64, 128)],
    *[("bf16", 8, 2, d, [16500], 64, 2, True) for d in (64, 128)],
    *[("f32", 32, 4, d, [1900, 5, 130], 32, 4, True) for d in (64, 128)],
]
# single tokens: ..., sequences, slices of a state
SINGLES = [(t, 4 * g, 4, d, n, s) for t in ("bf16", "f32") for g in (1, 2, 4, 8)
           for d, n, s in ((64, 80, 1), (64, 40, 2), (128, 80, 1), (128, 40, 2), (128, 32, 4))]
