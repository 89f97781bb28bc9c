"""CPU test of the parts into which the gradients of weights from few tokens are cut (csrc/few_items.hpp, compiled with the host compiler): the waves of a
launch take each part of both products once, wherever one of the two is empty, and the spare waves of the last workgroup take none."""
import os
import subprocess

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2009_12263_amd", "csrc")

PROGRAM = r"""
#include "few_items.hpp"
#include <cstdio>
#include <vector>
using namespace fg;
int main() {
    setbuf(stdout, nullptr);
    const int64_t sizes[][2] = {{0, 0}, {0, 300}, {1, 1}, {1, 129}, {130, 128}, {129, 300}, {513, 64}};
    int spare[4] = {};
    for (auto &p : sizes)
        for (auto &q : sizes)
            for (int64_t each : {64, 128}) {
                const int64_t n0 = few_items(p[0], p[1], each), n1 = few_items(q[0], q[1], each), waves = (n0 + n1 + 3) / 4 * 4;
                printf("%ld x %ld and %ld x %ld\n", (long)p[0], (long)p[1], (long)q[0], (long)q[1]);
                std::vector<int> taken((size_t)(n0 + n1));
                ++spare[waves - n0 - n1];
                for (int64_t w = 0; w < waves; ++w) {
                    FewItem at;
                    const bool some = few_item(w, n0, p[1], n1, q[1], each, at);
                    if (some != (w < n0 + n1)) return 1;
                    if (!some) continue;
                    const auto &of = at.second ? q : p;
                    const int64_t strips = (of[1] + 127) / 128;
                    if (at.word < 0 || at.word >= of[0] || at.word % each || at.strip < 0 || at.strip >= strips) return 1;
                    ++taken[(size_t)((at.second ? n0 : 0) + at.word / each * strips + at.strip)];
                }
                for (int n : taken) if (n != 1) return 1;
            }
    for (int n : spare) if (!n) return 1;
    puts("ok");
}
"""


def test_waves_take_each_part_once(tmp_path):
    src, exe = tmp_path / "t.cpp", tmp_path / "t"
    src.write_text(PROGRAM)
    subprocess.run(["g++", "-O1", "-std=c++17", "-Wall", "-I", CSRC, str(src), "-o", str(exe)], check=True)
    r = subprocess.run([str(exe)], stdout=subprocess.PIPE, text=True)
    assert r.returncode == 0 and r.stdout.endswith("ok\n"), (r.returncode, r.stdout.splitlines()[-1])
