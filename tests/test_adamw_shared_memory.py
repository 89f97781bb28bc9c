"""CPU tests of AdamW's arrays that share memory: how they are found (csrc/shared_spans.hpp, compiled with the host compiler, against marking every byte), and that such calls are
refused."""
import os
import subprocess

import pytest

from paper_2009_12263_amd import binding as fg
from tests.test_middle_operators_abi import adamw, apart

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2009_12263_amd", "csrc")

PROGRAM = r"""
#include "shared_spans.hpp"
#include <cstdio>
#include <cstring>
using namespace fg;
int main() {
    unsigned seed = 7;
    auto below = [&](int n) { seed = seed * 1664525u + 1013904223u; return (int)((seed >> 8) % (unsigned)n); };
    long shared = 0, apart = 0, merged = 0;
    for (int n = 0; n < 300000; ++n) {
        const int lists = 1 + below(5), room = 20 << below(6);
        std::vector<std::vector<Span>> spans((size_t)lists, std::vector<Span>(8));          // (some of 8 each, at places of their own)
        static signed char memory[800];             // 1: read, 2: written
        memset(memory, 0, sizeof memory);
        bool want = false;
        int of = 0, at = 0;
        const bool rising = below(2);
        for (auto &list : spans) {
            const bool written = below(3) > 0;
            if (rising && below(2)) at = below(4);
            for (int k = 0; k < 8; ++k) {
                list[(size_t)k] = {(uintptr_t)below(2) * 1000, 0, -1, written};
                if (below(2)) continue;
                const int begin = rising ? at + below(6) : below(room), end = begin + 1 + below(8);
                at = end;
                if (end > 780) break;
                for (int i = begin; i < end; ++i) {
                    want |= memory[i] == 2 || (memory[i] && written);
                    if (!memory[i] || written) memory[i] = written ? 2 : 1;
                }
                list[(size_t)k] = {(uintptr_t)(1000 + begin), (uintptr_t)(1000 + end), of++, written};
            }
            if (below(3) == 0) std::reverse(list.begin(), list.end());
        }
        const auto &all = spans;
        Span a, b;
        const bool found = shared_spans(lists, 8, [&](int list, int64_t i) { return all[(size_t)list][(size_t)i]; }, a, b);
        if (found != want) { printf("%d: %d found, %d wanted\n", n, (int)found, (int)want); return 1; }
        if (found) {
            ++shared;
            if (!(a.written || b.written) || a.of == b.of || a.begin > b.begin || a.end <= b.begin) return 1;
            int seen = 0;
            for (auto &list : all) for (const Span &s : list) for (const Span *t : {&a, &b}) seen += s.of == t->of && s.begin == t->begin && s.end == t->end && s.written == t->written;
            if (seen != 2) return 1;
        } else {
            ++apart;
            int filled = 0;
            for (auto &list : all) for (const Span &s : list) filled += s.of >= 0;
            merged += filled > 8;
        }
    }
    puts(shared > 50000 && apart > 50000 && merged > 10000 ? "ok" : "too few of a kind");
}
"""


def test_what_is_found(tmp_path):
    src, exe = tmp_path / "t.cpp", tmp_path / "t"
    src.write_text(PROGRAM)
    subprocess.run(["g++", "-O2", "-std=c++17", "-Wall", "-I", CSRC, str(src), "-o", str(exe)], check=True)
    r = subprocess.run([str(exe)], stdout=subprocess.PIPE, text=True)
    assert r.returncode == 0 and r.stdout == "ok\n", r.stdout


# apart(i): 100 values of bfloat16 parameters and gradients (200 bytes each) and FP32 moments (400)
A, B = apart(0), apart(1)
EIGHT = dict(avg_scale=1 << 20, sq_scale=1 << 21)           # (a scale of 4 bytes each)


@pytest.mark.parametrize("tensors,words", [
    ([apart(0, exp_avg_sq=A.exp_avg + 396)], "exp_avg of tensor 0 and exp_avg_sq of tensor 0"),
    ([apart(0, exp_avg=A.exp_avg_sq + 4)], "exp_avg_sq of tensor 0 and exp_avg of tensor 0"),
    ([apart(0), apart(1, exp_avg=A.exp_avg_sq)], "exp_avg_sq of tensor 0 and exp_avg of tensor 1"),
    ([apart(0, master=B.param + 196), apart(1)], "param of tensor 1 and master of tensor 0"),
    ([apart(0, grad=A.param + 2)], "param of tensor 0 and grad of tensor 0"),
    ([apart(0, grad=A.param)], "grad of tensor 0 and param of tensor 0"),
    ([apart(0), apart(1), apart(2, grad=B.exp_avg + 200)], "exp_avg of tensor 1 and grad of tensor 2"),
    ([apart(0, **EIGHT), apart(1, avg_scale=A.param + 196, sq_scale=1 << 22)], "param of tensor 0 and avg_scale of tensor 1"),
    ([apart(0, **EIGHT, grad=(1 << 20) - 196)], "grad of tensor 0 and avg_scale of tensor 0"),
    ([apart(k, master=None) for k in range(40)] + [apart(50, exp_avg=apart(17).exp_avg_sq + 12)], "exp_avg_sq of tensor 17 and exp_avg of tensor 40"),
    ([apart(k) for k in range(40, 0, -1)] + [apart(50, exp_avg=apart(17).param + 4)], "param of tensor 23 and exp_avg of tensor 40"),
])
def test_shared_arrays_are_refused(tensors, words):
    assert adamw(tensors) == fg.FG_ERR_LAYOUT and words in fg.fg_last_error(), fg.fg_last_error()


@pytest.mark.parametrize("args,words", [
    (dict(step=A.exp_avg + 8), "step is in exp_avg of tensor 0"),
    (dict(step=A.param - 8, factor=A.param + 196), "grad_factor is in param of tensor 0"),
    (dict(lr_factor=B.exp_avg_sq), "lr_factor is in exp_avg_sq of tensor 1"),
])
def test_values_in_arrays_that_are_written(args, words):
    assert adamw([apart(0), apart(1)], **args) == fg.FG_ERR_LAYOUT and words in fg.fg_last_error(), fg.fg_last_error()
