"""CPU tests of results of the gated feed-forward block that would share memory with operands or with each other: what counts as shared (csrc/shared_rows.hpp, compiled with the
host compiler, against marking every byte), and that such calls are refused."""
import ctypes as C
import os
import subprocess

import pytest

from paper_2009_12263_amd import binding as fg
from tests.test_middle_operators_abi import PTR, ffn, ffn_grad, row

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2009_12263_amd", "csrc")

PROGRAM = r"""
#include "shared_rows.hpp"
#include <cstdio>
#include <cstring>
using namespace fg;
static bool marked(const RowSpan &a, const RowSpan &b) {
    static unsigned char memory[4096];
    memset(memory, 0, sizeof memory);
    for (int64_t r = 0; r < a.rows; ++r) memset(memory + a.at + r * a.step, 1, (size_t)a.bytes);
    for (int64_t r = 0; r < b.rows; ++r)
        for (int64_t i = 0; i < b.bytes; ++i) if (memory[b.at + r * b.step + i]) return true;
    return false;
}
int main() {
    unsigned seed = 1;
    auto below = [&](int n) { seed = seed * 1664525u + 1013904223u; return (int64_t)((seed >> 8) % (unsigned)n); };
    long shared = 0, apart = 0, between = 0;
    for (int n = 0; n < 2000000; ++n) {
        RowSpan s[2];
        for (auto &v : s) {
            v = {(uintptr_t)below(60), below(7), 0, below(9)};
            v.step = v.bytes + below(20);
        }
        if (n % 2) {                    // the same distance, as columns of one matrix have
            const int64_t step = s[0].step > s[1].step ? s[0].step : s[1].step;
            s[0].step = s[1].step = step;
        }
        if (n % 5 == 0) { s[0].rows = 1; s[0].step = below(3) ? s[0].step : 0; }
        const bool want = marked(s[0], s[1]);
        for (int turn = 0; turn < 2; ++turn)
            if (share_bytes(s[turn], s[1 - turn]) != want) {
                printf("%d: at %ld, %ld x %ld of %ld; at %ld, %ld x %ld of %ld\n", (int)want, (long)s[0].at, (long)s[0].rows, (long)s[0].bytes, (long)s[0].step, (long)s[1].at,
                       (long)s[1].rows, (long)s[1].bytes, (long)s[1].step);
                return 1;
            }
        want ? ++shared : ++apart;
        const bool some = s[0].rows > 1 && s[1].rows > 1 && s[0].bytes && s[1].bytes;
        if (!want && some && s[0].at < s[1].at + s[1].step && s[1].at < s[0].at + s[0].step) ++between;
    }
    // long ones
    const uintptr_t far = 1ull << 46;
    const int64_t many = 1 << 30;
    if (share_bytes({far, many, 256, 128}, {far + 128, many, 256, 128}) || !share_bytes({far, many, 256, 129}, {far + 128, many, 256, 128})) return 1;
    if (!share_bytes({far, many, 256, 128}, {far + 256 * (uintptr_t)(many - 1) + 127, 4, 256, 1}) || share_bytes({far, many, 256, 128}, {far + 256 * (uintptr_t)(many - 1) + 128, 4, 256, 1})) return 1;
    if (share_bytes({far, 1, INT64_MAX, 64}, {far + 64, 1, INT64_MAX, 64})) return 1;
    puts(shared > 100000 && apart > 100000 && between > 10000 ? "ok" : "too few of a kind");
}
"""


def test_what_is_shared(tmp_path):
    src, exe = tmp_path / "t.cpp", tmp_path / "t"
    src.write_text(PROGRAM)
    subprocess.run(["g++", "-O2", "-std=c++17", "-Wall", "-I", CSRC, str(src), "-o", str(exe)], check=True)
    r = subprocess.run([str(exe)], stdout=subprocess.PIPE, text=True)
    assert r.returncode == 0 and r.stdout == "ok\n", r.stdout


# 4 tokens of 64 values, 48 hidden: X, dY, Y and dX have rows of 128 bytes, GU of 384, W_in 96 of 128, W_out 64 of 96; 256 bytes apart, GU's 512
HERE = 0x1000000


@pytest.mark.parametrize("call,args,word", [
    (ffn, dict(X=row(re=HERE), Y=row(re=HERE + 256)), "Y must be in other memory than X"),
    (ffn, dict(X=row(re=HERE), Y=row(re=HERE + 126)), "Y must be in other memory than X"),
    (ffn, dict(X=row(re=HERE + 2), Y=row(re=HERE + 256 * 3 + 128)), "Y must be in other memory than X"),
    (ffn, dict(W_in=row(re=HERE), Y=row(re=HERE + 256 * 95 + 64)), "Y must be in other memory than W_in"),
    (ffn, dict(W_out=row(re=HERE), Y=row(re=HERE - 256)), "Y must be in other memory than W_out"),
    (ffn, dict(X=row(re=HERE), GU=row(fg.FG_F32, re=HERE - 512 - 260)), "GU must be in other memory than X"),
    (ffn, dict(W_in=row(re=HERE), GU=row(fg.FG_F32, re=HERE + 256 * 94)), "GU must be in other memory than W_in"),
    (ffn, dict(Y=row(re=HERE), GU=row(fg.FG_F32, re=HERE + 4)), "GU must be in other memory than Y"),
    (ffn_grad, dict(X=row(re=HERE), dX=row(re=HERE + 256)), "dX must be in other memory than X"),
    (ffn_grad, dict(dY=row(re=HERE), dX=row(re=HERE + 2)), "dX must be in other memory than dY"),
    (ffn_grad, dict(W_in=row(re=HERE), dW_in=row(re=HERE + 256 * 50)), "dW_in must be in other memory than W_in"),
    (ffn_grad, dict(GU=row(fg.FG_F32, re=HERE), dW_out=row(re=HERE + 512)), "dW_out must be in other memory than GU"),
    (ffn_grad, dict(dX=row(re=HERE), dW_in=row(re=HERE + 64)), "dX must be in other memory than dW_in"),
    (ffn_grad, dict(dX=row(re=HERE), dW_out=row(re=HERE + 256)), "dX must be in other memory than dW_out"),
    (ffn_grad, dict(dW_in=row(re=HERE), dW_out=row(re=HERE + 256 * 90)), "dW_in must be in other memory than dW_out"),
    # the operand is refused before a workspace that is too small
    (ffn, dict(X=row(re=HERE), Y=row(re=HERE + 256), size=0), "Y must be in other memory than X"),
])
def test_shared_results_are_refused(call, args, word):
    assert call(**args) == fg.FG_ERR_LAYOUT and word in fg.fg_last_error(), fg.fg_last_error()


@pytest.mark.parametrize("call,args", [
    (ffn, dict(X=row(re=HERE), Y=row(re=HERE + 128))),                          # two halves of a matrix
    (ffn, dict(X=row(re=HERE + 128), Y=row(re=HERE))),
    (ffn, dict(X=row(re=HERE, ld=512), Y=row(re=HERE + 128, ld=512), GU=row(fg.FG_F32, re=HERE + 256, ld=256))),
    (ffn, dict(X=row(re=HERE), Y=row(re=HERE + 256 * 3 + 128))),
    (ffn_grad, dict(dY=row(re=HERE), X=row(re=HERE))),                          # operands may be the same
    (ffn_grad, dict(dX=row(re=HERE), dW_in=row(re=HERE + 128))),
    (ffn_grad, dict(dW_in=row(re=HERE), dW_out=row(re=HERE + 128))),
])
def test_rows_between_each_other_are_not(call, args):
    # (refused for its workspace, which is looked at last: nothing is launched)
    assert call(**args, size=0) == fg.FG_ERR_SHAPE and "workspace" in fg.fg_last_error(), fg.fg_last_error()
