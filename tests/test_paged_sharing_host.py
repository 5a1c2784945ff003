"""Host build of what the attention over pages makes of a batch's arrays (csrc/paged_work.h): whatever they hold, the rows that units are made
of lie among the call's tokens, so that no kernel addresses anything outside them (CPU only)."""
import os
import shutil
import subprocess

import pytest

PROGRAM = r"""
#include <climits>
#include <cstdio>
#include "paged_work.h"
using namespace infmllm;

template <int R> long check(long& bad)
{
    long cases = 0;
    const int at[] = {INT_MIN, INT_MIN + 1, INT_MIN + 9, -(1 << 30), -7, -1, 0, 1, 2, 6, 7, 8, 63, 64, 1000, 1 << 24, (1 << 24) + 1, 1 << 30, INT_MAX - 1, INT_MAX};
    const int groups[] = {1, 4, 5, 64, 4096}, windows[] = {0, 1, 300, 1 << 30};
    for (int tokens : {1, 7, 64, 1000, 1 << 18, 1 << 24}) for (int G : groups) for (int window : windows) {
        if ((long)tokens * G > 1 << 30) continue;
        Work<R, 32, 192> w{};
        w.tokens = tokens; w.G = G; w.Hkv = 2; w.window = window; w.row_lo = 0; w.row_hi = INT_MAX; w.most_keys = 5000; w.seqs = 1;
        for (int s0 : at) for (int s1 : at) for (int len : at) {
            const auto q = w.describe(s0, s1, len);
            const long rows = (long)q.n * G;
            const bool in = q.first >= 0 && q.n >= 0 && (long)q.first + q.n <= tokens && q.ntile == (rows + R - 1) / R;
            // positions: the new ones are the last of the sequence
            const bool there = q.n == 0 || (s1 > q.first && q.pos0 == (long)(len > 0 ? len : 0) - ((long)s1 - q.first) && (long)q.pos0 + q.n - 1 < INT_MAX);
            // entries that ascend within the call's tokens: as they stand
            const bool plain = !(0 <= s0 && s0 <= s1 && s1 <= tokens) || (q.first == s0 && q.n == s1 - s0);
            const bool cost = q.base > 0 && q.inc >= 0 && q.base < 1e11;
            ++cases;
            if (!(in && there && plain && cost)) {
                if (!bad++) std::printf("R %d tokens %d G %d window %d starts %d %d len %d: first %d n %d pos0 %d tiles %d base %g\n", R, tokens, G, window, s0, s1, len,
                                        q.first, q.n, q.pos0, q.ntile, q.base);
            }
        }
    }
    return cases;
}
int main()
{
    long bad = 0;
    const long cases = check<16>(bad) + check<32>(bad) + check<256>(bad);
    std::printf("%ld of %ld wrong\n", bad, cases);
    return bad != 0 || cases < 100000;
}
"""


@pytest.mark.skipif(shutil.which("hipcc") is None, reason="hipcc not found")
def test_rows_of_units_lie_among_the_tokens(tmp_path):
    from paper_2409_09086_amd.build import CSRC
    src, exe = tmp_path / "sharing.hip", tmp_path / "sharing"
    src.write_text(PROGRAM)
    subprocess.run(["hipcc", "--cuda-host-only", "-O1", "-std=c++17", "-I" + os.path.abspath(CSRC), str(src), "-o", str(exe)], check=True, capture_output=True)
    r = subprocess.run([str(exe)], capture_output=True, text=True, timeout=60)
    assert r.returncode == 0, r.stdout
