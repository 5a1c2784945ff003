"""Host build of what the attention over pages makes of a batch's arrays (csrc/paged_work.h): whatever they hold, the rows that units are made
of lie among the call's tokens and the units that shares begin in exist, so that no kernel addresses anything outside them (CPU only)."""
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
// the unit at a place of a sequence's cost: one that exists, and the right one where the costs are exact
template <int R> long places(long& bad)
{
    typedef Work<R, 32, 192> W;
    long cases = 0;
    for (int n : {1, 15, 1000, 1 << 24}) for (int G : {1, 5, 64}) for (int window : {0, 300}) for (int len : {1, 5000, INT_MAX}) for (int heads : {1, 3, 16384}) {
        W w{};
        w.tokens = n; w.G = G; w.Hkv = heads; w.window = window; w.row_hi = INT_MAX; w.most_keys = INT_MAX - 65536; w.seqs = 1;
        const auto q = w.describe(0, n, len);
        const double head = W::before(q, q.ntile), all = head * heads;
        auto look = [&](double rem) {
            const auto p = W::locate(q, heads, head, rem);
            bool good = p.h >= 0 && p.h < heads && p.tile >= 0 && p.tile < q.ntile;
            if (rem >= 0 && rem < all && all < 9e15) good &= W::before(q, p.tile) <= p.rem && p.rem < W::before(q, p.tile + 1) && p.h * head + p.rem == rem;
            ++cases;
            if (!good && !bad++) std::printf("R %d n %d G %d window %d len %d heads %d rem %.17g: head %d tile %d rem %.17g\n", R, n, G, window, len, heads, rem, p.h, p.tile, p.rem);
        };
        for (double x : {-1.0, 0.0, 1.0, all - 1, all, all + 1, all * (1 + 1e-12)}) look(x);
        for (int h : {0, 1, heads / 2, heads - 1})
            for (int t : {0, 1, q.ntile / 3, q.ntile - 1})
                for (double d : {-1.0, 0.0, 1.0}) look(h * head + W::before(q, t) + d);
    }
    return cases;
}
int main()
{
    long bad = 0;
    const long cases = check<16>(bad) + check<32>(bad) + check<256>(bad) + places<16>(bad) + places<256>(bad);
    std::printf("%ld of %ld wrong\n", bad, cases);
    return bad != 0 || cases < 100000;
}
"""


@pytest.mark.skipif(shutil.which("hipcc") is None, reason="hipcc not found")
def test_units_exist_and_their_rows_lie_among_the_tokens(tmp_path):
    from paper_2409_09086_amd.build import CSRC
    src, exe = tmp_path / "sharing.hip", tmp_path / "sharing"
    src.write_text(PROGRAM)
    subprocess.run(["hipcc", "--cuda-host-only", "-O1", "-std=c++17", "-I" + os.path.abspath(CSRC), str(src), "-o", str(exe)], check=True, capture_output=True)
    r = subprocess.run([str(exe)], capture_output=True, text=True, timeout=60)
    assert r.returncode == 0, r.stdout
