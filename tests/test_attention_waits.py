"""The waits at the end of a piece of prompt attention, against a model of a barrier whose phases are told apart by
parity: whatever has not been shown to be over may still be running."""
import os
import subprocess

CSRC = os.path.join(os.path.dirname(__file__), "..", "paper_2110_06037_gb300", "csrc")

PROGRAM = r"""
#include <cassert>
#include <initializer_list>
#include "attn_order.h"
// products before `over` are over; a wait for product p's parity passes at once where the phase under way has the
// other one, and else lasts until that phase is over.  Nothing ends before it is waited for.
struct Barrier {
    int over;
    void wait(int p) {
        if ((over & 1) == (p & 1)) ++over;
    }
};
int main() {
    for (int ahead : {1, 2}) {
        int sums = 0, missed = 0;
        for (int round = 0; round < 8; ++round)
            for (int n = 1; n <= 6; ++n) {
                // the last scores have come: of this piece's products all but the last `ahead` are over
                Barrier b{sums + (n > ahead ? n - ahead : 0)}, last = b;
                for (int j = sn::k::first_open_product(n, ahead); j < n; ++j) b.wait(sums + j);
                assert(b.over == sums + n);
                last.wait(sums + n - 1);
                missed += last.over != sums + n;
                sums += n;
            }
        assert((missed > 0) == (ahead > 1));  // to wait for the last one alone is enough with one product open, not with two
    }
}
"""


def test_the_end_of_a_piece_waits_for_every_product(tmp_path):
    src, exe = tmp_path / "t.cpp", tmp_path / "t"
    src.write_text(PROGRAM)
    subprocess.run(["g++", "-std=c++17", "-I", CSRC, str(src), "-o", str(exe)], check=True)
    subprocess.run([str(exe)], check=True)
