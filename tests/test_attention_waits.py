"""The waits of prompt attention, in every order that its warps and products can take: a model of the softmax's warps, of the
warp that issues products, and of barriers whose phases are told apart by parity."""
import os
import subprocess

import pytest

CSRC = os.path.join(os.path.dirname(__file__), "..", "paper_2110_06037_gb300", "csrc")

PROGRAM = r"""
#include <cstdio>
#include <cstdlib>
#include <cstring>
#include <set>
#include <string>
#include <vector>
#include "attn_order.h"

const int WARPS = 2, PIECES = 3;
int AHEAD, n[PIECES], first[PIECES];
bool by_header;  // (otherwise nothing is waited for before weights)

struct State {
    // a warp: piece, tile (n: behind the last), step of it; meetings it came to; the issuing warp likewise
    signed char piece[WARPS], tile[WARPS], step[WARPS], came[WARPS];
    signed char ip, ij, istep, met;
    signed char scores_asked, scores_over, products_asked, products_over;
    bool operator<(const State &o) const { return memcmp(this, &o, sizeof *this) < 0; }
};
bool over(int phases, int phase) { return (phases & 1) != (phase & 1); }  // what a wait by parity sees
[[noreturn]] void fail(const char *what) {
    printf("ahead %d, tiles %d %d %d: %s\n", AHEAD, n[0], n[1], n[2], what);
    exit(1);
}
// one score at a time on a barrier, or two barriers in turn
bool scores_seen(int have, int i) { return AHEAD == 1 ? over(have, i) : over((have + 1 - i % 2) / 2, i / 2); }

void check(bool ok, const char *what) {
    if (!ok) fail(what);
}
std::vector<State> next(const State &s) {
    std::vector<State> r;
    for (int w = 0; w < WARPS; ++w) {
        if (s.piece[w] == PIECES) continue;
        const int p = s.piece[w], j = s.tile[w], at = first[p] + j;
        State t = s;
        auto come = [&] {
            check(++t.came[w] - s.met <= (AHEAD == 1 ? 1 : 2), "a meeting is counted for another");
        };
        if (s.step[w] == 0) {  // the queries
            come(), t.step[w] = 1;
            r.push_back(t);
        } else if (s.step[w] == 1 && j < n[p]) {  // its scores
            if (!scores_seen(s.scores_over, at)) continue;
            check(s.scores_over > at, "scores before they are there");
            t.step[w] = 2;
            r.push_back(t);
            if (j > 0) t.step[w] = 3, r.push_back(t);  // the largest grew
        } else if (s.step[w] == 3) {  // sums are scaled again
            if (!over(s.products_over, at - 1)) continue;
            check(s.products_over == at, "sums scaled while a product adds to them");
            t.step[w] = 2;
            r.push_back(t);
        } else if (s.step[w] == 2) {  // weights
            if (by_header && sn::k::waits_before_weights(j, n[p], AHEAD) && !over(s.products_over, at - 1)) continue;
            come(), t.tile[w] = j + 1, t.step[w] = 1;
            r.push_back(t);
        } else {  // the end
            if (!over(s.products_over, at - 1)) continue;
            check(s.products_over == at, "sums read before the last product is over");
            t.piece[w] = p + 1, t.tile[w] = t.step[w] = 0;
            r.push_back(t);
        }
    }
    if (s.ip < PIECES) {
        State t = s;
        const int p = s.ip;
        int least = s.came[0];
        for (int w = 1; w < WARPS; ++w) least = s.came[w] < least ? s.came[w] : least;
        auto on = [&] {
            if (++t.ij == n[p]) t.ip = p + 1, t.ij = t.istep = 0;
            else t.istep = 1;
        };
        if (s.istep == 0 && least > s.met) {  // the queries are there: the first scores
            ++t.met, t.istep = 1, t.scores_asked += n[p] < AHEAD ? n[p] : AHEAD;
            r.push_back(t);
        } else if (s.istep == 1 && least > s.met) {  // weights are there: a product
            ++t.met, ++t.products_asked;
            if (s.ij + AHEAD < n[p]) t.istep = 2;
            else on();
            r.push_back(t);
        } else if (s.istep == 2 && over(s.products_over, first[p] + s.ij)) {
            check(s.products_over > first[p] + s.ij, "scores over weights that are still read");
            ++t.scores_asked, on();
            r.push_back(t);
        }
    }
    if (s.scores_over < s.scores_asked) r.push_back(s), ++r.back().scores_over;
    if (s.products_over < s.products_asked) r.push_back(s), ++r.back().products_over;
    return r;
}

int main(int argc, char **argv) {
    AHEAD = atoi(argv[1]), by_header = atoi(argv[2]);
    for (int c = 0; c < 64; ++c) {
        int sum = 0;
        for (int i = 0; i < PIECES; ++i) first[i] = sum, sum += n[i] = 1 + (c >> 2 * i) % 4;
        State s;
        memset(&s, 0, sizeof s);
        std::set<State> seen{s};
        std::vector<State> open{s};
        while (!open.empty()) {
            s = open.back(), open.pop_back();
            bool done = s.ip == PIECES;
            for (int w = 0; w < WARPS; ++w) done &= s.piece[w] == PIECES;
            const std::vector<State> all = next(s);
            if (all.empty() && !done) fail("a wait that does not end");
            for (const State &t : all)
                if (seen.insert(t).second) open.push_back(t);
        }
    }
}
"""


@pytest.fixture(scope="module")
def model(tmp_path_factory):
    src, exe = (tmp_path_factory.mktemp("waits") / name for name in ("t.cpp", "t"))
    src.write_text(PROGRAM)
    subprocess.run(["g++", "-std=c++17", "-O2", "-I", CSRC, str(src), "-o", str(exe)], check=True)
    return lambda *args: subprocess.run([str(exe), *map(str, args)], capture_output=True, text=True)


@pytest.mark.parametrize("ahead", [1, 2])
def test_every_wait_holds_and_ends(model, ahead):
    r = model(ahead, 1)
    assert r.returncode == 0, r.stdout


def test_without_the_wait_before_the_last_weights(model):
    """With one tile of scores ahead nothing is missing, with two the sums are read too early."""
    assert model(1, 0).returncode == 0
    r = model(2, 0)
    assert r.returncode == 1 and "sums read before" in r.stdout
