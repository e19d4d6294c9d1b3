"""How the wavefronts of a work-group learn their next piece of work (csrc/rl_turns.h,
compiled here with g++): every order in which they can run is gone through (CPU)."""
import os
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

# A wavefront's turn t, as the kernel runs it: wavefront 0 writes the turn's place (100 +
# t), all arrive at the barrier, all read.  The work itself holds no barrier.  A state
# is every wavefront's step number and the words; each step of each wavefront that can run
# is tried.
SOURCE = r"""
#include <set>
#include <vector>
#include <cstdio>
#include <cstdlib>
#include "rl_turns.h"
using namespace rl_da;

struct OneWord {  // what does not do
    int32_t words[1];
    int32_t& of(int) { return words[0]; }
};

constexpr int kTurns = 5;
enum { kWrite, kArrive, kRead, kSteps };

template <class Place>
struct World {
    Place place = {};
    std::vector<int> at;  // step of each wavefront, kSteps a turn
};

template <class Place>
static void go(World<Place> w, std::set<std::vector<int>>& seen, int& wrong, int& ends)
{
    std::vector<int> key = w.at;
    for (int32_t x : w.place.words)
        key.push_back(x);
    if (!seen.insert(key).second)
        return;
    bool over = true;
    for (size_t i = 0; i < w.at.size(); ++i) {
        const int turn = w.at[i] / kSteps, step = w.at[i] % kSteps;
        if (turn == kTurns)
            continue;
        over = false;
        World<Place> n = w;
        if (step == kWrite && i == 0)
            n.place.of(turn) = 100 + turn;
        if (step == kRead) {
            // past the barrier only once all have arrived there
            bool all = true;
            for (int a : w.at)
                all &= a >= turn * kSteps + kRead;
            if (!all)
                continue;
            if (n.place.of(turn) != 100 + turn) {
                ++wrong;
                continue;
            }
        }
        ++n.at[i];
        go(n, seen, wrong, ends);
    }
    ends += over;
}

template <class Place>
static int late_reads(int waves, int* ends)
{
    World<Place> w;
    w.at.assign(waves, 0);
    std::set<std::vector<int>> seen;
    int wrong = 0;
    *ends = 0;
    go(w, seen, wrong, *ends);
    return wrong;
}

int main(int, char** argv)
{
    int ends = 0, ends_one = 0;
    const int waves = atoi(argv[1]);
    const int wrong = late_reads<NextPlace>(waves, &ends);
    const int wrong_one = late_reads<OneWord>(waves, &ends_one);
    printf("%d %d %d %d\n", wrong, ends, wrong_one, ends_one);
}
"""


@pytest.fixture(scope="module")
def program(tmp_path_factory):
    d = tmp_path_factory.mktemp("turns")
    src, exe = str(d / "turns.cpp"), str(d / "turns")
    with open(src, "w") as f:
        f.write(SOURCE)
    subprocess.run(["g++", "-O1", "-std=c++17", "-Wall", "-Werror", "-I",
                    os.path.join(ROOT, "paper_2512_22492_amd", "csrc"), src, "-o", exe], check=True)
    return exe


@pytest.mark.parametrize("waves", [2, 3, 4])
def test_every_wavefront_reads_the_place_of_its_turn(program, waves):
    out = subprocess.run([program, str(waves)], check=True, stdout=subprocess.PIPE).stdout
    wrong, ends, wrong_one, _ = (int(x) for x in out.split())
    assert wrong == 0 and ends > 0
    assert wrong_one > 0      # one word for all turns: some order reads another turn's place
