"""The order in which a group of warps goes through its tiles (csrc/attend_walk.h), with host threads in the place of the warps: one that gives up on a
tile must not leave the others standing at the barrier where they meet."""
import ctypes as C
import os
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

SHIM = r"""
#include "attend_walk.h"

#include <chrono>
#include <condition_variable>
#include <mutex>
#include <thread>
#include <vector>

// A barrier of `n` threads that says so when somebody stands at it for too long (the device's has no limit).
struct Meeting {
    std::mutex m;
    std::condition_variable c;
    int n, here = 0, round = 0;
    bool stuck = false;
    explicit Meeting(int n) : n(n) {}
    void meet()
    {
        std::unique_lock<std::mutex> lock(m);
        const int mine = round;
        if (++here == n) { here = 0; ++round; c.notify_all(); return; }
        if (!c.wait_for(lock, std::chrono::milliseconds(300), [&] { return round != mine || stuck; })) { stuck = true; c.notify_all(); }
    }
};
// A walk that leaves at the first wait that gives up.
template <class Meet, class Wait, class Work>
bool walk_leaving(int first, int n, int step, Meet meet, Wait wait, Work work)
{
    for (int i = first; i < n; i += step) {
        meet(i);
        if (!wait(i) || !work(i)) return false;
    }
    return true;
}
// Four threads over `tiles` tiles, which meet in the tiles of `masked`; thread t gives up on tile wait_at[t] (-1: on none) before its work, or inside it
// on work_at[t].  done[t]: tiles that thread t worked on.  Returns whether all came through; ok[t]: what the walk said.
extern "C" int walk(int leaving, int first, int tiles, int step, const int* masked, const int* wait_at, const int* work_at, int* done, int* ok)
{
    Meeting meeting(4);
    std::vector<std::thread> threads;
    for (int t = 0; t < 4; ++t)
        threads.emplace_back([&, t] {
            const auto meet = [&](int i) { if (masked[i]) { meeting.meet(); meeting.meet(); } };
            const auto wait = [&](int i) { return wait_at[t] != i; };
            const auto work = [&](int i) { if (work_at[t] == i) return false; ++done[t]; return true; };
            ok[t] = leaving ? walk_leaving(first, tiles, step, meet, wait, work) : mvla::walk_tiles(first, tiles, step, meet, wait, work);
        });
    for (auto& t : threads) t.join();
    return !meeting.stuck;
}
"""


@pytest.fixture(scope="module")
def shim(tmp_path_factory):
    d = tmp_path_factory.mktemp("walk")
    src, lib = str(d / "shim.cpp"), str(d / "shim.so")
    open(src, "w").write(SHIM)
    subprocess.run(["g++", "-std=c++17", "-O1", "-fPIC", "-shared", "-pthread", "-I", os.path.join(ROOT, "paper_2604_09244_b200", "csrc"), src, "-o", lib],
                   check=True)
    return C.CDLL(lib)


def run(shim, leaving, tiles, masked, wait_at, work_at=(-1, -1, -1, -1), first=0, step=1):
    ints = lambda x: (C.c_int * len(x))(*x)  # noqa: E731
    done, ok = ints([0] * 4), ints([0] * 4)
    through = shim.walk(leaving, first, tiles, step, ints(masked), ints(wait_at), ints(work_at), done, ok)
    return bool(through), list(done), [bool(x) for x in ok]


@pytest.mark.parametrize("masked", [[1] * 9, [0, 1, 0, 0, 1, 0, 0, 0, 1], [0] * 9])
def test_nobody_gives_up(shim, masked):
    assert run(shim, 0, 9, masked, [-1] * 4) == (True, [9] * 4, [True] * 4)
    assert run(shim, 0, 9, masked, [-1] * 4, first=1, step=2) == (True, [4] * 4, [True] * 4)
    assert run(shim, 0, 0, masked, [-1] * 4) == (True, [0] * 4, [True] * 4)


@pytest.mark.parametrize("wait_at,work_at", [
    ([3, -1, -1, -1], [-1] * 4), ([-1, -1, 0, -1], [-1] * 4), ([8, 2, -1, 5], [-1] * 4), ([4] * 4, [-1] * 4),
    ([-1] * 4, [-1, 3, -1, -1]), ([-1, -1, 6, -1], [1, -1, -1, 7]),
])
def test_those_that_go_on_are_not_left_at_the_barrier(shim, wait_at, work_at):
    masked = [1, 0, 0, 1, 1, 0, 1, 0, 1]
    through, done, ok = run(shim, 0, 9, masked, wait_at, work_at)
    assert through
    for t in range(4):
        gave_up = [i for i in (wait_at[t], work_at[t]) if i >= 0]
        assert done[t] == min(gave_up, default=9) and ok[t] == (not gave_up)


def test_the_trial_notices_threads_that_are_left_behind(shim):
    assert not run(shim, 1, 9, [1] * 9, [3, -1, -1, -1])[0]
