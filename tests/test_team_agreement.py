"""Threads whose branch holds barriers or votes take it as one.  A team of warps (csrc/team.cuh) has to, whatever each of its
threads would have found by asking for itself.  Runs the header's function on host threads; no kernel is launched."""
import os
import shutil
import subprocess

import pytest

from paper_2512_09238_b200 import _build

# A piece of work as the paged kernel's teams do it: a question, barriers inside the branch that depends on it, one behind.  The
# answer changes with every time it is asked.  A barrier at which somebody waits for five seconds ends the program with 3.
SOURCE = r"""
#define __host__
#define __device__
#define __forceinline__ inline
#include "team.cuh"

#include <atomic>
#include <chrono>
#include <condition_variable>
#include <cstdio>
#include <cstdlib>
#include <cstring>
#include <mutex>
#include <thread>
#include <vector>

constexpr int kThreads = 8, kPieces = 400;
std::mutex mu;
std::condition_variable cv;
int arrived = 0, phase = 0;
std::atomic<int> asked{0};

void meet() {
  std::unique_lock<std::mutex> lock(mu);
  const int mine = phase;
  if (++arrived == kThreads) {
    arrived = 0;
    ++phase;
    cv.notify_all();
  } else if (!cv.wait_for(lock, std::chrono::seconds(5), [&] { return phase != mine; })) {
    std::puts("stuck");
    std::fflush(stdout);
    std::_Exit(3);
  }
}

int main(int, char** argv) {
  const bool together = !std::strcmp(argv[1], "together");
  static volatile int said;
  std::vector<int> taken(kThreads);
  std::vector<std::thread> team;
  for (int t = 0; t < kThreads; ++t)
    team.emplace_back([&, t] {
      auto ask = [&] { return asked++ % 3 != 0; };
      for (int p = 0; p < kPieces; ++p) {
        bool go;
        if (together) {
          go = tca::team_agrees(t == 0, &said, ask, meet);
        } else {
          meet();
          go = ask();
        }
        if (go) { meet(); ++taken[t]; meet(); }
        meet();
      }
    });
  for (auto& t : team) t.join();
  for (int n : taken) if (n != taken[0]) return 4;
  std::printf("%d %d\n", taken[0], asked.load());
  return 0;
}
"""


@pytest.fixture(scope="module")
def program(tmp_path_factory):
    if shutil.which("g++") is None:
        pytest.skip("no g++")
    d = tmp_path_factory.mktemp("team")
    (d / "team.cpp").write_text(SOURCE)
    subprocess.run(["g++", "-std=c++17", "-O2", "-pthread", "-I", _build.CSRC, "-o", str(d / "team"), str(d / "team.cpp")], check=True)
    return str(d / "team")


def test_a_team_that_agrees_gets_through(program):
    r = subprocess.run([program, "together"], capture_output=True, text=True, timeout=100)
    assert r.returncode == 0 and r.stdout.split() == ["266", "400"]     # asked once a piece; two answers of three are yes


def test_threads_that_ask_for_themselves_do_not(program):
    """That the program above can tell."""
    r = subprocess.run([program, "alone"], capture_output=True, text=True, timeout=100)
    assert r.returncode != 0


def test_the_paged_kernel_asks_as_a_team():
    """The branch that holds the merge's barriers hangs on that one answer."""
    src = open(os.path.join(_build.CSRC, "paged.cu")).read()
    assert src.count("if (team_agrees(") == 1 and "if (!*abort_flag" not in src


def test_the_mainloop_votes_on_the_abort_flag():
    """The softmax warps of flash_tc.cuh leave their loop over items together: what is in it needs whole warps."""
    src = open(os.path.join(_build.CSRC, "flash_tc.cuh")).read()
    assert "!*abort_flag &&" not in src and "__any_sync(0xffffffffu, *abort_flag != 0)" in src
