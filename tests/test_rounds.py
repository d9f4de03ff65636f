"""Which copies a thread of the token log probabilities still waits for when it leaves (csrc/rounds.h), on the host."""
import os
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

# Two rounds on the way, a new one behind each that landed, as the kernel does it; prints the rounds waited for at the end.
PROGRAM = r"""
#include <cstdio>
#include <cstdlib>
#include "rounds.h"
int main(int argc, char** argv) {
  const unsigned all = atoi(argv[1]), fails = atoi(argv[2]);  // rounds of the row; the first that does not land in time
  gf::Rounds r;
  for (unsigned i = 0; i < 2 && r.started < all; ++i) r.start();
  for (unsigned i = 0; i < all; ++i) {
    r.waited(r.ok && i != fails);
    if (r.ok && r.started < all) r.start();
  }
  if (r.on_the_way() > 2 || r.started > all) return 1;
  for (unsigned i = r.landed; i < r.started; ++i) printf("%u ", i);
}
"""


@pytest.fixture(scope="module")
def program(tmp_path_factory):
    at = tmp_path_factory.mktemp("rounds")
    (at / "rounds.cc").write_text(PROGRAM)
    subprocess.run(["g++", "-std=c++17", "-I", os.path.join(ROOT, "paper_2605_22566_b200", "csrc"), str(at / "rounds.cc"), "-o", str(at / "rounds")], check=True)
    return str(at / "rounds")


@pytest.mark.parametrize("rounds", [0, 1, 2, 3, 9])
def test_what_is_on_the_way_when_a_wait_gave_up(program, rounds):
    for fails in range(rounds + 1):
        out = subprocess.run([program, str(rounds), str(fails)], check=True, capture_output=True, text=True).stdout
        # the one that was not there in time, and the one behind it where there is one; nothing where all landed
        assert [int(x) for x in out.split()] == list(range(fails, min(fails + 2, rounds))), (rounds, fails)
