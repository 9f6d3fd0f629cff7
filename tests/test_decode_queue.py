"""What the work queue of moe_decode makes of tickets and experts that it reads back from the workspace
(csrc/decode_queue.h, compiled for the host), where another call has changed them: a call's items and experts are its own
ones whatever it reads."""
import os
import random
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2512_14080_amd", "csrc")
MIN, MAX = -2 ** 31, 2 ** 31 - 1

MAIN = """
#include "decode_queue.h"
#include <cstdio>
int main() {
  int kind, n;
  while (std::scanf("%d %d", &kind, &n) == 2) {
    if (kind == 0) {  // the items of a workgroup that reads n tickets
      int item = -1;
      for (int i = 0, t; i < n && std::scanf("%d", &t) == 1; ++i) std::printf("%d ", item = smoe::next_item(item, t));
    } else {  // an expert of n
      unsigned e;
      if (std::scanf("%u", &e) == 1) std::printf("%d", smoe::expert_within(e, n));
    }
    std::puts("");
  }
}
"""


@pytest.fixture(scope="module")
def ask(tmp_path_factory):
    d = tmp_path_factory.mktemp("queue")
    src, exe = d / "main.cpp", d / "main"
    src.write_text(MAIN)
    subprocess.run(["g++", "-O1", "-fsanitize=undefined", "-fno-sanitize-recover", "-I", CSRC, "-o", exe, src], check=True)

    def run(lines):
        r = subprocess.run([exe], input="\n".join(lines) + "\n", text=True, capture_output=True, check=True)
        return [[int(x) for x in l.split()] for l in r.stdout.splitlines()]

    return run


def test_tickets_of_a_call_alone_are_its_items(ask):
    rng = random.Random(0)
    seqs = [sorted(rng.sample(range(5000), rng.randint(1, 60))) for _ in range(50)]
    assert ask([f"0 {len(s)} " + " ".join(map(str, s)) for s in seqs]) == seqs


def test_items_increase_whatever_the_tickets(ask):
    """Counters set back to 0, counted on by two calls, or any bits at all: the items begin at 0 or above and increase, so
    that they end and no index formed from them is below its range."""
    rng = random.Random(1)
    seqs = [[7, 0, 1, 2, 9], [0, 0, 0], [5, 4, 3], [-1, -2, MIN], [MIN, MAX - 1], [3, MIN, 4, 4]]
    seqs += [[rng.choice([rng.randint(0, 300), rng.randint(MIN, MAX - 100)]) for _ in range(40)] for _ in range(200)]
    for s, items in zip(seqs, ask([f"0 {len(s)} " + " ".join(map(str, s)) for s in seqs])):
        assert items[0] >= 0 and all(a < b for a, b in zip(items, items[1:])), s


def test_experts_exist(ask):
    cases = [(E, e) for E in (8, 128, 1024) for e in (0, 1, E - 1, E, E + 1, 1023, 2 ** 31, 2 ** 32 - 1)]
    for (E, e), (got,) in zip(cases, ask([f"1 {E} {e}" for E, e in cases])):
        assert 0 <= got < E and (got == e or e >= E)
