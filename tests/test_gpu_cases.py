"""The cases of perf/more_operators.py whose outputs are moved or whole: their plain forms and the library's calls, each against the definition.

In a process of its own: the HIP runtime that torch brings along does not see the GPU once the library's has initialised it."""
import os
import subprocess
import sys

import pytest

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CHILD = """
import random, sys
import torch
torch.zeros(1, device="cuda")
from perf import more_operators as cases
op, what, names = sys.argv[1], sys.argv[2] or None, sys.argv[3].split(",")
rng, drawn = random.Random(5), []
while len(drawn) < 40:
    c = cases.draw(rng)
    if c["op"] == op and c.get("what") == what and c.get("batch", 1) * c.get("beams", 1) * c.get("vocab", 1) < 1 << 22:
        drawn.append(c)
wrong = []
for cases.own in (False, True):
    for i, c in enumerate(drawn):
        want, got = cases.exact(c, 100 + i), cases.run(cases.prepare(c, 100 + i))
        wrong += [(cases.own, name, c) for name in names if not bool((got[name].view(want[name].shape) == want[name]).all())]
    print(len(drawn), "cases, own", cases.own, flush=True)
for w in wrong:
    print("WRONG", *w)
sys.exit(1 if wrong else 0)
"""


@pytest.mark.parametrize("op,what,names", [("pages", "compact", "table,lengths,refs,codes,scales,used"), ("pages", "beams", "table,lengths,refs,codes,scales"),
                                           ("beams", "", "parents,tokens,lengths,finished,history")])
def test_moved_and_whole_outputs(op, what, names):
    r = subprocess.run([sys.executable, "-c", CHILD, op, what, names], cwd=ROOT, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True, timeout=100)
    assert r.returncode == 0, r.stdout[-4000:]
    assert r.stdout.count("40 cases") == 2
