"""Calls listed cases of perf/operators.py, for a profiler around it:  python3 profiles/paged_case.py <name>[,<name>] <passes>"""
import os
import sys

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
sys.path.insert(0, ROOT)
os.chdir(ROOT)
import torch  # noqa: E402

from perf import operators as O  # noqa: E402

O.own = True
cases = {c["name"]: c for c in O.listed()}
for name in sys.argv[1].split(","):
    state = O.prepare(cases[name], 1)
    for _ in range(int(sys.argv[2])):
        O.run(state)
    torch.cuda.synchronize()
    print("ran", name, flush=True)
