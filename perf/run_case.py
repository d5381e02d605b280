"""Runs one listed case of perf/more_operators.py through the library N times, for a profiler to watch:

    rocprofv3 --kernel-trace --stats -d OUT -o r -f csv -- python3 perf/run_case.py CASE N
"""
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from perf import more_operators as ops  # noqa: E402


def main():
    if len(sys.argv) != 3:
        sys.exit(__doc__)
    ops.own = True
    case = next((c for c in ops.listed() if c["name"] == sys.argv[1]), None)
    if case is None:
        sys.exit("no case %s; there are: %s" % (sys.argv[1], " ".join(c["name"] for c in ops.listed())))
    state = ops.prepare(case, 1)
    torch.cuda.synchronize()
    for _ in range(int(sys.argv[2])):
        ops.run(state)
    torch.cuda.synchronize()


if __name__ == "__main__":
    main()
