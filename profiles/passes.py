"""Runs the listed cases of perf/operators.py one after the other through the public entry points, n
times each on two states in turn: the program that the profiler runs for profiles/operators.md.

    rocprofv3 --kernel-trace --stats -f csv -d <out> -- python3 profiles/passes.py 30
"""
import os
import sys

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import torch  # noqa: E402

from perf import operators  # noqa: E402

if __name__ == "__main__":
    operators.own = True
    for case in operators.listed():
        states = [operators.prepare(case, 5 + i) for i in range(2)]
        for i in range(int(sys.argv[1])):
            operators.run(states[i % 2])
        torch.cuda.synchronize()
        print(case["name"], flush=True)
