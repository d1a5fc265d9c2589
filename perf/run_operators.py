"""Runs cases of `perf/operators.py` through the framework's kernels, for a profiler:

    rocprofv3 --kernel-trace --stats -f csv -d OUT -o n -- python3 perf/run_operators.py [NAME ...]

Each named case (all of them without names) is prepared three times and run 30
times on the three states in turn."""
import os
import sys

sys.path[:0] = [os.path.dirname(os.path.dirname(os.path.abspath(__file__)))]

import torch  # noqa: E402

from perf import operators  # noqa: E402


def main(names):
    operators.own = True
    for case in operators.listed():
        if names and case["name"] not in names:
            continue
        states = [operators.prepare(case, seed) for seed in range(3)]
        for i in range(30):
            operators.run(states[i % 3])
        torch.cuda.synchronize()
        print(case["name"], flush=True)


if __name__ == "__main__":
    main(sys.argv[1:])
