"""Barriers of thread-block clusters in the CUDA sources: a wait belongs to an arrival.  A wait without one passes at once or never, so
that a block may write to the shared memory of another that has not started; no run shows it reliably, the source does."""
import os
import re

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2105_13890_b200", "csrc")


def code_of(name):
    with open(os.path.join(CSRC, name)) as f:
        return re.sub(r"//[^\n]*", "", f.read())


@pytest.mark.parametrize("name", sorted(f for f in os.listdir(CSRC) if f.endswith(".cu")))
def test_every_wait_has_its_arrival(name):
    text = code_of(name)
    # by kernel: from one __global__ to the next
    for kernel in text.split("__global__")[1:]:
        steps = re.findall(r"ptx::cluster_(arrive|wait|sync)\(\)", kernel)
        open_arrivals = 0
        for step in steps:
            assert step != "sync" or open_arrivals == 0, "a sync between an arrival and its wait"
            open_arrivals += {"arrive": 1, "wait": -1, "sync": 0}[step]
            assert 0 <= open_arrivals <= 1, "a wait without an arrival, or two arrivals in one phase"
        assert open_arrivals == 0, "an arrival without a wait"
