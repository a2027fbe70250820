"""The DRAM traffic that the bench line quotes for its kernels was captured on the
kernels that are there: a change of their source calls for a new capture, not for
a line without one."""
import json
import os

import pytest

import bench

with open(os.path.join(bench.ROOT, "profiles", "traffic.json")) as f:
    KERNELS = [k for k in json.load(f) if not k.startswith("_")]


@pytest.mark.parametrize("kernel", KERNELS)
def test_traffic_is_of_the_present_kernels(kernel):
    assert bench.traffic_for(kernel) > 0
