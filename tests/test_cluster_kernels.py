"""Orders that no run can show, by the sources.  A block's shared memory is reached from another only behind a barrier of the cluster, before which nothing says that it has begun;
tensor memory is asked for when the kernel in front has ended."""
import os
import re

import pytest

from paper_2411_04975_b200 import build

BARRIER = re.compile(r"barrier_wait\(\)|cluster\.sync\(\)|cluster_sync\(\)|barrier\.cluster\.wait")


def kernels():
    """(name, body) of the kernels in the sources that reach other blocks' memory."""
    for f in sorted(os.listdir(build.CSRC)):
        if f.endswith((".cu", ".cuh")):
            with open(os.path.join(build.CSRC, f)) as h:
                parts = re.split(r"__global__", h.read())[1:]
            for p in parts:
                body = p.split("\n}\n")[0]
                if "map_shared_rank" in body:
                    yield pytest.param(body, id=f + ":" + re.search(r"(\w+_kernel)\(", body).group(1))


@pytest.mark.parametrize("body", list(kernels()))
def test_blocks_of_a_cluster_are_there_before_their_memory_is_reached(body):
    barrier = BARRIER.search(body)
    assert barrier and barrier.start() < body.index("map_shared_rank")


def test_there_are_such_kernels():
    assert len(list(kernels())) >= 2


def test_tensor_memory_is_asked_for_behind_the_kernel_before():
    """Asked for while the kernel in front still runs, it could be what that kernel asks for next, and each would wait for the other."""
    with open(os.path.join(build.CSRC, "attend.cu")) as h:
        body = re.split(r"__global__", h.read())[1].split("\n}\n")[0]
    assert body.index("griddepcontrol.wait") < body.index("bw_tmem_alloc(")
