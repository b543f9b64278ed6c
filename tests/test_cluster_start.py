"""A kernel that writes into the shared memory of its cluster's other CTAs has to know first that they have started.  A missing wait
shows as nothing on almost every run, so that the sources are read instead: in a kernel's text a cluster barrier, or the wait for the
cluster's start, stands ahead of the first remote access."""
import re
from pathlib import Path

import pytest

CSRC = Path(__file__).resolve().parent.parent / "paper_2605_13319_b200" / "csrc"
REMOTE = re.compile(r"shared::cluster\.f64 \[|\bdsmem_st_f(32|64)\(|\bmbar_arrive_cluster\(")
BARRIER = re.compile(r"\bcluster_sync_all\(\)|\bcluster_started_wait\(\)")


def _kernel(file, name):
    """The text of a kernel, from its name to the next kernel or the file's end."""
    text = re.sub(r"//[^\n]*", "", (CSRC / file).read_text())
    start = re.search(r"__global__[^;{]*\b" + name + r"\(", text).end()
    end = text.find("__global__", start)
    return text[start:end if end >= 0 else len(text)]


@pytest.mark.parametrize("file,name", [("serving/shape.cuh", "accept_shaped_kernel"), ("reject.cuh", "accept_sample_kernel"),
                                       ("gemm.cuh", "gemm_wstream_kernel"), ("gemm_dense.cuh", "gemm_dense_kernel")])
def test_a_cluster_has_started_before_it_is_written_to(file, name):
    body = _kernel(file, name)
    remote, barrier = REMOTE.search(body), BARRIER.search(body)
    assert remote and barrier and barrier.start() < remote.start()
    # a thread that waits has arrived, and whoever arrives waits: no return between the two
    arrive = body.find("cluster_started_arrive()")
    if arrive >= 0:
        assert arrive < barrier.start() and "return;" not in body[arrive:barrier.start()]
