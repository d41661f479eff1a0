"""Blocks of a cluster may touch each other's shared memory only once all of them are known to run: a kernel that names an
address of another block passes a barrier of the cluster first.  Read from the sources, without a GPU."""
import glob
import os
import re

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2401_04044_b200", "csrc")
COMMENT = re.compile(r"//[^\n]*|/\*.*?\*/", re.S)
REMOTE = re.compile(r"map_to_cta\(|(?:ld|st)\.shared::cluster|\bmapa\b")


def kernels():
    """(file, name, body) of every kernel: its text up to the next one's."""
    out = []
    for path in sorted(glob.glob(os.path.join(CSRC, "*.cu"))):
        text = COMMENT.sub("", open(path).read())
        starts = [m.start() for m in re.finditer(r"__global__", text)] + [len(text)]
        for a, b in zip(starts, starts[1:]):
            body = text[a:b]
            out.append((os.path.basename(path), re.search(r"(\w+_kernel)\b", body).group(1), body))
    return out


FOUND = [k for k in kernels() if REMOTE.search(k[2])]


def test_there_are_such_kernels():
    assert {"thin_solve_kernel", "muon_gemm_kernel", "muon_square_kernel", "shrink_tc_kernel", "train_gemm_kernel"} <= {k[1] for k in FOUND}


@pytest.mark.parametrize("file,name,body", FOUND, ids=[k[1] for k in FOUND])
def test_a_barrier_of_the_cluster_comes_first(file, name, body):
    barrier = body.find("cluster_sync_all(")
    assert 0 <= barrier < REMOTE.search(body).start(), f"{file}: {name} names another block's shared memory before a barrier of the cluster"
