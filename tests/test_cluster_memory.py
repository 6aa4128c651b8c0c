"""Shared memory of other CTAs of a cluster: it may be touched only once all of them are known to run, which a cluster barrier alone tells, and as long as
none has left.  No run shows a missing barrier reliably, so the kernels' sources are read."""
import re
from pathlib import Path

import pytest

CSRC = Path(__file__).resolve().parent.parent / "paper_2609_07883_b200" / "csrc"
# barriers that a kernel passes by itself (not where a lambda is defined)
BARRIER = re.compile(r"^\s*(?:if \(ranks > 1\) )?(?:cluster_wait\(\)|cluster\.sync\(\)|all_here\(\));", re.M)
REMOTE = re.compile(r"\bmap_shared_rank\(|\bmapa\b")


def without_comments(text):
    return re.sub(r"//[^\n]*|/\*.*?\*/", "", text, flags=re.S)


def kernels_with_remote_memory():
    found = []
    for path in sorted([*CSRC.glob("*.cu"), *CSRC.glob("*.cuh")]):
        text = without_comments(path.read_text())
        for m in re.finditer(r"__global__", text):
            end = text.find("\n}", m.start())
            if REMOTE.search(text[m.start():end]):
                found.append(pytest.param(text[m.start():end], id=f"{path.name}-{len(found)}"))
    return found


def without_lambdas(body):
    """The kernel's own statements: lambdas run where they are called, behind whatever stands in front of that."""
    return re.sub(r"^    auto (\w+) = \[&\].*?^    \};|^    auto \w+ = \[&\][^\n]*\};$", "", body, flags=re.S | re.M)


def test_there_are_such_kernels():
    assert len(kernels_with_remote_memory()) == 2


@pytest.mark.parametrize("body", kernels_with_remote_memory())
def test_a_cluster_barrier_comes_before_the_first_remote_access(body):
    own = without_lambdas(body)
    assert REMOTE.search(own) and BARRIER.search(own)
    assert BARRIER.search(own).start() < REMOTE.search(own).start()


@pytest.mark.parametrize("body", kernels_with_remote_memory())
def test_a_cluster_barrier_comes_behind_the_last_remote_access(body):
    own = without_lambdas(body)
    assert [m.start() for m in BARRIER.finditer(own)][-1] > [m.start() for m in REMOTE.finditer(own)][-1]
