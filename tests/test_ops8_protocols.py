"""Order of accesses and waits in the kernels of the 8-bit operators and of the sampler, checked on their source: what blocks of a
cluster and roles of a pipeline may assume of one another. (A kernel that breaks one of these rules can hang or fault, and mostly
does not.) No GPU."""
import os
import re

import paper_2605_08696_b200

CSRC = os.path.join(os.path.dirname(paper_2605_08696_b200.__file__), "csrc")


def _source(name):
    """A source file without its comments."""
    with open(os.path.join(CSRC, name)) as f:
        return re.sub(r"//[^\n]*", "", f.read())


def _body(text, start):
    """The braces' content that follows position `start`."""
    i = text.index("{", start)
    depth = 0
    for j in range(i, len(text)):
        depth += {"{": 1, "}": -1}.get(text[j], 0)
        if depth == 0:
            return text[i + 1: j]
    raise AssertionError("unbalanced braces")


def _sampler():
    text = _source("sample.cuh")
    return _body(text, text.index("sample_kernel("))


def test_sampler_waits_for_the_cluster_before_it_reaches_into_another_block():
    """A block's shared memory may be accessed from others once all blocks of the cluster are known to run. The first access is
    the reduction of the maximum (what stands above it in lambdas runs later); all threads arrive and wait before it."""
    k = _sampler()
    first = k.index("g.max_of(")
    assert first < min(k.index(f"g.{f}(", first) for f in ("min_of", "add64", "add7")) and not re.search(r"\blead\.", k[:first])
    arrive, wait = k.find("cluster_arrive();"), k.find("cluster_wait();")
    assert 0 <= arrive < wait < first
    for at in (arrive, wait):                        # unconditional in the cluster's kernel: no thread is left out
        assert k[:at].rstrip().endswith("if (CL)")
        assert k[:at].count("{") == k[:at].count("}")
