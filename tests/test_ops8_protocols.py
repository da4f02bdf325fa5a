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


def test_sampler_flips_its_sets_of_places_only_where_all_ranks_wait():
    """Reductions use two sets of places in turn: the one after the next may write a set again, which is safe if every rank has
    passed a barrier of the whole cluster in between, that of the next one. A reduction of one block alone that flipped the set
    would leave none between a set's readers and its next writers."""
    text = _source("sample.cuh")
    group = _body(text, text.index("struct Group"))
    members = {m.group(1): _body(group, m.end()) for m in re.finditer(r"__device__ \w+ (\w+)\([^{]*\)\s*(?={)", group)}
    flips = {name for name, b in members.items() if "turn ^= 1" in b}
    assert {"max_of", "min_of", "add7", "add64"} <= flips <= set(members)
    for name in flips:
        assert "sync_all();" in members[name], name
        assert len(re.findall(r"\bturn\b", members[name])) == 2      # one set, taken and flipped
    # and a reduction of the block alone has places that no other one writes
    own = re.findall(r"\bs\.(\w+)\[warp\] = ", members["block_max"])
    assert len(own) == 1
    assert not any(re.search(rf"\bs\.{own[0]}\b", b) for name, b in members.items() if name != "block_max")
    assert not re.search(rf"\bs\.{own[0]}\b", _sampler())
