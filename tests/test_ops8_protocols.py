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


def _pipeline_of_many_rows():
    """What gates what in gemm8_many_kernel, read from its source: whether a block's MMAs need its scales to have been asked for."""
    text = _source("gemm8.cuh")
    k = _body(text, text.index("gemm8_many_kernel(") - 1)
    arrivals = int(re.search(r"bar_init\(&full\[s\], (\d+)\)", k).group(1))
    scales = _body(k, k.index("else if (warp == 2)"))
    loop = _body(scales, scales.index("for (int kb = 0"))
    # one arrival per CTA's loads, one per CTA's scale warp; that one after every lane has seen the stage free
    gated = re.search(r"__all_sync\(0xffffffffu, bar_wait\(&empty\[stage\], [^)]*\)\)", loop) is not None
    gated = gated and re.search(r"if \(lane == 0\) bar_arrive\(peer_addr\(smem_addr\(&full\[stage\]\), 0\)\);", loop) is not None
    assert arrivals == (4 if gated else 2)
    return gated


def test_no_wait_of_the_product_of_many_rows_can_miss_its_phase():
    """A wait by parity misses its phase if the barrier completes the following one before the waiter has looked. It cannot where
    that following completion is a consequence of the waiter's own going on. Events of block i, over both CTAs c: L (tile loads
    asked for), S (scales asked for), M (products done), A (sums added, accumulator given back); edges are what each waits for."""
    gated = _pipeline_of_many_rows()
    for stages in (3, 4):
        slots, n = stages + 2, 40
        before = {}
        for i in range(n):
            for c in (0, 1):
                free = [("M", i - stages)]           # both wait for the same phase of empty[stage]
                before["L", c, i] = free + [("L", c, i - 1)]
                before["S", c, i] = free + [("S", c, i - 1)]
                before["A", c, i] = [("M", i), ("S", c, i), ("A", c, i - 1)]
            before["M", i] = [("M", i - 1)] + [("L", c, i) for c in (0, 1)] + [("A", c, i - 2) for c in (0, 1)]
            if gated:
                before["M", i] += [("S", c, i) for c in (0, 1)]

        def ancestors(e):
            seen, todo = set(), [e]
            while todo:
                for x in before.get(todo.pop(), []):
                    if x in before and x not in seen:
                        seen.add(x)
                        todo.append(x)
            return seen

        for i in range(n):
            past = ancestors(("M", i))
            for c in (0, 1):
                # empty[stage], completed by M(i - stages) and next by M(i): waited for by L(i) and S(i)
                assert ("L", c, i) in past, ("the loads", stages, i)
                assert ("S", c, i) in past, ("the scales", stages, i)
                # the two accumulators' barriers: tfull by M(i) and next by M(i + 2), tempty by A(i) and next by A(i + 2)
                if i + 2 < n:
                    assert ("A", c, i) in ancestors(("M", i + 2)) and ("M", i + 2) in ancestors(("A", c, i + 2))
                # a slot's scales are taken before the slot is written again, and its barrier's next phase comes after that
                if i + slots < n:
                    assert ("A", c, i) in ancestors(("S", c, i + slots))
