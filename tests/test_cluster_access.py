"""Kernels that access the shared memory of another block of their cluster: every block has to have started first,
which only a barrier of the whole cluster says (an access to a block that has not started is an error that no
test on a GPU may provoke).  Checked by reading the sources."""
import os
import re

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2509_08721_b200", "csrc")


def source(name):
    text = open(os.path.join(CSRC, name)).read()
    return re.sub(r"//[^\n]*", "", text)


def body(text, signature):
    """The braces that follow `signature`, their contents included."""
    at = text.index("{", text.index(signature))
    depth = 0
    for i in range(at, len(text)):
        depth += {"{": 1, "}": -1}.get(text[i], 0)
        if depth == 0:
            return text[at:i + 1]
    raise AssertionError("unbalanced braces")


def test_preference_kernel_waits_for_its_cluster_before_it_accesses_the_first_block():
    text = source("preference.cu")
    kernel = body(text, "preference_kernel(PrefArgs a)")
    remote = {"store_to_first", "load_from_first", "to_first"}      # what accesses the first block's shared memory
    # the lambda that names store_to_first is defined early and called later: calls count, its definition does not
    calls = re.sub(r"auto to_first = .*?;\s*\};", "", kernel, flags=re.S)
    first = min(m.start() for m in re.finditer(r"\b(%s)\(" % "|".join(remote), calls))
    assert "to_first(&" in calls
    arrive, wait = calls.index("cluster_arrive()"), calls.index("cluster_wait()")
    assert arrive < wait < first
    # every thread of every block takes part: nothing returns or branches off in between
    assert not re.search(r"\b(return|for|while)\b", calls[:wait])
    # and no block leaves while another may still read from it
    last = max(m.start() for m in re.finditer(r"\b(%s)\(" % "|".join(remote), calls))
    assert "cluster_barrier()" in calls[last:]


def test_no_other_source_maps_shared_memory_of_a_cluster_without_a_barrier():
    for name in sorted(os.listdir(CSRC)):
        text = source(name)
        if "shared::cluster" not in text or name in ("preference.cu", "umma.cuh"):
            continue
        assert "cluster_sync_all" in text, name
