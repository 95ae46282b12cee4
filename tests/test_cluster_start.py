"""Kernels whose CTAs share memory in a cluster: another CTA's shared memory is touched only once that CTA is known to have started.

A barrier behind the access covers the end of the other CTA, not its start.  A missing one is a race that hardly ever shows, so the
sources are read instead: before every access to another CTA's memory stands a wait at the cluster's barrier, and what waits there has
arrived at the beginning of its kernel."""
import os
import re

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2605_05802_b200", "csrc")
ACCESS = re.compile(r"map_shared_rank\(|store_at\(")
WHOLE = re.compile(r"(cluster|this_cluster\(\))\.sync\(\)")                  # arrives and waits
WAIT = re.compile(r"cluster_wait\(\)|barrier\.cluster\.wait")
ARRIVE = re.compile(r"cluster_arrive\(\)|barrier\.cluster\.arrive")


def functions(name):
    """(name, body) of every function at the top level of a source file, without comments."""
    text = re.sub(r"//[^\n]*", "", open(os.path.join(CSRC, name)).read())
    for m in re.finditer(r"^[^\s#/}][^\n;]*\(", text, re.M):
        begin = text.find("{", m.start())
        if begin < 0 or ";" in re.sub(r"\([^()]*(\([^()]*\)[^()]*)*\)", "", text[m.start():begin]):
            continue
        depth = 0
        for at in range(begin, len(text)):
            depth += (text[at] == "{") - (text[at] == "}")
            if depth == 0:
                break
        head = text[m.start():begin]
        names = re.findall(r"(\w+)\s*\(", head)
        if names:
            yield names[-1 if "__launch_bounds__" in head else 0], text[begin:at + 1]


@pytest.mark.parametrize("name", sorted(f for f in os.listdir(CSRC) if f.endswith((".cu", ".cuh"))))
def test_nobody_writes_to_a_cta_that_may_not_have_started(name):
    waits = {}
    for function, body in functions(name):
        # a lambda's body runs where it is called: behind the waits of the function that it stands in
        accesses = [m.start() for m in ACCESS.finditer(re.sub(r"auto settle = .*?\n        };", lambda m: " " * len(m.group()), body, flags=re.S))]
        if not accesses or (name == "ring.cuh" and function == "store_at"):
            continue
        before = body[:accesses[0]]
        assert WHOLE.search(before) or WAIT.search(before), f"{name}: {function} touches another CTA's memory before any wait"
        if not WHOLE.search(before):
            waits[function] = bool(ARRIVE.search(before))
    # where the arrival is not the function's own, every kernel that calls it has one before the call
    for function in (f for f, own in waits.items() if not own):
        callers = [(n, b) for n, b in functions(name) if re.search(rf"\b{function}<", b)]
        assert callers
        for caller, body in callers:
            assert ARRIVE.search(body[:re.search(rf"\b{function}<", body).start()]), f"{name}: {caller} calls {function} without an arrival"


def test_the_reading_finds_functions():
    names = {n: [f for f, _ in functions(n)] for n in os.listdir(CSRC) if n.endswith(".cu")}
    assert "combine" in names["logprob.cu"] and "held_policy_loss_kernel" in names["logprob.cu"] and "token_list_kernel" in names["logprob.cu"]
    assert "leave_sum" in names["policy.cu"] and "loss_weights_kernel" in names["policy.cu"] and "policy_loss_kernel" in names["policy.cu"]
