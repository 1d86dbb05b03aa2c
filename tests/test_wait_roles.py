"""Who may wait how, read from the kernels' source.

A bounded wait (mbar_wait) answers each lane by itself: its own clock may run out while its neighbours see the barrier complete.  Lanes that
disagree and then meet in an instruction of the whole warp stand there for ever.  So a wait is either one lane's, or the warp
decides together (a vote), or the verdict goes to a barrier that carries it before anything else of the warp's or block's, or it is kept
(`in_time`) and looked at in votes only."""
import glob
import os
import re

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2609_20744_b200", "csrc")
ONE_LANE = re.compile(r"\b(lane|tid|et|threadIdx\.x)\s*==\s*(0|W::WALKERS)\b")
COLLECTIVE = re.compile(r"__syncthreads\w*|named_barrier_or|__syncwarp|__(?:shfl|any|all|ballot|reduce|match)\w*_sync|__shfl\w*|tmem_\w+|"
                        r"mbar_arrive_warp|cluster_sync|elect_one|registers_\w+")
CARRIES = re.compile(r"(__syncthreads_or|named_barrier_or)\([^;]*(!ok|landed \?)")


def source(path):
    text = open(path).read()
    text = re.sub(r"//[^\n]*", lambda m: " " * len(m.group()), text)
    return re.sub(r"/\*.*?\*/", lambda m: re.sub(r"[^\n]", " ", m.group()), text, flags=re.S)


def headers(text, at):
    """What stands before each open brace around `at`, and the statement that `at` is in."""
    found, depth, i = [], 0, at
    start = max(text.rfind(c, 0, at) for c in ";{}")
    found.append(text[start + 1: at])
    while i > 0:
        i -= 1
        if text[i] == "}":
            depth += 1
        elif text[i] == "{":
            if depth:
                depth -= 1
            else:
                j = max(text.rfind(c, 0, i) for c in ";{}")
                found.append(text[j + 1: i])
    return found


def kept_for_votes(text):
    """Every look at in_time is inside a vote."""
    text = re.sub(r"\bbool in_time = true;|\bin_time\s*=\s*mbar_wait\([^;]*&& in_time;", "", text)
    return not re.search(r"\bin_time\b", re.sub(r"__any_sync\(0xffffffffu,[^;{]*!in_time\)", "", text))


def lonely_waits(text):
    """Lines of waits whose lanes may go different ways."""
    bad = []
    for m in re.finditer(r"\bmbar_wait\(", text):
        around = headers(text, m.start())
        if re.search(r"\bbool\s+$", around[0]):                              # the definition
            continue
        if any(ONE_LANE.search(h) for h in around) or "__all_sync(" in around[0]:
            continue
        rest = text[text.index(";", m.end()):]
        first = COLLECTIVE.search(rest)
        if re.search(r"\b(ok|landed)\s*=\s*$", around[0]) and first and CARRIES.match(rest, first.start()):
            continue
        if re.search(r"\bin_time\s*=\s*$", around[0]) and kept_for_votes(text):
            continue
        bad.append(text[: m.start()].count("\n") + 1)
    return bad


@pytest.mark.parametrize("path", sorted(glob.glob(os.path.join(CSRC, "*.cuh"))), ids=os.path.basename)
def test_lanes_of_a_warp_leave_a_wait_together(path):
    assert lonely_waits(source(path)) == []


def test_the_rule_tells_them_apart():
    wait = "mbar_wait(FULL, 0, wc)"
    assert lonely_waits("{ if (!%s) { ok = false; break; } tmem_ld16(a, b); }" % wait) == [1]
    assert lonely_waits("{ ok = %s; tmem_ld16(a, b); __syncthreads_or(!ok); }" % wait) == [1]
    assert lonely_waits("{ ok = %s; if (__syncthreads_or(!ok)) break; tmem_ld16(a, b); }" % wait) == []
    kept = "{ bool in_time = true; for (;;) { in_time = mbar_wait(FULL(a), (it >> 1) & 1, wc) && in_time; %s } }"
    assert lonely_waits(kept % "odd = __any_sync(0xffffffffu, !normal_number(s) || !in_time);") == []
    assert lonely_waits(kept % "if (odd) { if (__any_sync(0xffffffffu, !in_time)) break; }") == []
    assert lonely_waits(kept % "if (!in_time) break;") == [1]
    assert lonely_waits("{ if (lane == 0) { for (;;) { if (!%s) break; } } }" % wait) == []
    assert lonely_waits("{ if (!__all_sync(0xffffffffu, %s)) break; }" % wait) == []
    assert lonely_waits("{ if (!mbar_wait_warp(FULL, 0, wc)) break; tmem_ld16(a, b); }") == []


@pytest.mark.parametrize("path", sorted(glob.glob(os.path.join(CSRC, "*.cuh"))), ids=os.path.basename)
def test_a_block_that_gave_up_settles_before_it_goes(path):
    """What is on its way into a block's shared and tensor memory is given time before either goes to another: between the last barrier
    and the return of tensor memory (which a cluster's last barrier follows)."""
    text = source(path)
    for m in re.finditer(r"\btmem_dealloc(_pair)?\(", text):
        if re.search(r"\bvoid\s+$", text[: m.start()]):                       # the definition
            continue
        end = text[text.rindex("__syncthreads();", 0, m.start()): m.start()]
        assert "settle(" in end, text[: m.start()].count("\n") + 1
