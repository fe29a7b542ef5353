"""A named barrier knows no limit, so every warp that it counts has to come to it, one whose bounded wait gave up as well: a loop that holds
such a barrier is left by all of them or by none.  Read from the sources, as a wait that runs out is nothing to bring about on a GPU."""
import os
import re

import pytest

from tests.test_bounded_waits_cpu import SOURCES, block

BARRIER = re.compile(r"\b(?:bar|barrier\.cta)\.(?:sync|red)[.\w]*\s+(?:\w+\s*,\s*)?(?!0\b)[%\w]+\s*,\s*[%\w]+")


def bodies(text, head):
    """(first line, body) of every block behind a match of `head`."""
    return [(m.group(0), m.end(), block(text, m.end() - 1)) for m in re.finditer(head, text)]


def left_alone(text):
    """Loops around a named barrier that a warp may leave by itself: the statement that does it."""
    text = re.sub(r"//[^\n]*", "", text)
    meets, votes = set(), set()                      # what a call of meets everybody; what also tells all of them the same
    for head, _, body in bodies(text, r"auto \w+ = \[[^\]]*\]\s*(?:\([^)]*\))?\s*\{") + bodies(text, r"__device__ [^;{}()]*\w+\([^;{}]*\)\s*\{"):
        name = re.search(r"auto (\w+)|(\w+)\(", head)
        if BARRIER.search(body) and not re.search(r"\b(for|while)\b", body):
            meets.add(name.group(1) or name.group(2))
            if ".red." in body:
                votes.add(name.group(1) or name.group(2))
    call = lambda names: re.compile(r"\b(?:%s)\(" % "|".join(sorted(names) or ["-"]))
    found = []
    for head, at, body in bodies(text, r"\b(?:for|while) \((?:[^(){}]|\([^()]*\))*\) \{"):
        own = body                                   # without the loops inside, which are looked at by themselves
        for _, i, inner in reversed(bodies(body, r"\b(?:for|while) \((?:[^(){}]|\([^()]*\))*\) \{")):
            own = own.replace(inner, " ")
        if not (BARRIER.search(own) or call(meets).search(own)):
            continue
        if re.search(r"\bok\b", head):
            found.append(head)
        for m in re.finditer(r"[^;{}]*\b(?:break|return)\b[^;]*;", own):
            if not call(votes).search(m.group(0)):
                found.append(m.group(0).strip())
    return found


@pytest.mark.parametrize("path", SOURCES, ids=os.path.basename)
def test_nobody_leaves_a_loop_with_a_named_barrier_alone(path):
    assert left_alone(open(path).read()) == []


def test_such_a_loop_is_seen():
    one = 'for (int t = 0; t < n; ++t) { bool ok = mbar_wait_warp(b, 0); if (!ok) break; asm volatile("bar.sync 3, 128;" ::: "memory"); }\n'
    lambda_ = 'auto meet = [&] { asm volatile("bar.sync 3, 128;" ::: "memory"); };\n'
    vote = '__device__ bool everybody(bool mine) { asm volatile("bar.red.and.pred q, 3, 128, p;" : "=r"(all)); return all; }\n'
    assert left_alone(one) and left_alone(one.replace("bar.sync", "barrier.cta.sync"))
    assert left_alone(lambda_ + "for (int i = 0; i < n; ++i) { if (!ok) break; meet(); }")
    assert left_alone(lambda_ + "for (int i = 0; i < n && ok; ++i) { meet(); }")
    assert left_alone(vote + "for (int i = 0; i < n; ++i) { everybody(ok); if (!ok) break; }")
    assert not left_alone(vote + "for (int i = 0; i < n; ++i) { ok = wait(); if (!everybody(ok)) break; }")
    assert not left_alone(lambda_ + "for (int i = 0; i < n; ++i) { ok = ok && wait(); if (ok) go(); meet(); }")
    assert not left_alone('for (int i = 0; i < n; ++i) { if (!ok) break; __syncthreads(); asm volatile("bar.sync 0, 128;"); }')
