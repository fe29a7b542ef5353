"""What a CTA of the tile kernel leaves behind when one of its waits gives up, read from the source: a wait that runs out inside a kernel at work
is nothing to bring about on a GPU."""
import os
import re

from tests.test_bounded_waits_cpu import CSRC, block

SOURCE = re.sub(r"//[^\n]*", "", open(os.path.join(CSRC, "paged_tile.cuh")).read())


def role(head):
    """A role's block, and what of it stands in no loop and under no condition that the role's own success decides."""
    at = SOURCE.index(head)
    return block(SOURCE, at + len(head) - 1)


def always(body):
    """The block without inner blocks: the statements that a warp comes to whatever became of its waits (a role has no return)."""
    out, depth = [], 0
    for c in body:
        depth -= c == "}"
        if depth == 0:
            out.append(c)
        depth += c == "{"
    return "".join(out)


def test_the_issuer_sees_its_products_through():
    """A role that has issued all it had to is through with its loop while another one gives up, so its own success says nothing."""
    body = role("if (warp == 0 && rows > 0) {")
    drains = re.findall(r"(if \([^;{}]*\)\s*)?drain\(latest, latest_parity\);", always(body))
    assert len(drains) == 1 and "ok" not in drains[0]
    # `latest` names the commit behind all products: between a product and the next wait there is a commit, and its name is taken
    loops = body[body.index("bool ok = true;"):]
    products = list(re.finditer(r"\b(?:mma_s|tc_mma_ts_n<[^;(]*>)\(", loops))
    assert len(products) == 4
    for product in products:
        behind = re.split(r"\b(?:mbar_wait_warp|ring_full)\(", loops[product.start():])[0]
        name = re.search(r"latest = (bar\(Y::\w+ \+ qt\));", behind)
        assert name and f"tc_commit({name.group(1)})" in behind[:name.start()], product.group(0)


def test_the_producer_sees_its_copies_through():
    body = role("else if (warp == 1 && rows > 0) {")
    assert re.search(r"for \(int k = max\(t - kStages, 0\); k < t; \+\+k\) drain\(bar\(kLanded \+ k % kStages\), \(k / kStages\) & 1\);", always(body))
