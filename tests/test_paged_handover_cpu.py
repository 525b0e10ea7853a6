"""What the warps of the paged attention kernels hand to one another, read in the source: which of two warps is ahead cannot be
arranged on a GPU at will."""
import os
import re

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2502_08923_b200", "csrc")


def _end(text, at):
    """Index behind the brace that closes the one before `at`."""
    depth = 1
    while depth:
        depth += {"{": 1, "}": -1}.get(text[at], 0)
        at += 1
    return at


def _source(name):
    return re.sub(r"//[^\n]*", "", open(os.path.join(CSRC, name)).read())


def _kernel(source, name):
    text = _source(source)
    at = re.search(rf"\b{name}\s*\([^;{{]*\)\s*\{{", text).end()
    return text[at:_end(text, at)]


def _without_lambdas(body):
    while m := re.search(r"auto \w+ = \[[^\]]*\]\([^)]*\)[^{;]*\{", body):
        body = body[:m.start()] + body[_end(body, m.end()):]
    return body


def test_queries_are_read_by_all_warps_before_any_warp_fetches_again():
    """The ring has one place more than a warp fetches tiles ahead.  Of pieces of one tile each it is full when a piece begins, and the fetch behind its tile goes to the
    piece's own place; every warp writes two of the sixteen rows that every warp reads.  So a barrier lies between."""
    body = _kernel("cs_paged_attn.cu", "k_paged_few")
    assert re.search(r"queries\(\);", re.search(r"auto fetch = .*?\n  \};", body, flags=re.S).group(0)) and "s_q" in re.search(r"auto begin = .*?\n  \};", body, flags=re.S).group(0)
    body = _without_lambdas(body)
    loop = re.search(r"for \(bool more = true; more;\) \{", body)
    calls = lambda text: re.findall(r"\b(begin\(\)|fetch\(\)|__syncthreads\(\));", text)
    inside = calls(body[loop.end():_end(body, loop.end())])
    order = calls(body[:loop.start()]) + 2 * inside
    assert order.count("begin()") >= 2 and order.count("fetch()") >= 3
    for i, call in enumerate(order):
        if call == "begin()":
            rest = order[i + 1:]
            assert "fetch()" not in rest or "__syncthreads()" in rest[:rest.index("fetch()")], order
            # (and they are there: a barrier lies behind the wait for their copies as well)
            before = order[:i][::-1]
            assert "__syncthreads()" in before and "fetch()" not in before[:before.index("__syncthreads()")], order
