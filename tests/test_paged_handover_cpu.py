"""What the warps of the paged attention kernels hand to one another, read in the source: which of two warps is ahead cannot be
arranged on a GPU at will."""
import itertools
import os
import re

import pytest

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


# ---------------------------------------------------------------- the roles of k_paged_tc, as far as they wait for one another
class _Roles:
    """Pieces (slots have rows of their own, steps); a generator per role that yields the condition it waits for.  `stall`: this slot never
    gets further than `stall_at` of the waits it comes by in piece 0."""

    def __init__(self, pieces, apart, stall=None, stall_at=0):
        self.pieces, self.apart, self.stall, self.stall_at = pieces, apart, stall, stall_at
        self.done, self.published = set(), -1

    def has(self, *what):
        return lambda: what in self.done

    def queries(self):
        for i in range(len(self.pieces)):
            self.published = i
            self.done.add(("known", i))
            if i > 0:
                yield self.has("q free", i - 1)
            self.done.add(("q", i))

    def products(self):
        for i, (both, n) in enumerate(self.pieces):
            yield self.has("known", i)
            yield self.has("q", i)

            def scores(s):
                self.done.add(("s", i, s))
                if s == n - 1:
                    self.done.add(("q free", i))
            scores(0)
            if n > 1:
                scores(1)
            for s in range(n):
                if self.apart and s + 2 < n:
                    yield self.has("taken", i, s)
                    scores(s + 2)
                yield self.has("p", i, s)
                self.done.add(("o", i, s))
                if not self.apart and s + 2 < n:
                    scores(s + 2)

    def softmax(self, slot):
        for i, (both, n) in enumerate(self.pieces):
            yield self.has("known", i)
            for s in range(slot, n, 2):
                yield self.has("s", i, s)
                self.done.add(("taken", i, s))
                if self.apart and s > 1:
                    yield self.has("o", i, s - 2)
                self.done.add(("p", i, s))
            for s in range(n):
                if not both or s % 2 == slot:
                    yield self.has("o", i, s)
            for meeting in () if both else ("sums", "read"):
                self.done.add((meeting, i, slot))
                yield self.has(meeting, i, 1 - slot)

    def run(self):
        roles = [self.queries(), self.products(), self.softmax(0), self.softmax(1)]
        wants, passed = [next(r) for r in roles], [0] * 4
        moved = True
        while moved:
            moved = False
            for k, r in enumerate(roles):
                while wants[k] is not None and wants[k]() and not (self.stall is not None and k == 2 + self.stall and passed[k] == self.stall_at):
                    moved = True
                    passed[k] += 1
                    wants[k] = next(r, None)
        self.passed = passed
        return all(w is None for w in wants)


KINDS = [(False, 1), (False, 2), (False, 3), (True, 2), (True, 4)]


@pytest.mark.parametrize("apart", [False, True])
def test_descriptors_outlive_the_slot_that_lags(apart):
    """A piece's descriptor is read until its results are written; the one that takes its place is published only then.  Whatever the next pieces are, and wherever in the
    first one a slot stops, the others come to a halt before."""
    places = int(re.search(r"constexpr int kPieces = (\d+);", _source("cs_paged_attn_tc.cu")).group(1))
    furthest = 0
    for pieces in itertools.product(KINDS, repeat=5):
        run = _Roles(pieces + ((False, 1),) * 6, apart)
        assert run.run() and run.published == 10           # (nobody stops: all comes to its end)
        for slot in (0, 1):
            both, n = pieces[0]
            waits = 1 + sum((2 if apart and s > 1 else 1) for s in range(slot, n, 2)) + sum(not both or s % 2 == slot for s in range(n))      # ahead of its results
            for at in range(1, waits + 1 + (not both)):
                run = _Roles(pieces + ((False, 1),) * 6, apart, slot, at)
                assert not run.run() and run.passed[2 + slot] == at
                furthest = max(furthest, run.published)
    assert furthest == 4 and furthest < places, (furthest, places)


def test_a_second_pass_is_agreed_on():
    """Where a pass ends all roles meet.  One whose wait has run out leaves there, so the others may go on to a second pass, and to its end, only if the
    meeting itself has found that none has: a flag looked at before or after it may be another one for every role."""
    body = _kernel("cs_paged_attn_tc.cu", "k_paged_tc")
    again = re.search(r"auto again = \[&\]\(bool second\) -> bool \{(.*?)\n  \};", body, flags=re.S).group(1)
    asked = re.search(r"setp\.eq\.b32 p, %1, 0;\\n(bar\.red\.and\.pred) q, 0, p;.*?: \"=r\"\((\w+)\) : \"r\"\(flag\(f_abort\)\)", again, flags=re.S)
    assert asked and re.search(rf"return !second && {asked.group(2)} != 0 &&", again)
    # every way out of a role's loop comes by exactly one meeting: the one at a pass's end, or the one behind the loop
    assert body.count("if (!met) again(true);") == 2 and body.count("met = true;") == 4 and len(re.findall(r"\bagain\(", body)) == 6
