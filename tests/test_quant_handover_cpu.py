"""What the warps of the attention of tall blocks over 4 bits hand to one another, as a model of its barriers: two warps fetch tiles as they lie in the cache, four write them out in 16 bits, a half of a tile's rows each, and the ring,
the products and the softmax go on from there.  Barriers have phases, parities and counts as on the device, copies land and products end in their own time, and any role may lag as far as the others let it."""
import itertools
import random
import re

import pytest

from test_paged_handover_cpu import KINDS, _kernel, _source

NAME = "cs_paged_attn_tc.cu"


def constants():
    text = _source(NAME)
    number = lambda pattern: int(re.search(pattern, text).group(1))
    return dict(pieces=number(r"constexpr int kPieces = (\d+);"), packed=number(r"constexpr int kPackedTiles = (\d+);"),
                stages={True: number(r"constexpr int kStages = DH == 128 \? \(kQuant \? \d+ : \d+\) : (\d+);"), False: number(r"constexpr int kStages = DH == 128 \? \(kQuant \? (\d+)")},
                full=number(r"mbar_init\(b_full \+ 8 \* s, kQuant \? (\d+)"), empty=number(r"mbar_init\(b_empty \+ 8 \* s, (\d+)\)"),
                unpacked=number(r"mbar_init\(b_unpacked \+ 8 \* s, (\d+)\)"), landed=number(r"mbar_init\(b_packed \+ 8 \* s, (\d+)\)"))


class Wrong(Exception):
    pass


class Bar:
    def __init__(self, count):
        self.count, self.left, self.phase = count, count, 0

    def arrive(self):
        self.left -= 1
        if self.left == 0:
            self.left, self.phase = self.count, self.phase + 1


class Call:
    """A CTA's pieces (slots have rows of their own, steps), gone through once or twice; `apart`: weights have columns of their own, and scores are made ahead."""

    def __init__(self, pieces, apart, passes=1, **changed):
        c = constants()
        self.ns, self.np, self.nd = c["stages"][apart], c["packed"], c["pieces"]
        self.apart, self.passes = apart, passes
        count = {n: changed.get(n, c[n]) for n in ("full", "empty", "unpacked", "landed")}
        self.no_wait = changed.get("no_wait")             # a wait left out
        self.line = [(i, second, p) for second in range(passes) for i, p in enumerate(pieces + [None])]
        bars = lambda n, k: [Bar(k) for _ in range(n)]
        self.full, self.empty = bars(self.ns, count["full"]), bars(self.ns, count["empty"])
        self.landed, self.unpacked = {k: bars(self.np, count["landed"]) for k in "KV"}, {k: bars(self.np, count["unpacked"]) for k in "KV"}
        self.piece, self.qfull, self.qfree = bars(self.nd, 1), Bar(1), Bar(1)
        self.s, self.p, self.o, self.taken = bars(2, 1), bars(2, 1), bars(2, 1), bars(2, 1)
        self.ml, self.read, self.met = Bar(2), Bar(2), Bar(10)
        self.described, self.queries = [None] * self.nd, None
        self.ring, self.packed = [None] * self.ns, {k: [None] * self.np for k in "KV"}
        self.scores, self.weights = [None, None], [None, None]
        self.flying, self.queue = [], []                   # copies, products under way
        self.roles = {"queries": self._queries(), "products": self._products(), "softmax 0": self._softmax(0), "softmax 1": self._softmax(1)}
        for k in "KV":
            self.roles["fetch " + k] = self._fetch(k)
            for half in (0, 1):
                self.roles[f"expand {k}{half}"] = self._expand(k, half)

    # ---- the order of the ring
    def _ahead(self, both):
        return (1 if both else 2) + (1 if self.apart else 0)

    def _k_entry(self, both, s):
        i, ahead = s >> 1 if both else s, self._ahead(both)
        return i if i < ahead else 2 * i - ahead + 1

    def _v_entry(self, both, s, n):
        i, tiles = (s >> 1, n >> 1) if both else (s, n)
        return i + min(i + self._ahead(both), tiles)

    def _entry(self, kind, both, s, n):
        return self._k_entry(both, s) if kind == "K" else self._v_entry(both, s, n)

    # ---- roles: generators that yield (barrier, parity) to wait for
    def _known(self, number):
        yield self.piece[number % self.nd], number // self.nd & 1
        return self._look(number)

    def _look(self, number):
        if self.described[number % self.nd] != number:
            raise Wrong(f"descriptor of piece {number} has been overwritten")
        return self.line[number][2], self.line[number][1]

    def _meet(self):
        phase = self.met.phase
        self.met.arrive()
        yield self.met, phase & 1

    def _queries(self):
        for number, (_, second, d) in enumerate(self.line):
            self.described[number % self.nd] = number
            self.piece[number % self.nd].arrive()
            if d is None:
                yield from self._meet()
                continue
            if number - second > 0:
                yield self.qfree, (number - second - 1) & 1
            self.flying.append(("queries", number, None))

    def _fetch(self, kind):
        no = 0
        for number in range(len(self.line)):
            d, _ = yield from self._known(number)
            if d is None:
                yield from self._meet()
                continue
            both, n = d
            for s in range(0, n, 2 if both else 1):
                b = no % self.np
                if self.no_wait != "unpacked":
                    yield self.unpacked[kind][b], (no // self.np & 1) ^ 1
                self._look(number)
                self.flying.append((kind, (number, s), b))
                no += 1

    def _expand(self, kind, half):
        no = base = 0
        for number in range(len(self.line)):
            d, _ = yield from self._known(number)
            if d is None:
                yield from self._meet()
                continue
            both, n = d
            for s in range(0, n, 2 if both else 1):
                e = base + self._entry(kind, both, s, n)
                b, st = no % self.np, e % self.ns
                if self.no_wait != "packed":
                    yield self.landed[kind][b], no // self.np & 1
                if self.no_wait != "empty":
                    yield self.empty[st], (e // self.ns & 1) ^ 1
                tile = self.packed[kind][b]
                if tile is None or tile["what"] != (number, s) or half in tile["read"]:
                    raise Wrong(f"{kind} tile {number, s} is not where it is read")
                place = self.ring[st]
                if place is None or place["entry"] != e:
                    if place is not None and not place["free"]:
                        raise Wrong(f"ring entry {place['entry']} is overwritten")
                    place = self.ring[st] = {"entry": e, "what": (kind, number, s), "halves": set(), "free": False}
                place["halves"].add(half)
                tile["read"].add(half)
                self.unpacked[kind][b].arrive()
                self.full[st].arrive()
                no += 1
            base += n if both else 2 * n

    def _products(self):
        base, p_phase, t_phase = 0, [0, 0], [0, 0]
        for number in range(len(self.line)):
            d, second = yield from self._known(number)
            if d is None:
                yield from self._meet()
                continue
            both, n = d
            yield self.qfull, (number - second) & 1
            at, k_at, v_at = base, 0, 0

            def scores(s):
                nonlocal at, k_at
                if not both or not s & 1:
                    k_at = at
                    at += 1
                    yield self.full[k_at % self.ns], k_at // self.ns & 1
                self.queue.append(("s", number, s, k_at, both, [self.s[s & 1]] + ([self.empty[k_at % self.ns]] if not both or s & 1 else []) + ([self.qfree] if s == n - 1 else [])))
            yield from scores(0)
            if n > 1:
                yield from scores(1)
            for s in range(n):
                slot = s & 1
                if self.apart and s + 2 < n:
                    yield self.taken[slot], t_phase[slot]
                    yield from scores(s + 2)
                t_phase[slot] ^= self.apart
                if not both or not slot:
                    v_at = at
                    at += 1
                    yield self.full[v_at % self.ns], v_at // self.ns & 1
                yield self.p[slot], p_phase[slot]
                p_phase[slot] ^= 1
                self.queue.append(("o", number, s, v_at, both, ([self.empty[v_at % self.ns]] if not both or slot else []) + [self.o[slot]]))
                if not self.apart and s + 2 < n:
                    yield from scores(s + 2)
            base += n if both else 2 * n

    def _softmax(self, slot):
        base = s_phase = turns = mine = other = 0
        for number in range(len(self.line)):
            d, _ = yield from self._known(number)
            if d is None:
                yield from self._meet()
                continue
            both, n = d
            for s in range(slot, n, 2):
                yield self.s[slot], s_phase
                s_phase ^= 1
                e = base + self._v_entry(both, s, n)
                yield self.full[e % self.ns], e // self.ns & 1       # (V rows that nobody sees become zeros)
                if self.ring[e % self.ns]["what"] != ("V", number, s - (s & 1 if both else 0)):
                    raise Wrong("V rows of another tile become zeros")
                if self.scores[slot] != (number, s):
                    raise Wrong(f"scores {number, s} are not there")
                if self.apart:
                    self.scores[slot] = None
                    self.taken[slot].arrive()
                    if s > 1:
                        yield self.o[slot], (mine - 1) & 1
                if self.weights[slot] is not None:
                    raise Wrong(f"weights {self.weights[slot]} are overwritten")
                self.weights[slot] = (number, s)
                self.p[slot].arrive()
                mine += 1
            other += (n + slot) >> 1
            if n > slot:
                yield self.o[slot], (mine - 1) & 1
            if not both and n > 1 - slot:
                yield self.o[1 - slot], (other - 1) & 1
            if not both:
                self.ml.arrive()
                yield self.ml, turns & 1
            self._look(number)
            if not both:
                self.read.arrive()
                yield self.read, turns & 1
                turns += 1
            base += n if both else 2 * n

    # ---- what lands and ends by itself
    def _land(self, i):
        kind, what, b = self.flying.pop(i)
        if kind == "queries":
            self.queries = what
            self.qfull.arrive()
            return
        old = self.packed[kind][b]
        if old is not None and len(old["read"]) < 2:
            raise Wrong(f"{kind} tile {old['what']} is overwritten")
        self.packed[kind][b] = {"what": what, "read": set()}
        self.landed[kind][b].arrive()

    def _finish(self):
        op, number, s, e, both, bars = self.queue.pop(0)
        place, first = self.ring[e % self.ns], s - (s & 1 if both else 0)
        if place is None or place["entry"] != e or place["what"] != ("K" if op == "s" else "V", number, first) or len(place["halves"]) < 2:
            raise Wrong(f"a product of {number, s} without its tile")
        if op == "s":
            if self.queries != number or (self.apart and self.scores[s & 1] is not None):
                raise Wrong(f"scores of {number, s}")
            self.scores[s & 1] = (number, s)
        else:
            if self.weights[s & 1] != (number, s):
                raise Wrong(f"weights of {number, s}")
            self.weights[s & 1] = None
        if self.empty[e % self.ns] in bars:
            place["free"] = True
        for b in bars:
            b.arrive()

    def run(self, choose):
        """To its end, or until nothing moves; `choose` picks one of what can move."""
        wants = {name: next(r) if name != "queries" else None for name, r in self.roles.items()}
        wants["queries"] = next(self.roles["queries"])
        while True:
            able = [n for n, w in wants.items() if w is not None and (w[0].phase & 1) != w[1]]
            able += [f"copy {i}" for i in range(len(self.flying))] + (["product"] if self.queue else [])
            if not able:
                return all(w is None for w in wants.values())
            name = choose(able)
            if name == "product":
                self._finish()
            elif name.startswith("copy "):
                self._land(int(name[5:]))
            else:
                wants[name] = next(self.roles[name], None)


def by_chance(seed):
    rng = random.Random(seed)
    return lambda able: rng.choice(able)


def lagging(name, seed):
    """What bears that name moves only when nothing else can."""
    rng = random.Random(seed)

    def choose(able):
        rest = [x for x in able if not x.startswith(name)]
        return rng.choice(rest or able)
    return choose


LAGS = ["queries", "products", "softmax 0", "softmax 1", "fetch K", "fetch V", "expand K0", "expand K1", "expand V0", "expand V1", "expand K", "expand V", "copy", "product"]


@pytest.mark.parametrize("apart", [False, True])
def test_all_comes_to_its_end(apart):
    """Whatever the pieces are and whoever lags: no wait is for ever, no tile, packed place, descriptor, score or weight is taken for another or written over."""
    for seed, pieces in enumerate(itertools.product(KINDS, repeat=3)):
        for i, name in enumerate(LAGS):
            if (seed + i) % 4 == 0:
                assert Call(list(pieces), apart).run(lagging(name, seed)), (pieces, name)
        assert Call(list(pieces), apart, passes=2).run(by_chance(seed)), pieces


@pytest.mark.parametrize("apart", [False, True])
@pytest.mark.parametrize("name", LAGS)
def test_long_runs(apart, name):
    """Pieces of many steps, so that every ring goes round several times, and many pieces, so that descriptors do; two passes."""
    for seed in range(6):
        rng = random.Random(seed)
        pieces = [(both, rng.randint(1, 12) * (2 if both else 1)) for both in (rng.random() < 0.5 for _ in range(12))]
        assert Call(pieces, apart, passes=1 + seed % 2).run(lagging(name, seed)), (pieces, name)
        assert Call([(False, 1)] * 30, apart, passes=2).run(lagging(name, seed))


@pytest.mark.parametrize("apart", [False, True])
@pytest.mark.parametrize("changed", [dict(full=1), dict(unpacked=1), dict(no_wait="unpacked"), dict(no_wait="packed"), dict(no_wait="empty")])
def test_the_model_sees_mistakes(apart, changed):
    """A count of one where two warps arrive, or a wait left out: some run goes wrong."""
    def goes_wrong(name, seed):
        try:
            return not Call([(False, 5), (True, 8), (False, 20)], apart, **changed).run(lagging(name, seed))
        except (Wrong, TypeError):
            return True
    assert any(goes_wrong(name, seed) for name in LAGS for seed in range(3))


def test_the_source_hands_over_so():
    """The order of waits, reads and arrivals that the model has, in the source."""
    body = _kernel(NAME, "k_paged_tc")
    expand = body[body.index("else {", body.index("if (here && there) {")):]
    steps = [r"wait_warp\(b_packed \+ 8 \* buffer, \(packed_no / kTiles\) & 1\)", r"wait_warp\(b_empty \+ 8 \* st, \(\(e / kNS\) & 1\) \^ 1\)", r"expand_group<T>", r"fence\.proxy\.async\.shared::cta", r"__syncwarp\(\)",
             r"mbar_arrive\(b_unpacked \+ 8 \* buffer\)", r"mbar_arrive\(b_full \+ 8 \* st\)"]
    at = 0
    for s in steps:
        at += re.search(s, expand[at:]).end()
    fetch = body[:body.index("expand_group<T>")]
    at = fetch.rindex("wait_warp(b_unpacked + 8 * buffer, ((packed_no / kTiles) & 1) ^ 1)")
    assert re.search(r"mbar_expect_tx\(bar, bytes\);.*?bulk_load.*?bulk_load", fetch[at:], flags=re.S)
    # (a place that holds zeros instead of a copy is written to before the copy that follows in it)
    assert re.search(r"= 0u;.*?fence\.proxy\.async\.shared::cta.*?mbar_expect_tx", fetch[at:], flags=re.S)
    # (registers: three shares of the 512 x 128 that a block is launched with)
    text = _source(NAME)
    threads = int(re.search(r"kThreads = kQuant \? (\d+)", text).group(1))
    other, softmax = (int(re.search(rf"constexpr int {n} = kQuant \? (\d+)", text).group(1)) for n in ("kOtherRegs", "kSoftmaxRegs"))
    expanding = int(re.search(r"constexpr int kExpandRegs = (\d+);", text).group(1))
    assert 256 * softmax + 128 * other + 128 * expanding <= 65536 and threads == 512
