"""The prompt attention's warp roles (csrc/attention_tile.cu) as a model on the host: barriers with phases, copies and products
that land later or never, warps that run in any order.  The model checks, at every access, that what is read has landed and what is
written over has been used, that a CTA ends with no copy in flight, and that it ends at all when a copy never lands.  Each design that was found unsound is a variant of the
model that has to fail, which shows that the model would see it."""
import os
import random
import re

import pytest

SOURCE = open(os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2109_09868_b200", "csrc", "attention_tile.cu")).read()


def constant(name):
    return int(re.search(r"\b%s = (\d+)\b" % name, SOURCE).group(1))


STAGES, CLEANS, MASKS = constant("kStages"), constant("kCleans"), constant("kMasks")
FULLS = int(re.search(r"\bkFulls = (\d+) \* kStages\b", SOURCE).group(1)) * STAGES


class Unsound(Exception):
    pass


def need(ok, what):
    if not ok:
        raise Unsound(what)


class Bar:
    """A barrier that counts arrivals and bytes; a wait names the parity of the phase that has to be over."""

    def __init__(self, count):
        self.count, self.left, self.bytes, self.phase = count, count, 0, 0

    def _step(self):
        if self.left == 0 and self.bytes == 0:
            self.phase, self.left = self.phase + 1, self.count

    def arrive(self, expect=0):
        self.bytes += expect
        self.left -= 1
        need(self.left >= 0, "more arrivals than a phase takes")
        self._step()

    def land(self, count):
        self.bytes -= count
        self._step()

    def over(self, parity):
        return self.phase & 1 != parity


class Meeting:
    """Warps that meet, with an or over what they bring."""

    def __init__(self, count):
        self.count, self.here, self.any, self.turn, self.said = count, 0, False, 0, {}

    def come(self, want=False):
        turn = self.turn
        self.here, self.any = self.here + 1, self.any or want
        if self.here == self.count:
            self.said[turn] = self.any
            self.here, self.any, self.turn = 0, False, turn + 1
        return turn


class Cta:
    """One CTA of `tiles` query tiles that take part in `steps` of the key tiles; the two warps of one quarter of the rows stand
    for all softmax warps of a tile."""

    def __init__(self, rng, steps, queries="steps", rows=None, cluster=False, fulls=FULLS, lost=None, softmax="keeps meetings"):
        self.rng, self.steps_of, self.TQ, self.cluster = rng, steps, len(steps), cluster
        self.steps = max(steps)
        self.rows = rows or [True] * self.TQ  # tiles that have rows at all
        self.queries, self.softmax = queries, softmax
        self.lost = lost         # the copy that never lands: an entry of the ring, or "queries"
        self.gave_up = False     # a wait has run out: the CTA's flag; from then on nothing that is read or written counts
        self.full, self.empty = [Bar(1) for _ in range(fulls)], [Bar(1) for _ in range(STAGES)]
        self.clean, self.q_full, self.s_free = [Bar(1) for _ in range(CLEANS)], Bar(1), Bar(2)
        self.s_ready = [Bar(1) for _ in steps]
        self.p_ready = [[Bar(1), Bar(1)] for _ in steps]
        self.pv_done = [Bar(1) for _ in steps]
        self.meet, self.all_meet = [Meeting(2) for _ in steps], Meeting(2 * self.TQ)
        self.place = [None] * STAGES       # (entry, landed)
        self.used = set()                  # entries that all their products, and the look through them, are done with
        self.q = [None] * self.TQ          # None, "flying", "here"
        self.flying = []                   # copies: (barrier, landing)
        self.queues = {"score": [], "out": []}
        self.s, self.p, self.o = [None] * self.TQ, [[None, None] for _ in steps], [-1] * self.TQ
        self.read = [[-1, -1] for _ in steps]
        self.cleaned, self.masks = set(), {}

    # entry i = 2 j (keys of tile j) or 2 j + 1 (values)
    def full_of(self, i):
        if len(self.full) == STAGES:  # one barrier to a place
            return self.full[i % STAGES], (i // STAGES) & 1
        return self.full[i % STAGES + (i & 1) * STAGES], (i // STAGES >> 1) & 1

    def need(self, ok, what):
        need(ok or self.gave_up, what)

    def here(self, i):
        return self.place[i % STAGES] == (i, True)

    def copy_in(self, i):
        at, bar = i % STAGES, self.full_of(i)[0]
        if self.place[at] is not None:
            self.need(self.place[at][1] and self.place[at][0] in self.used, "entry %d is copied over what is still needed" % i)
        self.place[at] = (i, False)

        def landed():
            self.place[at] = (i, True)
            bar.land(1)

        bar.arrive(expect=1)
        if i != self.lost:
            self.flying.append(landed)

    # ---- roles: what they yield they wait for ----
    def copies(self):
        if self.queries == "steps":
            asked = [t for t in range(self.TQ) if self.steps_of[t] > 0]
        else:  # every tile with rows
            asked = [t for t in range(self.TQ) if self.rows[t]]
        if asked:
            self.q_full.arrive(expect=len(asked))
        for t in asked:
            self.q[t] = "flying"

            def landed(t=t):
                self.q[t] = "here"
                self.q_full.land(1)

            if self.lost != "queries":
                self.flying.append(landed)
            yield
        for i in range(2 * self.steps):
            if i >= STAGES:
                if not (yield self.empty[i % STAGES], (i // STAGES - 1) & 1):
                    return
            if i % 2 == 0:
                self.masks[i // 2 % MASKS] = i // 2
            self.copy_in(i)
            yield

    def scores(self, t, j):  # the product S, when it runs
        def run():
            self.need(self.q[t] == "here", "S of queries that have not landed")
            self.need(self.here(2 * j), "S of keys that have not landed")
            self.need(j == 0 or min(self.read[t]) == j - 1, "S over scores that have not been read")
            if self.TQ == 2:
                self.need(j == 0 or self.o[t] == j - 1, "S over weights that have not been used")
            self.s[t] = j

        return run

    def values(self, t, j, half):
        def run():
            self.need(self.here(2 * j + 1), "O of values that have not landed")
            self.need(j in self.cleaned, "O of values that have not been looked through")
            self.need(self.p[t][half] == j, "O of other weights")
            if half == 1:
                self.o[t] = j

        return run

    def give_back(self, i):
        def run():
            self.used.add(i)
            self.empty[i % STAGES].arrive()

        return run

    def score_warp(self):
        if self.TQ != 1 or self.steps == 0:
            return
        if not (yield self.q_full, 0):
            return
        for j in range(self.steps):
            if not (yield self.full_of(2 * j)):
                return
            if j > 0 and not (yield self.s_free, (j - 1) & 1):
                return
            self.queues["score"] += [self.scores(0, j), self.s_ready[0].arrive, self.give_back(2 * j)]

    def out_warp(self):
        items, queue = sum(self.steps_of), self.queues["out"]
        if items == 0:
            return
        keys_in = 1
        if self.TQ == 2:
            if not (yield self.q_full, 0) or not (yield self.full_of(0)):
                return
            for t in range(2):
                if self.steps_of[t] > 0:
                    queue += [self.scores(t, 0), self.s_ready[t].arrive]
            queue.append(self.give_back(0))
        both = min(self.steps_of) if self.TQ == 2 else 0
        for n in range(items):
            if self.TQ == 1:
                t, j, first, last = 0, n, True, True
            elif n < 2 * both:
                t, j, first, last = n & 1, n >> 1, n & 1 == 0, n & 1 == 1
            else:
                t, j, first, last = (1 if self.steps_of[1] > 0 else 0), n - both, True, True
            more = j + 1 < self.steps_of[t]
            if first:
                if not (yield self.clean[j % CLEANS], (j // CLEANS) & 1):
                    return
            if self.TQ == 2 and more and keys_in == j + 1:
                if not (yield self.full_of(2 * j + 2)):
                    return
                keys_in += 1
            for half in range(2):
                if not (yield self.p_ready[t][half], j & 1):
                    return
                queue.append(self.values(t, j, half))
            if self.TQ == 1 or not more:
                queue.append(self.pv_done[t].arrive)
            if last:
                queue.append(self.give_back(2 * j + 1))
            if self.TQ == 2 and more:
                queue += [self.scores(t, j + 1), self.s_ready[t].arrive]
                if t == 1 or j + 1 >= self.steps_of[1]:
                    queue.append(self.give_back(2 * j + 2))

    def clean_warp(self):
        for j in range(self.steps):
            if not (yield self.full_of(2 * j + 1)):
                return
            self.need(self.here(2 * j + 1), "values are looked through before they have landed")
            yield
            self.need(self.here(2 * j + 1), "values are looked through before they have landed")
            self.cleaned.add(j)
            self.clean[j % CLEANS].arrive()

    def softmax_warp(self, t, half):
        def together(want=False):
            return self.meet[t].come(want), self.meet[t]

        ok, left = True, 0  # left: steps that a wait which gave up leaves out
        for j in range(self.steps_of[t]):
            left = self.steps_of[t] - j
            ok = yield self.s_ready[t], j & 1
            if not ok:
                break
            self.need(self.s[t] == j, "scores are read before they are there")
            self.need(self.masks.get(j % MASKS) == j, "the pages of another tile of keys")
            self.read[t][half] = j
            if self.TQ == 1:
                self.s_free.arrive()
                if j > 0:
                    ok = yield self.pv_done[0], (j - 1) & 1
                    if not ok:
                        break
            turn, meeting = together(self.rng.random() < 0.3)
            yield meeting, turn
            if meeting.said[turn]:
                for _ in range(2):
                    yield tuple(reversed(together()))
                self.need(self.o[t] == j - 1, "O is scaled while products are added to it")
                yield tuple(reversed(together()))
            self.need(self.o[t] == j - 1, "weights are written over those in use")
            if self.TQ == 2:
                self.need(min(self.read[t]) == j, "weights are written over scores that have not been read")
            self.p[t][half] = j
            self.p_ready[t][half].arrive()
        for _ in range(0 if ok or self.softmax == "leaves" else left):
            turn, meeting = together()
            yield meeting, turn
            for _ in range(3 if meeting.said[turn] else 0):
                yield tuple(reversed(together()))
        if self.steps_of[t] > 0 and (ok or self.softmax != "leaves"):
            for _ in range(2):
                yield tuple(reversed(together()))
            if ok:
                ok = yield self.pv_done[t], (self.steps_of[t] - 1) & 1 if self.TQ == 1 else 0
            self.need(self.o[t] == self.steps_of[t] - 1, "O is read before it is whole")
        if self.cluster:
            turn = self.all_meet.come()
            yield self.all_meet, turn
        for u in range(self.TQ) if self.cluster else [t]:  # the output is staged where the queries were (a cluster: over all)
            self.need(self.q[u] != "flying", "the output is staged where queries still land")

    def run(self, order):
        roles = [self.copies(), self.score_warp(), self.out_warp(), self.clean_warp()] + [self.softmax_warp(t, h) for t in range(self.TQ) for h in range(2)]
        waits = {r: None for r in roles}

        def ready(w):
            return w is None or (w[0].over(w[1]) if isinstance(w[0], Bar) else w[1] in w[0].said)

        def step(r, ok):
            try:
                waits[r] = next(r) if waits[r] is None else r.send(ok)
            except StopIteration:
                del waits[r]

        while waits:
            can = [("role", r) for r, w in waits.items() if ready(w)]
            can += [("queue", q) for q in self.queues.values() if q]
            can += [("land", n) for n in range(len(self.flying) if order == "any" else min(1, len(self.flying)))]
            late = [r for r, w in waits.items() if w is not None and isinstance(w[0], Bar) and not ready(w)]
            # a wait runs out: where nothing else happens, now and then before; once one has, the others may soon
            if late and (not can or self.rng.random() < (0.2 if self.gave_up else 0.01 if self.lost is not None else 0)):
                self.gave_up = True
                step(late[self.rng.randrange(len(late))], False)
                continue
            need(can, "everything waits")
            # copies are slow or fast against the rest, by the draw
            kind, x = can[self.rng.randrange(len(can))] if self.rng.random() < 0.7 else can[0]
            if kind == "role":
                step(x, True)
            elif kind == "queue":
                x.pop(0)()
            else:
                self.flying.pop(x)()
        self.need(not self.flying, "the CTA ends with a copy in flight")


JOBS = [([n], [True]) for n in (0, 1, 2, 3, 5, 8, 13)] + [
    ([0, 0], [True, True]), ([0, 0], [True, False]), ([0, 1], [True, True]), ([0, 7], [True, True]), ([1, 1], [True, True]), ([2, 3], [True, True]),
    ([5, 5], [True, True]), ([4, 9], [True, True]), ([9, 0], [True, False]), ([12, 12], [True, True])]


def trial(steps, rows, cluster, order, seed, **variant):
    Cta(random.Random(seed), steps, rows=rows, cluster=cluster, **variant).run(order)


@pytest.mark.parametrize("cluster", [False, True])
@pytest.mark.parametrize("steps,rows", JOBS)
def test_every_access_waits_for_what_it_needs(steps, rows, cluster):
    for seed in range(60):
        trial(steps, rows, cluster, "in turn", seed)
        trial(steps, rows, cluster, "any", seed)


@pytest.mark.parametrize("steps,rows", JOBS)
def test_a_copy_that_never_lands_ends_the_kernel(steps, rows):
    for seed in range(60):
        lost = random.Random(seed).choice(["queries"] + list(range(2 * max(steps))))
        for cluster in (False, True):
            trial(steps, rows, cluster, "any", seed, lost=lost)


def finds(what, **variant):
    """The model finds fault with a variant, in some job and order."""
    for steps, rows in JOBS:
        for seed in range(60):
            try:
                trial(steps, rows, False, variant.get("order", "in turn"), seed, **{k: v for k, v in variant.items() if k != "order"})
            except Unsound as e:
                if what in str(e):
                    return True
    return False


def test_queries_of_tiles_without_steps_must_not_be_asked_for():
    assert finds("the output is staged where queries still land", queries="rows")
    assert finds("the CTA ends with a copy in flight", queries="rows")
    # the copies' byte count and their loop go by the tiles' steps
    assert "((job.steps0 > 0) + (job.steps1 > 0)) * (DP / 64) * g.group * job.tokens * 128" in SOURCE
    assert "job.steps_of(t) > 0; ++c)" in SOURCE


def test_keys_and_values_must_not_land_on_one_barrier():
    # (the copies of one CTA may land in any order)
    assert finds("values are looked through before they have landed", fulls=STAGES, order="any")
    assert "full + 8 * (i % kStages + (i & 1) * kStages)" in SOURCE and "(i / kStages >> 1) & 1" in SOURCE
    assert SOURCE.count("landed(i), landed_parity(i)") == 2 and "full + 8 * s," not in SOURCE.replace("bar_init(full + 8 * s, 1)", "")


def test_a_softmax_warp_must_not_leave_the_warp_it_meets():
    assert finds("everything waits", softmax="leaves", lost=4, order="any")
    softmax = SOURCE[SOURCE.index("---- softmax and output"): SOURCE.index("---- copies ----")]
    assert softmax.count("break;") == 2 and "if (any_of_both(meet, false)) warps_meet(meet), warps_meet(meet), warps_meet(meet);" in softmax
