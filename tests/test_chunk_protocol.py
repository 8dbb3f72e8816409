"""CPU model of the chunk-attention kernel's barriers: loader, making, matrix and softmax warps of one CTA, which takes one
item after another, as coroutines under random interleavings, with the copies and the matrix pipe as asynchronous agents.
Checks that no barrier gets an arrival its phase does not expect, that every product reads what it should, that nothing is
overwritten while it is read (a key tile's notes among it), that all roles end, and that nothing asynchronous is left then."""
import random

import pytest

from test_prompt_protocol import Bar

MAKERS, NOTES, AHEAD = 6, 8, 4  # the last two makers take the notes too


class Cta:
    def __init__(self, items, stages, grans, rng):
        """items: (key tiles of tile 0, of tile 1, granules of the last tile) each."""
        self.items, self.S, self.G, self.rng = items, stages, grans, rng
        self.full, self.empty = [Bar(MAKERS) for _ in range(stages)], [Bar(1) for _ in range(stages)]
        self.gran_full, self.gran_empty = [Bar(1) for _ in range(grans)], [Bar(MAKERS) for _ in range(grans)]
        self.q_full, self.q_empty, self.s_full, self.o_done = ([Bar(1) for _ in range(2)] for _ in range(4))
        self.p_ready = [Bar(4) for _ in range(2)]
        self.gran, self.q = [None] * grans, [None, None]
        self.stage = [{} for _ in range(stages)]  # by making warp: what it put there
        self.notes = [{} for _ in range(NOTES)]
        self.copies, self.pipe = [], []  # in flight; the pipe runs in order
        self.sp, self.o = [None, None], [None, None]
        self.work = [None] * AHEAD
        self.item_full, self.item_empty = [Bar(1) for _ in range(AHEAD)], [Bar(8 + MAKERS + 1) for _ in range(AHEAD)]
        self.stored = [set(), set()]
        self.speed = rng.choice((0.5, 0.02)), rng.choice((0.5, 0.05))
        self.rescale = rng.choice((0.0, 0.3))

    def read_item(self, n):
        while not self.item_full[n % AHEAD].done(n // AHEAD & 1):
            yield
        return self.work[n % AHEAD]

    def grans_of(self, x, j):
        n0, n1, tail = self.items[x]
        return tail if j == max(n0, n1) - 1 else 8

    def loader(self):
        count, nq = 0, [0, 0]
        for x in range(len(self.items) + 1):
            while x >= AHEAD and not self.item_empty[x % AHEAD].done((x // AHEAD + 1) & 1):
                yield
            self.work[x % AHEAD] = x if x < len(self.items) else "end"
            yield
            self.item_full[x % AHEAD].arrive()
            if x == len(self.items):
                break
            n0, n1, _ = self.items[x]
            for j in range(max(n0, n1)):
                lanes = list(range(self.grans_of(x, j)))
                self.rng.shuffle(lanes)
                for g in lanes:
                    c = count + g
                    while c >= self.G and not self.gran_empty[c % self.G].done((c // self.G + 1) & 1):
                        yield
                    self.gran_full[c % self.G].arrive(tx=1)
                    self.gran[c % self.G] = None
                    self.copies.append((self.gran, c % self.G, (x, j, g), self.gran_full[c % self.G]))
                    yield
                count += len(lanes)
                for t in (0, 1) if j == 0 else ():
                    if not (n0, n1)[t]:
                        continue
                    while nq[t] and not self.q_empty[t].done((nq[t] - 1) & 1):
                        yield
                    self.q_full[t].arrive(tx=1)
                    self.q[t] = None
                    self.copies.append((self.q, t, x, self.q_full[t]))
                    nq[t] += 1
                    yield
        for c in range(max(0, count - self.G), count):
            while not self.gran_full[c % self.G].done((c // self.G) & 1):
                yield
        for t in (0, 1):
            while nq[t] and not self.q_full[t].done((nq[t] - 1) & 1):
                yield

    def maker(self, w):
        n, count, tiles, taken = 0, 0, 0, 0
        steps = 16 if self.S == 3 else 8
        grans = sorted({s * 8 // steps for s in range(w, steps, MAKERS)})  # that it unpacks a part of

        def wait_empty(n):
            while n >= self.S and not self.empty[n % self.S].done((n // self.S + 1) & 1):
                yield

        while True:
            x = yield from self.read_item(taken)
            yield
            assert self.work[taken % AHEAD] == x
            self.item_empty[taken % AHEAD].arrive()
            taken += 1
            if x == "end":
                return
            n0, n1, _ = self.items[x]
            for j in range(max(n0, n1)):
                have = self.grans_of(x, j)
                notes = w - (MAKERS - 2)
                mine = [g for g in sorted({*grans, *(range(4 * notes, 4 * notes + 4) if notes >= 0 else ())}) if g < have]
                for g in range(have):
                    c = count + g
                    while not self.gran_full[c % self.G].done((c // self.G) & 1):
                        yield
                for kv in "KV":
                    yield from wait_empty(n)
                    for g in mine:
                        assert self.gran[(count + g) % self.G] == (x, j, g)
                    if kv == "K" and notes >= 0:
                        self.notes[tiles % NOTES][w] = (x, j)
                    self.stage[n % self.S][w] = None
                    yield
                    self.stage[n % self.S][w] = (kv, x, j)
                    if kv == "V":
                        for g in range(have):
                            self.gran_empty[(count + g) % self.G].arrive()
                    self.full[n % self.S].arrive()
                    n += 1
                    yield
                count += have
                tiles += 1

    def mma(self):
        base, ni, nq, taken = 0, [0, 0], [0, 0], 0

        def wait_full(n):
            while not self.full[n % self.S].done((n // self.S) & 1):
                yield

        def qk(x, t, j, n, last):
            self.pipe += [("QK", t, x, j, n % self.S), ("commit", self.s_full[t])]
            if last:
                self.pipe.append(("commit", self.q_empty[t]))

        freed = [0] * self.S

        def release(n):
            freed[n % self.S] += 1
            self.pipe.append(("commit", self.empty[n % self.S]))

        while True:
            x = yield from self.read_item(taken)
            yield
            assert self.work[taken % AHEAD] == x
            self.item_empty[taken % AHEAD].arrive()
            taken += 1
            if x == "end":
                break
            n0, n1, _ = self.items[x]
            nt, n_all = (n0, n1), max(n0, n1)
            if n_all == 0:
                continue
            yield from wait_full(base)
            for t in (0, 1):
                if nt[t]:
                    while not self.q_full[t].done(nq[t] & 1):
                        yield
                    nq[t] += 1
                    qk(x, t, 0, base, nt[t] == 1)
            release(base)
            yield
            for j in range(n_all):
                nv, nk = base + 2 * j + 1, base + 2 * j + 2
                yield from wait_full(nv)
                for t in (0, 1):
                    if j >= nt[t]:
                        continue
                    while not self.p_ready[t].done(ni[t] & 1):
                        yield
                    ni[t] += 1
                    self.pipe += [("PV", t, x, j, nv % self.S), ("commit", self.o_done[t])]
                    if t:
                        release(nv)
                    yield
                    if j + 1 < nt[t]:
                        yield from wait_full(nk)
                        qk(x, t, j + 1, nk, j + 2 == nt[t])
                    yield
                if j >= n1:
                    release(nv)
                if j + 1 < n_all:
                    release(nk)
            base += 2 * n_all
        for bars, counts in ((self.empty, freed), (self.s_full, ni), (self.o_done, ni), (self.q_empty, nq)):
            for bar, k in zip(bars, counts):
                while k and not bar.done((k - 1) & 1):
                    yield

    def softmax(self, t, warp):
        ni, tiles, taken = 0, 0, 0
        while True:
            x = yield from self.read_item(taken)
            if x == "end":
                return
            item = self.items[x]
            for j in range(item[t]):
                while not self.s_full[t].done(ni & 1):
                    yield
                for _ in range(self.rng.choice((1, 1, 30))):
                    assert self.sp[t] == ("S", x, j)
                    yield
                if j and self.rng.random() < self.rescale:
                    while not self.o_done[t].done((ni - 1) & 1):
                        yield
                    assert self.o[t] == (x, j - 1)
                    yield
                self.stored[t].add((warp, x, j))
                if all((w, x, j) in self.stored[t] for w in range(4)):
                    self.sp[t] = ("P", x, j)
                for _ in range(self.rng.choice((1, 1, 60))):
                    assert all(self.notes[(tiles + j) % NOTES].get(w) == (x, j) for w in (MAKERS - 2, MAKERS - 1)), "notes gone"
                    yield
                self.p_ready[t].arrive()
                ni += 1
            tiles += max(item[:2])
            if item[t]:
                while not self.o_done[t].done((ni - 1) & 1):
                    yield
                for _ in range(self.rng.choice((1, 1, 40))):
                    assert self.o[t] == (x, item[t] - 1), "O overwritten before it was read"
                    yield
            assert self.work[taken % AHEAD] == x, "an item overwritten before all had read it"
            self.item_empty[taken % AHEAD].arrive()
            taken += 1

    def agents(self):
        if self.copies and self.rng.random() < self.speed[0]:
            where, at, content, bar = self.copies.pop(self.rng.randrange(len(self.copies)))
            where[at] = content
            bar.landed(1)
        if self.pipe and self.rng.random() < self.speed[1]:
            op = self.pipe.pop(0)
            if op[0] == "commit":
                op[1].arrive()
                return
            kind, t, x, j, st = op
            want = {w: ("K" if kind == "QK" else "V", x, j) for w in range(MAKERS)}
            assert self.stage[st] == want
            if kind == "QK":
                assert self.q[t] == x and (self.sp[t] is None or self.sp[t][0] == "P")
                self.sp[t] = ("S", x, j)
            else:
                assert self.sp[t] == ("P", x, j) and (j == 0 or self.o[t] == (x, j - 1))
                self.o[t] = (x, j)

    def run(self):
        roles = [self.loader(), self.mma()] + [self.maker(w) for w in range(MAKERS)]
        roles += [self.softmax(t, w) for t in (0, 1) for w in range(4)]
        slow = {id(x): self.rng.choice((1.0, 0.3, 0.03)) for x in roles}
        for _ in range(3000000):
            if not roles:
                break
            x = self.rng.choice(roles)
            if self.rng.random() < slow[id(x)]:
                try:
                    next(x)
                except StopIteration:
                    roles.remove(x)
            self.agents()
        assert not roles, "a role never ended"
        assert not self.copies, "a copy is in flight after the CTA's end"
        assert not self.pipe, "a product or an arrival is left after the CTA's end"


@pytest.mark.parametrize("stages,grans", [(3, 28), (8, 32)])
def test_every_interleaving_tried_is_sound(stages, grans):
    rng = random.Random(11)
    for _ in range(60):
        items = []
        for _ in range(rng.randint(1, 9)):
            n1 = rng.choice((0, 0, 1, 1, 2, 5))
            n0 = rng.randint(max(0, n1 - 2), n1) if n1 else rng.choice((0, 1, 1, 2, 4))
            items.append((n0, n1, rng.randint(1, 8)))
        Cta(items, stages, grans, rng).run()


def test_many_short_items():
    """Items of one key tile, where the warps run furthest ahead of one another."""
    rng = random.Random(12)
    for stages, grans in ((3, 28), (8, 32)):
        for _ in range(20):
            Cta([(rng.choice((0, 1)), rng.choice((0, 1)), rng.choice((1, 1, 2))) for _ in range(30)], stages, grans, rng).run()


@pytest.mark.parametrize("stages,grans", [(3, 28), (8, 32)])
def test_long_items_of_one_tile_alone(stages, grans):
    """Items that one of the two warpgroups has no part in, while it still reads the notes of its last tile."""
    rng = random.Random(13)
    for _ in range(40):
        items = []
        for _ in range(3):
            items += [rng.choice(((1, 1), (2, 2), (0, 1), (1, 0))) + (8,)]
            items += [rng.choice(((10, 0), (9, 0), (0, 12))) + (1,)] * rng.randint(1, 2)
        Cta(items, stages, grans, rng).run()
