"""CPU model of the prompt-attention kernel's barriers: loader, matrix, cleaning and softmax warps of one CTA, which
takes one item after another, as coroutines under random interleavings, with the copies, the answers on the next item
and the matrix pipe as asynchronous agents.  Checks that no
barrier gets an arrival its phase does not expect, that every product reads what it should, that nothing is overwritten
while it is read, that all roles end, and that nothing asynchronous is left when they have."""
import random

import pytest


class Bar:
    def __init__(self, count):
        self.count, self.pending, self.tx, self.phase = count, count, 0, 0

    def _turn(self):
        if self.pending == 0 and self.tx == 0:
            self.phase += 1
            self.pending = self.count

    def arrive(self, tx=0):
        assert self.pending > 0, "arrival outside the phase"
        self.tx += tx
        self.pending -= 1
        self._turn()

    def landed(self, n):
        self.tx -= n
        assert self.tx >= 0
        self._turn()

    def done(self, parity):  # what a try answers: the phase of this parity is not the current one
        return self.phase % 2 != parity


class Cta:
    def __init__(self, items, stages, rng):
        """items: (key tiles of tile 0, of tile 1, first edge tile) each."""
        self.items, self.S, self.rng = items, stages, rng
        self.full = [Bar(2) for _ in range(stages)]
        self.empty = [Bar(1) for _ in range(stages)]
        self.q_full, self.q_empty, self.s_full, self.o_done = ([Bar(1) for _ in range(2)] for _ in range(4))
        self.p_ready, self.edge_v = [Bar(4) for _ in range(2)], [Bar(1) for _ in range(4)]
        self.stage, self.q = [None] * stages, [None, None]
        self.copies, self.pipe = [], []   # in flight; the pipe runs in order
        self.sp, self.o = [None, None], [None, None]
        self.work = [None] * 8
        self.epilogues, self.notes = [0] * 8, [None, None]
        self.stored = [set(), set()]
        self.speed = rng.choice((0.5, 0.02)), rng.choice((0.5, 0.05))
        self.next, self.given = [None] * 4, 1  # answers; items given out
        self.next_full, self.next_empty = [Bar(1) for _ in range(4)], [Bar(10) for _ in range(4)]
        self.rescale = rng.choice((0.0, 0.3))

    def ask(self, turn):
        while turn >= 4 and not self.next_empty[turn & 3].done((turn // 4 + 1) & 1):
            yield
        self.next_full[turn & 3].arrive(tx=1)
        self.next[turn & 3] = None
        self.copies.append((self.next, turn & 3, "next", self.next_full[turn & 3]))

    def read(self, turn, reader=True):
        while not self.next_full[turn & 3].done(turn >> 2 & 1):
            yield
        x = self.next[turn & 3]
        assert x is not None
        yield
        if reader:
            self.next_empty[turn & 3].arrive()
        return x

    def walk(self):
        """The items that a cleaning or softmax warp goes through, read as the kernel does; None: not there yet."""
        turn, x = 0, 0
        while x != "end":
            yield x
            step = self.read(turn)
            while True:
                try:
                    next(step)
                except StopIteration as e:
                    x = e.value
                    break
                yield None
            turn += 1

    def loader(self):
        n, edges, nq, sent, x, turn = 0, 0, [0, 0], 0, 0, 0
        while x != "end":
            n0, n1, fe = self.items[x]
            if max(n0, n1) <= 3:
                yield from self.ask(turn)
            if max(n0, n1):
                assert self.work[sent & 7] is None, "an item's note overwritten before it was read"
                self.work[sent & 7] = x
                sent += 1
            for j in range(max(n0, n1)):
                for kv in (0, 1):
                    st = n % self.S
                    dirty = kv and j >= fe
                    bar = self.edge_v[edges & 3] if dirty else self.full[st]
                    while n >= self.S and not self.empty[st].done((n // self.S + 1) & 1):
                        yield
                    if not dirty:
                        bar.arrive()
                    yield
                    bar.arrive(tx=1)
                    self.stage[st] = None
                    self.copies.append((self.stage, st, ("KV"[kv], x, j, not dirty), bar))
                    n, edges = n + 1, edges + dirty
                    yield
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
                if max(n0, n1) > 3 and j == max(n0, n1) - 3:
                    yield from self.ask(turn)
            x = yield from self.read(turn, False)
            turn += 1
        st = n % self.S
        while n >= self.S and not self.empty[st].done((n // self.S + 1) & 1):
            yield
        self.work[sent & 7] = "end"
        for _ in range(2):
            self.full[st].arrive()
            yield
        n += 1
        for i in range(max(0, n - self.S), n):
            while not self.full[i % self.S].done((i // self.S) & 1):
                yield
        for t in (0, 1):
            while nq[t] and not self.q_full[t].done((nq[t] - 1) & 1):
                yield

    def mma(self):
        base, ni, nq = 0, [0, 0], [0, 0]

        def wait_full(n):
            while not self.full[n % self.S].done((n // self.S) & 1):
                yield

        def qk(x, t, j, n, last):
            self.pipe += [("QK", t, x, j, n % self.S), ("commit", self.s_full[t])]
            if last:
                self.pipe.append(("commit", self.q_empty[t]))

        taken = 0
        while True:
            yield from wait_full(base)
            x = self.work[taken & 7]
            self.work[taken & 7] = None
            taken += 1
            if x == "end":
                return
            n0, n1, _ = self.items[x]
            nt, n_all = (n0, n1), max(n0, n1)
            for t in (0, 1):
                if nt[t]:
                    while not self.q_full[t].done(nq[t] & 1):
                        yield
                    nq[t] += 1
                    qk(x, t, 0, base, nt[t] == 1)
            self.pipe.append(("commit", self.empty[base % self.S]))
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
                        self.pipe.append(("commit", self.empty[nv % self.S]))
                    yield
                    if j + 1 < nt[t]:
                        yield from wait_full(nk)
                        qk(x, t, j + 1, nk, j + 2 == nt[t])
                    yield
                if j >= n1:
                    self.pipe.append(("commit", self.empty[nv % self.S]))
                if j + 1 < n_all:
                    self.pipe.append(("commit", self.empty[nk % self.S]))
            base += 2 * n_all

    def cleaner(self, half):
        base, edges = 0, 0
        for x in self.walk():
            if x is None:
                yield
                continue
            n0, n1, fe = self.items[x]
            n_all = max(n0, n1)
            if fe < n_all:
                while x >= 2 and min(self.epilogues) < x - 1:
                    yield
                self.notes[x & 1] = x
                yield
            for j in range(fe, n_all):
                st = (base + 2 * j + 1) % self.S
                while not self.edge_v[edges & 3].done((edges >> 2) & 1):
                    yield
                edges += 1
                yield
                assert self.stage[st] and self.stage[st][:3] == ("V", x, j)
                self.stage[st] = ("V", x, j, self.stage[st][3] + 1 if self.stage[st][3] else 1)
                yield
                self.full[st].arrive()
            base += 2 * n_all

    def softmax(self, t, warp):
        ni = 0
        turn, x = 0, 0
        while x != "end":
            item = self.items[x]
            fe = item[2]
            for j in range(item[t]):
                while not self.s_full[t].done(ni & 1):
                    yield
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
                self.p_ready[t].arrive()
                ni += 1
            here, x = x, (yield from self.read(turn))
            turn += 1
            if item[t]:
                while not self.o_done[t].done((ni - 1) & 1):
                    yield
                for _ in range(self.rng.choice((1, 1, 40))):
                    assert self.o[t] == (here, item[t] - 1), "O overwritten before it was read"
                    assert fe >= item[t] or self.notes[here & 1] == here
                    yield
            self.epilogues[4 * t + warp] = here + 1

    def agents(self):
        if self.copies and self.rng.random() < self.speed[0]:
            where, at, content, bar = self.copies.pop(self.rng.randrange(len(self.copies)))
            if content == "next":
                content, self.given = (self.given if self.given < len(self.items) else "end"), self.given + 1
            where[at] = content
            bar.landed(1)
        if self.pipe and self.rng.random() < self.speed[1]:
            op = self.pipe.pop(0)
            if op[0] == "commit":
                op[1].arrive()
                return
            kind, t, x, j, st = op
            if kind == "QK":
                assert self.stage[st] == ("K", x, j, True) and self.q[t] == x
                assert self.sp[t] is None or self.sp[t][0] == "P"
                self.sp[t] = ("S", x, j)
            else:
                v = self.stage[st]
                assert v and v[:3] == ("V", x, j) and v[3] == (2 if j >= self.items[x][2] else True)
                assert self.sp[t] == ("P", x, j) and (j == 0 or self.o[t] == (x, j - 1))
                self.o[t] = (x, j)

    def run(self):
        roles = [self.loader(), self.mma(), self.cleaner(0), self.cleaner(1)]
        roles += [self.softmax(t, w) for t in (0, 1) for w in range(4)]
        slow = {id(x): self.rng.choice((1.0, 0.3, 0.03)) for x in roles}
        for _ in range(2000000):
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
        assert all(op[0] == "commit" for op in self.pipe), "a product runs after the CTA's end"


@pytest.mark.parametrize("stages", [5, 8])
def test_every_interleaving_tried_is_sound(stages):
    rng = random.Random(7)
    for _ in range(150):
        items = []
        for _ in range(rng.randint(1, 7)):
            n1 = rng.choice((0, 0, 1, 1, 2, 5))
            n0 = rng.randint(max(0, n1 - 2), n1) if n1 else rng.choice((0, 1, 1, 2, 4))
            items.append((n0, n1, max(0, max(n0, n1) - rng.randint(0, 3))))
        Cta(items, stages, rng).run()
