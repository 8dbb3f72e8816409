"""CPU model of the prompt-attention kernel's barriers: loader, matrix, cleaning and softmax warps of one CTA as
coroutines under random interleavings, with the copies and the matrix pipe as asynchronous agents.  Checks that no
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
    def __init__(self, n_tiles, first_edge, stages, rng, rescale):
        self.nt, self.n_all, self.fe, self.S, self.rng = n_tiles, max(n_tiles), first_edge, stages, rng
        self.full = [Bar(2) for _ in range(stages)]
        self.empty = [Bar(1) for _ in range(stages)]
        self.s_full, self.p_ready, self.o_done = ([Bar(c) for _ in range(2)] for c in (1, 4, 1))
        self.q_ready, self.edge_v = Bar(8), [Bar(1) for _ in range(4)]
        self.stage = [None] * stages      # content: ("K"|"V", j, clean)
        self.copies, self.pipe = [], []   # in flight; the pipe runs in order
        self.sp = [None, None]            # S / P columns of a tile: ("S", j) or ("P", j)
        self.o = [-1, -1]                 # last PV accumulated
        self.rescale = rescale
        self.speed = rng.choice((0.5, 0.02)), rng.choice((0.5, 0.05))

    def loader(self):
        n = 0
        for j in range(self.n_all):
            for kv in (0, 1):
                st = n % self.S
                dirty = kv and j >= self.fe
                bar = self.edge_v[j - self.fe] if dirty else self.full[st]
                if n >= self.S:
                    while not self.empty[st].done((n // self.S + 1) & 1):
                        yield
                yield
                if not dirty:
                    bar.arrive()
                yield
                bar.arrive(tx=1)
                self.stage[st] = None
                self.copies.append((st, ("KV"[kv], j, not dirty), bar))
                n += 1
        for i in range(max(0, n - self.S), n):
            while not self.full[i % self.S].done((i // self.S) & 1):
                yield

    def mma(self):
        def wait_full(n):
            while not self.full[n % self.S].done((n // self.S) & 1):
                yield
        if not self.n_all:
            return
        while not self.q_ready.done(0):
            yield
        yield from wait_full(0)
        for t in (0, 1):
            if self.nt[t]:
                self.pipe += [("QK", t, 0, 0), ("commit", self.s_full[t])]
        self.pipe.append(("commit", self.empty[0]))
        for j in range(self.n_all):
            nv, nk = 2 * j + 1, 2 * j + 2
            yield from wait_full(nv)
            for t in (0, 1):
                if j >= self.nt[t]:
                    continue
                while not self.p_ready[t].done(j & 1):
                    yield
                self.pipe += [("PV", t, j, nv % self.S), ("commit", self.o_done[t])]
                yield
                if j + 1 < self.nt[t]:
                    yield from wait_full(nk)
                    self.pipe += [("QK", t, j + 1, nk % self.S), ("commit", self.s_full[t])]
                yield
            self.pipe.append(("commit", self.empty[nv % self.S]))
            if j + 1 < self.n_all:
                self.pipe.append(("commit", self.empty[nk % self.S]))

    def cleaner(self):
        for j in range(self.fe, self.n_all):
            st = (2 * j + 1) % self.S
            while not self.edge_v[j - self.fe].done(0):
                yield
            yield
            assert self.stage[st] and self.stage[st][:2] == ("V", j)
            self.stage[st] = ("V", j, True)
            yield
            self.full[st].arrive()

    def softmax(self, t, warp, shared):
        self.q_ready.arrive()
        for j in range(self.nt[t]):
            while not self.s_full[t].done(j & 1):
                yield
            assert self.sp[t] == ("S", j)
            yield
            if j and self.rescale(t, j):
                while not self.o_done[t].done((j - 1) & 1):
                    yield
                assert self.o[t] == j - 1
                yield
            shared[t].add((warp, j))
            if len([1 for w, i in shared[t] if i == j]) == 4:
                self.sp[t] = ("P", j)
            self.p_ready[t].arrive()
        if self.nt[t]:
            while not self.o_done[t].done((self.nt[t] - 1) & 1):
                yield
            assert self.o[t] == self.nt[t] - 1

    def agents(self):
        if self.copies and self.rng.random() < self.speed[0]:
            st, content, bar = self.copies.pop(self.rng.randrange(len(self.copies)))
            self.stage[st] = content
            bar.landed(1)
        if self.pipe and self.rng.random() < self.speed[1]:
            op = self.pipe.pop(0)
            if op[0] == "commit":
                op[1].arrive()
            elif op[0] == "QK":
                assert self.stage[op[3]] == ("K", op[2], True)
                assert self.sp[op[1]] == (None if op[2] == 0 else ("P", op[2] - 1))
                self.sp[op[1]] = ("S", op[2])
            else:
                assert self.stage[op[3]] == ("V", op[2], True)
                assert self.sp[op[1]] == ("P", op[2]) and self.o[op[1]] == op[2] - 1
                self.o[op[1]] = op[2]

    def run(self):
        shared = [set(), set()]
        roles = [self.loader(), self.mma(), self.cleaner(), self.cleaner()]
        roles += [self.softmax(t, w, shared) for t in (0, 1) for w in range(4)]
        slow = {id(x): self.rng.choice((1.0, 0.3, 0.03)) for x in roles}
        for _ in range(200000):
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


@pytest.mark.parametrize("stages", [4, 8])
def test_every_interleaving_tried_is_sound(stages):
    rng = random.Random(7)
    for _ in range(400):
        n1 = rng.randint(0, 9)
        n0 = rng.randint(max(0, n1 - 2), n1) if n1 else rng.randint(0, 9)
        fe = max(0, max(n0, n1) - rng.randint(0, 3))
        Cta((n0, n1), fe, stages, rng, lambda t, j: rng.random() < 0.3).run()
