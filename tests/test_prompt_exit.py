"""CPU model of how a CTA of the prompt-attention kernel ends (the roles and barriers of test_prompt_protocol): when its
warps have left, no copy, product or commit of its own is on its way, whose arrival could find the shared memory in another
block's hands.  Also where a warp's wait runs out and the others' do in turn."""
import random

import pytest

from test_prompt_protocol import Cta


class GaveUp(Exception):
    pass


class Pipe(list):
    """The matrix pipe, which counts the commits to each barrier."""

    def __init__(self):
        super().__init__()
        self.commits = {}

    def append(self, op):
        if op[0] == "commit":
            self.commits[op[1]] = self.commits.get(op[1], 0) + 1
        super().append(op)

    def __iadd__(self, ops):
        for op in ops:
            self.append(op)
        return self


class Ending(Cta):
    """`waits`: the matrix warp waits for the last commit on every barrier before it leaves."""

    def __init__(self, items, stages, rng, waits=True):
        super().__init__(items, stages, rng)
        self.pipe, self.waits, self.stuck = Pipe(), waits, set()

    def mma(self):
        try:
            yield from super().mma()
        except GaveUp:
            pass
        if self.waits:
            for bar, n in self.pipe.commits.items():
                while not bar.done((n - 1) & 1):
                    yield

    def loader(self):
        try:
            yield from super().loader()
        except GaveUp:  # each copy is waited for by the barrier that counts it alone
            while self.copies:
                yield

    def until_given_up(self, role):
        try:
            yield from role
        except GaveUp:
            pass

    def roles(self):
        r = [self.loader(), self.mma()]
        others = [self.cleaner(0), self.cleaner(1)] + [self.softmax(t, w) for t in (0, 1) for w in range(4)]
        return r + [self.until_given_up(x) for x in others]

    def run_and_give_up(self, at):
        """A role's wait runs out at step `at`; the others' do some time later, one after another."""
        roles = self.roles()
        for x in list(roles):
            next(x)
        waiting, limit = list(roles), at
        for step in range(400000):
            if not roles:
                break
            if step >= limit and waiting:
                x = self.rng.choice(waiting)
                waiting.remove(x)
                limit = step + self.rng.choice((0, 50, 2000))
                if x in roles:
                    try:
                        x.throw(GaveUp())
                    except StopIteration:
                        roles.remove(x)
            else:
                x = self.rng.choice(roles)
                try:
                    next(x)
                except StopIteration:
                    roles.remove(x)
            self.agents()
        assert not roles, "a role never ended"


def left_over(cta):
    return bool(cta.copies or cta.pipe)


def some_items(rng):
    items = []
    for _ in range(rng.randint(1, 6)):
        n1 = rng.choice((0, 0, 1, 1, 2, 5))
        n0 = rng.randint(max(0, n1 - 2), n1) if n1 else rng.choice((0, 1, 1, 2, 4))
        items.append((n0, n1, max(0, max(n0, n1) - rng.randint(0, 3))))
    return items


@pytest.mark.parametrize("stages", [5, 8])
def test_nothing_is_on_its_way_when_the_warps_have_left(stages):
    rng = random.Random(11)
    for _ in range(120):
        cta = Ending(some_items(rng), stages, rng)
        cta.run()
        assert not left_over(cta)


@pytest.mark.parametrize("stages", [5, 8])
def test_without_the_last_waits_commits_are_left(stages):
    rng = random.Random(12)
    found = 0
    for _ in range(60):
        cta = Ending(some_items(rng), stages, rng, waits=False)
        cta.run()
        found += left_over(cta)
    assert found


@pytest.mark.parametrize("stages", [5, 8])
def test_waits_that_run_out_leave_nothing_either(stages):
    rng = random.Random(13)
    for _ in range(150):
        cta = Ending(some_items(rng), stages, rng)
        cta.run_and_give_up(rng.choice((0, 30, 300, 1500, 5000)))
        assert not left_over(cta)


def source():
    import os
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    with open(os.path.join(root, "paper_2609_38706_gb300", "csrc", "pk_attend_prompt.cu")) as f:
        return f.read()


def test_the_kernel_waits_for_every_barrier_that_it_commits_to():
    """The model's waits are the kernel's: each barrier that a commit names is waited for behind the matrix warp's loop."""
    import re
    text = source()
    role = text[text.index("} else if (warp == kWarpMma) {"):text.index("// V of the tiles at the causal edge")]
    committed = set(re.findall(r"mma_commit\(pk::smem_addr\(&sm\.(\w+)\[", role))
    assert committed == {"empty", "s_full", "o_done", "q_empty"}
    waited = set(re.findall(r"last_commit\(sm\.(\w+)\[", role))
    assert waited == committed
