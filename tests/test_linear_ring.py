"""Model of the few-token product's rings: one warp of copies, two groups of converters that take blocks in turn, one warp
of products, all waiting on barriers by phase parity.  Copies land in any order.  A parity wait cannot tell a phase from
the one two before it, so what keeps a converter from reading a stage too early is the order of its two waits."""
import random

import pytest


class Barrier:
    def __init__(self, count):
        self.count, self.left, self.phase = count, count, 0

    def arrive(self):
        self.left -= 1
        assert self.left >= 0
        if self.left == 0:
            self.left, self.phase = self.count, self.phase + 1

    def passed(self, parity):  # mbarrier.try_wait.parity
        return (self.phase & 1) != parity


def simulate(rng, stages, blocks, empty_first):
    """Runs a random schedule to its end; False if a converter read a stage that did not hold its block."""
    raw_full, raw_empty = [Barrier(1) for _ in range(stages)], [Barrier(1) for _ in range(stages)]
    conv_full, conv_empty = [Barrier(1) for _ in range(2)], [Barrier(1) for _ in range(2)]
    held, flying, right = [None] * stages, [], [True]

    def copies():
        for i in range(blocks):
            s = i % stages
            while not raw_empty[s].passed((i // stages & 1) ^ 1):
                yield
            flying.append((i, s))
            yield

    def converters(g):
        for i in range(g, blocks, 2):
            s = i % stages
            waits = [(conv_empty[g], (i >> 1 & 1) ^ 1), (raw_full[s], i // stages & 1)]
            for bar, parity in waits if empty_first else waits[::-1]:
                while not bar.passed(parity):
                    yield
            right[0] &= held[s] == i
            yield
            raw_empty[s].arrive()
            conv_full[g].arrive()
            yield

    def products():
        for i in range(blocks):
            while not conv_full[i & 1].passed(i >> 1 & 1):
                yield
            yield
            conv_empty[i & 1].arrive()

    roles = [copies(), converters(0), converters(1), products()]
    for _ in range(200 * blocks):
        if not right[0]:
            return False  # (what follows a wrong read means nothing)
        if flying and rng.random() < 0.3:
            i, s = flying.pop(rng.randrange(len(flying)))  # lands
            held[s] = i
            raw_full[s].arrive()
            continue
        r = rng.choice(roles) if roles else None
        if r is None:
            break
        try:
            next(r)
        except StopIteration:
            roles.remove(r)
    assert not roles, "a role waits for ever"
    return right[0]


@pytest.mark.parametrize("stages", [2, 3, 4, 5])
def test_every_block_is_read_from_its_own_copy(stages):
    rng = random.Random(stages)
    assert all(simulate(rng, stages, rng.randint(1, 24), True) for _ in range(1500))


def test_the_other_order_of_waits_reads_too_early_with_an_odd_ring():
    rng = random.Random(0)
    assert not all(simulate(rng, 3, 24, False) for _ in range(1500))
    assert all(simulate(rng, 4, 24, False) for _ in range(500))


def test_the_kernel_waits_in_that_order():
    import os
    src = open(os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2203_12091_gb300", "csrc", "fxpq_linear.cu")).read()
    converters = src[src.index("const int grp = "):]
    assert converters.index("wait_warp(conv_empty + 8 * grp") < converters.index("wait_warp(raw_full + 8 * s, (i / ST)")
