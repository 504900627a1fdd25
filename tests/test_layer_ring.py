"""Model of the rings of the product of few rows: one warp of copies, two groups of converters that take blocks in turn, several operands
in tensor memory, one warp of products, all waiting on barriers by phase parity; copies land in any order.  In the form whose rows
come as fp16 (`freed_by_products`), a stage is free when its products are complete, else when it was converted."""
import os
import random

import pytest

SRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2203_12091_gb300", "csrc", "fxpq_layer_few.cuh")


class Barrier:
    def __init__(self):
        self.done = 0  # completed phases

    def arrive(self):
        self.done += 1

    def passed(self, parity):  # mbarrier.try_wait.parity
        return (self.done & 1) != parity


def turns(first, by, count, size):
    """(place, phase) of blocks first, first + by, ... as the kernel counts them."""
    at, phase = 0, 0
    out, step = [], first
    for _ in range(count):
        at += step
        if at >= size:
            at, phase = at - size, phase ^ 1
        out.append((at, phase))
        step = by
    return out


@pytest.mark.parametrize("size", [3, 4, 5, 8])
def test_turns_are_places_and_parities(size):
    for first, by in ((0, 1), (0, 2), (1, 2)):
        for n, (at, phase) in enumerate(turns(first, by, 40, size)):
            i = first + n * by
            assert (at, phase) == (i % size, i // size & 1)


def simulate(rng, stages, operands, blocks, freed_by_products, empty_first=True):
    """Runs a random schedule to its end; False if a role worked on a block that was not there."""
    raw_full, raw_empty = [Barrier() for _ in range(stages)], [Barrier() for _ in range(stages)]
    conv_full, conv_empty = [Barrier() for _ in range(operands)], [Barrier() for _ in range(operands)]
    held, formed, flying, right = [None] * stages, [None] * operands, [], [True]

    def copies():
        for i, (s, ph) in enumerate(turns(0, 1, blocks, stages)):
            while not raw_empty[s].passed(ph ^ 1):
                yield
            flying.append((i, s))
            yield

    def converters(g):
        n = (blocks - g + 1) // 2
        for i, (s, ps), (c, pc) in zip(range(g, blocks, 2), turns(g, 2, n, stages), turns(g, 2, n, operands)):
            waits = [(conv_empty[c], pc ^ 1), (raw_full[s], ps)]
            for bar, parity in waits if empty_first else waits[::-1]:
                while not bar.passed(parity):
                    yield
            right[0] &= held[s] == i
            yield
            right[0] &= held[s] == i
            formed[c] = i
            if not freed_by_products:
                raw_empty[s].arrive()
            conv_full[c].arrive()
            yield

    def products():
        for i, (s, ps), (c, pc) in zip(range(blocks), turns(0, 1, blocks, stages), turns(0, 1, blocks, operands)):
            for bar, parity in [(conv_full[c], pc)] + [(raw_full[s], ps)] * freed_by_products:
                while not bar.passed(parity):
                    yield
            right[0] &= formed[c] == i and (held[s] == i or not freed_by_products)
            yield
            right[0] &= formed[c] == i and (held[s] == i or not freed_by_products)
            conv_empty[c].arrive()
            if freed_by_products:
                raw_empty[s].arrive()

    roles = [copies(), converters(0), converters(1), products()]
    for _ in range(400 * blocks):
        if not right[0]:
            return False  # (what follows means nothing)
        if flying and rng.random() < 0.3:
            i, s = flying.pop(rng.randrange(len(flying)))  # lands
            held[s] = i
            raw_full[s].arrive()
            continue
        if not roles:
            break
        r = rng.choice(roles)
        try:
            next(r)
        except StopIteration:
            roles.remove(r)
    assert not roles, "a role waits for ever"
    return right[0]


@pytest.mark.parametrize("stages,operands", [(3, 3), (4, 3), (4, 4), (5, 3), (8, 3)])
@pytest.mark.parametrize("freed_by_products", [False, True])
def test_every_role_finds_its_block(stages, operands, freed_by_products):
    rng = random.Random(stages * 8 + operands)
    assert all(simulate(rng, stages, operands, rng.randint(1, 30), freed_by_products) for _ in range(800))


def test_more_operands_than_stages_or_the_other_order_of_waits_would_not_do():
    """What the kernel's comment rests on: with fewer stages than operands, or with the copy waited for first, a converter can read a
    stage two phases early."""
    rng = random.Random(0)
    assert not all(simulate(rng, 3, 5, 30, False) for _ in range(3000)) or not all(simulate(rng, 3, 4, 30, False, False) for _ in range(3000))


def test_the_kernel_waits_in_that_order():
    src = open(SRC).read()
    converters = src[src.index("const int grp = "):]
    assert converters.index("wait_warp(conv_empty + 8 * c.at") < converters.index("wait_warp(raw_full + 8 * s.at, s.phase")


def test_what_would_not_do():
    """Each of the comment's conditions by itself: more operands than stages fail although the waits are in order, and as many fail with the
    copy waited for first but not in order."""
    rng = random.Random(1)
    assert not all(simulate(rng, 3, 4, 30, False) for _ in range(3000))
    assert not all(simulate(rng, 3, 3, 30, False, empty_first=False) for _ in range(3000))
    assert all(simulate(rng, 3, 3, 30, False) for _ in range(3000))
