"""Model of the prompt attention kernel's barriers: copies, converters, products and two softmax groups, waiting by phase
parity (which cannot tell a phase from the one two before it).  Products complete in order, some time after their issue.
Random schedules check that every step uses its own scores, weights and operand tiles, and that nobody waits for ever."""
import random

import pytest

from tests.test_linear_ring import Barrier

RAWS, CONVS = 4, 3  # as in the kernel


def simulate(rng, n2, tiles, shared_p=False, last_wait_alone=False):
    n = (n2 + 1) // 2
    raw_full, raw_empty = [Barrier(1) for _ in range(RAWS)], [Barrier(1) for _ in range(RAWS)]
    conv_full, conv_empty = [Barrier(1) for _ in range(CONVS)], [Barrier(1) for _ in range(CONVS)]
    tab_full = [Barrier(1) for _ in range(8)]
    s_full = [Barrier(1) for _ in range(2)]
    p_full = [[Barrier(1) for _ in range(2)] for _ in range(2)]
    pv_done, o_full = ([Barrier(1) for _ in range(2)] for _ in range(2))
    raw, conv, tab = [None] * RAWS, [None] * CONVS, [None] * 8
    scores, weights = ([[None] * 2 for _ in range(2)] for _ in range(2))
    summed = [-1, -1]
    landing, pipe, wrong = [], [], []

    def check(what, ok):
        if not ok:
            wrong.append(what)

    def copies():
        u = 0
        for i in range(n):
            tab[i % 8] = i
            tab_full[i % 8].arrive()
            for _ in range(2):
                while not raw_empty[u % RAWS].passed((u // RAWS & 1) ^ 1):
                    yield
                landing.append(u)
                u += 1
                yield

    def converters():
        for u in range(2 * n):
            while not raw_full[u % RAWS].passed(u // RAWS & 1):
                yield
            while not conv_empty[u % CONVS].passed((u // CONVS & 1) ^ 1):
                yield
            check("raw", raw[u % RAWS] == u)
            conv[u % CONVS] = u
            yield
            raw_empty[u % RAWS].arrive()
            conv_full[u % CONVS].arrive()
            yield

    def products():
        def have(u):
            while not conv_full[u % CONVS].passed(u // CONVS & 1):
                yield

        def qk(t, j):
            pipe.append(("qk", t, 2 * j))
            pipe.append(("arrive", s_full[t]))
            if t == tiles - 1:
                pipe.append(("arrive", conv_empty[2 * j % CONVS]))
        yield from have(0)
        for t in range(tiles):
            qk(t, 0)
            yield
        for i in range(n2):
            if not i & 1:
                yield from have(i + 1)
            for t in range(tiles):
                bar, parity = (p_full[t][0], i & 1) if shared_p else (p_full[t][i & 1], i >> 1 & 1)
                while not bar.passed(parity):
                    yield
                pipe.append(("pv", t, i))
                pipe.append(("arrive", pv_done[t]))
                if i == n2 - 1:
                    pipe.append(("arrive", o_full[t]))
                if t == tiles - 1 and (i & 1 or i == n2 - 1):
                    pipe.append(("arrive", conv_empty[(2 * (i >> 1) + 1) % CONVS]))
                if i & 1 and (i >> 1) + 1 < n:
                    if t == 0:
                        yield from have(i + 1)
                    qk(t, (i >> 1) + 1)
                yield

    def softmax(t):
        for i in range(n2):
            slot = (i >> 1) % 8
            if not i & 1:
                while not tab_full[slot].passed((i >> 1) // 8 & 1):
                    yield
            while not i & 1 and not s_full[t].passed(i >> 1 & 1):
                yield
            check("scores", scores[t][i & 1] == i)
            check("table", tab[slot] == i >> 1)
            if i and rng.random() < 0.4:  # the maximum has grown
                while not pv_done[t].passed((i - 1) & 1):
                    yield
                check("rescaled", summed[t] == i - 1)
            yield
            check("table", tab[slot] == i >> 1)
            scores[t][i & 1], weights[t][i & 1] = None, i
            (p_full[t][0] if shared_p else p_full[t][i & 1]).arrive()
            yield
        while not (pv_done[t].passed((n2 - 1) & 1) if last_wait_alone else o_full[t].passed(0)):
            yield
        check("result", summed[t] == n2 - 1)

    roles = [copies(), converters(), products()] + [softmax(t) for t in range(tiles)]
    for _ in range(2000 + 1500 * n2):
        if wrong:
            return wrong[0]
        if landing and rng.random() < 0.2:
            u = landing.pop(rng.randrange(len(landing)))
            raw[u % RAWS] = u
            raw_full[u % RAWS].arrive()
        elif pipe and rng.random() < 0.3:
            what, *a = pipe.pop(0)
            if what == "arrive":
                a[0].arrive()
            else:
                t, i = a
                u = 2 * (i >> 1) + (what == "pv")
                check("operand", conv[u % CONVS] == u)
                if what == "qk":
                    scores[t] = [i, i + 1]
                else:
                    check("weights", weights[t][i & 1] == i)
                    summed[t] = i
        elif roles:
            r = rng.choice(roles)
            try:
                next(r)
            except StopIteration:
                roles.remove(r)
        elif not pipe and not landing:
            return wrong[0] if wrong else ""
    return wrong[0] if wrong else "waits for ever"


@pytest.mark.parametrize("tiles", [1, 2])
@pytest.mark.parametrize("n2", [1, 2, 3, 4, 5, 8, 21, 40])
def test_every_step_uses_its_own_data(n2, tiles):
    rng = random.Random(n2 * 10 + tiles)
    for _ in range(60):
        assert simulate(rng, n2, tiles) == ""


def test_one_barrier_for_both_steps_weights_is_not_enough():
    rng = random.Random(1)
    assert any(simulate(rng, 8, 2, shared_p=True) for _ in range(60))


def test_the_last_phase_of_every_step_s_barrier_is_not_enough_to_wait_for():
    rng = random.Random(2)
    assert any(simulate(rng, 8, 2, last_wait_alone=True) == "result" for _ in range(300))
