"""Model of the prompt attention kernel's barriers: copies, converters, products and for each tile of rows two softmax
groups X and Y that share a maximum, all waiting by phase parity (which cannot tell a phase from the one two before it).
Products complete in order, some time after their issue.  Random schedules check that every step uses its own scores,
weights, operand tiles and maximum, and that nobody waits for ever."""
import random

import pytest

from tests.test_linear_ring import Barrier

RAWS = 3  # as in the kernel


def simulate(rng, n2, tiles, one_p=False, deaf=False, CONVS=3):
    """"" or what went wrong.  one_p: one barrier for X's and Y's weights; deaf: X does not wait for Y's maximum; CONVS: 3, or 4
    as where the codes come expanded."""
    n = (n2 + 1) // 2
    raw_full, raw_empty = [Barrier(1) for _ in range(RAWS)], [Barrier(1) for _ in range(RAWS)]
    conv_full, conv_empty = [Barrier(1) for _ in range(CONVS)], [Barrier(1) for _ in range(CONVS)]
    tab_full = [Barrier(1) for _ in range(8)]
    s_full, pva_done, o_full = ([Barrier(1) for _ in range(2)] for _ in range(3))
    p_full, told = ([[Barrier(1) for _ in range(2)] for _ in range(2)] for _ in range(2))
    raw, conv, tab = [None] * RAWS, [None] * CONVS, [None] * 8
    scores, weights = ([[None] * 2 for _ in range(2)] for _ in range(2))
    summed, shared, scale = [-1, -1], [0, 0], [0, 0]  # value products done, the shared maximum, what O is scaled by
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
            pipe.append(("qk", t, j))
            pipe.append(("arrive", s_full[t]))
            if t == tiles - 1:
                pipe.append(("arrive", conv_empty[2 * j % CONVS]))
        yield from have(0)
        for t in range(tiles):
            qk(t, 0)
            yield
        for j in range(n):
            yield from have(2 * j + 1)
            for t in range(tiles):
                for y in range(2 if 2 * j + 1 < n2 else 1):
                    while not p_full[t][0 if one_p else y].passed((2 * j + y if one_p else j) & 1):
                        yield
                    pipe.append(("pv", t, 2 * j + y))
                    if y == 0:
                        pipe.append(("arrive", pva_done[t]))
                if j == n - 1:
                    pipe.append(("arrive", o_full[t]))
                if t == tiles - 1:
                    pipe.append(("arrive", conv_empty[(2 * j + 1) % CONVS]))
                if j + 1 < n:
                    if t == 0:
                        yield from have(2 * j + 2)
                    qk(t, j + 1)
                yield

    def softmax(t, y):
        m = 0
        for i in range((n2 + 1 - y) // 2):
            while not tab_full[i % 8].passed(i // 8 & 1):
                yield
            while not s_full[t].passed(i & 1):
                yield
            if not y and i and not deaf:
                while not told[t][1].passed((i - 1) & 1):
                    yield
                m = shared[t]
            check("scores", scores[t][y] == i)
            check("table", tab[i % 8] == i)
            yield
            if y:
                while not told[t][0].passed(i & 1):
                    yield
                m = shared[t]
            if rng.random() < 0.4:  # the maximum has grown
                m += 1
                shared[t] = m
                if y:
                    while not pva_done[t].passed(i & 1):
                        yield
                check("rescaled", summed[t] == 2 * i + y - 1)
                scale[t] = m
            yield
            told[t][y].arrive()
            check("table", tab[i % 8] == i)
            scores[t][y], weights[t][y] = None, (i, m)
            yield
            p_full[t][0 if one_p else y].arrive()
            yield
        while not o_full[t].passed(0):
            yield
        check("result", summed[t] == n2 - 1)

    roles = [copies(), converters(), products()] + [softmax(t, y) for t in range(tiles) for y in range(2)]
    for _ in range(3000 + 2500 * n2):
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
                u = 2 * i if what == "qk" else 2 * (i >> 1) + 1
                check("operand", conv[u % CONVS] == u)
                if what == "qk":
                    scores[t] = [i, i]
                else:
                    check("weights", weights[t][i & 1] == (i >> 1, scale[t]))
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
@pytest.mark.parametrize("convs", [3, 4])
@pytest.mark.parametrize("n2", [1, 2, 3, 4, 5, 8, 21, 40])
def test_every_step_uses_its_own_data(n2, convs, tiles):
    rng = random.Random(n2 * 10 + tiles)
    for _ in range(40):
        assert simulate(rng, n2, tiles, CONVS=convs) == ""


def test_one_barrier_for_both_groups_weights_is_not_enough():
    rng = random.Random(1)
    assert any(simulate(rng, 8, 2, one_p=True) for _ in range(60))


def test_a_maximum_that_is_not_passed_on_is_noticed():
    rng = random.Random(2)
    assert any(simulate(rng, 8, 2, deaf=True) == "weights" for _ in range(60))
