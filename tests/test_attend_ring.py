"""Model of the prompt attention kernel's barriers: copies, converters, products and for each tile of rows two softmax
groups X and Y that share a maximum, all waiting by phase parity (which cannot tell a phase from the one two before it);
X and Y meet in every step and once more where the maximum grows.
Products complete in order, some time after their issue.  Random schedules check that every step uses its own scores,
weights, operand tiles and maximum, and that nobody waits for ever."""
import random

import pytest

from tests.test_linear_ring import Barrier

RAWS = 3  # as in the kernel


def simulate(rng, n, tiles, deaf=False, late=0, CONVS=3):
    """"" or what went wrong.  deaf: X does not take the maximum from Y; late: the step in which a group's wait runs out;
    CONVS: 3, or 4 as where the codes come expanded."""
    raw_full, raw_empty = [Barrier(1) for _ in range(RAWS)], [Barrier(1) for _ in range(RAWS)]
    conv_full, conv_empty = [Barrier(1) for _ in range(CONVS)], [Barrier(1) for _ in range(CONVS)]
    tab_full = [Barrier(1) for _ in range(8)]
    s_full, o_full = ([Barrier(1) for _ in range(2)] for _ in range(2))
    p_full = [Barrier(2) for _ in range(2)]
    raw, conv, tab = [None] * RAWS, [None] * CONVS, [None] * 8
    scores, weights, quits = ([[None] * 2 for _ in range(2)] for _ in range(3))
    summed, scale = [-1, -1], [[0, 0], [0, 0]]  # value products done, what each half of O is scaled by
    meetings, tops = [[], []], [[0, 0], [0, 0]]  # who has come, with what; what either wants the maximum to be
    landing, pipe, wrong, aborted = [], [], [], []

    def check(what, ok):
        if not ok:
            wrong.append(what)

    def wait(bar, parity):
        while not bar.passed(parity):
            if aborted:
                return False
            yield
        return True

    def meet(t, k, pred):  # barrier k of the tile: both wait for both; any of their predicates
        while len(meetings[t]) <= k:
            meetings[t].append([])
        here = meetings[t][k]
        here.append(pred)
        while len(here) < 2:
            yield
        return any(here)

    def copies():
        u = 0
        for i in range(n):
            tab[i % 8] = i
            tab_full[i % 8].arrive()
            for _ in range(2):
                if not (yield from wait(raw_empty[u % RAWS], (u // RAWS & 1) ^ 1)):
                    return
                landing.append(u)
                u += 1
                yield

    def converters():
        for u in range(2 * n):
            if not (yield from wait(raw_full[u % RAWS], u // RAWS & 1)):
                return
            if not (yield from wait(conv_empty[u % CONVS], (u // CONVS & 1) ^ 1)):
                return
            check("raw", raw[u % RAWS] == u)
            conv[u % CONVS] = u
            yield
            raw_empty[u % RAWS].arrive()
            conv_full[u % CONVS].arrive()
            yield

    def products():
        def have(u):
            return (yield from wait(conv_full[u % CONVS], u // CONVS & 1))

        def qk(t, j):
            pipe.append(("qk", t, j))
            pipe.append(("arrive", s_full[t]))
            if t == tiles - 1:
                pipe.append(("arrive", conv_empty[2 * j % CONVS]))
        if not (yield from have(0)):
            return
        for t in range(tiles):
            qk(t, 0)
            yield
        for j in range(n):
            if not (yield from have(2 * j + 1)):
                return
            for t in range(tiles):
                if not (yield from wait(p_full[t], j & 1)):
                    return
                pipe.append(("pv", t, j))
                if j == n - 1:
                    pipe.append(("arrive", o_full[t]))
                if t == tiles - 1:
                    pipe.append(("arrive", conv_empty[(2 * j + 1) % CONVS]))
                if j + 1 < n:
                    if t == 0 and not (yield from have(2 * j + 2)):
                        return
                    qk(t, j + 1)
                yield

    def softmax(t, y):
        m, k, ok = 0, 0, True
        for i in range(n):
            if late and (t, y, i) == (0, late & 1, late >> 1):
                aborted.append(1)
            if not (yield from wait(tab_full[i % 8], i // 8 & 1)) or aborted or not (yield from wait(s_full[t], i & 1)):
                quits[t][y] = 1
                yield from meet(t, k, True)
                ok = False
                break
            check("scores", scores[t][y] == i)
            check("table", tab[i % 8] == i)
            yield
            grow = rng.random() < 0.3
            k += 1
            if (yield from meet(t, k - 1, grow)):
                if any(quits[t]):
                    ok = False
                    break
                yield
                tops[t][y] = m + 1 if grow else m
                k += 1
                yield from meet(t, k - 1, False)
                m = tops[t][y] if deaf and not y else max(tops[t])
                check("rescaled", summed[t] == i - 1)
                scale[t][y] = m
                yield
                k += 1
                yield from meet(t, k - 1, False)
            check("table", tab[i % 8] == i)
            scores[t][y], weights[t][y] = None, (i, m)
            yield
            p_full[t].arrive()
            yield
        if ok and (yield from wait(o_full[t], 0)):
            check("result", summed[t] == n - 1)
        yield from meet(t, 3 * n + 1, False)

    roles = [copies(), converters(), products()] + [softmax(t, y) for t in range(tiles) for y in range(2)]
    for _ in range(3000 + 5000 * n):
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
                t, j = a
                u = 2 * j if what == "qk" else 2 * j + 1
                check("operand", conv[u % CONVS] == u)
                if what == "qk":
                    scores[t] = [j, j]
                else:
                    check("weights", weights[t] == [(j, scale[t][0])] * 2 and scale[t][0] == scale[t][1])
                    summed[t] = j
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
@pytest.mark.parametrize("n", [1, 2, 3, 4, 5, 8, 21, 40])
def test_every_step_uses_its_own_data(n, convs, tiles):
    rng = random.Random(n * 10 + tiles)
    for _ in range(40):
        assert simulate(rng, n, tiles, CONVS=convs) == ""


@pytest.mark.parametrize("late", [2, 3, 9, 14])
def test_a_wait_that_runs_out_leaves_nobody_waiting(late):
    rng = random.Random(late)
    for _ in range(60):
        assert simulate(rng, 9, 2, late=late) == ""


def test_a_maximum_that_is_not_passed_on_is_noticed():
    rng = random.Random(2)
    assert any(simulate(rng, 8, 2, deaf=True) == "weights" for _ in range(60))
