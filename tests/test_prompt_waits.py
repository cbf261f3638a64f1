"""A model of the waits of the attention kernel for prompts, on the CPU: its warps run at any relative speed, products finish
in order but at any time, and a wait by parity passes whenever the phase before the current one has that parity.  No wait may
last for ever, none may pass before what it waits for (csrc/prompt.cu)."""
import os
import random
import re

import pytest

from conftest import ROOT


class Barrier:
    def __init__(self, count):
        self.count = self.pending = count
        self.phase = 0                                      # the one that is not complete

    def arrive(self):
        self.pending -= 1
        if self.pending == 0:
            self.phase, self.pending = self.phase + 1, self.count


def run(items, seed, no_handshake=False, idle_ahead=False, one_weight_barrier=False):
    """items: (steps, halves).  Returns None, or what went wrong."""
    rnd = random.Random(seed)
    B = {"queries": Barrier(2 + (0 if no_handshake else 2))}          # one arrival stands for the four warps of a half
    for i in (0, 1):
        for name, n in (("keys_full", 1), ("keys_free", 2), ("values_full", 1), ("values_free", 2), ("scores_done", 1),
                        ("scores_read", 1), ("weights0", 1), ("weights1", 1), ("sums0", 1), ("sums1", 1)):
            B[name, i] = Barrier(n)
    wrong, ready, done = [], {0: -1, 1: -1}, {0: 0, 1: 0}   # item whose queries are written; steps whose sums are complete
    queue = {0: [], 1: []}                                  # what a half's products do when they finish

    def wait(key, phase):
        while B[key].phase % 2 == phase % 2:
            yield
        if B[key].phase <= phase:
            wrong.append(f"{key} passed in phase {B[key].phase}, waited for {phase}")

    def sums(h, step):
        return (f"sums{step % 2}", h), step >> 1

    def weights(h, step):
        return (("weights0", h), step) if one_weight_barrier else ((f"weights{step % 2}", h), step >> 1)

    def softmax(h):
        n = item = 0
        for steps, halves in items:
            if steps == 0:
                continue
            ready[h] = item
            B["queries"].arrive()
            if h >= halves:
                if not idle_ahead:
                    yield from wait("queries", item)
                item += 1
                continue
            item += 1
            for i in range(steps):
                yield from wait(("scores_done", h), n)
                yield
                B["scores_read", h].arrive()
                if i > 0 and rnd.random() < 0.3:            # the maximum has risen
                    yield from wait(*sums(h, n - 1))
                yield
                if i > 1 and done[h] < n - 1:
                    wrong.append("weights written over those of a product that has not finished")
                B[weights(h, n)[0]].arrive()
                n += 1
            yield from wait(*sums(h, n - 1))

    def spread():
        count = 0
        for steps, _ in items:
            for _ in range((steps + 1) // 2):
                stage, use = count % 2, count >> 1
                if use > 0:
                    yield from wait(("keys_free", stage), use - 1)
                yield
                B["keys_full", stage].arrive()
                if use > 0:
                    yield from wait(("values_free", stage), use - 1)
                yield
                B["values_full", stage].arrive()
                count += 1

    def products(h):
        count = item = n = 0
        for steps, halves in items:
            if steps == 0:
                continue
            if not no_handshake:
                B["queries"].arrive()
            yield from wait("queries", item)
            if h < halves and ready[h] < item:
                wrong.append("products of queries that have not been written")
            item += 1
            if h >= halves:
                for _ in range((steps + 1) // 2):
                    for name in ("keys", "values"):
                        yield from wait((name + "_full", count % 2), count >> 1)
                        B[name + "_free", count % 2].arrive()
                    count += 1
                continue

            def keys(i):
                tile = count + i // 2
                if i % 2 == 0:
                    yield from wait(("keys_full", tile % 2), tile >> 1)
                free = [("keys_free", tile % 2)] if i % 2 or i + 1 == steps else []
                queue[h].append([("scores_done", h)] + free)

            yield from keys(0)
            for i in range(steps):
                yield from wait(("scores_read", h), n)
                if i + 1 < steps:
                    yield from keys(i + 1)
                tile = count + i // 2
                yield from wait(*weights(h, n))
                if i % 2 == 0:
                    yield from wait(("values_full", tile % 2), tile >> 1)
                free = [("values_free", tile % 2)] if i % 2 or i + 1 == steps else []
                queue[h].append([sums(h, n)[0]] + free)
                n += 1
            count += (steps + 1) // 2

    agents = [softmax(0), softmax(1), spread(), products(0), products(1)]
    speed = [rnd.choice((1, 1, 4, 20)) for _ in agents] + [rnd.choice((1, 4, 20))]
    for turn in range(60000):
        if wrong:
            return wrong[0]
        if not agents or not any(agents):
            return None
        k = rnd.choices(range(6), weights=speed)[0]
        if k == 5:
            for h in (0, 1):
                if queue[h] and rnd.random() < 0.7:
                    for key in queue[h].pop(0):
                        done[h] += key[0].startswith("sums")
                        B[key].arrive()
        elif agents[k] is not None:
            try:
                next(agents[k])
            except StopIteration:
                agents[k] = None
    return "stuck"


ITEMS = [[(1, 1)] * 6, [(1, 2), (2, 1), (3, 2), (1, 1), (4, 2)], [(7, 2), (0, 1), (5, 1), (6, 2)], [(2, 1), (1, 1), (1, 1), (9, 2)],
         [(12, 2), (3, 1)]]


@pytest.mark.parametrize("items", ITEMS)
def test_no_wait_lasts_and_none_passes_early(items):
    for seed in range(120):
        assert run(items, seed) is None, seed


def test_the_model_sees_the_mistakes():
    """One barrier for even and odd steps' weights: a wait that is two steps late meets the next phase of the same parity.  Without the
    products' part in the queries' barrier, the warp of a half without rows can be left behind by two items; a half without
    rows that does not wait for that barrier arrives for later items on it."""
    assert any(run([(12, 2)], s, one_weight_barrier=True) for s in range(60))
    assert any(run([(1, 1)] * 12, s, no_handshake=True) for s in range(400))
    assert any(run([(1, 1), (2, 1), (2, 1)], s, idle_ahead=True) for s in range(60))


def test_the_model_is_of_the_kernel():
    text = re.sub(r"//[^\n]*", "", open(os.path.join(ROOT, "paper_2407_11062_b200", "csrc", "prompt.cu")).read())
    for name, count in (("queries_full", "2 * kHalfWarps + 2"), ("keys_full[i]", "kSpreadWarps"), ("keys_free[i]", "2"), ("values_free[i]", "2"),
                        ("scores_done[i]", "1"), ("scores_read[i]", "kHalfWarps"), ("weights_full[i][0]", "kHalfWarps"), ("sums_done[i][0]", "1")):
        assert f"ptx::mbar_init(ptx::smem_addr(&ctl->{name}), {count});" in text
    assert "wait(ctl->sums_done[h][step & 1u], step >> 1)" in text and "kTile = 128, kStep = 64" in text
    assert "if (h >= job.halves) {\n        if (job.tiles > 0) wait(ctl->queries_full, items++);" in re.sub(r" +\n", "\n", text)
    steps = text[text.index("for (int i = 0; i < job.steps; ++i, ++n) {\n        const int t0"):]
    order = ["wait(ctl->scores_done[h], n)", "arrive(ctl->scores_read[h])", "wait_sums(n - 1)", "arrive(ctl->weights_full[h][n & 1u])"]
    assert [steps.index(x) for x in order] == sorted(steps.index(x) for x in order)
    products = text[text.index("multiply_keys(0);"):]
    order = ["wait(ctl->scores_read[h], n)", "multiply_keys(i + 1)", "wait(ctl->weights_full[h][n & 1u], n >> 1)", "ctl->values_full[stage], tile >> 1",
             "ctl->sums_done[h][n & 1u]"]
    assert [products.index(x) for x in order] == sorted(products.index(x) for x in order)
