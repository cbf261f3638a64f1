"""What the attention kernel for prompts says of its tiles in shared memory (tokens whose keys were scaled, values that bf16 cannot
hold) is written by the spreading warps into one of eight places in turn and read by the softmax warps, which wait for the products
of the tile and for nothing else.  A model of the waits of csrc/prompt.cu with both halves, at any relative speed of the warps: a
table is there when it is read, and still that of its tile."""
import random

import pytest


class Barrier:
    def __init__(self, count):
        self.count = self.pending = count
        self.phase = 0

    def arrive(self):
        self.pending -= 1
        if self.pending == 0:
            self.phase, self.pending = self.phase + 1, self.count


def run(items, seed, places=8):
    """items: steps of each item, of both halves.  Returns None, or what went wrong."""
    rnd, wrong, table, queue = random.Random(seed), [], {}, {0: [], 1: []}
    B = {(name, i): Barrier(n) for i in (0, 1) for name, n in (
        ("scores_done", 1), ("scores_read", 1), ("weights0", 1), ("weights1", 1), ("sums0", 1), ("sums1", 1), ("keys_full", 1),
        ("keys_free", 2), ("values_full", 1), ("values_free", 2))}
    B["queries"] = Barrier(4)

    def wait(key, phase):
        while B[key].phase % 2 == phase % 2:
            yield

    def read(kind, tile):
        if table.get((kind, tile % places)) != tile:
            wrong.append(f"{kind} of tile {tile}: the place holds {table.get((kind, tile % places))}")

    def softmax(h):
        n = tile0 = 0
        for steps in items:
            B["queries"].arrive()
            for i in range(steps):
                yield from wait(("scores_done", h), n)
                if rnd.random() < 0.5:
                    B["scores_read", h].arrive()
                    yield
                    read("keys", tile0 + i // 2)                # keys' scales may be read after the next scores are let in
                else:
                    read("keys", tile0 + i // 2)
                    B["scores_read", h].arrive()
                yield
                if i > 1 and i % 2 == 0:
                    read("values", tile0 + i // 2 - 1)
                B[f"weights{n % 2}", h].arrive()
                n += 1
            yield from wait((f"sums{(n - 1) % 2}", h), (n - 1) >> 1)
            tiles = (steps + 1) // 2
            for tile in range(max(0, tiles - 2), tiles):
                yield
                read("values", tile0 + tile)
            tile0 += tiles

    def spread():
        count = 0
        for steps in items:
            for _ in range((steps + 1) // 2):
                for name in ("keys", "values"):
                    if count >> 1 > 0:
                        yield from wait((name + "_free", count % 2), (count >> 1) - 1)
                    table[name, count % places] = count
                    yield
                    B[name + "_full", count % 2].arrive()
                count += 1

    def products(h):
        count = n = 0
        for item, steps in enumerate(items):
            B["queries"].arrive()
            yield from wait("queries", item)

            def keys(i):
                tile = count + i // 2
                if i % 2 == 0:
                    yield from wait(("keys_full", tile % 2), tile >> 1)
                queue[h].append([("scores_done", h)] + ([("keys_free", tile % 2)] if i % 2 or i + 1 == steps else []))

            yield from keys(0)
            for i in range(steps):
                yield from wait(("scores_read", h), n)
                if i + 1 < steps:
                    yield from keys(i + 1)
                tile = count + i // 2
                yield from wait((f"weights{n % 2}", h), n >> 1)
                if i % 2 == 0:
                    yield from wait(("values_full", tile % 2), tile >> 1)
                queue[h].append([(f"sums{n % 2}", h)] + ([("values_free", tile % 2)] if i % 2 or i + 1 == steps else []))
                n += 1
            count += (steps + 1) // 2

    agents = [softmax(0), softmax(1), spread(), products(0), products(1)]
    speed = [rnd.choice((1, 1, 4, 20)) for _ in range(6)]
    for _ in range(60000):
        if wrong:
            return wrong[0]
        if not any(agents):
            return None
        k = rnd.choices(range(6), weights=speed)[0]
        if k == 5:
            for h in (0, 1):
                if queue[h] and rnd.random() < 0.7:
                    for key in queue[h].pop(0):
                        B[key].arrive()
        elif agents[k] is not None:
            try:
                next(agents[k])
            except StopIteration:
                agents[k] = None
    return "stuck"


@pytest.mark.parametrize("items", [[1] * 8, [1, 2, 3, 1, 4], [7, 5, 6], [2, 1, 1, 9], [18, 3]])
def test_a_table_is_that_of_its_tile_when_it_is_read(items):
    for seed in range(100):
        assert run(items, seed) is None, seed


def test_the_model_sees_too_few_places():
    """With a place for each of the two stages the values' tables are overwritten before they are read."""
    assert any("place holds" in str(run([12, 9], s, places=2)) for s in range(60))
