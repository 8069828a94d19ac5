"""The barriers of the tcgen05 tree attention, without a GPU: its warps as processes that take their steps in drawn orders, with
barriers that tell phases apart by parity alone, as the hardware's do.  Whatever the order, every run ends, no product writes over
scores or weights that are still needed, and outputs are read when their products are done."""
import os
import random

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
SOURCE = open(os.path.join(ROOT, "paper_1811_03115_b200", "csrc", "tree_attention_tc.cuh")).read()


class Barrier:
    def __init__(self, count):
        self.count = self.left = count
        self.phase = 0

    def arrive(self):
        self.left -= 1
        if self.left == 0:
            self.phase, self.left = self.phase + 1, self.count

    def passed(self, parity):
        return self.phase & 1 != parity


class Stalled(Exception):
    pass


def run(tiles, seed, kv_stages, in_turn):
    """tiles: (chunks of the CTA's run, how many of them are the tree's) for each tile.  in_turn: the products with the values arrive
    on two barriers in turn, and the end of a tile waits for the last of them; else on one, and for the last two."""
    rng, total, KK = random.Random(seed), sum(n for n, _ in tiles), 2
    k_full, k_empty = [Barrier(1) for _ in range(KK)], [Barrier(1) for _ in range(KK)]
    v_full, v_empty = [Barrier(1) for _ in range(kv_stages)], [Barrier(1) for _ in range(kv_stages)]
    s_full, p_ready, pv_done = [Barrier(1) for _ in range(2)], [Barrier(4) for _ in range(2)], [Barrier(1) for _ in range(2)]
    q_ready, rows = Barrier(4), Barrier(4)
    products, loads, ended = [], [], 0                       # products end in order, loads in any
    rescales = [[rng.random() < 0.3 for _ in range(total)] for _ in range(4)]

    def until(bar, parity):
        while not bar.passed(parity):
            yield False

    def product(n):
        return until(pv_done[n & 1], n >> 1 & 1) if in_turn else until(pv_done[0], n & 1)

    def load(full, empty):
        for n in range(total):
            yield from until(empty[n % len(empty)], (n // len(empty) & 1) ^ 1)
            loads.append(full[n % len(full)])
            yield True

    def mma():
        def scores(n, first):
            yield from until(k_full[n % KK], n // KK & 1)
            if n >= 2 and (in_turn or not first):
                yield from product(n - 2)
            assert n < 2 or ended >= n - 1                   # the weights in their place have been used
            products.append([s_full[n & 1], k_empty[n % KK]])
            yield True
        n = 0
        for tile, (count, _) in enumerate(tiles):
            yield from until(q_ready, tile & 1)
            yield from scores(n, True)
            for i in range(count):
                if i + 1 < count:
                    yield from scores(n + 1, False)
                yield from until(p_ready[n & 1], n >> 1 & 1)
                yield from until(v_full[n % kv_stages], n // kv_stages & 1)
                products.append([v_empty[n % kv_stages], pv_done[n & 1 if in_turn else 0], None])
                yield True
                n += 1

    def softmax(warp):
        n, met = 0, 0

        def meet():
            nonlocal met
            rows.arrive()
            yield True
            yield from until(rows, met & 1)
            met += 1
        for count, tree in tiles:
            q_ready.arrive()
            yield True
            if tree:
                yield from meet()
                yield from meet()
            for i in range(count):
                yield from until(s_full[n & 1], n >> 1 & 1)
                if i >= count - tree:
                    yield from until(v_full[n % kv_stages], n // kv_stages & 1)
                if i > 0 and rescales[warp][n]:
                    yield from product(n - 1)
                    assert ended >= n
                p_ready[n & 1].arrive()
                n += 1
                yield True
            if not in_turn and count > 1:
                yield from product(n - 2)
            yield from product(n - 1)
            assert ended >= n                                # the outputs are whole
            if tree:
                yield from meet()
    going = {"keys": load(k_full, k_empty), "values": load(v_full, v_empty), "mma": mma(), **{f"softmax {w}": softmax(w) for w in range(4)}}
    pace = {name: 10 ** rng.uniform(-2, 0) for name in [*going, "products", "loads"]}
    idle = 0
    while going:
        names = [*going, "products", "loads"]
        name = rng.choices(names, [pace[x] for x in names])[0]
        moved = True
        if name == "products":
            moved = bool(products)
            if moved:
                bars = products.pop(0)
                ended += len(bars) == 3
                for bar in bars[:2]:
                    bar.arrive()
        elif name == "loads":
            moved = bool(loads)
            if moved:
                loads.pop(rng.randrange(len(loads))).arrive()
        else:
            try:
                moved = next(going[name])
            except StopIteration:
                del going[name]
        idle = 0 if moved else idle + 1
        if idle > 20000:
            raise Stalled(sorted(going))


RUNS = [[(1, 0)], [(2, 2)], [(5, 0)], [(9, 1)], [(1, 1), (6, 0)], [(2, 2), (5, 0)], [(3, 2), (4, 2), (1, 0)], [(6, 1), (1, 1), (7, 0)]]


@pytest.mark.parametrize("kv_stages", [2, 4])
@pytest.mark.parametrize("tiles", RUNS)
def test_every_run_ends(tiles, kv_stages):
    in_turn = "pv_done = [&](int s)" in SOURCE and SOURCE.count("umma_commit(pv_done(n & 1))") == 1 and "(n - 2) & 1" not in SOURCE
    for seed in range(60):
        run(tiles, seed, kv_stages, in_turn)


def test_one_barrier_for_all_products_would_not_do():
    stalls = 0
    for seed in range(40):
        try:
            run([(9, 1)], seed, 2, False)
        except Stalled:
            stalls += 1
    assert stalls > 0
